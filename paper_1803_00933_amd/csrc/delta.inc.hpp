// The gated delta rule and its gradient.  Included by apex_replay.hip (one translation unit).
//
// Per sequence and value head, with a state S [Dk,Dv]:  L = e^g S,  u = beta (v - L^T k),  S' = L + k u^T,  o = scale S'^T q.
//
// A piece of 64 steps at once.  With G the sum of g from the piece's begin on, S0 the state it starts from,
//     D_ti = exp(G_t - G_i) where no episode ends between them, else 0;   c_t = exp(G_t) where none has ended yet, else 0;
//     L = the part below the diagonal of (K K^T) o D,   M = L - L diag(beta) M  (row by row);
//     X = V - c K S0,   E = X - M (beta X),   U = beta E;
//     O = scale (c Q S0 + P U),   P = (Q K^T) o D on and below the diagonal;
//     S = c_last S0 + K^T (D_last U).
// M does not depend on the state, so all pieces' come first, side by side; then a sequence's pieces follow one another, with the
// columns of a state shared out.  E and not U = T beta X with T = (1 + beta L)^-1, since the gradient of beta is Y . E below and
// beta may be 0.
// The gradient, with dS that of the state behind the piece:
//     dU = scale P^T dO + D_last K dS,   Y = dU - M^T (beta dU),   dV = beta Y;
//     dS0 = scale Q^T (c dO) + c_last dS - K^T (c dV);
//     B = scale (dO U^T) o D on and below the diagonal,   C = (dV U^T) o D below it;
//     dQ = scale c dO S0^T + B K,   dK = D_last U dS^T + B^T Q - c dV S0^T - C K - C^T K;
//     dbeta_t = Y_t . E_t;
//     dg_t = the sum of q_s . dq_s - v_s . dv_s over s >= t of its episode, and <dS, S> where that reaches the piece's end: what
//     scales with exp(G_s) are o_s (linear in q_s) and what is taken from v_s.
// Here the pieces' dS come first, from the last to the first, and all else side by side.
#include "elements.hpp"

namespace apex {

constexpr uint32_t kPiece = 64;                                // steps
constexpr uint32_t kDeltaThreads = 256, kDeltaWaves = kDeltaThreads / kWave;
constexpr uint32_t kDeltaMaxWidth = 128;
constexpr uint32_t kPieceRow = kPiece + 4;                     // of a [64][64] matrix in LDS: lanes of a tile hit different banks

typedef float Tile __attribute__((ext_vector_type(4)));        // of 16 x 16: column lane % 16, rows 4 (lane / 16) + 0..3

struct DeltaArgs {
  uint32_t S, T, Hk, H, Dk, Dv, pieces, share;
  uint64_t q_seq, q_time, k_seq, k_time, v_seq, v_time;
  const void *q, *k, *v;
  const float *g, *beta;
  float scale;
  const float *discount;
  const int32_t *length;
  float *M;  // [S][pieces][H][64][64]
};

struct DeltaForward {
  DeltaArgs n;
  const float *h0;
  void *o;
  float *h_last, *carry;
};

struct DeltaBack {
  DeltaArgs n;
  const float *carry;
  const void *d_o;
  const float *dh_last;
  uint64_t dq_seq, dq_time, dk_seq, dk_time, dv_seq, dv_time;
  void *dq, *dk, *dv;
  float *dg, *dbeta, *dh0;
  float *dS;  // [S][pieces][H][Dk][Dv]: of the state behind a piece
  float *Y;   // [S][T][H][Dv]
};

__device__ __forceinline__ uint32_t delta_length(const DeltaArgs &a, uint32_t s)
{
  return a.length ? (uint32_t)min(max(a.length[s], 0), (int32_t)a.T) : a.T;
}

// e^g, and whether anything passes into the step.
__device__ __forceinline__ bool delta_cuts(float g) { return expf(g) == 0.0f; }
__device__ __forceinline__ bool delta_passes(const DeltaArgs &a, uint32_t s, uint32_t t)
{
  return !a.discount || a.discount[(uint64_t)s * a.T + t] != 0.0f;
}

// What a piece's steps have of their gates, in LDS.  Steps that a sequence does not have: g = beta = 0.
struct Gates {
  double G[kPiece];       // sum of g from the piece's begin on: differences of 32-bit sums would lose what is small beside them
  uint32_t episode[kPiece];  // episodes that ended in the piece in front of the step or on its begin
  float beta[kPiece], begin[kPiece], end[kPiece];  // strength; what is left of the start state, and of the step at the end
  uint32_t cut[kPiece];   // nothing passes into the step
  float last;             // what is left of the start state at the end
};

// By one wave.
__device__ __forceinline__ void load_gates(const DeltaArgs &a, uint32_t s, uint32_t h, uint32_t t0, uint32_t len, Gates &x)
{
  const uint32_t lane = lane_id(), t = t0 + lane;
  const bool have = t < len;
  const uint64_t at = ((uint64_t)s * a.T + t) * a.H + h;
  float g = have ? a.g[at] : 0.0f;
  const bool cut = have && (delta_cuts(g) || (t > 0 && !delta_passes(a, s, t - 1)));
  if (cut) g = 0.0f;
  double sum = g;
  uint32_t episode = cut;
  for (int d = 1; d < kWave; d *= 2) {
    const double up = __shfl_up(sum, d);
    const uint32_t e = __shfl_up(episode, d);
    if ((int)lane >= d) sum += up, episode += e;
  }
  const double all = __shfl(sum, kWave - 1);
  const uint32_t episodes = __shfl(episode, kWave - 1);
  x.G[lane] = sum;
  x.episode[lane] = episode;
  x.beta[lane] = have ? a.beta[at] : 0.0f;
  x.begin[lane] = episode == 0 ? expf((float)sum) : 0.0f;
  x.end[lane] = episode == episodes ? expf((float)(all - sum)) : 0.0f;
  x.cut[lane] = cut;
  if (lane == 0) x.last = episodes == 0 ? expf((float)all) : 0.0f;
}

// D of a step t and an earlier one.
__device__ __forceinline__ float decay(const Gates &x, uint32_t t, uint32_t i)
{
  return x.episode[t] == x.episode[i] ? expf((float)(x.G[t] - x.G[i])) : 0.0f;
}

// acc + A B over `depth` (a multiple of 16): a(k) of row lane % 16, b(k) of column lane % 16.
template <typename A, typename B>
__device__ __forceinline__ Tile product(Tile acc, uint32_t depth, A a, B b)
{
  const uint32_t k0 = lane_id() / 16;
  for (uint32_t k = 0; k < depth; k += 16)
#pragma unroll
    for (uint32_t i = 0; i < 16; i += 4) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a(k + i + k0), b(k + i + k0), acc, 0, 0, 0);
  return acc;
}

__device__ __forceinline__ uint32_t up16(uint32_t n) { return (n + 15) / 16 * 16; }

// Rows [0, 64) of one head, columns [c0, c0 + columns), of a strided array into LDS rows of `row` numbers; zeros beyond `have` rows and `width`.
template <typename T>
__device__ __forceinline__ void load_rows(float *to, uint32_t row, uint32_t columns, const T *from, uint64_t stride, uint32_t have,
                                          uint32_t width, uint32_t threads)
{
  for (uint32_t i = threadIdx.x; i < kPiece * columns; i += threads) {
    const uint32_t t = i / columns, d = i % columns;
    to[t * row + d] = t < have && d < width ? (float)from[t * stride + d] : 0.0f;
  }
}

// M of a piece: products of its keys, decayed, and the substitution row by row, a lane per column.
template <typename T>
__global__ __launch_bounds__(kDeltaThreads) void delta_solve_kernel(DeltaArgs a)
{
  __shared__ Gates gates;
  __shared__ float K[kPiece * (kDeltaMaxWidth + 4)], L[kPiece * kPieceRow];
  const uint32_t h = blockIdx.x % a.H, piece = blockIdx.x / a.H % a.pieces, s = blockIdx.x / a.H / a.pieces;
  const uint32_t len = delta_length(a, s), t0 = piece * kPiece;
  if (t0 >= len) return;
  const uint32_t lane = lane_id(), wave = threadIdx.x / kWave, depth = up16(a.Dk), row = depth + 4;
  const T *const k = static_cast<const T *>(a.k) + s * a.k_seq + t0 * a.k_time + (uint64_t)(h / a.share) * a.Dk;
  load_rows(K, row, depth, k, a.k_time, len - t0, a.Dk, kDeltaThreads);
  if (wave == 0) load_gates(a, s, h, t0, len, gates);
  __syncthreads();
  for (uint32_t tile = wave; tile < 16; tile += kDeltaWaves) {
    const uint32_t r = tile / 4 * 16, c = tile % 4 * 16;
    if (c > r) continue;
    const Tile kk = product(Tile{}, depth, [&](uint32_t i) { return K[(r + lane % 16) * row + i]; },
                            [&](uint32_t i) { return K[(c + lane % 16) * row + i]; });
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const uint32_t t = r + lane / 16 * 4 + i, j = c + lane % 16;
      L[t * kPieceRow + j] = j < t ? kk[i] * decay(gates, t, j) : 0.0f;
    }
  }
  __syncthreads();
  if (wave) return;
  // a lane's column of M, from the top
  float m[kPiece];
  float *const out = a.M + (uint64_t)blockIdx.x * kPiece * kPiece;
#pragma unroll
  for (uint32_t t = 0; t < kPiece; ++t) {
    float sum = lane < t ? L[t * kPieceRow + lane] : 0.0f;
#pragma unroll
    for (uint32_t i = 1; i < t; ++i) sum -= L[t * kPieceRow + i] * m[i];
    out[t * kPiece + lane] = sum;
    m[t] = sum * gates.beta[t];  // (as the rows below take it)
  }
}

template <uint32_t kColumns>
struct DeltaSpace {
  static constexpr uint32_t kRow = kColumns + 4;
  Gates gates;
  float K[kPiece * (kDeltaMaxWidth + 4)], Q[kPiece * (kDeltaMaxWidth + 4)];
  float M[kPiece * kPieceRow], P[kPiece * kPieceRow];
  float S[kDeltaMaxWidth * kRow];
  float X[kPiece * kRow], U[kPiece * kRow];
};

// P of a wave's 16 rows.
template <typename Space>
__device__ __forceinline__ void attend(Space &x, uint32_t depth, uint32_t row)
{
  const uint32_t lane = lane_id(), r = threadIdx.x / kWave * 16;
  for (uint32_t c = 0; c < kPiece; c += 16) {
    Tile p{};
    if (c <= r)
      p = product(p, depth, [&](uint32_t i) { return x.Q[(r + lane % 16) * row + i]; }, [&](uint32_t i) { return x.K[(c + lane % 16) * row + i]; });
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const uint32_t t = r + lane / 16 * 4 + i, j = c + lane % 16;
      x.P[t * kPieceRow + j] = j <= t ? p[i] * decay(x.gates, t, j) : 0.0f;
    }
  }
}

__device__ __forceinline__ void load_piece_matrix(float *to, const float *from)
{
  for (uint32_t i = threadIdx.x; i < kPiece * kPiece; i += kDeltaThreads) to[i / kPiece * kPieceRow + i % kPiece] = from[i];
}

// A workgroup per sequence, value head and kColumns columns of its state goes through the pieces.  A wave holds 32 rows of the
// state, as two rows of tiles, and writes them to LDS for the products of all; of what belongs to steps it has 16.
template <typename T, uint32_t kColumns>
__global__ __launch_bounds__(kDeltaThreads) void delta_pieces_kernel(DeltaForward f)
{
  constexpr uint32_t kTiles = kColumns / 16, kRow = DeltaSpace<kColumns>::kRow;
  const DeltaArgs &a = f.n;
  __shared__ DeltaSpace<kColumns> x;
  const uint32_t blocks = (a.Dv + kColumns - 1) / kColumns;
  const uint32_t c0 = blockIdx.x % blocks * kColumns, h = blockIdx.x / blocks % a.H, s = blockIdx.x / blocks / a.H;
  const uint32_t lane = lane_id(), wave = threadIdx.x / kWave, col = lane % 16, quad = lane / 16 * 4;
  const uint32_t len = delta_length(a, s), depth = up16(a.Dk), row = depth + 4, r = wave * 16;
  const uint64_t state = ((uint64_t)s * a.H + h) * a.Dk * a.Dv;
  const auto each = [&](auto do_) {  // of this wave's part of the state: (tile, element, row, column)
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
      for (uint32_t j = 0; j < kTiles; ++j)
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) do_(i, j, e, (wave * 2 + i) * 16 + quad + e, j * 16 + col);
  };
  Tile S[2][kTiles];
  each([&](uint32_t i, uint32_t j, uint32_t e, uint32_t d, uint32_t c) {
    S[i][j][e] = f.h0 && d < a.Dk && c0 + c < a.Dv ? f.h0[state + (uint64_t)d * a.Dv + c0 + c] : 0.0f;
  });
  const uint32_t hk = h / a.share;
  for (uint32_t piece = 0; piece < a.pieces; ++piece) {
    const uint32_t t0 = piece * kPiece, steps = min(kPiece, a.T - t0);
    T *const o = static_cast<T *>(f.o) + (((uint64_t)s * a.T + t0) * a.H + h) * a.Dv + c0;
    const uint64_t o_row = (uint64_t)a.H * a.Dv;
    if (t0 >= len) {
      for (uint32_t i = threadIdx.x; i < steps * kColumns; i += kDeltaThreads)
        if (c0 + i % kColumns < a.Dv) o[i / kColumns * o_row + i % kColumns] = (T)0.0f;
      continue;
    }
    __syncthreads();
    load_rows(x.K, row, depth, static_cast<const T *>(a.k) + s * a.k_seq + t0 * a.k_time + (uint64_t)hk * a.Dk, a.k_time, len - t0, a.Dk, kDeltaThreads);
    load_rows(x.Q, row, depth, static_cast<const T *>(a.q) + s * a.q_seq + t0 * a.q_time + (uint64_t)hk * a.Dk, a.q_time, len - t0, a.Dk, kDeltaThreads);
    load_rows(x.X, kRow, kColumns, static_cast<const T *>(a.v) + s * a.v_seq + t0 * a.v_time + (uint64_t)h * a.Dv + c0, a.v_time, len - t0, a.Dv - c0,
              kDeltaThreads);
    load_piece_matrix(x.M, a.M + (((uint64_t)s * a.pieces + piece) * a.H + h) * kPiece * kPiece);
    if (wave == 0) load_gates(a, s, h, t0, len, x.gates);
    each([&](uint32_t i, uint32_t j, uint32_t e, uint32_t d, uint32_t c) {
      x.S[d * kRow + c] = S[i][j][e];
      if (f.carry && d < a.Dk && c0 + c < a.Dv)
        f.carry[(((uint64_t)s * a.pieces + piece) * a.H + h) * a.Dk * a.Dv + (uint64_t)d * a.Dv + c0 + c] = S[i][j][e];
    });
    __syncthreads();
    attend(x, depth, row);
    Tile X[kTiles], O[kTiles];
#pragma unroll
    for (uint32_t j = 0; j < kTiles; ++j) {
      const auto state_of = [&](uint32_t i) { return x.S[i * kRow + j * 16 + col]; };
      const Tile kS = product(Tile{}, depth, [&](uint32_t i) { return x.K[(r + col) * row + i]; }, state_of);
      O[j] = product(Tile{}, depth, [&](uint32_t i) { return x.Q[(r + col) * row + i]; }, state_of);
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t t = r + quad + e;
        const bool passes = x.gates.episode[t] == 0;  // a selection: nothing of what has ended
        float &v = x.X[t * kRow + j * 16 + col];
        X[j][e] = v - (passes ? x.gates.begin[t] * kS[e] : 0.0f);
        O[j][e] = passes ? x.gates.begin[t] * O[j][e] : 0.0f;
        v = x.gates.beta[t] * X[j][e];
      }
    }
    __syncthreads();
#pragma unroll
    for (uint32_t j = 0; j < kTiles; ++j) {
      const Tile mX = product(Tile{}, kPiece, [&](uint32_t i) { return x.M[(r + col) * kPieceRow + i]; },
                              [&](uint32_t i) { return x.X[i * kRow + j * 16 + col]; });
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t t = r + quad + e;
        x.U[t * kRow + j * 16 + col] = x.gates.beta[t] * (X[j][e] - mX[e]);
      }
    }
    __syncthreads();
#pragma unroll
    for (uint32_t j = 0; j < kTiles; ++j) {
      O[j] = product(O[j], kPiece, [&](uint32_t i) { return x.P[(r + col) * kPieceRow + i]; },
                     [&](uint32_t i) { return x.U[i * kRow + j * 16 + col]; });
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t t = r + quad + e, c = j * 16 + col;
        if (t < steps && c0 + c < a.Dv) o[t * o_row + c] = t0 + t < len ? (T)(a.scale * O[j][e]) : (T)0.0f;
      }
#pragma unroll
      for (uint32_t i = 0; i < 2; ++i) {
        const uint32_t d0 = (wave * 2 + i) * 16;
        if (d0 >= depth) continue;
        const Tile left = x.gates.episode[kPiece - 1] == 0 ? S[i][j] * x.gates.last : Tile{};
        S[i][j] = product(left, kPiece, [&](uint32_t t) { return x.K[t * row + d0 + col]; },
                          [&](uint32_t t) { return x.U[t * kRow + j * 16 + col] * x.gates.end[t]; });
      }
    }
  }
  if (f.h_last) {
    const bool passes = len == 0 || delta_passes(a, s, len - 1);
    each([&](uint32_t i, uint32_t j, uint32_t e, uint32_t d, uint32_t c) {
      if (d < a.Dk && c0 + c < a.Dv) f.h_last[state + (uint64_t)d * a.Dv + c0 + c] = passes ? S[i][j][e] : 0.0f;
    });
  }
}

// The same from the last piece to the first, with dS: its values for every piece, Y and dV.
template <typename T, uint32_t kColumns>
__global__ __launch_bounds__(kDeltaThreads) void delta_pieces_back_kernel(DeltaBack b)
{
  constexpr uint32_t kTiles = kColumns / 16, kRow = DeltaSpace<kColumns>::kRow;
  const DeltaArgs &a = b.n;
  __shared__ DeltaSpace<kColumns> x;  // X: dO, U: beta dU, then c dV
  const uint32_t blocks = (a.Dv + kColumns - 1) / kColumns;
  const uint32_t c0 = blockIdx.x % blocks * kColumns, h = blockIdx.x / blocks % a.H, s = blockIdx.x / blocks / a.H;
  const uint32_t lane = lane_id(), wave = threadIdx.x / kWave, col = lane % 16, quad = lane / 16 * 4;
  const uint32_t len = delta_length(a, s), depth = up16(a.Dk), row = depth + 4, r = wave * 16;
  const uint64_t state = ((uint64_t)s * a.H + h) * a.Dk * a.Dv;
  const auto each = [&](auto do_) {
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
      for (uint32_t j = 0; j < kTiles; ++j)
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) do_(i, j, e, (wave * 2 + i) * 16 + quad + e, j * 16 + col);
  };
  Tile S[2][kTiles];
  const bool passes = len == 0 || delta_passes(a, s, len - 1);
  each([&](uint32_t i, uint32_t j, uint32_t e, uint32_t d, uint32_t c) {
    S[i][j][e] = b.dh_last && passes && d < a.Dk && c0 + c < a.Dv ? b.dh_last[state + (uint64_t)d * a.Dv + c0 + c] : 0.0f;
  });
  const uint32_t hk = h / a.share;
  for (uint32_t piece = a.pieces; piece-- > 0;) {
    const uint32_t t0 = piece * kPiece, steps = min(kPiece, a.T - t0);
    T *const dv = static_cast<T *>(b.dv) + s * b.dv_seq + t0 * b.dv_time + (uint64_t)h * a.Dv + c0;
    if (t0 >= len) {
      for (uint32_t i = threadIdx.x; i < steps * kColumns; i += kDeltaThreads)
        if (c0 + i % kColumns < a.Dv) dv[i / kColumns * b.dv_time + i % kColumns] = (T)0.0f;
      continue;
    }
    __syncthreads();
    load_rows(x.K, row, depth, static_cast<const T *>(a.k) + s * a.k_seq + t0 * a.k_time + (uint64_t)hk * a.Dk, a.k_time, len - t0, a.Dk, kDeltaThreads);
    load_rows(x.Q, row, depth, static_cast<const T *>(a.q) + s * a.q_seq + t0 * a.q_time + (uint64_t)hk * a.Dk, a.q_time, len - t0, a.Dk, kDeltaThreads);
    load_rows(x.X, kRow, kColumns, static_cast<const T *>(b.d_o) + (((uint64_t)s * a.T + t0) * a.H + h) * a.Dv + c0, (uint64_t)a.H * a.Dv, len - t0,
              a.Dv - c0, kDeltaThreads);
    load_piece_matrix(x.M, a.M + (((uint64_t)s * a.pieces + piece) * a.H + h) * kPiece * kPiece);
    if (wave == 0) load_gates(a, s, h, t0, len, x.gates);
    each([&](uint32_t i, uint32_t j, uint32_t e, uint32_t d, uint32_t c) {
      x.S[d * kRow + c] = S[i][j][e];
      if (d < a.Dk && c0 + c < a.Dv)
        b.dS[(((uint64_t)s * a.pieces + piece) * a.H + h) * a.Dk * a.Dv + (uint64_t)d * a.Dv + c0 + c] = S[i][j][e];
    });
    __syncthreads();
    attend(x, depth, row);
    __syncthreads();
    Tile dU[kTiles];
#pragma unroll
    for (uint32_t j = 0; j < kTiles; ++j) {
      const Tile of_o = product(Tile{}, kPiece, [&](uint32_t t) { return x.P[t * kPieceRow + r + col]; },
                                [&](uint32_t t) { return x.X[t * kRow + j * 16 + col]; });
      const Tile kS = product(Tile{}, depth, [&](uint32_t i) { return x.K[(r + col) * row + i]; },
                              [&](uint32_t i) { return x.S[i * kRow + j * 16 + col]; });
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t t = r + quad + e;
        dU[j][e] = a.scale * of_o[e] + x.gates.end[t] * kS[e];
        x.U[t * kRow + j * 16 + col] = x.gates.beta[t] * dU[j][e];
      }
    }
    __syncthreads();
#pragma unroll
    for (uint32_t j = 0; j < kTiles; ++j) {
      const Tile mU = product(Tile{}, kPiece, [&](uint32_t t) { return x.M[t * kPieceRow + r + col]; },
                              [&](uint32_t t) { return x.U[t * kRow + j * 16 + col]; });
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) dU[j][e] -= mU[e];  // Y
    }
    __syncthreads();
#pragma unroll
    for (uint32_t j = 0; j < kTiles; ++j)
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t t = r + quad + e, c = j * 16 + col;
        const float of_v = x.gates.beta[t] * dU[j][e];
        x.U[t * kRow + c] = x.gates.begin[t] * of_v;
        if (t < steps && c0 + c < a.Dv) {
          dv[t * b.dv_time + c] = t0 + t < len ? (T)of_v : (T)0.0f;
          b.Y[(((uint64_t)s * a.T + t0 + t) * a.H + h) * a.Dv + c0 + c] = dU[j][e];
        }
      }
    __syncthreads();
#pragma unroll
    for (uint32_t j = 0; j < kTiles; ++j)
#pragma unroll
      for (uint32_t i = 0; i < 2; ++i) {
        const uint32_t d0 = (wave * 2 + i) * 16;
        if (d0 >= depth) continue;
        const Tile of_q = product(Tile{}, kPiece, [&](uint32_t t) { return x.Q[t * row + d0 + col]; },
                                  [&](uint32_t t) { return x.X[t * kRow + j * 16 + col] * (a.scale * x.gates.begin[t]); });
        const Tile of_k = product(Tile{}, kPiece, [&](uint32_t t) { return x.K[t * row + d0 + col]; },
                                  [&](uint32_t t) { return x.U[t * kRow + j * 16 + col]; });
        const Tile left = x.gates.episode[kPiece - 1] == 0 ? S[i][j] * x.gates.last : Tile{};
        S[i][j] = of_q + left - of_k;
      }
  }
  if (b.dh0)
    each([&](uint32_t i, uint32_t j, uint32_t e, uint32_t d, uint32_t c) {
      if (d < a.Dk && c0 + c < a.Dv) b.dh0[state + (uint64_t)d * a.Dv + c0 + c] = S[i][j][e];
    });
}

// What is left of the gradient, a workgroup per piece and key head: eight waves, of which wave w has rows 16 (w % 4) of what
// belongs to steps, and of their columns one half.
constexpr uint32_t kGradThreads = 512, kGradWaves = kGradThreads / kWave, kGradColumns = 32;

struct GradSpace {
  static constexpr uint32_t kRow = kGradColumns + 4;
  Gates gates;
  float K[kPiece * (kDeltaMaxWidth + 4)];
  union {
    struct {
      float S0[kDeltaMaxWidth * kRow], dS[kDeltaMaxWidth * kRow];
    };
    float Q[kPiece * (kDeltaMaxWidth + 4)];
  };
  union {
    struct {
      float X[kPiece * kRow], U[kPiece * kRow], dO[kPiece * kRow], dV[kPiece * kRow];
    };
    struct {
      float B[kPiece * kPieceRow], C[kPiece * kPieceRow];
    };
  };
  float M[kPiece * kPieceRow];
  float of_g[2][kPiece], of_v[2][kPiece], of_beta[2][kPiece];  // sums over a half of the columns
  double at_end[kGradWaves];
};

// The sum over the 16 lanes of a row of a tile, in each of them.
__device__ __forceinline__ float row_sum(float v)
{
  for (int d = 1; d < 16; d *= 2) v += __shfl_xor(v, d);
  return v;
}

template <typename T>
__global__ __launch_bounds__(kGradThreads) void delta_gradients_kernel(DeltaBack b)
{
  constexpr uint32_t kRow = GradSpace::kRow, kMaxTiles = kDeltaMaxWidth / 16 / 2;
  const DeltaArgs &a = b.n;
  __shared__ GradSpace x;
  const uint32_t hk = blockIdx.x % a.Hk, piece = blockIdx.x / a.Hk % a.pieces, s = blockIdx.x / a.Hk / a.pieces;
  const uint32_t lane = lane_id(), wave = threadIdx.x / kWave, col = lane % 16, quad = lane / 16 * 4;
  const uint32_t r = wave % 4 * 16, half = wave / 4;
  const uint32_t len = delta_length(a, s), t0 = piece * kPiece, steps = min(kPiece, a.T - t0);
  const uint32_t depth = up16(a.Dk), row = depth + 4;
  T *const dq = static_cast<T *>(b.dq) + s * b.dq_seq + t0 * b.dq_time + (uint64_t)hk * a.Dk;
  T *const dk = static_cast<T *>(b.dk) + s * b.dk_seq + t0 * b.dk_time + (uint64_t)hk * a.Dk;
  const uint64_t gates_at = ((uint64_t)s * a.T + t0) * a.H;
  if (t0 >= len) {
    for (uint32_t i = threadIdx.x; i < steps * a.Dk; i += kGradThreads) {
      dq[i / a.Dk * b.dq_time + i % a.Dk] = (T)0.0f;
      dk[i / a.Dk * b.dk_time + i % a.Dk] = (T)0.0f;
    }
    for (uint32_t i = threadIdx.x; i < steps * a.share; i += kGradThreads) {
      const uint64_t at = gates_at + (uint64_t)(i / a.share) * a.H + hk * a.share + i % a.share;
      b.dg[at] = b.dbeta[at] = 0.0f;
    }
    return;
  }
  load_rows(x.K, row, depth, static_cast<const T *>(a.k) + s * a.k_seq + t0 * a.k_time + (uint64_t)hk * a.Dk, a.k_time, len - t0, a.Dk, kGradThreads);
  Tile dq_all[kMaxTiles] = {}, dk_all[kMaxTiles] = {};  // tile i: columns 16 (2 i + half)
  for (uint32_t h = hk * a.share; h < (hk + 1) * a.share; ++h) {
    __syncthreads();
    const uint64_t piece_head = ((uint64_t)s * a.pieces + piece) * a.H + h;
    if (wave == 0) load_gates(a, s, h, t0, len, x.gates);
    for (uint32_t i = threadIdx.x; i < kPiece * kPiece; i += kGradThreads)
      x.M[i / kPiece * kPieceRow + i % kPiece] = a.M[piece_head * kPiece * kPiece + i];
    Tile dq_h[kMaxTiles] = {}, B[2] = {}, C[2] = {};  // B and C: columns 16 (2 half + i)
    float of_v[4] = {}, of_beta[4] = {};
    double at_end = 0.0;
    for (uint32_t c0 = 0; c0 < a.Dv; c0 += kGradColumns) {
      __syncthreads();
      const float *const S0 = b.carry + piece_head * a.Dk * a.Dv + c0, *const dS = b.dS + piece_head * a.Dk * a.Dv + c0;
      for (uint32_t i = threadIdx.x; i < depth * kGradColumns; i += kGradThreads) {
        const uint32_t d = i / kGradColumns, c = i % kGradColumns;
        const bool have = d < a.Dk && c0 + c < a.Dv;
        x.S0[d * kRow + c] = have ? S0[(uint64_t)d * a.Dv + c] : 0.0f;
        x.dS[d * kRow + c] = have ? dS[(uint64_t)d * a.Dv + c] : 0.0f;
      }
      load_rows(x.X, kRow, kGradColumns, static_cast<const T *>(a.v) + s * a.v_seq + t0 * a.v_time + (uint64_t)h * a.Dv + c0, a.v_time, len - t0,
                a.Dv - c0, kGradThreads);
      load_rows(x.dO, kRow, kGradColumns, static_cast<const T *>(b.d_o) + gates_at * a.Dv + (uint64_t)h * a.Dv + c0, (uint64_t)a.H * a.Dv, len - t0,
                a.Dv - c0, kGradThreads);
      load_rows(x.dV, kRow, kGradColumns, b.Y + gates_at * a.Dv + (uint64_t)h * a.Dv + c0, (uint64_t)a.H * a.Dv, len - t0, a.Dv - c0, kGradThreads);
      __syncthreads();
      const uint32_t c = half * 16 + col;
      const Tile kS = product(Tile{}, depth, [&](uint32_t i) { return x.K[(r + col) * row + i]; }, [&](uint32_t i) { return x.S0[i * kRow + c]; });
      Tile X, Y, V;
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t t = r + quad + e;
        V[e] = x.X[t * kRow + c];
        Y[e] = x.dV[t * kRow + c];
        X[e] = V[e] - (x.gates.episode[t] == 0 ? x.gates.begin[t] * kS[e] : 0.0f);
        x.X[t * kRow + c] = x.gates.beta[t] * X[e];
        x.dV[t * kRow + c] = x.gates.beta[t] * Y[e];
      }
      __syncthreads();
      const Tile mX = product(Tile{}, kPiece, [&](uint32_t i) { return x.M[(r + col) * kPieceRow + i]; }, [&](uint32_t i) { return x.X[i * kRow + c]; });
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t t = r + quad + e;
        const float E = X[e] - mX[e];
        of_beta[e] += Y[e] * E;
        of_v[e] += V[e] * (x.gates.beta[t] * Y[e]);
        x.U[t * kRow + c] = x.gates.beta[t] * E;
      }
      if (x.gates.episode[kPiece - 1] == 0)
        for (uint32_t i = threadIdx.x; i < depth * kGradColumns; i += kGradThreads) {
          const uint32_t at = i / kGradColumns * kRow + i % kGradColumns;
          at_end += (double)(x.gates.last * x.S0[at]) * x.dS[at];
        }
      __syncthreads();
#pragma unroll
      for (uint32_t i = 0; i < kMaxTiles; ++i) {
        const uint32_t d0 = (2 * i + half) * 16;
        if (d0 >= depth) continue;
        const auto start = [&](uint32_t k) { return x.S0[(d0 + col) * kRow + k]; };
        const Tile oS = product(Tile{}, kGradColumns, [&](uint32_t k) { return x.dO[(r + col) * kRow + k]; }, start);
        const Tile vS = product(Tile{}, kGradColumns, [&](uint32_t k) { return x.dV[(r + col) * kRow + k]; }, start);
        const Tile uS = product(Tile{}, kGradColumns, [&](uint32_t k) { return x.U[(r + col) * kRow + k]; },
                                [&](uint32_t k) { return x.dS[(d0 + col) * kRow + k]; });
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
          const uint32_t t = r + quad + e;
          const bool passes = x.gates.episode[t] == 0;
          const float begin = x.gates.begin[t], end = x.gates.end[t];
          dq_h[i][e] += passes ? a.scale * begin * oS[e] : 0.0f;
          dk_all[i][e] += end * uS[e] - (passes ? begin * vS[e] : 0.0f);
          at_end += (double)(end * uS[e]) * x.K[t * row + d0 + col];
        }
      }
#pragma unroll
      for (uint32_t i = 0; i < 2; ++i) {
        const uint32_t j0 = (2 * half + i) * 16;
        if (j0 > r) continue;
        const auto u = [&](uint32_t k) { return x.U[(j0 + col) * kRow + k]; };
        B[i] = product(B[i], kGradColumns, [&](uint32_t k) { return x.dO[(r + col) * kRow + k]; }, u);
        C[i] = product(C[i], kGradColumns, [&](uint32_t k) { return x.dV[(r + col) * kRow + k]; }, u);
      }
    }
    __syncthreads();
    load_rows(x.Q, row, depth, static_cast<const T *>(a.q) + s * a.q_seq + t0 * a.q_time + (uint64_t)hk * a.Dk, a.q_time, len - t0, a.Dk, kGradThreads);
#pragma unroll
    for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t t = r + quad + e, j = (2 * half + i) * 16 + col;
        const float d = j <= t ? decay(x.gates, t, j) : 0.0f;
        x.B[t * kPieceRow + j] = j <= t ? a.scale * B[i][e] * d : 0.0f;
        x.C[t * kPieceRow + j] = j < t ? C[i][e] * d : 0.0f;
      }
    __syncthreads();
    float of_g[4] = {};
#pragma unroll
    for (uint32_t i = 0; i < kMaxTiles; ++i) {
      const uint32_t d0 = (2 * i + half) * 16;
      if (d0 >= depth) continue;
      const auto key = [&](uint32_t k) { return x.K[k * row + d0 + col]; };
      dq_h[i] = product(dq_h[i], kPiece, [&](uint32_t k) { return x.B[(r + col) * kPieceRow + k]; }, key);
      const Tile bQ = product(Tile{}, kPiece, [&](uint32_t k) { return x.B[k * kPieceRow + r + col]; }, [&](uint32_t k) { return x.Q[k * row + d0 + col]; });
      const Tile cK = product(Tile{}, kPiece, [&](uint32_t k) { return x.C[(r + col) * kPieceRow + k] + x.C[k * kPieceRow + r + col]; }, key);
      dk_all[i] += bQ - cK;
      dq_all[i] += dq_h[i];
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) of_g[e] += x.Q[(r + quad + e) * row + d0 + col] * dq_h[i][e];
    }
    at_end = wave_sum(at_end);
    if (lane == 0) x.at_end[wave] = at_end;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
      const uint32_t t = r + quad + e;
      const float g = row_sum(of_g[e]), v = row_sum(of_v[e]), beta = row_sum(of_beta[e]);
      if (col == 0) x.of_g[half][t] = g, x.of_v[half][t] = v, x.of_beta[half][t] = beta;
    }
    __syncthreads();
    if (threadIdx.x < steps) {
      const uint32_t t = threadIdx.x;
      const uint64_t at = gates_at + (uint64_t)t * a.H + h;
      double sum = 0.0;
      for (uint32_t i = t; i < kPiece && x.gates.episode[i] == x.gates.episode[t]; ++i)
        sum += (double)x.of_g[0][i] + x.of_g[1][i] - ((double)x.of_v[0][i] + x.of_v[1][i]);
      if (x.gates.episode[t] == x.gates.episode[kPiece - 1])
        for (uint32_t w = 0; w < kGradWaves; ++w) sum += x.at_end[w];
      const bool have = t0 + t < len;
      b.dg[at] = have && !x.gates.cut[t] ? (float)sum : 0.0f;
      b.dbeta[at] = have ? x.of_beta[0][t] + x.of_beta[1][t] : 0.0f;
    }
  }
#pragma unroll
  for (uint32_t i = 0; i < kMaxTiles; ++i) {
    const uint32_t d = (2 * i + half) * 16 + col;
    if (d >= a.Dk) continue;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
      const uint32_t t = r + quad + e;
      if (t >= steps) continue;
      dq[t * b.dq_time + d] = t0 + t < len ? (T)dq_all[i][e] : (T)0.0f;
      dk[t * b.dk_time + d] = t0 + t < len ? (T)dk_all[i][e] : (T)0.0f;
    }
  }
}

// ---- few steps: one after the other, the state in registers.  A workgroup has 64 columns of a state, a thread 8 rows of 4 of
// them; what crosses between rows are three sums a step: k . S, q . S and q . k, so that a step has one barrier.
constexpr uint32_t kStepColumns = 64, kStepRows = 8;

template <typename T>
__global__ __launch_bounds__(kDeltaThreads) void delta_steps_kernel(DeltaForward f)
{
  constexpr uint32_t C = 4;
  const DeltaArgs &a = f.n;
  __shared__ float red[2][kDeltaWaves][2 * kStepColumns + 1];
  const uint32_t blocks = (a.Dv + kStepColumns - 1) / kStepColumns;
  const uint32_t h = blockIdx.x / blocks % a.H, s = blockIdx.x / blocks / a.H, hk = h / a.share;
  const uint32_t lane = lane_id(), wave = threadIdx.x / kWave;
  const uint32_t in_block = lane % 16 * C, c0 = blockIdx.x % blocks * kStepColumns + in_block, d0 = threadIdx.x / 16 * kStepRows;
  const uint32_t len = delta_length(a, s);
  const uint64_t state = ((uint64_t)s * a.H + h) * a.Dk * a.Dv;
  float S[kStepRows][C];
  const auto load = [&](const float *from) {
#pragma unroll
    for (uint32_t i = 0; i < kStepRows; ++i) {
      const float *const p = from + state + (uint64_t)(d0 + i) * a.Dv + c0;
      if (d0 + i < a.Dk && c0 + C <= a.Dv) {
        const Run<float, C> v = load_run<float, C>(p);
#pragma unroll
        for (uint32_t c = 0; c < C; ++c) S[i][c] = v[c];
      } else {
#pragma unroll
        for (uint32_t c = 0; c < C; ++c) S[i][c] = d0 + i < a.Dk && c0 + c < a.Dv ? p[c] : 0.0f;
      }
    }
  };
  const auto store = [&](float *to, bool passes) {
#pragma unroll
    for (uint32_t i = 0; i < kStepRows; ++i) {
      if (d0 + i >= a.Dk) continue;
      float *const p = to + (uint64_t)(d0 + i) * a.Dv + c0;
      if (c0 + C <= a.Dv) {
        Run<float, C> v;
#pragma unroll
        for (uint32_t c = 0; c < C; ++c) v[c] = passes ? S[i][c] : 0.0f;
        *reinterpret_cast<Run<float, C> *>(p) = v;
      } else {
#pragma unroll
        for (uint32_t c = 0; c < C; ++c)
          if (c0 + c < a.Dv) p[c] = passes ? S[i][c] : 0.0f;
      }
    }
  };
  if (f.h0) {
    load(f.h0);
  } else {
#pragma unroll
    for (uint32_t i = 0; i < kStepRows; ++i)
#pragma unroll
      for (uint32_t c = 0; c < C; ++c) S[i][c] = 0.0f;
  }
  bool passes = true;
  for (uint32_t t = 0; t < a.T; ++t) {
    T *const o = static_cast<T *>(f.o) + (((uint64_t)s * a.T + t) * a.H + h) * a.Dv + c0;
    if (t >= len) {
      if (d0 == 0)
        for (uint32_t c = 0; c < C; ++c)
          if (c0 + c < a.Dv) o[c] = (T)0.0f;
      continue;
    }
    const uint64_t at = ((uint64_t)s * a.T + t) * a.H + h;
    const float beta = a.beta[at], keep = expf(a.g[at]);
    const T *const k_row = static_cast<const T *>(a.k) + s * a.k_seq + t * a.k_time + (uint64_t)hk * a.Dk;
    const T *const q_row = static_cast<const T *>(a.q) + s * a.q_seq + t * a.q_time + (uint64_t)hk * a.Dk;
    const T *const v_row = static_cast<const T *>(a.v) + s * a.v_seq + t * a.v_time + (uint64_t)h * a.Dv + c0;
    float k[kStepRows], q[kStepRows], v[C];
    if (d0 + kStepRows <= a.Dk) {
      const Run<T, kStepRows> kr = load_run<T, kStepRows>(k_row + d0), qr = load_run<T, kStepRows>(q_row + d0);
#pragma unroll
      for (uint32_t i = 0; i < kStepRows; ++i) k[i] = element<kStepRows, T>(kr, i), q[i] = element<kStepRows, T>(qr, i);
    } else {
#pragma unroll
      for (uint32_t i = 0; i < kStepRows; ++i) {
        k[i] = d0 + i < a.Dk ? (float)k_row[d0 + i] : 0.0f;
        q[i] = d0 + i < a.Dk ? (float)q_row[d0 + i] : 0.0f;
      }
    }
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) v[c] = c0 + c < a.Dv ? (float)v_row[c] : 0.0f;
    if (f.carry && t % kPiece == 0) store(f.carry + (((uint64_t)s * a.pieces + t / kPiece) * a.H + h) * a.Dk * a.Dv, passes);
    const bool in = passes && keep != 0.0f;  // a selection: nothing of what has ended
    float kS[C] = {}, qS[C] = {}, qk = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < kStepRows; ++i) {
      qk = __builtin_fmaf(q[i], k[i], qk);
#pragma unroll
      for (uint32_t c = 0; c < C; ++c) {
        S[i][c] = in ? S[i][c] * keep : 0.0f;
        kS[c] = __builtin_fmaf(k[i], S[i][c], kS[c]);
        qS[c] = __builtin_fmaf(q[i], S[i][c], qS[c]);
      }
    }
    // over the four groups of rows of the wave, then over the waves
    const auto of_wave = [](float y) {
      y += __shfl_xor(y, 16);
      return y + __shfl_xor(y, 32);
    };
    qk = of_wave(qk);
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) kS[c] = of_wave(kS[c]), qS[c] = of_wave(qS[c]);
    float(*const to)[2 * kStepColumns + 1] = red[t % 2];
    if (lane < 16) {
#pragma unroll
      for (uint32_t c = 0; c < C; ++c) to[wave][in_block + c] = kS[c], to[wave][kStepColumns + in_block + c] = qS[c];
      if (lane == 0) to[wave][2 * kStepColumns] = qk;
    }
    __syncthreads();
    qk = 0.0f;
#pragma unroll
    for (uint32_t w = 0; w < kDeltaWaves; ++w) qk += to[w][2 * kStepColumns];
#pragma unroll
    for (uint32_t c = 0; c < C; ++c) {
      float ks = 0.0f, qs = 0.0f;
#pragma unroll
      for (uint32_t w = 0; w < kDeltaWaves; ++w) ks += to[w][in_block + c], qs += to[w][kStepColumns + in_block + c];
      const float u = beta * (v[c] - ks);
#pragma unroll
      for (uint32_t i = 0; i < kStepRows; ++i) S[i][c] = __builtin_fmaf(k[i], u, S[i][c]);
      if (d0 == 0 && c0 + c < a.Dv) o[c] = (T)(a.scale * __builtin_fmaf(qk, u, qs));
    }
    passes = delta_passes(a, s, t);
  }
  if (f.h_last) store(f.h_last + state, passes);
}

}  // namespace apex

namespace {

constexpr uint32_t kDeltaSteps = 16;  // sequences of at most so many steps are computed step by step

uint32_t delta_columns(uint32_t S, uint32_t H, uint32_t Dv) { return (uint64_t)S * H * blocks_for(Dv, 32) >= kChipCus ? 32 : 16; }

// f(integral_constant<uint32_t>): the columns of a state that a workgroup takes.
template <typename F>
void with_columns(uint32_t columns, F f)
{
  if (columns == 32)
    f(std::integral_constant<uint32_t, 32>());
  else
    f(std::integral_constant<uint32_t, 16>());
}

struct DeltaBytes {
  uint64_t M, dS, Y, bytes;
};

int delta_sizes(uint32_t S, uint32_t T, uint32_t H, uint32_t Dk, uint32_t Dv, bool backward, DeltaBytes *n)
{
  if (!S || !T || !H || !Dk || !Dv || T > 0x7fffffffu) return APEX_ERR_INVALID_ARG;
  if (Dk > kDeltaMaxWidth || Dv > kDeltaMaxWidth) return APEX_ERR_TOO_LARGE;
  // workgroups of 512 threads, fewer than 2^32 threads in all
  uint64_t heads;
  if (__builtin_mul_overflow((uint64_t)S * blocks_for(T, kPiece), (uint64_t)H, &heads) || heads >= 1u << 23) return APEX_ERR_TOO_LARGE;
  n->M = n->dS = n->Y = 0;
  uint64_t at = 0;
  if (backward || T > kDeltaSteps) at = heads * kPiece * kPiece * 4;
  if (backward) {
    n->dS = at;
    at += round_up(heads * Dk * Dv * 4, 256);
    n->Y = at;
    at += round_up((uint64_t)S * T * H * Dv * 4, 256);
  }
  n->bytes = at;
  return APEX_OK;
}

int delta_check(const DeltaArgs &a, int dtype)
{
  const uint32_t size = element_size(dtype);
  if (!size || !a.Hk || a.H % a.Hk || !a.q || !a.k || !a.v || !a.g || !a.beta || !(a.scale - a.scale == 0.0f)) return APEX_ERR_INVALID_ARG;
  if (!rows_fit(a.q, size, a.S, a.q_seq, a.T, a.q_time, (uint64_t)a.Hk * a.Dk) || !rows_fit(a.k, size, a.S, a.k_seq, a.T, a.k_time, (uint64_t)a.Hk * a.Dk) ||
      !rows_fit(a.v, size, a.S, a.v_seq, a.T, a.v_time, (uint64_t)a.H * a.Dv))
    return APEX_ERR_INVALID_ARG;
  if (((uintptr_t)a.g | (uintptr_t)a.beta | (uintptr_t)a.discount | (uintptr_t)a.length) % 4) return APEX_ERR_INVALID_ARG;
  return APEX_OK;
}

}  // namespace

extern "C" {

int apex_delta_rule_workspace_bytes(uint32_t S, uint32_t T, uint32_t H, uint32_t Dk, uint32_t Dv, int backward, size_t *bytes)
{
  DeltaBytes n;
  if (!bytes) return APEX_ERR_INVALID_ARG;
  if (const int rc = delta_sizes(S, T, H, Dk, Dv, backward != 0, &n)) return rc;
  *bytes = n.bytes;
  return APEX_OK;
}

int apex_delta_rule(uint32_t S, uint32_t T, uint32_t Hk, uint32_t H, uint32_t Dk, uint32_t Dv, int dtype, const void *q,
                    uint64_t q_seq_stride, uint64_t q_time_stride, const void *k, uint64_t k_seq_stride, uint64_t k_time_stride,
                    const void *v, uint64_t v_seq_stride, uint64_t v_time_stride, const float *g, const float *beta, float scale,
                    const float *discount, const int32_t *length, const float *h0, void *o, float *h_last, float *carry,
                    void *workspace, void *hip_stream)
{
  DeltaBytes n;
  if (const int rc = delta_sizes(S, T, H, Dk, Dv, false, &n)) return rc;
  DeltaForward f{{S, T, Hk, H, Dk, Dv, blocks_for(T, kPiece), Hk ? H / Hk : 0, q_seq_stride, q_time_stride, k_seq_stride, k_time_stride,
                  v_seq_stride, v_time_stride, q, k, v, g, beta, scale, discount, length, static_cast<float *>(workspace)},
                 h0, o, h_last, carry};
  if (const int rc = delta_check(f.n, dtype)) return rc;
  if (!o || (uintptr_t)o % element_size(dtype) || ((uintptr_t)h0 | (uintptr_t)h_last | (uintptr_t)carry) % 4 ||
      (n.bytes && (!workspace || (uintptr_t)workspace % 256)))
    return APEX_ERR_INVALID_ARG;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (T <= kDeltaSteps) {
    with_type(dtype, [&](auto t) {
      delta_steps_kernel<decltype(t)><<<dim3(S * H * blocks_for(Dv, kStepColumns)), dim3(kDeltaThreads), 0, stream>>>(f);
    });
    APEX_HIP(hipGetLastError());
    return APEX_OK;
  }
  const uint32_t columns = delta_columns(S, H, Dv);
  with_type(dtype, [&](auto t) {
    typedef decltype(t) E;
    delta_solve_kernel<E><<<dim3(S * f.n.pieces * H), dim3(kDeltaThreads), 0, stream>>>(f.n);
    with_columns(columns, [&](auto c) {
      constexpr uint32_t kC = decltype(c)::value;
      delta_pieces_kernel<E, kC><<<dim3(S * H * blocks_for(Dv, kC)), dim3(kDeltaThreads), 0, stream>>>(f);
    });
  });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

int apex_delta_rule_backward(uint32_t S, uint32_t T, uint32_t Hk, uint32_t H, uint32_t Dk, uint32_t Dv, int dtype, const void *q,
                             uint64_t q_seq_stride, uint64_t q_time_stride, const void *k, uint64_t k_seq_stride,
                             uint64_t k_time_stride, const void *v, uint64_t v_seq_stride, uint64_t v_time_stride, const float *g,
                             const float *beta, float scale, const float *discount, const int32_t *length, const float *carry,
                             const void *d_o, const float *dh_last, void *dq, uint64_t dq_seq_stride, uint64_t dq_time_stride, void *dk,
                             uint64_t dk_seq_stride, uint64_t dk_time_stride, void *dv, uint64_t dv_seq_stride, uint64_t dv_time_stride,
                             float *dg, float *dbeta, float *dh0, void *workspace, void *hip_stream)
{
  DeltaBytes n;
  if (const int rc = delta_sizes(S, T, H, Dk, Dv, true, &n)) return rc;
  char *const space = static_cast<char *>(workspace);
  DeltaBack b{{S, T, Hk, H, Dk, Dv, blocks_for(T, kPiece), Hk ? H / Hk : 0, q_seq_stride, q_time_stride, k_seq_stride, k_time_stride,
               v_seq_stride, v_time_stride, q, k, v, g, beta, scale, discount, length, reinterpret_cast<float *>(space)},
              carry, d_o, dh_last, dq_seq_stride, dq_time_stride, dk_seq_stride, dk_time_stride, dv_seq_stride, dv_time_stride, dq, dk, dv, dg,
              dbeta, dh0, reinterpret_cast<float *>(space + n.dS), reinterpret_cast<float *>(space + n.Y)};
  if (const int rc = delta_check(b.n, dtype)) return rc;
  const uint32_t size = element_size(dtype);
  if (!carry || !d_o || !dg || !dbeta || !workspace || (uintptr_t)workspace % 256 || (uintptr_t)d_o % size ||
      ((uintptr_t)carry | (uintptr_t)dh_last | (uintptr_t)dg | (uintptr_t)dbeta | (uintptr_t)dh0) % 4 || !dq || !dk || !dv ||
      !rows_apart(dq, size, S, dq_seq_stride, T, dq_time_stride, (uint64_t)Hk * Dk) ||
      !rows_apart(dk, size, S, dk_seq_stride, T, dk_time_stride, (uint64_t)Hk * Dk) ||
      !rows_apart(dv, size, S, dv_seq_stride, T, dv_time_stride, (uint64_t)H * Dv))
    return APEX_ERR_INVALID_ARG;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const uint32_t columns = delta_columns(S, H, Dv);
  with_type(dtype, [&](auto t) {
    typedef decltype(t) E;
    delta_solve_kernel<E><<<dim3(S * b.n.pieces * H), dim3(kDeltaThreads), 0, stream>>>(b.n);
    with_columns(columns, [&](auto c) {
      constexpr uint32_t kC = decltype(c)::value;
      delta_pieces_back_kernel<E, kC><<<dim3(S * H * blocks_for(Dv, kC)), dim3(kDeltaThreads), 0, stream>>>(b);
    });
    delta_gradients_kernel<E><<<dim3(S * b.n.pieces * Hk), dim3(kGradThreads), 0, stream>>>(b);
  });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

}  // extern "C"
