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
  float *dS;  // [S][pieces][H]: of the state behind a piece, by 16 columns
  float *Y;   // [S][pieces][H][ceil(Dv / 16)][kWave][16]
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
struct alignas(16) Gates {
  double G[kPiece];       // sum of g log2(e) from the piece's begin on: differences of 32-bit sums would lose what is small beside them
  uint32_t episode[kPiece];  // episodes that ended in the piece in front of the step or on its begin
  float beta[kPiece], begin[kPiece], end[kPiece];  // strength; what is left of the start state, and of the step at the end
  uint32_t cut[kPiece];   // nothing passes into the step
  float last;             // what is left of the start state at the end
  uint32_t enters;        // the step in front of the piece did not end an episode: the start state is one
};

// By one wave.
__device__ __forceinline__ void load_gates(const DeltaArgs &a, uint32_t s, uint32_t h, uint32_t t0, uint32_t len, Gates &x)
{
  const uint32_t lane = lane_id(), t = t0 + lane;
  const bool have = t < len;
  const uint64_t at = ((uint64_t)s * a.T + t) * a.H + h;
  float g = have ? a.g[at] : 0.0f;
  const bool enters = !have || t == 0 || delta_passes(a, s, t - 1), cut = have && (delta_cuts(g) || !enters);
  if (cut) g = 0.0f;
  double sum = (double)g * 1.4426950408889634;
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
  x.begin[lane] = episode == 0 ? exp2_of((float)sum) : 0.0f;
  x.end[lane] = episode == episodes ? exp2_of((float)(all - sum)) : 0.0f;
  x.cut[lane] = cut;
  if (lane == 0) {
    x.last = episodes == 0 ? exp2_of((float)all) : 0.0f;
    x.enters = enters;
  }
}

// D of a step t and an earlier one.
__device__ __forceinline__ float decay(const Gates &x, uint32_t t, uint32_t i)
{
  const float d = exp2_of((float)(x.G[t] - x.G[i]));
  return x.episode[t] == x.episode[i] ? d : 0.0f;
}

// ---- products.  Matrix instructions take numbers of 8 bits (bf16), 16 times as many as of 32 bits, so a 32-bit number is the sum
// of three of them, each what is left rounded to nearest even: of a number in [1, 2) the second is at most 2^-8, the third 2^-17 and a
// multiple of 2^-23, so the sum is exact.  A product of two numbers is the sum of six products of parts; what the other three
// come to is at most 2 * 2^-8 * 2^-17 of it, half a unit of its last place, on either side of 0.  (Parts that are cut off instead all
// have the number's sign, and leave out up to 2^-21, always towards 0.)  Numbers of 16 bits are one part (bf16) or two (f16).  A number
// within 2^-9 of the largest of 32 bits has an infinite first part.  Beside one part nothing is left out, and parts might be cut off there,
// which takes half of the conversion's time, but brought nothing (4 x 8192 steps of 16 heads in bf16: the pieces 603 us in place of 595, the
// gradient's last kernel 1131 of 1140).
typedef __bf16 Parts8 __attribute__((ext_vector_type(8)));  // one part of 8 numbers: an operand's share of a lane

template <typename T>
constexpr uint32_t kPartsOf = std::is_same<T, __bf16>::value ? 1 : std::is_same<T, _Float16>::value ? 2 : 3;

template <uint32_t N>
struct Operand {
  Parts8 part[N];
};

// Two numbers' next parts, the first in the low half; x and y are what is left of them.  (Both at once, and taken apart as a word: one by
// one the compiler converts each twice.)
__device__ __forceinline__ uint32_t next_parts(float &x, float &y)
{
  typedef float Two __attribute__((ext_vector_type(2)));
  typedef __bf16 TwoParts __attribute__((ext_vector_type(2)));
  const uint32_t word = __builtin_bit_cast(uint32_t, __builtin_convertvector((Two{x, y}), TwoParts));
  x -= __uint_as_float(word << 16), y -= __uint_as_float(word & 0xffff0000u);
  return word;
}

template <uint32_t N>
__device__ __forceinline__ Operand<N> split(const float (&x)[8])
{
  Operand<N> r;
  float left[8];
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) left[i] = x[i];
#pragma unroll
  for (uint32_t p = 0; p < N; ++p) {
    uint32_t word[4];
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) word[i] = next_parts(left[2 * i], left[2 * i + 1]);
    __builtin_memcpy(&r.part[p], word, 16);
  }
  return r;
}

template <typename T>
__device__ __forceinline__ Operand<kPartsOf<T>> operand(const Run<T, 8> &x)
{
  if constexpr (std::is_same<T, __bf16>::value) {
    Operand<1> r;
    r.part[0] = __builtin_bit_cast(Parts8, x);
    return r;
  } else {
    float f[8];
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) f[i] = element<8, T>(x, i);
    return split<kPartsOf<T>>(f);
  }
}

// Eight numbers as prepared operands hold them: as they are, or f16 in its parts, as many bytes as 32 bits.  Parts spare a wave that takes
// a piece's keys 960 instructions, and are more to ask for; so they are for a few workgroups (1 x 16384 steps of 8 heads of 128 x 128
// 1.24 ms without, 1.03 with them) and not for many (4 x 4096 of 16 heads 522 us and 558, its gradient 1230 and 1409).
template <typename T, uint32_t KS, uint32_t kSlices>
constexpr bool kInParts = std::is_same<T, _Float16>::value && KS == 4 && kSlices == 1;
template <typename T, bool kParts>
using Stored = std::conditional_t<kParts, Operand<kPartsOf<T>>, Run<T, 8>>;
template <typename T>
__device__ __forceinline__ Operand<kPartsOf<T>> prepared(const Run<T, 8> &x) { return operand<T>(x); }
template <typename T>
__device__ __forceinline__ Operand<kPartsOf<T>> prepared(const Operand<kPartsOf<T>> &x) { return x; }

// acc + A B over 32: of the parts' products all but second with third and third with third.
template <uint32_t NA, uint32_t NB>
__device__ __forceinline__ void multiply(Tile &acc, const Operand<NA> &a, const Operand<NB> &b)
{
#pragma unroll
  for (uint32_t i = 0; i < NA; ++i)
#pragma unroll
    for (uint32_t j = 0; j < NB; ++j)
      if (i + j < 3) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.part[i], b.part[j], acc, 0, 0, 0);
}

// Two tiles on top of each other as the right operand of the next product: a lane of group q has rows 8 q .. 8 q + 7 of the 32 if
// row 4 q + e of the first tile is row 8 q + e, and of the second row 8 q + 4 + e.  Tiles of steps and of a state's rows are
// laid out that way, so that what one product leaves is what the next one takes, without a lane's data leaving it.
__device__ __forceinline__ uint32_t tile_row(uint32_t tile, uint32_t m) { return tile / 2 * 32 + m / 4 * 8 + tile % 2 * 4 + m % 4; }

template <uint32_t N>
__device__ __forceinline__ Operand<N> operand_of(const Tile &x, const Tile &y)
{
  const float f[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
  return split<N>(f);
}

// ---- what does not depend on a state, for every piece: its gates, M and P (or their transposes) and, by the first of the value
// heads that share them, the keys and queries and their transposes, in the order in which the kernels behind take them as operands:
// 64 lanes times 8 numbers, lane l has row l % 16 of the tile and numbers 8 (l / 16) .. + 7 of the 32.  (Rows of a strided array are far
// apart, often in the same channel of a cache, and were asked for by every 16 columns of every head: 773 us in place of 684.)
// Bound by what it writes, 78 KB for a piece and head in 16 bits: 216 us for 4 x 8192 steps of 16 heads, 3.0 TB/s, forwards, and 254
// backwards.  M's substitution is by blocks of 16: the inverses on the diagonal by a lane per column, all else by 32-bit
// matrix instructions, with what they leave taken as it lies (row by row for all 64, and keys by 32-bit instructions, 485 us when this was 240).
constexpr uint32_t kOperand = 64 * 8;                         // numbers
constexpr uint32_t kTriangle = 6;                             // operands of a triangular matrix: 4 tiles of rows by 2 of 32 steps, less 2
constexpr uint32_t kGateWords = 512;

static_assert(sizeof(Gates) <= kGateWords * 4);

struct Prepared {
  uint32_t *gates;   // [heads][kGateWords]: Gates
  __bf16 *M, *P;     // [heads][kTriangle][3][kOperand]
  void *K, *Q;       // [key heads][4][KS][kWave] of Stored: keys and queries
  void *Kt, *Qt;     // [key heads][2 KS][2][kWave] of Stored: their transposes
  void *V;           // [heads][ceil(Dv / 16)][kWave][16]: values, backwards dO, as a wave that has 16 columns takes them
  __bf16 *rows;      // M beside its transpose (for the gradient)
};

// The operand of rows and columns of a triangular matrix: f -> (tile of rows, 32 steps).
__device__ __forceinline__ void triangle(uint32_t f, bool upper, uint32_t *r, uint32_t *s)
{
  if (upper)
    *r = f < 4 ? f / 2 : f - 2, *s = f < 4 ? f % 2 : 1;
  else
    *r = f < 2 ? f : 2 + (f - 2) / 2, *s = f < 2 ? 0 : (f - 2) % 2;
}

// Eight numbers of a row from `d` on, zeros beyond `width`: one by one, without a branch, so that many such loads are on their way
// at once.
template <typename T>
__device__ __forceinline__ Run<T, 8> load_eight(const T *row, uint32_t d, uint32_t width)
{
  Run<T, 8> r;
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) {
    const T x = row[min(d + i, width - 1)];
    r[i] = d + i < width ? x : (T)0.0f;
  }
  return r;
}

// Row t of a piece's `have` steps; beyond them zeros, and the last one is fetched.  kWhole: eights end within the width.
template <typename T, bool kWhole>
__device__ __forceinline__ Run<T, 8> load_step(const T *piece, uint64_t stride, uint32_t t, uint32_t have, uint32_t d, uint32_t width)
{
  const T *const row = piece + min(t, have - 1) * stride;
  const Run<T, 8> r = kWhole ? load_run<T, 8>(row + d) : load_eight<T>(row, d, width);
  return t < have ? r : Run<T, 8>{};
}

template <typename T, uint32_t KS, bool kBack, bool kParts>
__global__ __launch_bounds__(kDeltaThreads) void delta_prepare_kernel(DeltaArgs a, const void *d_o, Prepared w)
{
  constexpr uint32_t kRaw = KS * 32 + 16 / sizeof(T);  // (rows begin on 16 bytes)
  __shared__ Gates gates;
  __shared__ __align__(16) float L[kPiece * kPieceRow], P[kPiece * kPieceRow];
  __shared__ __align__(16) T raw[kPiece][kRaw];  // (three workgroups a compute unit)
  const auto inverse = [&](uint32_t block, uint32_t t, uint32_t j) -> float & {  // in the blocks above L's diagonal
    return L[((block == 3 ? 16 : 0) + t) * kPieceRow + (block == 3 ? 32 : 16 * block + 16) + j];
  };
  const uint32_t h = blockIdx.x % a.H, piece = blockIdx.x / a.H % a.pieces, s = blockIdx.x / a.H / a.pieces, hk = h / a.share;
  const uint32_t len = delta_length(a, s), t0 = piece * kPiece;
  if (t0 >= len) return;
  const uint32_t have = min(kPiece, len - t0);
  const uint32_t lane = lane_id(), wave = threadIdx.x / kWave, m = lane % 16, q = lane / 16;
  const bool first = h % a.share == 0;  // of those that share a key head
  {
    const T *const rows = kBack ? static_cast<const T *>(d_o) + (((uint64_t)s * a.T + t0) * a.H + h) * a.Dv
                                : static_cast<const T *>(a.v) + s * a.v_seq + t0 * a.v_time + (uint64_t)h * a.Dv;
    const uint64_t stride = kBack ? (uint64_t)a.H * a.Dv : a.v_time;
    const uint32_t slices = (a.Dv + 15) / 16;
    for (uint32_t c0 = 0; c0 < a.Dv; c0 += KS * 32) {
      const auto load = [&](auto whole) {
        constexpr uint32_t kEach = kPiece * KS * 4 / kDeltaThreads;
        Run<T, 8> x[kEach];
#pragma unroll
        for (uint32_t n = 0; n < kEach; ++n) {
          const uint32_t i = n * kDeltaThreads + threadIdx.x;
          x[n] = load_step<T, decltype(whole)::value>(rows, stride, i / (KS * 4), have, c0 + i % (KS * 4) * 8, a.Dv);
        }
#pragma unroll
        for (uint32_t n = 0; n < kEach; ++n) {
          const uint32_t i = n * kDeltaThreads + threadIdx.x;
          *reinterpret_cast<Run<T, 8> *>(&raw[i / (KS * 4)][i % (KS * 4) * 8]) = x[n];
        }
      };
      if (a.Dv % (KS * 32))
        load(std::false_type());
      else
        load(std::true_type());
      __syncthreads();
      for (uint32_t i = wave; i < 2 * KS; i += kDeltaWaves) {
        if (c0 / 16 + i >= slices) break;
        T *const to = static_cast<T *>(w.V) + (((uint64_t)blockIdx.x * slices + c0 / 16 + i) * kWave + lane) * 16;
#pragma unroll
        for (uint32_t n = 0; n < 2; ++n) {
          Run<T, 8> x;
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) x[e] = raw[tile_row(2 * n + e / 4, q * 4 + e % 4)][i * 16 + m];
          *reinterpret_cast<Run<T, 8> *>(to + n * 8) = x;
        }
      }
      __syncthreads();
    }
  }
  const T *const k_rows = static_cast<const T *>(a.k) + s * a.k_seq + t0 * a.k_time + (uint64_t)hk * a.Dk;
  const T *const q_rows = static_cast<const T *>(a.q) + s * a.q_seq + t0 * a.q_time + (uint64_t)hk * a.Dk;
  Run<T, 8> k_own[KS], q_own[KS];
  const auto load_own = [&](auto whole) {
#pragma unroll
    for (uint32_t i = 0; i < KS; ++i) {
      k_own[i] = load_step<T, decltype(whole)::value>(k_rows, a.k_time, wave * 16 + m, have, i * 32 + q * 8, a.Dk);
      q_own[i] = load_step<T, decltype(whole)::value>(q_rows, a.q_time, wave * 16 + m, have, i * 32 + q * 8, a.Dk);
    }
  };
  if (a.Dk == KS * 32)
    load_own(std::true_type());
  else
    load_own(std::false_type());
  if (wave == 0) load_gates(a, s, h, t0, len, gates);
  const auto put_raw = [&](const Run<T, 8>(&x)[KS]) {
#pragma unroll
    for (uint32_t i = 0; i < KS; ++i) *reinterpret_cast<Run<T, 8> *>(&raw[wave * 16 + m][i * 32 + q * 8]) = x[i];
  };
  const uint64_t key_head = ((uint64_t)s * a.pieces + piece) * a.Hk + hk;
  const auto put_eight = [&](void *to_all, uint64_t at, const Run<T, 8> &x) {
    if constexpr (kParts)
      static_cast<Stored<T, true> *>(to_all)[at] = operand<T>(x);
    else
      static_cast<Stored<T, false> *>(to_all)[at] = x;
  };
  const auto put_columns = [&](void *to_all) {
    for (uint32_t i = threadIdx.x; i < 2 * KS * 2 * kWave; i += kDeltaThreads) {
      const uint32_t l = i % kWave, ks = i / kWave % 2, tile = i / kWave / 2, d = tile_row(tile, l % 16), t = ks * 32 + l / 16 * 8;
      Run<T, 8> x;
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e) x[e] = raw[t + e][d];
      put_eight(to_all, ((key_head * 2 * KS + tile) * 2 + ks) * kWave + l, x);
    }
  };
  // this wave's rows as operands: row t is row m of tile r
  const auto put_rows = [&](void *to_all, const Run<T, 8>(&x)[KS]) {
    const uint32_t t = wave * 16 + m, r = t / 32 * 2 + t / 4 % 2, row = t / 8 % 4 * 4 + t % 4;
#pragma unroll
    for (uint32_t i = 0; i < KS; ++i)
      put_eight(to_all, (key_head * 4 * KS + r * KS + i) * kWave + q * 16 + row, x[i]);
  };
  put_raw(k_own);
  __syncthreads();
  for (uint32_t c = 0; c < 4; ++c) {
    Tile kk{}, qk{};
    if (c <= wave) {
#pragma unroll
      for (uint32_t i = 0; i < KS; ++i) {
        Run<T, 8> key;
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) key[e] = raw[c * 16 + m][i * 32 + q * 8 + e];
        multiply(kk, operand<T>(k_own[i]), operand<T>(key));
        multiply(qk, operand<T>(q_own[i]), operand<T>(key));
      }
    }
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
      const uint32_t t = wave * 16 + q * 4 + e, j = c * 16 + m;
      const float d = decay(gates, t, j);
      L[t * kPieceRow + j] = j < t ? kk[e] * d : 0.0f;
      P[t * kPieceRow + j] = j <= t ? qk[e] * d : 0.0f;
    }
  }
  if (first) {
    put_rows(w.K, k_own);
    put_columns(w.Kt);
    if (!kBack) put_rows(w.Q, q_own);
  }
  __syncthreads();
  if (kBack) put_raw(q_own);
  // (1 + L diag(beta))^-1 of the four blocks on the diagonal: a lane has a column
  if (wave == 0) {
    float x[16];
#pragma unroll
    for (uint32_t t = 0; t < 16; ++t) {
      x[t] = t == m ? 1.0f : 0.0f;
#pragma unroll
      for (uint32_t i = 0; i < t; ++i) x[t] -= L[(q * 16 + t) * kPieceRow + q * 16 + i] * x[i];
      inverse(q, t, m) = x[t];
      x[t] *= gates.beta[q * 16 + t];  // (as the rows below take it)
    }
  }
  __syncthreads();
  if (kBack && first) put_columns(w.Qt);
  // M, block row by block row: a wave has a column of blocks, in the layout that the next product takes
  Tile M[4];
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    M[i] = Tile{};
    if (i < wave) continue;
    Tile x;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) x[e] = L[(i * 16 + q * 4 + e) * kPieceRow + wave * 16 + m];
#pragma unroll
    for (uint32_t j = 0; j < i; ++j)
      if (j >= wave) {
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
          const uint32_t k = j * 16 + q * 4 + e;
          x = __builtin_amdgcn_mfma_f32_16x16x4f32(-L[(i * 16 + m) * kPieceRow + k] * gates.beta[k], M[j][e], x, 0, 0, 0);
        }
      }
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) M[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(inverse(i, m, q * 4 + e), x[e], M[i], 0, 0, 0);
  }
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) L[(i * 16 + q * 4 + e) * kPieceRow + wave * 16 + m] = M[i][e];
  __syncthreads();
  const uint64_t head = blockIdx.x;
  for (uint32_t i = threadIdx.x; i < (kBack ? 3 : 2) * kTriangle * kWave; i += kDeltaThreads) {
    const uint32_t f = i / kWave % kTriangle, l = i % kWave, which = i / kWave / kTriangle;  // M, P, M beside its transpose
    const float *const from = which == 1 ? P : L;
    const bool turned = kBack && which < 2;
    uint32_t r, ks;
    triangle(f, turned, &r, &ks);
    const uint32_t row = tile_row(r, l % 16), col = ks * 32 + l / 16 * 8;
    float x[8];
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) x[e] = turned ? from[(col + e) * kPieceRow + row] : from[row * kPieceRow + col + e];
    const Operand<3> parts = split<3>(x);
    __bf16 *const to = (which == 0 ? w.M : which == 1 ? w.P : w.rows) + ((head * kTriangle + f) * 3) * kOperand + l * 8;
#pragma unroll
    for (uint32_t p = 0; p < 3; ++p) *reinterpret_cast<Parts8 *>(to + p * kOperand) = parts.part[p];
  }
  for (uint32_t i = threadIdx.x; i < sizeof(Gates) / 4; i += kDeltaThreads) w.gates[head * kGateWords + i] = reinterpret_cast<const uint32_t *>(&gates)[i];
}

// ---- from piece to piece.  A workgroup of two waves has 16 columns of a state, all its rows, and a wave's products need nothing
// but what the wave has itself and left operands from memory: no barrier within a piece.  One wave carries the state on, the other
// does what nobody waits for, a piece behind (outputs) or ahead (what the gradient of the state takes in from outside).
// Workgroups of a head, which read the same operands, are 8 apart: on one chiplet, whose L2 cache they share.
struct PiecePlace {
  uint32_t s, h, c0;
  bool none;
};
template <uint32_t kSlices>
__device__ __forceinline__ PiecePlace piece_place(const DeltaArgs &a, uint32_t slice)
{
  const uint32_t groups = (a.Dv + 16 * kSlices - 1) / (16 * kSlices), heads = a.S * a.H;
  const uint32_t head = blockIdx.x / (8 * groups) * 8 + blockIdx.x % 8;
  return PiecePlace{head / a.H, head % a.H, (blockIdx.x / 8 % groups * kSlices + slice) * 16, head >= heads};
}

// Both waves have arrived, and what they wrote to LDS is there.  Loads from memory stay on their way.
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <uint32_t N>
__device__ __forceinline__ void put(__bf16 *to, const Operand<N> &x)
{
#pragma unroll
  for (uint32_t p = 0; p < N; ++p) *reinterpret_cast<Parts8 *>(to + p * kOperand + lane_id() * 8) = x.part[p];
}
template <uint32_t N>
__device__ __forceinline__ Operand<N> get(const __bf16 *from)
{
  Operand<N> x;
#pragma unroll
  for (uint32_t p = 0; p < N; ++p) x.part[p] = *reinterpret_cast<const Parts8 *>(from + p * kOperand + lane_id() * 8);
  return x;
}

// The gates of the rows of a lane's part of a tile of steps.
struct RowGates {
  Tile tile[4];
};
struct AllGates {
  RowGates beta, begin, end;
  float last;
};
__device__ __forceinline__ RowGates row_gates(const float *gates)
{
  RowGates r;
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) r.tile[i] = *reinterpret_cast<const Tile *>(gates + i / 2 * 32 + lane_id() / 16 * 8 + i % 2 * 4);
  return r;
}

__device__ __forceinline__ const Gates &gates_of(const Prepared &w, uint64_t head) { return *reinterpret_cast<const Gates *>(w.gates + head * kGateWords); }
__device__ __forceinline__ AllGates all_gates(const Gates &gates)
{
  return AllGates{row_gates(gates.beta), row_gates(gates.begin), row_gates(gates.end), gates.last};
}

__device__ __forceinline__ Tile scaled(const Tile &x, const Tile &by)
{
  Tile r;
#pragma unroll
  for (uint32_t e = 0; e < 4; ++e) r[e] = x[e] * by[e];
  return r;
}
// by x, or 0 where by is, whatever x is: nothing of what has ended passes.
__device__ __forceinline__ Tile passed(const Tile &x, const Tile &by)
{
  Tile r;
#pragma unroll
  for (uint32_t e = 0; e < 4; ++e) r[e] = by[e] != 0.0f ? x[e] * by[e] : 0.0f;
  return r;
}

// x, of which the compiler knows nothing more: what is computed from it is computed where it is used, not ahead of a loop and kept
// in registers through it.
__device__ __forceinline__ uint32_t anew(uint32_t x)
{
  asm volatile("" : "+v"(x));
  return x;
}

// A product's result in registers that ordinary instructions take, once for all that is computed from it (else the compiler copies a state
// of a piece twice, 32 instructions of 1070).
__device__ __forceinline__ void held(Tile &x) { asm("" : "+v"(x)); }

// What the kernels take of a piece, as it is in memory: asked for a piece ahead, made operands when it is used.  Behind a
// sequence's last step that one is fetched again: its strength there is 0, and so is all that comes of it.
// `near`: 64 rows apart are less than 2^32 bytes apart, and there are 64: a lane's place is an offset from an address that all share.
constexpr uint64_t kNearStride = 1u << 23;

template <typename T>
struct PieceColumn {  // a lane's numbers of tiles of steps: rows of a strided array, this lane's column
  T x[4][4];
  __device__ __forceinline__ void load(const T *piece, uint64_t stride, uint32_t have, uint32_t column)
  {
    const uint32_t q = lane_id() / 16;
    if (have == kPiece && stride <= kNearStride) {
      const uint32_t offset = (q * 8 * (uint32_t)stride + column) * sizeof(T);
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) x[i][e] = *reinterpret_cast<const T *>(reinterpret_cast<const char *>(piece + (i / 2 * 32 + i % 2 * 4 + e) * stride) + offset);
    } else {
      const uint32_t m = anew(q * 4);
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) x[i][e] = piece[min(tile_row(i, m + e), have - 1) * stride + column];
    }
  }
  __device__ __forceinline__ Tile tile(uint32_t i) const { return Tile{(float)x[i][0], (float)x[i][1], (float)x[i][2], (float)x[i][3]}; }
};
template <typename T>
struct PieceSlice {  // the same, prepared
  Run<T, 8> x[2];
  __device__ __forceinline__ void load(const void *from, uint64_t slice)
  {
    const T *const p = static_cast<const T *>(from) + (slice * kWave + lane_id()) * 16;
#pragma unroll
    for (uint32_t n = 0; n < 2; ++n) x[n] = *reinterpret_cast<const Run<T, 8> *>(p + n * 8);
  }
  __device__ __forceinline__ Tile tile(uint32_t i) const
  {
    Tile r;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) r[e] = element<8, T>(x[i / 2], i % 2 * 4 + e);
    return r;
  }
};
// f(t, address): every step of a lane's part of tiles of steps that a sequence has, and where its number is.
template <typename T, typename F>
__device__ __forceinline__ void each_step(T *piece, uint64_t stride, uint32_t have, uint32_t column, F f)
{
  const uint32_t q = lane_id() / 16;
  if (have == kPiece && stride <= kNearStride) {
    const uint32_t offset = (q * 8 * (uint32_t)stride + column) * sizeof(T);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) f(i, e, reinterpret_cast<T *>(reinterpret_cast<char *>(piece + (i / 2 * 32 + i % 2 * 4 + e) * stride) + offset));
  } else {
    const uint32_t m = anew(q * 4);
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t t = tile_row(i, m + e);
        if (t < have) f(i, e, piece + t * stride + column);
      }
  }
}
template <typename T, uint32_t KS, bool kParts, uint32_t kTiles = 4>
struct PieceKeys {  // rows of keys or queries, prepared: tiles of steps from `first` on
  Stored<T, kParts> x[kTiles][KS];
  __device__ __forceinline__ void load(const void *from, uint64_t key_head, uint32_t first = 0)
  {
    const Stored<T, kParts> *const p = static_cast<const Stored<T, kParts> *>(from) + (key_head * 4 + first) * KS * kWave + lane_id();
#pragma unroll
    for (uint32_t i = 0; i < kTiles; ++i)
#pragma unroll
      for (uint32_t s = 0; s < KS; ++s) x[i][s] = p[(i * KS + s) * kWave];
  }
};
template <typename T, uint32_t KS, bool kParts>
struct PieceColumns {  // their transposes, prepared
  Stored<T, kParts> x[2 * KS][2];
  __device__ __forceinline__ void load(const void *from, uint64_t key_head)
  {
    const Stored<T, kParts> *const p = static_cast<const Stored<T, kParts> *>(from) + key_head * (2 * KS * 2 * kWave) + lane_id();
#pragma unroll
    for (uint32_t i = 0; i < 2 * KS; ++i)
#pragma unroll
      for (uint32_t s = 0; s < 2; ++s) x[i][s] = p[(i * 2 + s) * kWave];
  }
};
struct PieceTriangle {
  Operand<3> x[kTriangle];
  __device__ __forceinline__ void load(const __bf16 *from, uint64_t head)
  {
    const __bf16 *const p = from + head * (kTriangle * 3 * kOperand) + lane_id() * 8;
#pragma unroll
    for (uint32_t f = 0; f < kTriangle; ++f)
#pragma unroll
      for (uint32_t n = 0; n < 3; ++n) x[f].part[n] = *reinterpret_cast<const Parts8 *>(p + (f * 3 + n) * kOperand);
  }
  // acc + the matrix times right, whose operands are its rows 0..31 and 32..63
  template <bool kUpper, uint32_t NB>
  __device__ __forceinline__ void times(Tile (&acc)[4], const Operand<NB> (&right)[2]) const
  {
#pragma unroll
    for (uint32_t f = 0; f < kTriangle; ++f) {
      const uint32_t r = kUpper ? (f < 4 ? f / 2 : f - 2) : (f < 2 ? f : 2 + (f - 2) / 2);
      const uint32_t s = kUpper ? (f < 4 ? f % 2 : 1) : (f < 2 ? 0 : (f - 2) % 2);
      multiply(acc[r], x[f], right[s]);
    }
  }
};

// A state's tile i, element e of a lane is its row.
__device__ __forceinline__ uint32_t state_row(uint32_t tile, uint32_t e) { return tile_row(tile, lane_id() / 16 * 4 + e); }

template <uint32_t KS>
__device__ __forceinline__ void load_state(Tile (&S)[2 * KS], const float *from, uint32_t Dk, uint32_t Dv, uint32_t c0)
{
  const uint32_t q = lane_id() / 16, c = c0 + lane_id() % 16;
  if (Dk == KS * 32 && c0 + 16 <= Dv) {
    const uint32_t offset = (q * 8 * Dv + c) * 4;
#pragma unroll
    for (uint32_t i = 0; i < 2 * KS; ++i)
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) S[i][e] = *reinterpret_cast<const float *>(reinterpret_cast<const char *>(from + (i / 2 * 32 + i % 2 * 4 + e) * Dv) + offset);
  } else {
    const uint32_t m = anew(q * 4);
#pragma unroll
    for (uint32_t i = 0; i < 2 * KS; ++i)
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t d = tile_row(i, m + e);
        const float x = from[min(d, Dk - 1) * Dv + min(c, Dv - 1)];
        S[i][e] = d < Dk && c < Dv ? x : 0.0f;
      }
  }
}
template <uint32_t KS>
__device__ __forceinline__ void store_state(const Tile (&S)[2 * KS], float *to, uint32_t Dk, uint32_t Dv, uint32_t c0)
{
  const uint32_t q = lane_id() / 16, c = c0 + lane_id() % 16;
  if (Dk == KS * 32 && c0 + 16 <= Dv) {
    const uint32_t offset = (q * 8 * Dv + c) * 4;
#pragma unroll
    for (uint32_t i = 0; i < 2 * KS; ++i)
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) *reinterpret_cast<float *>(reinterpret_cast<char *>(to + (i / 2 * 32 + i % 2 * 4 + e) * Dv) + offset) = S[i][e];
  } else if (c < Dv) {
    const uint32_t m = anew(q * 4);
#pragma unroll
    for (uint32_t i = 0; i < 2 * KS; ++i)
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t d = tile_row(i, m + e);
        if (d < Dk) to[d * Dv + c] = S[i][e];
      }
  }
}
// States that only these kernels read (the carry and its gradient) lie by 16 columns, [ceil(Dv / 16)][rows][16], the rows of every
// 32 in the order 0, 8, 16, 24, 1, 9 ..: what a wave reads or writes of them with one instruction is 256 bytes in one place.  (By rows of Dv an instruction has 64 bytes
// out of every 512: without the carry's stores the forward kernel of 4 x 8192 steps of 16 heads took 480 us in place of 621.)
__device__ __forceinline__ uint32_t slice_size(uint32_t Dk) { return (Dk + 31) / 32 * 32 * 16; }
__device__ __forceinline__ uint64_t slices_size(uint32_t Dk, uint32_t Dv) { return (uint64_t)((Dv + 15) / 16) * slice_size(Dk); }
__device__ __forceinline__ uint32_t slice_row(uint32_t d) { return d / 32 * 32 + d % 8 * 4 + d / 8 % 4; }

// A state of which the three parts are held: their sum is exact.  Zeros where `column` is false.
template <uint32_t KS>
__device__ __forceinline__ void store_slice(const Operand<3> (&S)[KS], float *to, uint32_t Dk, uint32_t slice, bool column)
{
  float *const lane_to = to + slice * slice_size(Dk) + lane_id();
#pragma unroll
  for (uint32_t s = 0; s < KS; ++s) {
    if (s * 32 >= Dk) break;
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) {
      const float x = ((float)S[s].part[2][e] + (float)S[s].part[1][e]) + (float)S[s].part[0][e];
      lane_to[(s * 8 + e) * kWave] = column ? x : 0.0f;  // (rows beyond Dk: zeros, as the keys' are)
    }
  }
}
template <uint32_t KS>
__device__ __forceinline__ void load_slice(Tile (&S)[2 * KS], const float *from, uint32_t Dk, uint32_t slice)
{
  const float *const lane_from = from + slice * slice_size(Dk) + lane_id();
#pragma unroll
  for (uint32_t s = 0; s < KS; ++s)
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) S[2 * s + e / 4][e % 4] = s * 32 < Dk ? lane_from[(s * 8 + e) * kWave] : 0.0f;
}

// What the next piece takes is asked for as soon as this one has taken its own: in the same registers, which a wave has 512 of.
// (Numbers of 32 bits are twice as many; there a piece's are asked for at its begin.)
// Bound by the chain from piece to piece: X, E, U and the state, 132 products of tiles and some 850 other instructions of one wave in
// bf16, 5900 cycles, and as long again for the requests to be taken while four waves of a compute unit ask for 330 KB a piece: 4 x 8192
// steps of 16 heads of 128 x 128 in bf16 595 us, 4.6 us a piece (without any loads and stores 163); f16, whose keys are two parts,
// 1 x 16384 of 8 heads 930 us, 3.6 a piece (1125, with keys that were cut into parts where they were taken); f32 6.7 a piece, with 7 registers
// of wide states in scratch.  With 32-bit matrix instructions, all in LDS, 52 us a piece.
template <typename T, uint32_t KS, uint32_t kSlices>
__global__ __launch_bounds__(2 * kSlices * kWave) void delta_pieces_kernel(DeltaForward f, Prepared w)
{
  constexpr bool kAhead = sizeof(T) == 2, kParts = kInParts<T, KS, kSlices>;
  __shared__ __align__(16) __bf16 all_states[kSlices][2][KS][3 * kOperand];
  __shared__ Tile all_corrections[kSlices][2][4][kWave];  // U
  const uint32_t slice = threadIdx.x / kWave % kSlices;
  auto &states = all_states[slice];
  auto &corrections = all_corrections[slice];
  const DeltaArgs &a = f.n;
  const PiecePlace place = piece_place<kSlices>(a, slice);
  if (place.none) return;
  const uint32_t s = place.s, h = place.h, hk = h / a.share, lane = lane_id(), c = place.c0 + lane % 16;
  const bool column = c < a.Dv, carries = threadIdx.x < kSlices * kWave;
  const uint32_t len = delta_length(a, s), pieces = (len + kPiece - 1) / kPiece, slices = (a.Dv + 15) / 16;
  const uint64_t state = ((uint64_t)s * a.H + h) * a.Dk * a.Dv;
  const auto head_of = [&](uint32_t piece) { return ((uint64_t)s * a.pieces + piece) * a.H + h; };
  const auto have_of = [&](uint32_t piece) { return min(kPiece, len - piece * kPiece); };
  if (carries) {
    Tile S[2 * KS] = {};
    if (f.h0) load_state<KS>(S, f.h0 + state, a.Dk, a.Dv, place.c0);
    PieceKeys<T, KS, kParts> K;
    PieceSlice<T> V;
    PieceTriangle M;
    PieceColumns<T, KS, kParts> Kt;
    AllGates gates;
    const auto load_keys = [&](uint32_t piece) {
      K.load(w.K, ((uint64_t)s * a.pieces + piece) * a.Hk + hk);
      V.load(w.V, head_of(piece) * slices + min(place.c0 / 16, slices - 1));
    };
    const auto load_columns = [&](uint32_t piece) {
      Kt.load(w.Kt, ((uint64_t)s * a.pieces + piece) * a.Hk + hk);
      gates = all_gates(gates_of(w, head_of(piece)));
    };
    if (pieces) load_keys(0), M.load(w.M, head_of(0)), load_columns(0);
    for (uint32_t piece = 0; piece < pieces; ++piece) {
      const uint32_t next = min(piece + 1, pieces - 1);
      if (!kAhead && piece) load_keys(piece), M.load(w.M, head_of(piece)), load_columns(piece);
      Tile kS[4] = {}, X[4];
#pragma unroll
      for (uint32_t i = 0; i < KS; ++i) {
        held(S[2 * i]), held(S[2 * i + 1]);
        const Operand<3> parts = operand_of<3>(S[2 * i], S[2 * i + 1]);
        put(states[piece % 2][i], parts);
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) multiply(kS[r], prepared<T>(K.x[r][i]), parts);
      }
#pragma unroll
      for (uint32_t r = 0; r < 4; ++r) X[r] = V.tile(r) - passed(kS[r], gates.begin.tile[r]);
      if (kAhead) load_keys(next);
      const Operand<3> bX[2] = {operand_of<3>(scaled(X[0], gates.beta.tile[0]), scaled(X[1], gates.beta.tile[1])),
                                operand_of<3>(scaled(X[2], gates.beta.tile[2]), scaled(X[3], gates.beta.tile[3]))};
      Tile mX[4] = {}, U[4];
      M.times<false>(mX, bX);
      if (kAhead) M.load(w.M, head_of(next));
#pragma unroll
      for (uint32_t r = 0; r < 4; ++r) U[r] = scaled(X[r] - mX[r], gates.beta.tile[r]);
#pragma unroll
      for (uint32_t r = 0; r < 4; ++r) corrections[piece % 2][r][lane] = U[r];
      const Operand<3> left[2] = {operand_of<3>(scaled(U[0], gates.end.tile[0]), scaled(U[1], gates.end.tile[1])),
                                  operand_of<3>(scaled(U[2], gates.end.tile[2]), scaled(U[3], gates.end.tile[3]))};
#pragma unroll
      for (uint32_t i = 0; i < 2 * KS; ++i) {
        S[i] = gates.last != 0.0f ? S[i] * gates.last : Tile{};
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) multiply(S[i], prepared<T>(Kt.x[i][j]), left[j]);
      }
      if (kAhead) load_columns(next);
      meet();
    }
    if (f.h_last) {
      if (len && !delta_passes(a, s, len - 1)) {
#pragma unroll
        for (uint32_t i = 0; i < 2 * KS; ++i) S[i] = Tile{};
      }
      store_state<KS>(S, f.h_last + state, a.Dk, a.Dv, place.c0);
    }
  } else {
    T *const o = static_cast<T *>(f.o) + ((uint64_t)s * a.T * a.H + h) * a.Dv;
    const uint64_t o_row = (uint64_t)a.H * a.Dv;
    PieceKeys<T, KS, kParts> Q;
    PieceTriangle P;
    RowGates begin;
    uint32_t enters = 0;
    const auto load = [&](uint32_t piece) {
      Q.load(w.Q, ((uint64_t)s * a.pieces + piece) * a.Hk + hk);
      P.load(w.P, head_of(piece));
      begin = row_gates(gates_of(w, head_of(piece)).begin);
      enters = gates_of(w, head_of(piece)).enters;
    };
    if (pieces) load(0);
    for (uint32_t piece = 0; piece < pieces; ++piece) {
      if (!kAhead && piece) load(piece);
      meet();
      Tile O[4] = {};
      Operand<3> S[KS];
#pragma unroll
      for (uint32_t i = 0; i < KS; ++i) {
        S[i] = get<3>(states[piece % 2][i]);
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) multiply(O[r], prepared<T>(Q.x[r][i]), S[i]);
      }
#pragma unroll
      for (uint32_t r = 0; r < 4; ++r) O[r] = passed(O[r], begin.tile[r]);
      const Tile(&found)[4][kWave] = corrections[piece % 2];
      const Operand<3> U[2] = {operand_of<3>(found[0][lane], found[1][lane]), operand_of<3>(found[2][lane], found[3][lane])};
      P.times<false>(O, U);
      // (the state is carried as the last step left it: what an episode's end keeps out of the piece is not stored)
      const bool stored = column && enters;
      if (kAhead) load(min(piece + 1, pieces - 1));
      if (f.carry && place.c0 < a.Dv) store_slice<KS>(S, f.carry + head_of(piece) * slices_size(a.Dk, a.Dv), a.Dk, place.c0 / 16, stored);
      if (column)
        each_step(o + (uint64_t)piece * kPiece * o_row, o_row, have_of(piece), c, [&](uint32_t r, uint32_t e, T *to) { *to = (T)(a.scale * O[r][e]); });
    }
    if (column)
      for (uint64_t t = len + lane / 16; t < a.T; t += 4) o[t * o_row + c] = (T)0.0f;
  }
}

// The same from the last piece to the first, with dS.  The first wave carries it, the second brings P^T dO and Q^T (c dO) and
// stores dS, Y and dV.  Bound as the way there: 712 us, 5.6 us a piece, of 4 x 8192 steps of 16 heads of 128 x 128 in bf16.
template <typename T, uint32_t KS, uint32_t kSlices>
__global__ __launch_bounds__(2 * kSlices * kWave) void delta_pieces_back_kernel(DeltaBack b, Prepared w)
{
  constexpr bool kAhead = sizeof(T) == 2;
  struct Brought {
    Tile o[4][kWave], state[2 * KS][kWave];
  };
  __shared__ Brought all_brought[kSlices][2];
  __shared__ __align__(16) __bf16 all_states[kSlices][2][KS][3 * kOperand];
  __shared__ Tile all_found[kSlices][2][4][kWave];  // Y
  const uint32_t slice = threadIdx.x / kWave % kSlices;
  auto &brought = all_brought[slice];
  auto &states = all_states[slice];
  auto &found = all_found[slice];
  const DeltaArgs &a = b.n;
  const PiecePlace place = piece_place<kSlices>(a, slice);
  if (place.none) return;
  const uint32_t s = place.s, h = place.h, hk = h / a.share, lane = lane_id(), c = place.c0 + lane % 16;
  const bool column = c < a.Dv, carries = threadIdx.x < kSlices * kWave;
  const uint32_t len = delta_length(a, s), pieces = (len + kPiece - 1) / kPiece, slices = (a.Dv + 15) / 16;
  const uint64_t state = ((uint64_t)s * a.H + h) * a.Dk * a.Dv;
  const auto head_of = [&](uint32_t piece) { return ((uint64_t)s * a.pieces + piece) * a.H + h; };
  const auto key_head_of = [&](uint32_t piece) { return ((uint64_t)s * a.pieces + piece) * a.Hk + hk; };
  const auto have_of = [&](uint32_t piece) { return min(kPiece, len - piece * kPiece); };
  if (carries) {
    Tile S[2 * KS] = {};
    if (b.dh_last && (len == 0 || delta_passes(a, s, len - 1))) load_state<KS>(S, b.dh_last + state, a.Dk, a.Dv, place.c0);
    PieceKeys<T, KS, false> K;
    PieceTriangle M;
    PieceColumns<T, KS, false> Kt;
    AllGates gates;
    const auto load_keys = [&](uint32_t piece) { K.load(w.K, key_head_of(piece)); };
    const auto load_columns = [&](uint32_t piece) {
      Kt.load(w.Kt, key_head_of(piece));
      gates = all_gates(gates_of(w, head_of(piece)));
    };
    if (pieces) {
      load_keys(pieces - 1), M.load(w.M, head_of(pieces - 1)), load_columns(pieces - 1);
      meet();
    }
    for (uint32_t piece = pieces; piece-- > 0;) {
      const uint32_t next = piece ? piece - 1 : 0;
      if (!kAhead && piece + 1 < pieces) load_keys(piece), M.load(w.M, head_of(piece)), load_columns(piece);
      Tile kS[4] = {};
#pragma unroll
      for (uint32_t i = 0; i < KS; ++i) {
        held(S[2 * i]), held(S[2 * i + 1]);
        const Operand<3> parts = operand_of<3>(S[2 * i], S[2 * i + 1]);
        put(states[piece % 2][i], parts);
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) multiply(kS[r], prepared<T>(K.x[r][i]), parts);
      }
      if (kAhead) load_keys(next);
      Tile dU[4];
#pragma unroll
      for (uint32_t r = 0; r < 4; ++r) dU[r] = brought[piece % 2].o[r][lane] + scaled(kS[r], gates.end.tile[r]);
      const Operand<3> bU[2] = {operand_of<3>(scaled(dU[0], gates.beta.tile[0]), scaled(dU[1], gates.beta.tile[1])),
                                operand_of<3>(scaled(dU[2], gates.beta.tile[2]), scaled(dU[3], gates.beta.tile[3]))};
      Tile mU[4] = {}, V[4];
      M.times<true>(mU, bU);
      if (kAhead) M.load(w.M, head_of(next));
#pragma unroll
      for (uint32_t r = 0; r < 4; ++r) {
        dU[r] -= mU[r];  // Y
        found[piece % 2][r][lane] = dU[r];
        V[r] = -scaled(scaled(dU[r], gates.beta.tile[r]), gates.begin.tile[r]);
      }
      const Operand<3> left[2] = {operand_of<3>(V[0], V[1]), operand_of<3>(V[2], V[3])};
#pragma unroll
      for (uint32_t i = 0; i < 2 * KS; ++i) {
        S[i] = (gates.last != 0.0f ? S[i] * gates.last : Tile{}) + brought[piece % 2].state[i][lane];
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) multiply(S[i], prepared<T>(Kt.x[i][j]), left[j]);
      }
      if (kAhead) load_columns(next);
      meet();
    }
    if (b.dh0) store_state<KS>(S, b.dh0 + state, a.Dk, a.Dv, place.c0);
  } else {
    T *const dv = static_cast<T *>(b.dv) + s * b.dv_seq + (uint64_t)h * a.Dv;
    PieceSlice<T> taken;
    PieceTriangle P;
    PieceColumns<T, KS, false> Qt;
    RowGates begin;
    const auto load = [&](uint32_t piece) {
      taken.load(w.V, head_of(piece) * slices + min(place.c0 / 16, slices - 1));
      P.load(w.P, head_of(piece));
      Qt.load(w.Qt, key_head_of(piece));
      begin = row_gates(gates_of(w, head_of(piece)).begin);
    };
    const auto bring = [&](uint32_t piece) {
      Tile dO[4];
#pragma unroll
      for (uint32_t r = 0; r < 4; ++r) dO[r] = taken.tile(r);  // (zeros behind the sequence's end)
      const Operand<kPartsOf<T>> right[2] = {operand_of<kPartsOf<T>>(dO[0], dO[1]), operand_of<kPartsOf<T>>(dO[2], dO[3])};
      Tile of_o[4] = {};
      P.times<true>(of_o, right);
#pragma unroll
      for (uint32_t r = 0; r < 4; ++r) {
        brought[piece % 2].o[r][lane] = a.scale * of_o[r];
        dO[r] = scaled(a.scale * dO[r], begin.tile[r]);
      }
      const Operand<3> left[2] = {operand_of<3>(dO[0], dO[1]), operand_of<3>(dO[2], dO[3])};
#pragma unroll
      for (uint32_t i = 0; i < 2 * KS; ++i) {
        Tile x{};
#pragma unroll
        for (uint32_t j = 0; j < 2; ++j) multiply(x, prepared<T>(Qt.x[i][j]), left[j]);
        brought[piece % 2].state[i][lane] = x;
      }
      if (piece) load(piece - 1);
    };
    const auto store = [&](uint32_t piece) {
      const uint64_t head = head_of(piece);
      const uint32_t have = have_of(piece);
      Operand<3> S[KS];
#pragma unroll
      for (uint32_t i = 0; i < KS; ++i) S[i] = get<3>(states[piece % 2][i]);
      if (place.c0 < a.Dv) store_slice<KS>(S, b.dS + head * slices_size(a.Dk, a.Dv), a.Dk, place.c0 / 16, column);
      const RowGates beta = row_gates(gates_of(w, head).beta);
      Tile y[4];
#pragma unroll
      for (uint32_t r = 0; r < 4; ++r) {
        y[r] = found[piece % 2][r][lane];
        if (place.c0 < a.Dv) *reinterpret_cast<Tile *>(b.Y + ((head * slices + place.c0 / 16) * kWave + lane) * 16 + r * 4) = y[r];
      }
      if (column) {
        each_step(dv + (uint64_t)piece * kPiece * b.dv_time, b.dv_time, have, c, [&](uint32_t r, uint32_t e, T *to) { *to = (T)(beta.tile[r][e] * y[r][e]); });
      }
    };
    if (pieces) {
      load(pieces - 1);
      bring(pieces - 1);
      meet();
      for (uint32_t piece = pieces; piece-- > 0;) {
        if (piece) bring(piece - 1);
        if (piece + 1 < pieces) store(piece + 1);
        meet();
      }
      store(0);
    }
    if (column)
      for (uint64_t t = len + lane / 16; t < a.T; t += 4) dv[t * b.dv_time + c] = (T)0.0f;
  }
}

// What is left of the gradient, a workgroup of eight waves (narrow states: four) per piece and key head: first a wave has 16 of the state's columns and all
// steps, and finds U anew; then a wave has a tile of the state's rows and two or four tiles of steps, and sums over the columns.  Between the
// two U and dV cross LDS, in parts.
// Bound by the chain of its phases, one workgroup a compute unit: keys and state, M, 32 columns after another, B and C, their products
// with keys and queries, a wait for memory or for all waves between any two.  4 x 8192 steps of 16 heads of 128 x 128 in bf16 1.08 ms, of
// which its products are 0.19; with 32-bit matrix instructions 3.6.  A wave has 256 registers, and what does not fit lies in scratch: of 16
// bits and wide states 3 to 5 numbers a lane, 28 where columns are no multiple of 32 (narrow 0 and 7); of 32 bits 37 and 68 (15 and 48).
constexpr uint32_t kGradWaves = kDeltaMaxWidth / 16, kGradNarrowWaves = 4;

template <uint32_t kWaves>
struct GradSpace {
  static constexpr uint32_t kRow = kWaves * 16 + 8;
  Gates gates;
  union alignas(16) {  // (eight at a time: at half the alignment a read of them took eight times as long)
    __bf16 part[2][3][kPiece][kRow];  // U, dV; zeros beyond the state's columns
    float B[2][kPiece * kPieceRow];       // B, C
  };
  alignas(16) float of_g[kWaves][kPiece], of_v[kWaves][kPiece], of_beta[kWaves][kPiece];  // sums over a wave's share
  double at_end[kWaves];
};

// The sum over the 16 lanes of a row of a tile, in each of them: rotated by 8, 4, 2 and 1 lanes.
__device__ __forceinline__ float row_sum(float v)
{
  v += dpp_from<0x128, 0xf>(v, 0.0f);
  v += dpp_from<0x124, 0xf>(v, 0.0f);
  v += dpp_from<0x122, 0xf>(v, 0.0f);
  return v + dpp_from<0x121, 0xf>(v, 0.0f);
}

// The parts of a number of each of two matrices, and eight numbers of a row as an operand.  Row: 16 times the tile of steps, and its row
// of that (neighbours are 4 banks apart, whatever steps they are).
template <uint32_t kRow>
__device__ __forceinline__ void put_parts(__bf16 (*part)[3][kPiece][kRow], uint32_t t, uint32_t c, float x, float y)
{
#pragma unroll
  for (uint32_t p = 0; p < 3; ++p) {
    const uint32_t word = next_parts(x, y);
    part[0][p][t][c] = __builtin_bit_cast(__bf16, (uint16_t)word);
    part[1][p][t][c] = __builtin_bit_cast(__bf16, (uint16_t)(word >> 16));
  }
}
template <uint32_t kRow>
__device__ __forceinline__ Operand<3> get_parts(const __bf16 (*part)[kPiece][kRow], uint32_t t, uint32_t c)
{
  Operand<3> x;
#pragma unroll
  for (uint32_t p = 0; p < 3; ++p) x.part[p] = *reinterpret_cast<const Parts8 *>(&part[p][t][c]);
  return x;
}
template <typename T, uint32_t KS, uint32_t kWaves, bool kWhole>
__global__ __launch_bounds__(kWaves * kWave, 2) void delta_gradients_kernel(DeltaBack b, Prepared w)
{
  constexpr uint32_t kGradThreads = kWaves * kWave, kWidths = kWaves / 2;  // (32 columns each)
  constexpr uint32_t kSteps = 8 * KS / kWaves;                             // tiles of steps of a wave
  static_assert((KS == 2 || KS == 4) && kSteps <= 4);
  __shared__ __align__(16) GradSpace<kWaves> x;
  const DeltaArgs &a = b.n;
  const uint32_t hk = blockIdx.x % a.Hk, piece = blockIdx.x / a.Hk % a.pieces, s = blockIdx.x / a.Hk / a.pieces;
  const uint32_t lane = lane_id(), wave = threadIdx.x / kWave;
  const uint32_t len = delta_length(a, s), t0 = piece * kPiece, steps = min(kPiece, a.T - t0);
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
  const uint32_t have = min(kPiece, len - t0);
  const T *const k_rows = static_cast<const T *>(a.k) + s * a.k_seq + t0 * a.k_time + (uint64_t)hk * a.Dk;
  const T *const q_rows = static_cast<const T *>(a.q) + s * a.q_seq + t0 * a.q_time + (uint64_t)hk * a.Dk;
  const uint64_t o_row = (uint64_t)a.H * a.Dv, key_head = ((uint64_t)s * a.pieces + piece) * a.Hk + hk;
  // this wave's tile of the state's rows, and its first tile of steps
  const uint32_t own = wave % (2 * KS), r0 = wave / (2 * KS) * kSteps;
  Tile dq_all[kSteps] = {}, dk_all[kSteps] = {};
#pragma unroll 1
  for (uint32_t h = hk * a.share; h < (hk + 1) * a.share; ++h) {
    const uint64_t head = ((uint64_t)s * a.pieces + piece) * a.H + h;
    const uint32_t m = anew(lane % 16), q = anew(lane / 16), own_d = tile_row(own, m);
    const auto state_row = [&](uint32_t tile, uint32_t e) { return tile_row(tile, q * 4 + e); };
    const float *const S0 = b.carry + head * slices_size(a.Dk, a.Dv), *const dS = b.dS + head * slices_size(a.Dk, a.Dv);
    const T *const v_rows = static_cast<const T *>(a.v) + s * a.v_seq + t0 * a.v_time + (uint64_t)h * a.Dv;
    const T *const o_rows = static_cast<const T *>(b.d_o) + gates_at * a.Dv + (uint64_t)h * a.Dv;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < sizeof(Gates) / 4; i += kGradThreads) reinterpret_cast<uint32_t *>(&x.gates)[i] = w.gates[head * kGateWords + i];
    __syncthreads();
    {
      const uint32_t column = wave * 16 + m, c = min(column, a.Dv - 1);
      Tile U[4] = {}, Y[4] = {}, of_v[4] = {}, of_beta[4] = {};
      if (wave * 16 < a.Dv) {
        Tile kS[4] = {}, S[2 * KS];
        load_slice<KS>(S, S0, a.Dk, wave);
        // (half of the keys at a time, and so on: a wave has 256 registers here)
        PieceKeys<T, KS, false, 2> K;
        K.load(w.K, key_head);
        Operand<3> parts[KS];
#pragma unroll
        for (uint32_t i = 0; i < KS; ++i) {
          parts[i] = operand_of<3>(S[2 * i], S[2 * i + 1]);
#pragma unroll
          for (uint32_t r = 0; r < 2; ++r) multiply(kS[r], prepared<T>(K.x[r][i]), parts[i]);
        }
        __builtin_amdgcn_sched_barrier(0);
        K.load(w.K, key_head, 2);
        PieceColumn<T> V;
        PieceSlice<float> y;
        V.load(v_rows, a.v_time, have, c);
        y.load(b.Y, head * ((a.Dv + 15) / 16) + wave);
#pragma unroll
        for (uint32_t i = 0; i < KS; ++i)
#pragma unroll
          for (uint32_t r = 0; r < 2; ++r) multiply(kS[2 + r], prepared<T>(K.x[r][i]), parts[i]);
        __builtin_amdgcn_sched_barrier(0);
        PieceTriangle M;
        M.load(w.rows, head);
        const RowGates beta = row_gates(x.gates.beta), begin = row_gates(x.gates.begin);
        Tile X[4], mX[4] = {};
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) X[r] = V.tile(r) - passed(kS[r], begin.tile[r]);
        const Operand<3> bX[2] = {operand_of<3>(scaled(X[0], beta.tile[0]), scaled(X[1], beta.tile[1])),
                                  operand_of<3>(scaled(X[2], beta.tile[2]), scaled(X[3], beta.tile[3]))};
        M.times<false>(mX, bX);
        if (column < a.Dv) {
#pragma unroll
          for (uint32_t r = 0; r < 4; ++r) {
            const Tile E = X[r] - mX[r];
            U[r] = scaled(E, beta.tile[r]);
            Y[r] = scaled(y.tile(r), beta.tile[r]);
            of_beta[r] = scaled(y.tile(r), E);
            of_v[r] = scaled(V.tile(r), Y[r]);
          }
        }
      }
#pragma unroll
      for (uint32_t r = 0; r < 4; ++r)
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
          put_parts(x.part, r * 16 + q * 4 + e, column, U[r][e], Y[r][e]);
          of_v[r][e] = row_sum(of_v[r][e]), of_beta[r][e] = row_sum(of_beta[r][e]);
        }
      if (m == 0) {
#pragma unroll
        for (uint32_t r = 0; r < 4; ++r) {
          *reinterpret_cast<Tile *>(&x.of_v[wave][state_row(r, 0)]) = of_v[r];
          *reinterpret_cast<Tile *>(&x.of_beta[wave][state_row(r, 0)]) = of_beta[r];
        }
      }
    }
    __syncthreads();
    Tile oS[kSteps] = {}, uS[kSteps] = {}, vS[kSteps] = {};
    double at_end = 0.0;
    // what 32 columns take from memory, asked for 32 columns ahead
    struct Taken {
      Run<T, 8> o[kSteps];
      Run<float, 8> start, end;
    } next;
    // (clamped: what is fetched beyond the widths meets zeros)
    const auto eight = [&](auto *row, uint32_t c) {
      typedef std::remove_cv_t<std::remove_pointer_t<decltype(row)>> E;
      Run<E, 8> r;
      if constexpr (kWhole) {
        r = load_run<E, 8>(row + min(c, a.Dv - 8));
      } else {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) r[e] = row[min(c + e, a.Dv - 1)];
      }
      return r;
    };
    const uint32_t own_row = slice_row(min(own_d, a.Dk - 1)) * 16 + q % 2 * 8, slices = (a.Dv + 15) / 16;
    const auto take = [&](uint32_t c0) {
      const uint32_t at = min(c0 / 16 + q / 2, slices - 1) * slice_size(a.Dk) + own_row;
      next.start = *reinterpret_cast<const Run<float, 8> *>(S0 + at), next.end = *reinterpret_cast<const Run<float, 8> *>(dS + at);
#pragma unroll
      for (uint32_t i = 0; i < kSteps; ++i) next.o[i] = eight(o_rows + min(tile_row(r0 + i, m), have - 1) * o_row, c0 + q * 8);
    };
    take(0);
#pragma unroll 1
    for (uint32_t c0 = 0; c0 < a.Dv; c0 += 32) {
      const uint32_t c = c0 + q * 8;
      Taken now = next;
      if (c0 + 32 < a.Dv) take(c0 + 32);
      if (!kWhole && c >= slices * 16) now.start = Run<float, 8>{};  // (a slice that there is not)
      const Operand<3> start = operand<float>(now.start), end = operand<float>(now.end);
      if (x.gates.last != 0.0f && own_d < a.Dk && r0 == 0) {
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) at_end += (double)(x.gates.last * now.start[e]) * now.end[e];
      }
#pragma unroll
      for (uint32_t i = 0; i < kSteps; ++i) {
        multiply(oS[i], operand<T>(now.o[i]), start);
        multiply(uS[i], get_parts(x.part[0], (r0 + i) * 16 + m, c), end);
        multiply(vS[i], get_parts(x.part[1], (r0 + i) * 16 + m, c), start);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // B and C: of 16 tiles, those four of later columns than rows are left out; a wave has one, four waves another one
    constexpr uint32_t kRounds = (12 + kWaves - 1) / kWaves;
    Tile B[kRounds] = {}, C[kRounds] = {};
    const auto tile_of = [&](uint32_t i, uint32_t *r, uint32_t *j) {
      const uint32_t f = wave + i * kWaves;
      *r = f < 4 ? f / 2 : 2 + (f - 4) / 4, *j = f < 4 ? f % 2 : (f - 4) % 4;
      return f < 12;
    };
    Run<T, 8> of_tile[kRounds][kWidths];
#pragma unroll
    for (uint32_t i = 0; i < kRounds; ++i) {
      uint32_t r, j;
      tile_of(i, &r, &j);
#pragma unroll
      for (uint32_t n = 0; n < kWidths; ++n) of_tile[i][n] = eight(o_rows + min(tile_row(min(r, 3u), m), have - 1) * o_row, n * 32 + q * 8);
    }
#pragma unroll
    for (uint32_t i = 0; i < kRounds; ++i) {
      uint32_t r, j;
      if (!tile_of(i, &r, &j)) continue;
#pragma unroll
      for (uint32_t n = 0; n < kWidths; ++n) {
        const Operand<3> u = get_parts(x.part[0], j * 16 + m, n * 32 + q * 8);
        multiply(B[i], operand<T>(of_tile[i][n]), u);
        multiply(C[i], get_parts(x.part[1], r * 16 + m, n * 32 + q * 8), u);
      }
    }
    T key_at[kSteps][4], query_at[kSteps][4];  // this lane's of the keys and queries, as tiles
#pragma unroll
    for (uint32_t i = 0; i < kSteps; ++i)
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint64_t t = min(state_row(r0 + i, e), have - 1);
        key_at[i][e] = k_rows[t * a.k_time + min(own_d, a.Dk - 1)], query_at[i][e] = q_rows[t * a.q_time + min(own_d, a.Dk - 1)];
      }
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < kRounds; ++i) {
      uint32_t r, j;
      if (!tile_of(i, &r, &j)) continue;
      j = tile_row(j, m);
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        const uint32_t t = state_row(r, e);
        const float d = decay(x.gates, t, j);
        x.B[0][t * kPieceRow + j] = j <= t && t < have ? a.scale * B[i][e] * d : 0.0f;
        x.B[1][t * kPieceRow + j] = j < t ? C[i][e] * d : 0.0f;
      }
    }
    __syncthreads();
    const Stored<T, false> *const kt = static_cast<const Stored<T, false> *>(w.Kt) + (key_head * 2 * KS + own) * 2 * kWave + lane;
    const Stored<T, false> *const qt = static_cast<const Stored<T, false> *>(w.Qt) + (key_head * 2 * KS + own) * 2 * kWave + lane;
#pragma unroll
    for (uint32_t i = 0; i < kSteps; ++i) {
      const Tile begin = *reinterpret_cast<const Tile *>(&x.gates.begin[state_row(r0 + i, 0)]);
      const Tile end = *reinterpret_cast<const Tile *>(&x.gates.end[state_row(r0 + i, 0)]);
      oS[i] = a.scale * passed(oS[i], begin);
      uS[i] = scaled(uS[i], end);
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) at_end += own_d < a.Dk ? (double)uS[i][e] * (float)key_at[i][e] : 0.0;
      dk_all[i] += uS[i] - passed(vS[i], begin);
    }
#pragma unroll
    for (uint32_t ks = 0; ks < 2; ++ks) {
      const Operand<kPartsOf<T>> key = prepared<T>(kt[ks * kWave]);
      const Operand<kPartsOf<T>> query = prepared<T>(qt[ks * kWave]);
#pragma unroll
      for (uint32_t i = 0; i < kSteps; ++i) {
        const uint32_t r = r0 + i, t = tile_row(r, m), j = ks * 32 + q * 8;
        const bool lower = ks <= r / 2, upper = ks >= r / 2;  // (of the matrix: what lies there is not all zeros)
        float f[8];
        if (lower) {
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) f[e] = x.B[0][t * kPieceRow + j + e];
          multiply(oS[i], split<3>(f), key);
        }
        if (upper) {
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) f[e] = x.B[0][(j + e) * kPieceRow + t];
          multiply(dk_all[i], split<3>(f), query);
        }
#pragma unroll
        for (uint32_t e = 0; e < 8; ++e) f[e] = -((lower ? x.B[1][t * kPieceRow + j + e] : 0.0f) + (upper ? x.B[1][(j + e) * kPieceRow + t] : 0.0f));
        multiply(dk_all[i], split<3>(f), key);
      }
    }
    at_end = wave_sum(at_end);
    if (lane == 0) x.at_end[wave] = at_end;
    Tile of_g[kSteps];
#pragma unroll
    for (uint32_t i = 0; i < kSteps; ++i) {
      dq_all[i] += oS[i];
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) of_g[i][e] = row_sum(own_d < a.Dk ? (float)query_at[i][e] * oS[i][e] : 0.0f);
    }
    if (m == 0) {
#pragma unroll
      for (uint32_t i = 0; i < kSteps; ++i) *reinterpret_cast<Tile *>(&x.of_g[own][state_row(r0 + i, 0)]) = of_g[i];
    }
    __syncthreads();
    if (wave == 0) {
      const uint32_t t = lane, episode = x.gates.episode[t];
      double sum = 0.0, to_end = 0.0;
      float beta = 0.0f;
      if (t < have)
        for (uint32_t n = 0; n < 2 * KS; ++n) sum += x.of_g[n][t];
      for (uint32_t n = 0; n < kWaves; ++n) {
        if (t < have) sum -= x.of_v[n][t];
        beta += x.of_beta[n][t];
        to_end += x.at_end[n];
      }
      // from t to the end of its episode
      for (uint32_t d = 1; d < kPiece; d *= 2) {
        const double next = __shfl_down(sum, d);
        const uint32_t its = __shfl_down(episode, d);
        if (t + d < kPiece && its == episode) sum += next;
      }
      if (episode == x.gates.episode[kPiece - 1]) sum += to_end;
      if (t < steps) {
        const uint64_t at = gates_at + (uint64_t)t * a.H + h;
        b.dg[at] = t < have && !x.gates.cut[t] ? (float)sum : 0.0f;
        b.dbeta[at] = t < have ? beta : 0.0f;
      }
    }
  }
  const uint32_t own_d = tile_row(own, lane % 16);
  if (own_d >= a.Dk) return;
#pragma unroll
  for (uint32_t i = 0; i < kSteps; ++i)
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
      const uint32_t t = state_row(r0 + i, e);
      if (t >= steps) continue;
      dq[t * b.dq_time + own_d] = t < have ? (T)dq_all[i][e] : (T)0.0f;
      dk[t * b.dk_time + own_d] = t < have ? (T)dk_all[i][e] : (T)0.0f;
    }
}

// ---- few steps: one after the other, the state in registers.  A workgroup has 64 columns of a state, a thread 8 rows of 4 of
// them; what crosses between rows are three sums a step: k . S, q . S and q . k, so that a step has one barrier.
// One step is bound by memory, the states read and written once: 64 sequences of 16 heads of 128 x 128 30 us, 4.5 TB/s
// (25.4 on the states of the pass before, which are in the caches in part).
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
    if (f.carry && t % kPiece == 0 && c0 < (a.Dv + 15) / 16 * 16) {
      float *const to = f.carry + (((uint64_t)s * a.pieces + t / kPiece) * a.H + h) * slices_size(a.Dk, a.Dv) + (c0 / 16) * slice_size(a.Dk) + c0 % 16;
#pragma unroll
      for (uint32_t i = 0; i < kStepRows; ++i) {
        Run<float, C> v;
#pragma unroll
        for (uint32_t c = 0; c < C; ++c) v[c] = passes && c0 + c < a.Dv ? S[i][c] : 0.0f;
        if (d0 + i < (a.Dk + 31) / 32 * 32) *reinterpret_cast<Run<float, C> *>(to + slice_row(d0 + i) * 16) = v;  // (0 beyond Dk)
      }
    }
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

// Sequences of at most so many steps are computed step by step, of the second number where workgroups are more than compute units.
// (A step takes 1.5 us, the pieces' two launches 17 where there are few workgroups: 8 heads of 128 x 128 8 steps 16 us, 12 steps 22,
// by pieces 17; 64 sequences of 16 of them 16 steps 103 us, by pieces 150, of 8 heads of 64 x 64 35 and 36.)
constexpr uint32_t kDeltaFew = 8, kDeltaSteps = 16;

bool delta_by_steps(uint32_t S, uint32_t T, uint32_t H, uint32_t Dv)
{
  return T <= kDeltaFew || (T <= kDeltaSteps && (uint64_t)S * H * blocks_for(Dv, kStepColumns) > kChipCus);
}

// f(integral_constant<uint32_t>): the width of keys and queries, in 32.
template <typename F>
void with_width(uint32_t Dk, F f)
{
  if (Dk > 64)
    f(std::integral_constant<uint32_t, 4>());
  else
    f(std::integral_constant<uint32_t, 2>());
}

struct DeltaBytes {
  uint64_t gates, M, P, K, Q, Kt, Qt, V, rows, dS, Y, bytes;
};

int delta_sizes(uint32_t S, uint32_t T, uint32_t H, uint32_t Dk, uint32_t Dv, bool backward, DeltaBytes *n)
{
  if (!S || !T || !H || !Dk || !Dv || T > 0x7fffffffu) return APEX_ERR_INVALID_ARG;
  if (Dk > kDeltaMaxWidth || Dv > kDeltaMaxWidth) return APEX_ERR_TOO_LARGE;
  // (no launch has 2^32 threads: eight slices of a head, two waves each)
  uint64_t heads;
  if (__builtin_mul_overflow((uint64_t)S * blocks_for(T, kPiece), (uint64_t)H, &heads) || heads > APEX_DELTA_MAX_PIECES) return APEX_ERR_TOO_LARGE;
  *n = DeltaBytes{};
  if (!backward && T <= kDeltaFew) return APEX_OK;  // (sizes grow with the sequences, whether or not a call takes the steps)
  const auto take = [&](uint64_t bytes) {
    const uint64_t at = n->bytes;
    n->bytes += round_up(bytes, 256);
    return at;
  };
  const uint64_t columns = heads * (Dk > 64 ? 8 : 4) * 2 * kOperand * 4;  // (for the widest type, and every head with a key of its own)
  n->gates = take(heads * kGateWords * 4);
  n->M = take(heads * kTriangle * 3 * kOperand * 2);
  n->P = take(heads * kTriangle * 3 * kOperand * 2);
  n->K = take(columns);
  n->Q = take(columns);  // (the gradient takes no rows of queries, and has their transposes there)
  n->Qt = n->Q;
  n->Kt = take(columns);
  n->V = take(heads * blocks_for(Dv, 16) * kWave * 16 * 4);
  if (backward) {
    n->rows = take(heads * kTriangle * 3 * kOperand * 2);
    n->dS = take(heads * round_up(Dk, 32) * round_up(Dv, 16) * 4);
    n->Y = take(heads * blocks_for(Dv, 16) * kWave * 16 * 4);
  }
  return APEX_OK;
}

Prepared delta_prepared(const DeltaBytes &n, void *workspace)
{
  char *const p = static_cast<char *>(workspace);
  return Prepared{reinterpret_cast<uint32_t *>(p + n.gates), reinterpret_cast<__bf16 *>(p + n.M), reinterpret_cast<__bf16 *>(p + n.P), p + n.K, p + n.Q, p + n.Kt, p + n.Qt, p + n.V,
                  reinterpret_cast<__bf16 *>(p + n.rows)};
}

// Workgroups of the kernels that go from piece to piece, of `slices` slices of 16 columns each: eight heads' at a time.
uint32_t delta_groups(uint32_t S, uint32_t H, uint32_t Dv, uint32_t slices) { return blocks_for((uint64_t)S * H, 8) * 8 * blocks_for(Dv, 16 * slices); }

// f(integral_constant<uint32_t>): slices of a workgroup.
// Two, which read the same operands at the same time, where a compute unit has two anyway and operands are large (4 x 8192 steps of
// 16 heads of 128 x 128 684 us by one, 621 by two); else one (1 x 16384 of 8 heads, keys of f16 not in parts, 1131 and 1289, 64 x 96 of 8 heads of 64 x 64 33.7
// and 36).
template <uint32_t KS, typename F>
void with_slices(uint32_t S, uint32_t H, uint32_t Dv, F f)
{
  if (KS == 4 && Dv > 16 && (uint64_t)S * H * blocks_for(Dv, 16) > kChipCus)
    f(std::integral_constant<uint32_t, KS / 2>());
  else
    f(std::integral_constant<uint32_t, 1>());
}

// f(integral_constant<uint32_t>): waves of a workgroup of the gradient's last kernel.
// Four for narrow states, a wave per 16 columns and per 16 rows, so that a compute unit has two workgroups, one of which works while the
// other waits: the gradient of 64 x 96 steps of 8 heads of 64 x 64 in bf16 144 -> 121 us, in f32 186 -> 165, of 4 x 4096 399 -> 339;
// where there is a workgroup a compute unit or less, 1 x 4096 of 4 heads, 184 as before.
template <uint32_t KS, typename F>
void with_waves(uint32_t Dv, F f)
{
  if (KS == 2 && Dv <= 16 * kGradNarrowWaves)
    f(std::integral_constant<uint32_t, KS == 2 ? kGradNarrowWaves : kGradWaves>());
  else
    f(std::integral_constant<uint32_t, kGradWaves>());
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
                  v_seq_stride, v_time_stride, q, k, v, g, beta, scale, discount, length},
                 h0, o, h_last, carry};
  if (const int rc = delta_check(f.n, dtype)) return rc;
  if (!o || (uintptr_t)o % element_size(dtype) || ((uintptr_t)h0 | (uintptr_t)h_last | (uintptr_t)carry) % 4 ||
      (n.bytes && (!workspace || (uintptr_t)workspace % 256)))
    return APEX_ERR_INVALID_ARG;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (delta_by_steps(S, T, H, Dv)) {
    with_type(dtype, [&](auto t) {
      delta_steps_kernel<decltype(t)><<<dim3(S * H * blocks_for(Dv, kStepColumns)), dim3(kDeltaThreads), 0, stream>>>(f);
    });
    APEX_HIP(hipGetLastError());
    return APEX_OK;
  }
  const Prepared w = delta_prepared(n, workspace);
  with_type(dtype, [&](auto t) {
    typedef decltype(t) E;
    with_width(Dk, [&](auto width) {
      constexpr uint32_t KS = decltype(width)::value;
      with_slices<KS>(S, H, Dv, [&](auto slices) {
        constexpr uint32_t kSlices = decltype(slices)::value;
        delta_prepare_kernel<E, KS, false, kInParts<E, KS, kSlices>><<<dim3(S * f.n.pieces * H), dim3(kDeltaThreads), 0, stream>>>(f.n, nullptr, w);
        delta_pieces_kernel<E, KS, kSlices><<<dim3(delta_groups(S, H, Dv, kSlices)), dim3(2 * kSlices * kWave), 0, stream>>>(f, w);
      });
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
  DeltaBack b{{S, T, Hk, H, Dk, Dv, blocks_for(T, kPiece), Hk ? H / Hk : 0, q_seq_stride, q_time_stride, k_seq_stride, k_time_stride,
               v_seq_stride, v_time_stride, q, k, v, g, beta, scale, discount, length},
              carry, d_o, dh_last, dq_seq_stride, dq_time_stride, dk_seq_stride, dk_time_stride, dv_seq_stride, dv_time_stride, dq, dk, dv, dg,
              dbeta, dh0, nullptr, nullptr};
  if (const int rc = delta_check(b.n, dtype)) return rc;
  const uint32_t size = element_size(dtype);
  if (!carry || !d_o || !dg || !dbeta || !workspace || (uintptr_t)workspace % 256 || (uintptr_t)d_o % size ||
      ((uintptr_t)carry | (uintptr_t)dh_last | (uintptr_t)dg | (uintptr_t)dbeta | (uintptr_t)dh0) % 4 || !dq || !dk || !dv ||
      !rows_apart(dq, size, S, dq_seq_stride, T, dq_time_stride, (uint64_t)Hk * Dk) ||
      !rows_apart(dk, size, S, dk_seq_stride, T, dk_time_stride, (uint64_t)Hk * Dk) ||
      !rows_apart(dv, size, S, dv_seq_stride, T, dv_time_stride, (uint64_t)H * Dv))
    return APEX_ERR_INVALID_ARG;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const Prepared w = delta_prepared(n, workspace);
  b.dS = reinterpret_cast<float *>(static_cast<char *>(workspace) + n.dS), b.Y = reinterpret_cast<float *>(static_cast<char *>(workspace) + n.Y);
  with_type(dtype, [&](auto t) {
    typedef decltype(t) E;
    with_width(Dk, [&](auto width) {
      constexpr uint32_t KS = decltype(width)::value;
      delta_prepare_kernel<E, KS, true, false><<<dim3(S * b.n.pieces * H), dim3(kDeltaThreads), 0, stream>>>(b.n, b.d_o, w);
      with_slices<KS>(S, H, Dv, [&](auto slices) {
        constexpr uint32_t kSlices = decltype(slices)::value;
        delta_pieces_back_kernel<E, KS, kSlices><<<dim3(delta_groups(S, H, Dv, kSlices)), dim3(2 * kSlices * kWave), 0, stream>>>(b, w);
      });
      with_waves<KS>(Dv, [&](auto waves) {
        constexpr uint32_t kWaves = decltype(waves)::value;
        if (Dv % 32)
          delta_gradients_kernel<E, KS, kWaves, false><<<dim3(S * b.n.pieces * Hk), dim3(kWaves * kWave), 0, stream>>>(b, w);
        else
          delta_gradients_kernel<E, KS, kWaves, true><<<dim3(S * b.n.pieces * Hk), dim3(kWaves * kWave), 0, stream>>>(b, w);
      });
    });
  });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

}  // extern "C"
