// Verification of drafted tokens.  Included by apex_replay.hip (one translation unit).
//
// Probabilities are compared, subtracted and summed as integers of 2^-40, so that sums do not depend on their order and
// the draw is the same however a row is shared out: what the sum tree does with priorities.
#include "elements.hpp"

namespace apex {

constexpr uint32_t kVerifyThreads = 512, kVerifyShares = 64;  // threads per workgroup, workgroups per sequence at most
constexpr uint32_t kVerifyItems = 8;                          // neighbouring tokens of a thread when a share is searched

// Per sequence: a word that counts its workgroups (0 before and after every call) and, in a line of their own, their sums.
struct VerifyShare {
  uint64_t left, target;  // sums of max(0, m(p) - m(q)) and of m(p)
};
struct VerifySpace {
  uint32_t done;
  uint32_t pad[31];
  VerifyShare share[kVerifyShares];
};

struct VerifyArgs {
  uint32_t B, G, V, shares, share_tokens;  // a share: a multiple of the tokens that a workgroup takes at once
  uint64_t target_seq, target_row, draft_seq, draft_row;
  const void *target, *draft;
  const int32_t *token;
  const uint64_t *rnd;
  const int32_t *length;
  int32_t *accepted, *token_out;
  VerifySpace *space;
};

constexpr int kMassBits = 40;

// floor(min(x, 1) 2^40), 0 for what is not above 0.  In two conversions of 32 bits: the multiple of 2^-20 below x, and the
// rest, which is exact, in 2^-40.
__device__ __forceinline__ uint64_t probability_mass(float x)
{
  x = x > 0.0f ? fminf(x, 1.0f) : 0.0f;
  const float scaled = x * 0x1p+20f, whole = __builtin_floorf(scaled);
  return ((uint64_t)(uint32_t)whole << 20) + (uint32_t)((scaled - whole) * 0x1p+20f);
}

__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v)
{
  const uint64_t s = wave_inclusive_scan(v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)s, kWave - 1);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(s >> 32), kWave - 1);
  return ((uint64_t)hi << 32) | lo;
}

// The row that a sequence's next token is drawn from.
struct VerifyRows {
  uint32_t n;     // drafted tokens that stand
  bool turned;    // the one behind them was turned down
};

// By one wave: a lane per drafted token.
template <typename T>
__device__ __forceinline__ VerifyRows tokens_that_stand(const VerifyArgs &a, uint32_t b)
{
  const uint32_t i = lane_id();
  const uint32_t len = a.length ? (uint32_t)min(max(a.length[b], 0), (int32_t)a.G) : a.G;
  bool stands = false;
  if (i < len) {
    const int32_t token = a.token[(uint64_t)b * a.G + i];
    const uint64_t u = a.rnd[(uint64_t)b * (a.G + 1) + i];
    if (token >= 0 && (uint32_t)token < a.V) {
      const uint64_t p = probability_mass((float)static_cast<const T *>(a.target)[b * a.target_seq + i * a.target_row + token]);
      const uint64_t q = probability_mass((float)static_cast<const T *>(a.draft)[b * a.draft_seq + i * a.draft_row + token]);
      stands = __umul64hi(u, q) < p;
    }
  }
  const uint64_t down = ~__ballot(stands);  // a lane beyond the draft does not stand
  const uint32_t n = len == kWave && down == 0 ? kWave : (uint32_t)__builtin_ctzll(down);
  return VerifyRows{n, n < len};
}

// Masses of tokens [at, at + N) of the two rows; none beyond V.
template <typename T, int N>
__device__ __forceinline__ void masses_of(const T *p_row, const T *q_row, bool turned, uint32_t at, uint32_t V, uint64_t (&left)[N],
                                          uint64_t (&target)[N])
{
  float p[N], q[N];
  if (at + N <= V) {
    const Run<T, N> pr = load_run<T, N>(p_row + at);
    Run<T, N> qr{};
    if (turned) qr = load_run<T, N>(q_row + at);
#pragma unroll
    for (int e = 0; e < N; ++e) p[e] = element<N, T>(pr, e), q[e] = element<N, T>(qr, e);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      p[e] = at + e < V ? (float)p_row[at + e] : 0.0f;
      q[e] = turned && at + e < V ? (float)q_row[at + e] : 0.0f;
    }
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    target[e] = probability_mass(p[e]);
    const uint64_t m = probability_mass(q[e]);
    left[e] = target[e] > m ? target[e] - m : 0;
  }
}

// Every sequence's row is shared by `shares` workgroups, which sum their parts; the last of them to be done knows the
// total, finds the part that the drawn point lies in and goes through it once more.
template <typename T>
__global__ __launch_bounds__(kVerifyThreads) void verify_kernel(VerifyArgs a)
{
  constexpr int N = 16 / sizeof(T);
  constexpr uint32_t kWaves = kVerifyThreads / kWave;
  __shared__ uint64_t red[2][kWaves];
  __shared__ VerifyRows sh_rows;
  __shared__ uint32_t sh_done;
  const uint32_t thread = threadIdx.x, lane = lane_id(), wave = thread / kWave;
  const uint32_t b = blockIdx.x / a.shares, share = blockIdx.x % a.shares;
  if (wave == 0) {
    const VerifyRows r = tokens_that_stand<T>(a, b);
    if (lane == 0) sh_rows = r;
  }
  __syncthreads();
  const VerifyRows rows = sh_rows;
  const T *const p_row = static_cast<const T *>(a.target) + b * a.target_seq + rows.n * a.target_row;
  const T *const q_row = rows.turned ? static_cast<const T *>(a.draft) + b * a.draft_seq + rows.n * a.draft_row : nullptr;

  const uint32_t begin = share * a.share_tokens, end = min(a.V, begin + a.share_tokens);
  uint64_t left_sum = 0, target_sum = 0;
  for (uint32_t at = begin + thread * N; at < end; at += kVerifyThreads * N) {
    uint64_t left[N], target[N];
    masses_of<T, N>(p_row, q_row, rows.turned, at, a.V, left, target);
#pragma unroll
    for (int e = 0; e < N; ++e) left_sum += left[e], target_sum += target[e];
  }
  left_sum = wave_sum_u64(left_sum);
  target_sum = wave_sum_u64(target_sum);
  if (lane == 0) red[0][wave] = left_sum, red[1][wave] = target_sum;
  __syncthreads();
  VerifySpace *const space = a.space + b;
  if (wave == 0) {
    left_sum = wave_sum_u64(lane < kWaves ? red[0][lane] : 0);
    target_sum = wave_sum_u64(lane < kWaves ? red[1][lane] : 0);
    if (lane == 0) {
      // only these words cross between workgroups: written through to memory, and waited for before the word is counted
      __hip_atomic_store(&space->share[share].left, left_sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(&space->share[share].target, target_sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      sh_done = __hip_atomic_fetch_add(&space->done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  __syncthreads();
  if (sh_done != a.shares - 1) return;
  if (thread == 0) __hip_atomic_store(&space->done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

  // which share (every wave finds it for itself)
  static_assert(kVerifyShares == kWave);
  uint64_t of_left = 0, of_target = 0;
  if (lane < a.shares) {
    of_left = __hip_atomic_load(&space->share[lane].left, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    of_target = __hip_atomic_load(&space->share[lane].target, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  const uint64_t left_up_to = wave_inclusive_scan(of_left), target_up_to = wave_inclusive_scan(of_target);
  const uint64_t left_total = __shfl(left_up_to, kWave - 1), target_total = __shfl(target_up_to, kWave - 1);
  const bool use_left = left_total != 0;
  const uint64_t total = use_left ? left_total : target_total, up_to = use_left ? left_up_to : target_up_to;
  const uint64_t of_share = use_left ? of_left : of_target;
  const uint64_t point = __umul64hi(a.rnd[(uint64_t)b * (a.G + 1) + a.G], total);
  const uint64_t over = __ballot(up_to > point);
  int32_t drawn = -1;
  if (over) {  // total is above 0, and point below it
    const int found = __builtin_ctzll(over);
    uint64_t base = __shfl(up_to - of_share, found);  // mass in front of the tokens looked at
    const uint32_t from = (uint32_t)found * a.share_tokens;
    for (uint32_t at0 = from;; at0 += kVerifyThreads * kVerifyItems) {
      const uint32_t at = at0 + thread * kVerifyItems;
      uint64_t left[kVerifyItems], target[kVerifyItems], mine = 0;
      masses_of<T, kVerifyItems>(p_row, q_row, rows.turned, at, a.V, left, target);
#pragma unroll
      for (uint32_t e = 0; e < kVerifyItems; ++e) {
        if (!use_left) left[e] = target[e];
        mine += left[e];
      }
      const uint64_t in_wave = wave_inclusive_scan(mine);
      __syncthreads();  // the words of the round before have been read
      if (lane == kWave - 1) red[0][wave] = in_wave;
      __syncthreads();
      uint64_t before = base, all = 0;
#pragma unroll
      for (uint32_t w = 0; w < kWaves; ++w) {
        if (w < wave) before += red[0][w];
        all += red[0][w];
      }
      before += in_wave - mine;
      if (point >= before && point < before + mine) {  // one thread of the workgroup, in one of the rounds
        uint32_t e = 0;
        for (uint64_t x = point - before; e < kVerifyItems - 1 && x >= left[e]; ++e) x -= left[e];
        a.token_out[(uint64_t)b * (a.G + 1) + rows.n] = (int32_t)(at + e);
      }
      base += all;
      if (base > point || at0 + kVerifyThreads * kVerifyItems >= a.V) break;
    }
    drawn = 0;
  }
  if (thread <= a.G && thread != rows.n)
    a.token_out[(uint64_t)b * (a.G + 1) + thread] = thread < rows.n ? a.token[(uint64_t)b * a.G + thread] : -1;
  if (thread == 0) {
    a.accepted[b] = (int32_t)rows.n;
    if (drawn < 0) a.token_out[(uint64_t)b * (a.G + 1) + rows.n] = -1;
  }
}

}  // namespace apex

namespace {

// Workgroups per sequence and tokens of each.
void verify_shares(uint32_t B, uint32_t V, uint32_t *shares, uint32_t *tokens)
{
  constexpr uint32_t kRound = kVerifyThreads * kVerifyItems;
  const uint32_t rounds = (V + kRound - 1) / kRound;
  const uint32_t most = std::clamp<uint32_t>(4 * kChipCus / B, 1, std::min(kVerifyShares, rounds));
  *tokens = (rounds + most - 1) / most * kRound;
  *shares = (V + *tokens - 1) / *tokens;
}

}  // namespace

extern "C" {

int apex_verify_draft_workspace_bytes(uint32_t B, uint32_t V, size_t *bytes)
{
  if (!B || !V || !bytes) return APEX_ERR_INVALID_ARG;
  if (V > APEX_MAX_VOCABULARY) return APEX_ERR_TOO_LARGE;
  *bytes = (size_t)B * sizeof(VerifySpace);
  return APEX_OK;
}

int apex_verify_draft(uint32_t B, uint32_t G, uint32_t V, int dtype, const void *target, uint64_t target_seq_stride,
                      uint64_t target_row_stride, const void *draft, uint64_t draft_seq_stride, uint64_t draft_row_stride,
                      const int32_t *token, const uint64_t *rnd, const int32_t *length, int32_t *accepted,
                      int32_t *token_out, void *workspace, void *hip_stream)
{
  const uint32_t size = element_size(dtype);
  if (!B || !V || !size || !target || !rnd || !accepted || !token_out || !workspace || (G && (!draft || !token)))
    return APEX_ERR_INVALID_ARG;
  if (V > APEX_MAX_VOCABULARY || G > APEX_MAX_DRAFT || B > 0xffffffffu / (kVerifyShares * kVerifyThreads)) return APEX_ERR_TOO_LARGE;
  if (!rows_fit(target, size, B, target_seq_stride, G + 1, target_row_stride, V) ||
      (G && !rows_fit(draft, size, B, draft_seq_stride, G, draft_row_stride, V)))
    return APEX_ERR_INVALID_ARG;
  if (((uintptr_t)token | (uintptr_t)length | (uintptr_t)accepted | (uintptr_t)token_out) % 4 || (uintptr_t)rnd % 8 ||
      (uintptr_t)workspace % 256)
    return APEX_ERR_INVALID_ARG;
  VerifyArgs a{B, G, V, 1, V, target_seq_stride, target_row_stride, draft_seq_stride, draft_row_stride, target, draft, token, rnd,
               length, accepted, token_out, static_cast<VerifySpace *>(workspace)};
  verify_shares(B, V, &a.shares, &a.share_tokens);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  with_type(dtype, [&](auto t) { verify_kernel<decltype(t)><<<dim3(B * a.shares), dim3(kVerifyThreads), 0, stream>>>(a); });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

}  // extern "C"
