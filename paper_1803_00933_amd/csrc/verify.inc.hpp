// Verification of drafted tokens.  Included by apex_replay.hip (one translation unit).
//
// Probabilities are compared, subtracted and summed as integers of 2^-40, so that sums do not depend on their order and
// the draw is the same however a row is shared out: what the sum tree does with priorities.
#include "elements.hpp"

namespace apex {

constexpr uint32_t kVerifyThreads = 512, kVerifyShares = 64;  // threads per workgroup, workgroups per sequence at most
constexpr uint32_t kVerifyItems = 8;                          // neighbouring tokens of a thread when a share is searched
constexpr uint32_t kVerifyMaxShare = 1u << 19;                // tokens of a share at most: a thread's sums stay within 31 bits

// Per sequence: a word that counts its workgroups (0 before and after every call) and, in lines of their own, their sums.
struct VerifySpace {
  uint32_t done;
  uint32_t pad[31];
  uint64_t share[kVerifyShares];
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

// m(x) = floor(min(x, 1) 2^40), 0 for what is not above 0, as high 2^20 + low: the multiple of 2^-20 below x, and the rest,
// which is exact, in 2^-40.
struct Mass {
  float scaled;
  uint32_t high, low;
  __device__ __forceinline__ explicit Mass(float x)
  {
    scaled = __builtin_amdgcn_fmed3f(x, 0.0f, 1.0f) * 0x1p+20f;  // (NaN: 0)
    high = (uint32_t)scaled;
    low = (uint32_t)(__builtin_amdgcn_fractf(scaled) * 0x1p+20f);
  }
  __device__ __forceinline__ uint64_t whole() const { return ((uint64_t)high << 20) + low; }
};

// max(0, m(p) - m(q)): what is scaled decides, which is a number where p or q is none.
__device__ __forceinline__ uint64_t mass_left(float p, float q)
{
  const Mass mp(p), mq(q);
  return mp.scaled > mq.scaled ? mp.whole() - mq.whole() : 0;
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
      const uint64_t p = Mass((float)static_cast<const T *>(a.target)[b * a.target_seq + i * a.target_row + token]).whole();
      const uint64_t q = Mass((float)static_cast<const T *>(a.draft)[b * a.draft_seq + i * a.draft_row + token]).whole();
      stands = __umul64hi(u, q) < p;
    }
  }
  const uint64_t down = ~__ballot(stands);  // a lane beyond the draft does not stand
  const uint32_t n = len == kWave && down == 0 ? kWave : (uint32_t)__builtin_ctzll(down);
  return VerifyRows{n, n < len};
}

// What a thread has summed up: differences of masses, the two parts apart.  Up to 2^10 tokens of 2^20.
struct MassSum {
  int32_t high = 0, low = 0;
  __device__ __forceinline__ void add(float p, float q)
  {
    const Mass mp(p), mq(q);
    const bool more = mp.scaled > mq.scaled;
    high += more ? (int32_t)(mp.high - mq.high) : 0;
    low += more ? (int32_t)(mp.low - mq.low) : 0;
  }
  __device__ __forceinline__ uint64_t whole() const { return (uint64_t)(((int64_t)high << 20) + low); }
};

// The probabilities of tokens [at, at + N), 0 beyond V.
template <typename T, int N>
__device__ __forceinline__ void probabilities(const T *row, uint32_t at, uint32_t V, float (&x)[N])
{
  if (at + N <= V) {
    const Run<T, N> r = load_run<T, N>(row + at);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = element<N, T>(r, e);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = at + e < V ? (float)row[at + e] : 0.0f;
  }
}

// This thread's part of the mass that is left of tokens [begin, end), in rounds of the whole workgroup; kTwo: with a row q.
template <typename T, bool kTwo>
__device__ __forceinline__ uint64_t sum_of(const T *p_row, const T *q_row, uint32_t begin, uint32_t end, uint32_t V)
{
  constexpr uint32_t N = 16 / sizeof(T), kRound = kVerifyThreads * N, kAhead = 4;
  static_assert(kVerifyMaxShare / kVerifyThreads <= 1u << 10);
  MassSum sum;
  uint32_t at = begin + threadIdx.x * N;
  for (; at + (kAhead - 1) * kRound + N <= min(end, V); at += kAhead * kRound) {
    Run<T, N> p[kAhead], q[kAhead];
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) {
      p[i] = load_run<T, N>(p_row + at + i * kRound);
      if (kTwo) q[i] = load_run<T, N>(q_row + at + i * kRound);
    }
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i)
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) sum.add(element<N, T>(p[i], e), kTwo ? element<N, T>(q[i], e) : 0.0f);
  }
  for (; at < end; at += kRound) {
    float p[N], q[N] = {};
    probabilities<T, N>(p_row, at, V, p);
    if (kTwo) probabilities<T, N>(q_row, at, V, q);
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) sum.add(p[e], q[e]);
  }
  return sum.whole();
}

// Every sequence's row is shared by `shares` workgroups, which sum their parts; the last of them to be done knows the
// total, finds the part that the drawn point lies in and goes through it once more.
// Bound by memory for many sequences (256 x 128001 in 32 bits 52-53 us for 228 MB, 4.3 TB/s; 67 in 16 bits, for
// half as much), for few by a chain of round trips: token, its two probabilities, the row, the sums, the part of the row again (one
// sequence of 131072: 5.4-6.4 us).
// One sum a row: with the target's own beside what is left of it, for the row of which nothing is left, the first took 61 us;
// that row is summed up again when it comes.  Masses in two parts of 32 bits: with 64-bit masses and sums 76.
template <typename T>
__global__ __launch_bounds__(kVerifyThreads) void verify_kernel(VerifyArgs a)
{
  constexpr uint32_t kWaves = kVerifyThreads / kWave;
  __shared__ uint64_t red[kWaves];
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
  bool two = rows.turned;
  const T *const p_row = static_cast<const T *>(a.target) + b * a.target_seq + rows.n * a.target_row;
  const T *const q_row = two ? static_cast<const T *>(a.draft) + b * a.draft_seq + rows.n * a.draft_row : nullptr;
  // the sum over the workgroup, in every thread of wave 0
  const auto of_workgroup = [&](uint64_t mine) {
    mine = wave_sum_u64(mine);
    if (lane == 0) red[wave] = mine;
    __syncthreads();
    return wave == 0 ? wave_sum_u64(lane < kWaves ? red[lane] : 0) : 0;
  };

  const uint32_t begin = share * a.share_tokens, end = min(a.V, begin + a.share_tokens);
  const uint64_t sum = of_workgroup(two ? sum_of<T, true>(p_row, q_row, begin, end, a.V) : sum_of<T, false>(p_row, q_row, begin, end, a.V));
  VerifySpace *const space = a.space + b;
  if (thread == 0) {
    // only these words cross between workgroups: written through to memory, and waited for before the workgroup is counted
    __hip_atomic_store(&space->share[share], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    sh_done = __hip_atomic_fetch_add(&space->done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (sh_done != a.shares - 1) return;
  if (thread == 0) __hip_atomic_store(&space->done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);

  // which share (every wave finds it for itself)
  static_assert(kVerifyShares == kWave);
  const uint64_t of_share = lane < a.shares ? __hip_atomic_load(&space->share[lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
  const uint64_t u = a.rnd[(uint64_t)b * (a.G + 1) + a.G];
  const uint64_t up_to = wave_inclusive_scan(of_share);
  uint64_t total = __shfl(up_to, kWave - 1), point = __umul64hi(u, total), base = 0;  // base: mass in front of the tokens looked at
  uint32_t from = 0;
  if (total) {  // point is below it
    const int found = __builtin_ctzll(__ballot(up_to > point));
    base = __shfl(up_to - of_share, found);
    from = (uint32_t)found * a.share_tokens;
  } else if (two) {  // nothing is left of a row that was turned down: the target's own, all of it by this workgroup
    two = false;
    uint64_t all = 0;
    for (uint32_t at = 0; at < a.V; at += a.share_tokens) all += sum_of<T, false>(p_row, nullptr, at, min(a.V, at + a.share_tokens), a.V);
    all = of_workgroup(all);
    if (thread == 0) red[0] = all;
    __syncthreads();
    total = red[0];
    point = __umul64hi(u, total);
  }
  if (total) {
    for (uint32_t at0 = from;; at0 += kVerifyThreads * kVerifyItems) {
      const uint32_t at = at0 + thread * kVerifyItems;
      float p[kVerifyItems], q[kVerifyItems] = {};
      probabilities<T, kVerifyItems>(p_row, at, a.V, p);
      if (two) probabilities<T, kVerifyItems>(q_row, at, a.V, q);
      uint64_t left[kVerifyItems], mine = 0;
#pragma unroll
      for (uint32_t e = 0; e < kVerifyItems; ++e) mine += left[e] = mass_left(p[e], q[e]);
      const uint64_t in_wave = wave_inclusive_scan(mine);
      __syncthreads();  // the words of the round before have been read
      if (lane == kWave - 1) red[wave] = in_wave;
      __syncthreads();
      uint64_t before = base, all = 0;
#pragma unroll
      for (uint32_t w = 0; w < kWaves; ++w) {
        if (w < wave) before += red[w];
        all += red[w];
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
  }
  if (thread <= a.G && thread != rows.n)
    a.token_out[(uint64_t)b * (a.G + 1) + thread] = thread < rows.n ? a.token[(uint64_t)b * a.G + thread] : -1;
  if (thread == 0) {
    a.accepted[b] = (int32_t)rows.n;
    if (!total) a.token_out[(uint64_t)b * (a.G + 1) + rows.n] = -1;
  }
}

}  // namespace apex

namespace {

// Workgroups per sequence and tokens of each: as many as keep the chip in sixteen times its compute units, no smaller than a
// round of the search.  (256 x 128001 in 32 bits 68.8 us with 2 workgroups a sequence, 59.6 with 4, 53.5 with 8, 52.8 with 16.)
void verify_shares(uint32_t B, uint32_t V, uint32_t *shares, uint32_t *tokens)
{
  constexpr uint32_t kRound = kVerifyThreads * kVerifyItems;
  const uint32_t rounds = blocks_for(V, kRound);
  const uint32_t most = std::clamp<uint32_t>(16 * kChipCus / B, blocks_for(V, kVerifyMaxShare), std::min(kVerifyShares, rounds));
  *tokens = blocks_for(rounds, most) * kRound;
  *shares = blocks_for(V, *tokens);
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
