// The norm over many tensors, and the tensors scaled by what keeps it below a limit.  Included by apex_replay.hip (one
// translation unit).
#include <memory>

#include "elements.hpp"

namespace apex {

constexpr uint32_t kClipThreads = 256, kClipTensors = 96;      // tensors of a launch: their table is an argument of the kernel
constexpr uint32_t kClipMinPiece = 8192;                       // elements that a workgroup takes, where there are few
constexpr uint32_t kClipPieces = 4096;                         // pieces at most, beside one more per tensor

struct ClipTensor {
  const void *grad;
  void *out;
  uint64_t elements;
  uint32_t first;  // its first piece within the launch
  uint32_t dtype;
};

// Counts the workgroups that have stored their sums (0 before and after every call); factor and sums in lines of their own.
// The factor is a product, factor times power, so that it has all its bits below the normal range, too.
struct ClipSpace {
  uint32_t done;
  uint32_t pad[31];
  float factor, power;
  uint32_t pad2[30];
  double sum[];
};

struct ClipArgs {
  uint32_t tensors, pieces;          // of this launch
  uint32_t before, all;              // pieces of the launches in front of it, and of all of them
  uint32_t piece;                    // elements
  float max_norm;
  bool in_place, past_caches;
  float *norm;
  ClipSpace *space;
  ClipTensor tensor[kClipTensors];
};

// The tensor that a piece is of: the last whose first piece is not behind it.
__device__ __forceinline__ uint32_t clip_tensor(const ClipArgs &a, uint32_t piece)
{
  uint32_t low = 0, high = a.tensors;
  while (high - low > 1) {
    const uint32_t mid = (low + high) / 2;
    if (a.tensor[mid].first <= piece)
      low = mid;
    else
      high = mid;
  }
  return low;
}

// f(value of the element type)
template <typename F>
__device__ __forceinline__ void with_element(uint32_t dtype, F f)
{
  if (dtype == APEX_F32)
    f(float());
  else if (dtype == APEX_BF16)
    f(__bf16());
  else
    f(_Float16());
}

// This thread's squares of [begin, end): in 64 bits, where no square of a 32-bit number overflows.
template <typename T>
__device__ __forceinline__ double squares(const T *x, uint64_t begin, uint64_t end)
{
  constexpr uint32_t N = 16 / sizeof(T), kRound = kClipThreads * N, kAhead = 4;
  double sum[2] = {0.0, 0.0};
  uint64_t at = begin + threadIdx.x * N;
  for (; at + (kAhead - 1) * kRound + N <= end; at += kAhead * kRound) {
    Run<T, N> r[kAhead];
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) r[i] = load_run<T, N>(x + at + i * kRound);
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i)
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        const double v = element<N, T>(r[i], e);
        sum[e % 2] = __builtin_fma(v, v, sum[e % 2]);
      }
  }
  for (; at < end; at += kRound)
    for (uint32_t e = 0; e < N && at + e < end; ++e) {
      const double v = (float)x[at + e];
      sum[e % 2] = __builtin_fma(v, v, sum[e % 2]);
    }
  return sum[0] + sum[1];
}

// A workgroup per piece; the last of all of them to be done sums the pieces up, in their order.  Many elements are bound by memory, 729 M of
// bf16 270 us, 5.4 TB/s; fewer by the counter, at which workgroups arrive one after the other, 14 ns each: 80 M in 3259 pieces 55 us, 46 of
// it the counter's.  So there are not too many (8192 pieces 70 us and 267, 2048 45 and 300).
__global__ __launch_bounds__(kClipThreads) void clip_norm_kernel(ClipArgs a)
{
  constexpr uint32_t kWaves = kClipThreads / kWave;
  __shared__ double red[kWaves];
  __shared__ uint32_t sh_done;
  const uint32_t lane = lane_id(), wave = threadIdx.x / kWave;
  const auto of_workgroup = [&](double mine) {  // in thread 0
    mine = wave_sum(mine);
    if (lane == 0) red[wave] = mine;
    __syncthreads();
    double sum = 0.0;
    for (uint32_t w = 0; w < kWaves; ++w) sum += red[w];
    __syncthreads();
    return sum;
  };
  double mine = 0.0;
  if (a.pieces) {
    const ClipTensor &t = a.tensor[clip_tensor(a, blockIdx.x)];
    const uint64_t begin = (uint64_t)(blockIdx.x - t.first) * a.piece, end = min(t.elements, begin + a.piece);
    with_element(t.dtype, [&](auto e) { mine = squares(static_cast<const decltype(e) *>(t.grad), begin, end); });
  }
  const double sum = of_workgroup(mine);
  ClipSpace *const space = a.space;
  if (threadIdx.x == 0) {
    // only these words cross between workgroups: written through to memory, and waited for before the workgroup is counted
    if (a.pieces)
      __hip_atomic_store(reinterpret_cast<uint64_t *>(&space->sum[a.before + blockIdx.x]), __builtin_bit_cast(uint64_t, sum), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    sh_done = __hip_atomic_fetch_add(&space->done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
  }
  __syncthreads();
  if (sh_done != max(a.all, 1u)) return;
  double total = 0.0;
  for (uint32_t i = threadIdx.x; i < a.all; i += kClipThreads)
    total += __builtin_bit_cast(double, __hip_atomic_load(reinterpret_cast<uint64_t *>(&space->sum[i]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
  total = of_workgroup(total);
  if (threadIdx.x == 0) {
    __hip_atomic_store(&space->done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const double norm = __builtin_sqrt(total);
    // (a norm that is no number, or infinite, scales nothing)
    const bool clips = norm > (double)a.max_norm && norm < __builtin_huge_val();
    const double factor = clips ? (double)a.max_norm / norm : 1.0;
    const bool small = factor < 0x1p-100;
    space->factor = (float)(small ? factor * 0x1p100 : factor);
    space->power = small ? 0x1p-100f : 1.0f;
    if (a.norm) a.norm[0] = (float)norm;
  }
}

// The pieces from the last one of the last tensor on: what the sums have read last is still in the caches.  Bound by memory: 729 M elements
// of bf16 559 us, 5.2 TB/s read and written (571 where the tensors of a launch come from the first one on).
__global__ __launch_bounds__(kClipThreads) void clip_scale_kernel(ClipArgs a)
{
  const float factor = a.space->factor, power = a.space->power;
  if (a.in_place && factor == 1.0f && power == 1.0f) return;
  const uint32_t piece = a.pieces - 1 - blockIdx.x;
  const ClipTensor &t = a.tensor[clip_tensor(a, piece)];
  const uint64_t begin = (uint64_t)(piece - t.first) * a.piece, end = min(t.elements, begin + a.piece);
  with_element(t.dtype, [&](auto of) {
    typedef decltype(of) T;
    constexpr uint32_t N = 16 / sizeof(T), kRound = kClipThreads * N, kAhead = 4;
    const T *const x = static_cast<const T *>(t.grad);
    T *const out = static_cast<T *>(t.out);
    in_either_way(a.past_caches, [&](auto past) {
      const auto put = [&](uint64_t at, Run<T, N> r) {
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) r[e] = (T)(element<N, T>(r, e) * factor * power);
        if (decltype(past)::value)
          __builtin_nontemporal_store(r, reinterpret_cast<Run<T, N> *>(out + at));
        else
          *reinterpret_cast<Run<T, N> *>(out + at) = r;
      };
      uint64_t at = begin + threadIdx.x * N;
      for (; at + (kAhead - 1) * kRound + N <= end; at += kAhead * kRound) {
        Run<T, N> r[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) r[i] = load_run<T, N>(x + at + i * kRound);
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) put(at + i * kRound, r[i]);
      }
      for (; at < end; at += kRound) {
        if (at + N <= end)
          put(at, load_run<T, N>(x + at));
        else
          for (uint64_t i = at; i < end; ++i) out[i] = (T)((float)x[i] * factor * power);
      }
    });
  });
}

}  // namespace apex

namespace {

// No output lies over another one, or over a gradient that is not its own: workgroups read some while others write, and a tensor that is
// named twice would be scaled once or twice.
bool clip_apart(uint32_t count, const void *const *grad, void *const *out, const uint64_t *elements, const int *dtype)
{
  struct Range {
    uint64_t begin, end;
  };
  const auto range = [&](const void *p, uint32_t i) { return Range{(uintptr_t)p, (uintptr_t)p + elements[i] * element_size(dtype[i])}; };
  const std::unique_ptr<Range[]> written(new (std::nothrow) Range[count]);
  if (count && !written) return false;
  Range *last = written.get();
  for (uint32_t i = 0; i < count; ++i)
    if (elements[i]) *last++ = range(out[i], i);
  std::sort(written.get(), last, [](const Range &a, const Range &b) { return a.begin < b.begin; });
  for (Range *r = written.get(); r + 1 < last; ++r)
    if (r->end > r[1].begin) return false;
  for (uint32_t i = 0; i < count; ++i) {
    if (!elements[i] || out[i] == grad[i]) continue;
    const Range read = range(grad[i], i);
    const Range *const w = std::lower_bound(written.get(), last, read, [](const Range &a, const Range &b) { return a.end <= b.begin; });
    if (w != last && w->begin < read.end) return false;
  }
  return true;
}

}  // namespace

extern "C" {

int apex_clip_gradients_workspace_bytes(uint32_t count, size_t *bytes)
{
  if (!bytes) return APEX_ERR_INVALID_ARG;
  if (count > APEX_MAX_TENSORS) return APEX_ERR_TOO_LARGE;
  *bytes = round_up(sizeof(ClipSpace) + 8 * ((uint64_t)kClipPieces + count), 256);
  return APEX_OK;
}

int apex_clip_gradients(uint32_t count, const void *const *grad, void *const *out, const uint64_t *elements, const int *dtype,
                        float max_norm, float *norm, void *workspace, void *hip_stream)
{
  if ((count && (!grad || !elements || !dtype)) || !workspace || (uintptr_t)workspace % 256 || (uintptr_t)norm % 4 || !(max_norm > 0.0f))
    return APEX_ERR_INVALID_ARG;
  if (count > APEX_MAX_TENSORS) return APEX_ERR_TOO_LARGE;
  uint64_t total = 0, bytes = 0;
  bool in_place = true;
  for (uint32_t i = 0; i < count; ++i) {
    if (!elements[i]) continue;
    const uint32_t size = element_size(dtype[i]);
    if (!size || !grad[i] || (uintptr_t)grad[i] % size || (out && (!out[i] || (uintptr_t)out[i] % size))) return APEX_ERR_INVALID_ARG;
    if (elements[i] > 1ull << 48 || total > 1ull << 48) return APEX_ERR_TOO_LARGE;
    total += elements[i];
    bytes += elements[i] * size;
    in_place = in_place && (!out || out[i] == grad[i]);
  }
  if (!(in_place && max_norm == __builtin_inff()) && !clip_apart(count, grad, out ? out : const_cast<void *const *>(grad), elements, dtype))
    return APEX_ERR_INVALID_ARG;
  // pieces of whole rounds of a workgroup, so few that their sums are soon summed up
  const uint64_t piece = std::max<uint64_t>(kClipMinPiece, round_up((total + kClipPieces - 1) / kClipPieces, kClipMinPiece));
  if (piece > 0x7fffffffu) return APEX_ERR_TOO_LARGE;
  uint32_t all = 0;
  for (uint32_t i = 0; i < count; ++i) all += (uint32_t)((elements[i] + piece - 1) / piece);
  ClipArgs a{};
  a.all = all;
  a.piece = (uint32_t)piece;
  a.max_norm = max_norm;
  a.past_caches = bytes > kPastCachesBytes;
  a.norm = norm;
  a.space = static_cast<ClipSpace *>(workspace);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  // f for every launch's tensors, the launches forwards or backwards; a launch's table is in the tensors' order both ways
  const auto launches = [&](bool backwards, auto f) {
    for (uint32_t at = backwards ? count : 0; at != (backwards ? 0 : count);) {
      uint32_t from = at, to = at, some = 0;
      while (some < kClipTensors && (backwards ? from > 0 : to < count)) some += elements[backwards ? --from : to++] != 0;
      at = backwards ? from : to;
      a.tensors = a.pieces = 0;
      for (uint32_t i = from; i < to; ++i) {
        if (!elements[i]) continue;
        a.tensor[a.tensors++] = ClipTensor{grad[i], out ? out[i] : const_cast<void *>(grad[i]), elements[i], a.pieces, (uint32_t)dtype[i]};
        a.pieces += (uint32_t)((elements[i] + piece - 1) / piece);
      }
      if (a.pieces) f();
      a.before += a.pieces;
    }
  };
  if (!all) {  // nothing to sum up: the norm is 0
    clip_norm_kernel<<<dim3(1), dim3(kClipThreads), 0, stream>>>(a);
    APEX_HIP(hipGetLastError());
    return APEX_OK;
  }
  launches(false, [&] { clip_norm_kernel<<<dim3(a.pieces), dim3(kClipThreads), 0, stream>>>(a); });
  a.in_place = in_place;
  if (!(in_place && max_norm == __builtin_inff()))
    launches(true, [&] { clip_scale_kernel<<<dim3(a.pieces), dim3(kClipThreads), 0, stream>>>(a); });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

}  // extern "C"
