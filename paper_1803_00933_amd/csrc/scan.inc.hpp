// A gated linear recurrence and its gradient.  Included by apex_replay.hip (one translation unit).
//
//   h_t = a_t k_{t-1} h_{t-1} + b_t        k: 0 where the episode ended one step before
#include "elements.hpp"

namespace apex {

struct ScanArgs {
  uint32_t S, T, D;
  uint64_t g_seq, g_time, x_seq, x_time;  // strides in elements
  const void *g, *x;
  const float *discount;
  const int32_t *length;
  const float *h0;
  void *h;
  float *h_last, *carry;
};

struct ScanBackArgs {
  uint32_t S, T, D;
  uint64_t g_seq, g_time, x_seq, x_time;
  const void *g, *x;
  const float *discount;
  const int32_t *length;
  const float *carry;
  const void *dh;
  const float *dh_last;
  uint64_t dg_seq, dg_time, dx_seq, dx_time;
  void *dg, *dx;
  float *dh0;
};

__device__ __forceinline__ uint32_t scan_length(const int32_t *length, uint32_t s, uint32_t T)
{
  return length ? (uint32_t)min(max(length[s], 0), (int32_t)T) : T;
}

// sigma(g) and 1 - sigma(g), each to full precision: the smaller of the two is e^-|g| times the larger.
__device__ __forceinline__ void sigmoid_pair(float g, float *s, float *rest)
{
  const float e = exp2_of(-__builtin_fabsf(g) * kLog2e);
  const float big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
  *s = g >= 0.0f ? big : small;
  *rest = g >= 0.0f ? small : big;
}

// The step's factor and its term.
template <int kGate>
__device__ __forceinline__ void scan_gate(float g, float x, float *a, float *b)
{
  if (kGate == APEX_GATE_SIGMOID) {
    float rest;
    sigmoid_pair(g, a, &rest);
    *b = rest * x;
  } else {
    *a = g;
    *b = x;
  }
}

// Gradients of g and x from lambda and the state that came in.
template <int kGate>
__device__ __forceinline__ void scan_gate_back(float g, float x, float prev, float lambda, float *dg, float *dx)
{
  if (kGate == APEX_GATE_SIGMOID) {
    float a, rest;
    sigmoid_pair(g, &a, &rest);
    *dg = lambda * (prev - x) * (a * rest);
    *dx = lambda * rest;
  } else {
    *dg = lambda * prev;
    *dx = lambda;
  }
}

constexpr uint32_t kChannelThreads = 64;

// A thread per channel, step after step.
template <typename T, int kGate>
__global__ __launch_bounds__(kChannelThreads) void scan_channel_kernel(ScanArgs a)
{
  const uint32_t tiles = (a.D + kChannelThreads - 1) / kChannelThreads;
  const uint32_t s = blockIdx.x / tiles, d = blockIdx.x % tiles * kChannelThreads + threadIdx.x;
  if (d >= a.D) return;
  const uint32_t len = scan_length(a.length, s, a.T);
  const T *g = static_cast<const T *>(a.g) + s * a.g_seq + d;
  const T *x = static_cast<const T *>(a.x) + s * a.x_seq + d;
  T *h = static_cast<T *>(a.h) + (uint64_t)s * a.T * a.D + d;
  const float *const discount = a.discount ? a.discount + (uint64_t)s * a.T : nullptr;
  const uint32_t chunks = (a.T + APEX_SCAN_CHUNK - 1) / APEX_SCAN_CHUNK;
  float state = a.h0 ? a.h0[(uint64_t)s * a.D + d] : 0.0f;  // what passes into step t
  for (uint32_t t = 0; t < len; ++t) {
    if (a.carry && t % APEX_SCAN_CHUNK == 0) a.carry[((uint64_t)s * chunks + t / APEX_SCAN_CHUNK) * a.D + d] = state;
    float f, b;
    scan_gate<kGate>((float)g[t * a.g_time], (float)x[t * a.x_time], &f, &b);
    const float now = __builtin_fmaf(f, state, b);
    h[(uint64_t)t * a.D] = (T)now;
    state = discount && discount[t] == 0.0f ? 0.0f : now;
  }
  for (uint32_t t = len; t < a.T; ++t) h[(uint64_t)t * a.D] = (T)0.0f;
  if (a.h_last) a.h_last[(uint64_t)s * a.D + d] = state;
}

// The same backwards: chunk by chunk from the end, the states of a chunk computed again from what passes into it.
template <typename T, int kGate>
__global__ __launch_bounds__(kChannelThreads) void scan_channel_back_kernel(ScanBackArgs a)
{
  __shared__ float prev[APEX_SCAN_CHUNK][kChannelThreads];  // what passes into each step; a column is one thread's own
  const uint32_t tiles = (a.D + kChannelThreads - 1) / kChannelThreads;
  const uint32_t s = blockIdx.x / tiles, d = blockIdx.x % tiles * kChannelThreads + threadIdx.x;
  if (d >= a.D) return;
  const uint32_t len = scan_length(a.length, s, a.T);
  const T *g = static_cast<const T *>(a.g) + s * a.g_seq + d, *x = static_cast<const T *>(a.x) + s * a.x_seq + d;
  T *dg = static_cast<T *>(a.dg) + s * a.dg_seq + d, *dx = static_cast<T *>(a.dx) + s * a.dx_seq + d;
  const T *dh = static_cast<const T *>(a.dh) + (uint64_t)s * a.T * a.D + d;
  const float *const discount = a.discount ? a.discount + (uint64_t)s * a.T : nullptr;
  const uint32_t chunks = (a.T + APEX_SCAN_CHUNK - 1) / APEX_SCAN_CHUNK;
  for (uint32_t t = len; t < a.T; ++t) dg[t * a.dg_time] = dx[t * a.dx_time] = (T)0.0f;
  float back = a.dh_last ? a.dh_last[(uint64_t)s * a.D + d] : 0.0f;  // gradient of what step t passes on
  for (uint32_t end = len; end > 0;) {
    const uint32_t c = (end - 1) / APEX_SCAN_CHUNK, begin = c * APEX_SCAN_CHUNK;
    float state = a.carry[((uint64_t)s * chunks + c) * a.D + d];
    for (uint32_t t = begin; t < end; ++t) {
      prev[t - begin][threadIdx.x] = state;
      float f, b;
      scan_gate<kGate>((float)g[t * a.g_time], (float)x[t * a.x_time], &f, &b);
      const float now = __builtin_fmaf(f, state, b);
      state = discount && discount[t] == 0.0f ? 0.0f : now;
    }
    for (uint32_t t = end; t-- > begin;) {
      const float gt = (float)g[t * a.g_time], xt = (float)x[t * a.x_time];
      const float lambda = (float)dh[(uint64_t)t * a.D] + (discount && discount[t] == 0.0f ? 0.0f : back);
      float f, b, dgt, dxt;
      scan_gate<kGate>(gt, xt, &f, &b);
      scan_gate_back<kGate>(gt, xt, prev[t - begin][threadIdx.x], lambda, &dgt, &dxt);
      dg[t * a.dg_time] = (T)dgt;
      dx[t * a.dx_time] = (T)dxt;
      back = f * lambda;
    }
    end = begin;
  }
  if (a.dh0) a.dh0[(uint64_t)s * a.D + d] = back;
}

}  // namespace apex

namespace {

// Whether `rows` rows of `stride` elements and a last one of `width` can be addressed, and p is aligned to an element.
bool rows_fit(const void *p, uint32_t size, uint64_t rows, uint64_t stride, uint64_t rows2, uint64_t stride2, uint64_t width)
{
  uint64_t a, b, n;
  return (uintptr_t)p % size == 0 && !__builtin_mul_overflow(rows - 1, stride, &a) && !__builtin_mul_overflow(rows2 - 1, stride2, &b) &&
         !__builtin_add_overflow(a, b, &n) && !__builtin_add_overflow(n, width, &n) && n <= (1ull << 60);
}

// The same, and no two of the rows overlap: what is written.
bool rows_apart(const void *p, uint32_t size, uint64_t rows, uint64_t stride, uint64_t rows2, uint64_t stride2, uint64_t width)
{
  if (!rows_fit(p, size, rows, stride, rows2, stride2, width)) return false;
  if (rows < 2) return rows2 < 2 || stride2 >= width;
  if (rows2 < 2) return stride >= width;
  return (stride2 >= width && stride >= (rows2 - 1) * stride2 + width) || (stride >= width && stride2 >= (rows - 1) * stride + width);
}

uint32_t element_size(int dtype) { return dtype == APEX_F32 ? 4 : dtype == APEX_BF16 || dtype == APEX_F16 ? 2 : 0; }

// Calls f with a value of the element type.
template <typename F>
void with_type(int dtype, F f)
{
  if (dtype == APEX_F32)
    f(float());
  else if (dtype == APEX_BF16)
    f(__bf16());
  else
    f(_Float16());
}

int scan_check(uint32_t S, uint32_t T, uint32_t D, int dtype, int gate, const void *g, uint64_t g_seq, uint64_t g_time, const void *x,
               uint64_t x_seq, uint64_t x_time, const void *discount, const void *length)
{
  const uint32_t size = element_size(dtype);
  if (!S || !T || !D || T > 0x7fffffffu || !size || (gate != APEX_GATE_GIVEN && gate != APEX_GATE_SIGMOID) || !g || !x)
    return APEX_ERR_INVALID_ARG;
  if (!rows_fit(g, size, S, g_seq, T, g_time, D) || !rows_fit(x, size, S, x_seq, T, x_time, D)) return APEX_ERR_INVALID_ARG;
  if (((uintptr_t)discount | (uintptr_t)length) % 4) return APEX_ERR_INVALID_ARG;
  if ((uint64_t)S * ((D - 1) / kChannelThreads + 1) > 0xffffffffull / 1024 || (uint64_t)S * T > (1ull << 40)) return APEX_ERR_TOO_LARGE;
  return APEX_OK;
}

}  // namespace

extern "C" {

int apex_gated_scan_workspace_bytes(uint32_t S, uint32_t T, uint32_t D, size_t *bytes)
{
  if (!S || !T || !D || !bytes) return APEX_ERR_INVALID_ARG;
  *bytes = 0;
  return APEX_OK;
}

int apex_gated_scan(uint32_t S, uint32_t T, uint32_t D, int dtype, int gate, const void *g, uint64_t g_seq_stride,
                    uint64_t g_time_stride, const void *x, uint64_t x_seq_stride, uint64_t x_time_stride,
                    const float *discount, const int32_t *length, const float *h0, void *h, float *h_last, float *carry,
                    void *workspace, void *hip_stream)
{
  if (const int rc = scan_check(S, T, D, dtype, gate, g, g_seq_stride, g_time_stride, x, x_seq_stride, x_time_stride, discount, length))
    return rc;
  if (!h || (uintptr_t)h % element_size(dtype) || ((uintptr_t)h0 | (uintptr_t)h_last | (uintptr_t)carry) % 4) return APEX_ERR_INVALID_ARG;
  const ScanArgs a{S, T, D, g_seq_stride, g_time_stride, x_seq_stride, x_time_stride, g, x, discount, length, h0, h, h_last, carry};
  const dim3 grid(S * ((D - 1) / kChannelThreads + 1)), block(kChannelThreads);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  with_type(dtype, [&](auto t) {
    typedef decltype(t) E;
    if (gate == APEX_GATE_SIGMOID)
      scan_channel_kernel<E, APEX_GATE_SIGMOID><<<grid, block, 0, stream>>>(a);
    else
      scan_channel_kernel<E, APEX_GATE_GIVEN><<<grid, block, 0, stream>>>(a);
  });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

int apex_gated_scan_backward(uint32_t S, uint32_t T, uint32_t D, int dtype, int gate, const void *g, uint64_t g_seq_stride,
                             uint64_t g_time_stride, const void *x, uint64_t x_seq_stride, uint64_t x_time_stride,
                             const float *discount, const int32_t *length, const float *carry, const void *dh,
                             const float *dh_last, void *dg, uint64_t dg_seq_stride, uint64_t dg_time_stride, void *dx,
                             uint64_t dx_seq_stride, uint64_t dx_time_stride, float *dh0, void *workspace, void *hip_stream)
{
  if (const int rc = scan_check(S, T, D, dtype, gate, g, g_seq_stride, g_time_stride, x, x_seq_stride, x_time_stride, discount, length))
    return rc;
  const uint32_t size = element_size(dtype);
  if (!carry || !dh || !dg || !dx || (uintptr_t)dh % size || ((uintptr_t)carry | (uintptr_t)dh_last | (uintptr_t)dh0) % 4 ||
      !rows_apart(dg, size, S, dg_seq_stride, T, dg_time_stride, D) || !rows_apart(dx, size, S, dx_seq_stride, T, dx_time_stride, D))
    return APEX_ERR_INVALID_ARG;
  const ScanBackArgs a{S, T, D, g_seq_stride, g_time_stride, x_seq_stride, x_time_stride, g, x, discount, length, carry, dh, dh_last,
                       dg_seq_stride, dg_time_stride, dx_seq_stride, dx_time_stride, dg, dx, dh0};
  const dim3 grid(S * ((D - 1) / kChannelThreads + 1)), block(kChannelThreads);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  with_type(dtype, [&](auto t) {
    typedef decltype(t) E;
    if (gate == APEX_GATE_SIGMOID)
      scan_channel_back_kernel<E, APEX_GATE_SIGMOID><<<grid, block, 0, stream>>>(a);
    else
      scan_channel_back_kernel<E, APEX_GATE_GIVEN><<<grid, block, 0, stream>>>(a);
  });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

}  // extern "C"
