// Distillation from a teacher's top logits, with the gradient.  Included by apex_replay.hip (one translation unit).
//
// With c = log2(e) / tau everything that is summed over the vocabulary is 2^(z c - R), R the whole number next to max z c: one
// fused multiply-add and one instruction of the transcendental unit an element, and R, a whole number, adds and cancels exactly.
// With a rest class the sum runs over the tokens that are not named, with a maximum of its own, and the named ones, which are
// gathered, join it afterwards: the rest's share keeps its precision however little of the student's mass it has.
#include "elements.hpp"

namespace apex {

struct DistillArgs {
  uint32_t N, V, K, H, value_dtype;  // H: places of the table of named tokens, a power of two of at least 2 K
  uint64_t row_stride, grad_stride;
  const void *logits;
  const int32_t *top_index;
  const void *top_value;
  const float *top_lse, *weight;
  double inv_tau;
  float c, grad_scale;  // log2(e) / tau, 1 / tau
  float *loss, *lse;
  void *grad;
};

// The named tokens of a row, in LDS: a table by open addressing, and a bit for each run of the row that holds one.
struct Named {
  int32_t *key;       // [H] token, or -1
  uint32_t *place;    // [H] the first place that names it; later, as a float, the token's gradient
  int32_t *slot;      // [K] the table's entry of a place; -1: empty
  float *value, *z;   // [K] teacher's and student's logits
  uint64_t *runs;
  uint32_t H;

  __device__ __forceinline__ uint32_t hash(int32_t token) const { return ((uint32_t)token * 2654435761u) >> (32 - __builtin_ctz(H)); }

  __device__ __forceinline__ int32_t find(int32_t token) const
  {
    for (uint32_t i = hash(token);; i = (i + 1) & (H - 1)) {  // at most half of the entries are in use
      if (key[i] == token) return (int32_t)i;
      if (key[i] < 0) return -1;
    }
  }
};

__host__ __device__ constexpr uint32_t distill_table(uint32_t K)
{
  uint32_t H = 64;
  while (H < 2 * K) H *= 2;
  return H;
}
// Bytes of LDS of a row of `runs` runs.
__host__ __device__ constexpr uint32_t distill_lds(uint32_t K, uint32_t runs)
{
  return (runs + 63) / 64 * 8 + distill_table(K) * 8 + K * 12;
}

__device__ __forceinline__ Named named_in(uint64_t *lds, uint32_t K, uint32_t H, uint32_t runs)
{
  Named n;
  n.H = H;
  n.runs = lds;
  n.key = reinterpret_cast<int32_t *>(lds + (runs + 63) / 64);
  n.place = reinterpret_cast<uint32_t *>(n.key + H);
  n.slot = reinterpret_cast<int32_t *>(n.place + H);
  n.value = reinterpret_cast<float *>(n.slot + K);
  n.z = n.value + K;
  return n;
}

__device__ __forceinline__ float typed_element(const void *p, uint32_t dtype, uint64_t i)
{
  if (dtype == APEX_F32) return static_cast<const float *>(p)[i];
  if (dtype == APEX_BF16) return (float)static_cast<const __bf16 *>(p)[i];
  return (float)static_cast<const _Float16 *>(p)[i];
}

// The sum of 2^(z c - R) over logits whose largest is m, R = m c rounded to a whole number (0 while m is -inf).
struct Sum {
  float m, s;
  __device__ __forceinline__ static float ref(float m, float c) { return m == -__builtin_inff() ? 0.0f : __builtin_rintf(m * c); }
};

// Logits [run * N, run * N + N) of a row, -inf beyond its end.
template <typename T, int N>
__device__ __forceinline__ void logits_of(const T *row, uint32_t run, uint32_t V, float (&z)[N])
{
  const uint32_t at = run * N;
  if (at + N <= V) {
    const Run<T, N> r = load_run<T, N>(row + at);
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = element<N, T>(r, e);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = at + e < V ? (float)row[at + e] : -__builtin_inff();
  }
}

template <int N>
__device__ __forceinline__ void add_to(Sum &a, const float (&z)[N], float c)
{
  float top = z[0];
#pragma unroll
  for (int e = 1; e < N; ++e) top = fmaxf(top, z[e]);
  const float m = fmaxf(a.m, top), R = Sum::ref(m, c);
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < N; ++e) s += exp2_of(__builtin_fmaf(z[e], c, -R));
  a.s = __builtin_fmaf(a.s, a.m == -__builtin_inff() ? 1.0f : exp2_of(Sum::ref(a.m, c) - R), s);  // (NaN may be there without a maximum)
  a.m = m;
}

// 2^x scale, an element of the gradient: gradual down to the smallest numbers where the gradient has them (scale_low = scale
// 2^-64); of one of 16 bits a power below 2^-126 is 0.
template <typename T>
__device__ __forceinline__ float power(float x, float scale, float scale_low)
{
  if (sizeof(T) < 4) return exp2_of(x) * scale;
  const bool low = x < -125.0f;
  return exp2_of(low ? x + 64.0f : x) * (low ? scale_low : scale);
}

// e^x for the teacher's and the student's places: the exponent keeps 48 bits until its whole part is split off.
__device__ __forceinline__ double exp_of(double x)
{
  if (x < -200.0) return 0.0;
  const double y = x * 1.4426950408889634, n = __builtin_rint(y);
  return __builtin_ldexp((double)exp2_of((float)(y - n)), (int)fmin(n, 1000.0));
}

// ln x, x > 0: the exponent apart, so that the error is that of a logarithm next to 0.
__device__ __forceinline__ double ln_of(float x)
{
  int e = (int)(__float_as_uint(x) >> 23) - 127;
  if (!(x >= 0x1p-126f && x < __builtin_inff())) return (double)log2_of(x) * 0.6931471805599453;
  float m = __uint_as_float((__float_as_uint(x) & 0x007fffffu) | 0x3f800000u);
  if (m > 1.41421354f) m *= 0.5f, ++e;
  return ((double)e + (double)log2_of(m)) * 0.6931471805599453;
}

// What a row's gradient is made of: of a token not named 2^(z c - R) * scale.
struct RowGradient {
  float R, scale;
  bool zero;  // the row's weight is 0
};

// The teacher's side, by one wave, once the row's sum `all` (without the named tokens if there is a rest class) is known:
// writes loss and lse, leaves the gradients of the named tokens in the table.
__device__ __forceinline__ RowGradient settle_row(const DistillArgs &a, const Named &n, uint32_t row, Sum all)
{
  const uint32_t lane = lane_id();
  const float c = a.c;
  const bool rest_class = a.top_lse != nullptr;
  uint32_t mine = 0;
  float t_top = -__builtin_inff(), z_top = -__builtin_inff();
  for (uint32_t k = lane; k < a.K; k += kWave)
    if (n.slot[k] >= 0) {
      ++mine;
      t_top = fmaxf(t_top, n.value[k]);
      z_top = fmaxf(z_top, n.z[k]);
    }
  const uint32_t named = (uint32_t)wave_sum((float)mine);  // at most APEX_MAX_TOP
  t_top = wave_max(t_top);
  const float t_R = Sum::ref(t_top, c);
  const float R_rest = Sum::ref(all.m, c), s_rest = all.s;
  float R = R_rest, s = s_rest;
  if (rest_class) {
    z_top = fmaxf(wave_max(z_top), all.m);
    R = Sum::ref(z_top, c);
  }
  float t_sum = 0.0f, z_sum = 0.0f;
  for (uint32_t k = lane; k < a.K; k += kWave)
    if (n.slot[k] >= 0) {
      t_sum += exp2_of(__builtin_fmaf(n.value[k], c, -t_R));
      z_sum += exp2_of(__builtin_fmaf(n.z[k], c, -R));
    }
  t_sum = wave_sum(t_sum);
  if (rest_class) s = wave_sum(z_sum) + (s_rest == 0.0f ? 0.0f : s_rest * exp2_of(R_rest - R));
  if (s == 0.0f) s = __builtin_nanf("");  // no finite logit
  const float inv_s = 1.0f / s;
  // Logarithms of nearly equal numbers are subtracted below: in 64 bits, a few operations for each named token.
  const auto log_sum = [&](float m, float ref, float sum) {  // of a Sum; c, as rounded, only scales what is relative to m
    if (m == -__builtin_inff()) return -__builtin_inf();
    return __builtin_fma((double)m, a.inv_tau, (ln_of(sum) + 0.6931471805599453 * __builtin_fma(-(double)m, (double)c, (double)ref)));
  };
  const double ln_all = log_sum(rest_class ? z_top : all.m, R, s);
  const double ln_teacher = rest_class ? (double)a.top_lse[row] : log_sum(t_top, t_R, t_sum);
  const auto ln_q = [&](uint32_t k) { return __builtin_fma((double)n.value[k], a.inv_tau, -ln_teacher); };
  const auto ln_p = [&](uint32_t k) { return __builtin_fma((double)n.z[k], a.inv_tau, -ln_all); };
  const bool teaches = t_sum != 0.0f;  // not -inf for every place
  float mass = 0.0f, loss = 0.0f;
  for (uint32_t k = lane; k < a.K; k += kWave)
    if (n.slot[k] >= 0 && teaches) {
      const double l = ln_q(k);
      const float q = (float)exp_of(l);
      mass += q;
      loss += q == 0.0f ? 0.0f : q * (float)(l - ln_p(k));
    }
  mass = wave_sum(mass);
  loss = wave_sum(loss);
  float rest = 0.0f;
  if (rest_class && named < a.V) {
    rest = mass > 1.0f ? 0.0f : 1.0f - mass;
    if (rest != 0.0f) loss += rest * (float)(ln_of(rest) - (log_sum(all.m, R_rest, s_rest) - ln_all));
  }
  if (s != s) loss = s;
  if (lane == 0) {
    a.loss[row] = loss;
    if (a.lse) a.lse[row] = (float)ln_all;
  }
  const float w = a.weight ? a.weight[row] : 1.0f, wt = w * a.grad_scale;
  for (uint32_t k = lane; k < a.K; k += kWave)
    if (n.slot[k] >= 0) {
      const double q = teaches ? exp_of(ln_q(k)) : 0.0;
      n.place[n.slot[k]] = __float_as_uint(w == 0.0f ? 0.0f : (float)(wt * (((double)mass + (double)rest) * exp_of(ln_p(k)) - q)));
    }
  RowGradient g{R_rest, wt * (mass * inv_s), w == 0.0f};
  if (rest_class) g.scale = s_rest == 0.0f ? 0.0f : wt * ((mass + rest) * inv_s * exp2_of(R_rest - R) - rest / s_rest);
  return g;
}

constexpr uint32_t kDistillThreads = 512;

// A workgroup per row, which it reads twice: for the sum, and for the gradient.
template <typename T>
__global__ __launch_bounds__(kDistillThreads) void distill_rows_kernel(DistillArgs a)
{
  constexpr int N = 16 / sizeof(T);
  extern __shared__ uint64_t lds[];
  __shared__ float red_m[kDistillThreads / kWave], red_s[kDistillThreads / kWave];
  __shared__ RowGradient sh_gradient;
  const uint32_t thread = threadIdx.x, lane = lane_id(), wave = thread / kWave, row = blockIdx.x;
  const uint32_t runs = (a.V + N - 1) / N;
  const Named n = named_in(lds, a.K, a.H, runs);
  const T *const z_row = static_cast<const T *>(a.logits) + row * a.row_stride;
  for (uint32_t i = thread; i < (runs + 63) / 64; i += kDistillThreads) n.runs[i] = 0;
  for (uint32_t i = thread; i < a.H; i += kDistillThreads) n.key[i] = -1, n.place[i] = 0xffffffffu;
  __syncthreads();
  for (uint32_t k = thread; k < a.K; k += kDistillThreads) {
    const uint64_t at = (uint64_t)row * a.K + k;
    const int32_t token = a.top_index[at];
    int32_t slot = -1;
    if (token >= 0 && (uint32_t)token < a.V) {
      n.value[k] = typed_element(a.top_value, a.value_dtype, at);
      n.z[k] = (float)z_row[token];
      for (uint32_t i = n.hash(token); slot < 0; i = (i + 1) & (a.H - 1)) {
        const int32_t had = atomicCAS(n.key + i, -1, token);
        if (had == -1 || had == token) slot = (int32_t)i;
      }
      atomicMin(n.place + slot, k);
      atomicOr(reinterpret_cast<unsigned long long *>(n.runs + (token / N) / 64), 1ull << ((token / N) % 64));
    }
    n.slot[k] = slot;
  }
  __syncthreads();
  for (uint32_t k = thread; k < a.K; k += kDistillThreads)
    if (n.slot[k] >= 0 && n.place[n.slot[k]] != k) n.slot[k] = -1;  // named by an earlier place

  Sum sum{-__builtin_inff(), 0.0f};
  for (uint32_t run = thread; run < runs; run += kDistillThreads) {
    float z[N];
    logits_of<T, N>(z_row, run, a.V, z);
    if (a.top_lse && (n.runs[run / 64] >> (run % 64) & 1)) {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (n.find((int32_t)(run * N + e)) >= 0) z[e] = -__builtin_inff();
    }
    add_to<N>(sum, z, a.c);
  }
  const float m = wave_max(sum.m), R = Sum::ref(m, a.c);
  const float s = wave_sum(sum.m == -__builtin_inff() ? sum.s : sum.s * exp2_of(Sum::ref(sum.m, a.c) - R));
  if (lane == 0) red_m[wave] = m, red_s[wave] = s;
  __syncthreads();
  if (wave == 0) {
    constexpr uint32_t kWaves = kDistillThreads / kWave;
    const float wm = lane < kWaves ? red_m[lane] : -__builtin_inff(), ws = lane < kWaves ? red_s[lane] : 0.0f;
    const float top = wave_max(wm), top_R = Sum::ref(top, a.c);
    const Sum all{top, wave_sum(wm == -__builtin_inff() ? ws : ws * exp2_of(Sum::ref(wm, a.c) - top_R))};
    const RowGradient g = settle_row(a, n, row, all);
    if (lane == 0) sh_gradient = g;
  }
  if (!a.grad) return;
  __syncthreads();
  const RowGradient g = sh_gradient;
  T *const out = static_cast<T *>(a.grad) + row * a.grad_stride;
  for (uint32_t run = thread; run < runs; run += kDistillThreads) {
    float z[N];
    logits_of<T, N>(z_row, run, a.V, z);
    const bool has_named = n.runs[run / 64] >> (run % 64) & 1;
    const uint32_t at = run * N;
    Run<T, N> r;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float v = g.zero ? 0.0f : power<T>(__builtin_fmaf(z[e], a.c, -g.R), g.scale, g.scale * 0x1p-64f);
      if (has_named) {
        const int32_t slot = n.find((int32_t)(at + e));
        if (slot >= 0) v = __uint_as_float(n.place[slot]);
      }
      r[e] = (T)v;
    }
    if (at + N <= a.V) {
      *reinterpret_cast<Run<T, N> *>(out + at) = r;
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (at + e < a.V) out[at + e] = r[e];
    }
  }
}

}  // namespace apex

extern "C" {

int apex_distill_topk_workspace_bytes(uint32_t N, uint32_t V, size_t *bytes)
{
  if (!N || !V || !bytes) return APEX_ERR_INVALID_ARG;
  if (V > APEX_MAX_VOCABULARY) return APEX_ERR_TOO_LARGE;
  *bytes = 0;
  return APEX_OK;
}

int apex_distill_topk(uint32_t N, uint32_t V, uint32_t K, int dtype, const void *logits, uint64_t row_stride,
                      const int32_t *top_index, int value_dtype, const void *top_value, const float *top_lse,
                      const float *weight, float temperature, float *loss, float *lse, void *grad, uint64_t grad_stride,
                      void *workspace, void *hip_stream)
{
  const uint32_t size = element_size(dtype), value_size = element_size(value_dtype);
  if (!N || !V || !K || !size || !value_size || !logits || !top_index || !top_value || !loss) return APEX_ERR_INVALID_ARG;
  if (!(temperature > 0.0f) || !(temperature < __builtin_inff())) return APEX_ERR_INVALID_ARG;
  if (!rows_fit(logits, size, N, row_stride, 1, 0, V) || (grad && !rows_apart(grad, size, N, grad_stride, 1, 0, V)))
    return APEX_ERR_INVALID_ARG;
  if (((uintptr_t)top_index | (uintptr_t)top_lse | (uintptr_t)weight | (uintptr_t)loss | (uintptr_t)lse) % 4 ||
      (uintptr_t)top_value % value_size)
    return APEX_ERR_INVALID_ARG;
  if (V > APEX_MAX_VOCABULARY || K > APEX_MAX_TOP || N > 0xffffffffu / 1024) return APEX_ERR_TOO_LARGE;
  const double inv_tau = 1.0 / (double)temperature;
  const DistillArgs a{N, V, K, distill_table(K), (uint32_t)value_dtype, row_stride, grad_stride, logits, top_index, top_value, top_lse,
                      weight, inv_tau, (float)(1.4426950408889634 * inv_tau), (float)inv_tau, loss, lse, grad};
  const uint32_t lds = distill_lds(K, (V + 16 / size - 1) / (16 / size));
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  with_type(dtype, [&](auto t) { distill_rows_kernel<decltype(t)><<<dim3(N), dim3(kDistillThreads), lds, stream>>>(a); });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

}  // extern "C"
