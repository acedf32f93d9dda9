// Distillation from a teacher's top logits, with the gradient.  Included by apex_replay.hip (one translation unit).
//
// With c = log2(e) / tau everything that is summed over the vocabulary is 2^(z c - R), R the whole number next to max z c: one
// fused multiply-add and one instruction of the transcendental unit an element, and R, a whole number, adds and cancels exactly.
// (Far from 0 it is no longer next to max z c: Sum.)
// With a rest class the sum runs over the tokens that are not named, with a maximum of its own, and the named ones, which are
// gathered, join it afterwards: the rest's share keeps its precision however little of the student's mass it has.  Where that is
// nearly all of it, or the student is near its teacher, what cancels is not subtracted: settle.
#include "elements.hpp"

namespace apex {

struct DistillArgs {
  uint32_t N, V, K, value_dtype;
  uint64_t row_stride, grad_stride;
  const void *logits;
  const int32_t *top_index;
  const void *top_value;
  const float *top_lse, *weight;
  double inv_tau;
  float c, grad_scale;  // log2(e) / tau, 1 / tau
  float *loss, *lse;
  void *grad;
  bool past_caches, whole_lines;  // the gradient is stored past the caches; rows begin with cache lines
};

// The named tokens of a row, in LDS.
struct Named {
  uint32_t *bits;        // [ceil(V / 64)] words of 64 bits: a bit for every token
  double *q;             // [K] the teacher's probability
  int32_t *token;        // [K] -1: a place that does not count
  float *value, *z;      // [K] the teacher's and the student's logits

  // Which of the N tokens of a run are named.
  template <uint32_t N>
  __device__ __forceinline__ uint32_t mask(uint32_t run) const
  {
    const uint32_t byte = reinterpret_cast<const uint8_t *>(bits)[run * N / 8];
    return N == 8 ? byte : byte >> (run % 2 * 4) & 15u;
  }
};

__host__ __device__ constexpr uint32_t distill_lds(uint32_t K, uint32_t V)  // bytes
{
  return (V + 63) / 64 * 8 + K * 20;
}

__device__ __forceinline__ Named named_in(uint64_t *lds, uint32_t K, uint32_t V)
{
  Named n;
  n.bits = reinterpret_cast<uint32_t *>(lds);
  n.q = reinterpret_cast<double *>(lds + (V + 63) / 64);
  n.token = reinterpret_cast<int32_t *>(n.q + K);
  n.value = reinterpret_cast<float *>(n.token + K);
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
// In 32 bits R misses m c by up to 64 where that is next to 2^31: the sum is relative to R all the same.  Beyond that, as with logits
// masked by their type's lowest value, R is m c itself, and the power is 1 for z = m and 0 for every other z.
struct Sum {
  float m, s;
  __device__ __forceinline__ static bool far(float m, float c) { return !(__builtin_fabsf(m * c) < 0x1p31f) && m != -__builtin_inff(); }
  __device__ __forceinline__ static double ref(float m, float c)
  {
    if (far(m, c)) return (double)m * (double)c;
    return m == -__builtin_inff() ? 0.0 : (double)__builtin_rintf(m * c);
  }
};

// z c - R as z times + plus.  Far from 0 `times` is the power of 2 that brings m into [2^32, 2^33): whatever differs from m is 2^8 away.
struct Exponent {
  float times, plus;
  __device__ __forceinline__ Exponent(float m, float c)
  {
    if (Sum::far(m, c)) {
      times = __uint_as_float(min(286u - (__float_as_uint(m) >> 23 & 255u), 254u) << 23);
      plus = -m * times;
    } else {
      times = c;
      plus = m == -__builtin_inff() ? 0.0f : -__builtin_rintf(m * c);
    }
  }
  __device__ __forceinline__ float of(float z) const { return __builtin_fmaf(z, times, plus); }
};

// What a sum relative to `from` is multiplied by to be relative to `to`, from <= to, neither of them -inf.
__device__ __forceinline__ float relative(float from, float to, float c)
{
  if (Sum::far(to, c)) return exp2_of((float)(((double)from - (double)to) * (double)c));
  return exp2_of(__builtin_rintf(from * c) - __builtin_rintf(to * c));
}

// Adds a run; x is that of the sum's largest.
template <int N>
__device__ __forceinline__ void add_to(Sum &a, Exponent &x, const float (&z)[N], float c)
{
  float top = z[0];
#pragma unroll
  for (int e = 1; e < N; ++e) top = fmaxf(top, z[e]);
  if (top > a.m) {  // (NaN may be there without a maximum)
    if (a.m != -__builtin_inff()) a.s *= relative(a.m, top, c);
    a.m = top;
    x = Exponent(top, c);
  }
  float s = 0.0f;
#pragma unroll
  for (int e = 0; e < N; ++e) s += exp2_of(x.of(z[e]));
  a.s += s;
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

constexpr double kLn2d = 0.6931471805599453;

// ln x, x > 0: the exponent apart, so that the error is that of a logarithm next to 0.
__device__ __forceinline__ double ln_of(float x)
{
  int e = (int)(__float_as_uint(x) >> 23) - 127;
  if (!(x >= 0x1p-126f && x < __builtin_inff())) return (double)log2_of(x) * 0.6931471805599453;
  float m = __uint_as_float((__float_as_uint(x) & 0x007fffffu) | 0x3f800000u);
  if (m > 1.41421354f) m *= 0.5f, ++e;
  return ((double)e + (double)log2_of(m)) * 0.6931471805599453;
}

// e^x for the teacher's and the student's places: the exponent keeps 48 bits until its whole part is split off.
__device__ __forceinline__ double exp_of(double x)
{
  if (x < -200.0) return 0.0;
  const double y = x * 1.4426950408889634, n = __builtin_rint(y);
  return __builtin_ldexp((double)exp2_of((float)(y - n)), (int)fmin(n, 1000.0));
}

// The same to 1e-12, for what is subtracted from 1: the series within ln 2 / 2 of a whole power of 2.
__device__ __forceinline__ double exactly_exp_of(double x)
{
  if (x < -200.0) return 0.0;
  const double n = __builtin_rint(x * 1.4426950408889634), f = __builtin_fma(-n, kLn2d, x);
  double e = 1.0 / 3628800;
  constexpr double kFactor[] = {1.0 / 362880, 1.0 / 40320, 1.0 / 5040, 1.0 / 720, 1.0 / 120, 1.0 / 24, 1.0 / 6, 0.5, 1.0, 1.0};
#pragma unroll
  for (double k : kFactor) e = __builtin_fma(e, f, k);
  return __builtin_ldexp(e, (int)fmin(n, 1000.0));
}

// e^u - 1 - u for |u| < 1, not by that difference: u^2 times its series.
__device__ __forceinline__ float exp_beyond(float u)
{
  float e = 1.0f / 39916800;
  constexpr float kFactor[] = {1.0f / 3628800, 1.0f / 362880, 1.0f / 40320, 1.0f / 5040, 1.0f / 720, 1.0f / 120, 1.0f / 24, 1.0f / 6, 0.5f};
#pragma unroll
  for (float k : kFactor) e = __builtin_fmaf(e, u, k);
  return e * u * u;
}

// w - ln(1 + w) for -1/2 <= w: up to 1 by ln(1 + w) = 2 artanh t, t = w / (2 + w), of which w - 2 t = w t.
__device__ __forceinline__ float log_short_of(float w)
{
  if (w > 1.0f) return w - (float)ln_of(1.0f + w);
  const float t = w / (2.0f + w), tt = t * t;
  float e = 1.0f / 19;
  constexpr float kFactor[] = {1.0f / 17, 1.0f / 15, 1.0f / 13, 1.0f / 11, 1.0f / 9, 1.0f / 7, 1.0f / 5, 1.0f / 3};
#pragma unroll
  for (float k : kFactor) e = __builtin_fmaf(e, tt, k);
  return w * t - 2.0f * t * tt * e;
}

// What a row's gradient is made of: of a token not named 2^(z c - R) * scale, R that of m.
struct RowGradient {
  float m, scale;
  bool zero;  // the row's weight is 0
};

// Enters place k's token; whether another place names it too.
__device__ __forceinline__ bool enter_named(const DistillArgs &a, const Named &n, uint32_t k, int32_t token, float value)
{
  const bool counts = token >= 0 && (uint32_t)token < a.V;
  n.token[k] = counts ? token : -1;
  n.value[k] = value;
  return counts && (atomicOr(n.bits + token / 32, 1u << (token % 32)) >> (token % 32) & 1);
}

// What a wave knows of a row's teacher.
struct Teacher {
  double top, ln_sum;  // ln q = (value - top) / tau - ln_sum
  double mass, part;   // sum of q: 1 without a rest class, off which the lanes' parts are by 1e-7
  uint32_t named;      // places that count
  bool teaches;        // not -inf for every one of them
};

// ln of a sum of 2^(z c - R) whose largest z is m, less m / tau; c, as rounded, only scales what is relative to m.
__device__ __forceinline__ double log_sum(const DistillArgs &a, float m, double R, float sum)
{
  if (m == -__builtin_inff()) return -__builtin_inf();
  return ln_of(sum) + kLn2d * __builtin_fma(-(double)m, (double)a.c, R);
}

// The part of a row that needs no sum over the vocabulary, by one wave: drops places whose token an earlier one names (if there
// are any: `repeated`), and leaves the q of the others.
__device__ __forceinline__ Teacher teach(const DistillArgs &a, const Named &n, uint32_t row, bool repeated)
{
  const uint32_t lane = lane_id();
  uint32_t mine = 0;
  float top = -__builtin_inff();
  if (repeated)
    for (uint32_t k = lane; k < a.K; k += kWave)
      for (uint32_t i = 0; i < k; ++i)
        if (n.token[i] == n.token[k]) n.token[k] = -1;  // (whatever goes first, the first place of a token stays, and drops the others)
  for (uint32_t k = lane; k < a.K; k += kWave)
    if (n.token[k] >= 0) ++mine, top = fmaxf(top, n.value[k]);
  Teacher t;
  t.named = (uint32_t)wave_sum((float)mine);  // at most APEX_MAX_TOP
  top = wave_max(top);
  const Exponent x(top, a.c);
  float sum = 0.0f;
  for (uint32_t k = lane; k < a.K; k += kWave)
    if (n.token[k] >= 0) sum += exp2_of(x.of(n.value[k]));
  sum = wave_sum(sum);
  t.teaches = sum != 0.0f;
  t.top = a.top_lse || top == -__builtin_inff() ? 0.0 : (double)top;
  t.ln_sum = a.top_lse ? (double)a.top_lse[row] : log_sum(a, top, Sum::ref(top, a.c), sum);
  double mass = 0.0;
  for (uint32_t k = lane; k < a.K; k += kWave)
    if (n.token[k] >= 0) {
      const double ln_q = __builtin_fma((double)n.value[k] - t.top, a.inv_tau, -t.ln_sum);
      const double q = !t.teaches ? 0.0 : a.top_lse ? exactly_exp_of(ln_q) : exp_of(ln_q);
      n.q[k] = q;
      mass += q;
    }
  t.part = mass;
  t.mass = a.top_lse ? wave_sum(mass) : t.teaches ? 1.0 : 0.0;
  return t;
}

// The rest of it, by the same wave, once the row's sum `all` (without the named tokens if there is a rest class) is known: writes
// the gradients of the named tokens (out: the row's gradient, or null).
// The loss is not summed up as it is defined: q ln(q/p) and r ln(r/s) cancel to second order where the student is near its teacher,
// and r and s to first where little is named.  With u = ln(p/q) and w = s/r - 1 (-sum (p - q) / r unless s is the smaller part) it is
//     sum q (e^u - 1 - u) + r (w - ln(1 + w)),     with - sum (p - q) in place of the second where there is no rest,
// terms that are not negative, each by a form of its own that does not cancel; and the gradient has p - q = q (e^u - 1), and
// (M + r) - r/s = w / (1 + w) for the rest.  Errors of p's common factor, from the sum in 32 bits, enter times p - q.  (As defined:
// losses of V = 40000, K = 1, tau = 4 off by 2e-3.)  64 bits, a few operations for each named token.
struct Settled {
  RowGradient gradient;
  double base, ln_all;       // ln p = (z - base) / tau - ln_all
  double rest, more, ratio;  // r; sum q - 1 where r is 0; w
  double terms;              // a lane's part of the sum of q (e^u - 1 - u)
  float apart;               // of p - q: the sum if there is a rest class, else a lane's part
  bool plain;                // w is not below -1/2
};

template <typename T>
__device__ __forceinline__ Settled settle(const DistillArgs &a, const Named &n, uint32_t row, const Teacher &t, Sum all, T *out)
{
  const uint32_t lane = lane_id();
  const float w = a.weight ? a.weight[row] : 1.0f, wt = w * a.grad_scale;
  Settled r;
  float top = all.m, s = all.s, to_all = 1.0f;  // to_all: from a sum over the rest to one over the row
  if (a.top_lse) {
    float z_top = -__builtin_inff(), z_sum = 0.0f;
    for (uint32_t k = lane; k < a.K; k += kWave)
      if (n.token[k] >= 0) z_top = fmaxf(z_top, n.z[k]);
    top = fmaxf(wave_max(z_top), all.m);
    const Exponent x(top, a.c);
    for (uint32_t k = lane; k < a.K; k += kWave)
      if (n.token[k] >= 0) z_sum += exp2_of(x.of(n.z[k]));
    to_all = all.s == 0.0f ? 0.0f : relative(all.m, top, a.c);
    s = wave_sum(z_sum) + (all.s == 0.0f ? 0.0f : all.s * to_all);
  }
  if (s == 0.0f) s = __builtin_nanf("");  // no finite logit
  const float inv_s = 1.0f / s;
  r.gradient = RowGradient{all.m, wt * ((float)t.mass * inv_s), w == 0.0f};
  r.base = top == -__builtin_inff() ? 0.0 : (double)top;
  r.ln_all = log_sum(a, top, Sum::ref(top, a.c), s);
  r.rest = 0.0;
  if (a.top_lse && t.named < a.V) r.rest = t.mass > 1.0 ? 0.0 : 1.0 - t.mass;
  r.more = r.rest > 0.0 ? 0.0 : t.mass - 1.0;
  r.terms = 0.0, r.apart = 0.0f;
  for (uint32_t k = lane; k < a.K; k += kWave)
    if (n.token[k] >= 0) {
      const double q = n.q[k], ln_p = __builtin_fma((double)n.z[k] - r.base, a.inv_tau, -r.ln_all);
      const double u = ln_p - __builtin_fma((double)n.value[k] - t.top, a.inv_tau, -t.ln_sum);
      double diff, term;
      if (__builtin_fabs(u) < 1.0) {
        const float beyond = exp_beyond((float)u);
        term = q * beyond;
        diff = q * (beyond + u);
      } else {
        diff = exp_of(ln_p) - q;
        term = q == 0.0 ? diff : diff - q * u;
      }
      r.terms += term;
      r.apart += (float)diff;
      if (out) out[n.token[k]] = (T)(w == 0.0f ? 0.0f : (float)(wt * (diff + r.more * (q + diff))));
    }
  if (!a.top_lse) return r;
  r.apart = wave_sum(r.apart);
  const float share = inv_s * to_all, others = all.s == 0.0f ? 0.0f : all.s * share;  // others: s
  r.ratio = others < 0.5f ? (double)others / r.rest - 1.0 : -(double)r.apart / r.rest;
  r.plain = r.rest == 0.0 || !(r.ratio < -0.5);
  if (all.s == 0.0f)
    r.gradient.scale = 0.0f;
  else if (r.plain)
    r.gradient.scale = wt * (share * (r.rest == 0.0 ? (float)t.mass : (float)r.ratio / (1.0f + (float)r.ratio)));
  else
    r.gradient.scale = wt * (share - (float)r.rest / all.s);
  return r;
}

// loss and lse of a settled row: the other waves do not wait for them.
__device__ __forceinline__ void conclude(const DistillArgs &a, uint32_t row, const Teacher &t, Sum all, const Settled &r)
{
  double loss = wave_sum(r.terms);
  if (r.rest == 0.0)
    loss += t.named == a.V ? r.more : -(double)(a.top_lse ? r.apart : wave_sum(r.apart));
  else if (r.plain)
    loss += (float)r.rest * log_short_of((float)r.ratio);
  else  // far less than the teacher gives the rest
    loss += r.rest * (r.ratio + ln_of((float)r.rest) -
                      __builtin_fma((double)all.m - r.base, a.inv_tau, log_sum(a, all.m, Sum::ref(all.m, a.c), all.s) - r.ln_all));
  if (!a.top_lse) {  // q as if it summed up to 1
    const double off = wave_sum(t.part) - 1.0;
    loss = t.teaches ? loss - off * (t.named == a.V ? loss : 1.0 + loss) : 0.0;
  }
  if (!(__builtin_fabs(r.ln_all) < __builtin_inf())) loss = __builtin_nan("");  // the sum was NaN
  if (lane_id() == 0) {
    a.loss[row] = (float)loss;
    if (a.lse) a.lse[row] = (float)__builtin_fma(r.base, a.inv_tau, r.ln_all);
  }
}

// A workgroup per row.  kHeld runs of 16 bytes of the row stay in a thread's registers from the sum to the gradient, so that the
// row is read once; kMore: what a row has beyond them is read again.
// Bound by memory: 2048 x 32768 bf16 58.5 us for 269 MB (4.6 TB/s; a copy reaches 5.1), 777 x 49999 f16 34-37 us (4.2-4.6), 3001 x
// 131072 bf16 with a rest class 370 us for 1.58 GB (4.3): there a compute unit has one row at a time, and its memory waits while
// the row is settled.  Reading every row twice took 115, 56 and 588.  The loss alone 27 us for the first.
// Named tokens cost instructions where the row is gone through: looking every element of a marked run up in a table took 804 us
// for the third, looking marked elements up 423, a bit each and no look-up this.  Their logits are fetched by themselves, and the
// wave that settles the row writes their gradients; the others write around them.
// What is beyond 256 KB of a row is read twice (512 x 200000 bf16 95 us; 116 with all of it read twice).
// Registers are bounded so that as many workgroups share a compute unit as the rows that they hold leave room for: unbounded,
// what settles a row took 96 and 136, the first 63 us, the second 49.
// (Rows one after the other by a workgroup that stays, the next row's loads beside the gradient's stores: 510 us for the third.)
template <typename T, uint32_t kThreads, uint32_t kHeld, bool kMore = false>
__global__ __launch_bounds__(kThreads, kHeld == 16 || kThreads == 1024 ? 4 : kHeld == 8 ? 6 : 8) void distill_rows_kernel(DistillArgs a)
{
  constexpr uint32_t N = 16 / sizeof(T), kWaves = kThreads / kWave;
  extern __shared__ uint64_t lds[];
  __shared__ float red_m[kWaves], red_s[kWaves];
  __shared__ RowGradient sh_gradient;
  __shared__ uint32_t sh_repeated;
  const uint32_t thread = threadIdx.x, lane = lane_id(), wave = thread / kWave, row = blockIdx.x;
  const uint32_t runs = a.V / N, left = a.V % N;  // whole runs; the elements behind them: one each
  const Named n = named_in(lds, a.K, a.V);
  const T *const z_row = static_cast<const T *>(a.logits) + row * a.row_stride;
  T *const out = a.grad ? static_cast<T *>(a.grad) + row * a.grad_stride : nullptr;
  // The named tokens first: loads come back in order, and their bits have to be there before the row is looked at.
  int32_t token = -1;
  float value = 0.0f;
  if (thread < a.K) {
    const uint64_t at = (uint64_t)row * a.K + thread;
    token = a.top_index[at];
    value = typed_element(a.top_value, a.value_dtype, at);
  }
  Run<T, N> held[kHeld];
  // (A row that is read once, past the caches too where no line is shared by two loads: 3001 x 131072 373 us through them, 364
  // past them; 777 rows that begin inside lines 33.9 and 39.2.)
  in_either_way(a.past_caches && a.whole_lines, [&](auto past) {
#pragma unroll
    for (uint32_t i = 0; i < kHeld; ++i) {
      const uint32_t run = thread + i * kThreads;
      if (run < runs) held[i] = fetch_run<decltype(past)::value, T, N>(z_row + run * N);
    }
  });
  float z_left = thread < left ? (float)z_row[runs * N + thread] : -__builtin_inff();
  for (uint32_t i = thread; i < (a.V + 63) / 64 * 2; i += kThreads) n.bits[i] = 0;
  if (thread == 0) sh_repeated = 0;
  lds_barrier();
  float z_named = 0.0f;
  if (thread < a.K) {
    if (enter_named(a, n, thread, token, value)) sh_repeated = 1;
    if (token >= 0 && (uint32_t)token < a.V) z_named = (float)z_row[token];  // on its way while the row is looked at
  }
  for (uint32_t k = thread + kThreads; k < a.K; k += kThreads) {
    const uint64_t at = (uint64_t)row * a.K + k;
    const int32_t other = a.top_index[at];
    if (enter_named(a, n, k, other, typed_element(a.top_value, a.value_dtype, at))) sh_repeated = 1;
    if (other >= 0 && (uint32_t)other < a.V) n.z[k] = (float)z_row[other];
  }
  lds_barrier();
  Teacher teacher;
  if (wave == 0) teacher = teach(a, n, row, sh_repeated);
  const bool left_named = thread < left && (n.bits[(runs * N + thread) / 32] >> (runs * N + thread) % 32 & 1);

  // the sum of this thread's part of the row, without the named tokens if there is a rest class
  Sum sum{-__builtin_inff(), 0.0f};
  Exponent x(sum.m, a.c);
  if (a.top_lse && left_named) z_left = -__builtin_inff();
  {
    float top = z_left;
#pragma unroll
    for (uint32_t i = 0; i < kHeld; ++i) {
      const uint32_t run = thread + i * kThreads;
      if (run >= runs) continue;
      const uint32_t named = a.top_lse ? n.mask<N>(run) : 0;
      if (named) {
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) held[i][e] = named >> e & 1 ? (T)-__builtin_inff() : (T)held[i][e];
      }
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) top = fmaxf(top, element<N, T>(held[i], e));
      hold_packed<N, T>(held[i]);
    }
    x = Exponent(top, a.c);
    float s = exp2_of(x.of(z_left));
#pragma unroll
    for (uint32_t i = 0; i < kHeld; ++i) {
      if (thread + i * kThreads >= runs) continue;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) s += exp2_of(x.of(element<N, T>(held[i], e)));
      hold_packed<N, T>(held[i]);
    }
    sum = Sum{top, s};
  }
  if (kMore) {
    uint32_t run = thread + kHeld * kThreads;
    Run<T, N> next{};
    if (run < runs) next = load_run<T, N>(z_row + run * N);
    for (; run < runs; run += kThreads) {  // the run behind it is on its way
      const Run<T, N> r = next;
      if (run + kThreads < runs) next = load_run<T, N>(z_row + (run + kThreads) * N);
      const uint32_t named = a.top_lse ? n.mask<N>(run) : 0;
      float z[N];
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) z[e] = named >> e & 1 ? -__builtin_inff() : element<N, T>(r, e);
      add_to<N>(sum, x, z, a.c);
    }
  }
  const float m = wave_max(sum.m), s = wave_sum(sum.m == -__builtin_inff() ? sum.s : sum.s * relative(sum.m, m, a.c));
  if (lane == 0) red_m[wave] = m, red_s[wave] = s;
  if (thread < a.K) n.z[thread] = z_named;
  lds_barrier();
  Settled settled;
  Sum all;
  if (wave == 0) {
    const float wm = lane < kWaves ? red_m[lane] : -__builtin_inff(), ws = lane < kWaves ? red_s[lane] : 0.0f;
    const float top = wave_max(wm);
    all = Sum{top, wave_sum(wm == -__builtin_inff() ? ws : ws * relative(wm, top, a.c))};
    settled = settle(a, n, row, teacher, all, out);
    if (lane == 0) sh_gradient = settled.gradient;
  }
  lds_barrier();
  if (wave == 0) conclude(a, row, teacher, all, settled);
  if (!out) return;
  const RowGradient g = sh_gradient;
  const float scale_low = g.scale * 0x1p-64f;
  const Exponent of_row(g.m, a.c);
  const auto gradient = [&](float z) { return power<T>(of_row.of(z), g.scale, scale_low); };
  // The named tokens' elements are the first wave's, all others of the row are written here.
  if (thread < left && !left_named) out[runs * N + thread] = (T)(g.zero ? 0.0f : gradient(z_left));
  const auto write = [&](uint32_t run, const Run<T, N> &z) {
    Run<T, N> r;
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) r[e] = (T)gradient(element<N, T>(z, e));
    if (g.zero) r = Run<T, N>{};
    const uint32_t named = n.mask<N>(run);
    if (!named) {
      store_run<T, N>(out + run * N, r, a.past_caches);
    } else {
#pragma unroll
      for (uint32_t e = 0; e < N; ++e)
        if (!(named >> e & 1)) out[run * N + e] = r[e];
    }
  };
#pragma unroll
  for (uint32_t i = 0; i < kHeld; ++i)
    if (thread + i * kThreads < runs) write(thread + i * kThreads, held[i]);
  if (kMore)
    for (uint32_t run = thread + kHeld * kThreads; run < runs; run += kThreads) write(run, load_run<T, N>(z_row + run * N));
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
  if (!((float)(1.4426950408889634 * inv_tau) < __builtin_inff())) return APEX_ERR_INVALID_ARG;
  constexpr uint32_t kLine = 128;
  const DistillArgs a{N, V, K, (uint32_t)value_dtype, row_stride, grad_stride, logits, top_index, top_value, top_lse, weight, inv_tau,
                      (float)(1.4426950408889634 * inv_tau), (float)inv_tau, loss, lse, grad,
                      grad && (uint64_t)N * V * size > kPastCachesBytes, (uintptr_t)logits % kLine == 0 && row_stride * size % kLine == 0};
  const uint32_t runs = V / (16 / size), lds = distill_lds(K, V);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  // As few threads as hold a row, for the registers of more rows on a compute unit; where the chip has a compute unit for every
  // row, as many as there are runs (12 x 32000 in 32 bits 10.4 us with 512 threads, 8.8 with 1024).
  with_type(dtype, [&](auto t) {
    typedef decltype(t) E;
    if (runs <= 256 * 4)
      distill_rows_kernel<E, 256, 4><<<N, 256, lds, stream>>>(a);
    else if (runs <= 1024 * 8 && N <= kChipCus)
      distill_rows_kernel<E, 1024, 8><<<N, 1024, lds, stream>>>(a);
    else if (runs <= 512 * 8)
      distill_rows_kernel<E, 512, 8><<<N, 512, lds, stream>>>(a);
    else if (runs <= 512 * 16)
      distill_rows_kernel<E, 512, 16><<<N, 512, lds, stream>>>(a);
    else if (runs <= 1024 * 16)
      distill_rows_kernel<E, 1024, 16><<<N, 1024, lds, stream>>>(a);
    else
      distill_rows_kernel<E, 1024, 16, true><<<N, 1024, lds, stream>>>(a);
  });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

}  // extern "C"
