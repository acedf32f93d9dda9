// Elements of 32 and 16 bits in runs that are aligned to the element only, and reductions over a wave, for the operators.
#pragma once
#include <type_traits>

#include "wave.hpp"

namespace apex {

// N neighbouring elements as one load or store.  The target takes global accesses of 16 bytes at any address, so that rows
// of odd lengths and strides need no path of their own.
template <typename T, int N>
struct RunOf {
  typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};
template <typename T>
struct RunOf<T, 1> {
  typedef T type;
};
template <typename T, int N>
using Run = typename RunOf<T, N>::type;

template <typename T, int N>
__device__ __forceinline__ Run<T, N> load_run(const T *p)
{
  return *reinterpret_cast<const Run<T, N> *>(p);
}

// Outputs beyond this size are stored past the caches: nobody finds them there afterwards, and the inputs of the workgroups to
// come lose their places to them (distillation of 777 x 49999 43.5 us through the caches, 33.9 past them, 2048 x 32768 62.6 and
// 57.7; scan of 1 x 32768 x 768 65.5 and 58.1).
constexpr uint64_t kPastCachesBytes = 32ull << 20;  // what the L2 caches of the chip hold

// f(integral_constant<bool>), the accesses of one way apart from those of the other: the comments in the assembly differ, on both
// sides, so that the compiler does not make one ordinary access of two.
template <typename F>
__device__ __forceinline__ void in_either_way(bool past_caches, F f)
{
  if (past_caches) {
    asm volatile("; past the caches");
    f(std::integral_constant<bool, true>());
    asm volatile("; past the caches");
  } else {
    asm volatile("; through the caches");
    f(std::integral_constant<bool, false>());
    asm volatile("; through the caches");
  }
}

template <typename T, int N>
__device__ __forceinline__ void store_run(T *p, const Run<T, N> &r, bool past_caches)
{
  in_either_way(past_caches, [&](auto past) {
    if (decltype(past)::value)
      __builtin_nontemporal_store(r, reinterpret_cast<Run<T, N> *>(p));
    else
      *reinterpret_cast<Run<T, N> *>(p) = r;
  });
}
template <bool kPast, typename T, int N>
__device__ __forceinline__ Run<T, N> fetch_run(const T *p)
{
  if (kPast) return __builtin_nontemporal_load(reinterpret_cast<const Run<T, N> *>(p));
  return load_run<T, N>(p);
}

template <int N, typename T>
__device__ __forceinline__ float element(const Run<T, N> &r, int i)
{
  if constexpr (N == 1)
    return (float)r;
  else
    return (float)r[i];
}

// Keeps a run of 16-bit elements as it is from here on: what they are in 32 bits, where it was needed before, is not held in
// registers until it is needed again.
template <int N, typename T>
__device__ __forceinline__ void hold_packed(Run<T, N> &r)
{
  if constexpr (sizeof(T) == 2 && N % 4 == 0) {
    struct Bits {
      uint64_t word[N / 4];
    } bits = __builtin_bit_cast(Bits, r);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) asm volatile("" : "+v"(bits.word[i]));
    r = __builtin_bit_cast(Run<T, N>, bits);
  }
}

// One step of a reduction with data-parallel primitives: a lane to which the control routes no value takes `none`.
template <int kCtrl, int kRowMask>
__device__ __forceinline__ float dpp_from(float v, float none)
{
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(none), (int)__float_as_uint(v), kCtrl, kRowMask,
                                                               0xf, false));
}

// f over the 64 lanes in a fixed order, the same in every lane.  `none` is f's neutral element.
template <typename F>
__device__ __forceinline__ float wave_reduce(float v, float none, F f)
{
  v = f(v, dpp_from<0x111, 0xf>(v, none));  // row_shr:1, the steps of wave_inclusive_scan
  v = f(v, dpp_from<0x112, 0xf>(v, none));
  v = f(v, dpp_from<0x114, 0xf>(v, none));
  v = f(v, dpp_from<0x118, 0xf>(v, none));
  v = f(v, dpp_from<0x142, 0xa>(v, none));
  v = f(v, dpp_from<0x143, 0xc>(v, none));
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), kWave - 1));
}
__device__ __forceinline__ float wave_sum(float v)
{
  return wave_reduce(v, 0.0f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v)
{
  return wave_reduce(v, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); });
}

__device__ __forceinline__ double wave_sum(double v)
{
  const auto step = [&](auto from) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __float_as_uint(from(__uint_as_float((uint32_t)bits))), hi = __float_as_uint(from(__uint_as_float((uint32_t)(bits >> 32))));
    v += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  step([](float x) { return dpp_from<0x111, 0xf>(x, 0.0f); });
  step([](float x) { return dpp_from<0x112, 0xf>(x, 0.0f); });
  step([](float x) { return dpp_from<0x114, 0xf>(x, 0.0f); });
  step([](float x) { return dpp_from<0x118, 0xf>(x, 0.0f); });
  step([](float x) { return dpp_from<0x142, 0xa>(x, 0.0f); });
  step([](float x) { return dpp_from<0x143, 0xc>(x, 0.0f); });
  const uint64_t bits = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)bits, kWave - 1);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(bits >> 32), kWave - 1);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// 2^x and log2 x as the hardware has them: within 1 ulp; results of 2^x below the normal range are 0.
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_of(float x) { return __builtin_amdgcn_logf(x); }

constexpr float kLog2e = 0x1.715476p+0f, kLn2 = 0x1.62e430p-1f;

}  // namespace apex
