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
  bool past_caches;  // h is stored past the caches
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
  bool past_caches;  // dg and dx are stored past the caches
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

// The step's factor, what is left beside it, and its term.
template <int kGate>
__device__ __forceinline__ void scan_gate(float g, float x, float *a, float *rest, float *b)
{
  if (kGate == APEX_GATE_SIGMOID) {
    sigmoid_pair(g, a, rest);
    *b = *rest * x;
  } else {
    *a = g;
    *rest = 1.0f;
    *b = x;
  }
}

// Gradients of g and x from lambda, the state that came in, and the step's own a and rest.
template <int kGate>
__device__ __forceinline__ void scan_gate_back(float a, float rest, float x, float prev, float lambda, float *dg, float *dx)
{
  if (kGate == APEX_GATE_SIGMOID) {
    *dg = lambda * (prev - x) * (a * rest);
    *dx = lambda * rest;
  } else {
    *dg = lambda * prev;
    *dx = lambda;
  }
}

// ---- tiles ----
//
// A tile is a stretch of steps of kTileWidth channels, held in the registers of one workgroup: a thread has kTileRun channels in
// kTileRows steps.  h -> A h + B composes: every thread composes its own steps, the compositions go through
// LDS (segments of kSegment groups of steps, then the segments), and with the state that enters the tile every thread goes through
// its steps once more.  Reads every input once.
//
// A sequence longer than a tile is a chain of tiles, whose states are handed on while they run: a tile publishes its
// composition as soon as it has it and goes back to the nearest place whose state is there.  However far it goes back, the
// operations on a state are the same, so the bits are.  Only words of 64 bits cross between workgroups, a number and a tag in
// one, written and read at agent scope.
// The tiles of a column of channels are taken by tickets, earlier ones first, so that whatever a tile waits for is held by a
// workgroup that runs, and the first one waits for nobody.  (A counter per column: atomics on one address take turns of some
// 14 ns.)
constexpr uint32_t kTileRows = 4, kTileRun = 4, kTileLanes = 32, kTileWidth = kTileLanes * kTileRun, kTileMaxThreads = 1024;
constexpr uint32_t kTileMaxSteps = kTileMaxThreads / kTileLanes * kTileRows;
constexpr uint32_t kChainThreads = 512, kChainSteps = kChainThreads / kTileLanes * kTileRows;  // of tiles in a chain
constexpr uint32_t kSegment = kTileWidth / kTileLanes;  // groups of a segment: as many segments as a tile has threads per channel

// Shared by all tiles of a call.  Zero before the first call; a call leaves the counters at 0 and moves epoch on, so that no
// word of an earlier call carries the tag of a later one, whatever its shape was.
constexpr uint32_t kScanCounters = 1024;
struct ScanCounter {
  uint32_t taken, done, pad[30];
};
struct ScanSpace {
  uint32_t epoch, done, pad[62];
  ScanCounter counter[kScanCounters];
  uint64_t word[1];  // [column][tile][3][kTileWidth]
};
constexpr size_t kScanSpaceHead = offsetof(ScanSpace, word);

// The tiles of a call: `columns` pieces of kTileWidth channels of a sequence, `tiles` tiles each.  Column c's tickets come from
// counter c mod groups.
struct Chain {
  ScanSpace *space;
  uint32_t columns, tiles, groups;
};

// The tile of a workgroup: where in its chain, and in which column.  By one thread.
__device__ __forceinline__ uint2 take_tile(const Chain &c)
{
  const uint32_t g = blockIdx.x % c.columns % c.groups, columns = (c.columns - g + c.groups - 1) / c.groups;  // of this counter
  const uint32_t n = __hip_atomic_fetch_add(&c.space->counter[g].taken, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_uint2(n / columns, g + c.groups * (n % columns));
}

// What is the same in every lane, in a scalar register.
__device__ __forceinline__ uint32_t one_for_all(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

__device__ __forceinline__ uint64_t tagged(float v, uint32_t tag) { return ((uint64_t)tag << 32) | __float_as_uint(v); }
__device__ __forceinline__ void publish(uint64_t *word, uint64_t v)
{
  __hip_atomic_store(word, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t seen(const uint64_t *word)
{
  return __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

constexpr uint32_t kCutTag = 0x80000000u;  // of a composition: the state that enters does not get through
__device__ __forceinline__ uint32_t next_tag(uint32_t epoch)  // never that of memory filled with zeros
{
  const uint32_t tag = (epoch + 1) & ~kCutTag;
  return tag ? tag : 1;
}
constexpr uint32_t kMostTiles = 1u << 22;  // of a chain: its words are counted in 32 bits
constexpr uint32_t kMostPolls = 1u << 20;  // a wait gives up (and hands on NaN) where a word never comes: the workspace was not zero

constexpr uint32_t kStretch = 4;  // tiles of a stretch
constexpr uint32_t kWindow = 8;   // compositions that a workgroup fetches at once

__device__ __forceinline__ bool carries(uint64_t word, uint32_t tag) { return ((uint32_t)(word >> 32) & ~kCutTag) == tag; }
__device__ __forceinline__ float number(uint64_t word) { return __uint_as_float((uint32_t)word); }
// The word once it carries the tag (w: what it was just now); NaN if it never does.
__device__ __forceinline__ uint64_t waited_for(uint64_t w, const uint64_t *word, uint32_t tag)
{
  for (uint32_t polls = 0; !carries(w, tag); w = seen(word))
    if (++polls == kMostPolls) return tagged(__builtin_nanf(""), tag);
  return w;
}

// Compositions fetched by a workgroup, in LDS.
template <uint32_t kCount>
struct Fetched {
  float a[kCount][kTileWidth], b[kCount][kTileWidth];
  uint32_t cut[kCount];

  // `count` compositions at word + offset(i, 0), + offset(i, 1); by all threads, behind a barrier and before the next.
  template <typename F>
  __device__ __forceinline__ void fetch(const uint64_t *word, uint32_t count, bool is, uint32_t tag, F offset)
  {
    constexpr uint32_t kSlots = kChainThreads / kTileWidth, kEach = (kCount + kSlots - 1) / kSlots;
    const uint32_t channel = threadIdx.x % kTileWidth, slot = threadIdx.x / kTileWidth;
    uint64_t wa[kEach], wb[kEach];
#pragma unroll
    for (uint32_t u = 0; u < kEach; ++u) {
      const uint32_t i = slot + u * kSlots;
      if (i < count && is) wa[u] = seen(word + (offset(i, 0) + channel)), wb[u] = seen(word + (offset(i, 1) + channel));
    }
#pragma unroll
    for (uint32_t u = 0; u < kEach; ++u) {
      const uint32_t i = slot + u * kSlots;
      if (i < count && is) {
        wa[u] = waited_for(wa[u], word + (offset(i, 0) + channel), tag);
        wb[u] = waited_for(wb[u], word + (offset(i, 1) + channel), tag);
        a[i][channel] = number(wa[u]);
        b[i][channel] = number(wb[u]);
        if (channel == 0) cut[i] = (uint32_t)(wa[u] >> 32) & kCutTag;
      }
    }
  }
  __device__ __forceinline__ float through(uint32_t i, uint32_t channel, float state) const
  {
    return cut[i] ? b[i][channel] : __builtin_fmaf(a[i][channel], state, b[i][channel]);
  }
};

struct ChainSpace {
  Fetched<kStretch - 1> tiles;
  Fetched<kWindow> stretches;
  uint32_t nearest;
};

// The state that enters the tile at position q of a chain, for thread < kTileWidth and its channel (`is`: there is one), from
// the composition (A, B) of the tile (`cut`: B is its outgoing state whatever enters) and the state that enters the chain.  By
// the whole workgroup.  Publishes what the tiles behind ask for, unless the tile has no composition (`composed`): then what comes out
// of it is said by hand_on, once it is known.
//
// kStretch tiles are a stretch: a tile publishes its composition, the last one of a stretch the stretch's and the state behind
// it.  A tile goes back to the nearest stretch whose state is there (the first wave looks at 64 at once), through the
// compositions of the stretches from there on, and through those of the tiles of its own stretch before it, which all threads
// fetch, up to kWindow with one round trip.  (Without stretches, from tile to tile, by the threads that have a channel: 1 x
// 32768 x 768 109 us, where a state comes past 64 tiles at a time.  Stretches of 8: gradient of 4 x 8192 x 2048 208 us, 200 of 4.)
// Words of position p: word + p * 3 * kTileWidth: A, B, and a third row that the last three tiles of a stretch lend to the
// stretch: its A, its B, and the state behind it.
__device__ __forceinline__ float chain_state(uint64_t *word, uint32_t q, bool is, float A, float B, bool cut, float start, uint32_t tag,
                                             ChainSpace &w, bool composed)
{
  const uint32_t thread = threadIdx.x, channel = thread % kTileWidth, stretch = q / kStretch, place = q % kStretch;
  const bool speaks = thread < kTileWidth && is;
  const auto row = [&](uint32_t position, uint32_t i) { return (position * 3 + i) * kTileWidth; };  // (kMostTiles)
  const auto stretch_row = [&](uint32_t k, uint32_t i) { return row(k * kStretch + kStretch - 3 + i, 2); };
  const auto say = [&](uint32_t at, uint64_t v) { publish(word + (at + channel), v); };
  if (speaks && composed && place < kStretch - 1) {
    say(row(q, 0), tagged(A, cut ? tag | kCutTag : tag));
    say(row(q, 1), tagged(B, tag));
  }
  if (q == 0) return start;
  w.tiles.fetch(word, place, is, tag, [&](uint32_t i, uint32_t r) { return row(q - place + i, r); });
  if (thread >= kChainThreads - kWave && stretch > 0) {
    const uint32_t lane = lane_id(), reach = min(stretch, (uint32_t)kWave);
    uint64_t there = 0;
    for (uint32_t polls = 0; polls < kMostPolls; ++polls) {
      const uint64_t v = lane < reach ? seen(word + stretch_row(stretch - 1 - lane, 2)) : 0;
      there = __ballot(lane < reach && carries(v, tag));
      if (there) break;
      __builtin_amdgcn_s_sleep(1);
    }
    if (lane == 0) w.nearest = there ? (uint32_t)__builtin_ctzll(there) : 0;
  }
  __syncthreads();
  float SA = 1.0f, SB = 0.0f;
  bool stretch_cut = cut;
  const bool last = place == kStretch - 1 && composed;
  if (last && thread < kTileWidth) {
    for (uint32_t i = 0; i < kStretch - 1; ++i) {
      stretch_cut = stretch_cut || w.tiles.cut[i];
      SB = w.tiles.through(i, channel, SB);
      SA *= w.tiles.a[i][channel];
    }
    SB = cut ? B : __builtin_fmaf(A, SB, B);
    SA = A * SA;
    if (is) {
      say(stretch_row(stretch, 0), tagged(SA, stretch_cut ? tag | kCutTag : tag));
      say(stretch_row(stretch, 1), tagged(SB, tag));
      if (stretch_cut) say(stretch_row(stretch, 2), tagged(SB, tag));
    }
  }
  float state = start;
  if (stretch > 0) {
    const uint32_t nearest = w.nearest;
    const uint64_t *const from = word + (stretch_row(stretch - 1 - nearest, 2) + channel);
    uint64_t v = 0;
    if (speaks) v = seen(from);
    for (uint32_t left = nearest; left > 0;) {
      const uint32_t count = min(left, kWindow), first = stretch - left;
      w.stretches.fetch(word, count, is, tag, [&](uint32_t i, uint32_t r) { return stretch_row(first + i, r); });
      if (left == nearest && speaks) state = number(waited_for(v, from, tag));
      __syncthreads();
      if (thread < kTileWidth)
        for (uint32_t i = 0; i < count; ++i) state = w.stretches.through(i, channel, state);
      left -= count;
      if (left) __syncthreads();
    }
    if (nearest == 0 && speaks) state = number(waited_for(v, from, tag));
  }
  if (speaks && last && !stretch_cut) say(stretch_row(stretch, 2), tagged(__builtin_fmaf(SA, state, SB), tag));
  if (thread < kTileWidth)
    for (uint32_t i = 0; i < place; ++i) state = w.tiles.through(i, channel, state);
  return state;
}

// The state behind a tile that has no composition, by the threads that speak for a channel: to those that ask it is a composition
// with a cut.
__device__ __forceinline__ void hand_on(uint64_t *word, uint32_t q, float state, uint32_t tag)
{
  const uint32_t channel = threadIdx.x % kTileWidth, place = q % kStretch, first = q - place;
  if (place < kStretch - 1) {
    publish(word + ((q * 3 + 0) * kTileWidth + channel), tagged(0.0f, tag | kCutTag));
    publish(word + ((q * 3 + 1) * kTileWidth + channel), tagged(state, tag));
  } else {
    for (uint32_t i = 0; i < 3; ++i)
      publish(word + (((first + kStretch - 3 + i) * 3 + 2) * kTileWidth + channel), i == 0 ? tagged(0.0f, tag | kCutTag) : tagged(state, tag));
  }
}

// How far given factors above 1 may multiply up over a tile, in powers of 2, as kGrowthUnit-ths: four tiles make a stretch, whose
// product has to be a number.  (A product that falls below the numbers is 0: what is lost of a state is 2^-149 of it, and 2^30
// times that where it grows again.)  Beyond, an overflow could meet a state of 0, or come back within range: such a tile has no
// composition.  It waits for the state that enters it and goes from step to step, some 7 us a tile.  (64 steps of 1.38 are within
// the bound.  4 x 8192 x 2048 bf16 112 us forward, 854 with tiles that all go from step to step; 1 x 32768 x 768 54 and 3850.)
constexpr uint32_t kGrowthUnit = 16, kMostGrowth = 30 * kGrowthUnit;

// Adds a wave's part to the tile's.
template <uint32_t N>
__device__ __forceinline__ void add_growth(const float (&f)[kTileRows][N], uint32_t *growth)
{
  float most = 0.0f;
#pragma unroll
  for (uint32_t l = 0; l < kTileRows; ++l)
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) most = fmaxf(most, __builtin_fabsf(f[l][e]));
  if (__ballot(most > 1.0f) == 0) return;
  most = 1.0f;
#pragma unroll
  for (uint32_t e = 0; e < N; ++e) {
    float product = 1.0f;
#pragma unroll
    for (uint32_t l = 0; l < kTileRows; ++l) product *= fmaxf(__builtin_fabsf(f[l][e]), 1.0f);
    most = fmaxf(most, product);
  }
  most = fminf(wave_max(most), 0x1p126f);
  constexpr uint32_t kGroups = kWave / kTileLanes;
  if (lane_id() == 0) atomicAdd(growth, kGroups * ((uint32_t)(log2_of(most) * kGrowthUnit) + 1));
}

// Where h_last is h0, nothing of the chain orders the tiles that read h0, those of the first stretch, before the one that
// writes h_last: a stretch with a cut in it hands its state on before anything in front of it is there.  So they say that they have
// read it, in words of position 0 that nothing else uses, and the writer waits for that.
__device__ __forceinline__ uint64_t *start_read(const Chain &c, uint32_t column, uint32_t tile)
{
  return c.space->word + ((uint64_t)column * c.tiles * 3 + 2) * kTileWidth + tile;
}
static_assert(kStretch == 4);  // position 0 lends its third row to nobody: chain_state

// A workgroup that waits for nothing any more: the last one of a counter, and of them the last of the call, leave the counters as
// the next call has to find them.  By one thread; leaving() is the round trip, left() looks at what it brought.
__device__ __forceinline__ uint32_t leaving(const Chain &c)
{
  return __hip_atomic_fetch_add(&c.space->counter[blockIdx.x % c.columns % c.groups].done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void left(const Chain &c, uint32_t before, uint32_t tag)
{
  const uint32_t g = blockIdx.x % c.columns % c.groups, columns = (c.columns - g + c.groups - 1) / c.groups;
  if (before != columns * c.tiles - 1) return;
  ScanCounter *const counter = c.space->counter + g;
  __hip_atomic_store(&counter->taken, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(&counter->done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (__hip_atomic_fetch_add(&c.space->done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != c.groups - 1) return;
  __hip_atomic_store(&c.space->done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(&c.space->epoch, tag, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Bits of a tile's rows, in LDS.
struct RowBits {
  uint64_t word[kTileMaxSteps / kWave];
  __device__ __forceinline__ uint32_t of_group(uint32_t g) const { return (uint32_t)(word[g / 16] >> (g % 16 * 4)) & 15u; }
  __device__ __forceinline__ bool all_of_segment(uint32_t i) const { return (uint16_t)(word[i / 4] >> (i % 4 * 16)) == 0xffffu; }
};

// Elements [d, d + N) of a row, 0 beyond D.
template <typename T, int N>
__device__ __forceinline__ Run<T, N> run_of(const T *row, uint32_t d, uint32_t D)
{
  if (d + N <= D) return load_run<T, N>(row + d);
  Run<T, N> r;
#pragma unroll
  for (int e = 0; e < N; ++e) r[e] = d + e < D ? row[d + e] : (T)0.0f;
  return r;
}
template <typename T, int N>
__device__ __forceinline__ void store_run_of(T *row, uint32_t d, uint32_t D, const Run<T, N> &r)
{
  if (d + N <= D) {
    *reinterpret_cast<Run<T, N> *>(row + d) = r;
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (d + e < D) row[d + e] = r[e];
  }
}

constexpr uint32_t tile_lds(uint32_t threads)  // bytes: compositions of the groups, of the segments, states that enter segments
{
  return threads * kTileRun * 8 + threads * 12;
}

// What a workgroup's threads are to its tile.
struct TileShape {
  uint32_t threads, thread, groups, segments, steps;
  uint32_t group, run;        // a thread's steps and channels ...
  uint32_t segment, channel;  // ... and what it does when the compositions are gone through
  __device__ __forceinline__ TileShape()
  {
    threads = blockDim.x, thread = threadIdx.x;
    groups = threads / kTileLanes, segments = threads / kTileWidth, steps = groups * kTileRows;
    group = thread / kTileLanes, run = thread % kTileLanes * kTileRun;
    segment = thread / kTileWidth, channel = thread % kTileWidth;
  }
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
static_assert(kTileRun == 4);

// Whether every row of the tile passes on; behind the barrier that the bits were written before.
__device__ __forceinline__ bool uncut(const RowBits &bits, uint32_t steps)
{
  uint64_t missing = 0;
  for (uint32_t i = 0; i * kWave < steps; ++i)
    missing |= ~bits.word[i] & (steps - i * kWave >= kWave ? ~0ull : (1ull << (steps - i * kWave)) - 1);
  return missing == 0;
}

// f(integral_constant<bool>): tiles in which every row passes on apart, without the branches that would keep the rows' gates
// from running side by side.  Not where a call is one tile deep: twice the code to fetch cost more there (64 x 96 x 1024 13.8 us
// with, 11.4 without).
template <bool kApart, typename F>
__device__ __forceinline__ void plainly(bool plain, F f)
{
  if (kApart && plain)
    f(std::integral_constant<bool, true>());
  else
    f(std::integral_constant<bool, false>());
}

// What stands for a step that a sequence does not have: one that leaves a state as it is, a = 1, b = 0.
template <typename T, int kGate, int N>
__device__ __forceinline__ void no_step(Run<T, N> *g, Run<T, N> *x)
{
#pragma unroll
  for (int e = 0; e < N; ++e) (*g)[e] = (T)(kGate == APEX_GATE_SIGMOID ? __builtin_inff() : 1.0f), (*x)[e] = (T)0.0f;
}

// kChained: tiles of a sequence wait for one another; else a sequence has one tile.
// Chained bound by memory and by waits for states: 4 x 8192 x 2048 bf16 125 us for 403 MB (3.2 TB/s), 101 without the waits; one
// prompt of 32768 x 768 61 and 38.  Else by loads, gates, barriers and stores one after the other, of one round of workgroups: 64 x
// 96 x 1024 bf16 12 us.
template <typename T, int kGate, bool kChained>
__global__ __launch_bounds__(kChained ? kChainThreads : kTileMaxThreads, kChained ? 6 : 4) void scan_tile_kernel(ScanArgs a, Chain chain)
{
  constexpr uint32_t N = kTileRun, kWidth = kTileWidth;
  extern __shared__ __align__(16) float scan_lds[];
  __shared__ RowBits into;  // whether the state passes into a row
  __shared__ uint2 sh_tile;
  __shared__ uint32_t sh_growth;
  __shared__ typename std::conditional<kChained, ChainSpace, uint32_t>::type sh_chain;
  const TileShape w;
  float *const group_a = scan_lds, *const group_b = group_a + w.groups * kWidth;  // [groups][kWidth]; group_a later: the state that enters
  float *const segment_a = group_b + w.groups * kWidth, *const segment_b = segment_a + w.threads;  // [segments][kWidth]
  float *const segment_in = segment_b + w.threads;
  const uint32_t pieces = (a.D + kWidth - 1) / kWidth;  // of a row
  const uint32_t chunks = (a.T + APEX_SCAN_CHUNK - 1) / APEX_SCAN_CHUNK;
  uint32_t tag = 0, tile = 0, column = blockIdx.x;
  if (kChained) {
    tag = next_tag(chain.space->epoch);
    if (w.thread == 0) sh_tile = take_tile(chain);
    __syncthreads();
    tile = one_for_all(sh_tile.x), column = one_for_all(sh_tile.y);
    if (tile >= chain.tiles) return;  // no ticket of this call: the counters were not zero
  }
  const uint32_t s = column / pieces, d0 = column % pieces * kWidth, t0 = tile * w.steps;
  const uint32_t len = scan_length(a.length, s, a.T);
  const uint32_t t_group = t0 + w.group * kTileRows, d = d0 + w.run;
  const bool exists = d < a.D, whole = t0 + w.steps <= len && d0 + kWidth <= a.D;
  if (t0 >= len) {  // nothing but what a sequence's end leaves
    T *const h = static_cast<T *>(a.h) + ((uint64_t)s * a.T + t_group) * a.D;
    for (uint32_t l = 0; l < kTileRows; ++l)
      if (exists && t_group + l < a.T) store_run_of<T, N>(h + (uint64_t)l * a.D, d, a.D, Run<T, N>{});
    if (tile == 0 && a.h_last && w.thread < kWidth && d0 + w.channel < a.D) {
      const uint64_t at = (uint64_t)s * a.D + d0 + w.channel;
      a.h_last[at] = a.h0 ? a.h0[at] : 0.0f;
    }
    if (kChained && w.thread == w.threads - 1) left(chain, leaving(chain), tag);
    return;
  }
  // the rows of this thread
  Run<T, N> gr[kTileRows], xr[kTileRows];
  {
    const T *const g = static_cast<const T *>(a.g) + s * a.g_seq + t_group * a.g_time;
    const T *const x = static_cast<const T *>(a.x) + s * a.x_seq + t_group * a.x_time;
    if (whole) {
#pragma unroll
      for (uint32_t l = 0; l < kTileRows; ++l) gr[l] = load_run<T, N>(g + l * a.g_time + d), xr[l] = load_run<T, N>(x + l * a.x_time + d);
    } else {
#pragma unroll
      for (uint32_t l = 0; l < kTileRows; ++l)
        if (exists && t_group + l < len)
          gr[l] = run_of<T, N>(g + l * a.g_time, d, a.D), xr[l] = run_of<T, N>(x + l * a.x_time, d, a.D);
        else
          no_step<T, kGate, N>(&gr[l], &xr[l]);
    }
  }
  if (w.thread < w.steps) {
    const uint32_t t = t0 + w.thread;
    const uint64_t bits = __ballot(!a.discount || t == 0 || t >= len || a.discount[(uint64_t)s * a.T + t - 1] != 0.0f);
    if (lane_id() == 0) into.word[w.thread / kWave] = bits;
  }
  if (kGate == APEX_GATE_GIVEN && w.thread == 0) sh_growth = 0;
  __syncthreads();
  const uint32_t bits = into.of_group(w.group);
  const bool no_cut = uncut(into, w.steps);
  float fa[kTileRows][N], fb[kTileRows][N];
  plainly<kChained>(no_cut, [&](auto is_plain) {
    constexpr bool kPlain = decltype(is_plain)::value;
    f32x4 A, B;
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) A[e] = 1.0f, B[e] = 0.0f;
#pragma unroll
    for (uint32_t l = 0; l < kTileRows; ++l) {
      if (!kPlain && !(bits >> l & 1)) A = B = f32x4{};
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        float rest;
        scan_gate<kGate>(element<N, T>(gr[l], e), element<N, T>(xr[l], e), &fa[l][e], &rest, &fb[l][e]);
        A[e] *= fa[l][e];
        B[e] = __builtin_fmaf(fa[l][e], B[e], fb[l][e]);
      }
    }
    *reinterpret_cast<f32x4 *>(group_a + w.group * kWidth + w.run) = A;
    *reinterpret_cast<f32x4 *>(group_b + w.group * kWidth + w.run) = B;
  });
  if (kGate == APEX_GATE_GIVEN) add_growth(fa, &sh_growth);
  __syncthreads();
  const bool composed = kGate != APEX_GATE_GIVEN || sh_growth <= kMostGrowth;
  if (w.segments > 1) {
    float A = 1.0f, B = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < kSegment; ++i) {
      const uint32_t at = (w.segment * kSegment + i) * kWidth + w.channel;
      const float ga = group_a[at], gb = group_b[at];
      const bool passes = no_cut || into.of_group(w.segment * kSegment + i) == 15u;
      A = passes ? A * ga : 0.0f;
      B = passes ? __builtin_fmaf(ga, B, gb) : gb;
    }
    segment_a[w.thread] = A;
    segment_b[w.thread] = B;
    __syncthreads();
  }
  const bool speaks = w.thread < kWidth && d0 + w.channel < a.D;
  float state_in = 0.0f;  // what enters the chain; then what enters the tile
  if (speaks && a.h0 && tile < kStretch) state_in = a.h0[(uint64_t)s * a.D + d0 + w.channel];
  const bool in_place = a.h0 && a.h0 == a.h_last;
  if constexpr (kChained) {
    if (__builtin_expect(in_place, false)) {
      if (tile < kStretch) asm volatile("s_waitcnt vmcnt(0)" : "+v"(state_in) : : "memory");  // it is here, not on its way
      if (len - t0 <= w.steps && w.thread < min(tile, kStretch)) waited_for(0, start_read(chain, column, w.thread), tag);
    }
    float A = 1.0f, B = 0.0f;
    if (w.thread < kWidth)
      for (uint32_t i = 0; i < w.segments; ++i) {
        const float sa = segment_a[i * kWidth + w.channel], sb = segment_b[i * kWidth + w.channel];
        const bool passes = into.all_of_segment(i);
        A = passes ? A * sa : 0.0f;
        B = passes ? __builtin_fmaf(sa, B, sb) : sb;
      }
    state_in = chain_state(chain.space->word + (uint64_t)column * chain.tiles * 3 * kWidth, tile, d0 + w.channel < a.D, A, B, !no_cut,
                           state_in, tag, sh_chain, composed);
  }
  if (!composed) {
    if (w.thread < kWidth) {
      const uint64_t at = d0 + min(w.channel, a.D - 1 - d0);
      const T *const g = static_cast<const T *>(a.g) + s * a.g_seq + t0 * a.g_time + at;
      const T *const x = static_cast<const T *>(a.x) + s * a.x_seq + t0 * a.x_time + at;
      const uint32_t steps = min(len - t0, w.steps);
      for (uint32_t i = 0; i < w.groups; ++i) {
        group_a[i * kWidth + w.channel] = state_in;
        float gt[kTileRows], xt[kTileRows];
#pragma unroll
        for (uint32_t l = 0; l < kTileRows; ++l) {
          const uint32_t t = min(i * kTileRows + l, steps - 1);
          gt[l] = (float)g[t * a.g_time], xt[l] = (float)x[t * a.x_time];
        }
#pragma unroll
        for (uint32_t l = 0; l < kTileRows; ++l)
          if (i * kTileRows + l < steps) state_in = __builtin_fmaf(gt[l], into.of_group(i) >> l & 1 ? state_in : 0.0f, xt[l]);
      }
      if (kChained && speaks) hand_on(chain.space->word + (uint64_t)column * chain.tiles * 3 * kWidth, tile, state_in, tag);
    }
  } else if (w.thread < kWidth) {
    segment_in[w.channel] = state_in;
    for (uint32_t i = 0; i + 1 < w.segments; ++i) {
      const float sa = segment_a[i * kWidth + w.channel], sb = segment_b[i * kWidth + w.channel];
      state_in = into.all_of_segment(i) ? __builtin_fmaf(sa, state_in, sb) : sb;
      segment_in[(i + 1) * kWidth + w.channel] = state_in;
    }
  }
  __syncthreads();
  uint32_t before = 0;
  if constexpr (kChained) {
    if (__builtin_expect(in_place && tile < kStretch, false) && w.thread == 0) publish(start_read(chain, column, tile), tagged(0.0f, tag));
    if (w.thread == w.threads - 1) before = leaving(chain);
  }
  if (composed) {
    float state = segment_in[w.thread];
#pragma unroll
    for (uint32_t i = 0; i < kSegment; ++i) {
      const uint32_t at = (w.segment * kSegment + i) * kWidth + w.channel;
      const float ga = group_a[at], gb = group_b[at];
      group_a[at] = state;
      state = no_cut || into.of_group(w.segment * kSegment + i) == 15u ? __builtin_fmaf(ga, state, gb) : gb;
    }
  }
  __syncthreads();
  if (exists) {
    f32x4 state = *reinterpret_cast<const f32x4 *>(group_a + w.group * kWidth + w.run);
    if (a.carry && t_group % APEX_SCAN_CHUNK == 0 && t_group < len) {
      float *const c = a.carry + ((uint64_t)s * chunks + t_group / APEX_SCAN_CHUNK) * a.D;
      f32x4 r;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) r[e] = bits & 1 ? state[e] : 0.0f;
      store_run_of<float, N>(c, d, a.D, r);
    }
    T *const h = static_cast<T *>(a.h) + ((uint64_t)s * a.T + t_group) * a.D;
    plainly<kChained>(no_cut, [&](auto is_plain) {
      constexpr bool kPlain = decltype(is_plain)::value;
#pragma unroll
      for (uint32_t l = 0; l < kTileRows; ++l) {
        const uint32_t t = t_group + l;
        if (!kPlain && !(bits >> l & 1)) state = f32x4{};
        Run<T, N> r;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) {
          state[e] = __builtin_fmaf(fa[l][e], state[e], fb[l][e]);
          r[e] = (T)state[e];
        }
        T *const to = h + (uint64_t)l * a.D;
        if (whole) {
          store_run<T, N>(to + d, r, a.past_caches);
        } else if (t < a.T) {
          if (t >= len) r = Run<T, N>{};
          store_run_of<T, N>(to, d, a.D, r);
        }
        if (a.h_last && t + 1 == len) {
          const bool on = !a.discount || a.discount[(uint64_t)s * a.T + t] != 0.0f;
          store_run_of<float, N>(a.h_last + (uint64_t)s * a.D, d, a.D, on ? state : f32x4{});
        }
      }
    });
  }
  if (kChained && w.thread == w.threads - 1) left(chain, before, tag);
}

// The gradient in tiles: the states from `carry`, which begins anew every APEX_SCAN_CHUNK steps, and lambda by a chain from the
// last step to the first.  A row's bit says whether its state passes on; the rows of a chunk take each other's, and what enters
// a chunk's first row has been through its bit already.
// Bound as the forward pass is: 4 x 8192 x 2048 bf16 193 us for 671 MB (3.5 TB/s), 179 without the waits; 64 x 96 x 1024 18 us.  In
// fp32, 2 x 8192 x 2048, 140 us for as much (4.8), 97 forward.
constexpr uint32_t tile_back_lds(uint32_t threads)  // both kinds of compositions of the groups, segments' compositions, what enters
{
  return threads * kTileRun * 16 + threads * 12;
}

template <typename T, int kGate, bool kChained>
__global__ __launch_bounds__(kChained ? kChainThreads : kTileMaxThreads, kChained || sizeof(T) == 4 ? 4 : 6) void scan_tile_back_kernel(ScanBackArgs a, Chain chain)
{
  constexpr uint32_t N = kTileRun, kWidth = kTileWidth;
  constexpr uint32_t kChunkGroups = APEX_SCAN_CHUNK / kTileRows, kChunkSegments = kChunkGroups / kSegment;
  static_assert(APEX_SCAN_CHUNK == kWave);  // a word of RowBits is a chunk
  extern __shared__ __align__(16) float scan_lds[];
  __shared__ RowBits on;  // whether a row's state passes on
  __shared__ uint2 sh_tile;
  __shared__ uint32_t sh_growth;
  __shared__ typename std::conditional<kChained, ChainSpace, uint32_t>::type sh_chain;
  const TileShape w;
  float *const group_a = scan_lds, *const group_b = group_a + w.groups * kWidth;                 // [groups][kWidth]; group_a later: the state that enters
  float *const group_p = group_b + w.groups * kWidth, *const group_q = group_p + w.groups * kWidth;  // group_p: the gradient that enters
  float *const segment_p = group_q + w.groups * kWidth, *const segment_q = segment_p + w.threads;    // [segments][kWidth]
  float *const segment_in = segment_q + w.threads;
  const uint32_t pieces = (a.D + kWidth - 1) / kWidth;
  const uint32_t chunks = (a.T + APEX_SCAN_CHUNK - 1) / APEX_SCAN_CHUNK;
  uint32_t tag = 0, tile = 0, column = blockIdx.x;
  if (kChained) {
    tag = next_tag(chain.space->epoch);
    if (w.thread == 0) sh_tile = take_tile(chain);
    __syncthreads();
    tile = one_for_all(sh_tile.x), column = one_for_all(sh_tile.y);
    if (tile >= chain.tiles) return;  // no ticket of this call: the counters were not zero
    tile = chain.tiles - 1 - tile;
  }
  const uint32_t s = column / pieces, d0 = column % pieces * kWidth, t0 = tile * w.steps;
  const uint32_t len = scan_length(a.length, s, a.T);
  const uint32_t t_group = t0 + w.group * kTileRows, d = d0 + w.run;
  const bool exists = d < a.D, whole = t0 + w.steps <= len && d0 + kWidth <= a.D;
  if (t0 >= len) {
    T *const dg = static_cast<T *>(a.dg) + s * a.dg_seq + t_group * a.dg_time;
    T *const dx = static_cast<T *>(a.dx) + s * a.dx_seq + t_group * a.dx_time;
    for (uint32_t l = 0; l < kTileRows; ++l)
      if (exists && t_group + l < a.T) {
        store_run_of<T, N>(dg + l * a.dg_time, d, a.D, Run<T, N>{});
        store_run_of<T, N>(dx + l * a.dx_time, d, a.D, Run<T, N>{});
      }
    if (tile == 0 && a.dh0 && w.thread < kWidth && d0 + w.channel < a.D) {
      const uint64_t at = (uint64_t)s * a.D + d0 + w.channel;
      a.dh0[at] = a.dh_last ? a.dh_last[at] : 0.0f;
    }
    if (kChained && w.thread == w.threads - 1) left(chain, leaving(chain), tag);
    return;
  }
  Run<T, N> gr[kTileRows], xr[kTileRows], hr[kTileRows];
  {
    const T *const g = static_cast<const T *>(a.g) + s * a.g_seq + t_group * a.g_time;
    const T *const x = static_cast<const T *>(a.x) + s * a.x_seq + t_group * a.x_time;
    const T *const dh = static_cast<const T *>(a.dh) + ((uint64_t)s * a.T + t_group) * a.D;
    if (whole) {
#pragma unroll
      for (uint32_t l = 0; l < kTileRows; ++l) {
        gr[l] = load_run<T, N>(g + l * a.g_time + d);
        xr[l] = load_run<T, N>(x + l * a.x_time + d);
        hr[l] = load_run<T, N>(dh + (uint64_t)l * a.D + d);
      }
    } else {
#pragma unroll
      for (uint32_t l = 0; l < kTileRows; ++l)
        if (exists && t_group + l < len) {
          gr[l] = run_of<T, N>(g + l * a.g_time, d, a.D);
          xr[l] = run_of<T, N>(x + l * a.x_time, d, a.D);
          hr[l] = run_of<T, N>(dh + (uint64_t)l * a.D, d, a.D);
        } else {
          no_step<T, kGate, N>(&gr[l], &xr[l]);
          hr[l] = Run<T, N>{};
        }
    }
  }
  // the state that enters the chunk of this thread's segment
  const bool is = d0 + w.channel < a.D, speaks = w.thread < kWidth && is;
  const uint32_t chunk = t0 / APEX_SCAN_CHUNK + w.segment / kChunkSegments;
  float state = 0.0f;
  if (is && chunk * APEX_SCAN_CHUNK < len) state = a.carry[((uint64_t)s * chunks + chunk) * a.D + d0 + w.channel];
  if (w.thread < w.steps) {
    const uint32_t t = t0 + w.thread;
    const uint64_t bits = __ballot(!a.discount || t >= len || a.discount[(uint64_t)s * a.T + t] != 0.0f);
    if (lane_id() == 0) on.word[w.thread / kWave] = bits;
  }
  if (kGate == APEX_GATE_GIVEN && w.thread == 0) sh_growth = 0;
  __syncthreads();
  const uint32_t bits = on.of_group(w.group);
  const bool no_cut = uncut(on, w.steps);
  const uint32_t into = (uint32_t)((on.word[w.group / kChunkGroups] << 1 | 1) >> (w.group % kChunkGroups * kTileRows)) & 15u;
  float f[kTileRows][N], rest[kTileRows][N];
  plainly<kChained>(no_cut, [&](auto is_plain) {
    constexpr bool kPlain = decltype(is_plain)::value;
    f32x4 A, B, P, Q;
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) A[e] = P[e] = 1.0f, B[e] = Q[e] = 0.0f;
#pragma unroll
    for (uint32_t l = 0; l < kTileRows; ++l) {
      if (!kPlain && !(into >> l & 1)) A = B = f32x4{};
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        float b;
        scan_gate<kGate>(element<N, T>(gr[l], e), element<N, T>(xr[l], e), &f[l][e], &rest[l][e], &b);
        A[e] *= f[l][e];
        B[e] = __builtin_fmaf(f[l][e], B[e], b);
      }
    }
#pragma unroll
    for (uint32_t l = kTileRows; l-- > 0;) {
      if (!kPlain && !(bits >> l & 1)) P = Q = f32x4{};
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        P[e] *= f[l][e];
        Q[e] = f[l][e] * (Q[e] + element<N, T>(hr[l], e));
      }
    }
    const uint32_t at = w.group * kWidth + w.run;
    *reinterpret_cast<f32x4 *>(group_a + at) = A;
    *reinterpret_cast<f32x4 *>(group_b + at) = B;
    *reinterpret_cast<f32x4 *>(group_p + at) = P;
    *reinterpret_cast<f32x4 *>(group_q + at) = Q;
  });
  if (kGate == APEX_GATE_GIVEN) add_growth(f, &sh_growth);
#pragma unroll
  for (uint32_t l = 0; l < kTileRows; ++l) {
    hold_packed<N, T>(xr[l]);
    hold_packed<N, T>(hr[l]);
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) asm volatile("" : "+v"(rest[l][e]));  // nor are its products held
  }
  __syncthreads();
  const bool composed = kGate != APEX_GATE_GIVEN || sh_growth <= kMostGrowth;
  // the states that enter the groups of a segment, from the chunk's; the segment's composition, from its last group
  float states[kSegment];
  const uint64_t at_channel = d0 + min(w.channel, a.D - 1 - d0);
  const uint32_t steps = min(len - t0, w.steps);
  if (!composed) {
    const T *const g = static_cast<const T *>(a.g) + s * a.g_seq + t0 * a.g_time + at_channel;
    const T *const x = static_cast<const T *>(a.x) + s * a.x_seq + t0 * a.x_time + at_channel;
    const uint32_t first = w.segment / kChunkSegments * kChunkGroups, mine = w.segment * kSegment;
    const uint64_t chunk_bits = on.word[first / kChunkGroups] << 1 | 1;
    for (uint32_t i = first; i < mine + kSegment; ++i) {
      if (i >= mine) group_a[i * kWidth + w.channel] = state;
      float gt[kTileRows], xt[kTileRows];
#pragma unroll
      for (uint32_t l = 0; l < kTileRows; ++l) {
        const uint32_t t = min(i * kTileRows + l, steps - 1);
        gt[l] = (float)g[t * a.g_time], xt[l] = (float)x[t * a.x_time];
      }
#pragma unroll
      for (uint32_t l = 0; l < kTileRows; ++l)
        if (i * kTileRows + l < steps)
          state = __builtin_fmaf(gt[l], chunk_bits >> ((i - first) * kTileRows + l) & 1 ? state : 0.0f, xt[l]);
    }
  } else {
    const uint32_t first = w.segment / kChunkSegments * kChunkGroups;
    const uint64_t chunk_bits = on.word[first / kChunkGroups] << 1 | 1;
    const auto go_through = [&](uint32_t i) {
      const float ga = group_a[i * kWidth + w.channel], gb = group_b[i * kWidth + w.channel];
      state = no_cut || ((uint32_t)(chunk_bits >> (i - first) * kTileRows) & 15u) == 15u ? __builtin_fmaf(ga, state, gb) : gb;
    };
    for (uint32_t i = first; i < w.segment * kSegment; ++i) go_through(i);
#pragma unroll
    for (uint32_t i = 0; i < kSegment; ++i) {
      states[i] = state;
      go_through(w.segment * kSegment + i);
    }
    float P = 1.0f, Q = 0.0f;
#pragma unroll
    for (uint32_t i = kSegment; i-- > 0;) {
      const uint32_t at = (w.segment * kSegment + i) * kWidth + w.channel;
      const float gp = group_p[at], gq = group_q[at];
      const bool passes = no_cut || on.of_group(w.segment * kSegment + i) == 15u;
      P = passes ? P * gp : 0.0f;
      Q = passes ? __builtin_fmaf(gp, Q, gq) : gq;
    }
    segment_p[w.thread] = P;
    segment_q[w.thread] = Q;
  }
  __syncthreads();
  if (composed)
#pragma unroll
    for (uint32_t i = 0; i < kSegment; ++i) group_a[(w.segment * kSegment + i) * kWidth + w.channel] = states[i];
  const uint32_t last = (len - 1) / w.steps;
  float back_in = 0.0f;  // what enters the chain from behind; then what enters the tile
  if (speaks && a.dh_last && tile <= last && last - tile < kStretch) back_in = a.dh_last[(uint64_t)s * a.D + d0 + w.channel];
  if constexpr (kChained) {
    float P = 1.0f, Q = 0.0f;
    if (w.thread < kWidth)
      for (uint32_t i = w.segments; i-- > 0;) {
        const float sp = segment_p[i * kWidth + w.channel], sq = segment_q[i * kWidth + w.channel];
        const bool passes = on.all_of_segment(i);
        P = passes ? P * sp : 0.0f;
        Q = passes ? __builtin_fmaf(sp, Q, sq) : sq;
      }
    back_in = chain_state(chain.space->word + (uint64_t)column * chain.tiles * 3 * kWidth, last - tile, is, P, Q, !no_cut, back_in, tag,
                          sh_chain, composed);
  }
  if (!composed) {
    if (w.thread < kWidth) {
      const T *const g = static_cast<const T *>(a.g) + s * a.g_seq + t0 * a.g_time + at_channel;
      const T *const dh = static_cast<const T *>(a.dh) + ((uint64_t)s * a.T + t0) * a.D + at_channel;
      for (uint32_t i = w.groups; i-- > 0;) {
        group_p[i * kWidth + w.channel] = back_in;
        float gt[kTileRows], ht[kTileRows];
#pragma unroll
        for (uint32_t l = 0; l < kTileRows; ++l) {
          const uint32_t t = min(i * kTileRows + l, steps - 1);
          gt[l] = (float)g[t * a.g_time], ht[l] = (float)dh[(uint64_t)t * a.D];
        }
#pragma unroll
        for (uint32_t l = kTileRows; l-- > 0;)
          if (i * kTileRows + l < steps) back_in = gt[l] * (ht[l] + (on.of_group(i) >> l & 1 ? back_in : 0.0f));
      }
      if (kChained && speaks) hand_on(chain.space->word + (uint64_t)column * chain.tiles * 3 * kWidth, last - tile, back_in, tag);
    }
  } else if (w.thread < kWidth)
    for (uint32_t i = w.segments; i-- > 0;) {
      segment_in[i * kWidth + w.channel] = back_in;
      const float sp = segment_p[i * kWidth + w.channel], sq = segment_q[i * kWidth + w.channel];
      back_in = on.all_of_segment(i) ? __builtin_fmaf(sp, back_in, sq) : sq;
    }
  __syncthreads();
  uint32_t before = 0;
  if (kChained && w.thread == w.threads - 1) before = leaving(chain);
  if (composed) {
    float back = segment_in[w.thread];
#pragma unroll
    for (uint32_t i = kSegment; i-- > 0;) {
      const uint32_t at = (w.segment * kSegment + i) * kWidth + w.channel;
      const float gp = group_p[at], gq = group_q[at];
      group_p[at] = back;
      back = no_cut || on.of_group(w.segment * kSegment + i) == 15u ? __builtin_fmaf(gp, back, gq) : gq;
    }
  }
  __syncthreads();
  if (exists) {
    f32x4 back = *reinterpret_cast<const f32x4 *>(group_p + w.group * kWidth + w.run);
    f32x4 prev[kTileRows];
    prev[0] = *reinterpret_cast<const f32x4 *>(group_a + w.group * kWidth + w.run);
    T *const dg = static_cast<T *>(a.dg) + s * a.dg_seq + t_group * a.dg_time;
    T *const dx = static_cast<T *>(a.dx) + s * a.dx_seq + t_group * a.dx_time;
    plainly<kChained>(no_cut, [&](auto is_plain) {
      constexpr bool kPlain = decltype(is_plain)::value;
#pragma unroll
      for (uint32_t l = 0; l < kTileRows; ++l) {
        if (!kPlain && !(into >> l & 1)) prev[l] = f32x4{};
        if (l + 1 < kTileRows)
#pragma unroll
          for (uint32_t e = 0; e < N; ++e) {
            const float xt = element<N, T>(xr[l], e);
            prev[(l + 1) % kTileRows][e] = __builtin_fmaf(f[l][e], prev[l][e], kGate == APEX_GATE_SIGMOID ? rest[l][e] * xt : xt);
          }
      }
#pragma unroll
      for (uint32_t l = kTileRows; l-- > 0;) {
        const uint32_t t = t_group + l;
        if (!kPlain && !(bits >> l & 1)) back = f32x4{};
        Run<T, N> dgr, dxr;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) {
          float dgt, dxt;
          const float lambda = element<N, T>(hr[l], e) + back[e];
          scan_gate_back<kGate>(f[l][e], rest[l][e], element<N, T>(xr[l], e), prev[l][e], lambda, &dgt, &dxt);
          back[e] = f[l][e] * lambda;
          dgr[e] = (T)dgt;
          dxr[e] = (T)dxt;
        }
        if (whole) {
          store_run<T, N>(dg + l * a.dg_time + d, dgr, a.past_caches);
          store_run<T, N>(dx + l * a.dx_time + d, dxr, a.past_caches);
        } else if (t < a.T) {
          if (t >= len) dgr = dxr = Run<T, N>{};
          store_run_of<T, N>(dg + l * a.dg_time, d, a.D, dgr);
          store_run_of<T, N>(dx + l * a.dx_time, d, a.D, dxr);
        }
      }
    });
    if (a.dh0 && t_group == 0) store_run_of<float, N>(a.dh0 + (uint64_t)s * a.D, d, a.D, back);
  }
  if (kChained && w.thread == w.threads - 1) left(chain, before, tag);
}

constexpr uint32_t kChannelThreads = 64;

// A thread per channel, step after step: for an actor's single tokens.  Bound by the round trip of a launch and two loads
// (64 x 1 x 1024: 2.5 us), and for longer sequences by one step's loads after the other's.
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
    float f, rest, b;
    scan_gate<kGate>((float)g[t * a.g_time], (float)x[t * a.x_time], &f, &rest, &b);
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
      float f, rest, b;
      scan_gate<kGate>((float)g[t * a.g_time], (float)x[t * a.x_time], &f, &rest, &b);
      const float now = __builtin_fmaf(f, state, b);
      state = discount && discount[t] == 0.0f ? 0.0f : now;
    }
    for (uint32_t t = end; t-- > begin;) {
      const float gt = (float)g[t * a.g_time], xt = (float)x[t * a.x_time];
      const float lambda = (float)dh[(uint64_t)t * a.D] + (discount && discount[t] == 0.0f ? 0.0f : back);
      float f, rest, b, dgt, dxt;
      scan_gate<kGate>(gt, xt, &f, &rest, &b);
      scan_gate_back<kGate>(f, rest, xt, prev[t - begin][threadIdx.x], lambda, &dgt, &dxt);
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

template <typename F>
void with_gate(int gate, F f)
{
  if (gate == APEX_GATE_SIGMOID)
    f(std::integral_constant<int, APEX_GATE_SIGMOID>());
  else
    f(std::integral_constant<int, APEX_GATE_GIVEN>());
}

// Shorter sequences go by a thread per channel.  us, forward / gradient, by channel and by tile (bf16, a row of workgroups deep):
//     64 x T x 1024   T = 1   2.3 / 2.6   4.2 / 6.1      512 x T x 512   T = 1    3.3 / 4.3    5.9 / 9.5
//                         8   3.8 / 5.4   4.6 / 6.9                          8    5.4 / 10.6   6.7 / 11.2
//                        12   4.6 / 7.1   4.6 / 7.1                         12    6.5 / 16.2   7.1 / 12.7
//                        16   5.5 / 8.7   4.3 / 6.9                         16    7.5 / 26.4   6.9 / 13.6
constexpr uint32_t kTileMinSteps = 12;

struct ScanLaunch {
  bool by_channel;
  uint32_t grid, threads, lds;
  Chain chain;
};

int scan_launch(uint32_t S, uint32_t T, uint32_t D, bool back, void *workspace, ScanLaunch *l)
{
  if (T < kTileMinSteps) {
    *l = ScanLaunch{true, S * blocks_for(D, kChannelThreads), kChannelThreads, 0, {}};
    return APEX_OK;
  }
  l->by_channel = false;
  const uint32_t columns = S * blocks_for(D, kTileWidth);
  l->chain = Chain{static_cast<ScanSpace *>(workspace), columns, 1, std::min(columns, kScanCounters)};
  if (T <= kTileMaxSteps) {
    l->threads = (uint32_t)round_up(blocks_for(T, kTileRows) * kTileLanes, kTileWidth);
    l->grid = columns;
  } else {
    if (!workspace || (uintptr_t)workspace % 256) return APEX_ERR_INVALID_ARG;
    l->threads = kChainThreads;
    l->chain.tiles = blocks_for(T, kChainSteps);
    const uint64_t tiles = (uint64_t)columns * l->chain.tiles;
    if (l->chain.tiles > kMostTiles || tiles > 0xffffffffull / kChainThreads) return APEX_ERR_TOO_LARGE;
    l->grid = (uint32_t)tiles;
  }
  l->lds = back ? tile_back_lds(l->threads) : tile_lds(l->threads);
  return APEX_OK;
}

}  // namespace

extern "C" {

int apex_gated_scan_workspace_bytes(uint32_t S, uint32_t T, uint32_t D, size_t *bytes)
{
  if (!S || !T || !D || !bytes) return APEX_ERR_INVALID_ARG;
  size_t n = 0, words;
  if (T > kTileMaxSteps &&
      (__builtin_mul_overflow((uint64_t)S * blocks_for(T, kChainSteps), round_up(D, kTileWidth) * 3 * 8, &words) ||
       __builtin_add_overflow(words, kScanSpaceHead, &n)))
    return APEX_ERR_TOO_LARGE;
  *bytes = n;
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
  const ScanArgs a{S, T, D, g_seq_stride, g_time_stride, x_seq_stride, x_time_stride, g, x, discount, length, h0, h, h_last, carry,
                   (uint64_t)S * T * D * element_size(dtype) > kPastCachesBytes};
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  ScanLaunch l;
  if (const int rc = scan_launch(S, T, D, false, workspace, &l)) return rc;
  with_type(dtype, [&](auto t) {
    typedef decltype(t) E;
    with_gate(gate, [&](auto gate_of) {
      constexpr int kGate = decltype(gate_of)::value;
      if (l.by_channel)
        scan_channel_kernel<E, kGate><<<l.grid, l.threads, 0, stream>>>(a);
      else if (l.chain.tiles > 1)
        scan_tile_kernel<E, kGate, true><<<l.grid, l.threads, l.lds, stream>>>(a, l.chain);
      else
        scan_tile_kernel<E, kGate, false><<<l.grid, l.threads, l.lds, stream>>>(a, l.chain);
    });
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
                       dg_seq_stride, dg_time_stride, dx_seq_stride, dx_time_stride, dg, dx, dh0,
                       (uint64_t)S * T * D * size > kPastCachesBytes};
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  ScanLaunch l;
  if (const int rc = scan_launch(S, T, D, true, workspace, &l)) return rc;
  with_type(dtype, [&](auto t) {
    typedef decltype(t) E;
    with_gate(gate, [&](auto gate_of) {
      constexpr int kGate = decltype(gate_of)::value;
      if (l.by_channel)
        scan_channel_back_kernel<E, kGate><<<l.grid, l.threads, 0, stream>>>(a);
      else if (l.chain.tiles > 1)
        scan_tile_back_kernel<E, kGate, true><<<l.grid, l.threads, l.lds, stream>>>(a, l.chain);
      else
        scan_tile_back_kernel<E, kGate, false><<<l.grid, l.threads, l.lds, stream>>>(a, l.chain);
    });
  });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

}  // extern "C"
