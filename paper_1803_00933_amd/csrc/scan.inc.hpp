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
// composition as soon as it has it, looks back for the nearest tile whose outgoing state is there, applies the compositions
// in between one after the other, and publishes its own.  However far it looks back, the operations on a state are the same, so
// the bits are.  Only words of 64 bits cross between workgroups, a number and a tag in one, written and read at agent scope.
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
constexpr uint32_t kMostPolls = 1u << 20;  // a wait gives up (and hands on NaN) where the workspace was not as required

// The words of one tile: compositions A and B, state.
struct TileWords {
  uint64_t *a, *b, *state;
  __device__ __forceinline__ TileWords(ScanSpace *space, uint64_t tile, uint32_t width)
      : a(space->word + tile * 3 * width), b(a + width), state(b + width) {}
};

// The state that enters a tile from the one `behind` it, for the channel of this lane; called by a wave, whose first lane's
// channel exists.  word_of(i): the words of the tile i places away, i < reach.
template <typename F>
__device__ __forceinline__ float look_back(F word_of, uint32_t channel, bool exists, uint32_t reach, uint32_t tag)
{
  const uint32_t lane = lane_id();
  const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane((int)channel);
  uint64_t there = 0;
  uint32_t polls = 0;
  for (;;) {
    uint64_t w = 0;
    if (lane < reach) w = seen(word_of(lane).state + first);
    there = __ballot((uint32_t)(w >> 32) == tag);
    if (there || ++polls == kMostPolls) break;
    __builtin_amdgcn_s_sleep(1);
  }
  if (!there) return __builtin_nanf("");
  const uint32_t nearest = (uint32_t)__builtin_ctzll(there);
  if (!exists) return 0.0f;
  uint64_t w = seen(word_of(nearest).state + channel);
  while ((uint32_t)(w >> 32) != tag && ++polls < kMostPolls) w = seen(word_of(nearest).state + channel);
  float state = __uint_as_float((uint32_t)w);
  constexpr uint32_t kBatch = 2;
  for (uint32_t i = nearest; i > 0;) {
    uint64_t wa[kBatch], wb[kBatch];
#pragma unroll
    for (uint32_t j = 0; j < kBatch; ++j) {
      const TileWords t = word_of(i > j ? i - 1 - j : 0);
      wa[j] = seen(t.a + channel);
      wb[j] = seen(t.b + channel);
    }
#pragma unroll
    for (uint32_t j = 0; j < kBatch; ++j) {
      if (i == 0) break;
      const TileWords t = word_of(i - 1);
      while (((uint32_t)(wb[j] >> 32) != tag || ((uint32_t)(wa[j] >> 32) & ~kCutTag) != tag) && ++polls < kMostPolls)
        wa[j] = seen(t.a + channel), wb[j] = seen(t.b + channel);
      const float A = __uint_as_float((uint32_t)wa[j]), B = __uint_as_float((uint32_t)wb[j]);
      state = (uint32_t)(wa[j] >> 32) & kCutTag ? B : __builtin_fmaf(A, state, B);
      --i;
    }
  }
  return polls >= kMostPolls ? __builtin_nanf("") : state;
}

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

// kChained: tiles of a sequence wait for one another; else a sequence has one tile.
template <typename T, int kGate, bool kChained>
__global__ __launch_bounds__(kChained ? kChainThreads : kTileMaxThreads, 4) void scan_tile_kernel(ScanArgs a, Chain chain)
{
  constexpr uint32_t N = kTileRun, kWidth = kTileWidth;
  extern __shared__ uint64_t lds[];
  __shared__ RowBits into;  // whether the state passes into a row
  __shared__ uint2 sh_tile;
  const uint32_t threads = blockDim.x, thread = threadIdx.x, lane = lane_id(), wave = thread / kWave;
  const uint32_t groups = threads / kTileLanes, segments = threads / kWidth, steps = groups * kTileRows;
  float2 *const group_ab = reinterpret_cast<float2 *>(lds);                    // [groups][kWidth]; .x later: the state that enters
  float2 *const segment_ab = group_ab + groups * kWidth;                       // [segments][kWidth]
  float *const segment_in = reinterpret_cast<float *>(segment_ab + segments * kWidth);
  const uint32_t pieces = (a.D + kWidth - 1) / kWidth;  // of a row
  const uint32_t group = thread / kTileLanes, run = thread % kTileLanes * N;
  const uint32_t segment = thread / kWidth, channel = thread % kWidth;  // the same threads, when they go through compositions
  const uint32_t chunks = (a.T + APEX_SCAN_CHUNK - 1) / APEX_SCAN_CHUNK;
  uint32_t tag = 0, tile = 0, column = blockIdx.x;
  if (kChained) {
    tag = next_tag(chain.space->epoch);
    if (thread == 0) sh_tile = take_tile(chain);
    __syncthreads();
    tile = sh_tile.x, column = sh_tile.y;
  }
  const uint32_t s = column / pieces, d0 = column % pieces * kWidth, t0 = tile * steps;
  const uint32_t len = scan_length(a.length, s, a.T);
  const uint32_t t_group = t0 + group * kTileRows, d = d0 + run;
  const bool exists = d < a.D;
  // the rows of this thread
  const T *const g = static_cast<const T *>(a.g) + s * a.g_seq, *const x = static_cast<const T *>(a.x) + s * a.x_seq;
  Run<T, N> gr[kTileRows], xr[kTileRows];
#pragma unroll
  for (uint32_t l = 0; l < kTileRows; ++l) {
    const uint32_t t = t_group + l;
    if (exists && t < len) gr[l] = run_of<T, N>(g + t * a.g_time, d, a.D), xr[l] = run_of<T, N>(x + t * a.x_time, d, a.D);
  }
  if (thread < steps) {
    const uint32_t t = t0 + thread;
    const bool passes = !a.discount || t == 0 || t >= len || a.discount[(uint64_t)s * a.T + t - 1] != 0.0f;
    const uint64_t bits = __ballot(passes);
    if (lane == 0) into.word[wave] = bits;
  }
  __syncthreads();
  const uint32_t bits = into.of_group(group);
  float fa[kTileRows][N], fb[kTileRows][N];
  {
    float A[N], B[N];
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) A[e] = 1.0f, B[e] = 0.0f;
#pragma unroll
    for (uint32_t l = 0; l < kTileRows; ++l) {
      const bool inside = exists && t_group + l < len, passes = bits >> l & 1;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        float f = 1.0f, b = 0.0f, rest;
        if (inside) scan_gate<kGate>(element<N, T>(gr[l], e), element<N, T>(xr[l], e), &f, &rest, &b);
        fa[l][e] = f;
        fb[l][e] = b;
        A[e] = passes ? A[e] * f : 0.0f;
        B[e] = passes ? __builtin_fmaf(f, B[e], b) : b;
      }
    }
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) group_ab[group * kWidth + run + e] = make_float2(A[e], B[e]);
  }
  __syncthreads();
  if (segments > 1) {
    float A = 1.0f, B = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < kSegment; ++i) {
      const float2 c = group_ab[(segment * kSegment + i) * kWidth + channel];
      const bool passes = into.of_group(segment * kSegment + i) == 15u;
      A = passes ? A * c.x : 0.0f;
      B = passes ? __builtin_fmaf(c.x, B, c.y) : c.y;
    }
    segment_ab[segment * kWidth + channel] = make_float2(A, B);
    __syncthreads();
  }
  if (thread < kWidth) {
    const bool is = d0 + channel < a.D;
    const uint64_t at = (uint64_t)s * a.D + d0 + channel;
    float state = 0.0f;
    if (kChained && t0 < len && __ballot(is)) {
      float A = 1.0f, B = 0.0f;
      bool cut = false;
      for (uint32_t i = 0; i < segments; ++i) {
        const float2 c = segment_ab[i * kWidth + channel];
        const bool passes = into.all_of_segment(i);
        cut = cut || !passes;
        A = passes ? A * c.x : 0.0f;
        B = passes ? __builtin_fmaf(c.x, B, c.y) : c.y;
      }
      const auto words = [&](uint32_t behind) { return TileWords(chain.space, (uint64_t)column * chain.tiles + tile - 1 - behind, kWidth); };
      const TileWords own(chain.space, (uint64_t)column * chain.tiles + tile, kWidth);
      if (is && tile > 0) {
        publish(own.a + channel, tagged(A, cut ? tag | kCutTag : tag));
        publish(own.b + channel, tagged(B, tag));
      }
      if (is && cut) publish(own.state + channel, tagged(B, tag));
      if (tile == 0)
        state = a.h0 && is ? a.h0[at] : 0.0f;
      else
        state = look_back(words, channel, is, min(tile, kWave), tag);
      if (is && !cut) publish(own.state + channel, tagged(__builtin_fmaf(A, state, B), tag));
    } else if (!kChained && is) {
      state = a.h0 ? a.h0[at] : 0.0f;
    }
    if (t0 == 0 && len == 0 && is && a.h_last) a.h_last[at] = a.h0 ? a.h0[at] : 0.0f;
    segment_in[channel] = state;
    for (uint32_t i = 0; i + 1 < segments; ++i) {
      const float2 c = segment_ab[i * kWidth + channel];
      state = into.all_of_segment(i) ? __builtin_fmaf(c.x, state, c.y) : c.y;
      segment_in[(i + 1) * kWidth + channel] = state;
    }
  }
  __syncthreads();
  uint32_t before = 0;
  if (kChained && thread == threads - 1) before = leaving(chain);
  {
    float state = segment_in[segment * kWidth + channel];
#pragma unroll
    for (uint32_t i = 0; i < kSegment; ++i) {
      float2 *const at = group_ab + (segment * kSegment + i) * kWidth + channel;
      const float2 c = *at;
      at->x = state;
      state = into.of_group(segment * kSegment + i) == 15u ? __builtin_fmaf(c.x, state, c.y) : c.y;
    }
  }
  __syncthreads();
  if (exists) {
    float state[N];
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) state[e] = group_ab[group * kWidth + run + e].x;
    if (a.carry && t_group % APEX_SCAN_CHUNK == 0 && t_group < len) {
      float *const c = a.carry + ((uint64_t)s * chunks + t_group / APEX_SCAN_CHUNK) * a.D;
      Run<float, N> r;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) r[e] = bits & 1 ? state[e] : 0.0f;
      store_run_of<float, N>(c, d, a.D, r);
    }
    T *const h = static_cast<T *>(a.h) + (uint64_t)s * a.T * a.D;
#pragma unroll
    for (uint32_t l = 0; l < kTileRows; ++l) {
      const uint32_t t = t_group + l;
      const bool passes = bits >> l & 1;
      Run<T, N> r;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        state[e] = passes ? __builtin_fmaf(fa[l][e], state[e], fb[l][e]) : fb[l][e];
        r[e] = t < len ? (T)state[e] : (T)0.0f;
      }
      if (t < a.T) store_run_of<T, N>(h + (uint64_t)t * a.D, d, a.D, r);
      if (a.h_last && t + 1 == len) {
        const bool on = !a.discount || a.discount[(uint64_t)s * a.T + t] != 0.0f;
        Run<float, N> last;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) last[e] = on ? state[e] : 0.0f;
        store_run_of<float, N>(a.h_last + (uint64_t)s * a.D, d, a.D, last);
      }
    }
  }
  if (kChained && thread == threads - 1) left(chain, before, tag);
}

// The gradient in tiles: the states from `carry`, which begins anew every APEX_SCAN_CHUNK steps, and lambda by a chain from the
// last step to the first.  A row's bit says whether its state passes on; the rows of a chunk take each other's, and what enters
// a chunk's first row has been through its bit already.
constexpr uint32_t tile_back_lds(uint32_t threads)  // both kinds of compositions of the groups, segments' compositions, what enters
{
  return threads * kTileRun * 16 + threads * 12;
}

template <typename T, int kGate, bool kChained>
__global__ __launch_bounds__(kChained ? kChainThreads : kTileMaxThreads, 4) void scan_tile_back_kernel(ScanBackArgs a, Chain chain)
{
  constexpr uint32_t N = kTileRun, kWidth = kTileWidth;
  constexpr uint32_t kChunkGroups = APEX_SCAN_CHUNK / kTileRows, kChunkSegments = kChunkGroups / kSegment;
  static_assert(APEX_SCAN_CHUNK == kWave);  // a word of RowBits is a chunk

  extern __shared__ uint64_t lds[];
  __shared__ RowBits on;  // whether a row's state passes on
  __shared__ uint2 sh_tile;
  const uint32_t threads = blockDim.x, thread = threadIdx.x, lane = lane_id(), wave = thread / kWave;
  const uint32_t groups = threads / kTileLanes, segments = threads / kWidth, steps = groups * kTileRows;
  float2 *const group_ab = reinterpret_cast<float2 *>(lds);  // [groups][kWidth]; .x later: the state that enters
  float2 *const group_pq = group_ab + groups * kWidth;       // [groups][kWidth]; .x later: the gradient that enters from behind
  float2 *const segment_pq = group_pq + groups * kWidth;     // [segments][kWidth]
  float *const segment_in = reinterpret_cast<float *>(segment_pq + segments * kWidth);
  const uint32_t pieces = (a.D + kWidth - 1) / kWidth;
  const uint32_t group = thread / kTileLanes, run = thread % kTileLanes * N;
  const uint32_t segment = thread / kWidth, channel = thread % kWidth;
  const uint32_t chunks = (a.T + APEX_SCAN_CHUNK - 1) / APEX_SCAN_CHUNK;
  uint32_t tag = 0, tile = 0, column = blockIdx.x;
  if (kChained) {
    tag = next_tag(chain.space->epoch);
    if (thread == 0) sh_tile = take_tile(chain);
    __syncthreads();
    tile = chain.tiles - 1 - sh_tile.x, column = sh_tile.y;
  }
  const uint32_t s = column / pieces, d0 = column % pieces * kWidth, t0 = tile * steps;
  const uint32_t len = scan_length(a.length, s, a.T);
  const uint32_t t_group = t0 + group * kTileRows, d = d0 + run;
  const bool exists = d < a.D;
  const T *const g = static_cast<const T *>(a.g) + s * a.g_seq, *const x = static_cast<const T *>(a.x) + s * a.x_seq;
  const T *const dh = static_cast<const T *>(a.dh) + (uint64_t)s * a.T * a.D;
  Run<T, N> gr[kTileRows], xr[kTileRows], hr[kTileRows];
#pragma unroll
  for (uint32_t l = 0; l < kTileRows; ++l) {
    const uint32_t t = t_group + l;
    if (exists && t < len) {
      gr[l] = run_of<T, N>(g + t * a.g_time, d, a.D);
      xr[l] = run_of<T, N>(x + t * a.x_time, d, a.D);
      hr[l] = run_of<T, N>(dh + (uint64_t)t * a.D, d, a.D);
    }
  }
  // the state that enters the chunk of this thread's segment
  const bool is = d0 + channel < a.D;
  const uint32_t chunk = t0 / APEX_SCAN_CHUNK + segment / kChunkSegments;
  float state = 0.0f;
  if (is && chunk * APEX_SCAN_CHUNK < len) state = a.carry[((uint64_t)s * chunks + chunk) * a.D + d0 + channel];
  if (thread < steps) {
    const uint32_t t = t0 + thread;
    const uint64_t bits = __ballot(!a.discount || t >= len || a.discount[(uint64_t)s * a.T + t] != 0.0f);
    if (lane == 0) on.word[wave] = bits;
  }
  __syncthreads();
  const uint32_t bits = on.of_group(group);
  float f[kTileRows][N], rest[kTileRows][N];
  const uint32_t into = (uint32_t)((on.word[group / kChunkGroups] << 1 | 1) >> (group % kChunkGroups * kTileRows)) & 15u;
  {
    float A[N], B[N], P[N], Q[N];
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) A[e] = P[e] = 1.0f, B[e] = Q[e] = 0.0f;
#pragma unroll
    for (uint32_t l = 0; l < kTileRows; ++l) {
      const bool inside = exists && t_group + l < len, passes = into >> l & 1;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        float b = 0.0f;
        f[l][e] = 1.0f, rest[l][e] = 0.0f;
        if (inside) scan_gate<kGate>(element<N, T>(gr[l], e), element<N, T>(xr[l], e), &f[l][e], &rest[l][e], &b);
        A[e] = passes ? A[e] * f[l][e] : 0.0f;
        B[e] = passes ? __builtin_fmaf(f[l][e], B[e], b) : b;
      }
    }
#pragma unroll
    for (uint32_t l = kTileRows; l-- > 0;) {
      const bool inside = exists && t_group + l < len, passes = bits >> l & 1;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        const float dht = inside ? element<N, T>(hr[l], e) : 0.0f;
        P[e] = passes ? P[e] * f[l][e] : 0.0f;
        Q[e] = f[l][e] * (passes ? Q[e] + dht : dht);
      }
    }
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) {
      group_ab[group * kWidth + run + e] = make_float2(A[e], B[e]);
      group_pq[group * kWidth + run + e] = make_float2(P[e], Q[e]);
    }
  }
  __syncthreads();
  // the states that enter the groups of a segment, from the chunk's; the segment's composition, from its last group
  float states[kSegment];
  {
    const uint32_t first = segment / kChunkSegments * kChunkGroups;
    const uint64_t chunk_bits = on.word[first / kChunkGroups] << 1 | 1;
    const auto through = [&](uint32_t i) {
      const float2 c = group_ab[i * kWidth + channel];
      state = ((uint32_t)(chunk_bits >> (i - first) * kTileRows) & 15u) == 15u ? __builtin_fmaf(c.x, state, c.y) : c.y;
    };
    for (uint32_t i = first; i < segment * kSegment; ++i) through(i);
#pragma unroll
    for (uint32_t i = 0; i < kSegment; ++i) {
      states[i] = state;
      through(segment * kSegment + i);
    }
    float P = 1.0f, Q = 0.0f;
#pragma unroll
    for (uint32_t i = kSegment; i-- > 0;) {
      const float2 c = group_pq[(segment * kSegment + i) * kWidth + channel];
      const bool passes = on.of_group(segment * kSegment + i) == 15u;
      P = passes ? P * c.x : 0.0f;
      Q = passes ? __builtin_fmaf(c.x, Q, c.y) : c.y;
    }
    segment_pq[segment * kWidth + channel] = make_float2(P, Q);
  }
  __syncthreads();
#pragma unroll
  for (uint32_t i = 0; i < kSegment; ++i) group_ab[(segment * kSegment + i) * kWidth + channel].x = states[i];
  if (thread < kWidth) {
    const uint64_t at = (uint64_t)s * a.D + d0 + channel;
    const uint32_t last = len ? (len - 1) / steps : 0;
    float back = 0.0f;  // what enters the tile from behind
    if (is && a.dh_last && tile == last) back = a.dh_last[at];
    if (len == 0 && tile == 0 && is && a.dh0) a.dh0[at] = back;
    if (kChained && t0 < len && __ballot(is)) {
      float P = 1.0f, Q = 0.0f;
      bool cut = false;
      for (uint32_t i = segments; i-- > 0;) {
        const float2 c = segment_pq[i * kWidth + channel];
        const bool passes = on.all_of_segment(i);
        cut = cut || !passes;
        P = passes ? P * c.x : 0.0f;
        Q = passes ? __builtin_fmaf(c.x, Q, c.y) : c.y;
      }
      const auto words = [&](uint32_t behind) { return TileWords(chain.space, (uint64_t)column * chain.tiles + tile + 1 + behind, kWidth); };
      const TileWords own(chain.space, (uint64_t)column * chain.tiles + tile, kWidth);
      if (is && tile < last) {
        publish(own.a + channel, tagged(P, cut ? tag | kCutTag : tag));
        publish(own.b + channel, tagged(Q, tag));
      }
      if (is && cut) publish(own.state + channel, tagged(Q, tag));
      if (tile < last) back = look_back(words, channel, is, min(last - tile, kWave), tag);
      if (is && !cut) publish(own.state + channel, tagged(__builtin_fmaf(P, back, Q), tag));
    }
    for (uint32_t i = segments; i-- > 0;) {
      segment_in[i * kWidth + channel] = back;
      const float2 c = segment_pq[i * kWidth + channel];
      back = on.all_of_segment(i) ? __builtin_fmaf(c.x, back, c.y) : c.y;
    }
  }
  __syncthreads();
  uint32_t before = 0;
  if (kChained && thread == threads - 1) before = leaving(chain);
  {
    float back = segment_in[segment * kWidth + channel];
#pragma unroll
    for (uint32_t i = kSegment; i-- > 0;) {
      float2 *const at = group_pq + (segment * kSegment + i) * kWidth + channel;
      const float2 c = *at;
      at->x = back;
      back = on.of_group(segment * kSegment + i) == 15u ? __builtin_fmaf(c.x, back, c.y) : c.y;
    }
  }
  __syncthreads();
  if (exists) {
    float prev[kTileRows][N], back[N];
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) {
      prev[0][e] = group_ab[group * kWidth + run + e].x;
      back[e] = group_pq[group * kWidth + run + e].x;
    }
#pragma unroll
    for (uint32_t l = 0; l < kTileRows; ++l) {
      const bool inside = t_group + l < len, passes = into >> l & 1;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        if (!passes) prev[l][e] = 0.0f;
        if (l + 1 < kTileRows) {
          const float xt = inside ? element<N, T>(xr[l], e) : 0.0f;
          prev[(l + 1) % kTileRows][e] = __builtin_fmaf(f[l][e], prev[l][e], kGate == APEX_GATE_SIGMOID ? rest[l][e] * xt : xt);
        }
      }
    }
    T *const dg = static_cast<T *>(a.dg) + s * a.dg_seq, *const dx = static_cast<T *>(a.dx) + s * a.dx_seq;
#pragma unroll
    for (uint32_t l = kTileRows; l-- > 0;) {
      const uint32_t t = t_group + l;
      const bool inside = t < len, passes = bits >> l & 1;
      Run<T, N> dgr, dxr;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) {
        float dgt = 0.0f, dxt = 0.0f;
        if (inside) {
          const float lambda = element<N, T>(hr[l], e) + (passes ? back[e] : 0.0f);
          scan_gate_back<kGate>(f[l][e], rest[l][e], element<N, T>(xr[l], e), prev[l][e], lambda, &dgt, &dxt);
          back[e] = f[l][e] * lambda;
        }
        dgr[e] = (T)dgt;
        dxr[e] = (T)dxt;
      }
      if (t < a.T) {
        store_run_of<T, N>(dg + t * a.dg_time, d, a.D, dgr);
        store_run_of<T, N>(dx + t * a.dx_time, d, a.D, dxr);
      }
    }
    if (a.dh0 && t_group == 0 && len > 0) {
      Run<float, N> r;
#pragma unroll
      for (uint32_t e = 0; e < N; ++e) r[e] = back[e];
      store_run_of<float, N>(a.dh0 + (uint64_t)s * a.D, d, a.D, r);
    }
  }
  if (kChained && thread == threads - 1) left(chain, before, tag);
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

constexpr uint32_t kTileMinSteps = 16;  // shorter sequences: a thread per channel

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
    if (tiles > 0xffffffffull / kChainThreads) return APEX_ERR_TOO_LARGE;
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
  const ScanArgs a{S, T, D, g_seq_stride, g_time_stride, x_seq_stride, x_time_stride, g, x, discount, length, h0, h, h_last, carry};
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
                       dg_seq_stride, dg_time_stride, dx_seq_stride, dx_time_stride, dg, dx, dh0};
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
