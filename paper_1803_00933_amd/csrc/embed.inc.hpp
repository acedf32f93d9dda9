// Lookup of tokens' rows and the gradient of the table.  Included by apex_replay.hip (one translation unit).
#include "elements.hpp"

namespace apex {

constexpr uint32_t kEmbedThreads = 256;
constexpr uint32_t kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr uint32_t kDigitBits = 11, kDigits = 1u << kDigitBits;     // of a pass of the sort at most: two passes for any vocabulary
// Tokens that one workgroup sorts by itself, and of a tile else (never one tile of more tokens than the first).  The gradient of V x 64 in
// bf16, alone and in tiles: 2049 tokens of 2000 14.5 us and 20.3, of 49999 22.4 and 33.7; 8192 of 2000 21.0 and 22.3, of 49999 35.1 and 38.1.
constexpr uint32_t kSortAlone = 8192, kSortTile = 2048;
static_assert(kSortTile <= kSortAlone);
constexpr uint32_t kSlice = 64, kSlice2 = kSlice * kSlice;          // sorted tokens whose rows are summed up ahead, if they are one
// ... in two steps from so many tokens on.  The gradient of 32000 x 1024 in bf16, in one step and in two: 8192 tokens 77 us and 47 where all
// are one token, 72 and 73 where half are, 53.9 and 55.5 where a token is as frequent as one over its rank; 16384 125 and 53, 97 and 88, 59.7
// and 61.2; 32768 217 and 59, 154 and 107, 78.3 and 80.4.
constexpr uint32_t kSlice2From = 16384;

struct EmbedArgs {
  uint32_t N, V, D;
  uint32_t lanes_log2;  // lanes of a row
  uint64_t table_row, out_row;
  const void *table;
  const int32_t *token;
  float scale;
  void *out;
  bool past_caches;
};

// Rows of `lanes` lanes each; a token outside the table has a row of zeros.
// Bound by memory: every row is read where it is named and written once.  32768 rows of 2048 in bf16 42 us, 3.2 TB/s written and as
// much read, in part from the caches (30.5 on the rows of the pass before); 64 rows of 1024 2.2.
template <typename T>
__global__ __launch_bounds__(kEmbedThreads) void embed_kernel(EmbedArgs a)
{
  constexpr uint32_t N = 16 / sizeof(T);
  const uint32_t lanes = 1u << a.lanes_log2, rows = kEmbedThreads >> a.lanes_log2;
  const uint64_t n = (uint64_t)blockIdx.x * rows + (threadIdx.x >> a.lanes_log2);
  if (n >= a.N) return;
  const int32_t token = a.token[n];
  const bool named = token >= 0 && (uint32_t)token < a.V;
  const T *const row = static_cast<const T *>(a.table) + (named ? (uint64_t)token * a.table_row : 0);
  T *const out = static_cast<T *>(a.out) + n * a.out_row;
  in_either_way(a.past_caches, [&](auto past) {
    for (uint32_t at = (threadIdx.x & (lanes - 1)) * N; at < a.D; at += lanes * N) {
      if (at + N <= a.D) {
        Run<T, N> r{};
        if (named) r = load_run<T, N>(row + at);
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) r[e] = (T)(element<N, T>(r, e) * a.scale);
        if (!named) r = Run<T, N>{};  // (0 times a scale of -1)
        if (decltype(past)::value)
          __builtin_nontemporal_store(r, reinterpret_cast<Run<T, N> *>(out + at));
        else
          *reinterpret_cast<Run<T, N> *>(out + at) = r;
      } else {
        for (uint32_t d = at; d < a.D; ++d) out[d] = named ? (T)((float)row[d] * a.scale) : (T)0.0f;
      }
    }
  });
}

// ---- the gradient: tokens are sorted (stable, so that a token's rows keep their order), and every row of the table is the sum
// of the rows that name it, in that order.

struct SortArgs {
  uint32_t N, V, tiles, tile;
  uint32_t shift, bits;
  const int32_t *token;  // of the first pass (key_in is null)
  const uint32_t *key_in, *index_in;
  uint32_t *key_out, *index_out;
  uint32_t *count;  // [kDigits][tiles]: tokens of a digit in a tile, then in the tiles in front of it
  uint32_t *total;  // [kDigits]
};

// Tokens outside the table go behind all others.
__device__ __forceinline__ uint32_t sort_key(const SortArgs &a, uint32_t i)
{
  if (a.key_in) return a.key_in[i];
  const uint32_t t = (uint32_t)a.token[i];
  return t < a.V ? t : a.V;
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortArgs a)
{
  __shared__ uint32_t count[kDigits];
  const uint32_t digits = 1u << a.bits;
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
  __syncthreads();
  const uint32_t begin = blockIdx.x * a.tile, end = min(a.N, begin + a.tile);
  for (uint32_t i = begin + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&count[(sort_key(a, i) >> a.shift) & (digits - 1)], 1u);
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) a.count[(uint64_t)d * a.tiles + blockIdx.x] = count[d];
}

// A wave per digit: how many of it are in the tiles in front of each.
__global__ __launch_bounds__(kEmbedThreads) void sort_tiles_kernel(SortArgs a)
{
  const uint32_t d = blockIdx.x * (kEmbedThreads / kWave) + threadIdx.x / kWave, lane = lane_id();
  if (d >= 1u << a.bits) return;
  uint32_t *const count = a.count + (uint64_t)d * a.tiles;
  uint32_t before = 0;
  for (uint32_t t0 = 0; t0 < a.tiles; t0 += kWave) {
    const uint32_t mine = t0 + lane < a.tiles ? count[t0 + lane] : 0;
    const uint32_t up_to = (uint32_t)wave_inclusive_scan(mine);
    if (t0 + lane < a.tiles) count[t0 + lane] = before + up_to - mine;
    before += (uint32_t)__builtin_amdgcn_readlane((int)up_to, kWave - 1);
  }
  if (lane == 0) a.total[d] = before;
}

// Places of a tile's tokens: behind all of smaller digits, those of the same digit in earlier tiles, in earlier waves, and in
// front of it in its wave, which goes through its part in groups of 64: lanes of the same digit find one another by a ballot per
// bit.  One pass of the sort; kAlone: with the counts of a single tile, kGroups groups a wave at most.  count[digit][wave] holds what
// a wave has of a digit, then how many tokens of the tile go in front of those; base, of a digit, what the tile's places begin at.
// A workgroup that is alone keeps tokens and places in `held` from pass to pass, and writes them out in their order at the end: as
// scattered words, by one compute unit, 7777 took 32 us.
struct Held {
  uint32_t key, index;
};
template <bool kAlone>
__device__ __forceinline__ void sort_pass(const SortArgs &a, uint16_t *count, uint32_t *base, Held *held, bool second)
{
  constexpr uint32_t kGroups = (kAlone ? kSortAlone : kSortTile) / kSortThreads;
  __shared__ uint32_t of_wave[kSortWaves];
  const uint32_t digits = 1u << a.bits, lane = lane_id(), wave = threadIdx.x / kWave;
  for (uint32_t i = threadIdx.x; i < digits * kSortWaves / 2; i += kSortThreads) reinterpret_cast<uint32_t *>(count)[i] = 0;
  // a wave's part: consecutive groups
  const uint32_t tile_begin = kAlone ? 0 : blockIdx.x * a.tile, tile_end = kAlone ? a.N : min(a.N, tile_begin + a.tile);
  const uint32_t groups = ((tile_end - tile_begin) + kSortThreads - 1) / kSortThreads;
  const uint32_t begin = tile_begin + wave * groups * kWave + lane;
  uint32_t key[kGroups], index[kGroups], local[kGroups];
#pragma unroll
  for (uint32_t g = 0; g < kGroups; ++g) {
    const uint32_t i = begin + g * kWave;
    if (g < groups && i < tile_end) {
      if (kAlone && second) {
        key[g] = held[i].key, index[g] = held[i].index;
      } else {
        key[g] = sort_key(a, i);
        index[g] = a.key_in ? a.index_in[i] : i;
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (uint32_t g = 0; g < kGroups; ++g) {
    if (g >= groups) continue;  // (for all)
    const bool have = begin + g * kWave < tile_end;
    const uint32_t digit = have ? (key[g] >> a.shift) & (digits - 1) : 0;
    uint32_t low = 0, high = 0;  // lanes of which a bit differs
#pragma unroll
    for (uint32_t b = 0; b < kDigitBits; ++b) {
      const uint32_t mine = (uint32_t)__builtin_amdgcn_sbfe((int)digit, b, 1);  // all ones, or none
      const uint64_t ones = __ballot(mine != 0);
      low |= (uint32_t)ones ^ mine, high |= (uint32_t)(ones >> 32) ^ mine;
    }
    const uint64_t same = __ballot(have) & ~((uint64_t)high << 32 | low);
    if (have) {
      const uint32_t rank = __builtin_popcountll(same & ((1ull << lane) - 1));
      volatile uint16_t *const place = &count[digit * kSortWaves + wave];  // (other lanes of the wave write it)
      const uint32_t had = *place;
      local[g] = had + rank;
      __builtin_amdgcn_wave_barrier();
      if (rank == 0) *place = (uint16_t)(had + __builtin_popcountll(same));
    }
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  // what is in front, digit by digit and wave by wave: a thread has neighbouring counts
  const uint32_t each = max(digits * kSortWaves / kSortThreads, 1u), first = threadIdx.x * each;
  uint32_t sum = 0;
  if (first < digits * kSortWaves)
    for (uint32_t i = 0; i < each; ++i) sum += count[first + i];
  const auto in_front = [&](uint32_t mine) {  // of all threads
    const uint32_t up_to = (uint32_t)wave_inclusive_scan(mine);
    if (lane == kWave - 1) of_wave[wave] = up_to;
    __syncthreads();
    const uint32_t waves = (uint32_t)wave_inclusive_scan(lane < kSortWaves ? of_wave[lane] : 0);
    __syncthreads();
    return up_to - mine + (wave ? (uint32_t)__builtin_amdgcn_readlane((int)waves, (int)__builtin_amdgcn_readfirstlane((int)wave) - 1) : 0);
  };
  uint32_t before = in_front(sum);
  if (first < digits * kSortWaves)
    for (uint32_t i = 0; i < each; ++i) {
      const uint32_t c = count[first + i];
      count[first + i] = (uint16_t)before;
      before += c;
    }
  if (!kAlone) {
    // (a thread's two digits)
    const uint32_t d = threadIdx.x * 2;
    const uint32_t n0 = d < digits ? a.total[d] : 0, n1 = d + 1 < digits ? a.total[d + 1] : 0;
    const uint32_t front = in_front(n0 + n1);
    __syncthreads();
    if (d < digits) base[d] = front + a.count[(uint64_t)d * a.tiles + blockIdx.x] - count[d * kSortWaves];
    if (d + 1 < digits) base[d + 1] = front + n0 + a.count[(uint64_t)(d + 1) * a.tiles + blockIdx.x] - count[(d + 1) * kSortWaves];
  }
  __syncthreads();
#pragma unroll
  for (uint32_t g = 0; g < kGroups; ++g) {
    if (g >= groups || begin + g * kWave >= tile_end) continue;
    const uint32_t digit = (key[g] >> a.shift) & (digits - 1);
    const uint32_t to = (kAlone ? 0 : base[digit]) + count[digit * kSortWaves + wave] + local[g];
    if (kAlone) {
      held[to] = Held{key[g], index[g]};
    } else {
      a.key_out[to] = key[g];
      a.index_out[to] = index[g];
    }
  }
}

__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(SortArgs a)
{
  __shared__ __align__(16) uint16_t count[kDigits * kSortWaves];
  __shared__ uint32_t base[kDigits];
  sort_pass<false>(a, count, base, nullptr, false);
}

// Both passes by one workgroup: 6144 tokens of 32768 15.2 us, 7777 of 49999 21; groups of a wave one after the other, and LDS.  In tiles
// of 2048 by as many workgroups, three launches a pass, 32768 tokens of 131072 take 31.
__global__ __launch_bounds__(kSortThreads) void sort_alone_kernel(SortArgs first, SortArgs second)
{
  __shared__ __align__(16) uint16_t count[kDigits * kSortWaves];
  __shared__ Held held[kSortAlone];
  sort_pass<true>(first, count, nullptr, held, false);
  __syncthreads();
  if (second.bits) {
    sort_pass<true>(second, count, nullptr, held, true);
    __syncthreads();
  }
  const SortArgs &last = second.bits ? second : first;
  for (uint32_t i = threadIdx.x; i < first.N; i += kSortThreads) last.key_out[i] = held[i].key, last.index_out[i] = held[i].index;
}

struct EmbedBackArgs {
  uint32_t N, V, D;
  uint64_t dout_row, dtable_row;
  const void *dout;
  const uint32_t *key, *index;    // sorted
  uint32_t *begin, *end;          // [V]: a token's places, where it has any (else whatever was there)
  float *slice, *slice2;          // sums of slices of 64 and of 4096 that are one token's (null: of 64 alone)
  float scale;
  bool add;
  void *dtable;
  bool past_caches;
};

template <typename T, int N>
__device__ __forceinline__ void add_row(const T *row, uint32_t at, uint32_t D, float (&sum)[N])
{
  if (at + N <= D) {
    const Run<T, N> r = load_run<T, N>(row + at);
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] += element<N, T>(r, e);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (at + e < D) sum[e] += (float)row[at + e];
  }
}

// The rows of places [from, to), in their order, kAhead on their way at once.
template <typename T, int N, uint32_t kAhead>
__device__ __forceinline__ void add_places(const EmbedBackArgs &a, uint32_t from, uint32_t to, uint32_t at, float (&sum)[N])
{
  const T *const dout = static_cast<const T *>(a.dout);
  uint32_t i = from;
  if (at + N <= a.D) {
    for (; i + kAhead <= to; i += kAhead) {
      Run<T, N> r[kAhead];
#pragma unroll
      for (uint32_t j = 0; j < kAhead; ++j) r[j] = load_run<T, N>(dout + a.index[i + j] * a.dout_row + at);
#pragma unroll
      for (uint32_t j = 0; j < kAhead; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += element<N, T>(r[j], e);
    }
  }
  for (; i < to; ++i) add_row<T, N>(dout + a.index[i] * a.dout_row, at, a.D, sum);
}

template <int N>
__device__ __forceinline__ void put_sums(float *row, uint32_t at, uint32_t D, const float (&sum)[N])
{
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (at + e < D) row[at + e] = sum[e];
}

// Where a token's places begin and end; and the sums of the slices that are one token's, so that a frequent token is not one
// workgroup's alone.  A wave per slice and piece of a row.
template <typename T>
__global__ __launch_bounds__(kEmbedThreads) void embed_slices_kernel(EmbedBackArgs a)
{
  constexpr uint32_t N = 16 / sizeof(T);
  const uint32_t pieces = (a.D + kWave * N - 1) / (kWave * N);
  const uint64_t job = (uint64_t)blockIdx.x * (kEmbedThreads / kWave) + threadIdx.x / kWave;
  const uint32_t s = (uint32_t)(job / pieces), piece = (uint32_t)(job % pieces), lane = lane_id();
  const uint64_t from = (uint64_t)s * kSlice;
  if (from >= a.N) return;
  const uint32_t i = (uint32_t)from + lane;
  if (piece == 0 && i < a.N) {
    const uint32_t key = a.key[i];
    if (key < a.V) {
      if (i == 0 || a.key[i - 1] != key) a.begin[key] = i;
      if (i == a.N - 1 || a.key[i + 1] != key) a.end[key] = i + 1;
    }
  }
  if (from + kSlice > a.N) return;
  const uint32_t key = a.key[from];
  if (key >= a.V || a.key[from + kSlice - 1] != key) return;
  const uint32_t at = (piece * kWave + lane) * N;
  if (at >= a.D) return;
  float sum[N] = {};
  add_places<T, N, 8>(a, (uint32_t)from, (uint32_t)from + kSlice, at, sum);
  put_sums<N>(a.slice + (uint64_t)s * a.D, at, a.D, sum);
}

// 64 of them once more, where all are one token's.
__global__ __launch_bounds__(kEmbedThreads) void embed_slices2_kernel(EmbedBackArgs a)
{
  const uint32_t pieces = (a.D + kWave - 1) / kWave;
  const uint64_t job = (uint64_t)blockIdx.x * (kEmbedThreads / kWave) + threadIdx.x / kWave;
  const uint32_t s = (uint32_t)(job / pieces), at = (uint32_t)(job % pieces) * kWave + lane_id();
  const uint64_t from = (uint64_t)s * kSlice2;
  if (from + kSlice2 > a.N || at >= a.D) return;
  const uint32_t key = a.key[from];
  if (key >= a.V || a.key[from + kSlice2 - 1] != key) return;
  float sum = 0.0f;
#pragma unroll 8
  for (uint32_t j = 0; j < kSlice; ++j) sum += a.slice[((uint64_t)s * kSlice + j) * a.D + at];
  a.slice2[(uint64_t)s * a.D + at] = sum;
}

// A wave per row of the table and piece of it: the table's gradient is written once (zeros where a token is not named), the rows that name
// it are read once.  131072 x 2048 in bf16 with 32768 places 190 us, 3.5 TB/s read and written; with none 80, 6.7 TB/s: bound by a named row's
// loads, which come one behind the other (where it begins, its key, where it ends, its places, their rows).  On the inputs of the pass before
// 103, and eight rows on their way instead of four, or four slices, which cost registers and waves, 121 and 126.
template <typename T>
__global__ __launch_bounds__(kEmbedThreads) void embed_rows_kernel(EmbedBackArgs a)
{
  constexpr uint32_t N = 16 / sizeof(T);
  const uint32_t pieces = (a.D + kWave * N - 1) / (kWave * N);
  const uint64_t job = (uint64_t)blockIdx.x * (kEmbedThreads / kWave) + threadIdx.x / kWave;
  const uint32_t v = (uint32_t)(job / pieces), at = ((uint32_t)(job % pieces) * kWave + lane_id()) * N;
  if (v >= a.V || at >= a.D) return;
  // (begin holds a place of this call only where the sorted tokens say so)
  const uint32_t begin = a.begin[v];
  const bool named = begin < a.N && a.key[begin] == v;
  T *const row = static_cast<T *>(a.dtable) + v * a.dtable_row;
  float sum[N] = {};
  if (named) {
    const uint32_t end = a.end[v];
    const uint32_t whole = (begin + kSlice - 1) / kSlice * kSlice, last = end / kSlice * kSlice;   // (N stays below 2^31)
    if (whole >= last) {
      add_places<T, N, 4>(a, begin, end, at, sum);
    } else {
      add_places<T, N, 4>(a, begin, whole, at, sum);
      for (uint32_t i = whole; i < last;) {
        const bool many = a.slice2 && i % kSlice2 == 0 && last - i >= kSlice2;
        const float *const from = many ? a.slice2 + (uint64_t)(i / kSlice2) * a.D : a.slice + (uint64_t)(i / kSlice) * a.D;
        add_row<float, N>(from, at, a.D, sum);
        i += many ? kSlice2 : kSlice;
      }
      add_places<T, N, 4>(a, last, end, at, sum);
    }
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) sum[e] *= a.scale;
  }
  if (a.add) {
    if (!named) return;
    add_row<T, N>(row, at, a.D, sum);
  }
  if (at + N <= a.D) {
    Run<T, N> r;
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) r[e] = (T)sum[e];
    store_run<T, N>(row + at, r, a.past_caches);
  } else {
#pragma unroll
    for (uint32_t e = 0; e < N; ++e)
      if (at + e < a.D) row[at + e] = (T)sum[e];
  }
}

}  // namespace apex

namespace {

struct EmbedSpace {
  uint64_t key[2], index[2], begin, end, count, total, slice, slice2, bytes;
  uint32_t tiles, tile;
};

bool embed_space(uint32_t N, uint32_t V, uint32_t D, EmbedSpace *s)
{
  uint64_t at = 0;
  bool fits = true;
  const auto take = [&](uint64_t *offset, uint64_t words) {
    *offset = at;
    fits = !__builtin_add_overflow(at, round_up(words * 4, 256), &at) && fits;
  };
  s->tile = N <= kSortAlone ? N : kSortTile;
  s->tiles = blocks_for(N, s->tile);
  for (int i = 0; i < 2; ++i) take(&s->key[i], N), take(&s->index[i], N);
  take(&s->begin, V), take(&s->end, V);
  take(&s->count, s->tiles > 1 ? (uint64_t)kDigits * s->tiles : 0), take(&s->total, kDigits);
  take(&s->slice, (uint64_t)(N / kSlice) * D), take(&s->slice2, (uint64_t)(N / kSlice2) * D);
  s->bytes = at;
  return fits;
}

int embed_check(uint32_t N, uint32_t V, uint32_t D, int dtype, float scale)
{
  if (!N || !V || !D || !element_size(dtype) || !(scale - scale == 0.0f)) return APEX_ERR_INVALID_ARG;
  if (N > APEX_MAX_TOKENS || V > APEX_MAX_VOCABULARY || D > APEX_MAX_WIDTH) return APEX_ERR_TOO_LARGE;
  return APEX_OK;
}

}  // namespace

extern "C" {

int apex_embedding(uint32_t N, uint32_t V, uint32_t D, int dtype, const void *table, uint64_t table_stride, const int32_t *token,
                   float scale, void *out, uint64_t out_stride, void *hip_stream)
{
  if (const int rc = embed_check(N, V, D, dtype, scale)) return rc;
  const uint32_t size = element_size(dtype);
  if (!table || !token || !out || (uintptr_t)token % 4 || !rows_fit(table, size, V, table_stride, 1, 0, D) ||
      !rows_apart(out, size, N, out_stride, 1, 0, D))
    return APEX_ERR_INVALID_ARG;
  const uint32_t lanes_log2 = std::min(ceil_log2(blocks_for(D, 16 / size)), 8u);
  const EmbedArgs a{N, V, D, lanes_log2, table_stride, out_stride, table, token, scale, out, (uint64_t)N * D * size > kPastCachesBytes};
  const uint32_t blocks = blocks_for(N, kEmbedThreads >> lanes_log2);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  with_type(dtype, [&](auto t) { embed_kernel<decltype(t)><<<dim3(blocks), dim3(kEmbedThreads), 0, stream>>>(a); });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

int apex_embedding_backward_workspace_bytes(uint32_t N, uint32_t V, uint32_t D, size_t *bytes)
{
  if (!bytes) return APEX_ERR_INVALID_ARG;
  if (const int rc = embed_check(N, V, D, APEX_F32, 1.0f)) return rc;
  EmbedSpace s;
  if (!embed_space(N, V, D, &s)) return APEX_ERR_TOO_LARGE;
  *bytes = s.bytes;
  return APEX_OK;
}

int apex_embedding_backward(uint32_t N, uint32_t V, uint32_t D, int dtype, const void *dout, uint64_t dout_stride, const int32_t *token,
                            float scale, int add, void *dtable, uint64_t dtable_stride, void *workspace, void *hip_stream)
{
  if (const int rc = embed_check(N, V, D, dtype, scale)) return rc;
  const uint32_t size = element_size(dtype);
  if (!dout || !token || !dtable || !workspace || (uintptr_t)token % 4 || (uintptr_t)workspace % 256 ||
      !rows_fit(dout, size, N, dout_stride, 1, 0, D) || !rows_apart(dtable, size, V, dtable_stride, 1, 0, D))
    return APEX_ERR_INVALID_ARG;
  EmbedSpace s;
  if (!embed_space(N, V, D, &s)) return APEX_ERR_TOO_LARGE;
  char *const space = static_cast<char *>(workspace);
  const auto words = [&](uint64_t offset) { return reinterpret_cast<uint32_t *>(space + offset); };
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  // two passes, of half the bits each, where one does not reach
  const uint32_t bits = ceil_log2((uint64_t)V + 1), passes = blocks_for(bits, kDigitBits), each = blocks_for(bits, passes);
  SortArgs sort[2] = {{N, V, s.tiles, s.tile, 0, each, token, nullptr, nullptr, words(s.key[0]), words(s.index[0]), words(s.count),
                       words(s.total)}, {}};
  if (passes > 1)
    sort[1] = SortArgs{N, V, s.tiles, s.tile, each, bits - each, token, words(s.key[0]), words(s.index[0]), words(s.key[1]),
                       words(s.index[1]), words(s.count), words(s.total)};
  if (s.tiles == 1) {
    sort_alone_kernel<<<dim3(1), dim3(kSortThreads), 0, stream>>>(sort[0], sort[1]);
  } else {
    for (uint32_t p = 0; p < passes; ++p) {
      sort_count_kernel<<<dim3(s.tiles), dim3(kSortThreads), 0, stream>>>(sort[p]);
      sort_tiles_kernel<<<dim3(blocks_for(1u << sort[p].bits, kEmbedThreads / kWave)), dim3(kEmbedThreads), 0, stream>>>(sort[p]);
      sort_place_kernel<<<dim3(s.tiles), dim3(kSortThreads), 0, stream>>>(sort[p]);
    }
  }
  const EmbedBackArgs a{N, V, D, dout_stride, dtable_stride, dout, sort[passes - 1].key_out, sort[passes - 1].index_out, words(s.begin),
                        words(s.end), reinterpret_cast<float *>(space + s.slice),
                        N >= kSlice2From ? reinterpret_cast<float *>(space + s.slice2) : nullptr, scale,
                        add != 0, dtable, (uint64_t)V * D * size > kPastCachesBytes};
  with_type(dtype, [&](auto t) {
    typedef decltype(t) E;
    constexpr uint32_t kWaves = kEmbedThreads / kWave;
    const uint64_t pieces = blocks_for(D, kWave * 16 / sizeof(E));
    embed_slices_kernel<E><<<dim3(blocks_for(blocks_for(N, kSlice) * pieces, kWaves)), dim3(kEmbedThreads), 0, stream>>>(a);
    if (a.slice2)
      embed_slices2_kernel<<<dim3(blocks_for((uint64_t)(N / kSlice2) * blocks_for(D, kWave), kWaves)), dim3(kEmbedThreads), 0, stream>>>(a);
    embed_rows_kernel<E><<<dim3(blocks_for(V * pieces, kWaves)), dim3(kEmbedThreads), 0, stream>>>(a);
  });
  APEX_HIP(hipGetLastError());
  return APEX_OK;
}

}  // extern "C"
