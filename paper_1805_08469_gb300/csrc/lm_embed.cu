// Embedding of tokens and the gradient of its table (include/gem_lm.h).
//
// Lookup: a warp copies a slab of a row, a lane 16 bytes of what it writes (single elements where a row
// does not lie on such boundaries).  65,536 tokens of Zipf frequencies, rows of 1024 fp32 to bf16: 47 us (402 MB read and
// written, of which repeated rows come from L2; HBM at 48%, its warps wait for their loads).
//
// Gradient, in four launches:
//   zeros  to the table's rows that no token has (where they are not added to); each block looks through the
//          tokens for those of its rows.
//   sort   one cluster sorts the tokens with their places (stable, by digits of up to nine bits, the lowest first).  A block of it
//          takes all of an SM's registers, so it starts when the zeros of as many neighbouring SMs are written, beside the last.
//   sums   the sorted places are cut into chunks of L.  A warp takes a chunk and a slab of columns, adds up each run
//          of equal tokens in fp32 and writes the row of a run that lies inside the chunk.  What a run has in the
//          chunk where it began, and in each where it goes on, are partial sums.
//   join   adds a run's partial sums in the order of the chunks.
// Every dout row is read once and every row of the table written once, and a heavy token (one word in ten) is
// spread over as many warps as it has chunks.  The order of every sum is fixed by the tokens.  65,536 tokens of Zipf
// frequencies, 131,072 rows of 1024 fp32 from bf16: zeros 80 us (450 MB; the first of their blocks end at 55), sort from 66 to 89, sums
// 38 (5 TB/s), join 13 (the heaviest token's 120 partial rows).
#include <cooperative_groups.h>

#include <algorithm>

#include "lm_internal.h"

namespace gem {
namespace lm {
namespace {

namespace cg = cooperative_groups;

constexpr int kEmbedThreads = 128;

// 16 / sizeof(E) columns of a lane: neighbours where the rows of all tensors of the call lie at multiples of their
// pieces' size and have whole pieces (WIDE), else 32 apart.
template <typename E>
constexpr int kCols = 16 / int(sizeof(E));
template <typename E>
constexpr int kSlab = 32 * kCols<E>;   // columns of a warp

template <typename E, bool WIDE>
struct Columns {
  int first, D;
  __device__ Columns(int slab, int D) : first(slab * kSlab<E> + int(threadIdx.x % 32) * (WIDE ? kCols<E> : 1)), D(D) {}
  __device__ int operator()(int k) const { return first + (WIDE ? k : 32 * k); }
  __device__ bool has(int k) const { return WIDE ? first < D : (*this)(k) < D; }
};

// A lane's columns of a row of type X as they are in memory: in words, or one by one (so that loads of several rows are
// in flight: to pack single elements would wait for each).
template <typename E, bool WIDE, typename X>
struct Row;
template <typename E, typename X>
struct Row<E, true, X> {
  static constexpr int kWords = kCols<E> * int(sizeof(X)) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void read(const Columns<E, true>& c, const X* row) {
    if (!c.has(0)) return;
    const X* const at = row + c.first;
#pragma unroll
    for (int i = 0; i < kWords; i += kWords < 4 ? kWords : 4) {
      if constexpr (kWords >= 4)
        *reinterpret_cast<uint4*>(w + i) = *reinterpret_cast<const uint4*>(at + i * 4 / int(sizeof(X)));
      else
        *reinterpret_cast<uint2*>(w + i) = *reinterpret_cast<const uint2*>(at + i * 4 / int(sizeof(X)));
    }
  }
  __device__ __forceinline__ float operator[](int k) const {
    if constexpr (sizeof(X) == 4) {
      return __uint_as_float(w[k]);
    } else {
      const uint16_t half = uint16_t(w[k / 2] >> (k % 2 * 16));
      return to_f32(*reinterpret_cast<const X*>(&half));
    }
  }
};
template <typename E, typename X>
struct Row<E, false, X> {
  X x[kCols<E>];
  __device__ __forceinline__ void read(const Columns<E, false>& c, const X* row) {
#pragma unroll
    for (int k = 0; k < kCols<E>; ++k)
      if (c.has(k)) x[k] = row[c(k)];
  }
  __device__ __forceinline__ float operator[](int k) const { return to_f32(x[k]); }
};

template <typename X, int K>
struct alignas(sizeof(X) * K < 16 ? sizeof(X) * K : 16) Piece {
  X x[K];
};
template <typename E, bool WIDE, typename X>
__device__ __forceinline__ void write_row(const Columns<E, WIDE>& c, X* row, const float (&v)[kCols<E>]) {
  if constexpr (WIDE) {
    Piece<X, kCols<E>> p;
#pragma unroll
    for (int k = 0; k < kCols<E>; ++k) p.x[k] = from_f32<X>(v[k]);
    if (c.has(0)) *reinterpret_cast<Piece<X, kCols<E>>*>(row + c.first) = p;
  } else {
#pragma unroll
    for (int k = 0; k < kCols<E>; ++k)
      if (c.has(k)) row[c(k)] = from_f32<X>(v[k]);
  }
}

struct EmbedArgs {
  const void* table;
  void* out;
  int64_t table_ld, out_ld;
  int64_t N;
  int V, D, slabs;
  const int32_t* tokens;
  float scale;
};

template <typename T, typename E, bool WIDE>
__global__ void __launch_bounds__(kEmbedThreads) embed_kernel(const EmbedArgs p) {
  pdl_entry();
  const int64_t i = int64_t(blockIdx.x) * (kEmbedThreads / 32) + threadIdx.x / 32;
  const int64_t n = i / p.slabs;
  if (n >= p.N) return;
  const Columns<E, WIDE> c(int(i % p.slabs), p.D);
  const int token = p.tokens[n];
  float v[kCols<E>];
  if (token >= 0 && token < p.V) {
    Row<E, WIDE, T> row;
    row.read(c, static_cast<const T*>(p.table) + token * p.table_ld);
#pragma unroll
    for (int k = 0; k < kCols<E>; ++k) v[k] = row[k] * p.scale;
  } else {
#pragma unroll
    for (int k = 0; k < kCols<E>; ++k) v[k] = token < 0 ? 0.0f : NAN;
  }
  write_row<E, WIDE, E>(c, static_cast<E*>(p.out) + n * p.out_ld, v);
}

struct EmbedGradArgs {
  const void* dout;
  void* dtable;
  int64_t dout_ld, dtable_ld;
  int64_t N;
  int V, D;
  const int32_t* tokens;
  float scale;
  bool accumulate;
  int32_t *keys[2], *places[2];   // [N]: each pass of the sort writes one pair
  const int32_t *sorted_keys, *sorted_places;   // what the last pass wrote
  float* parts;                   // [chunks][2][pitch]: of a chunk's run that began before it, of its last run if that goes on
  int bits, passes;               // of a digit, of the sort
  int chunk, chunks, slabs, pitch;
};

// ---- sort, and zeros ----

constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kDigitBits = 9, kRadix = 1 << kDigitBits;
constexpr int kZeroBlocks = 152, kZeroRows = 1 << 17;   // rows of a block at a time

// A block's shared memory.
struct SortShared {
  unsigned counts[kSortWarps][kRadix];   // entries of each warp and digit, then where its next one goes
  unsigned total[kRadix];                // the block's entries of each digit
  unsigned lower[kRadix], half[kRadix], sums[kRadix / 32];
};
static_assert(kSortThreads == 2 * kRadix, "two threads a digit");

// The lanes with the same digit of `bits` bits as this one, of those in `on`.
__device__ __forceinline__ unsigned alike(unsigned digit, int bits, unsigned on) {
  unsigned same = on;
#pragma unroll
  for (int b = 0; b < kDigitBits; ++b) {
    if (b == bits) break;
    const bool set = digit >> b & 1;
    const unsigned with = __ballot_sync(~0u, set);
    same &= set ? with : ~with;
  }
  return same;
}

__device__ void sort_tokens(const EmbedGradArgs& p, SortShared& s, int rank, int blocks) {
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, digit_here = tid % kRadix, half = tid / kRadix;
  const int64_t warps = blocks * kSortWarps, each = ((p.N + warps - 1) / warps + 31) / 32 * 32;
  const int64_t begin = min((int64_t(rank) * kSortWarps + warp) * each, p.N), end = min(begin + each, p.N);
  const int radix = 1 << p.bits;
  constexpr int kBatch = 4;
  for (int pass = 0; pass < p.passes; ++pass) {
    const int32_t* const keys = pass == 0 ? p.tokens : pass & 1 ? p.keys[0] : p.keys[1];
    const int32_t* const places = pass & 1 ? p.places[0] : p.places[1];
    const int shift = pass * p.bits;
    // a token outside the table sorts behind all others, as V
    auto key_at = [&](int64_t i) {
      const int k = keys[i];
      return pass == 0 && unsigned(k) >= unsigned(p.V) ? p.V : k;
    };
    auto digit_of = [&](int key) { return unsigned(key) >> shift & (radix - 1); };
    for (int i = tid; i < kSortWarps * kRadix / 4; i += kSortThreads) reinterpret_cast<uint4*>(s.counts)[i] = make_uint4(0, 0, 0, 0);
    int key[kBatch], place[kBatch];
    unsigned same[kBatch];   // the lanes with the same digit
    auto load = [&](int64_t i0) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int64_t i = i0 + 32 * u + lane;
        key[u] = i < end ? key_at(i) : 0;
        place[u] = i < end ? pass == 0 ? int(i) : places[i] : 0;
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (i0 + 32 * u < end) same[u] = alike(digit_of(key[u]), p.bits, __ballot_sync(~0u, i0 + 32 * u + lane < end));
    };
    load(begin);
    __syncthreads();
    for (int64_t i0 = begin; i0 < end; i0 += 32 * kBatch) {
      if (i0 > begin) load(i0);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (i0 + 32 * u >= end) break;
        const bool in = i0 + 32 * u + lane < end;
        if (in && lane == __ffs(same[u]) - 1) s.counts[warp][digit_of(key[u])] += __popc(same[u]);
        __syncwarp();
      }
    }
    __syncthreads();
    // where each warp's first entry of a digit goes: behind all of lower digits, those of the blocks before and of the
    // warps before
    constexpr int kHalf = kSortWarps / 2;
    unsigned upto[kHalf], sum = 0;
#pragma unroll
    for (int w = 0; w < kHalf; ++w) upto[w] = s.counts[half * kHalf + w][digit_here];
#pragma unroll
    for (int w = 0; w < kHalf; ++w) {
      const unsigned here = upto[w];
      upto[w] = sum;
      sum += here;
    }
    if (half == 0) s.half[digit_here] = sum;
    __syncthreads();
    if (half == 1) s.total[digit_here] = s.half[digit_here] + sum;
    if (blocks > 1)
      cluster.sync();
    else
      __syncthreads();
    if (half == 0) {
      unsigned all = 0, before = 0;
      for (int r = 0; r < blocks; ++r) {
        const unsigned there = cluster.map_shared_rank(s.total, r)[digit_here];
        all += there;
        if (r < rank) before += there;
      }
      unsigned scan = all;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const unsigned other = __shfl_up_sync(~0u, scan, d);
        if (lane >= d) scan += other;
      }
      if (lane == 31) s.sums[warp] = scan;
      s.lower[digit_here] = scan - all + before;
    }
    __syncthreads();
    unsigned base = s.lower[digit_here] + (half ? s.half[digit_here] : 0);
    for (int w = 0; w < digit_here / 32; ++w) base += s.sums[w];
#pragma unroll
    for (int w = 0; w < kHalf; ++w) s.counts[half * kHalf + w][digit_here] = base + upto[w];
    __syncthreads();
    int32_t* const keys_out = pass & 1 ? p.keys[1] : p.keys[0];
    int32_t* const places_out = pass & 1 ? p.places[1] : p.places[0];
    for (int64_t i0 = begin; i0 < end; i0 += 32 * kBatch) {
      if (end - begin > 32 * kBatch) load(i0);   // (else the only batch is still there)
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (i0 + 32 * u >= end) break;
        const bool in = i0 + 32 * u + lane < end;
        const unsigned digit = digit_of(key[u]);
        unsigned to = 0;
        if (in) to = s.counts[warp][digit];
        __syncwarp();
        if (in && lane == __ffs(same[u]) - 1) s.counts[warp][digit] = to + __popc(same[u]);
        __syncwarp();
        to += __popc(same[u] & ((1u << lane) - 1));
        if (in) {
          keys_out[to] = key[u];
          places_out[to] = place[u];
        }
      }
    }
    // (what a pass wrote is read by all blocks in the next, which also replaces the totals)
    if (blocks > 1)
      cluster.sync();
    else
      __syncthreads();
  }
}

// Zeros to the rows from `first` on that no token has.  bitmap: of the rows that one has.
template <typename G>
__device__ void zero_rows(const EmbedGradArgs& p, unsigned* bitmap, int64_t first, int rows) {
  const int tid = threadIdx.x, lane = tid % 32;
  for (int i = tid; i < (rows + 31) / 32; i += kSortThreads) bitmap[i] = 0;
  __syncthreads();
#pragma unroll 4
  for (int64_t n = tid; n < p.N; n += kSortThreads) {
    const int64_t r = p.tokens[n] - first;
    if (r >= 0 && r < rows) atomicOr(&bitmap[r / 32], 1u << (r % 32));
  }
  __syncthreads();
  constexpr int kPer = 16 / int(sizeof(G));
  for (int r = tid / 32; r < rows; r += kSortWarps) {
    if (bitmap[r / 32] >> (r % 32) & 1) continue;
    G* const row = static_cast<G*>(p.dtable) + (first + r) * p.dtable_ld;
    const int lead = min(int((16 - reinterpret_cast<uintptr_t>(row) % 16) % 16 / sizeof(G)), p.D), whole = (p.D - lead) / kPer;
    for (int i = lane; i < whole; i += 32) *reinterpret_cast<uint4*>(row + lead + i * kPer) = make_uint4(0, 0, 0, 0);
    const int edge = lane < lead ? lane : lane + whole * kPer;
    if (edge < p.D && lane < p.D - whole * kPer) row[edge] = from_f32<G>(0.0f);
  }
  __syncthreads();
}

// A block per SM for an even range of rows each.  It lets the sort start before the last of them end, once what came before has ended.
template <typename G>
__global__ void __launch_bounds__(kSortThreads) embed_zeros_kernel(const EmbedGradArgs p) {
  __shared__ unsigned bitmap[kZeroRows / 32];
  pdl_entry();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t each = (p.V + gridDim.x - 1) / gridDim.x, begin = blockIdx.x * each, end = min(begin + each, int64_t(p.V));
  for (int64_t v = begin; v < end; v += kZeroRows) zero_rows<G>(p, bitmap, v, int(min(int64_t(kZeroRows), end - v)));
}

// AFTER_ZEROS: launched when every block of embed_zeros_kernel has passed its own wait, so what the call reads is there; the
// wait at the end is for that kernel itself, so that whatever waits for this one waits for both.
template <bool AFTER_ZEROS>
__global__ void __launch_bounds__(kSortThreads, 1) embed_sort_kernel(const EmbedGradArgs p) {
  extern __shared__ unsigned shared[];
  if (!AFTER_ZEROS) pdl_entry();
  sort_tokens(p, *reinterpret_cast<SortShared*>(shared), blockIdx.x, gridDim.x);
  if (AFTER_ZEROS) pdl_entry();
}

// ---- sums ----

// The row's sum: written, or added to what is there.  A row of fp32 is added to in L2, without waiting for what it holds
// (each element gets one addition, so nothing depends on an order).
template <typename E, bool WIDE, typename G>
__device__ __forceinline__ void finish_row(const EmbedGradArgs& p, const Columns<E, WIDE>& c, int key, const float (&sum)[kCols<E>]) {
  G* const row = static_cast<G*>(p.dtable) + key * p.dtable_ld;
  float v[kCols<E>];
#pragma unroll
  for (int k = 0; k < kCols<E>; ++k) v[k] = sum[k] * p.scale;
  if (!p.accumulate) {
    write_row<E, WIDE, G>(c, row, v);
  } else if constexpr (sizeof(G) == 4) {
#pragma unroll
    for (int k = 0; k < kCols<E>; k += WIDE ? 4 : 1) {
      if (!c.has(k)) continue;
      if constexpr (WIDE)
        asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(row + c(k)), "f"(v[k]), "f"(v[k + 1]), "f"(v[k + 2]), "f"(v[k + 3])
                     : "memory");
      else
        asm volatile("red.global.add.f32 [%0], %1;" ::"l"(row + c(k)), "f"(v[k]) : "memory");
    }
  } else {
    Row<E, WIDE, G> old;
    old.read(c, row);
#pragma unroll
    for (int k = 0; k < kCols<E>; ++k) v[k] += old[k];
    write_row<E, WIDE, G>(c, row, v);
  }
}

// A warp per chunk and slab.  The loads of four rows are in flight while four others are added.
template <typename E, typename G, bool WIDE>
__global__ void __launch_bounds__(kEmbedThreads) embed_sums_kernel(const EmbedGradArgs p) {
  pdl_entry();
  constexpr int K = kCols<E>, kBatch = 4;
  const int64_t w = int64_t(blockIdx.x) * (kEmbedThreads / 32) + threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  const int64_t chunk = w / p.slabs, first = chunk * p.chunk;
  if (chunk >= p.chunks) return;
  const Columns<E, WIDE> c(int(w % p.slabs), p.D);
  const int32_t *const keys = p.sorted_keys, *const places = p.sorted_places;
  const int L = int(min(int64_t(p.chunk), p.N - first));
  const int key = lane < L ? keys[first + lane] : p.V;
  const int place = lane < L ? places[first + lane] : 0;
  const int before = first > 0 ? keys[first - 1] : -1, after = first + L < p.N ? keys[first + L] : -1;
  const int count = __popc(__ballot_sync(~0u, key < p.V));   // entries with a row
  float* const parts = p.parts + chunk * 2 * p.pitch;
  float sum[K] = {};
  bool began = __shfl_sync(~0u, key, 0) != before;   // the run at hand began in this chunk
  Row<E, WIDE, E> rows[2][kBatch];
  auto load = [&](Row<E, WIDE, E> (&to)[kBatch], int j0) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int n = __shfl_sync(~0u, place, (j0 + u) & 31);
      if (j0 + u < count) to[u].read(c, static_cast<const E*>(p.dout) + n * p.dout_ld);
    }
  };
  auto add = [&](const Row<E, WIDE, E> (&from)[kBatch], int j0) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int j = j0 + u;
      if (j >= count) break;
#pragma unroll
      for (int k = 0; k < K; ++k) sum[k] += from[u][k];
      const int here = __shfl_sync(~0u, key, j), next = __shfl_sync(~0u, key, (j + 1) & 31);
      const bool ends = j + 1 < L ? next != here : after != here;
      if (j + 1 < L && !ends) continue;
      if (began && ends) {
        finish_row<E, WIDE, G>(p, c, here, sum);
      } else {
        write_row<E, WIDE, float>(c, parts + (began ? p.pitch : 0), sum);
      }
#pragma unroll
      for (int k = 0; k < K; ++k) sum[k] = 0.0f;
      began = true;
    }
  };
  load(rows[0], 0);
  for (int j0 = 0; j0 < count; j0 += 2 * kBatch) {
    load(rows[1], j0 + kBatch);
    add(rows[0], j0);
    load(rows[0], j0 + 2 * kBatch);
    add(rows[1], j0 + kBatch);
  }
}

// The runs that go on past the chunk where they began.  A block has up to kJoinSlabs slabs of 128 columns and looks at 32 chunks
// gridDim.x apart at a time; its warps are shares of `slabs` warps.  A run that ends in the next chunk is a share's own; of a longer
// one share q takes every shares-th partial row from the q-th on, and the first adds theirs up.  65,536 tokens, rows of 1024, in us for
// Zipf frequencies and for one token in all places (the whole call): 13.0, 112; a block for each chunk instead, most of which found
// nothing, 17.7, 187; two slabs of a block 18.9, 112; eight 17.6, 247.
constexpr int kJoinThreads = 512, kJoinWarps = kJoinThreads / 32, kJoinSlabs = 4, kJoinBlocks = 152 * 3;
template <typename G, bool WIDE>
__global__ void __launch_bounds__(kJoinThreads, 2) embed_join_kernel(const EmbedGradArgs p, int slabs) {
  __shared__ float parts[kJoinWarps][kSlab<float>];
  pdl_entry();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, share = warp / slabs, shares = kJoinWarps / slabs;
  const int32_t* const keys = p.sorted_keys;
  const Columns<float, WIDE> c(int(blockIdx.y) * slabs + warp % slabs, p.D);
  auto part = [&](int64_t at, int slot) {
    Row<float, WIDE, float> v = {};
    v.read(c, p.parts + (at * 2 + slot) * p.pitch);
    return v;
  };
  for (int64_t base = blockIdx.x; base < p.chunks - 1; base += 32 * int64_t(gridDim.x)) {
    const int64_t mine = base + lane * int64_t(gridDim.x), first = mine * p.chunk, next = first + p.chunk;
    int key = p.V, beyond = p.V;
    if (mine < p.chunks - 1) {
      const int start = keys[first], before = first > 0 ? keys[first - 1] : -1, after = keys[next];
      key = keys[next - 1];
      beyond = mine + 2 < p.chunks ? keys[next + p.chunk] : p.V;
      if (after != key || (start == key && before == key)) key = p.V;   // none, or it began earlier
    }
    unsigned runs = __ballot_sync(~0u, key < p.V && beyond != key);
    for (int i = 0; runs != 0; ++i, runs &= runs - 1) {
      if (i % shares != share) continue;
      const int from = __ffs(runs) - 1;
      const int64_t at = base + from * int64_t(gridDim.x);
      const Row<float, WIDE, float> v = part(at, 1), w = part(at + 1, 0);
      float sum[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) sum[k] = v[k] + w[k];
      finish_row<float, WIDE, G>(p, c, __shfl_sync(~0u, key, from), sum);
    }
    runs = __ballot_sync(~0u, key < p.V && beyond == key);
    for (; runs != 0; runs &= runs - 1) {
      const int from = __ffs(runs) - 1, run = __shfl_sync(~0u, key, from);
      const int64_t chunk = base + from * int64_t(gridDim.x);
      float sum[4] = {};
      if (share < shares) {
        auto add = [&](int64_t at, int slot) {
          const Row<float, WIDE, float> v = part(at, slot);
#pragma unroll
          for (int k = 0; k < 4; ++k) sum[k] += v[k];
        };
        if (share == 0) add(chunk, 1);
        // chunks from here on that begin with the run's token, 128 looked up at a time
        for (int64_t at = chunk + 1;; at += 128) {
          int count = 0;
          bool on[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int64_t i = at + q * 32 + lane;
            on[q] = i < p.chunks && keys[i * p.chunk] == run;
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const unsigned all = __ballot_sync(~0u, on[q]);
            if (count == q * 32) count += all == ~0u ? 32 : __ffs(~all) - 1;
          }
#pragma unroll 8
          for (int i = share; i < count; i += shares) add(at + i, 0);
          if (count < 128) break;
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) parts[warp][k * 32 + lane] = sum[k];
      __syncthreads();
      if (share == 0) {
        for (int q = 1; q < shares; ++q)
#pragma unroll
          for (int k = 0; k < 4; ++k) sum[k] += parts[q * slabs + warp][k * 32 + lane];
        finish_row<float, WIDE, G>(p, c, run, sum);
      }
      __syncthreads();
    }
  }
}

constexpr int64_t kMaxTokens = int64_t(1) << 27, kMaxRowsOfTable = int64_t(1) << 30, kMaxWidth = int64_t(1) << 23;

bool embed_sizes_ok(int64_t N, int64_t V, int64_t D) {
  if (N < 0 || N > kMaxTokens || V < 1 || V > kMaxRowsOfTable || D < 0 || D > kMaxWidth) return false;
  return N == 0 || (D + 127) / 128 <= kMaxExtent / N;   // a warp for each row's slabs
}
bool matrix_ok(const void* p, int dtype, int64_t D, int64_t ld) {
  return p && aligned_to(p, size_t(dtype_size(dtype))) && ld >= D && ld <= kMaxStride >> 16;
}
// Whether rows are whole pieces of `per` elements, which lie at multiples of their size (16 bytes at most).
bool wide(const void* p, int element, int64_t ld, int64_t D, int per) {
  const int bytes = per * element < 16 ? per * element : 16;
  return D % per == 0 && aligned_to(p, size_t(bytes)) && ld * element % bytes == 0;
}

// Few entries are cut into small chunks, so that there are warps for all SMs; the partial rows of small chunks cost more.
int chunk_of(int64_t N) { return N < 2048 ? 8 : N < 16384 ? 16 : 32; }

// Blocks of the sort's cluster: barriers between more blocks cost what few tokens do not earn (us with 1, 8, 16 blocks: 1024 tokens 9, -, -;
// 8192 37, 13, -; 32,768 -, 22, 18).
unsigned sort_blocks(int64_t N) { return N <= 2048 ? 1 : N <= 16384 ? 8 : 16; }

// Parts of the workspace, each a multiple of 16 bytes.
int64_t list_bytes(int64_t N) { return (N * 4 + 15) / 16 * 16; }
int64_t parts_bytes(int64_t N, int64_t D) { return (N + chunk_of(N) - 1) / chunk_of(N) * 2 * ((D + 3) / 4 * 4) * 4; }

template <typename E, typename T>
cudaError_t launch_embed_as(const EmbedArgs& p, cudaStream_t stream) {
  const dim3 grid(unsigned((p.N * p.slabs + kEmbedThreads / 32 - 1) / (kEmbedThreads / 32)));
  return wide(p.out, sizeof(E), p.out_ld, p.D, kCols<E>) && wide(p.table, sizeof(T), p.table_ld, p.D, kCols<E>)
             ? launch_pdl(embed_kernel<T, E, true>, grid, dim3(kEmbedThreads), 0, stream, p)
             : launch_pdl(embed_kernel<T, E, false>, grid, dim3(kEmbedThreads), 0, stream, p);
}
template <typename E>
cudaError_t launch_embed(EmbedArgs p, int table_dtype, cudaStream_t stream) {
  p.slabs = (p.D + kSlab<E> - 1) / kSlab<E>;
  return table_dtype == GEM_F32    ? launch_embed_as<E, float>(p, stream)
         : table_dtype == GEM_BF16 ? launch_embed_as<E, __nv_bfloat16>(p, stream)
                                   : launch_embed_as<E, __half>(p, stream);
}

template <bool AFTER_ZEROS>
cudaError_t launch_sort(const EmbedGradArgs& p, cudaStream_t stream) {
  const cudaError_t e = allow_shared<embed_sort_kernel<AFTER_ZEROS>, true>(sizeof(SortShared));
  if (e != cudaSuccess) return e;
  const unsigned blocks = sort_blocks(p.N);
  return launch_cluster_pdl(embed_sort_kernel<AFTER_ZEROS>, blocks, kSortThreads, blocks, sizeof(SortShared), stream, p);
}

template <typename E, typename G>
cudaError_t launch_embed_grad_as(EmbedGradArgs p, cudaStream_t stream) {
  constexpr int kWarps = kEmbedThreads / 32;
  p.slabs = (p.D + kSlab<E> - 1) / kSlab<E>;
  cudaError_t e = cudaSuccess;
  if (!p.accumulate) e = launch_pdl(embed_zeros_kernel<G>, dim3(kZeroBlocks), dim3(kSortThreads), 0, stream, p);
  if (e != cudaSuccess || p.N == 0) return e;
  e = p.accumulate ? launch_sort<false>(p, stream) : launch_sort<true>(p, stream);
  if (e != cudaSuccess) return e;
  const dim3 grid(unsigned((int64_t(p.chunks) * p.slabs + kWarps - 1) / kWarps));
  e = wide(p.dout, sizeof(E), p.dout_ld, p.D, kCols<E>) && wide(p.dtable, sizeof(G), p.dtable_ld, p.D, kCols<E>)
          ? launch_pdl(embed_sums_kernel<E, G, true>, grid, dim3(kEmbedThreads), 0, stream, p)
          : launch_pdl(embed_sums_kernel<E, G, false>, grid, dim3(kEmbedThreads), 0, stream, p);
  if (e != cudaSuccess || p.chunks == 1) return e;
  const int columns = kSlab<float>, slabs = std::min((p.D + columns - 1) / columns, kJoinSlabs);
  const int groups = (p.D + columns * slabs - 1) / (columns * slabs);   // (at most 2^14)
  const dim3 joins(unsigned(std::min(p.chunks - 1, std::max(kJoinBlocks / groups, 1))), unsigned(groups));
  return wide(p.dtable, sizeof(G), p.dtable_ld, p.D, kCols<float>) ? launch_pdl(embed_join_kernel<G, true>, joins, dim3(kJoinThreads), 0, stream, p, slabs)
                                                                   : launch_pdl(embed_join_kernel<G, false>, joins, dim3(kJoinThreads), 0, stream, p, slabs);
}
template <typename E>
cudaError_t launch_embed_grad(const EmbedGradArgs& p, int grad_dtype, cudaStream_t stream) {
  return grad_dtype == GEM_F32    ? launch_embed_grad_as<E, float>(p, stream)
         : grad_dtype == GEM_BF16 ? launch_embed_grad_as<E, __nv_bfloat16>(p, stream)
                                  : launch_embed_grad_as<E, __half>(p, stream);
}

}  // namespace
}  // namespace lm
}  // namespace gem

using namespace gem;
using namespace gem::lm;

extern "C" {

int gem_embed(int table_dtype, int dtype, int64_t N, int64_t V, int64_t D, const void* table,
              int64_t table_ld, const int32_t* tokens, float scale, void* out, int64_t out_ld,
              void* stream) {
  if (!dtype_ok(table_dtype) || !dtype_ok(dtype) || !embed_sizes_ok(N, V, D)) return GEM_EINVAL;
  if (N == 0 || D == 0) return GEM_OK;
  if (!matrix_ok(table, table_dtype, D, table_ld) || !matrix_ok(out, dtype, D, out_ld) || !array_ok(tokens)) return GEM_EINVAL;
  const EmbedArgs p = {table, out, table_ld, out_ld, N, int(V), int(D), 0, tokens, scale};
  return launch_status(BY_TYPE(launch_embed, p, table_dtype, static_cast<cudaStream_t>(stream)));
}

int64_t gem_embed_workspace(int64_t N, int64_t V, int64_t D) {
  if (!embed_sizes_ok(N, V, D)) return -1;
  return 4 * list_bytes(N) + parts_bytes(N, D);
}

int gem_embed_grad(int dtype, int grad_dtype, int64_t N, int64_t V, int64_t D, const void* dout,
                   int64_t dout_ld, const int32_t* tokens, float scale, int accumulate,
                   void* dtable, int64_t dtable_ld, void* workspace, void* stream) {
  if (!dtype_ok(dtype) || !dtype_ok(grad_dtype) || !embed_sizes_ok(N, V, D) || (accumulate & ~1)) return GEM_EINVAL;
  if (D == 0 || (N == 0 && accumulate)) return GEM_OK;
  if (!matrix_ok(dtable, grad_dtype, D, dtable_ld)) return GEM_EINVAL;
  if (N > 0 && (!matrix_ok(dout, dtype, D, dout_ld) || !array_ok(tokens))) return GEM_EINVAL;
  if (N > 0 && (!workspace || !aligned_to(workspace, 16))) return GEM_EINVAL;
  EmbedGradArgs p = {};
  p.dout = dout;
  p.dtable = dtable;
  p.dout_ld = dout_ld;
  p.dtable_ld = dtable_ld;
  p.N = N;
  p.V = int(V);
  p.D = int(D);
  p.tokens = tokens;
  p.scale = scale;
  p.accumulate = accumulate != 0;
  char* space = static_cast<char*>(workspace);
  if (N > 0)
    for (int i = 0; i < 4; ++i, space += list_bytes(N)) (i < 2 ? p.keys : p.places)[i % 2] = reinterpret_cast<int32_t*>(space);
  p.parts = reinterpret_cast<float*>(space);
  int bits = 1;
  while (V >> bits) ++bits;   // of V, the key of tokens outside the table
  p.passes = (bits + kDigitBits - 1) / kDigitBits;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.sorted_keys = p.keys[(p.passes - 1) & 1];
  p.sorted_places = p.places[(p.passes - 1) & 1];
  p.chunk = chunk_of(N);
  p.chunks = int((N + p.chunk - 1) / p.chunk);
  p.pitch = int((D + 3) / 4 * 4);
  return launch_status(BY_TYPE(launch_embed_grad, p, grad_dtype, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
