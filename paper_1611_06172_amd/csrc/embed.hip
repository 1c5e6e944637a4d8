// Rows of a matrix by word, scaled, and the gradient of that: rows of dy summed
// by word.
//
//   y_i = scale W[id_i]                       (0 where id_i is absent)
//   G_v = scale sum over {i : id_i = v} dy_i  (+ G_v when accumulating)
//
// Both move bytes and compute next to nothing: the lookup reads each different
// row once (again from the caches) and writes n rows; the gradient reads n rows
// and writes V, or reads and writes those that occur.
//
// The gradient's sums have one order, so that the same call gives the same bits:
// the positions are sorted by word (stable), the sorted list is cut into chunks
// of equal length, a wavefront adds a chunk's rows in registers and writes every
// word that lies within the chunk; words that go over a chunk's end leave a
// partial sum for each chunk they touch, and a second kernel adds these in the
// order of the chunks. A frequent word's tens of thousands of rows are thus
// added by as many wavefronts as they take chunks, without atomics.
#include "embed.h"
#include "head_types.h"
#include "kernel_args.h"

namespace w2v {
namespace {

constexpr int kE = 8;             // elements a lane takes of a row
constexpr int kBlock = 256;
constexpr int kBlockPacks = 1024;  // packs of a block's rows
constexpr int kMaxGrid = 1 << 22;
constexpr int kWave = 64;

__device__ __forceinline__ uint64_t lanes_below(int lane) { return (1ull << lane) - 1; }

// How rows of D elements are taken apart into packs of kE. The last pack of a
// row begins early (its first elements are also its neighbour's), so that all
// are loaded and stored whole.
struct RowPacks {
  int32_t n, D, per_row, rows_a_block;
  Divisor by_row;
};

RowPacks row_packs(int32_t n, int32_t D) {
  RowPacks p;
  p.n = n;
  p.D = D;
  p.per_row = (int32_t)(((int64_t)D + kE - 1) / kE);
  p.rows_a_block = p.per_row >= kBlockPacks ? 1 : kBlockPacks / p.per_row;
  p.by_row = divisor_of((uint32_t)p.per_row);
  return p;
}

int row_blocks(const RowPacks& p) {
  const int64_t blocks = ((int64_t)p.n + p.rows_a_block - 1) / p.rows_a_block;
  return (int)(blocks < kMaxGrid ? blocks : kMaxGrid);
}

// kE elements, or for rows shorter than that (SHORT) the `left` there are.
template <bool SHORT, typename T>
__device__ __forceinline__ Pack<T, kE> get(const T* p, int left) {
  if constexpr (SHORT) return load_some<T, kE>(p, left);
  return load_pack<T, kE>(p);
}
template <bool SHORT, typename T>
__device__ __forceinline__ void put(T* p, int left, const Pack<T, kE>& v) {
  if constexpr (SHORT) return store_some<T, kE>(p, left, v);
  return store_pack<T, kE>(p, v);
}

// Column where pack `i` of a row begins.
template <bool SHORT>
__device__ __forceinline__ int pack_column(int i, int D) {
  return SHORT || i * kE + kE <= D ? i * kE : D - kE;
}

// Four packs of a thread are in flight at once; an absent word's are loaded from
// row 0 and not used, so that no load has a test of its own.
template <typename TI, typename TO, bool SHORT>
__global__ __launch_bounds__(kBlock) void k_embed(EmbedArgs a, RowPacks p) {
  const TI* w = (const TI*)a.weight;
  TO* y = (TO*)a.y;
  for (int64_t b = (int64_t)blockIdx.x * p.rows_a_block; b < a.n;
       b += (int64_t)gridDim.x * p.rows_a_block) {
    const int rows = (int)(a.n - b < p.rows_a_block ? a.n - b : p.rows_a_block);
    const int packs = rows * p.per_row;
    for (int first = 0; first < packs; first += kBlockPacks) {
      int row[4], col[4];
      int32_t id[4];
#pragma unroll
      for (int u = 0; u < 4; u++) {
        const int i = first + u * kBlock + (int)threadIdx.x;
        const int at = i < packs ? i : packs - 1;
        row[u] = (int)divided((uint32_t)at, p.by_row);
        col[u] = pack_column<SHORT>(at - row[u] * p.per_row, a.D);
        id[u] = a.ids[b + row[u]];
      }
      Pack<TI, kE> in[4];
#pragma unroll
      for (int u = 0; u < 4; u++) {
        const bool there = id[u] >= 0 && id[u] < a.V;
        if (!there && id[u] != -1) report_row(a.status);
        in[u] = get<SHORT>(w + (there ? id[u] : 0) * a.ldw + col[u], a.D - col[u]);
        if (!there) id[u] = -1;
      }
#pragma unroll
      for (int u = 0; u < 4; u++) {
        if (first + u * kBlock + (int)threadIdx.x >= packs) continue;
        Pack<TO, kE> out;
#pragma unroll
        for (int e = 0; e < kE; e++)
          out.v[e] = from_f32<TO>(id[u] >= 0 ? a.scale * to_f32(in[u].v[e]) : 0.0f);
        put<SHORT>(y + (b + row[u]) * a.ldy + col[u], a.D - col[u], out);
      }
    }
  }
}

// ------------------------------------------------------------- gradient --

// Rows of zeros, in the packs of the block `b` of `grid`.
template <typename T>
__device__ __forceinline__ void clear_rows(T* g, int64_t ld, const RowPacks& p, int64_t b,
                                           int64_t grid) {
  Pack<T, kE> zero;
#pragma unroll
  for (int e = 0; e < kE; e++) zero.v[e] = T(0.0f);
  const bool whole = p.D >= kE;
  for (b *= p.rows_a_block; b < p.n; b += grid * p.rows_a_block) {
    const int rows = (int)(p.n - b < p.rows_a_block ? p.n - b : p.rows_a_block);
    const int packs = rows * p.per_row;
    for (int i = threadIdx.x; i < packs; i += (int)blockDim.x) {
      const int row = (int)divided((uint32_t)i, p.by_row);
      const int pack = i - row * p.per_row;
      if (whole) {
        store_pack<T, kE>(g + (b + row) * ld + pack_column<false>(pack, p.D), zero);
      } else {
        store_some<T, kE>(g + (b + row) * ld, p.D, zero);
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_embed_clear(T* g, int64_t ld, RowPacks p) {
  clear_rows<T>(g, ld, p, blockIdx.x, gridDim.x);
}

// The sort's key of a word: itself, V where there is none.
__device__ __forceinline__ uint32_t word_key(int32_t id, int32_t V, int32_t* status) {
  if (id >= 0 && id < V) return (uint32_t)id;
  if (id != -1) report_row(status);
  return (uint32_t)V;
}

__global__ __launch_bounds__(kBlock) void k_embed_keys(const int32_t* ids, int32_t n, int32_t V,
                                                       uint32_t* keys, int32_t* status) {
  const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  if (i < n) keys[i] = word_key(ids[i], V, status);
}

// Up to kSortMax words sorted by one block, stably, by digits of six bits as in
// radix_sort.hip, but with the elements in registers and the counters of a
// wavefront's 64 digits in its 64 lanes: lane l counts digit l. Blocks after the
// first clear the gradient meanwhile.
constexpr int kSortWaves = 16;
constexpr int kSortGroups = 8;
constexpr int kSortMax = kSortWaves * kSortGroups * kWave;  // 8,192

// Lanes whose digit is d, from the ballots of the digits' six bits.
__device__ __forceinline__ uint64_t lanes_with(const uint64_t (&set)[6], int d) {
  uint64_t m = ~0ull;
#pragma unroll
  for (int b = 0; b < 6; b++) m &= (d >> b) & 1 ? set[b] : ~set[b];
  return m;
}

template <typename TG>
__global__ __launch_bounds__(kSortWaves* kWave) void k_embed_sort(EmbedBackwardArgs a, int bits,
                                                                uint32_t* keys, int32_t* at,
                                                                RowPacks p) {
  if (blockIdx.x > 0) {
    clear_rows<TG>((TG*)a.grad, a.ldg, p, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  __shared__ uint32_t s_key[kSortMax];
  __shared__ uint16_t s_at[kSortMax];
  __shared__ int s_count[kSortWaves * kWave];  // [digit][wave], then its start
  __shared__ int s_total[kSortWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t key[kSortGroups];
  int from[kSortGroups];
#pragma unroll
  for (int g = 0; g < kSortGroups; g++) {
    const int i = (wave * kSortGroups + g) * kWave + lane;
    from[g] = i;
    // past the end: behind everything, since the sort is stable
    key[g] = i < a.n ? word_key(a.ids[i], a.V, a.status) : ~0u;
  }
  for (int shift = 0; shift < bits; shift += 6) {
    int count = 0, rank[kSortGroups];
#pragma unroll
    for (int g = 0; g < kSortGroups; g++) {
      const int d = (int)(key[g] >> shift) & 63;
      uint64_t set[6];
#pragma unroll
      for (int b = 0; b < 6; b++) set[b] = __ballot((d >> b) & 1);
      rank[g] = __shfl(count, d) + __popcll(lanes_with(set, d) & lanes_below(lane));
      count += __popcll(lanes_with(set, lane));
    }
    s_count[lane * kSortWaves + wave] = count;
    __syncthreads();
    // exclusive prefix sums over digits, and within a digit over the wavefronts
    const int c = s_count[threadIdx.x];
    int sum = c;
#pragma unroll
    for (int off = 1; off < kWave; off *= 2) {
      const int below = __shfl_up(sum, off);
      if (lane >= off) sum += below;
    }
    if (lane == kWave - 1) s_total[wave] = sum;
    __syncthreads();
    for (int w = 0; w < wave; w++) sum += s_total[w];
    s_count[threadIdx.x] = sum - c;
    __syncthreads();
#pragma unroll
    for (int g = 0; g < kSortGroups; g++) {
      const int d = (int)(key[g] >> shift) & 63;
      const int to = s_count[d * kSortWaves + wave] + rank[g];
      s_key[to] = key[g];
      s_at[to] = (uint16_t)from[g];
    }
    __syncthreads();
#pragma unroll
    for (int g = 0; g < kSortGroups; g++) {
      const int i = (wave * kSortGroups + g) * kWave + lane;
      key[g] = s_key[i];
      from[g] = s_at[i];
    }
    __syncthreads();
  }
#pragma unroll
  for (int g = 0; g < kSortGroups; g++) {
    const int i = (wave * kSortGroups + g) * kWave + lane;
    if (i < a.n) {
      keys[i] = key[g];
      at[i] = from[g];
    }
  }
}

// The columns of a row over the lanes of one wavefront or, for long rows, of
// several (blockIdx.y); lanes past the last pack take no part.
struct Columns {
  int32_t lanes, tiles;  // lanes a wavefront uses, wavefronts a row takes
  int64_t ld;            // floats of a partial sum
};

struct LaneColumns {
  int first, skip, left;  // first element, how many are the neighbour's, how many there are
  bool there;
};

template <bool SHORT>
__device__ __forceinline__ LaneColumns lane_columns(const Columns& c, int32_t D) {
  const int lane = threadIdx.x & 63;
  const int pack = (int)blockIdx.y * c.lanes + lane;
  LaneColumns l;
  l.there = lane < c.lanes && pack * kE < D;
  l.first = l.there ? pack_column<SHORT>(pack, D) : 0;
  l.skip = l.there ? pack * kE - l.first : 0;
  l.left = D - l.first;
  return l;
}

// One word's finished sum. Of a pack that begins early only the lane's own
// elements are written, since another wavefront may add to the others.
template <bool SHORT, typename TG>
__device__ __forceinline__ void write_word(const EmbedBackwardArgs& a, uint32_t word,
                                           const LaneColumns& l, const Pack<float, kE>& sum) {
  if (!l.there) return;
  TG* g = (TG*)a.grad + word * a.ldg + l.first;
  Pack<TG, kE> out;
  if (a.accumulate) {
    const Pack<TG, kE> old = get<SHORT>(g, l.left);
#pragma unroll
    for (int e = 0; e < kE; e++) out.v[e] = from_f32<TG>(fmaf(a.scale, sum.v[e], to_f32(old.v[e])));
  } else {
#pragma unroll
    for (int e = 0; e < kE; e++) out.v[e] = from_f32<TG>(a.scale * sum.v[e]);
  }
  if (l.skip == 0) {
    put<SHORT>(g, l.left, out);
  } else {
#pragma unroll
    for (int e = 0; e < kE; e++)
      if (e >= l.skip) g[e] = out.v[e];
  }
}

// One wavefront a chunk of `chunk` (up to 64) sorted positions: the chunk's keys
// are in its lanes, kAhead rows in flight. `head` and `tail`: partial sums of the
// word that comes into the chunk from the one before, and of the one that goes
// over its end and began within.
constexpr int kAhead = 8;

template <typename TI, typename TG, bool SHORT>
__global__ __launch_bounds__(kBlock) void k_embed_sums(EmbedBackwardArgs a, Columns cols,
                                                       const uint32_t* keys, const int32_t* at,
                                                       int chunk, float* head, float* tail) {
  const int lane = threadIdx.x & 63;
  const int64_t k = (int64_t)blockIdx.x * (kBlock / kWave) + (threadIdx.x >> 6);
  const int64_t begin = k * chunk;
  if (begin >= a.n) return;
  const int size = (int)(a.n - begin < chunk ? a.n - begin : chunk);
  const LaneColumns l = lane_columns<SHORT>(cols, a.D);
  const uint32_t V = (uint32_t)a.V;
  const uint32_t key = lane < size ? keys[begin + lane] : V;
  const int32_t row = lane < size ? at[begin + lane] : 0;
  const uint32_t before = begin > 0 ? keys[begin - 1] : ~0u;
  const uint32_t after = begin + size < a.n ? keys[begin + size] : ~0u;
  // words only: absent ones come last
  const int used = __popcll(__ballot(lane < size && key < V));
  if (used == 0) return;
  const TI* dy = (const TI*)a.dy + l.first;
  Pack<float, kE> sum{};
  uint32_t word = (uint32_t)__builtin_amdgcn_readfirstlane((int)key);
  bool came = word == before;
  for (int j0 = 0; j0 < used; j0 += kAhead) {
    Pack<TI, kE> in[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; u++) {
      const int j = j0 + u < used ? j0 + u : used - 1;
      const int32_t r = __builtin_amdgcn_readlane(row, j);
      in[u] = get<SHORT>(dy + r * a.lddy, l.left);
    }
#pragma unroll
    for (int u = 0; u < kAhead; u++) {
      if (j0 + u >= used) break;
      const uint32_t next = (uint32_t)__builtin_amdgcn_readlane((int)key, j0 + u);
      if (next != word) {
        if (came) {
          if (l.there) put<SHORT>(head + k * cols.ld + l.first, l.left, sum);
        } else {
          write_word<SHORT, TG>(a, word, l, sum);
        }
        word = next;
        came = false;
        sum = Pack<float, kE>{};
      }
#pragma unroll
      for (int e = 0; e < kE; e++) sum.v[e] += to_f32(in[u].v[e]);
    }
  }
  const bool goes = word == after;
  if (!came && !goes) {
    write_word<SHORT, TG>(a, word, l, sum);
  } else if (l.there) {
    put<SHORT>((came ? head : tail) + k * cols.ld + l.first, l.left, sum);
  }
}

// Joins the partial sums of the word that goes over chunk k's end and began in
// it: one block a chunk, most of which have none. The word's last chunk is the
// first one behind which another word follows.
template <typename TG, bool SHORT>
__device__ __forceinline__ void join_word(const EmbedBackwardArgs& a, const Columns& cols,
                                          const uint32_t* keys, int chunk, int64_t k,
                                          const float* head, const float* tail) {
  const int64_t begin = k * chunk, end = begin + chunk;
  const uint32_t word = keys[end - 1];
  if (word >= (uint32_t)a.V || keys[end] != word) return;
  if (keys[begin] == word && begin > 0 && keys[begin - 1] == word) return;
  __shared__ int s_last;
  __shared__ float s_sum[kBlock / kWave][kWave][kE];
  __syncthreads();
  if (threadIdx.x == 0) s_last = 0x7fffffff;
  __syncthreads();
  // the word ends in chunk k + 1 + s_last
  for (int64_t from = 0;; from += kBlock) {
    const int64_t stop = (k + 2 + from + threadIdx.x) * chunk;
    if (stop >= a.n || keys[stop] != word) atomicMin(&s_last, (int)(from + threadIdx.x));
    __syncthreads();
    const int found = s_last;
    __syncthreads();
    if (found != 0x7fffffff) break;
  }
  constexpr int kWaves = kBlock / kWave;
  const int count = s_last + 1;
  const LaneColumns l = lane_columns<SHORT>(cols, a.D);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float* from = head + (k + 1) * cols.ld + l.first;
  Pack<float, kE> sum{};
  for (int j0 = wave; j0 < count; j0 += kAhead * kWaves) {
    Pack<float, kE> in[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; u++) {
      const int j = j0 + u * kWaves;
      in[u] = get<SHORT>(from + (j < count ? j : j0) * cols.ld, l.left);
    }
#pragma unroll
    for (int u = 0; u < kAhead; u++) {
      if (j0 + u * kWaves >= count) break;
#pragma unroll
      for (int e = 0; e < kE; e++) sum.v[e] += in[u].v[e];
    }
  }
#pragma unroll
  for (int e = 0; e < kE; e++) s_sum[wave][lane][e] = sum.v[e];
  __syncthreads();
  if (wave != 0) return;
  sum = get<SHORT>(tail + k * cols.ld + l.first, l.left);
#pragma unroll
  for (int w = 0; w < kWaves; w++)
#pragma unroll
    for (int e = 0; e < kE; e++) sum.v[e] += s_sum[w][lane][e];
  write_word<SHORT, TG>(a, word, l, sum);
}

template <typename TG, bool SHORT>
__global__ __launch_bounds__(kBlock) void k_embed_join(EmbedBackwardArgs a, Columns cols,
                                                       const uint32_t* keys, int chunk,
                                                       const float* head, const float* tail) {
  for (int64_t k = blockIdx.x; (k + 1) * chunk < a.n; k += gridDim.x)
    join_word<TG, SHORT>(a, cols, keys, chunk, k, head, tail);
}

Columns columns_of(int32_t D) {
  const int64_t packs = ((int64_t)D + kE - 1) / kE;
  Columns c;
  c.tiles = (int32_t)((packs + kWave - 1) / kWave);
  c.lanes = (int32_t)((packs + c.tiles - 1) / c.tiles);
  c.ld = packs * kE;
  return c;
}

// Long chunks leave few partial sums, short ones fill the card.
int chunk_of(int32_t n) {
  int chunk = kWave;
  while (chunk > kAhead && (int64_t)n / chunk < 4096) chunk /= 2;
  return chunk;
}

int key_bits(int32_t V) {
  int bits = 1;
  while ((V >> bits) != 0) bits++;
  return bits;
}

size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }

struct Workspace {
  uint32_t *keys, *sorted;
  int32_t* at;
  float *head, *tail;
  void* temp;
  size_t bytes;
};

Workspace lay_out(void* base, int32_t n, int32_t D) {
  Workspace w{};
  size_t used = 0;
  const auto take = [&](size_t bytes) {
    char* p = (char*)base + used;
    used += aligned(bytes);
    return (void*)p;
  };
  const int64_t chunks = ((int64_t)n + chunk_of(n) - 1) / chunk_of(n);
  w.sorted = (uint32_t*)take(4 * (size_t)n);
  w.at = (int32_t*)take(4 * (size_t)n);
  const size_t partial = 4 * (size_t)chunks * (size_t)columns_of(D).ld;
  w.head = (float*)take(partial);
  w.tail = (float*)take(partial);
  if (n > kSortMax) {
    w.keys = (uint32_t*)take(4 * (size_t)n);
    w.temp = take(radix_sort_temp_bytes(n, 4));
  }
  w.bytes = used;
  return w;
}

template <typename TI, typename TG, bool SHORT>
hipError_t launch_sums(const EmbedBackwardArgs& a, const Workspace& w, hipStream_t s) {
  const Columns cols = columns_of(a.D);
  const int chunk = chunk_of(a.n);
  const int64_t chunks = ((int64_t)a.n + chunk - 1) / chunk;
  const dim3 grid((unsigned)((chunks + 3) / 4), (unsigned)cols.tiles);
  hipLaunchKernelGGL((k_embed_sums<TI, TG, SHORT>), grid, dim3(kBlock), 0, s, a, cols, w.sorted,
                     w.at, chunk, w.head, w.tail);
  const int64_t joins = chunks - 1 < kMaxGrid ? chunks - 1 : kMaxGrid;
  if (joins > 0)
    hipLaunchKernelGGL((k_embed_join<TG, SHORT>), dim3((unsigned)joins, (unsigned)cols.tiles),
                       dim3(kBlock), 0, s, a, cols, w.sorted, chunk, w.head, w.tail);
  return hipGetLastError();
}

template <typename TI, typename TG>
hipError_t launch_sums(const EmbedBackwardArgs& a, const Workspace& w, hipStream_t s) {
  return a.D < kE ? launch_sums<TI, TG, true>(a, w, s) : launch_sums<TI, TG, false>(a, w, s);
}

template <typename TG>
hipError_t launch_backward(const EmbedBackwardArgs& a, void* workspace, hipStream_t s) {
  const RowPacks p = row_packs(a.V, a.D);
  const int clear = a.accumulate ? 0 : row_blocks(p);
  if (a.n == 0) {
    if (clear > 0)
      hipLaunchKernelGGL(k_embed_clear<TG>, dim3(clear), dim3(kBlock), 0, s, (TG*)a.grad, a.ldg,
                         p);
    return hipGetLastError();
  }
  const Workspace w = lay_out(workspace, a.n, a.D);
  const int bits = key_bits(a.V);
  if (a.n <= kSortMax) {
    // four times the threads of k_embed_clear's blocks
    hipLaunchKernelGGL(k_embed_sort<TG>, dim3(1 + (clear + 3) / 4), dim3(kSortWaves * kWave), 0,
                       s, a, bits, w.sorted, w.at, p);
  } else {
    if (clear > 0)
      hipLaunchKernelGGL(k_embed_clear<TG>, dim3(clear), dim3(kBlock), 0, s, (TG*)a.grad, a.ldg,
                         p);
    hipLaunchKernelGGL(k_embed_keys, dim3((unsigned)(((int64_t)a.n + kBlock - 1) / kBlock)),
                       dim3(kBlock), 0, s, a.ids, a.n, a.V, w.keys, a.status);
    const hipError_t e =
        radix_sort_pairs(w.keys, nullptr, w.sorted, w.at, a.n, bits, w.temp, s);
    if (e != hipSuccess) return e;
  }
  switch (a.dtype) {
    case W2V_DTYPE_F32:
      return launch_sums<float, TG>(a, w, s);
    case W2V_DTYPE_BF16:
      return launch_sums<bf16_t, TG>(a, w, s);
    default:
      return launch_sums<f16_t, TG>(a, w, s);
  }
}

template <typename TI, typename TO>
hipError_t launch_lookup(const EmbedArgs& a, hipStream_t s) {
  const RowPacks p = row_packs(a.n, a.D);
  const dim3 grid(row_blocks(p));
  if (a.D < kE) {
    hipLaunchKernelGGL((k_embed<TI, TO, true>), grid, dim3(kBlock), 0, s, a, p);
  } else {
    hipLaunchKernelGGL((k_embed<TI, TO, false>), grid, dim3(kBlock), 0, s, a, p);
  }
  return hipGetLastError();
}

template <typename TI>
hipError_t launch_lookup(const EmbedArgs& a, hipStream_t s) {
  switch (a.out_dtype) {
    case W2V_DTYPE_F32:
      return launch_lookup<TI, float>(a, s);
    case W2V_DTYPE_BF16:
      return launch_lookup<TI, bf16_t>(a, s);
    default:
      return launch_lookup<TI, f16_t>(a, s);
  }
}

}  // namespace

hipError_t launch_embed(const EmbedArgs& a, hipStream_t s) {
  switch (a.dtype) {
    case W2V_DTYPE_F32:
      return launch_lookup<float>(a, s);
    case W2V_DTYPE_BF16:
      return launch_lookup<bf16_t>(a, s);
    default:
      return launch_lookup<f16_t>(a, s);
  }
}

size_t embed_backward_workspace_bytes(int32_t n, int32_t V, int32_t D) {
  return n == 0 ? 0 : lay_out(nullptr, n, D).bytes;
}

hipError_t launch_embed_backward(const EmbedBackwardArgs& a, void* workspace, hipStream_t s) {
  switch (a.grad_dtype) {
    case W2V_DTYPE_F32:
      return launch_backward<float>(a, workspace, s);
    case W2V_DTYPE_BF16:
      return launch_backward<bf16_t>(a, workspace, s);
    default:
      return launch_backward<f16_t>(a, workspace, s);
  }
}

}  // namespace w2v
