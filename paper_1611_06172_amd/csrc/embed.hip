// Rows of a matrix by word, scaled, and the gradient of that: rows of dy summed
// by word.
//
//   y_i = scale W[id_i]                       (0 where id_i is absent)
//   G_v = scale sum over {i : id_i = v} dy_i  (+ G_v when accumulating)
//
// Both move bytes and compute next to nothing: the lookup reads each different
// row once (again from the caches) and writes n rows; the gradient reads n rows
// and writes V, or reads and writes those that occur. Measured: 10^6 rows of 300 from
// 10^6, fp32 to bf16, 202 us (795 MB at 3.9 TB/s); their gradient, bf16 to fp32, 444 us
// (1.8 GB at 4.1 TB/s: sort and clearing 240, sums 171, joins 17); 4,096 rows of 300
// fp32 into 71,290, 26 us (91 MB at 3.5 TB/s); a lookup of 64 rows 9 us, 2.4 of them in
// the kernel.
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

namespace w2v {
namespace {

constexpr int kE = 8;             // elements a lane takes of a row
constexpr int kBlock = 256;
constexpr int kPacks = 2;  // packs a thread has in flight (1: 220 us, 4: 207, where 2 take 204)
constexpr int kBlockPacks = kPacks * kBlock;
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

// The same of a row that is read once, and of rows that are more than the caches
// hold (`large`).
template <bool SHORT, typename T>
__device__ __forceinline__ Pack<T, kE> get_once(const T* p, int left) {
  if constexpr (SHORT) return load_some<T, kE>(p, left);
  return load_once<Pack<T, kE>>(p);
}
template <bool SHORT, typename T>
__device__ __forceinline__ void put_once(T* p, int left, const Pack<T, kE>& v, bool large) {
  if constexpr (SHORT) return store_some<T, kE>(p, left, v);
  if (large) return store_once(p, v);
  return store_pack<T, kE>(p, v);
}

// Column where pack `i` of a row begins.
template <bool SHORT>
__device__ __forceinline__ int pack_column(int i, int D) {
  return SHORT || i * kE + kE <= D ? i * kE : D - kE;
}

// The packs of a thread are in flight at once; an absent word's are loaded from
// row 0 and not used, so that no load has a test of its own.
template <typename TI, typename TO, bool SHORT>
__global__ __launch_bounds__(kBlock) void k_embed(EmbedArgs a, RowPacks p) {
  const TI* w = (const TI*)a.weight;
  TO* y = (TO*)a.y;
  // rows of W stay in the L2s (32 MB) rather than y: 10^6 rows of 300 from 10^6,
  // fp32 to bf16, in 202 us instead of 244
  const bool large = (int64_t)a.n * a.D * (int64_t)sizeof(TO) > (32 << 20);
  for (int64_t b = (int64_t)blockIdx.x * p.rows_a_block; b < a.n;
       b += (int64_t)gridDim.x * p.rows_a_block) {
    const int rows = (int)(a.n - b < p.rows_a_block ? a.n - b : p.rows_a_block);
    const int packs = rows * p.per_row;
    for (int first = 0; first < packs; first += kBlockPacks) {
      int row[kPacks], col[kPacks];
      int32_t id[kPacks];
#pragma unroll
      for (int u = 0; u < kPacks; u++) {
        const int i = first + u * kBlock + (int)threadIdx.x;
        const int at = i < packs ? i : packs - 1;
        row[u] = (int)divided((uint32_t)at, p.by_row);
        col[u] = pack_column<SHORT>(at - row[u] * p.per_row, a.D);
        id[u] = a.ids[b + row[u]];
      }
      Pack<TI, kE> in[kPacks];
#pragma unroll
      for (int u = 0; u < kPacks; u++) {
        const bool there = id[u] >= 0 && id[u] < a.V;
        if (!there && id[u] != -1) report_row(a.status);
        in[u] = get<SHORT>(w + (there ? id[u] : 0) * a.ldw + col[u], a.D - col[u]);
        if (!there) id[u] = -1;
      }
      // every load is under way before the first is waited for
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < kPacks; u++) {
        if (first + u * kBlock + (int)threadIdx.x >= packs) continue;
        Pack<TO, kE> out;
#pragma unroll
        for (int e = 0; e < kE; e++)
          out.v[e] = from_f32<TO>(id[u] >= 0 ? a.scale * to_f32(in[u].v[e]) : 0.0f);
        put_once<SHORT>(y + (b + row[u]) * a.ldy + col[u], a.D - col[u], out, large);
      }
    }
  }
}

// ------------------------------------------------------------- gradient --

// Rows of zeros, by bytes, which are 0 in every type: chunks of 16, the last of a
// row moved back to its end. Rows without a gap between them are one long row, a
// chunk a thread: 10^6 x 300 fp32 in 180 us (6.7 TB/s), with four chunks a thread 202,
// by rows 266, so that it is no matter that rows with words are written again later.
struct Clear {
  char* rows;
  int64_t ld;  // bytes
  int32_t n, row_bytes, per_row, rows_a_block;
  Divisor by_row;
  int64_t flat;    // bytes of one long row, or 0
  int32_t blocks;  // 0: nothing to clear
};

__device__ __forceinline__ void clear_rows(const Clear& c, int64_t b) {
  const uint4 zero = make_uint4(0, 0, 0, 0);
  if (c.flat > 0) {
    const int64_t span = 16 * (int64_t)blockDim.x;
    for (int64_t at = b * span + threadIdx.x * 16; at < c.flat; at += c.blocks * span)
      store_once(c.rows + (at + 16 <= c.flat ? at : c.flat - 16), zero);
    return;
  }
  for (b *= c.rows_a_block; b < c.n; b += (int64_t)c.blocks * c.rows_a_block) {
    const int rows = (int)(c.n - b < c.rows_a_block ? c.n - b : c.rows_a_block);
    const int chunks = rows * c.per_row;
    for (int i = threadIdx.x; i < chunks; i += (int)blockDim.x) {
      const int row = (int)divided((uint32_t)i, c.by_row);
      const int at = (i - row * c.per_row) * 16;
      char* to = c.rows + (b + row) * c.ld;
      if (c.row_bytes >= 16) {
        store_once(to + (at + 16 <= c.row_bytes ? at : c.row_bytes - 16), zero);
      } else {
        for (int j = 0; j < c.row_bytes; j += 2) *(uint16_t*)(to + j) = 0;
      }
    }
  }
}

__global__ __launch_bounds__(kBlock) void k_embed_clear(Clear c) { clear_rows(c, blockIdx.x); }

// Rows [first, last) of the gradient, if they are to be cleared, by blocks of
// `threads`.
Clear clear_of(const EmbedBackwardArgs& a, int64_t first, int64_t last, int threads = kBlock) {
  Clear c{};
  if (a.accumulate || first == last) return c;
  const int64_t size = a.grad_dtype == W2V_DTYPE_F32 ? 4 : 2;
  c.ld = a.ldg * size;
  c.rows = (char*)a.grad + first * c.ld;
  c.n = (int32_t)(last - first);
  c.row_bytes = (int32_t)(a.D * size);
  c.per_row = (c.row_bytes + 15) / 16;
  c.rows_a_block = c.per_row >= 4 * threads ? 1 : 4 * threads / c.per_row;
  c.by_row = divisor_of((uint32_t)c.per_row);
  int64_t blocks = ((int64_t)c.n + c.rows_a_block - 1) / c.rows_a_block;
  if ((a.ldg == a.D || c.n == 1) && c.n * (int64_t)c.row_bytes >= 16) {
    c.flat = c.n * (int64_t)c.row_bytes;
    blocks = (c.flat + 16 * threads - 1) / (16 * threads);
  }
  const int64_t most = kMaxGrid / (threads / kBlock);  // 2^30 threads; a launch takes 2^32
  c.blocks = (int32_t)(blocks < most ? blocks : most);
  return c;
}

// The sort's key of a word: itself, V where there is none.
__device__ __forceinline__ uint32_t word_key(int32_t id, int32_t V, int32_t* status) {
  if (id >= 0 && id < V) return (uint32_t)id;
  if (id != -1) report_row(status);
  return (uint32_t)V;
}

// Up to 64 x 16 x GROUPS words sorted by one block, stably, by digits of six bits,
// the elements in registers and the counters of a wavefront's 64 digits in its 64
// lanes: lane l counts digit l. Blocks after the first clear the gradient
// meanwhile.
constexpr int kSortWaves = 16;
constexpr int kSortMax = kSortWaves * 8 * kWave;  // 8,192

// Lanes whose digit is d, from the ballots of the digits' bits.
template <int BITS>
__device__ __forceinline__ uint64_t lanes_with(const uint64_t (&set)[BITS], int d) {
  uint64_t m = ~0ull;
#pragma unroll
  for (int b = 0; b < BITS; b++) m &= (d >> b) & 1 ? set[b] : ~set[b];
  return m;
}

template <int GROUPS>
__global__ __launch_bounds__(kSortWaves* kWave) void k_embed_sort(
    const int32_t* ids, int32_t n, int32_t V, int bits, uint32_t* keys, int32_t* at,
    int32_t* status, Clear clear) {
  if (blockIdx.x > 0) {
    clear_rows(clear, blockIdx.x - 1);
    return;
  }
  __shared__ uint32_t s_key[kSortWaves * GROUPS * kWave];
  __shared__ uint16_t s_at[kSortWaves * GROUPS * kWave];
  __shared__ int s_count[kSortWaves * kWave];  // [digit][wave], then its start
  __shared__ int s_total[kSortWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t key[GROUPS];
  int from[GROUPS];
#pragma unroll
  for (int g = 0; g < GROUPS; g++) {
    const int i = (wave * GROUPS + g) * kWave + lane;
    from[g] = i;
    // past the end: behind everything, since the sort is stable
    key[g] = i < n ? word_key(ids[i], V, status) : ~0u;
  }
  for (int shift = 0; shift < bits; shift += 6) {
    int count = 0, rank[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; g++) {
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
#pragma unroll
    for (int w = 0; w < kSortWaves; w++) sum += w < wave ? s_total[w] : 0;
    s_count[threadIdx.x] = sum - c;
    __syncthreads();
#pragma unroll
    for (int g = 0; g < GROUPS; g++) {
      const int d = (int)(key[g] >> shift) & 63;
      const int to = s_count[d * kSortWaves + wave] + rank[g];
      s_key[to] = key[g];
      s_at[to] = (uint16_t)from[g];
    }
    __syncthreads();
#pragma unroll
    for (int g = 0; g < GROUPS; g++) {
      const int i = (wave * GROUPS + g) * kWave + lane;
      key[g] = s_key[i];
      from[g] = s_at[i];
    }
  }
#pragma unroll
  for (int g = 0; g < GROUPS; g++) {
    const int i = (wave * GROUPS + g) * kWave + lane;
    if (i < n) {
      keys[i] = key[g];
      at[i] = from[g];
    }
  }
}

// More words: passes over digits of up to ten bits, so that a vocabulary of up to
// 2^20 words takes two. A block counts the digits of a tile of 2,048 words in LDS;
// a block for 64 digits turns the tiles' counts into places (of few tiles, the next
// blocks do that for themselves); a block sends its tile there in order. The gradient
// is cleared by further blocks of these launches, which leave most of the card idle:
// 10^6 words and 10^6 x 300 fp32 in 240 us, 180 of them the clearing's 1.2 GB.
constexpr int kDigitBits = 10;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kTileGroups = 8;  // of a wavefront
constexpr int kTileWaves = kBlock / kWave;
constexpr int kTile = kTileWaves * kTileGroups * kWave;  // 2,048

// A pass's keys: words, which the first pass's counting copies, or the pass before's.
// Words are read that once: whatever becomes of them meanwhile, the counts are those of
// the keys that are sent, so that every place is taken, once.
struct SortPass {
  const int32_t* ids;  // or NULL
  uint32_t* copy;      // of their keys
  const uint32_t* keys;
  const int32_t* at;  // or NULL: where they are
  int32_t n, V, shift, digits, tiles;
  int32_t* status;

  __device__ __forceinline__ int digit(uint32_t k) const {
    return (int)(k >> shift) & (digits - 1);
  }
};

__global__ __launch_bounds__(kBlock) void k_embed_count(SortPass p, int32_t* hist, Clear clear) {
  if ((int)blockIdx.x >= p.tiles) {
    clear_rows(clear, (int)blockIdx.x - p.tiles);
    return;
  }
  __shared__ int s_count[kDigits];
  for (int d = threadIdx.x; d < p.digits; d += kBlock) s_count[d] = 0;
  const int64_t first = (int64_t)blockIdx.x * kTile + threadIdx.x;
  uint32_t key[kTileGroups];
#pragma unroll
  for (int g = 0; g < kTileGroups; g++) {
    const int64_t i = first + g * kBlock;
    key[g] = i >= p.n ? 0 : p.ids != nullptr ? word_key(p.ids[i], p.V, p.status) : p.keys[i];
    if (p.ids != nullptr && i < p.n) p.copy[i] = key[g];
  }
  __syncthreads();
#pragma unroll
  for (int g = 0; g < kTileGroups; g++)
    if (first + g * kBlock < p.n) atomicAdd(&s_count[p.digit(key[g])], 1);
  __syncthreads();
  for (int d = threadIdx.x; d < p.digits; d += kBlock)
    hist[(int64_t)blockIdx.x * p.digits + d] = s_count[d];
}

__device__ __forceinline__ int wave_prefix(int v, int lane) {
#pragma unroll
  for (int off = 1; off < kWave; off *= 2) {
    const int below = __shfl_up(v, off);
    if (lane >= off) v += below;
  }
  return v;
}

// The counts of a digit in the tiles [tile][digit] become the words of that digit
// before each tile: a lane a digit, a wavefront a sixteenth of up to 512 tiles at a
// time.
constexpr int kScanWaves = 16;
constexpr int kScanEach = 32;

__global__ __launch_bounds__(kScanWaves* kWave) void k_embed_scan(SortPass p, int32_t* hist,
                                                                int32_t* totals, Clear clear) {
  const int blocks = (p.digits + kWave - 1) / kWave;
  if ((int)blockIdx.x >= blocks) {
    clear_rows(clear, (int)blockIdx.x - blocks);
    return;
  }
  __shared__ int s_sum[kScanWaves][kWave];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int d = (int)blockIdx.x * kWave + lane;
  const bool there = d < p.digits;
  int carry = 0;
  for (int t0 = 0; t0 < p.tiles; t0 += kScanWaves * kScanEach) {
    const int left = p.tiles - t0 < kScanWaves * kScanEach ? p.tiles - t0 : kScanWaves * kScanEach;
    const int each = (left + kScanWaves - 1) / kScanWaves;
    const int first = wave * each < left ? wave * each : left;
    const int count = left - first < each ? left - first : each;
    int32_t* col = hist + (there ? d : 0);
    int v[kScanEach], own = 0;
    // no load has a test of its own
#pragma unroll
    for (int u = 0; u < kScanEach; u++) {
      const int t = t0 + first + u < p.tiles ? t0 + first + u : p.tiles - 1;
      v[u] = col[(int64_t)t * p.digits];
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < kScanEach; u++) {
      v[u] = u < count ? v[u] : 0;
      own += v[u];
    }
    s_sum[wave][lane] = own;
    __syncthreads();
    int at = carry, all = 0;
#pragma unroll
    for (int w = 0; w < kScanWaves; w++) {
      at += w < wave ? s_sum[w][lane] : 0;
      all += s_sum[w][lane];
    }
    carry += all;
#pragma unroll
    for (int u = 0; u < kScanEach; u++) {
      if (u < count && there) col[(int64_t)(t0 + first + u) * p.digits] = at;
      at += v[u];
    }
    __syncthreads();
  }
  if (wave == 0 && there) totals[d] = carry;
}

// Up to so many tiles need no launch for that (49 tiles of one pass: 50 us instead of 45
// without it).
constexpr int kFewTiles = 32;

__global__ __launch_bounds__(kBlock) void k_embed_scatter(SortPass p, const int32_t* hist,
                                                          const int32_t* totals, uint32_t* keys,
                                                          int32_t* at, Clear clear) {
  if ((int)blockIdx.x >= p.tiles) {
    clear_rows(clear, (int)blockIdx.x - p.tiles);
    return;
  }
  __shared__ int s_next[kTileWaves][kDigits];  // a wavefront's next place of a digit
  __shared__ int s_total[kTileWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int d = threadIdx.x; d < p.digits; d += kBlock)
    for (int w = 0; w < kTileWaves; w++) s_next[w][d] = 0;
  // a wavefront's words are consecutive
  const int64_t first = (int64_t)blockIdx.x * kTile + wave * (kTileGroups * kWave) + lane;
  uint32_t key[kTileGroups];
  int32_t from[kTileGroups];
#pragma unroll
  for (int g = 0; g < kTileGroups; g++) {
    const int64_t i = first + g * kWave;
    key[g] = i < p.n ? p.keys[i] : 0;
    from[g] = i < p.n ? (p.at == nullptr ? (int32_t)i : p.at[i]) : 0;
  }
  __syncthreads();
#pragma unroll
  for (int g = 0; g < kTileGroups; g++)
    if (first + g * kWave < p.n) atomicAdd(&s_next[wave][p.digit(key[g])], 1);
  // the words of smaller digits, and those of the digit before the tile, for digits
  // that are consecutive over the threads
  constexpr int kEach = kDigits / kBlock;
  const int d0 = (int)threadIdx.x * kEach;
  int total[kEach] = {}, before[kEach] = {}, own = 0;
  if (p.tiles <= kFewTiles) {
#pragma unroll 8
    for (int t = 0; t < p.tiles; t++)
#pragma unroll
      for (int j = 0; j < kEach; j++) {
        const int count = d0 + j < p.digits ? hist[(int64_t)t * p.digits + d0 + j] : 0;
        total[j] += count;
        before[j] += t < (int)blockIdx.x ? count : 0;
      }
  } else {
#pragma unroll
    for (int j = 0; j < kEach; j++)
      if (d0 + j < p.digits) {
        total[j] = totals[d0 + j];
        before[j] = hist[(int64_t)blockIdx.x * p.digits + d0 + j];
      }
  }
#pragma unroll
  for (int j = 0; j < kEach; j++) own += total[j];
  const int upto = wave_prefix(own, lane);
  if (lane == kWave - 1) s_total[wave] = upto;
  __syncthreads();
  int base = upto - own;
  for (int w = 0; w < wave; w++) base += s_total[w];
#pragma unroll
  for (int j = 0; j < kEach; j++) {
    const int d = d0 + j;
    if (d >= p.digits) break;
    int place = base + before[j];
    base += total[j];
#pragma unroll
    for (int w = 0; w < kTileWaves; w++) {
      const int count = s_next[w][d];
      s_next[w][d] = place;
      place += count;
    }
  }
  __syncthreads();
#pragma unroll
  for (int g = 0; g < kTileGroups; g++) {
    const bool there = first + g * kWave < p.n;
    const int d = p.digit(key[g]);
    uint64_t set[kDigitBits];
#pragma unroll
    for (int b = 0; b < kDigitBits; b++) set[b] = __ballot((d >> b) & 1);
    const uint64_t same = lanes_with(set, d) & __ballot(there);
    const int rank = __popcll(same & lanes_below(lane));
    const int place = s_next[wave][d] + rank;
    // places lie in [0, n) by construction. Should a workspace be written by another
    // call all the same, the test here and that of the sums' rows (row_in) keep what
    // is done within the arguments
    if (there && place >= 0 && place < p.n) {
      keys[place] = key[g];
      at[place] = from[g];
    }
    // the wavefront's own counters: its reads are before its writes
    __builtin_amdgcn_wave_barrier();
    if (there && rank == __popcll(same) - 1) s_next[wave][d] = place + 1;
    __builtin_amdgcn_wave_barrier();
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
__device__ __forceinline__ LaneColumns lane_columns(const Columns& c, int32_t D, int lane) {
  const int pack = (int)blockIdx.y * c.lanes + lane;
  LaneColumns l;
  l.there = lane < c.lanes && pack * kE < D;
  l.first = l.there ? pack_column<SHORT>(pack, D) : 0;
  l.skip = l.there ? pack * kE - l.first : 0;
  l.left = D - l.first;
  return l;
}

// A row of dy from the sorted list.
__device__ __forceinline__ int32_t row_in(int32_t at, int32_t n) {
  return (uint32_t)at < (uint32_t)n ? at : 0;
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

// The rows in flight together are added to each other before they are to the word's
// sum, and so are the partial sums of a long word: 10^6 normal rows of 64 fp32 over
// 1,000 words have an error of 1.1e-7 of their size, one after the other 1.4e-7.
__device__ __forceinline__ void fold(Pack<float, kE>& sum, Pack<float, kE>& some) {
#pragma unroll
  for (int e = 0; e < kE; e++) sum.v[e] += some.v[e];
  some = Pack<float, kE>{};
}

// Rows of more than 256 elements: one wavefront a chunk of `chunk` (up to 64) sorted
// positions, the chunk's keys in its lanes, kAhead rows in flight. `head` and `tail`:
// partial sums of the word that comes into the chunk from the one before, and of the
// one that goes over its end and began within.
constexpr int kAhead = 8;

template <typename TI, typename TG>
__global__ __launch_bounds__(kBlock) void k_embed_sums(EmbedBackwardArgs a, Columns cols,
                                                       const uint32_t* keys, const int32_t* at,
                                                       int chunk, float* head, float* tail) {
  const int lane = threadIdx.x & 63;
  const int64_t k = (int64_t)blockIdx.x * (kBlock / kWave) + (threadIdx.x >> 6);
  const int64_t begin = k * chunk;
  if (begin >= a.n) return;
  const int size = (int)(a.n - begin < chunk ? a.n - begin : chunk);
  const LaneColumns l = lane_columns<false>(cols, a.D, (int)threadIdx.x & 63);
  const uint32_t V = (uint32_t)a.V;
  const uint32_t key = lane < size ? keys[begin + lane] : V;
  const int32_t row = lane < size ? row_in(at[begin + lane], a.n) : 0;
  const uint32_t before = begin > 0 ? keys[begin - 1] : ~0u;
  const uint32_t after = begin + size < a.n ? keys[begin + size] : ~0u;
  // words only: absent ones come last
  const int used = __popcll(__ballot(lane < size && key < V));
  if (used == 0) return;
  const TI* dy = (const TI*)a.dy + l.first;
  Pack<float, kE> sum{}, some{};
  uint32_t word = (uint32_t)__builtin_amdgcn_readfirstlane((int)key);
  bool came = word == before;
  // `next`'s row comes after `word`'s
  const auto add = [&](const Pack<TI, kE>& in, uint32_t next) {
    if (next != word) {
      fold(sum, some);
      if (came) {
        if (l.there) put<false>(head + k * cols.ld + l.first, l.left, sum);
      } else {
        write_word<false, TG>(a, word, l, sum);
      }
      word = next;
      came = false;
      sum = Pack<float, kE>{};
    }
#pragma unroll
    for (int e = 0; e < kE; e++) some.v[e] += to_f32(in.v[e]);
  };
  const auto row_of = [&](int j) { return dy + __builtin_amdgcn_readlane(row, j) * a.lddy; };
  const auto key_of = [&](int j) { return (uint32_t)__builtin_amdgcn_readlane((int)key, j); };
  int j0 = 0;
  for (; j0 + kAhead <= used; j0 += kAhead) {
    Pack<TI, kE> in[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; u++) in[u] = get_once<false>(row_of(j0 + u), l.left);
    // every load is under way before the first is waited for
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < kAhead; u++) add(in[u], key_of(j0 + u));
    fold(sum, some);
  }
  for (; j0 < used; j0++) add(get_once<false>(row_of(j0), l.left), key_of(j0));
  fold(sum, some);
  const bool goes = word == after;
  if (!came && !goes) {
    write_word<false, TG>(a, word, l, sum);
  } else if (l.there) {
    put<false>((came ? head : tail) + k * cols.ld + l.first, l.left, sum);
  }
}

// Shorter rows: TEAM lanes a chunk, as many as a row has packs, so that a wavefront
// adds 2 to 8 rows at a time (10^6 rows of 64 bf16: 88 us with a wavefront a chunk).
template <typename TI, typename TG, bool SHORT, int TEAM>
__global__ __launch_bounds__(kBlock) void k_embed_team_sums(EmbedBackwardArgs a, Columns cols,
                                                            const uint32_t* keys,
                                                            const int32_t* at, int chunk,
                                                            float* head, float* tail) {
  const int64_t k = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / TEAM;
  const bool any = k * chunk < a.n;
  const int64_t begin = any ? k * chunk : 0;
  const int size = !any ? 0 : (int)(a.n - begin < chunk ? a.n - begin : chunk);
  const LaneColumns l = lane_columns<SHORT>(cols, a.D, (int)threadIdx.x & (TEAM - 1));
  const uint32_t V = (uint32_t)a.V;
  const uint32_t before = begin > 0 ? keys[begin - 1] : ~0u;
  const uint32_t after = any && begin + size < a.n ? keys[begin + size] : ~0u;
  const TI* dy = (const TI*)a.dy + l.first;
  Pack<float, kE> sum{}, some{};
  uint32_t word = any ? keys[begin] : V;
  bool came = word == before;
  // groups of kAhead lie within the arrays, which are of whole 256 bytes
  Pack<uint32_t, kAhead> next_key = load_pack<uint32_t, kAhead>(keys + begin);
  Pack<int32_t, kAhead> next_row = load_pack<int32_t, kAhead>(at + begin);
  for (int j0 = 0; j0 < chunk; j0 += kAhead) {
    const Pack<uint32_t, kAhead> key = next_key;
    const Pack<int32_t, kAhead> row = next_row;
    Pack<TI, kE> in[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; u++)
      in[u] = get_once<SHORT>(dy + (j0 + u < size ? row_in(row.v[u], a.n) : 0) * a.lddy, l.left);
    const int64_t from = j0 + kAhead < size ? begin + j0 + kAhead : begin;
    next_key = load_pack<uint32_t, kAhead>(keys + from);
    next_row = load_pack<int32_t, kAhead>(at + from);
    // every load is under way before the first is waited for
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < kAhead; u++) {
      if (j0 + u >= size || key.v[u] >= V) continue;  // absent words come last
      if (key.v[u] != word) {
        fold(sum, some);
        if (came) {
          if (l.there) put<SHORT>(head + k * cols.ld + l.first, l.left, sum);
        } else {
          write_word<SHORT, TG>(a, word, l, sum);
        }
        word = key.v[u];
        came = false;
        sum = Pack<float, kE>{};
      }
#pragma unroll
      for (int e = 0; e < kE; e++) some.v[e] += to_f32(in[u].v[e]);
    }
    fold(sum, some);
  }
  if (word >= V) return;
  if (!came && word != after) {
    write_word<SHORT, TG>(a, word, l, sum);
  } else if (l.there) {
    put<SHORT>((came ? head : tail) + k * cols.ld + l.first, l.left, sum);
  }
}

// Whether the word goes over the end of chunk c no further.
__device__ __forceinline__ bool ends_in(const uint32_t* keys, int64_t n, int chunk, int64_t c,
                                        uint32_t word) {
  const int64_t stop = (c + 1) * chunk;
  return stop >= n || keys[stop] != word;
}

// The chunk in which a word that goes over chunk k's end comes to its own: by 64
// probes at a time, first of the next chunks, then evenly over the others.
__device__ __forceinline__ int64_t last_chunk(const uint32_t* keys, int64_t n, int chunk,
                                              int64_t k, uint32_t word) {
  const int lane = threadIdx.x & 63;
  int64_t low = k + 1, high = (n - 1) / chunk, step = 1;
  for (;;) {
    const int64_t c = low + lane * step < high ? low + lane * step : high;
    const uint64_t m = __ballot(ends_in(keys, n, chunk, c, word));
    if (m == 0) {
      low += 63 * step + 1;
    } else {
      const int f = __builtin_ctzll(m);
      const int64_t found = low + f * step < high ? low + f * step : high;
      if (step == 1 || found == low) return found;
      low = f > 0 ? low + (f - 1) * step + 1 : low;
      high = found;
    }
    step = (high - low) / 63 > 1 ? (high - low) / 63 : 1;
  }
}

// Rows [first, first + count), every `stride`-th, of a table of partial sums.
template <bool SHORT>
__device__ __forceinline__ void add_rows(const float* rows, int64_t ld, int count, int first,
                                         int stride, int left, Pack<float, kE>& sum) {
  for (int j0 = first; j0 < count; j0 += kAhead * stride) {
    Pack<float, kE> in[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; u++) {
      const int j = j0 + u * stride;
      in[u] = get<SHORT>(rows + (j < count ? j : j0) * ld, left);
    }
    __builtin_amdgcn_sched_barrier(0);
    // to each other first, in pairs
#pragma unroll
    for (int u = 0; u < kAhead; u++)
#pragma unroll
      for (int e = 0; e < kE; e++) in[u].v[e] = j0 + u * stride < count ? in[u].v[e] : 0.0f;
#pragma unroll
    for (int d = 1; d < kAhead; d *= 2)
#pragma unroll
      for (int u = 0; u < kAhead; u += 2 * d)
#pragma unroll
        for (int e = 0; e < kE; e++) in[u].v[e] += in[u + d].v[e];
#pragma unroll
    for (int e = 0; e < kE; e++) sum.v[e] += in[0].v[e];
  }
}

// Long words' partial sums, kSpan chunks to one: for each span of chunks that lies
// wholly within a word that comes into it.
constexpr int kSpan = 32;
constexpr int kWaves = kBlock / kWave;

// The waves' sums, in their order, to wave 0.
__device__ __forceinline__ void join_waves(float (&s_sum)[kWaves][kWave][kE],
                                           Pack<float, kE>& sum) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int e = 0; e < kE; e++) s_sum[wave][lane][e] = sum.v[e];
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int w = 1; w < kWaves; w++)
#pragma unroll
    for (int e = 0; e < kE; e++) sum.v[e] += s_sum[w][lane][e];
}

template <bool SHORT>
__global__ __launch_bounds__(kBlock) void k_embed_spans(EmbedBackwardArgs a, Columns cols,
                                                        const uint32_t* keys, int chunk,
                                                        const float* head, float* spans) {
  __shared__ float s_sum[kWaves][kWave][kE];
  const int64_t first = (int64_t)blockIdx.x * kSpan * chunk, last = first + kSpan * chunk - 1;
  if (first == 0 || last >= a.n) return;
  const uint32_t word = keys[first];
  if (word >= (uint32_t)a.V || keys[first - 1] != word || keys[last] != word) return;
  const LaneColumns l = lane_columns<SHORT>(cols, a.D, (int)threadIdx.x & 63);
  Pack<float, kE> sum{};
  add_rows<SHORT>(head + (int64_t)blockIdx.x * kSpan * cols.ld + l.first, cols.ld, kSpan,
                  threadIdx.x >> 6, kWaves, l.left, sum);
  join_waves(s_sum, sum);
  if (threadIdx.x < kWave && l.there)
    put<SHORT>(spans + blockIdx.x * cols.ld + l.first, l.left, sum);
}

// Joins the partial sums of the words that go over their chunk's end and began in
// it. A wavefront looks at `each` chunks at once (1 to 16) and joins what it finds one
// after the other; words over many chunks are left to all four of a block. In order:
// the word's own tail, the chunks up to a span, the spans, the chunks behind.
constexpr int kMostEach = 16;

template <typename TG, bool SHORT>
__global__ __launch_bounds__(kBlock) void k_embed_join(EmbedBackwardArgs a, Columns cols,
                                                       const uint32_t* keys, int chunk,
                                                       int64_t chunks, int each,
                                                       const float* head, const float* tail,
                                                       const float* spans) {
  constexpr int kAlone = 2 * kAhead;
  __shared__ float s_sum[kWaves][kWave][kE];
  __shared__ int s_long, s_chunk[kMostEach * kWaves], s_count[kMostEach * kWaves];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const LaneColumns l = lane_columns<SHORT>(cols, a.D, lane);
  for (int64_t k0 = (int64_t)blockIdx.x * each * kWaves; k0 + 1 < chunks;
       k0 += (int64_t)gridDim.x * each * kWaves) {
    if (threadIdx.x == 0) s_long = 0;
    __syncthreads();
    const int64_t first = k0 + wave * each;
    const bool looks = lane < each && first + lane + 1 < chunks;
    const int64_t begin = looks ? (first + lane) * chunk : 0, end = looks ? begin + chunk : 1;
    const uint32_t word = keys[end - 1], behind = keys[looks ? end : 0], own = keys[begin],
                   before = keys[begin > 0 ? begin - 1 : 0];
    const bool came = own == word && begin > 0 && before == word;
    uint64_t found = __ballot(looks && word < (uint32_t)a.V && behind == word && !came);
    for (; found != 0; found &= found - 1) {
      const int at = __builtin_ctzll(found);
      const uint32_t w = (uint32_t)__builtin_amdgcn_readlane((int)word, at);
      const int64_t k = first + at;
      const int count = (int)(last_chunk(keys, a.n, chunk, k, w) - k);
      if (count <= kAlone) {
        Pack<float, kE> sum = get<SHORT>(tail + k * cols.ld + l.first, l.left);
        add_rows<SHORT>(head + (k + 1) * cols.ld + l.first, cols.ld, count, 0, 1, l.left, sum);
        write_word<SHORT, TG>(a, w, l, sum);
      } else if (lane == 0) {
        const int to = atomicAdd(&s_long, 1);
        s_chunk[to] = (int)(k - k0);
        s_count[to] = count;
      }
    }
    __syncthreads();
    const int longs = s_long;
    for (int i = 0; i < longs; i++) {
      const int64_t own_chunk = k0 + s_chunk[i], from = own_chunk + 1, to = from + s_count[i];
      // a span with the word's last chunk, which it may not fill, has no sum
      int64_t g0 = (from + kSpan - 1) / kSpan, g1 = (to - 1) / kSpan;
      if (spans == nullptr || g1 <= g0) g0 = g1 = to / kSpan + 1;
      const int64_t stop = g0 * kSpan < to ? g0 * kSpan : to;
      const int64_t on = g1 * kSpan < to ? g1 * kSpan : to;
      Pack<float, kE> sum{};
      if (wave == 0) sum = get<SHORT>(tail + own_chunk * cols.ld + l.first, l.left);
      add_rows<SHORT>(head + from * cols.ld + l.first, cols.ld, (int)(stop - from), wave, kWaves,
                      l.left, sum);
      if (g1 > g0)
        add_rows<SHORT>(spans + g0 * cols.ld + l.first, cols.ld, (int)(g1 - g0), wave, kWaves,
                        l.left, sum);
      add_rows<SHORT>(head + on * cols.ld + l.first, cols.ld, (int)(to - on), wave, kWaves, l.left,
                      sum);
      join_waves(s_sum, sum);
      if (wave == 0) write_word<SHORT, TG>(a, keys[own_chunk * chunk + chunk - 1], l, sum);
      __syncthreads();
    }
    __syncthreads();
  }
}

Columns columns_of(int32_t D) {
  const int64_t packs = ((int64_t)D + kE - 1) / kE;
  Columns c;
  c.tiles = (int32_t)((packs + kWave - 1) / kWave);
  c.lanes = (int32_t)((packs + c.tiles - 1) / c.tiles);
  c.ld = packs * kE;
  return c;
}

// Lanes that add a chunk.
int team_of(int32_t D) { return D <= 8 * kE ? 8 : D <= 16 * kE ? 16 : D <= 32 * kE ? 32 : kWave; }

// Long chunks leave few partial sums, short ones fill the card with wavefronts.
int chunk_of(int32_t n, int32_t D) {
  int chunk = kWave;
  while (chunk > kAhead && (int64_t)n / chunk * team_of(D) / kWave < 4096) chunk /= 2;
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
  int32_t *at, *at_before, *hist, *totals;
  float *head, *tail, *spans;
  size_t bytes;
};

int64_t tiles_of(int32_t n) { return ((int64_t)n + kTile - 1) / kTile; }

Workspace lay_out(void* base, int32_t n, int32_t D) {
  Workspace w{};
  size_t used = 0;
  const auto take = [&](size_t bytes) {
    char* p = (char*)base + used;
    used += aligned(bytes);
    return (void*)p;
  };
  const int64_t chunks = ((int64_t)n + chunk_of(n, D) - 1) / chunk_of(n, D);
  // of whole 256 bytes: read in groups of kAhead
  w.sorted = (uint32_t*)take(4 * (size_t)n);
  w.at = (int32_t*)take(4 * (size_t)n);
  const size_t row = 4 * (size_t)columns_of(D).ld;
  w.head = (float*)take((size_t)chunks * row);
  w.tail = (float*)take((size_t)chunks * row);
  w.spans = (float*)take((size_t)(chunks / kSpan) * row);
  if (n > kSortMax) {
    w.keys = (uint32_t*)take(4 * (size_t)n);
    w.at_before = (int32_t*)take(4 * (size_t)n);
    w.hist = (int32_t*)take(4 * (size_t)tiles_of(n) * kDigits);
    w.totals = (int32_t*)take(4 * kDigits);
  }
  w.bytes = used;
  return w;
}

template <int GROUPS>
void launch_sort(const EmbedBackwardArgs& a, const Workspace& w, const Clear& clear, int bits,
                 hipStream_t s) {
  hipLaunchKernelGGL(k_embed_sort<GROUPS>, dim3(1 + clear.blocks), dim3(kSortWaves * kWave), 0, s,
                     a.ids, a.n, a.V, bits, w.sorted, w.at, a.status, clear);
}

// Sorts the positions by word into w.sorted and w.at, and clears the gradient.
void launch_order(const EmbedBackwardArgs& a, const Workspace& w, hipStream_t s) {
  const int bits = key_bits(a.V);
  if (a.n <= kSortMax) {
    const Clear clear = clear_of(a, 0, a.V, kSortWaves * kWave);
    const int groups = (a.n + kSortWaves * kWave - 1) / (kSortWaves * kWave);
    if (groups <= 1) return launch_sort<1>(a, w, clear, bits, s);
    if (groups <= 2) return launch_sort<2>(a, w, clear, bits, s);
    if (groups <= 4) return launch_sort<4>(a, w, clear, bits, s);
    return launch_sort<8>(a, w, clear, bits, s);
  }
  const int passes = (bits + kDigitBits - 1) / kDigitBits;
  const int digit_bits = (bits + passes - 1) / passes < 2 ? 2 : (bits + passes - 1) / passes;
  SortPass p{};
  p.n = a.n;
  p.V = a.V;
  p.digits = 1 << digit_bits;
  p.tiles = (int32_t)tiles_of(a.n);
  p.status = a.status;
  p.ids = a.ids;
  const int launches = (p.tiles > kFewTiles ? 3 : 2) * passes;
  int launch = 0;
  const auto clear_next = [&](int threads = kBlock) {
    const int64_t first = (int64_t)a.V * launch / launches;
    launch++;
    return clear_of(a, first, (int64_t)a.V * launch / launches, threads);
  };
  for (int pass = 0; pass < passes; pass++) {
    p.shift = pass * digit_bits;
    // the last pass writes the result
    const bool to_out = (passes - 1 - pass) % 2 == 0;
    uint32_t* keys = to_out ? w.sorted : w.keys;
    int32_t* at = to_out ? w.at : w.at_before;
    p.copy = to_out ? w.keys : w.sorted;  // of the two, the one that the pass does not write
    Clear c = clear_next();
    hipLaunchKernelGGL(k_embed_count, dim3(p.tiles + c.blocks), dim3(kBlock), 0, s, p, w.hist, c);
    if (p.tiles > kFewTiles) {
      c = clear_next(kScanWaves * kWave);
      hipLaunchKernelGGL(k_embed_scan, dim3((p.digits + kWave - 1) / kWave + c.blocks),
                         dim3(kScanWaves * kWave), 0, s, p, w.hist, w.totals, c);
    }
    if (p.ids != nullptr) p.keys = p.copy;
    p.ids = nullptr;
    c = clear_next();
    hipLaunchKernelGGL(k_embed_scatter, dim3(p.tiles + c.blocks), dim3(kBlock), 0, s, p, w.hist,
                       w.totals, keys, at, c);
    p.keys = keys;
    p.at = at;
  }
}

template <typename TI, typename TG, bool SHORT>
hipError_t launch_sums(const EmbedBackwardArgs& a, const Workspace& w, hipStream_t s) {
  const Columns cols = columns_of(a.D);
  const int chunk = chunk_of(a.n, a.D);
  const int64_t chunks = ((int64_t)a.n + chunk - 1) / chunk;
  const unsigned tiles = (unsigned)cols.tiles;
  const int team = team_of(a.D), per_block = kBlock / team;
  const dim3 grid((unsigned)((chunks + per_block - 1) / per_block), tiles);
  const auto sums = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kBlock), 0, s, a, cols, w.sorted, w.at, chunk, w.head,
                       w.tail);
  };
  if constexpr (SHORT) {
    sums(k_embed_team_sums<TI, TG, true, 8>);
  } else if (team == 8) {
    sums(k_embed_team_sums<TI, TG, false, 8>);
  } else if (team == 16) {
    sums(k_embed_team_sums<TI, TG, false, 16>);
  } else if (team == 32) {
    sums(k_embed_team_sums<TI, TG, false, 32>);
  } else {
    sums(k_embed_sums<TI, TG>);
  }
  if (chunks == 1) return hipGetLastError();
  // spans shorten words over hundreds of chunks, for a launch
  const float* spans = chunks >= 64 * kSpan ? w.spans : nullptr;
  if (spans != nullptr)
    hipLaunchKernelGGL(k_embed_spans<SHORT>, dim3((unsigned)(chunks / kSpan), tiles), dim3(kBlock),
                       0, s, a, cols, w.sorted, chunk, w.head, w.spans);
  // a wavefront a chunk while the card holds them (62,500 chunks, D 64: 41 us so, 30
  // with 16 each; 3,125, D 300: 8 and 29)
  int each = 1;
  while (each < kMostEach && chunks / each > 16384) each *= 2;
  const int64_t joins = (chunks - 1 + each * kWaves - 1) / (each * kWaves);
  hipLaunchKernelGGL((k_embed_join<TG, SHORT>),
                     dim3((unsigned)(joins < kMaxGrid ? joins : kMaxGrid), tiles), dim3(kBlock), 0,
                     s, a, cols, w.sorted, chunk, chunks, each, w.head, w.tail, spans);
  return hipGetLastError();
}

template <typename TI, typename TG>
hipError_t launch_sums(const EmbedBackwardArgs& a, const Workspace& w, hipStream_t s) {
  return a.D < kE ? launch_sums<TI, TG, true>(a, w, s) : launch_sums<TI, TG, false>(a, w, s);
}

template <typename TG>
hipError_t launch_backward(const EmbedBackwardArgs& a, void* workspace, hipStream_t s) {
  if (a.n == 0) {
    const Clear clear = clear_of(a, 0, a.V);
    if (clear.blocks > 0)
      hipLaunchKernelGGL(k_embed_clear, dim3(clear.blocks), dim3(kBlock), 0, s, clear);
    return hipGetLastError();
  }
  const Workspace w = lay_out(workspace, a.n, a.D);
  launch_order(a, w, s);
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
