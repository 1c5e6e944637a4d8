// Words drawn from scores. Per row, with z the V scores and m their maximum:
//   x_j = (z_j - m) / T, w_j = exp(x_j); words are ranked by score, then by
//   index; a word is kept if its rank is below top_k, the weight of the words
//   ranked before it is below top_p of the top_k words' weight, and w_j >=
//   min_p. Each kept word races with x_j - log(-log u_j) (u_j its uniform
//   random number); the largest wins, which draws word j with probability
//   w_j over the kept words' weight.
// Every filter keeps a prefix of the ranking, so what is looked for is where
// it ends. The passes over a row, each split over blocks:
//   k_scan   maximum and sum of weights
//   k_bins   words or weight (in fixed point, so that sums have no order) by
//            bins of x, where a rank or a weight ends the prefix
//   k_race   the race of the words in bins that are kept whole; the words of
//            the bin in which the prefix ends (of all bins up to it where
//            top_k is on) go to a list
//   k_pick   one block a row: the end of the prefix within the list, the race
//            of the listed words, and the winner
#include "sample.h"

#include "head_types.h"

namespace w2v {
namespace {

constexpr int kThreads = 512;
constexpr int kPickThreads = 1024;
constexpr int kBins = 3072;
constexpr int kCapacity = 16384;  // words of a row's list
constexpr int kSmall = 1024;      // listed words that are ranked by counting

typedef unsigned long long u64;

struct Part {  // of one block's share of a row
  float max, sum;
  int32_t first;  // lowest index of the maximum
  int32_t nan;
  u64 best;  // the race's (score, index)
};

struct Ctx {
  SampleArgs a;
  int splits;
  int64_t range;
  int fixed_bits;  // a weight of 1 in fixed point
  bool bins;       // some row may need k_bins
  Part* parts;     // [rows][splits]
  u64* hist;       // [rows][kBins]
  uint32_t* listed;  // [rows]
  uint2* list;       // [rows][kCapacity]: score key, index
};

struct Setting {
  float inverse;  // 1 / T
  float p, floor;  // x >= floor = log min_p
  int32_t k;       // 0: off
  bool greedy, ok;
  __device__ bool by_rank() const { return k > 0; }
  __device__ bool by_weight() const { return p < 1.0f; }
  __device__ bool filters() const { return !greedy && ok && (by_rank() || by_weight()); }
};

__device__ __forceinline__ Setting setting(const Ctx& c, int row) {
  const SampleArgs& a = c.a;
  const float T = a.temperatures == nullptr ? a.temperature : a.temperatures[row];
  const int32_t k = a.top_ks == nullptr ? a.top_k : a.top_ks[row];
  const float p = a.top_ps == nullptr ? a.top_p : a.top_ps[row];
  const float least = a.min_ps == nullptr ? a.min_p : a.min_ps[row];
  Setting s;
  s.ok = T >= 0.0f && T < INFINITY && p > 0.0f && least >= 0.0f && least <= 1.0f && k >= 0 &&
         (k <= W2V_MAX_TOP_K || k >= a.V);
  s.greedy = T == 0.0f;
  s.inverse = 1.0f / T;
  s.k = k >= a.V ? 0 : k;
  s.p = p;
  s.floor = least > 0.0f ? logf(least) : -INFINITY;
  return s;
}

// Scores in an unsigned order.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __builtin_bit_cast(uint32_t, z == 0.0f ? 0.0f : z);  // -0 is 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float score_of(uint32_t key) {
  return __builtin_bit_cast(float, key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

__device__ __forceinline__ float x_of(float z, float max, float inverse) {
  return z == max ? 0.0f : (z - max) * inverse;
}

// Bins of x <= 0: 256 for every doubling of 1 - x, so 1/256 wide near the
// maximum and 1/16 at x = -16; the last takes all below -4095.
__device__ __forceinline__ int bin_of(float x) {
  const int b = (int)(__builtin_bit_cast(uint32_t, 1.0f - x) >> 15) - (127 << 8);
  return b < kBins - 1 ? b : kBins - 1;
}

__device__ __forceinline__ u64 weight_of(float x, int fixed_bits) {
  return (u64)(ldexpf(expf(x), fixed_bits));
}

// Larger is better: the score of the race, then the lower index. 0: none.
__device__ __forceinline__ u64 race_of(float x, float u, int32_t index) {
  float score = x - logf(-logf(u));
  if (score != score) score = -INFINITY;
  return (u64)key_of(score) << 32 | (uint32_t)~index;
}

__device__ __forceinline__ u64 wave_best(u64 v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const u64 o = __shfl_xor(v, d);
    v = o > v ? o : v;
  }
  return v;
}
__device__ __forceinline__ u64 wave_total(u64 v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ u64 block_best(u64 v, u64* scratch) {
  v = wave_best(v);
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
  __syncthreads();
  v = scratch[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); w++) v = scratch[w] > v ? scratch[w] : v;
  __syncthreads();
  return v;
}
__device__ u64 block_total(u64 v, u64* scratch) {
  v = wave_total(v);
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
  __syncthreads();
  v = scratch[0];
  for (int w = 1; w < (int)(blockDim.x >> 6); w++) v += scratch[w];
  __syncthreads();
  return v;
}

// f(index, z) for the thread's words of [lo, hi), 16 bytes at a time.
template <typename T, typename F>
__device__ __forceinline__ void each_word(const T* row, int64_t lo, int64_t hi, F f) {
  constexpr int N = 16 / (int)sizeof(T);
  const int step = blockDim.x;
  const int64_t packs = (hi - lo) / N;
  for (int64_t p = threadIdx.x; p < packs; p += step) {
    const int64_t at = lo + p * N;
    const Pack<T, N> in = load_pack<T, N>(row + at);
#pragma unroll
    for (int i = 0; i < N; i++) f((int32_t)(at + i), to_f32(in.v[i]));
  }
  const int64_t last = lo + packs * N + threadIdx.x;
  if (last < hi) f((int32_t)last, to_f32(row[last]));
}

// The row's maximum from its parts (a NaN in the row makes it NaN), in every
// thread.
__device__ float row_max(const Ctx& c, int row) {
  float m = -INFINITY;
  bool nan = false;
  for (int i = 0; i < c.splits; i++) {
    const Part& p = c.parts[(int64_t)row * c.splits + i];
    m = fmaxf(m, p.max);
    nan |= p.nan != 0;
  }
  return nan ? NAN : m;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_scan(Ctx c) {
  __shared__ float scratch[16];
  __shared__ u64 wide[16];
  const int row = blockIdx.x / c.splits, split = blockIdx.x % c.splits;
  const int64_t lo = split * c.range;
  const int64_t hi = lo + c.range < c.a.V ? lo + c.range : c.a.V;
  const T* z = (const T*)c.a.logits + row * c.a.ld;
  const Setting s = setting(c, row);
  // the share of what later passes add to
  if (c.bins)
    for (int i = split * kThreads + threadIdx.x; i < kBins; i += c.splits * kThreads)
      c.hist[(int64_t)row * kBins + i] = 0;
  if (split == 0 && threadIdx.x == 0) c.listed[row] = 0;
  float m = -INFINITY, nan = 0.0f;
  int32_t first = INT32_MAX;
  each_word(z, lo, hi, [&](int32_t i, float v) {
    if (v > m) {
      m = v;
      first = i;
    }
    if (v != v) nan = 1.0f;
  });
  const float max = block_max(m, scratch);
  nan = block_max(nan, scratch);
  const u64 index = block_best(m == max ? (u64)(uint32_t)~first : 0, wide);
  float sum = 0.0f;
  if (!s.greedy && max != -INFINITY)
    each_word(z, lo, hi, [&](int32_t, float v) { sum += expf(x_of(v, max, s.inverse)); });
  sum = block_sum(sum, scratch);
  if (threadIdx.x == 0) {
    Part& p = c.parts[(int64_t)row * c.splits + split];
    p.max = max;
    p.sum = sum;
    p.first = (int32_t)~(uint32_t)index;
    p.nan = nan > 0.0f;
    p.best = 0;
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_bins(Ctx c) {
  __shared__ u64 bins[kBins];
  const int row = blockIdx.x / c.splits, split = blockIdx.x % c.splits;
  const Setting s = setting(c, row);
  const float max = row_max(c, row);
  if (!s.filters() || !(max > -INFINITY)) return;
  const int64_t lo = split * c.range;
  const int64_t hi = lo + c.range < c.a.V ? lo + c.range : c.a.V;
  for (int i = threadIdx.x; i < kBins; i += kThreads) bins[i] = 0;
  __syncthreads();
  each_word((const T*)c.a.logits + row * c.a.ld, lo, hi, [&](int32_t, float v) {
    if (v == -INFINITY) return;
    const float x = x_of(v, max, s.inverse);
    atomicAdd(&bins[bin_of(x)], s.by_rank() ? 1ull : weight_of(x, c.fixed_bits));
  });
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kThreads)
    if (bins[i] != 0) atomicAdd(&c.hist[(int64_t)row * kBins + i], bins[i]);
}

// Where a row's prefix ends: bins below `bin` are kept whole, with `above`
// words or weight; the prefix has `target` in all.
struct End {
  int bin;
  u64 above, target;
};

// From the row's histogram, in every thread. Thread t sums neighbouring bins;
// the sums are scanned over the block.
__device__ End end_of(const Ctx& c, int row, const Setting& s, u64* wide) {
  __shared__ End end;
  const int tid = threadIdx.x, per = (kBins + (int)blockDim.x - 1) / (int)blockDim.x;
  const u64* h = c.hist + (int64_t)row * kBins;
  u64 own = 0;
  for (int i = 0; i < per; i++)
    if (tid * per + i < kBins) own += h[tid * per + i];
  u64 upto = own;  // inclusive scan over the wave
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const u64 o = __shfl_up(upto, d);
    if ((tid & 63) >= d) upto += o;
  }
  if ((tid & 63) == 63) wide[tid >> 6] = upto;
  __syncthreads();
  u64 total = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); w++) {
    if (w < tid >> 6) upto += wide[w];
    total += wide[w];
  }
  const u64 target = s.by_rank() ? (u64)s.k : (u64)ceil((double)s.p * (double)total);
  if (tid == 0) end = End{kBins, total, target};
  __syncthreads();
  u64 before = upto - own;
  if (before < target && upto >= target) {  // one thread, if any
    for (int i = 0; i < per; i++) {
      const u64 n = h[tid * per + i];
      if (before + n >= target) {
        end = End{tid * per + i, before, target};
        break;
      }
      before += n;
    }
  }
  __syncthreads();
  const End out = end;
  __syncthreads();
  return out;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_race(Ctx c) {
  __shared__ u64 wide[16];
  const int row = blockIdx.x / c.splits, split = blockIdx.x % c.splits;
  const Setting s = setting(c, row);
  const float max = row_max(c, row);
  if (s.greedy || !s.ok || !(max > -INFINITY)) return;
  const int64_t lo = split * c.range;
  const int64_t hi = lo + c.range < c.a.V ? lo + c.range : c.a.V;
  End end = {kBins, 0, 0};
  if (s.filters()) end = end_of(c, row, s, wide);
  const float* u = c.a.uniforms + row * c.a.ldu;
  uint2* list = c.list + (int64_t)row * kCapacity;
  u64 best = 0;
  each_word((const T*)c.a.logits + row * c.a.ld, lo, hi, [&](int32_t i, float v) {
    if (v == -INFINITY) return;
    const float x = x_of(v, max, s.inverse);
    const int bin = bin_of(x);
    if (bin > end.bin) return;
    if (s.by_rank() || bin == end.bin) {
      const uint32_t at = atomicAdd(&c.listed[row], 1u);
      if (at < kCapacity) list[at] = make_uint2(key_of(v), (uint32_t)i);
    } else if (x >= s.floor) {
      const u64 r = race_of(x, u[i], i);
      best = r > best ? r : best;
    }
  });
  best = block_best(best, wide);
  if (threadIdx.x == 0) c.parts[(int64_t)row * c.splits + split].best = best;
}

// f(key, index) for every listed word, from the list or, where it was too
// short, from the row itself.
template <typename T, typename F>
__device__ void each_listed(const Ctx& c, int row, const Setting& s, float max, const End& end,
                            uint32_t n, F f) {
  if (n <= kCapacity) {
    const uint2* list = c.list + (int64_t)row * kCapacity;
    for (uint32_t i = threadIdx.x; i < n; i += blockDim.x) f(list[i].x, list[i].y);
    return;
  }
  each_word((const T*)c.a.logits + row * c.a.ld, 0, c.a.V, [&](int32_t i, float v) {
    if (v == -INFINITY) return;
    const int bin = bin_of(x_of(v, max, s.inverse));
    if (bin == end.bin || (s.by_rank() && bin < end.bin)) f(key_of(v), (uint32_t)i);
  });
}

__device__ __forceinline__ u64 order_of(uint32_t key, uint32_t index) {
  return (u64)key << 32 | (uint32_t)~index;
}

template <typename T>
__global__ __launch_bounds__(kPickThreads) void k_pick(Ctx c) {
  __shared__ u64 wide[16];
  __shared__ u64 order[kSmall], weight[kSmall];
  __shared__ u64 digits[256];
  __shared__ u64 prefix_s, above_s;
  __shared__ uint32_t taken;
  const int row = blockIdx.x, tid = threadIdx.x;
  const Setting s = setting(c, row);
  const float max = row_max(c, row);
  const T* logits = (const T*)c.a.logits + row * c.a.ld;
  const float* u = c.a.uniforms + row * c.a.ldu;
  if (!s.ok || !(max > -INFINITY)) {  // no setting, no word, or NaN
    if (tid == 0) {
      c.a.ids[row] = -1;
      if (c.a.logprob != nullptr) c.a.logprob[row] = NAN;
      if (!s.ok)
        __hip_atomic_store(c.a.status, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
    }
    return;
  }
  const Part* parts = c.parts + (int64_t)row * c.splits;
  int32_t id = INT32_MAX;
  if (s.greedy) {
    for (int i = 0; i < c.splits; i++)
      if (parts[i].max == max && parts[i].first < id) id = parts[i].first;
    if (tid == 0) {
      c.a.ids[row] = id;
      if (c.a.logprob != nullptr) c.a.logprob[row] = 0.0f;
    }
    return;
  }
  u64 best = 0;
  for (int i = tid; i < c.splits; i += kPickThreads)
    best = parts[i].best > best ? parts[i].best : best;

  if (s.filters()) {
    const End end = end_of(c, row, s, wide);
    const uint32_t n = c.listed[row];
    // What the words of the list have to stay below, counted from its first.
    u64 target = s.by_rank() ? (u64)s.k : end.target - end.above;
    u64 lowest = 0;  // listed words of this order or above are kept
    if (n > kSmall) {
      // The order of the last kept word, 8 bits at a time.
      u64 prefix = 0, above = 0;
      for (int shift = 56; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += kPickThreads) digits[i] = 0;
        __syncthreads();
        each_listed<T>(c, row, s, max, end, n, [&](uint32_t key, uint32_t i) {
          const u64 o = order_of(key, i);
          if (shift < 56 && (o ^ prefix) >> (shift + 8) != 0) return;
          atomicAdd(&digits[(o >> shift) & 255],
                    s.by_rank() ? 1ull
                                : weight_of(x_of(score_of(key), max, s.inverse), c.fixed_bits));
        });
        __syncthreads();
        if (tid == 0) {
          int d = 255;
          u64 a = above;
          for (; d > 0 && a + digits[d] < target; d--) a += digits[d];
          prefix_s = prefix | (u64)d << shift;
          above_s = a;
        }
        __syncthreads();
        prefix = prefix_s;
        above = above_s;
        __syncthreads();
      }
      lowest = prefix;
    }
    if (s.by_rank() || n <= kSmall) {
      // Ranks by counting: each thread has one word.
      if (tid == 0) taken = 0;
      __syncthreads();
      each_listed<T>(c, row, s, max, end, n, [&](uint32_t key, uint32_t i) {
        const u64 o = order_of(key, i);
        if (o < lowest) return;
        const uint32_t at = atomicAdd(&taken, 1u);
        if (at < kSmall) {
          order[at] = o;
          weight[at] = weight_of(x_of(score_of(key), max, s.inverse), c.fixed_bits);
        }
      });
      __syncthreads();
      const int count = (int)(taken < kSmall ? taken : kSmall);
      const bool mine = tid < count;
      const u64 o = mine ? order[tid] : 0;
      u64 before = 0;
      int rank = 0;
      if (mine) {
        for (int i = 0; i < count; i++) {
          if (order[i] > o) {
            before += weight[i];
            rank++;
          }
        }
      }
      bool keep = mine;
      if (s.by_rank()) {
        keep = keep && rank < s.k;
        const u64 total = block_total(keep ? weight[tid] : 0, wide);
        if (s.by_weight())
          keep = keep && (rank == 0 || before < (u64)ceil((double)s.p * (double)total));
      } else {
        keep = keep && (before < target);
      }
      if (keep) {
        const uint32_t i = ~(uint32_t)o;
        const float x = x_of(score_of((uint32_t)(o >> 32)), max, s.inverse);
        if (x >= s.floor) {
          const u64 r = race_of(x, u[i], (int32_t)i);
          best = r > best ? r : best;
        }
      }
    } else {
      each_listed<T>(c, row, s, max, end, n, [&](uint32_t key, uint32_t i) {
        const float x = x_of(score_of(key), max, s.inverse);
        if (order_of(key, i) < lowest || !(x >= s.floor)) return;
        const u64 r = race_of(x, u[i], (int32_t)i);
        best = r > best ? r : best;
      });
    }
  }
  best = block_best(best, wide);
  if (tid == 0) {
    id = (int32_t)~(uint32_t)best;
    c.a.ids[row] = id;
    if (c.a.logprob != nullptr) {
      float sum = 0.0f;
      for (int i = 0; i < c.splits; i++)
        if (parts[i].max != -INFINITY)
          sum += parts[i].sum * expf(x_of(parts[i].max, max, s.inverse));
      c.a.logprob[row] = x_of(to_f32(logits[id]), max, s.inverse) - logf(sum);
    }
  }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Blocks of a row: enough for the GPU to be full with few rows, each with at
// least 4096 words.
int splits_of(int32_t rows, int32_t V) {
  const int64_t most = ceil_div(V, 4096);
  int64_t want = ceil_div(1024, rows > 0 ? rows : 1);
  if (want > most) want = most;
  if (want > 256) want = 256;
  return (int)(want < 1 ? 1 : want);
}

struct Layout {
  size_t parts, hist, listed, list, total;
};

Layout layout(int32_t rows, int32_t V) {
  Layout l;
  size_t at = 0;
  l.parts = at;
  at += aligned((size_t)rows * splits_of(rows, V) * sizeof(Part));
  l.listed = at;
  at += aligned((size_t)rows * 4);
  l.hist = at;
  at += aligned((size_t)rows * kBins * 8);
  l.list = at;
  at += aligned((size_t)rows * kCapacity * 8);
  l.total = at;
  return l;
}

template <typename T>
hipError_t launch_as(const Ctx& c, hipStream_t s) {
  const int grid = c.a.rows * c.splits;
  const bool greedy = c.a.temperatures == nullptr && c.a.temperature == 0.0f;
  k_scan<T><<<grid, kThreads, 0, s>>>(c);
  if (c.bins) k_bins<T><<<grid, kThreads, 0, s>>>(c);
  if (!greedy) k_race<T><<<grid, kThreads, 0, s>>>(c);
  k_pick<T><<<c.a.rows, kPickThreads, 0, s>>>(c);
  return hipGetLastError();
}

}  // namespace

size_t sample_workspace_bytes(int32_t rows, int32_t V) { return layout(rows, V).total; }

hipError_t launch_sample(const SampleArgs& a, void* workspace, hipStream_t s) {
  Ctx c{};
  c.a = a;
  c.splits = splits_of(a.rows, a.V);
  c.range = ceil_div(ceil_div(a.V, c.splits), 64) * 64;
  c.splits = (int)ceil_div(a.V, c.range);
  int bits = 1;
  while (bits < 31 && (int64_t(1) << bits) <= a.V) bits++;
  c.fixed_bits = 62 - bits < 40 ? 62 - bits : 40;
  const bool rank = a.top_ks != nullptr || (a.top_k > 0 && a.top_k < a.V);
  const bool weight = a.top_ps != nullptr || a.top_p < 1.0f;
  c.bins = (rank || weight) && !(a.temperatures == nullptr && a.temperature == 0.0f);
  const Layout l = layout(a.rows, a.V);
  char* ws = (char*)workspace;
  c.parts = (Part*)(ws + l.parts);
  c.hist = (u64*)(ws + l.hist);
  c.listed = (uint32_t*)(ws + l.listed);
  c.list = (uint2*)(ws + l.list);
  switch (a.dtype) {
    case W2V_DTYPE_F32:
      return launch_as<float>(c, s);
    case W2V_DTYPE_BF16:
      return launch_as<bf16_t>(c, s);
    default:
      return launch_as<f16_t>(c, s);
  }
}

}  // namespace w2v
