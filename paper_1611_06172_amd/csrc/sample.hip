// Words drawn from scores. Per row, with z the V scores and m their maximum:
//   x_j = (z_j - m) / T, w_j = exp(x_j); words are ranked by score, then by
//   index; a word is kept if its rank is below top_k, the weight of the words
//   ranked before it is below top_p of the top_k words' weight, and w_j >=
//   min_p. Each kept word races with x_j - log(-log u_j) (u_j its uniform
//   random number); the largest wins, which draws word j with probability
//   w_j over the kept words' weight.
// Every filter keeps a prefix of the ranking, so what is looked for is where
// it ends. The passes over a row:
//   scan   maximum and sum of weights; for a small top_k also a score that k
//          words reach: the k-th largest of the threads' own maxima
//   bins   otherwise: words or weight (in fixed point, so that sums have no
//          order) by bins of x, where a rank or a weight ends the prefix
//   race   the race of the words in bins that are kept whole; the words that
//          the end of the prefix may cut (those of its bin; with top_k all that
//          reach the score or the bin) go to a list
//   pick   the end of the prefix within the list, the race of the listed words,
//          and the winner
// One block does all of them for a row of few words, or where there are enough
// rows (k_row); otherwise each is a kernel over shares of the rows.
// Bound by memory over many rows and by the chain of barriers over few. Measured
// (us): 64 rows of 10^6 bf16 with top_p 187 (scan 25, bins 43, race 98: it reads
// the kept words' random numbers one by one, pick 23), 0.7 TB/s of one reading of
// the scores, which is read three times; 257 rows of 100,000 fp16 with top_k 50
// 46 (1.1 TB/s, read twice); one row of 71,290 fp32 20 in three kernels.
// Where the words that the end may cut are more than a list holds (nearly equal
// scores), one block reads the whole row again, up to eight times: 64 rows of 10^6
// scores within 1e-3 take 8,570 with top_p 0.9 and 1,780 with top_k 500, but 87 with
// top_k 50; 64 rows of 60,000 199, 175 and 32.
#include "sample.h"

#include "head_types.h"

namespace w2v {
namespace {

constexpr int kThreads = 256;
constexpr int kBins = 3072;
constexpr int kCapacity = 16384;  // words of a row's list in memory
constexpr int kLocal = 2048;      // and of a share's in LDS
constexpr int kLocalRow = 5120;   // and of a whole row's
// top_k up to which the threads' maxima bound the list well: with k of 1024
// threads' maxima above the bound, about k (1 + k / 2048) words are. Every
// block has as many threads.
constexpr int kBounded = 256;

typedef unsigned long long u64;

struct Part {  // of one block's share of a row
  float max;
  float rest;     // weights relative to max, but for one word at it
  float bound;    // a score that k of its words reach, or -inf
  int32_t first;  // lowest index of the maximum
  int32_t nan;
  u64 best;  // the race's (score, index)
};

struct Ctx {
  SampleArgs a;
  int splits;
  int64_t range;
  int fixed_bits;  // a weight of 1 in fixed point
  bool bins;       // some row may need bins
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
  // the list starts at a score instead of in a bin
  __device__ bool bounded() const { return by_rank() && k <= kBounded; }
  __device__ bool binned() const { return filters() && !bounded(); }
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
  // kept finite, with its multiple by log2(e): a row's maximum is 0 times it
  s.inverse = 1.0f / fmaxf(T, 0x1p-126f);
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
  return (u64)(ldexpf(exp2_fast(x * kLog2e), fixed_bits));
}

// A word's score in the race. The hardware's logarithm (base 2) is within a
// unit in the last place, so each logarithm's relative error is 2^-22 and the
// score's 2^-22 + 2^-23 |x|. u of 0 or NaN gives the lowest score.
__device__ __forceinline__ float score_in_race(float x, float u) {
  constexpr float kLn2 = 0.693147180559945309f;
  const float e = __builtin_amdgcn_logf(u) * -kLn2;
  return fmaxf(__builtin_fmaf(__builtin_amdgcn_logf(e), -kLn2, x), -3.402823466e38f);
}
// Larger is better: the score, then the lower index. 0: none.
__device__ __forceinline__ u64 entry_of(float score, int32_t index) {
  return (u64)key_of(score) << 32 | (uint32_t)~index;
}
__device__ __forceinline__ u64 race_of(float x, float u, int32_t index) {
  return entry_of(score_in_race(x, u), index);
}

__device__ __forceinline__ u64 wave_best(u64 v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const u64 o = __shfl_xor(v, d);
    v = o > v ? o : v;
  }
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
__device__ u64 block_or(u64 v, u64* scratch) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v |= __shfl_xor(v, d);
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); w++) v |= scratch[w];
  __syncthreads();
  return v;
}
// Inclusive sum over the block's threads, and the total.
__device__ u64 block_scan(u64 v, u64* scratch, u64& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const u64 o = __shfl_up(v, d);
    if (lane >= d) v += o;
  }
  if (lane == 63) scratch[wave] = v;
  __syncthreads();
  total = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); w++) {
    if (w < wave) v += scratch[w];
    total += scratch[w];
  }
  __syncthreads();
  return v;
}

// f(first index, z[N], n) for the thread's packs of [lo, hi): N neighbouring
// words, of which n are there; U packs' loads are in flight together.
template <typename T, int U, typename F>
__device__ __forceinline__ void each_pack(const T* row, int64_t lo, int64_t hi, F f) {
  constexpr int N = 16 / (int)sizeof(T);
  const int step = blockDim.x;
  const int64_t packs = (hi - lo) / N;
  for (int64_t p = threadIdx.x; p < packs; p += U * step) {
    uint4 in[U];
#pragma unroll
    for (int u = 0; u < U; u++)
      if (p + u * step < packs) in[u] = load_16(row + lo + (p + u * step) * N);
#pragma unroll
    for (int u = 0; u < U; u++) {
      if (p + u * step >= packs) break;
      float v[N];
      unpack_words<T>(in[u], v);
      f((int32_t)(lo + (p + u * step) * N), v, N);
    }
  }
  const int64_t last = lo + packs * N + threadIdx.x;
  if (last < hi) {
    float v[N];
#pragma unroll
    for (int i = 1; i < N; i++) v[i] = -INFINITY;
    v[0] = to_f32(row[last]);
    f((int32_t)last, v, 1);
  }
}

template <typename T>
__device__ __forceinline__ const T* logits_of(const Ctx& c, int row) {
  return (const T*)c.a.logits + (int64_t)row * c.a.ld;
}

// The thread's element of the block's sorted in descending order (bitonic; the
// block has a power of two of threads, `size` of them are sorted).
template <typename K>
__device__ __forceinline__ K sorted(K o, int size, K* buffer) {
  const int tid = threadIdx.x;
  for (int span = 2; span <= size; span <<= 1) {
    for (int step = span >> 1; step > 0; step >>= 1) {
      K other;
      if (step < 64) {
        other = __shfl_xor(o, step);
      } else {
        __syncthreads();
        buffer[tid] = o;
        __syncthreads();
        other = buffer[tid ^ step];
      }
      const bool larger = ((tid & step) == 0) == ((tid & span) == 0);
      o = larger == (other > o) ? other : o;
    }
  }
  return o;
}

// The part of [lo, hi), in every thread: one pass with a running maximum, which
// moves once a pack.
template <typename T>
__device__ Part scan(const Ctx& c, int row, const Setting& s, int64_t lo, int64_t hi,
                     float* scratch, u64* wide, uint32_t* buffer) {
  constexpr int N = 16 / (int)sizeof(T);
  float m = -INFINITY, sum = 0.0f, nan = 0.0f;
  int32_t first = INT32_MAX;
  const float scale = s.inverse * kLog2e;
  if (s.greedy) {
    each_pack<T, 4>(logits_of<T>(c, row), lo, hi, [&](int32_t i, const float(&v)[N], int) {
#pragma unroll
      for (int j = 0; j < N; j++) {
        if (v[j] > m) {
          m = v[j];
          first = i + j;
        }
        if (v[j] != v[j]) nan = 1.0f;
      }
    });
  } else {
    // (with a maximum of +inf the sum is only asked whether it is NaN)
    each_pack<T, 4>(logits_of<T>(c, row), lo, hi, [&](int32_t, const float(&v)[N], int) {
      float most = v[0];
#pragma unroll
      for (int j = 1; j < N; j++) most = fmaxf(most, v[j]);
      if (most > m) {
        sum *= m == -INFINITY ? 0.0f : exp2_fast(x_of(m, most, scale));
        m = most;
      }
      const float base = fabsf(m) == INFINITY ? 0.0f : m;
      float some = 0.0f;
#pragma unroll
      for (int j = 0; j < N; j++) some += exp2_fast((v[j] - base) * scale);
      sum += some;
    });
    if (sum != sum) nan = 1.0f;
  }
  float max = m;
  block_maxima(max, nan, scratch);
  Part p;
  p.max = max;
  p.nan = nan > 0.0f;
  p.best = 0;
  p.first = 0;
  p.rest = 0.0f;
  p.bound = -INFINITY;
  if (s.bounded() && !s.greedy && s.ok) {
    const uint32_t key = sorted(key_of(m), blockDim.x, buffer);
    __syncthreads();
    if ((int)threadIdx.x == s.k - 1) buffer[0] = key;
    __syncthreads();
    p.bound = score_of(buffer[0]);
  }
  if (max == INFINITY && !s.greedy) {  // words at +inf weigh 1, others nothing
    sum = 0.0f;
    each_pack<T, 4>(logits_of<T>(c, row), lo, hi, [&](int32_t, const float(&v)[N], int) {
#pragma unroll
      for (int j = 0; j < N; j++) sum += v[j] == INFINITY ? 1.0f : 0.0f;
    });
    m = max;
  }
  if (s.greedy)
    p.first = (int32_t)~(uint32_t)block_best(m == max ? (u64)(uint32_t)~first : 0, wide);
  else {
    float top = m == max ? sum : 0.0f;
    p.rest = m == max || m == -INFINITY ? 0.0f : sum * exp2_fast(x_of(m, max, scale));
    block_sums(top, p.rest, scratch);
    if (top - 1.0f + p.rest < 0.25f && max < INFINITY) {
      // The best word has nearly all of the weight, and beside it its thread's
      // other words were rounded to units of 2^-24: they are added up again.
      top = 0.0f;
      if (m == max)
        each_pack<T, 4>(logits_of<T>(c, row), lo, hi, [&](int32_t, const float(&v)[N], int) {
#pragma unroll
          for (int j = 0; j < N; j++)
            top += v[j] == max ? 0.0f : exp2_fast((v[j] - max) * scale);
        });
      p.rest += block_sum(top, scratch);
    } else {
      p.rest += top - 1.0f;
    }
  }
  return p;
}

// Adds the words of [lo, hi) to the bins in LDS.
template <typename T>
__device__ __forceinline__ void add_bins(const Ctx& c, int row, const Setting& s, float max,
                                         int64_t lo, int64_t hi, u64* bins) {
  constexpr int N = 16 / (int)sizeof(T);
  const bool by_rank = s.by_rank();
  each_pack<T, 4>(logits_of<T>(c, row), lo, hi, [&](int32_t, const float(&v)[N], int) {
#pragma unroll
    for (int j = 0; j < N; j++) {
      const float x = x_of(v[j], max, s.inverse);
      const u64 w = by_rank ? 1 : weight_of(x, c.fixed_bits);
      if (v[j] != -INFINITY && w != 0) atomicAdd(&bins[bin_of(x)], w);
    }
  });
}

// Where a row's prefix ends: bins below `bin` are kept whole, with `above`
// words or weight; the prefix has `target` in all.
struct End {
  int bin;
  u64 above, target;
  float bound;  // where the list starts at a score
};

// 1 - x from which on a word is in bin b or a later one; NaN, which nothing
// reaches, for the end of the last bin.
__device__ __forceinline__ float edge_of(int b) {
  return b >= kBins ? NAN : __builtin_bit_cast(float, (uint32_t)(b + (127 << 8)) << 15);
}

// From the row's bins (in LDS or memory), in every thread: thread t sums
// neighbouring bins and the sums are scanned over the block.
__device__ End end_of(const Setting& s, const u64* bins, u64* wide, End* shared) {
  const int tid = threadIdx.x, per = (kBins + (int)blockDim.x - 1) / (int)blockDim.x;
  u64 own = 0, total;
  for (int i = 0; i < per; i++)
    if (tid * per + i < kBins) own += bins[tid * per + i];
  const u64 upto = block_scan(own, wide, total);
  const u64 target = s.by_rank() ? (u64)s.k : (u64)ceil((double)s.p * (double)total);
  if (tid == 0) *shared = End{kBins, total, target, 0.0f};
  __syncthreads();
  u64 before = upto - own;
  if (before < target && upto >= target) {  // one thread, if any
    for (int i = 0; i < per; i++) {
      const u64 n = bins[tid * per + i];
      if (before + n >= target) {
        *shared = End{tid * per + i, before, target, 0.0f};
        break;
      }
      before += n;
    }
  }
  __syncthreads();
  const End out = *shared;
  __syncthreads();
  return out;
}

// The race of the words of [lo, hi) that are surely kept; those that the end of
// the prefix may cut are listed in LDS (`count` of them, more than `capacity`
// are only counted). Returns the thread's best.
template <typename T>
__device__ __forceinline__ u64 race(const Ctx& c, int row, const Setting& s, float max,
                                    const End& end, int64_t lo, int64_t hi, uint2* list,
                                    uint32_t capacity, uint32_t* count) {
  constexpr int N = 16 / (int)sizeof(T);
  const float* u = c.a.uniforms + (int64_t)row * c.a.ldu;
  float best = -INFINITY;
  int32_t at = -1;
  if (!s.filters() && s.floor == -INFINITY) {  // every word races
    each_pack<T, 2>(logits_of<T>(c, row), lo, hi, [&](int32_t i, const float(&v)[N], int n) {
      const Pack<float, N> r = load_some<float, N>(u + i, n);
#pragma unroll
      for (int j = 0; j < N; j++) {
        if (j >= n) break;
        const float score = score_in_race(x_of(v[j], max, s.inverse), r.v[j]);
        if (score > best && v[j] != -INFINITY) {
          best = score;
          at = i + j;
        }
      }
    });
  } else if (s.bounded()) {  // words that reach the bound are listed
    each_pack<T, 4>(logits_of<T>(c, row), lo, hi, [&](int32_t i, const float(&v)[N], int n) {
      bool any = false;
#pragma unroll
      for (int j = 0; j < N; j++) any |= v[j] >= end.bound;
      if (!any) return;
#pragma unroll
      for (int j = 0; j < N; j++) {
        if (v[j] >= end.bound && v[j] != -INFINITY) {
          const uint32_t slot = atomicAdd(count, 1u);
          if (slot < capacity) list[slot] = make_uint2(key_of(v[j]), (uint32_t)(i + j));
        }
      }
    });
  } else {
    // with top_k all bins up to the end's are listed and none races here
    const float lower = edge_of(s.by_rank() ? 0 : end.bin), upper = edge_of(end.bin + 1);
    each_pack<T, 1>(logits_of<T>(c, row), lo, hi, [&](int32_t i, const float(&v)[N], int) {
      // all random numbers of the pack's kept words are asked for before the
      // first is used
      float x[N], r[N];
      bool keep[N];
#pragma unroll
      for (int j = 0; j < N; j++) {
        x[j] = x_of(v[j], max, s.inverse);
        keep[j] = !(1.0f - x[j] >= lower) && x[j] >= s.floor && v[j] != -INFINITY;
        r[j] = 0.0f;
        if (keep[j]) r[j] = u[i + j];
      }
#pragma unroll
      for (int j = 0; j < N; j++) {
        if (keep[j]) {
          const float score = score_in_race(x[j], r[j]);
          if (score > best) {
            best = score;
            at = i + j;
          }
        }
        if (1.0f - x[j] >= lower && !(1.0f - x[j] >= upper) && v[j] != -INFINITY) {
          const uint32_t slot = atomicAdd(count, 1u);
          if (slot < capacity) list[slot] = make_uint2(key_of(v[j]), (uint32_t)(i + j));
        }
      }
    });
  }
  return at < 0 ? 0 : entry_of(best, at);
}

__device__ __forceinline__ u64 order_of(uint32_t key, uint32_t index) {
  return (u64)key << 32 | (uint32_t)~index;
}

// f(key, index) for the words that race() lists, found in the row again: for a
// list that did not fit.
template <typename T, typename F>
__device__ void each_listed(const Ctx& c, int row, const Setting& s, float max, const End& end,
                            F f) {
  constexpr int N = 16 / (int)sizeof(T);
  const float lower = edge_of(s.by_rank() ? 0 : end.bin), upper = edge_of(end.bin + 1);
  each_pack<T, 1>(logits_of<T>(c, row), 0, c.a.V, [&](int32_t i, const float(&v)[N], int) {
    for (int j = 0; j < N; j++) {
      const float t = 1.0f - x_of(v[j], max, s.inverse);
      if (v[j] != -INFINITY && (s.bounded() ? v[j] >= end.bound : t >= lower && !(t >= upper)))
        f(key_of(v[j]), (uint32_t)(i + j));
    }
  });
}

// LDS of a block of SMALL threads that picks; so many listed words are sorted.
template <int SMALL>
struct Pick {
  u64 order[SMALL], digits[256];
  u64 prefix, above;
  uint32_t taken;
};

// The winner among the listed words and `best`, in every thread. each(f) calls
// f(key, index) for the thread's share of the n listed words.
template <int SMALL, typename E>
__device__ u64 pick(const Ctx& c, int row, const Setting& s, float max, const End& end,
                    uint32_t n, u64 best, Pick<SMALL>& k, u64* wide, E each) {
  const int tid = threadIdx.x;
  const float* u = c.a.uniforms + (int64_t)row * c.a.ldu;
  const u64 target = s.by_rank() ? (u64)s.k : end.target - end.above;
  auto weight = [&](uint32_t key) {
    return weight_of(x_of(score_of(key), max, s.inverse), c.fixed_bits);
  };
  u64 lowest = 0;  // listed words of this order or above are kept
  if (n > SMALL) {
    // The order of the last kept word, by up to 8 bits at a time of those in
    // which the listed words differ.
    if (tid == 0) k.prefix = 0;
    __syncthreads();
    each([&](uint32_t key, uint32_t i) { k.prefix = order_of(key, i); });  // any of them
    __syncthreads();
    u64 prefix = k.prefix, differ = 0, above = 0;
    __syncthreads();
    each([&](uint32_t key, uint32_t i) { differ |= order_of(key, i) ^ prefix; });
    differ = block_or(differ, wide);
    int decided = 64;  // bits from here on are the prefix's
    while (differ != 0) {
      const int top = 63 - __builtin_clzll(differ), shift = top < 7 ? 0 : top - 7;
      for (int i = tid; i < 256; i += blockDim.x) k.digits[i] = 0;
      __syncthreads();
      each([&](uint32_t key, uint32_t i) {
        const u64 o = order_of(key, i);
        if (decided < 64 && (o ^ prefix) >> decided != 0) return;
        atomicAdd(&k.digits[(o >> shift) & 255], s.by_rank() ? 1ull : weight(key));
      });
      __syncthreads();
      if (tid < 64) {  // a lane has four digits, from the largest down
        u64 d[4], own = 0;
#pragma unroll
        for (int i = 0; i < 4; i++) own += d[i] = k.digits[255 - tid * 4 - i];
        u64 upto = own;
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
          const u64 o = __shfl_up(upto, i);
          if (tid >= i) upto += o;
        }
        u64 before = above + upto - own;
        // the lane that reaches the target; the last one if rounding left none
        const bool reached = above + upto >= target;
        const u64 lanes = __ballot(reached);
        const int first = lanes == 0 ? 63 : __builtin_ctzll(lanes);
        if (tid == first) {
          int i = 0;
#pragma unroll
          for (int j = 0; j < 3; j++) {
            if (i == j && before + d[j] < target) {
              before += d[j];
              i = j + 1;
            }
          }
          const u64 digit = (u64)(255 - tid * 4 - i);
          k.prefix = (prefix & ~(255ull << shift)) | digit << shift;
          k.above = before;
        }
      }
      __syncthreads();
      prefix = k.prefix;
      above = k.above;
      __syncthreads();
      decided = shift;
      differ &= (1ull << shift) - 1;
    }
    lowest = prefix;
  }
  if (!s.by_rank() && n > SMALL) {
    each([&](uint32_t key, uint32_t i) {
      const float x = x_of(score_of(key), max, s.inverse);
      if (order_of(key, i) < lowest || !(x >= s.floor)) return;
      const u64 r = race_of(x, u[i], (int32_t)i);
      best = r > best ? r : best;
    });
    return block_best(best, wide);
  }
  // Few words: sorted, a thread each.
  if (tid == 0) k.taken = 0;
  for (int i = tid; i < SMALL; i += blockDim.x) k.order[i] = 0;
  __syncthreads();
  each([&](uint32_t key, uint32_t i) {
    const u64 o = order_of(key, i);
    if (o < lowest) return;
    const uint32_t slot = atomicAdd(&k.taken, 1u);
    if (slot < SMALL) k.order[slot] = o;
  });
  __syncthreads();
  const int count = (int)(k.taken < SMALL ? k.taken : SMALL);
  int size = 64;
  while (size < count) size <<= 1;
  const u64 o = sorted(k.order[tid], size, k.order);
  const uint32_t key = (uint32_t)(o >> 32);
  const bool mine = tid < count;
  const float x = mine ? x_of(score_of(key), max, s.inverse) : -INFINITY;
  const u64 w = mine && (!s.by_rank() || tid < s.k) ? weight_of(x, c.fixed_bits) : 0;
  u64 total;
  const u64 before = block_scan(w, wide, total) - w;
  bool keep = mine && x >= s.floor;
  if (s.by_rank()) {
    keep = keep && tid < s.k;
    if (s.by_weight())
      keep = keep && (tid == 0 || before < (u64)ceil((double)s.p * (double)total));
  } else {
    keep = keep && before < target;
  }
  if (keep) {
    const int32_t i = (int32_t)~(uint32_t)o;
    const u64 r = race_of(x, u[i], i);
    best = r > best ? r : best;
  }
  return block_best(best, wide);
}

__device__ void write_none(const Ctx& c, int row, const Setting& s) {
  if (threadIdx.x != 0) return;
  c.a.ids[row] = -1;
  if (c.a.logprob != nullptr) c.a.logprob[row] = NAN;
  if (!s.ok) report_row(c.a.status);
}
// By one thread. The sum of all weights is 1 + rest; rest by itself keeps the
// log-probability of a nearly certain word as exact as any.
__device__ __forceinline__ void write_word(const Ctx& c, int row, int32_t id, float x,
                                           float rest) {
  c.a.ids[row] = id;
  if (c.a.logprob != nullptr) c.a.logprob[row] = x - log1pf(rest);
}

// A row by one block.
// (72 registers are enough for a block of 256 threads, whose LDS lets two share a
// CU; two of 1024 need 64)
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, THREADS == 1024 ? 8 : 2) void k_row(Ctx c) {
  __shared__ float scratch[32];
  __shared__ u64 wide[16];
  __shared__ u64 bins[kBins];
  __shared__ uint2 list[kLocalRow];
  static_assert(kLocalRow * 8 >= THREADS * 4, "the list holds the threads' maxima");
  __shared__ Pick<THREADS> k;
  __shared__ End shared_end;
  __shared__ uint32_t count;
  const int row = blockIdx.x, tid = threadIdx.x;
  const Setting s = setting(c, row);
  const bool filters = s.filters();
  if (s.binned())
    for (int i = tid; i < kBins; i += THREADS) bins[i] = 0;
  if (tid == 0) count = 0;
  const Part p = scan<T>(c, row, s, 0, c.a.V, scratch, wide, (uint32_t*)list);
  const float max = p.max;
  if (!s.ok || p.nan || !(max > -INFINITY)) return write_none(c, row, s);
  if (s.greedy) {
    if (tid == 0) write_word(c, row, p.first, 0.0f, 0.0f);
    return;
  }
  End end = {kBins, 0, 0, p.bound};
  if (s.binned()) {
    add_bins<T>(c, row, s, max, 0, c.a.V, bins);
    __syncthreads();
    end = end_of(s, bins, wide, &shared_end);
  }
  u64 best = race<T>(c, row, s, max, end, 0, c.a.V, list, kLocalRow, &count);
  __syncthreads();
  if (filters) {
    const uint32_t n = count;
    best = pick(c, row, s, max, end, n, best, k, wide, [&](auto f) {
      if (n <= kLocalRow) {
        for (uint32_t i = tid; i < n; i += THREADS) f(list[i].x, list[i].y);
      } else {
        each_listed<T>(c, row, s, max, end, f);
      }
    });
  } else {
    best = block_best(best, wide);
  }
  if (tid == 0) {
    const int32_t id = (int32_t)~(uint32_t)best;
    write_word(c, row, id, x_of(to_f32(logits_of<T>(c, row)[id]), max, s.inverse), p.rest);
  }
}

// The row's maximum from its parts (a NaN in the row makes it NaN) and the sum
// of its weights but for one word at the maximum, in every thread; the parts are
// read by the wave's lanes.
__device__ float row_max(const Ctx& c, int row, const Setting& s, float& rest, float& bound) {
  const Part* parts = c.parts + (int64_t)row * c.splits;
  float m = -INFINITY, nan = 0.0f;
  bound = -INFINITY;  // k words of one share reach its bound, so the largest serves
  for (int i = threadIdx.x & 63; i < c.splits; i += 64) {
    m = fmaxf(m, parts[i].max);
    bound = fmaxf(bound, parts[i].bound);
    nan = fmaxf(nan, parts[i].nan != 0 ? 1.0f : 0.0f);
  }
  m = wave_max(m);
  nan = wave_max(nan);
  bound = wave_max(bound);
  rest = 0.0f;
  float tops = 0.0f;  // parts at the maximum
  for (int i = threadIdx.x & 63; i < c.splits; i += 64) {
    const bool top = parts[i].max == m;
    tops += top ? 1.0f : 0.0f;
    if (top)
      rest += parts[i].rest;
    else if (parts[i].max != -INFINITY)
      rest += (1.0f + parts[i].rest) * exp2_fast(x_of(parts[i].max, m, s.inverse * kLog2e));
  }
  rest = wave_sum(rest) + (wave_sum(tops) - 1.0f);
  return nan > 0.0f ? NAN : m;
}

__device__ __forceinline__ void share_of(const Ctx& c, int& row, int& split, int64_t& lo,
                                         int64_t& hi) {
  row = blockIdx.x / c.splits;
  split = blockIdx.x % c.splits;
  lo = split * c.range;
  hi = lo + c.range < c.a.V ? lo + c.range : c.a.V;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_scan(Ctx c) {
  __shared__ float scratch[32];
  __shared__ u64 wide[16];
  __shared__ uint32_t buffer[kThreads];
  int row, split;
  int64_t lo, hi;
  share_of(c, row, split, lo, hi);
  const Setting s = setting(c, row);
  // the share of what later passes add to
  if (c.bins)
    for (int i = split * kThreads + threadIdx.x; i < kBins; i += c.splits * kThreads)
      c.hist[(int64_t)row * kBins + i] = 0;
  if (split == 0 && threadIdx.x == 0) c.listed[row] = 0;
  const Part p = scan<T>(c, row, s, lo, hi, scratch, wide, buffer);
  if (threadIdx.x == 0) c.parts[(int64_t)row * c.splits + split] = p;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_bins(Ctx c) {
  __shared__ u64 bins[kBins];
  int row, split;
  int64_t lo, hi;
  share_of(c, row, split, lo, hi);
  const Setting s = setting(c, row);
  float rest, bound;
  const float max = row_max(c, row, s, rest, bound);
  if (!s.binned() || !(max > -INFINITY)) return;
  for (int i = threadIdx.x; i < kBins; i += kThreads) bins[i] = 0;
  __syncthreads();
  add_bins<T>(c, row, s, max, lo, hi, bins);
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kThreads)
    if (bins[i] != 0) atomicAdd(&c.hist[(int64_t)row * kBins + i], bins[i]);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_race(Ctx c) {
  __shared__ u64 wide[16];
  __shared__ uint2 list[kLocal];
  __shared__ End shared_end;
  __shared__ uint32_t count, base;
  int row, split;
  int64_t lo, hi;
  share_of(c, row, split, lo, hi);
  const Setting s = setting(c, row);
  float rest, bound;
  const float max = row_max(c, row, s, rest, bound);
  if (s.greedy || !s.ok || !(max > -INFINITY)) return;
  if (threadIdx.x == 0) count = 0;
  End end = {kBins, 0, 0, bound};
  if (s.binned()) end = end_of(s, c.hist + (int64_t)row * kBins, wide, &shared_end);
  __syncthreads();
  u64 best = race<T>(c, row, s, max, end, lo, hi, list, kLocal, &count);
  best = block_best(best, wide);
  if (threadIdx.x == 0) {
    c.parts[(int64_t)row * c.splits + split].best = best;
    // a list that did not fit here cannot be whole in memory either
    base = count == 0 ? 0
                      : atomicAdd(&c.listed[row], count > kLocal ? kCapacity + 1u : count);
  }
  __syncthreads();
  if (count > kLocal) return;
  for (uint32_t i = threadIdx.x; i < count; i += kThreads)
    if (base + i < kCapacity) c.list[(int64_t)row * kCapacity + base + i] = list[i];
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS, 8) void k_pick(Ctx c) {
  __shared__ u64 wide[16];
  __shared__ Pick<THREADS> k;
  __shared__ End shared_end;
  const int row = blockIdx.x, tid = threadIdx.x;
  const Setting s = setting(c, row);
  float rest, bound;
  const float max = row_max(c, row, s, rest, bound);
  if (!s.ok || !(max > -INFINITY)) return write_none(c, row, s);
  const Part* parts = c.parts + (int64_t)row * c.splits;
  u64 best = 0;
  for (int i = tid; i < c.splits; i += THREADS) {
    const u64 b = s.greedy ? (parts[i].max == max ? (u64)(uint32_t)~parts[i].first : 0)
                           : parts[i].best;
    best = b > best ? b : best;
  }
  if (s.filters()) {
    End end = {kBins, 0, 0, bound};
    if (s.binned()) end = end_of(s, c.hist + (int64_t)row * kBins, wide, &shared_end);
    const uint32_t n = c.listed[row];
    best = pick(c, row, s, max, end, n, best, k, wide, [&](auto f) {
      if (n <= kCapacity) {
        const uint2* list = c.list + (int64_t)row * kCapacity;
        for (uint32_t i = tid; i < n; i += THREADS) f(list[i].x, list[i].y);
      } else {
        each_listed<T>(c, row, s, max, end, f);
      }
    });
  } else {
    best = block_best(best, wide);
  }
  if (tid == 0) {
    const int32_t id = (int32_t)~(uint32_t)best;
    if (s.greedy)
      write_word(c, row, id, 0.0f, 0.0f);
    else
      write_word(c, row, id, x_of(to_f32(logits_of<T>(c, row)[id]), max, s.inverse), rest);
  }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Blocks of a row: enough for the GPU to be full with few rows, each with at
// least 2048 words.
int splits_of(int32_t rows, int32_t V) {
  const int64_t most = ceil_div(V, 2048);
  int64_t want = ceil_div(2048, rows > 0 ? rows : 1);
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

// Words of a row that a block of 256 threads does as fast as one of 1024. With
// 256 and 1,024, fp32, us: 512 rows of 1,000 top_p 16 and 26; of 8,192 24 and 30,
// top_k 50 19 and 33; of 16,000 top_p 41 and 35; 64 rows of 8,192 22 and 20.
constexpr int kShortRow = 8192;

// Whether a block does a whole row: short rows, or enough rows to fill the GPU,
// fewer of them the shorter they are. By a block and by shares (us): 1 row of
// 71,290 fp32 words, top_p, 48 and 34; 100 of 50,000 bf16 38 and 59; 257 of
// 100,000 fp16 (top_k 50) 46 and 61; 64 of 10^6 bf16 (top_k 50) 112 and 69. Below
// the limit, one row of 8,192 fp32 words, top_p, 19 and 28, of 40,000 30 and 28, of
// 65,536 39 and 29 (top_k 40 27 and 22); 64 rows of 40,000 34 and 50, of 65,536 45
// and 63.
bool row_by_block(int32_t rows, int32_t V) {
  return V <= 65536 || (rows >= 128 && V <= 131072) || rows >= 512;
}

template <typename T>
hipError_t launch_as(const Ctx& c, hipStream_t s) {
  const int rows = c.a.rows, V = c.a.V;
  // a small block's barriers cost less; a top_k beyond its threads needs a
  // large one
  const bool few = c.a.top_ks == nullptr && (c.a.top_k <= kBounded || c.a.top_k >= V);
  if (row_by_block(rows, V)) {
    if (few && V <= kShortRow)
      k_row<T, 256><<<rows, 256, 0, s>>>(c);
    else
      k_row<T, 1024><<<rows, 1024, 0, s>>>(c);
    return hipGetLastError();
  }
  const int grid = rows * c.splits;
  const bool greedy = c.a.temperatures == nullptr && c.a.temperature == 0.0f;
  k_scan<T><<<grid, kThreads, 0, s>>>(c);
  if (c.bins) k_bins<T><<<grid, kThreads, 0, s>>>(c);
  if (!greedy) k_race<T><<<grid, kThreads, 0, s>>>(c);
  if (few)
    k_pick<T, 256><<<rows, 256, 0, s>>>(c);
  else
    k_pick<T, 1024><<<rows, 1024, 0, s>>>(c);
  return hipGetLastError();
}

}  // namespace

size_t sample_workspace_bytes(int32_t rows, int32_t V) {
  return row_by_block(rows, V) ? 0 : layout(rows, V).total;
}

static hipError_t launch_part(const SampleArgs& a, void* workspace, hipStream_t s) {
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
  const bool bounded = a.top_ks == nullptr && rank && a.top_k <= kBounded;
  c.bins = (rank || weight) && !bounded &&
           !(a.temperatures == nullptr && a.temperature == 0.0f);
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

hipError_t launch_sample(const SampleArgs& a, void* workspace, hipStream_t s) {
  const int most = rows_of_launch(a.rows);
  hipError_t e = hipSuccess;
  for (int64_t row = 0; row < a.rows && e == hipSuccess; row += most) {
    SampleArgs part = a;
    part.rows = (int32_t)(a.rows - row < most ? a.rows - row : most);
    part.logits = row_at(a.logits, row, a.ld, a.dtype);
    part.uniforms = row_at(a.uniforms, row, a.ldu);
    part.temperatures = row_at(a.temperatures, row);
    part.top_ks = row_at(a.top_ks, row);
    part.top_ps = row_at(a.top_ps, row);
    part.min_ps = row_at(a.min_ps, row);
    part.ids = row_at(a.ids, row);
    part.logprob = row_at(a.logprob, row);
    e = launch_part(part, workspace, s);
  }
  return e;
}

}  // namespace w2v
