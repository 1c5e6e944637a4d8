// A step of beam search: of an entry's live beams b, with running scores c_b, and
// the words v, the `width` pairs with the largest
//
//   c_b + log p_b(v) = (c_b - log sum exp z_b) + z_bv,
//
// and the beams' states moved to where their continuations are.
//
// The scores are read once. A row is cut into shares that one block holds in its
// registers; the block writes the share's maximum and sum, and its `width` best
// words, sorted. A second kernel, a block an entry, joins the sums and takes the
// best of all shares' words. Words of one beam are ranked by their score, equal
// ones by index, and no sum comes into that; pairs of different beams by the sum
// above in 64 bits, equal ones by beam.
//
// The best words of a share lie above a bound that at least `width` of them reach: the
// width-th largest of the maxima of groups of its threads. Packs of scores with such a
// word go to a list in LDS, its words to another one, and are ranked there by counting.
// Of too many words those above the bound are taken, and the first that equal it (32 x 8
// beams of 100,000 words all alike 45 us, one after the other 105); if that is still more
// than the list holds, one after the other.
//
// Of the instructions for a score the exponential takes four slots of about nine, which
// is about what reading 16-bit scores leaves time for. Measured: 16 x 16 beams of 10^6
// words fp16 107 us (512 MB at 4.8 TB/s; shares 96 with the scores partly cached, merge
// 17), 32 x 8 of 100,000 bf16 with two states 31 us (16, 9, and 5 for the states), 1 x 4
// of 71,290 fp32 29 us, 18 of them in the kernels.
#include "beam.h"
#include "head_types.h"

namespace w2v {
namespace {

constexpr int kWave = 64;
constexpr int kBlock = 256;
constexpr int kWaves = kBlock / kWave;
constexpr int kMaxGrid = 1 << 22;
constexpr int kList = 1024;
constexpr int kPackList = 512;
constexpr int kMany = 256;  // words that are ranked at once without a second look
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ bool live_score(float c) { return c > -kInf; }  // not NaN

// What a share leaves: {maximum, sum of exp(z - maximum)}, and `width` words.
struct Share {
  float most, sum;
};
struct Word {
  float z;
  int32_t id;
};
__device__ __forceinline__ bool better(const Word& a, const Word& b) {
  return (a.z > b.z) | ((a.z == b.z) & (a.id < b.id));
}

__device__ __forceinline__ Word best_of_wave(Word w) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const Word o = {__shfl_xor(w.z, d), __shfl_xor(w.id, d)};
    if (better(o, w)) w = o;
  }
  return w;
}

// The n-th largest of the maxima of 64 groups of four threads, or of all threads'
// values for n > 16 or ALL, by counting the larger ones: what at least n values of
// the block's threads reach. begin() and, behind a barrier, end() of all threads; the
// result is there behind another one.
struct Bound {
  float groups[kBlock];
  float waves[kWaves];

  template <bool ALL>
  __device__ __forceinline__ static bool few(int n) {
    return !ALL && n <= 16;
  }
  template <bool ALL = false>
  __device__ __forceinline__ void begin(float v, int n) {
    if (few<ALL>(n)) {
      v = fmaxf(v, __shfl_xor(v, 1));
      v = fmaxf(v, __shfl_xor(v, 2));
      if ((threadIdx.x & 3) == 0) groups[threadIdx.x >> 2] = v;
    } else {
      groups[threadIdx.x] = v;
    }
  }
  template <bool ALL = false>
  __device__ __forceinline__ void end(int n) {
    const int count = few<ALL>(n) ? kBlock / 4 : kBlock;
    if ((int)threadIdx.x >= count) return;
    const float mine = groups[threadIdx.x];
    int above = 0;
#pragma unroll 2
    for (int i = 0; i < count; i += 4) {
      const f32x4 o = *(const f32x4*)(groups + i);
      above += (o[0] > mine) + (o[1] > mine) + (o[2] > mine) + (o[3] > mine);
    }
    const float least = -wave_max(above < n ? -mine : -kInf);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = least;
  }
  template <bool ALL = false>
  __device__ __forceinline__ float get(int n) const {
    float least = waves[0];
    if (!few<ALL>(n))
      for (int w = 1; w < kWaves; w++) least = fminf(least, waves[w]);
    return least;
  }
};

template <typename T, int PACKS>
struct Row {
  static constexpr int kE = 16 / (int)sizeof(T);
  static constexpr int kShare = kBlock * PACKS * kE;
  word4 w[PACKS];

  __device__ __forceinline__ static word4 load(const T* p) {
    return __builtin_bit_cast(word4, load_16(p));
  }
  // Elements [first, first + kShare) of the n of a row; -inf past its end.
  __device__ __forceinline__ void load(const T* row, int64_t first, int64_t n) {
    const int64_t mine = first + threadIdx.x * kE;
    if (first + kShare <= n) {
#pragma unroll
      for (int p = 0; p < PACKS; p++) w[p] = load(row + mine + p * kBlock * kE);
      return;
    }
    // the row's last pack, where it is not whole
    const int64_t whole = n - n % kE;
    Pack<T, kE> tail, gone;
#pragma unroll
    for (int e = 0; e < kE; e++) {
      gone.v[e] = from_f32<T>(-kInf);
      tail.v[e] = whole + e < n ? row[whole + e] : gone.v[e];
    }
#pragma unroll
    for (int p = 0; p < PACKS; p++) {
      const int64_t i = mine + p * kBlock * kE;
      if (i < whole)
        w[p] = load(row + i);
      else
        w[p] = __builtin_bit_cast(word4, i < n ? tail : gone);
    }
  }
  // Keeps the compiler from holding what one reading unpacked for the next: 8
  // registers a pack instead of 4, and two wavefronts a SIMD instead of five.
  __device__ __forceinline__ void repack(int p) {
    asm volatile("" : "+v"(w[p]));
  }
  // The largest score of pack p, of NaN's others.
  __device__ __forceinline__ float most(int p) {
    float z[kE];
    repack(p);
    unpack_words<T>(__builtin_bit_cast(uint4, w[p]), z);
    float m = fmaxf(z[0], z[1]);
#pragma unroll
    for (int e = 2; e < kE; e += 2) m = fmaxf(m, fmaxf(z[e], z[e + 1]));
    asm volatile("" : "+v"(m));
    return m;
  }
  // Which scores of pack p equal v, as bits.
  __device__ __forceinline__ uint32_t equal(int p, float v) {
    float z[kE];
    repack(p);
    unpack_words<T>(__builtin_bit_cast(uint4, w[p]), z);
    uint32_t bits = 0;
#pragma unroll
    for (int e = 0; e < kE; e++) bits |= z[e] == v ? 1u << e : 0;
    asm volatile("" : "+v"(bits));
    return bits;
  }
  // Sum of exp(z - top). Of fp16 exp2(z k - t), t the rounded top k, is one
  // instruction before the exponential, with the conversion, where exp2((z - top) k)
  // takes three; that sum is 2^(top k - t) times too large or small, at most
  // 1 +- 0.006 as no fp16 is over 2^16, and the series of that factor is off by 4e-11.
  __device__ __forceinline__ float sum_exp(float top) {
    float sum = 0.0f;
    if constexpr (__is_same(T, f16_t)) {
      const float t = top * kLog2e;
      add(sum, [&](float v) { return fmaf(v, kLog2e, -t); });
      const float x = fmaf(-kLog2e, top, t) * 0.6931471805599453f;
      return fmaf(sum, fmaf(x * x, fmaf(x, 1.0f / 6, 0.5f), x), sum);
    } else {
      add(sum, [&](float v) { return (v - top) * kLog2e; });
      return sum;
    }
  }
  template <typename F>
  __device__ __forceinline__ void add(float& sum, F&& power) {
#pragma unroll
    for (int p = 0; p < PACKS; p++) {
      float z[kE];
      repack(p);
      unpack_words<T>(__builtin_bit_cast(uint4, w[p]), z);
#pragma unroll
      for (int e = 0; e < kE; e++) sum += exp2_fast(power(z[e]));
      asm volatile("" : "+v"(sum));
    }
  }
  // f(score, index in the share), in order of the index
  template <typename F>
  __device__ __forceinline__ void each(F&& f) {
#pragma unroll
    for (int p = 0; p < PACKS; p++) {
      float z[kE];
      repack(p);
      unpack_words<T>(__builtin_bit_cast(uint4, w[p]), z);
      int first = (int)threadIdx.x * kE;
      asm volatile("" : "+v"(first));  // not an index for each element at once
#pragma unroll
      for (int e = 0; e < kE; e++) f(z[e], first + p * kBlock * kE + e);
    }
  }
};

// The next larger fp32 number of a finite one.
__device__ __forceinline__ float next_above(float v) {
  const int32_t bits = __builtin_bit_cast(int32_t, v);
  if (v == 0.0f) return __builtin_bit_cast(float, 1);
  return __builtin_bit_cast(float, bits + (bits < 0 ? -1 : 1));
}

// Puts the first `most` of a share's scores that equal v, by index, into a list.
// Returns how many there are of them.
template <typename T, int PACKS>
__device__ __forceinline__ int take_equal(Row<T, PACKS>& z, float v, int most,
                                          int (&of_waves)[kWaves], Word* list) {
  constexpr int kE = Row<T, PACKS>::kE, kBits = PACKS * kE, kWords = (kBits + 31) / 32;
  uint32_t mask[kWords] = {};
#pragma unroll
  for (int p = 0; p < PACKS; p++) mask[p * kE / 32] |= z.equal(p, v) << (p * kE % 32);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int total = 0;
  for (int p = 0; p < PACKS && total < most; p++) {
    uint32_t here = 0;
#pragma unroll
    for (int i = 0; i < kWords; i++)
      if (p * kE / 32 == i) here = mask[i];
    here = here >> (p * kE % 32) & ((1u << kE) - 1);
    const int mine = __popc(here);
    int upto = mine;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const int below = __shfl_up(upto, d);
      if (lane >= d) upto += below;
    }
    if (lane == kWave - 1) of_waves[wave] = upto;
    __syncthreads();
    int at = total + upto - mine;
    for (int w = 0; w < kWaves; w++) {
      if (w < wave) at += of_waves[w];
      total += of_waves[w];
    }
    for (; here != 0 && at < most; here &= here - 1)
      list[at++] = {v, (p * kBlock + (int)threadIdx.x) * kE + __builtin_ctz(here)};
    __syncthreads();
  }
  return total < most ? total : most;
}

template <typename T, int PACKS>
__global__ __launch_bounds__(kBlock, 4) void k_beam_shares(BeamArgs a, int shares, Share* out,
                                                        Word* best) {
  __shared__ __attribute__((aligned(16))) Bound s_bound;
  __shared__ float s_wave[2 * kWaves];
  __shared__ int s_packs, s_count;
  __shared__ word4 s_pack[kPackList];
  __shared__ int s_first[kPackList];
  __shared__ Word s_list[kList];
  __shared__ int s_equal[kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  constexpr int kE = Row<T, PACKS>::kE;
  const int64_t units = (int64_t)a.batch * a.beams * shares;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t row = unit / shares;
    // of an ended beam and of one that is none, nothing is read
    if (a.finished != nullptr && a.finished[row] != 0) continue;
    if (!live_score(a.scores[row])) continue;
    const int64_t first = (unit - row * shares) * Row<T, PACKS>::kShare;
    Row<T, PACKS> z;
    z.load((const T*)a.logits + row * a.ld, first, a.V);
    // the largest of every kPer packs, so that the others are not read for words
    constexpr int kPer = PACKS > 1 ? 2 : 1;
    float most = -kInf, of_packs[PACKS / kPer];
#pragma unroll
    for (int p = 0; p < PACKS; p += kPer) {
      float m = z.most(p);
      if constexpr (kPer > 1) m = fmaxf(m, z.most(p + 1));
      most = fmaxf(most, of_packs[p / kPer] = m);
    }
    s_bound.begin(most, a.width);
    const float of_wave = wave_max(most);
    if (lane == 0) s_wave[wave] = of_wave;
    if (threadIdx.x == 0) s_packs = s_count = 0;
    __syncthreads();
    most = s_wave[0];
#pragma unroll
    for (int w = 1; w < kWaves; w++) most = fmaxf(most, s_wave[w]);
    s_bound.end(a.width);
    // a share of -inf alone has sum 0; NaN and +inf make it NaN
    float sum = wave_sum(z.sum_exp(most > -kInf ? most : 0.0f));
    if (lane == 0) s_wave[kWaves + wave] = sum;
    __syncthreads();
    // the packs that hold words to take, then those words; of a NaN neither
    const auto take = [&](float from) {
#pragma unroll
      for (int p = 0; p < PACKS; p += kPer)
        if (of_packs[p / kPer] >= from) {
          const int at = atomicAdd(&s_packs, kPer);
          if (at <= kPackList - kPer) {
#pragma unroll
            for (int u = 0; u < kPer; u++) {
              s_pack[at + u] = z.w[p + u];
              s_first[at + u] = ((p + u) * kBlock + (int)threadIdx.x) * kE;
            }
          }
        }
      __syncthreads();
      const int packs = s_packs;
      if (packs <= kPackList)
        for (int i = threadIdx.x; i < packs * kE; i += kBlock) {
          const float v = to_f32(((const T*)s_pack)[i]);
          if (v >= from) {
            const int at = atomicAdd(&s_count, 1);
            if (at < kList) s_list[at] = {v, s_first[i / kE] + i % kE};
          }
        }
      __syncthreads();
      return packs <= kPackList ? s_count : kList + 1;
    };
    const float bound = fmaxf(s_bound.get(a.width), -__FLT_MAX__);
    int count = take(bound);
    if (count > kMany) {
      // what is more than the bound, and the first `width` of those that equal it: a
      // model whose scores are all alike takes no longer
      __syncthreads();
      if (threadIdx.x == 0) s_packs = s_count = 0;
      __syncthreads();
      count = take(next_above(bound));
      if (count < a.width)
        count += take_equal(z, bound, a.width - count, s_equal, s_list + count);
    }
    Word* to = best + unit * a.width;
    if (count <= kList) {
      for (int i = threadIdx.x; i < count; i += kBlock) {
        const Word mine = s_list[i];
        int rank = 0;
#pragma unroll 4
        for (int j = 0; j < count; j++) rank += better(s_list[j], mine);
        if (rank < a.width) to[rank] = {mine.z, (int32_t)(first + mine.id)};
      }
      for (int i = count + threadIdx.x; i < a.width; i += kBlock) to[i] = {-kInf, -1};
    } else {
      Word last = {kInf, -1};
      for (int i = 0; i < a.width; i++) {
        Word mine = {-kInf, 0x7fffffff};
        z.each([&](float v, int id) {
          if (v > mine.z && better(last, {v, id})) mine = {v, id};
        });
        mine = best_of_wave(mine);
        __syncthreads();
        if (lane == 0) s_list[wave] = mine;
        __syncthreads();
        last = s_list[0];
#pragma unroll
        for (int w = 1; w < kWaves; w++)
          if (better(s_list[w], last)) last = s_list[w];
        if (threadIdx.x == 0)
          to[i] = {last.z, last.z > -kInf ? (int32_t)(first + last.id) : -1};
      }
    }
    if (threadIdx.x == 0) {
      sum = 0.0f;
      for (int w = 0; w < kWaves; w++) sum += s_wave[kWaves + w];
      out[unit] = {most, sum};
    }
    __syncthreads();
  }
}

// A pair of beam and word, in the order in which they are taken.
struct Pair {
  double key;
  float z;
  int32_t beam, id;
};
// Without a branch, so that loops over it are unrolled with their loads in flight.
__device__ __forceinline__ bool better(const Pair& a, const Pair& b) {
  const bool word = (a.z > b.z) | ((a.z == b.z) & (a.id < b.id));
  const bool beam = (a.beam < b.beam) | ((a.beam == b.beam) & word);
  return (a.key > b.key) | ((a.key == b.key) & beam);
}

__device__ __forceinline__ Pair best_of_wave(Pair p) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    const Pair o = {__shfl_xor(p.key, d), __shfl_xor(p.z, d), __shfl_xor(p.beam, d),
                    __shfl_xor(p.id, d)};
    if (better(o, p)) p = o;
  }
  return p;
}

__global__ __launch_bounds__(kBlock) void k_beam_merge(BeamArgs a, int shares, const Share* share,
                                                       const Word* best) {
  __shared__ double s_add[W2V_MAX_BEAMS];     // what a beam's scores are added to
  __shared__ uint8_t s_kind[W2V_MAX_BEAMS];   // 0: no word, 1: live, 2: ended
  __shared__ int s_bad, s_count, s_hot, s_lists[kList];
  __shared__ __attribute__((aligned(16))) Bound s_bound;
  __shared__ __attribute__((aligned(16))) double s_key[kList + 4];
  // beam, word: the order of equal keys
  __shared__ __attribute__((aligned(16))) uint64_t s_tie[kList + 4];
  __shared__ __attribute__((aligned(16))) float s_z[kList + 4];
  __shared__ Pair s_list[kList];
  const Pair none = {-(double)kInf, -kInf, 0x7fffffff, 0x7fffffff};
  int team = kWave;
  while (team > 4 && team * a.beams > kBlock) team /= 2;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int64_t entry = blockIdx.x; entry < a.batch; entry += gridDim.x) {
    if (threadIdx.x == 0) s_bad = s_count = s_hot = 0;
    __syncthreads();
    // a beam's shares are joined by a team of lanes, all beams at once
    for (int b0 = 0; b0 < a.beams; b0 += kBlock / team) {
      const int b = b0 + (int)threadIdx.x / team, part = (int)threadIdx.x & (team - 1);
      const int64_t row = entry * a.beams + (b < a.beams ? b : 0);
      const float c = a.scores[row];
      const bool ended = a.finished != nullptr && a.finished[row] != 0;
      const bool live = c > -kInf && c < kInf && !ended;
      float most = -kInf;
      double sum = 0.0;
      if (live)
        for (int i = part; i < shares; i += team) most = fmaxf(most, share[row * shares + i].most);
      for (int d = team / 2; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
      if (live)
        for (int i = part; i < shares; i += team) {
          const Share s = share[row * shares + i];
          // of a share of -inf alone the sum is 0, or NaN if it holds one
          sum += s.most > -kInf ? s.sum * exp((double)s.most - most) : (double)s.sum;
        }
      for (int d = team / 2; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
      if (part == 0 && b < a.beams) {
        int kind = 0;
        double add = 0.0;
        if (!(c < kInf) || sum != sum || most == kInf) {
          s_bad = 1;  // +inf or NaN
        } else if (c > -kInf && ended) {
          kind = 2;
          add = c;
        } else if (most > -kInf) {
          kind = 1;
          add = (double)c - ((double)most + log(sum));
        }
        s_add[b] = add;
        s_kind[b] = (uint8_t)kind;
      }
    }
    __syncthreads();
    const int64_t out = entry * a.width;
    const auto write = [&](int i, const Pair& p, bool there) {
      a.words[out + i] = there ? p.id : -1;
      a.parents[out + i] = there ? p.beam : -1;
      a.new_scores[out + i] = s_bad != 0 ? __builtin_nanf("") : (float)p.key;
      if (a.new_finished != nullptr)
        a.new_finished[out + i] = there && (s_kind[p.beam] == 2 || p.id == a.end) ? 1 : 0;
    };
    if (s_bad != 0) {
      for (int i = threadIdx.x; i < a.width; i += kBlock) write(i, none, false);
      __syncthreads();
      continue;
    }
    // Each list's words go to `ways` threads in turn (a thread has whole lists
    // where there are more lists than threads), so a thread's best pair is the
    // first of its first place.
    const int lists = a.beams * shares;
    const int ways = lists < kBlock ? kBlock / lists : 1;
    const int way = ways > 1 ? (int)threadIdx.x / lists : 0;
    const int list0 = ways > 1 ? (int)threadIdx.x - way * lists : (int)threadIdx.x;
    const int64_t list_base = entry * lists;
    const auto pair_of = [&](int list, int place) {
      const int b = list / shares;
      Pair p = none;
      if (s_kind[b] == 1) {
        const Word w = best[(list_base + list) * a.width + place];
        if (w.z > -kInf) p = {s_add[b] + (double)w.z, w.z, b, w.id};
      } else if (s_kind[b] == 2 && place == 0 && list == b * shares) {
        p = {s_add[b], 0.0f, b, a.end};
      }
      return p;
    };
    double first = -(double)kInf;
    if (way < ways && way < a.width)
      for (int list = list0; list < lists; list += kBlock)
        first = fmax(first, pair_of(list, way).key);
    // in fp32: rounding keeps the keys' order, so no pair above the bound is lost
    s_bound.begin((float)first, a.width);
    __syncthreads();
    s_bound.end(a.width);
    __syncthreads();
    // the lists that begin above the bound, then their words, all at once
    const float bound = s_bound.get(a.width);
    if (way == 0)
      for (int list = list0; list < lists; list += kBlock) {
        const Pair p = pair_of(list, 0);
        if ((float)p.key >= bound && p.key > -(double)kInf) {
          const int at = atomicAdd(&s_hot, 1);
          if (at < kList) s_lists[at] = list;
        }
      }
    __syncthreads();
    const auto put = [&](const Pair& p) {
      const int to = atomicAdd(&s_count, 1);
      s_list[to] = p;
      s_key[to] = p.key;
      s_tie[to] = (uint64_t)p.beam << 32 | (uint32_t)p.id;
      s_z[to] = p.z;
    };
    // They are taken into a list of kList, as many at a time as it has room for. Many
    // of them give a closer bound, the width-th largest of what the threads hold, and
    // those below it leave the list: 16 of 174 are ranked in 3 us, with the bound, 174
    // in 9. Equal scores can fill the list.
    const int hot = s_hot, words = hot <= kList ? hot * a.width : 0;
    int count = 0;
    float least = bound;
    for (int from = 0; from < words && count <= kList / 2;) {
      const int stop = words - from < kList - count ? words : from + kList - count;
      for (int i = from + (int)threadIdx.x; i < stop; i += kBlock) {
        const int at = i / a.width;
        const Pair p = pair_of(s_lists[at], i - at * a.width);
        if ((float)p.key >= least && p.key > -(double)kInf) put(p);
      }
      from = stop;
      __syncthreads();
      count = s_count;
      if (count > 4 * a.width) {
        Pair p[kList / kBlock];
        float most = -kInf;
#pragma unroll
        for (int u = 0; u < kList / kBlock; u++) {
          const int i = u * kBlock + (int)threadIdx.x;
          p[u] = none;
          if (i < count) p[u] = s_list[i];
          most = fmaxf(most, (float)p[u].key);
        }
        s_bound.begin<true>(most, a.width);
        __syncthreads();
        if (threadIdx.x == 0) s_count = 0;
        s_bound.end<true>(a.width);
        __syncthreads();
        least = s_bound.get<true>(a.width);
#pragma unroll
        for (int u = 0; u < kList / kBlock; u++)
          if ((float)p[u].key >= least && p[u].key > -(double)kInf) put(p[u]);
        __syncthreads();
        count = s_count;
      }
      __syncthreads();
      if (from < words && count > kList / 2) count = kList + 1;
    }
    if (hot > kList) count = kList + 1;
    // pairs are compared in fours
    if (count <= kList && threadIdx.x < 4) s_key[count + threadIdx.x] = none.key;
    __syncthreads();
    if (count <= kList) {
      // a pair's place by counting the better ones; few pairs have several threads.
      // Scores of one beam that differ, but not in their keys, are rare: such a
      // pair counts again by all that it is ranked by
      int split = kWave;
      while (split > 1 && split * count > kBlock) split /= 2;
      for (int i0 = 0; i0 < count; i0 += kBlock / split) {
        const int i = i0 + (int)threadIdx.x / split, part = (int)threadIdx.x & (split - 1);
        const int at = i < count ? i : 0;
        const double key = s_key[at];
        const uint64_t tie = s_tie[at];
        const float z = s_z[at];
        int rank = 0, merged = 0;
#pragma unroll 2
        for (int j = part * 4; j < count; j += split * 4) {
          const f32x4 zs = *(const f32x4*)(s_z + j);
#pragma unroll
          for (int u = 0; u < 4; u += 2) {
            const double2 keys = *(const double2*)(s_key + j + u);
            const ulonglong2 ties = *(const ulonglong2*)(s_tie + j + u);
            const bool same0 = keys.x == key, same1 = keys.y == key;
            rank += (keys.x > key) | (same0 & (ties.x < tie));
            rank += (keys.y > key) | (same1 & (ties.y < tie));
            merged |= same0 & (ties.x >> 32 == tie >> 32) & (zs[u] != z);
            merged |= same1 & (ties.y >> 32 == tie >> 32) & (zs[u + 1] != z);
          }
        }
        for (int d = split / 2; d > 0; d >>= 1) {
          rank += __shfl_xor(rank, d);
          merged |= __shfl_xor(merged, d);
        }
        if (part == 0 && i < count) {
          const Pair p = s_list[i];
          if (merged) {
            rank = 0;
            for (int j = 0; j < count; j++) rank += better(s_list[j], p);
          }
          if (rank < a.width) write(rank, p, true);
        }
      }
      for (int i = count + threadIdx.x; i < a.width; i += kBlock) write(i, none, false);
    } else {
      // one after the other: of each list the first pair behind the last taken, from
      // where a thread found it before in its first kHeld lists
      constexpr int kHeld = 4;
      Pair last = {(double)kInf, 0.0f, 0, 0};
      int next[kHeld];
#pragma unroll
      for (int u = 0; u < kHeld; u++) next[u] = way;
      for (int n = 0; n < a.width; n++) {
        Pair mine = none;
        const auto look = [&](int list, int& from) {
          for (; from < a.width; from += ways) {
            const Pair p = pair_of(list, from);
            if (!(p.key > -(double)kInf)) break;
            if (!better(last, p)) continue;
            if (better(p, mine)) mine = p;
            break;
          }
        };
        if (way < ways) {
#pragma unroll
          for (int u = 0; u < kHeld; u++)
            if (list0 + u * kBlock < lists) look(list0 + u * kBlock, next[u]);
          for (int list = list0 + kHeld * kBlock; list < lists; list += kBlock) {
            int from = way;
            look(list, from);
          }
        }
        mine = best_of_wave(mine);
        __syncthreads();
        if (lane == 0) s_list[wave] = mine;
        __syncthreads();
        last = s_list[0];
        for (int w = 1; w < kWaves; w++)
          if (better(s_list[w], last)) last = s_list[w];
        if (threadIdx.x == 0) write(n, last, last.key > -(double)kInf);
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- reorder --

constexpr int kChunk = 16;  // bytes
constexpr int kAtOnce = 4;

// Rows of every state (blockIdx.y) by parent, in chunks of 16 bytes, the last of a
// row moved back to its end. An absent parent's row is 0 and reads nothing of its
// own: the chunk of the entry's first beam is loaded and not used.
__global__ __launch_bounds__(kBlock) void k_beam_reorder(ReorderArgs a) {
  const w2v_beam_state st = a.states[blockIdx.y];
  const int64_t per_row = (st.row_bytes + kChunk - 1) / kChunk;
  const int64_t chunks = (int64_t)a.batch * a.width * per_row;
  const bool whole = st.row_bytes >= kChunk;
  constexpr int kStep = kBlock * kAtOnce;
  for (int64_t base = (int64_t)blockIdx.x * kStep; base < chunks;
       base += (int64_t)gridDim.x * kStep) {
    const int64_t row0 = base / per_row, rest = base - row0 * per_row;
    uint4 v[kAtOnce];
    char* to[kAtOnce];
    bool there[kAtOnce];
    const char* from[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; u++) {
      const int64_t i = rest + u * kBlock + threadIdx.x;
      const bool some = base - rest + i < chunks;
      const int64_t on = some ? divided((uint32_t)i, a.by_row[blockIdx.y]) : 0;
      const int64_t row = row0 + on, entry = row / a.width;
      const int64_t byte = some ? (i - on * per_row) * kChunk : 0;
      const int64_t at = whole && byte + kChunk > st.row_bytes ? st.row_bytes - kChunk : byte;
      const int32_t parent = a.parents[row];
      there[u] = parent >= 0 && parent < a.beams;
      if (!there[u] && parent != -1) report_row(a.status);
      from[u] =
          (const char*)st.src + (entry * a.beams + (there[u] ? parent : 0)) * st.src_stride + at;
      to[u] = some ? (char*)st.dst + row * st.dst_stride + at : nullptr;
    }
    if (whole) {
#pragma unroll
      for (int u = 0; u < kAtOnce; u++) v[u] = load_16(from[u]);
#pragma unroll
      for (int u = 0; u < kAtOnce; u++) {
        if (to[u] == nullptr) continue;
        if (!there[u]) v[u] = make_uint4(0, 0, 0, 0);
        __builtin_memcpy(to[u], &v[u], 16);
      }
    } else {
      for (int u = 0; u < kAtOnce; u++)
        if (to[u] != nullptr)
          for (int i = 0; i < (int)st.row_bytes; i++) to[u][i] = there[u] ? from[u][i] : 0;
    }
  }
}

// ------------------------------------------------------------------ launch --

// Packs a thread holds of a row, by an estimate of the time: a block takes 6 us and
// 0.6 for each pack, the card holds 1,024 blocks of 16 packs, 1,536 of 4 and 1,792 of
// 1 at once, and the merge 0.7 us for 256 lists of an entry. Measured with 16, 4, 1
// packs: 16 x 16 beams of 10^6 words fp16 109, 165, 464 us; 32 x 8 of 100,000 bf16 32,
// 33, 54; 64 x 32 of 2,000 fp32 44, 38, 49; 16 x 16 of 30,000 bf16 29, 29, 36.
int packs_of(int64_t batch, int64_t beams, int32_t V, int32_t dtype) {
  const int64_t e = dtype == W2V_DTYPE_F32 ? 4 : 8;
  const int packs[3] = {16, 4, 1};
  const double held[3] = {1024, 1536, 1792};
  int best = 0;
  double least = 0;
  for (int i = 0; i < 3; i++) {
    const int64_t of = kBlock * packs[i] * e, shares = (V + of - 1) / of;
    const double rounds = (double)(batch * beams * shares) / held[i];
    const double us = (rounds > 1 ? rounds : 1) * (6 + 0.6 * packs[i]) +
                      0.7 * (double)(beams * shares) / 256;
    if (i == 0 || us < least) {
      least = us;
      best = packs[i];
    }
  }
  return best;
}

int64_t share_count(int64_t batch, int64_t beams, int32_t V, int32_t dtype) {
  const int64_t of =
      (int64_t)kBlock * packs_of(batch, beams, V, dtype) * (dtype == W2V_DTYPE_F32 ? 4 : 8);
  return (V + of - 1) / of;
}

size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }

template <typename T, int PACKS>
void launch_shares(const BeamArgs& a, int shares, Share* share, Word* best, hipStream_t s) {
  const int64_t units = (int64_t)a.batch * a.beams * shares;
  const dim3 grid((unsigned)(units < kMaxGrid ? units : kMaxGrid));
  hipLaunchKernelGGL((k_beam_shares<T, PACKS>), grid, dim3(kBlock), 0, s, a, shares, share, best);
}

template <typename T>
void launch_shares(const BeamArgs& a, int shares, Share* share, Word* best, hipStream_t s) {
  switch (packs_of(a.batch, a.beams, a.V, a.dtype)) {
    case 16:
      return launch_shares<T, 16>(a, shares, share, best, s);
    case 4:
      return launch_shares<T, 4>(a, shares, share, best, s);
    default:
      return launch_shares<T, 1>(a, shares, share, best, s);
  }
}

}  // namespace

size_t beam_workspace_bytes(int32_t batch, int32_t beams, int32_t width, int32_t V,
                            int32_t dtype) {
  const int64_t rows = (int64_t)batch * beams;
  const size_t lists = (size_t)(rows * share_count(batch, beams, V, dtype));
  return aligned(lists * sizeof(Share)) + aligned(lists * (size_t)width * sizeof(Word));
}

hipError_t launch_beam_step(const BeamArgs& a, void* workspace, hipStream_t s) {
  const int64_t rows = (int64_t)a.batch * a.beams;
  const int shares = (int)share_count(a.batch, a.beams, a.V, a.dtype);
  Share* share = (Share*)workspace;
  Word* best = (Word*)((char*)workspace + aligned((size_t)rows * shares * sizeof(Share)));
  switch (a.dtype) {
    case W2V_DTYPE_F32:
      launch_shares<float>(a, shares, share, best, s);
      break;
    case W2V_DTYPE_BF16:
      launch_shares<bf16_t>(a, shares, share, best, s);
      break;
    default:
      launch_shares<f16_t>(a, shares, share, best, s);
  }
  hipLaunchKernelGGL(k_beam_merge, dim3((unsigned)(a.batch < kMaxGrid ? a.batch : kMaxGrid)),
                     dim3(kBlock), 0, s, a, shares, share, best);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(const ReorderArgs& args, hipStream_t s) {
  ReorderArgs a = args;
  int64_t most = 1;
  for (int i = 0; i < a.count; i++) {
    const int64_t per_row = (a.states[i].row_bytes + kChunk - 1) / kChunk;
    const int64_t chunks = (int64_t)a.batch * a.width * per_row;
    a.by_row[i] = divisor_of((uint32_t)per_row);
    const int64_t blocks = (chunks + kBlock * kAtOnce - 1) / (kBlock * kAtOnce);
    if (blocks > most) most = blocks;
  }
  const dim3 grid((unsigned)(most < (1 << 16) ? most : 1 << 16), (unsigned)a.count);
  hipLaunchKernelGGL(k_beam_reorder, grid, dim3(kBlock), 0, s, a);
  return hipGetLastError();
}

}  // namespace w2v
