// Distillation from a teacher's top logits. Per row, with s the student's V
// scores, (id_k, t_k) the teacher's list, T the temperature:
//   q = softmax(t / T) over the listed words, p_T = softmax(s / T),
//   p_1 = softmax(s),
//   loss = soft T^2 sum_k q_k (log q_k - log p_T(id_k)) - hard log p_1(label)
//   d loss / d s_j = soft T (Q p_T(j) - q_j) + hard (p_1(j) - [j = label])
// with Q = 1 where the row lists a word above -inf, else 0. A block that can
// hold a row in its registers reads it once (k_row); otherwise one pass over s
// keeps a running maximum and the two sums of exponentials relative to it, and a
// second one forms the gradient. All are bound by memory.
#include "distill.h"

#include "head_types.h"

namespace w2v {
namespace {

constexpr int kThreads = 512;

// How p_1 is formed beside p_T. Squaring for T = 1, 2, 4 and an exponential of its
// own, us: 4,096 rows of 71,290 bf16 269, 268, 277 and 296 (259 without labels), fp32
// 518, 529, 567 and 547; 65,536 of 1,000 bf16 90, 91, 93 and 96.
constexpr int kSoftOnly = -1;  // not at all: no row has a label
// 0, 1, 2: T is 1, 2 or 4, and exp(x) is exp(x / T) squared that often
constexpr int kBoth = 3;  // any T: an exponential of its own

struct Ctx {
  DistillArgs a;
  float scale;    // log2(e) / T
  int splits;     // of a row
  int64_t range;  // elements of a split
  float* parts;   // [rows][splits][3]
};

// Maximum of some of a row's scores and the sums of exp((s - max) / T) and
// exp(s - max) over them. An empty set has maximum -inf and sums 0.
struct Sums {
  float max, soft, hard;
};

// exp2((from - to) scale): what sums relative to `from` are multiplied with
// to be relative to `to` >= from.
__device__ __forceinline__ float rescale(float from, float to, float scale) {
  return from == to ? 1.0f : exp2_fast((from - to) * scale);
}

__device__ __forceinline__ Sums join(Sums a, Sums b, float scale) {
  Sums o;
  o.max = fmaxf(a.max, b.max);
  o.soft = a.soft * rescale(a.max, o.max, scale) + b.soft * rescale(b.max, o.max, scale);
  o.hard = a.hard * rescale(a.max, o.max, kLog2e) + b.hard * rescale(b.max, o.max, kLog2e);
  return o;
}

// exp(d) beside e = exp(d / T).
template <int MODE>
__device__ __forceinline__ float hard_of(float d, float e) {
  if constexpr (MODE == kBoth) return exp2_fast(d * kLog2e);
  for (int i = 0; i < MODE; i++) e *= e;
  return e;
}

// Adds N scores. The maximum is moved once for all of them.
template <int MODE, int N>
__device__ __forceinline__ void add(Sums& s, const float (&v)[N], float scale) {
  float m = v[0];
#pragma unroll
  for (int i = 1; i < N; i++) m = fmaxf(m, v[i]);
  if (m > s.max) {
    s.soft *= rescale(s.max, m, scale);
    if constexpr (MODE != kSoftOnly) s.hard *= rescale(s.max, m, kLog2e);
    s.max = m;
  }
  const float base = s.max == -INFINITY ? 0.0f : s.max;
  float soft = 0.0f, hard = 0.0f;
#pragma unroll
  for (int i = 0; i < N; i++) {
    const float d = v[i] - base;
    const float e = exp2_fast(d * scale);
    soft += e;
    if constexpr (MODE != kSoftOnly) hard += hard_of<MODE>(d, e);
  }
  s.soft += soft;
  s.hard += hard;
}

// The thread's share of the sums over [lo, hi) of a row.
template <typename T, int MODE, int THREADS>
__device__ __forceinline__ Sums scan(const T* row, int64_t lo, int64_t hi, const Ctx& c) {
  constexpr int N = 16 / (int)sizeof(T), U = 4;
  const int tid = threadIdx.x;
  Sums s = {-INFINITY, 0.0f, 0.0f};
  const int64_t packs = (hi - lo) / N;
  int64_t p = tid;
  for (; p + (U - 1) * THREADS < packs; p += U * THREADS) {
    uint4 in[U];
#pragma unroll
    for (int u = 0; u < U; u++) in[u] = load_16(row + lo + (p + u * THREADS) * N);
#pragma unroll
    for (int u = 0; u < U; u++) {
      float v[N];
      unpack_words<T>(in[u], v);
      add<MODE, N>(s, v, c.scale);
    }
  }
  for (; p < packs; p += THREADS) {
    float v[N];
    unpack_words<T>(load_16(row + lo + p * N), v);
    add<MODE, N>(s, v, c.scale);
  }
  if (lo + packs * N + tid < hi) {
    const float v[1] = {to_f32(row[lo + packs * N + tid])};
    add<MODE, 1>(s, v, c.scale);
  }
  return s;
}

// The block's sums from its threads', relative to the maximum m.
template <int MODE>
__device__ __forceinline__ Sums block_of(Sums s, float m, const Ctx& c, float* scratch) {
  s.soft *= rescale(s.max, m, c.scale);
  if constexpr (MODE == kSoftOnly) {
    s.soft = block_sum(s.soft, scratch);
  } else {
    s.hard *= rescale(s.max, m, kLog2e);
    block_sums(s.soft, s.hard, scratch);
  }
  s.max = m;
  return s;
}

// The teacher's list of a row in LDS, and its label as one more entry: the
// word (-1: absent), the teacher's logit (then what is taken from the entry's
// gradient) and the student's score.
struct List {
  int32_t* id;
  float* q;
  float* s;
  float* scratch;  // 32
};
__device__ __forceinline__ List list_of(const Ctx& c) {
  extern __shared__ float memory[];
  const int n = c.a.K + 1;
  return List{(int32_t*)(memory + 32), memory + 32 + n, memory + 32 + 2 * n, memory};
}

struct Row {
  bool some;       // has a soft term: lists a word whose logit is above -inf
  bool ok;         // every id is a word or -1
  int32_t label;   // or -1
  float weight;    // of the gradient
  float max, log;  // of the list's t / T: q_k = exp(t_k / T - max - log)
};

template <typename T>
__device__ __forceinline__ float teacher_at(const Ctx& c, int row, int k) {
  return to_f32(((const T*)c.a.teacher)[(int64_t)row * c.a.K + k]);
}
__device__ __forceinline__ float teacher_logit(const Ctx& c, int row, int k) {
  switch (c.a.teacher_dtype) {
    case W2V_DTYPE_F32:
      return teacher_at<float>(c, row, k);
    case W2V_DTYPE_BF16:
      return teacher_at<bf16_t>(c, row, k);
    default:
      return teacher_at<f16_t>(c, row, k);
  }
}

// Reads the row's list and its label with the student's scores of their words;
// q sums to 1 over the present entries. t - max comes first, so that any finite
// t / T is within range.
template <typename T>
__device__ __forceinline__ Row read_list(const Ctx& c, int row, const List& l) {
  const int tid = threadIdx.x, step = blockDim.x;
  const T* logits = (const T*)c.a.logits + row * c.a.ld;
  Row r;
  r.label = c.a.labels == nullptr ? -1 : c.a.labels[row];
  r.weight = c.a.row_weight == nullptr ? 1.0f : c.a.row_weight[row];
  float m = -INFINITY, fault = 0.0f;  // 1: NaN, which the row's loss shows; 2: an id
  for (int k = tid; k <= c.a.K; k += step) {
    const int32_t id = k == c.a.K ? r.label : c.a.ids[(int64_t)row * c.a.K + k];
    const bool word = id >= 0 && id < c.a.V;
    const float t = k == c.a.K || !word ? -INFINITY : teacher_logit(c, row, k);
    l.id[k] = id;
    l.q[k] = t;
    l.s[k] = word ? to_f32(logits[id]) : 0.0f;
    m = fmaxf(m, t);
    fault = fmaxf(fault, id < -1 || id >= c.a.V ? 2.0f : t != t ? 1.0f : 0.0f);
  }
  block_maxima(m, fault, l.scratch);
  if (fault == 1.0f) m = NAN;
  r.ok = fault < 2.0f;
  r.some = m != -INFINITY && c.a.soft != 0.0f;
  r.max = m;
  float sum = 0.0f;
  for (int k = tid; k < c.a.K; k += step)
    sum += r.some && l.id[k] >= 0 ? expf((l.q[k] - m) / c.a.temperature) : 0.0f;
  sum = block_sum(sum, l.scratch);
  r.log = r.some ? logf(sum) : 0.0f;
  return r;
}

// (t_k - max) / T - log: log q_k of a present entry.
__device__ __forceinline__ float log_q(const Ctx& c, const Row& r, float t) {
  return (t - r.max) / c.a.temperature - r.log;
}

template <typename T, int MODE>
__global__ __launch_bounds__(kThreads) void k_sums(Ctx c) {
  __shared__ float scratch[32];
  const int row = blockIdx.x / c.splits, split = blockIdx.x % c.splits;
  const int64_t lo = split * c.range;
  const int64_t hi = lo + c.range < c.a.V ? lo + c.range : c.a.V;
  Sums s = scan<T, MODE, kThreads>((const T*)c.a.logits + row * c.a.ld, lo, hi, c);
  s = block_of<MODE>(s, block_max(s.max, scratch), c, scratch);
  if (threadIdx.x == 0) {
    float* out = c.parts + ((int64_t)row * c.splits + split) * 3;
    out[0] = s.max;
    out[1] = s.soft;
    out[2] = s.hard;
  }
}

// log of a row's second sum, which is 0 where nothing was added to it. NaN, as a
// score of NaN or +inf makes it, stays.
__device__ __forceinline__ float log_hard_of(const Sums& s) {
  return s.hard == 0.0f ? 0.0f : logf(s.hard);
}

// A row's loss from its sums (every thread has them); thread 0 writes it.
__device__ __forceinline__ void write_loss(const Ctx& c, int row, const Row& r, const List& l,
                                           const Sums& s) {
  const float log_soft = logf(s.soft), log_hard = log_hard_of(s);
  const bool live = r.ok && log_soft != -INFINITY;  // some score is above -inf
  float v = 0.0f;
  if (live && r.some) {
    for (int k = threadIdx.x; k < c.a.K; k += blockDim.x) {
      if (l.id[k] < 0) continue;
      const float lq = log_q(c, r, l.q[k]), q = expf(lq);
      if (q == 0.0f) continue;
      v += q * (lq - ((l.s[k] - s.max) / c.a.temperature - log_soft));
    }
  }
  v = block_sum(v, l.scratch);
  if (threadIdx.x == 0) {
    float loss = c.a.soft * c.a.temperature * c.a.temperature * v;
    if (live && r.label >= 0 && c.a.hard != 0.0f)  // 0 times an infinite term is none
      loss += c.a.hard * (log_hard - (l.s[c.a.K] - s.max));
    if (log_soft != log_soft) loss = NAN;  // whatever terms the row has
    if (!live) loss = 0.0f;
    c.a.loss[row] = loss;
    c.a.stats[(int64_t)row * 3] = s.max;
    c.a.stats[(int64_t)row * 3 + 1] = log_soft;
    c.a.stats[(int64_t)row * 3 + 2] = log_hard;
    if (!r.ok) report_row(c.a.status);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_loss(Ctx c) {
  const List l = list_of(c);
  const int row = blockIdx.x;
  const Row r = read_list<T>(c, row, l);
  Sums s = {-INFINITY, 0.0f, 0.0f};
  for (int i = 0; i < c.splits; i++) {
    const float* in = c.parts + ((int64_t)row * c.splits + i) * 3;
    s = join(s, Sums{in[0], in[1], in[2]}, c.scale);
  }
  write_loss(c, row, r, l, s);
}

// What a row's gradient is made of: soft p_T + hard p_1 from the statistics,
// less the amounts of the listed words and the label.
struct Slope {
  float max, soft, hard;  // exp((s - max) / T) soft + exp(s - max) hard
  bool none;              // the row's gradient is 0
};

template <int MODE>
__device__ __forceinline__ float slope_at(const Slope& g, float s, const Ctx& c) {
  const float d = s - g.max, e = exp2_fast(d * c.scale);
  if constexpr (MODE == kSoftOnly) return g.soft * e;
  if constexpr (MODE == 0) return (g.soft + g.hard) * e;
  if constexpr (MODE == 1) return __builtin_fmaf(g.hard, e, g.soft) * e;
  return g.soft * e + g.hard * hard_of<MODE>(d, e);
}

// The gradient's N elements from the scores.
template <typename T, int MODE, int N>
__device__ __forceinline__ Pack<T, N> slopes(const Slope& g, const float (&v)[N],
                                             const Ctx& c) {
  Pack<T, N> o;
  if (g.none) {  // uniform over the block
#pragma unroll
    for (int j = 0; j < N; j++) o.v[j] = T(0.0f);
  } else {
#pragma unroll
    for (int j = 0; j < N; j++) o.v[j] = from_f32<T>(slope_at<MODE>(g, v[j], c));
  }
  return o;
}

// Turns the list into the entries of the gradient within [lo, hi): the amount
// to take off. The student's scores were read before the gradient may overwrite
// them.
__device__ __forceinline__ Slope begin_gradient(const Ctx& c, const Row& r, const List& l,
                                                float max, float log_soft, float log_hard,
                                                int64_t lo, int64_t hi) {
  const float soft = r.weight * c.a.soft * c.a.temperature, hard = r.weight * c.a.hard;
  const bool live = r.ok && log_soft != -INFINITY;
  for (int k = threadIdx.x; k <= c.a.K; k += blockDim.x) {
    // (where every present logit is -inf there is no q to form)
    const bool there = live && l.id[k] >= lo && l.id[k] < hi && (k == c.a.K || r.some);
    if (!there) l.id[k] = -1;
    l.q[k] = k == c.a.K ? hard : there ? soft * expf(log_q(c, r, l.q[k])) : 0.0f;
  }
  __syncthreads();
  Slope g = {max, 0.0f, 0.0f, true};
  if (live && (r.some || log_soft != log_soft)) {  // NaN reaches every row's gradient
    g.soft = soft * expf(-log_soft);
    g.none = false;
  }
  if (live && r.label >= 0) {
    g.hard = hard * expf(-log_hard);
    g.none = false;
  }
  return g;
}

// Replaces the entries' gradients. Entries of one word write the same value. Each
// entry goes through the list, which outweighs the row where that is short and
// the list long: 65,536 rows of 1,000 bf16 take 98 us with 16 entries, 134 with 64,
// 756 with 256, 7,880 with 1,000.
template <typename T, int MODE>
__device__ void end_gradient(const Ctx& c, int row, const List& l, const Slope& g) {
  T* grad = (T*)c.a.grad + row * c.a.ldg;
  for (int k = threadIdx.x; k <= c.a.K; k += blockDim.x) {
    const int32_t id = l.id[k];
    if (id < 0) continue;
    float off = 0.0f;
    for (int i = 0; i <= c.a.K; i++) off += l.id[i] == id ? l.q[i] : 0.0f;
    grad[id] = from_f32<T>(slope_at<MODE>(g, l.s[k], c) - off);
  }
}

template <typename T, int MODE>
__global__ __launch_bounds__(kThreads) void k_gradient(Ctx c) {
  const List l = list_of(c);
  constexpr int N = 16 / (int)sizeof(T);
  const int row = blockIdx.x / c.splits, split = blockIdx.x % c.splits, tid = threadIdx.x;
  const int64_t lo = split * c.range;
  const int64_t hi = lo + c.range < c.a.V ? lo + c.range : c.a.V;
  const Row r = read_list<T>(c, row, l);
  if (!r.ok && tid == 0) report_row(c.a.status);
  const float* stats = c.a.stats + (int64_t)row * 3;
  const Slope g = begin_gradient(c, r, l, stats[0], stats[1], stats[2], lo, hi);
  const T* in = (const T*)c.a.logits + row * c.a.ld;
  T* out = (T*)c.a.grad + row * c.a.ldg;
  const int64_t packs = (hi - lo) / N;
  for (int64_t p = tid; p < packs; p += kThreads) {
    const int64_t at = lo + p * N;
    float v[N];
    unpack_words<T>(load_16(in + at), v);
    store_pack<T, N>(out + at, slopes<T, MODE>(g, v, c));
  }
  const int64_t last = lo + packs * N + tid;
  if (last < hi) {
    const float v[1] = {to_f32(in[last])};
    out[last] = slopes<T, MODE>(g, v, c).v[0];
  }
  __syncthreads();
  end_gradient<T, MODE>(c, row, l, g);
}

// Keeps the compiler from carrying a pack's elements in unpacked form past this
// point, at twice the registers.
__device__ __forceinline__ void keep_packed(uint4& v) {
  asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w));
}

// Where a thread's pack of 16 bytes of a turn of the block is. The packs of the
// row's last turn that would pass its end are moved down to end there; so they
// hold elements of other packs again, which the sums leave out and the gradient
// writes twice, with the same values. That way no load and no store has a test
// of its own. (4,096 rows of 71,290 bf16 took 373 us with tests, 288 without.)
struct Place {
  int64_t from;
  uint32_t off;
};
template <int SPAN, int N>
__device__ __forceinline__ Place place_of(int64_t start, int64_t V) {
  Place p;
  const int64_t last = V - N;
  p.from = start < last ? start : last;
  const uint32_t room = last - p.from < SPAN ? (uint32_t)(last - p.from) : SPAN;
  uint32_t off = threadIdx.x * N;
  asm volatile("" : "+v"(off));  // made anew at each use: kept, all would need registers
  p.off = off < room ? off : room;
  return p;
}

// Elements at .. at + N - 1 of a row of fewer than N, -inf past its end.
template <typename T, int N>
__device__ __forceinline__ uint4 load_few(const T* row, int64_t at, int64_t V) {
  T v[N];
#pragma unroll
  for (int i = 0; i < N; i++) v[i] = at + i < V ? row[at + i] : T(-INFINITY);
  return __builtin_bit_cast(uint4, v);
}

// Loss and gradient of a row by one block. The end of the row stays in
// registers, NV packs of 16 bytes a thread, between the sums and the gradient;
// STREAM: of longer rows the first part is read twice, the second time
// backwards, from what was read last. Measured (us, bf16, K 64): 4,096 rows of
// 71,290 261 to 290, 4.0 to 4.5 TB/s, where a copy of them has 4.9; 65,536 of
// 1,000 87; 2,048 of 10^6 2,390, whose two readings and one writing pass at
// 4.9 TB/s of traffic.
// Between its sums and its gradient a block waits for its slowest wave; two
// blocks a CU (18 packs are 72 of 128 registers) fill each other's waits.
template <typename T, int MODE, int THREADS, int NV, bool STREAM>
__global__ __launch_bounds__(THREADS) void k_row(Ctx c) {
  const List l = list_of(c);
  constexpr int N = 16 / (int)sizeof(T);
  constexpr int kSpan = THREADS * N;  // of a turn of the block
  const int tid = threadIdx.x;
  const int64_t V = c.a.V;
  // what is read twice: whole turns of the block
  const int64_t over = V - (int64_t)NV * kSpan;
  const int64_t head = STREAM && over > 0 ? (over + kSpan - 1) / kSpan * kSpan : 0;
  uint4 kept[NV];
  const int64_t row = blockIdx.x;
  const T* in = (const T*)c.a.logits + row * c.a.ld;
  const bool few = NV <= 4 && V < N;
  if (!few) {
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const Place p = place_of<kSpan, N>(head + i * kSpan, V);
      kept[i] = load_16(in + p.from + p.off);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; i++) kept[i] = load_few<T, N>(in, (tid + i * THREADS) * N, V);
  }
  const Row r = read_list<T>(c, (int)row, l);
  Sums s = {-INFINITY, 0.0f, 0.0f};
  if (STREAM) s = scan<T, MODE, THREADS>(in, 0, head, c);
  float m = s.max;
#pragma unroll
  for (int i = 0; i < NV; i++) {
    float v[N];
    unpack_words<T>(kept[i], v);
#pragma unroll
    for (int j = 0; j < N; j++) m = fmaxf(m, v[j]);
    keep_packed(kept[i]);
    __builtin_amdgcn_sched_barrier(0);
  }
  m = block_max(m, l.scratch);
  s.soft *= rescale(s.max, m, c.scale);
  s.hard *= rescale(s.max, m, kLog2e);
  s.max = m;
  const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
  for (int i = 0; i < NV; i++) {
    const int64_t start = head + i * kSpan;
    if (start >= V) break;
    const bool whole = few || start + kSpan <= V;
    int skip = 0;  // elements that another pack has
    if (!whole) {
      const Place p = place_of<kSpan, N>(start, V);
      const int64_t n = start + tid * N - (p.from + p.off);
      skip = n < N ? (int)n : N;
    }
    float soft = 0.0f, hard = 0.0f, v[N];
    unpack_words<T>(kept[i], v);
#pragma unroll
    for (int j = 0; j < N; j++) {
      const float d = v[j] - base, e = exp2_fast(d * c.scale);
      const bool again = !whole && j < skip;
      soft += again ? 0.0f : e;
      if constexpr (MODE != kSoftOnly) hard += again ? 0.0f : hard_of<MODE>(d, e);
    }
    s.soft += soft;
    s.hard += hard;
    keep_packed(kept[i]);
    __builtin_amdgcn_sched_barrier(0);
  }
  s = block_of<MODE>(s, m, c, l.scratch);
  write_loss(c, (int)row, r, l, s);
  if (c.a.grad == nullptr) return;

  const float log_soft = logf(s.soft), log_hard = log_hard_of(s);
  const Slope g = begin_gradient(c, r, l, s.max, log_soft, log_hard, 0, V);
  T* out = (T*)c.a.grad + row * c.a.ldg;
#pragma unroll
  for (int i = 0; i < NV; i++) {
    const int64_t start = head + i * kSpan;
    if (start >= V) break;
    float v[N];
    unpack_words<T>(kept[i], v);
    const Pack<T, N> o = slopes<T, MODE>(g, v, c);
    if (!few) {
      const Place p = place_of<kSpan, N>(start, V);
      store_pack<T, N>(out + p.from + p.off, o);
    } else if (tid == 0) {
      store_some<T, N>(out, V, o);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  if (STREAM) {
    constexpr int U = 4;
    int64_t turn = head / kSpan;
    for (; turn >= U; turn -= U) {
      const T* from = in + (turn - U) * kSpan;
      T* to = out + (turn - U) * kSpan;
      uint4 w[U];
#pragma unroll
      for (int u = 0; u < U; u++) w[u] = load_16(from + u * kSpan + (uint32_t)(tid * N));
#pragma unroll
      for (int u = 0; u < U; u++) {
        float v[N];
        unpack_words<T>(w[u], v);
        store_pack<T, N>(to + u * kSpan + (uint32_t)(tid * N), slopes<T, MODE>(g, v, c));
      }
    }
    for (; turn > 0; turn--) {
      const int64_t at = (turn - 1) * kSpan + tid * N;
      float v[N];
      unpack_words<T>(load_16(in + at), v);
      store_pack<T, N>(out + at, slopes<T, MODE>(g, v, c));
    }
  }
  __syncthreads();
  end_gradient<T, MODE>(c, (int)row, l, g);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

constexpr int kCUs = 256;

// Blocks of a row: enough for the GPU to be full with few rows, each with at
// least 8192 elements.
int splits_of(int32_t rows, int32_t V) {
  const int64_t most = ceil_div(V, 8192);
  int64_t want = ceil_div(1024, rows > 0 ? rows : 1);
  if (want > most) want = most;
  return (int)(want < 1 ? 1 : want);
}

Ctx context(const DistillArgs& a) {
  Ctx c{};
  c.a = a;
  c.scale = kLog2e / a.temperature;
  c.splits = splits_of(a.rows, a.V);
  c.range = ceil_div(ceil_div(a.V, c.splits), 64) * 64;
  c.splits = (int)ceil_div(a.V, c.range);
  return c;
}

// A row goes to the smallest block whose registers hold it: of 65,536 rows of
// 1,000 bf16 one of 64 threads takes 87 us, of 256 253; 16,384 rows of 8,000 256
// threads 138, 512 291; 4,096 of 30,000 9 packs a thread 134, 18 165; 4,096 of
// 71,290 512 threads 261, 1,024 425. (K <= 128: a wave alone does not go through
// longer lists.) By shares (k_sums, k_loss, k_gradient) these take 399 (the
// last), and with few rows no less either: 8 rows of 71,290 24 beside 22, 16 of
// 1,000 28 beside 17.
// Longer rows, which a block reads twice in part, need enough rows to fill the
// GPU. By a block and by shares: 2,048 rows of 110,000 295 and 317, 64 30 and
// 29, one 28 and 25; 256 rows of 10^6 300 and 329, 128 194 and 166, 16 133 and 42.
template <typename T, int MODE>
hipError_t launch_as(const Ctx& c, bool forward, hipStream_t s) {
  constexpr int N = 16 / (int)sizeof(T);
  const int rows = c.a.rows, V = c.a.V;
  const size_t lds = 32 * 4 + (size_t)(c.a.K + 1) * 12;
  if (forward && V <= 64 * 4 * N && c.a.K <= 128) {
    k_row<T, MODE, 64, 4, false><<<rows, 64, lds, s>>>(c);
  } else if (forward && V <= 256 * 4 * N) {
    k_row<T, MODE, 256, 4, false><<<rows, 256, lds, s>>>(c);
  } else if (forward && V <= 512 * 9 * N) {
    k_row<T, MODE, 512, 9, false><<<rows, 512, lds, s>>>(c);
  } else if (forward && V <= 512 * 18 * N) {
    k_row<T, MODE, 512, 18, false><<<rows, 512, lds, s>>>(c);
  } else if (forward && rows >= kCUs) {
    k_row<T, MODE, 1024, 14, true><<<rows, 1024, lds, s>>>(c);
  } else {
    const int grid = rows * c.splits;
    if (forward) {
      k_sums<T, MODE><<<grid, kThreads, 0, s>>>(c);
      k_loss<T><<<rows, kThreads, lds, s>>>(c);
    }
    if (c.a.grad != nullptr) k_gradient<T, MODE><<<grid, kThreads, lds, s>>>(c);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const Ctx& c, bool forward, hipStream_t s) {
  if (c.a.labels == nullptr) return launch_as<T, kSoftOnly>(c, forward, s);
  const float t = c.a.temperature;
  if (t == 1.0f) return launch_as<T, 0>(c, forward, s);
  if (t == 2.0f) return launch_as<T, 1>(c, forward, s);
  if (t == 4.0f) return launch_as<T, 2>(c, forward, s);
  return launch_as<T, kBoth>(c, forward, s);
}

hipError_t launch_part(const Ctx& c, bool forward, hipStream_t s) {
  switch (c.a.dtype) {
    case W2V_DTYPE_F32:
      return launch_type<float>(c, forward, s);
    case W2V_DTYPE_BF16:
      return launch_type<bf16_t>(c, forward, s);
    default:
      return launch_type<f16_t>(c, forward, s);
  }
}

hipError_t launch(const DistillArgs& a, void* workspace, bool forward, hipStream_t s) {
  const int most = rows_of_launch(a.rows);
  hipError_t e = hipSuccess;
  for (int64_t row = 0; row < a.rows && e == hipSuccess; row += most) {
    DistillArgs part = a;
    part.rows = (int32_t)(a.rows - row < most ? a.rows - row : most);
    part.logits = row_at(a.logits, row, a.ld, a.dtype);
    part.ids = row_at(a.ids, row, a.K);
    part.teacher = row_at(a.teacher, row, a.K, a.teacher_dtype);
    part.labels = row_at(a.labels, row);
    part.row_weight = row_at(a.row_weight, row);
    part.loss = row_at(a.loss, row);
    part.stats = row_at(a.stats, row, 3);
    part.grad = const_cast<void*>(row_at(a.grad, row, a.ldg, a.dtype));
    Ctx c = context(part);
    c.parts = (float*)workspace;
    e = launch_part(c, forward, s);
  }
  return e;
}

}  // namespace

size_t distill_workspace_bytes(int32_t rows, int32_t V, int32_t dtype) {
  (void)dtype;
  return ((size_t)rows * splits_of(rows, V) * 12 + 255) / 256 * 256;
}

hipError_t launch_distill(const DistillArgs& a, void* workspace, hipStream_t s) {
  return launch(a, workspace, true, s);
}

hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t s) {
  return launch(a, nullptr, false, s);
}

}  // namespace w2v
