// Distillation from a teacher's top logits. Per row, with s the student's V
// scores, (id_k, t_k) the teacher's list, T the temperature:
//   q = softmax(t / T) over the listed words, p_T = softmax(s / T),
//   p_1 = softmax(s),
//   loss = soft T^2 sum_k q_k (log q_k - log p_T(id_k)) - hard log p_1(label)
//   d loss / d s_j = soft T (Q p_T(j) - q_j) + hard (p_1(j) - [j = label])
// with Q = 1 where the row lists a word, else 0. One pass over s keeps a
// running maximum and the two sums of exponentials relative to it; a second
// one forms the gradient. Both are bound by memory.
#include "distill.h"

#include "head_types.h"

namespace w2v {
namespace {

constexpr int kThreads = 512;
constexpr int kMaxList = W2V_MAX_TEACHER;

// How p_1 is formed beside p_T.
constexpr int kSoftOnly = 0;  // not at all: no row has a label
constexpr int kPower = 1;     // T = 2^n: exp(x) is exp(x / T) squared n times
constexpr int kBoth = 2;      // any T: an exponential of its own

struct Ctx {
  DistillArgs a;
  float scale;    // log2(e) / T
  int squarings;  // n of kPower
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

__device__ __forceinline__ float squared(float e, int squarings) {
  for (int i = 0; i < squarings; i++) e *= e;
  return e;
}

template <int MODE>
__device__ __forceinline__ float hard_of(float d, float e, int squarings) {
  if constexpr (MODE == kPower) return squared(e, squarings);
  if constexpr (MODE == kBoth) return exp2_fast(d * kLog2e);
  return 0.0f;
}

// Adds N scores. The maximum is moved once for all of them.
template <int MODE, int N>
__device__ __forceinline__ void add(Sums& s, const float (&v)[N], float scale,
                                    int squarings) {
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
    if constexpr (MODE != kSoftOnly) hard += hard_of<MODE>(d, e, squarings);
  }
  s.soft += soft;
  s.hard += hard;
}

// The sums over the block's share [lo, hi) of a row, in every thread.
template <typename T, int MODE>
__device__ Sums scan(const T* row, int64_t lo, int64_t hi, const Ctx& c, float* scratch) {
  constexpr int N = 16 / (int)sizeof(T);
  const int tid = threadIdx.x;
  Sums s = {-INFINITY, 0.0f, 0.0f};
  const int64_t packs = (hi - lo) / N;
  constexpr int U = 4;
  int64_t p = tid;
  for (; p + (U - 1) * kThreads < packs; p += U * kThreads) {
    Pack<T, N> in[U];
#pragma unroll
    for (int u = 0; u < U; u++) in[u] = load_pack<T, N>(row + lo + (p + u * kThreads) * N);
#pragma unroll
    for (int u = 0; u < U; u++) {
      float v[N];
#pragma unroll
      for (int i = 0; i < N; i++) v[i] = to_f32(in[u].v[i]);
      add<MODE, N>(s, v, c.scale, c.squarings);
    }
  }
  for (; p < packs; p += kThreads) {
    const Pack<T, N> in = load_pack<T, N>(row + lo + p * N);
    float v[N];
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = to_f32(in.v[i]);
    add<MODE, N>(s, v, c.scale, c.squarings);
  }
  if (lo + packs * N + tid < hi) {
    const float v[1] = {to_f32(row[lo + packs * N + tid])};
    add<MODE, 1>(s, v, c.scale, c.squarings);
  }
  const float m = block_max(s.max, scratch);
  s.soft *= rescale(s.max, m, c.scale);
  s.hard *= rescale(s.max, m, kLog2e);
  s.max = m;
  s.soft = block_sum(s.soft, scratch);
  if constexpr (MODE != kSoftOnly) s.hard = block_sum(s.hard, scratch);
  return s;
}

// The teacher's list of a row, in LDS: q of each entry (0 where absent).
struct List {
  int32_t id[kMaxList + 1];
  float q[kMaxList + 1];  // then what is taken from the entry's gradient
  float s[kMaxList + 1];  // the student's score
  float scratch[16];
  int bad;
};

struct Row {
  bool some;       // lists a word
  bool ok;         // every id is a word or -1
  int32_t label;   // or -1
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

// Reads the row's list and its label; q sums to 1 over the present entries.
// t - max comes first, so that any finite t / T is within range.
__device__ Row read_list(const Ctx& c, int row, List& l) {
  const int tid = threadIdx.x, step = blockDim.x;
  Row r;
  if (tid == 0) l.bad = 0;
  r.label = c.a.labels == nullptr ? -1 : c.a.labels[row];
  __syncthreads();
  float m = -INFINITY;
  bool bad = r.label < -1 || r.label >= c.a.V;
  for (int k = tid; k < c.a.K; k += step) {
    const int32_t id = c.a.ids[(int64_t)row * c.a.K + k];
    bad |= id < -1 || id >= c.a.V;
    const float t = id < 0 ? -INFINITY : teacher_logit(c, row, k);
    l.id[k] = id;
    l.q[k] = t;
    m = t > m || t != t ? t : m;  // NaN is kept: the row's loss shows it
  }
  if (bad) l.bad = 1;
  const float seen = block_sum(m != m ? 1.0f : 0.0f, l.scratch);
  m = block_max(m, l.scratch);
  if (seen > 0.0f) m = NAN;
  r.ok = l.bad == 0;
  r.some = m != -INFINITY;
  r.max = m;
  float sum = 0.0f;
  for (int k = tid; k < c.a.K; k += step) {
    const float e = r.some && l.id[k] >= 0 ? expf((l.q[k] - m) / c.a.temperature) : 0.0f;
    sum += e;
  }
  sum = block_sum(sum, l.scratch);
  r.log = r.some ? logf(sum) : 0.0f;
  __syncthreads();
  return r;
}

// (t_k - max) / T - log: log q_k of a present entry.
__device__ __forceinline__ float log_q(const Ctx& c, const Row& r, float t) {
  return (t - r.max) / c.a.temperature - r.log;
}

template <typename T, int MODE>
__global__ __launch_bounds__(kThreads) void k_sums(Ctx c) {
  __shared__ float scratch[16];
  const int row = blockIdx.x / c.splits, split = blockIdx.x % c.splits;
  const int64_t lo = split * c.range;
  const int64_t hi = lo + c.range < c.a.V ? lo + c.range : c.a.V;
  const Sums s = scan<T, MODE>((const T*)c.a.logits + row * c.a.ld, lo, hi, c, scratch);
  if (threadIdx.x == 0) {
    float* out = c.parts + ((int64_t)row * c.splits + split) * 3;
    out[0] = s.max;
    out[1] = s.soft;
    out[2] = s.hard;
  }
}

// A row's loss from its sums (every thread has them); thread 0 writes it.
template <typename T>
__device__ void write_loss(const Ctx& c, int row, const Row& r, const List& l, const Sums& s,
                           float* scratch) {
  const T* logits = (const T*)c.a.logits + row * c.a.ld;
  const float log_soft = logf(s.soft), log_hard = s.hard > 0.0f ? logf(s.hard) : 0.0f;
  const bool live = r.ok && log_soft != -INFINITY;  // some score is above -inf
  float v = 0.0f;
  if (live && r.some) {
    for (int k = threadIdx.x; k < c.a.K; k += blockDim.x) {
      if (l.id[k] < 0) continue;
      const float lq = log_q(c, r, l.q[k]), q = expf(lq);
      if (q == 0.0f) continue;
      const float x = (to_f32(logits[l.id[k]]) - s.max) / c.a.temperature;
      v += q * (lq - (x - log_soft));
    }
  }
  v = block_sum(v, scratch);
  if (threadIdx.x == 0) {
    float loss = c.a.soft * c.a.temperature * c.a.temperature * v;
    if (live && r.label >= 0)
      loss += c.a.hard * (log_hard - (to_f32(logits[r.label]) - s.max));
    if (!live) loss = 0.0f;
    c.a.loss[row] = loss;
    c.a.stats[(int64_t)row * 3] = s.max;
    c.a.stats[(int64_t)row * 3 + 1] = log_soft;
    c.a.stats[(int64_t)row * 3 + 2] = log_hard;
    if (!r.ok) __hip_atomic_store(c.a.status, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_loss(Ctx c) {
  __shared__ List l;
  const int row = blockIdx.x;
  const Row r = read_list(c, row, l);
  Sums s = {-INFINITY, 0.0f, 0.0f};
  for (int i = 0; i < c.splits; i++) {
    const float* in = c.parts + ((int64_t)row * c.splits + i) * 3;
    s = join(s, Sums{in[0], in[1], in[2]}, c.scale);
  }
  write_loss<T>(c, row, r, l, s, l.scratch);
}

// What a row's gradient is made of: soft p_T + hard p_1 from the statistics,
// less the amounts of the listed words and the label.
struct Slope {
  float max, soft, hard;  // exp2((s - max) scale) soft + exp2((s - max) log2e) hard
};

template <int MODE>
__device__ __forceinline__ float slope_at(const Slope& g, float s, const Ctx& c) {
  const float d = s - g.max, e = exp2_fast(d * c.scale);
  float v = g.soft * e;
  if constexpr (MODE != kSoftOnly) v += g.hard * hard_of<MODE>(d, e, c.squarings);
  return v;
}

// Turns the list into the entries of the gradient within [lo, hi): the
// student's score (read before the gradient may overwrite it) and the amount
// to take off; the label is one more entry.
template <typename T>
__device__ Slope begin_gradient(const Ctx& c, int row, const Row& r, List& l, float max,
                                float log_soft, float log_hard, int64_t lo, int64_t hi) {
  const T* logits = (const T*)c.a.logits + row * c.a.ld;
  const float w = c.a.row_weight == nullptr ? 1.0f : c.a.row_weight[row];
  const float soft = w * c.a.soft * c.a.temperature, hard = w * c.a.hard;
  const bool live = r.ok && log_soft != -INFINITY;
  for (int k = threadIdx.x; k <= c.a.K; k += blockDim.x) {
    if (k == c.a.K) {
      l.id[k] = r.label;
      l.q[k] = hard;
    } else {
      l.q[k] = l.id[k] < 0 ? 0.0f : soft * expf(log_q(c, r, l.q[k]));
    }
    if (!live || l.id[k] < lo || l.id[k] >= hi) l.id[k] = -1;
    if (l.id[k] >= 0) l.s[k] = to_f32(logits[l.id[k]]);
  }
  __syncthreads();
  Slope g = {max, 0.0f, 0.0f};
  if (live && r.some) g.soft = soft * expf(-log_soft);
  if (live && r.label >= 0) g.hard = hard * expf(-log_hard);
  if (!live) g.max = 0.0f;
  return g;
}

// Replaces the entries' gradients. Entries of one word write the same value.
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
  __shared__ List l;
  constexpr int N = 16 / (int)sizeof(T);
  const int row = blockIdx.x / c.splits, split = blockIdx.x % c.splits, tid = threadIdx.x;
  const int64_t lo = split * c.range;
  const int64_t hi = lo + c.range < c.a.V ? lo + c.range : c.a.V;
  const Row r = read_list(c, row, l);
  if (!r.ok && tid == 0)
    __hip_atomic_store(c.a.status, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
  const float* stats = c.a.stats + (int64_t)row * 3;
  const Slope g = begin_gradient<T>(c, row, r, l, stats[0], stats[1], stats[2], lo, hi);
  const bool none = g.soft == 0.0f && g.hard == 0.0f;
  const T* in = (const T*)c.a.logits + row * c.a.ld;
  T* out = (T*)c.a.grad + row * c.a.ldg;
  const int64_t packs = (hi - lo) / N;
  for (int64_t p = tid; p < packs; p += kThreads) {
    const int64_t at = lo + p * N;
    const Pack<T, N> v = load_pack<T, N>(in + at);
    Pack<T, N> o;
#pragma unroll
    for (int i = 0; i < N; i++)
      o.v[i] = from_f32<T>(none ? 0.0f : slope_at<MODE>(g, to_f32(v.v[i]), c));
    store_pack<T, N>(out + at, o);
  }
  const int64_t last = lo + packs * N + tid;
  if (last < hi) out[last] = from_f32<T>(none ? 0.0f : slope_at<MODE>(g, to_f32(in[last]), c));
  __syncthreads();
  end_gradient<T, MODE>(c, row, l, g);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

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
  c.squarings = a.temperature == 1.0f ? 0 : a.temperature == 2.0f ? 1 : 2;
  c.splits = splits_of(a.rows, a.V);
  c.range = ceil_div(ceil_div(a.V, c.splits), 64) * 64;
  c.splits = (int)ceil_div(a.V, c.range);
  return c;
}

template <typename T, int MODE>
hipError_t launch_as(const Ctx& c, bool forward, hipStream_t s) {
  const int grid = c.a.rows * c.splits;
  if (forward) {
    k_sums<T, MODE><<<grid, kThreads, 0, s>>>(c);
    k_loss<T><<<c.a.rows, kThreads, 0, s>>>(c);
  }
  if (c.a.grad != nullptr) k_gradient<T, MODE><<<grid, kThreads, 0, s>>>(c);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const Ctx& c, bool forward, hipStream_t s) {
  if (c.a.labels == nullptr) return launch_as<T, kSoftOnly>(c, forward, s);
  const float t = c.a.temperature;
  if (t == 1.0f || t == 2.0f || t == 4.0f) return launch_as<T, kPower>(c, forward, s);
  return launch_as<T, kBoth>(c, forward, s);
}

hipError_t launch(const Ctx& c, bool forward, hipStream_t s) {
  switch (c.a.dtype) {
    case W2V_DTYPE_F32:
      return launch_type<float>(c, forward, s);
    case W2V_DTYPE_BF16:
      return launch_type<bf16_t>(c, forward, s);
    default:
      return launch_type<f16_t>(c, forward, s);
  }
}

}  // namespace

size_t distill_workspace_bytes(int32_t rows, int32_t V, int32_t dtype) {
  (void)dtype;
  return ((size_t)rows * splits_of(rows, V) * 12 + 255) / 256 * 256;
}

hipError_t launch_distill(const DistillArgs& a, void* workspace, hipStream_t s) {
  Ctx c = context(a);
  c.parts = (float*)workspace;
  return launch(c, true, s);
}

hipError_t launch_distill_backward(const DistillArgs& a, hipStream_t s) {
  return launch(context(a), false, s);
}

}  // namespace w2v
