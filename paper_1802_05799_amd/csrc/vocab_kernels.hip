// Rows of logits over a vocabulary: log probabilities of given tokens with entropy and top
// alternatives, distillation from a teacher's alternatives, and the gradients of both.
//
// For a row z with scale s (one over the temperature): d_v = s (z_v - m) with m the row's
// largest logit, S = sum e^{d_v}, L = log S, so that log p_v = d_v - L, and the entropy is
// L - (sum e^{d_v} d_v) / S.  One pass gives all of it: m, S and the weighted sum are carried
// along, rescaled where the maximum grows.  Exponents are to base 2 (d times log2 e) for the
// hardware's exponential; z - m is formed before it is scaled, so logits near a type's lowest
// value (masks) do not overflow.  Everything is held in binary32.  Bound: memory, one read of
// the logits, and a gradient's one write.
#include "rows.hpp"

namespace hvdx {
namespace {

// Rows are split over blocks where there are too few of them to fill the chip: into parts of at least
// kPartLeast elements, until there are kBlocksWanted blocks.
constexpr int64_t kBlocksWanted = 1024, kPartLeast = 4096;
constexpr int kPartsMost = 64;  // one lane each when they are joined

constexpr float kNone = -3.402823466e38f;  // the maximum of nothing: finite, so that -inf minus it is no NaN
constexpr float kFar = -1000.f;            // 2^kFar is 0; a clamp for what 0 is multiplied by

// A row's elements in 16-byte vectors on 16-byte boundaries, and the few before and after them.
template <typename T>
struct Cut {
  static constexpr int n = RowTypes<T>::n;
  int head, nvec, edges;
  __device__ Cut(const T* row, int vocab) {
    head = (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) / sizeof(T)) % n;
    if (head > vocab) head = vocab;
    nvec = (vocab - head) / n;
    edges = vocab - nvec * n;
  }
  __device__ int start(int vec) const { return head + vec * n; }
  __device__ int edge(int i) const { return i < head ? i : nvec * n + i; }  // 0 <= i < edges
};

// max, sum of 2^(d - max) and the sum of those times their exponent, for a part of a row
struct Online {
  float m = kNone, s = 0.f, a = 0.f;
  __device__ void rise(float to, float c) {  // to >= m
    const float d = fmaxf((m - to) * c, kFar), r = exp2_hw(d);
    a = r * (a + d * s);
    s *= r;
    m = to;
  }
  __device__ void add(float z, float c) {
    const float d = (z - m) * c, e = exp2_hw(d);
    s += e;
    a += e * fmaxf(d, kFar);
  }
  __device__ void join(Online o, float c) {
    const float hi = fmaxf(m, o.m);
    rise(hi, c);
    o.rise(hi, c);
    s += o.s;
    a += o.a;
  }
};

template <int W>
__device__ Online block_join(Online o, float c, float (*lds)[3]) {  // the same in every thread
#pragma unroll
  for (int k = 1; k < 64; k *= 2) {
    Online other;
    other.m = __shfl_xor(o.m, k);
    other.s = __shfl_xor(o.s, k);
    other.a = __shfl_xor(o.a, k);
    o.join(other, c);
  }
  if constexpr (W > 1) {
    if (threadIdx.x % 64 == 0) {
      float* mine = lds[threadIdx.x / 64];
      mine[0] = o.m, mine[1] = o.s, mine[2] = o.a;
    }
    __syncthreads();
    o = Online{lds[0][0], lds[0][1], lds[0][2]};
    for (int w = 1; w < W; ++w) o.join(Online{lds[w][0], lds[w][1], lds[w][2]}, c);
  }
  return o;
}

// An order of (value, position): larger values first, then lower positions; -0 as +0.
__device__ __forceinline__ uint64_t key_of(float z, int position) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return (uint64_t)(b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) << 32 | (uint32_t)~position;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t b = (uint32_t)(k >> 32);
  return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ __forceinline__ int key_position(uint64_t k) { return (int)~(uint32_t)k; }

constexpr int kWaves = 4;

// The `k` first of a block's keys.  Each thread has the first of its own as `best`, at a coarser grain
// (the position of its vector); the block's 64 groups of W threads have one first key each, and the
// k-th of those is a bound that at least k keys reach: what lies below it cannot be among the k
// first.  Little reaches it (k = 32 of 131,072 normal values: about 45), so the threads with any
// collect those into LDS, where each finds its rank by counting.  Where more reach it than LDS
// holds, k rounds over all keys find them one by one.
constexpr int kCandidates = 1024;
template <int W>
struct TopLds {
  uint64_t group[64], candidate[kCandidates], best[W], bound;
  int count;
};
template <int W, typename Collect, typename Below, typename Emit>
__device__ void select_top(int k, uint64_t best, TopLds<W>& lds, Collect collect, Below below, Emit emit) {
  constexpr int NT = 64 * W;
  const int tid = threadIdx.x;
  uint64_t first = best;
#pragma unroll
  for (int j = 1; j < W; j *= 2) {
    const uint64_t other = __shfl_xor((unsigned long long)first, j);
    if (other > first) first = other;
  }
  if (tid % W == 0) lds.group[tid / W] = first;
  if (tid == 0) lds.count = 0;
  __syncthreads();
  if (tid < 64) {
    const uint64_t mine = lds.group[tid];
    int rank = 0;
#pragma unroll 16
    for (int j = 0; j < 64; ++j) {
      const uint64_t other = lds.group[j];
      rank += other > mine || (other == mine && j < tid);
    }
    if (rank == k - 1) lds.bound = mine;
  }
  __syncthreads();
  const uint64_t bound = lds.bound;
  if (best && best >= bound)
    collect(bound, [&](uint64_t key) {
      const int at = atomicAdd(&lds.count, 1);
      if (at < kCandidates) lds.candidate[at] = key;
    });
  __syncthreads();
  const int count = lds.count;
  if (count <= kCandidates) {
    for (int i = tid; i < count; i += NT) {
      const uint64_t mine = lds.candidate[i];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < count; ++j) rank += lds.candidate[j] > mine;
      if (rank < k) emit(rank, mine);
    }
    for (int i = count + tid; i < k; i += NT) emit(i, 0);  // there are no more
    return;
  }
  uint64_t last = ~0ull;
  for (int r = 0; r < k; ++r) {
    uint64_t next = below(last);
#pragma unroll
    for (int j = 1; j < 64; j *= 2) {
      const uint64_t other = __shfl_xor((unsigned long long)next, j);
      if (other > next) next = other;
    }
    __syncthreads();
    if (tid % 64 == 0) lds.best[tid / 64] = next;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w)
      if (lds.best[w] > next) next = lds.best[w];
    if (tid == 0) emit(r, next);
    last = next;
  }
}

// What a row's sums give, and one of its alternatives.
__device__ __forceinline__ void finish_logprobs(const LogprobArgs& g, int64_t row, float z_token, int64_t token, Online o) {
  const bool none = o.s == 0.f;
  const float lse = logf(o.s), entropy = none ? 0.f : lse - kLn2 * o.a / o.s;
  if (g.logprob) {
    float lp = 0.f;
    if (token >= g.vocab) lp = __builtin_nanf("");
    else if (token >= 0) lp = none ? -__builtin_inff() : (z_token - o.m) * g.scale - lse;
    g.logprob[row] = lp;
  }
  if (g.entropy) g.entropy[row] = entropy;
  if (g.stats) g.stats[row] = make_float4(o.m, lse, entropy, 0.f);
}
__device__ __forceinline__ void emit_top(const LogprobArgs& g, int64_t row, int rank, uint64_t key, Online o) {
  const bool broken = !(o.s == o.s);
  g.top_ids[row * g.top + rank] = broken ? -1 : key_position(key);
  g.top_logprobs[row * g.top + rank] = broken ? __builtin_nanf("")
                                       : o.s == 0.f ? -__builtin_inff()
                                                    : (key_value(key) - o.m) * g.scale - logf(o.s);
}

// A block has one of a row's `parts`: all of it, and the results, or a stretch of its vectors, whose sums and
// first keys go to the workspace for logprobs_join_kernel.  kBatch vectors are loaded at once, and
// the sums rescaled once for each batch.
constexpr int kBatch = 4;
template <typename T, int W>
__global__ __launch_bounds__(64 * W) void logprobs_kernel(LogprobArgs g) {
  constexpr int NT = 64 * W, N = RowTypes<T>::n;
  __shared__ float parts[W][3];
  __shared__ TopLds<W> top;
  const int64_t block = block_row();
  if (block >= g.rows * g.parts) return;
  const int64_t row = g.parts == 1 ? block : block / g.parts;
  const int part = g.parts == 1 ? 0 : (int)(block % g.parts);
  const T* z = static_cast<const T*>(g.logits) + row * g.stride;
  const float c = g.scale * kLog2e;
  const Cut<T> cut(z, g.vocab);
  const int v0 = (int)((int64_t)cut.nvec * part / g.parts), v1 = (int)((int64_t)cut.nvec * (part + 1) / g.parts);
  const int edges = part == 0 ? cut.edges : 0;
  const int64_t token = g.logprob ? g.tokens[row] : -1;
  const float z_token = token >= 0 && token < g.vocab ? (float)z[token] : 0.f;
  Online o;
  float high = -__builtin_inff();  // the thread's largest, and where its vector (or edge element) starts
  int high_at = v0 + (int)threadIdx.x < v1 ? cut.start(v0 + threadIdx.x) : (int)threadIdx.x < edges ? cut.edge(threadIdx.x) : -1;
  for (int i = v0 + threadIdx.x; i < v1; i += kBatch * NT) {
    Packed<T> p[kBatch];
    bool there[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      there[u] = i + u * NT < v1;
      if (there[u]) p[u] = load_packed(z + cut.start(i + u * NT));
    }
    Wide<T> x[kBatch];
    float hi = kNone;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      x[u] = there[u] ? widen<T>(p[u]) : Wide<T>(-__builtin_inff());
      float h = x[u][0];
#pragma unroll
      for (int k = 1; k < N; ++k) h = fmaxf(h, x[u][k]);
      if (h > high) {
        high = h;
        high_at = cut.start(i + u * NT);
      }
      hi = fmaxf(hi, h);
    }
    if (hi > o.m) o.rise(hi, c);
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
#pragma unroll
      for (int k = 0; k < N; ++k) o.add(x[u][k], c);
  }
  if ((int)threadIdx.x < edges) {
    const float x = (float)z[cut.edge(threadIdx.x)];
    if (high_at < 0 || key_of(x, cut.edge(threadIdx.x)) > key_of(high, high_at)) {  // it may stand before the vectors
      high = x;
      high_at = cut.edge(threadIdx.x);
    }
    if (x > o.m) o.rise(x, c);
    o.add(x, c);
  }
  o = block_join<W>(o, c, parts);
  const bool whole = g.parts == 1;
  if (threadIdx.x == 0) {
    if (whole) finish_logprobs(g, row, z_token, token, o);
    else g.part_sums[block] = make_float4(o.m, o.s, o.a, 0.f);
  }
  if (!g.top) return;
  select_top<W>(
      g.top, high_at < 0 ? 0 : key_of(high, high_at), top,
      [&](uint64_t bound, auto push) {
        for (int i = v0 + threadIdx.x; i < v1; i += kBatch * NT) {
          Packed<T> p[kBatch];
#pragma unroll
          for (int u = 0; u < kBatch; ++u)
            if (i + u * NT < v1) p[u] = load_packed(z + cut.start(i + u * NT));
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            if (i + u * NT >= v1) break;
            const int start = cut.start(i + u * NT);
            const Wide<T> x = widen<T>(p[u]);
            float h = x[0];
#pragma unroll
            for (int k = 1; k < N; ++k) h = fmaxf(h, x[k]);
            if (key_of(h, start) < bound) continue;
#pragma unroll
            for (int k = 0; k < N; ++k)
              if (key_of(x[k], start) >= bound) push(key_of(x[k], start + k));
          }
        }
        if ((int)threadIdx.x < edges) {
          const uint64_t key = key_of((float)z[cut.edge(threadIdx.x)], cut.edge(threadIdx.x));
          if (key >= bound) push(key);
        }
      },
      [&](uint64_t last) {
        uint64_t next = 0;
        auto take = [&](float x, int at) {
          const uint64_t key = key_of(x, at);
          if (key < last && key > next) next = key;
        };
        for (int i = v0 + threadIdx.x; i < v1; i += NT) {
          const Wide<T> x = widen<T>(load_packed(z + cut.start(i)));
#pragma unroll
          for (int k = 0; k < N; ++k) take(x[k], cut.start(i) + k);
        }
        if ((int)threadIdx.x < edges) take((float)z[cut.edge(threadIdx.x)], cut.edge(threadIdx.x));
        return next;
      },
      [&](int rank, uint64_t key) {
        if (whole) emit_top(g, row, rank, key, o);
        else g.part_keys[block * g.top + rank] = key;
      });
}

// A row's results from its parts'.
template <typename T>
__global__ __launch_bounds__(64 * kWaves) void logprobs_join_kernel(LogprobArgs g) {
  constexpr int NT = 64 * kWaves;
  __shared__ float parts[kWaves][3];
  __shared__ TopLds<kWaves> top;
  const int64_t row = block_row();
  if (row >= g.rows) return;
  const T* z = static_cast<const T*>(g.logits) + row * g.stride;
  const float c = g.scale * kLog2e;
  const int64_t token = g.logprob ? g.tokens[row] : -1;
  const float z_token = token >= 0 && token < g.vocab ? (float)z[token] : 0.f;
  const uint64_t* keys = g.part_keys + row * g.parts * g.top;
  const int nkeys = g.parts * g.top;
  Online o;
  if ((int)threadIdx.x < g.parts) {
    const float4 s = g.part_sums[row * g.parts + threadIdx.x];
    o = Online{s.x, s.y, s.z};
  }
  uint64_t best = 0;
  for (int i = threadIdx.x; i < nkeys; i += NT)
    if (keys[i] > best) best = keys[i];
  o = block_join<kWaves>(o, c, parts);
  if (threadIdx.x == 0) finish_logprobs(g, row, z_token, token, o);
  if (!g.top) return;
  select_top<kWaves>(
      g.top, best, top,
      [&](uint64_t bound, auto push) {
        for (int i = threadIdx.x; i < nkeys; i += NT)
          if (keys[i] && keys[i] >= bound) push(keys[i]);
      },
      [&](uint64_t last) {
        uint64_t next = 0;
        for (int i = threadIdx.x; i < nkeys; i += NT)
          if (keys[i] < last && keys[i] > next) next = keys[i];
        return next;
      },
      [&](int rank, uint64_t key) { emit_top(g, row, rank, key, o); });
}

// dz_v = s [ a (delta - p_v) - b p_v (log p_v + H) ] = p_v (C0 + C1 d_v) + s a delta, d_v in base 2.
template <typename T>
__global__ __launch_bounds__(64 * kWaves) void logprobs_grad_kernel(LogprobGradArgs g) {
  constexpr int NT = 64 * kWaves, N = RowTypes<T>::n;
  const int64_t row = block_row();
  if (row >= g.rows) return;
  const T* z = static_cast<const T*>(g.logits) + row * g.stride;
  T* out = static_cast<T*>(g.grad) + row * g.grad_stride;
  const float c = g.scale * kLog2e;
  const Cut<T> cut(z, g.vocab);
  const float4 st = g.stats[row];
  const float m = st.x, lse = st.y, entropy = st.z;
  const int64_t t = g.tokens ? g.tokens[row] : -1;
  float a = g.grad_logprob && t >= 0 ? g.grad_logprob[row] : 0.f;
  if (g.grad_logprob && t >= g.vocab) a = __builtin_nanf("");
  const float b = g.grad_entropy ? g.grad_entropy[row] : 0.f;
  const bool none = lse == -__builtin_inff();
  const float inv = none ? 0.f : expf(-lse);
  if (none) a = 0.f;
  const float c1 = -g.scale * b * kLn2, c0 = -g.scale * (a + b * (none ? 0.f : entropy - lse));
  const float peak = g.scale * a;
  auto one = [&](float x, int at) {
    const float d = (x - m) * c;
    float v = exp2_hw(d) * inv * (c0 + c1 * fmaxf(d, kFar));
    return at == t ? v + peak : v;
  };
  for (int i = threadIdx.x; i < cut.nvec; i += NT) {
    Wide<T> x = widen<T>(load_packed(z + cut.start(i)));
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = one(x[k], cut.start(i) + k);
    store_packed(out + cut.start(i), narrow<T>(x));
  }
  if ((int)threadIdx.x < cut.edges) {
    const int at = cut.edge(threadIdx.x);
    out[at] = (T)one((float)z[at], at);
  }
}

// What the teacher's alternatives ask of a row, in lane j of one wavefront for entry j.
struct Entry {
  int64_t id;     // -1 where absent
  float z, q;     // the student's logit there, the teacher's probability
  float log_q;
  bool first;     // of the entries with this token
  float q_token;  // the probability of all of them
};

constexpr int kBitmapMost = 32768;  // bytes: one for each vector of a row, by its number modulo their count

// Distillation.  `rest`: what is left of the teacher's mass, q_R, stands against the unlisted tokens'
// p_R, whose sum is taken over them alone (subtracting the listed ones' from the whole would lose
// it where they hold nearly everything): the pass leaves the listed tokens out, which a bitmap in LDS
// marks, and the wavefront that holds the entries adds theirs afterwards.  An unlisted token's
// gradient is then s g 2^(d) F with d from the unlisted maximum m_R and
// F = Q 2^(m_R - m) / S - q_R / S_R; a listed one's is s g (Q p - q), written over it.
template <typename T, bool REST>
struct DistillRow {
  static constexpr int N = RowTypes<T>::n;
  const T* z;
  Cut<T> cut;
  int vocab, entries;
  uint32_t mask;
  bool exact;
  const uint8_t* bitmap;
  const int* listed;  // LDS [64], -1 for absent entries

  __device__ uint32_t marks(int vec) const {
    uint32_t b = bitmap[vec & mask];
    if (b && !exact) {
      b = 0;
      for (int j = 0; j < entries; ++j) {
        const int d = listed[j] - cut.start(vec);
        if (listed[j] >= 0 && d >= 0 && d < N) b |= 1u << d;
      }
    }
    return b;
  }
  __device__ bool is_listed(int at) const {
    for (int j = 0; j < entries; ++j)
      if (listed[j] == at) return true;
    return false;
  }
};

template <typename T, bool REST>
__device__ __forceinline__ Entry entry_of(const DistillArgs& g, const T* z, int64_t row, int lane, bool& bad) {
  Entry e{-1, 0.f, 0.f, 0.f, true, 0.f};
  float t = -__builtin_inff();
  if (lane < g.entries) {
    e.id = g.ids[row * g.entries + lane];
    if (e.id >= g.vocab) bad = true;
    if (e.id < 0 || e.id >= g.vocab) e.id = -1;
    if (e.id >= 0) {
      t = g.teacher[row * g.entries + lane];
      e.z = (float)z[e.id];
    }
  }
  bad = __any(bad);
  if constexpr (!REST) {
    const float high = wave_max(t);
    const float x = high == -__builtin_inff() ? t : t - high;
    const float sum = wave_sum(e.id >= 0 ? expf(x) : 0.f);
    t = sum == 0.f ? t : x - logf(sum);
  }
  e.q = e.id >= 0 ? expf(t) : 0.f;
  e.log_q = t;
  e.q_token = 0.f;
  for (int j = 0; j < g.entries; ++j) {
    const int id = __shfl((int)e.id, j);
    const float q = __shfl(e.q, j);
    if (id == (int)e.id) {
      e.q_token += q;
      if (j < lane) e.first = false;
    }
  }
  return e;
}

// The row's loss and what its gradient takes, from the pass over the unlisted (REST) or all tokens.
struct DistillResult {
  float loss, f, m, lse, total;
};
template <bool REST>
__device__ __forceinline__ DistillResult distill_finish(const Entry& e, Online o, float scale, bool bad) {
  const float c = scale * kLog2e, inf = __builtin_inff();
  const bool there = e.id >= 0;
  float m = o.m, s = o.s, down = 1.f;
  if constexpr (REST) {
    m = fmaxf(m, wave_max(there ? e.z : kNone));
    down = exp2_hw(fmaxf((o.m - m) * c, kFar));
    s = o.s * down + wave_sum(there && e.first ? exp2_hw((e.z - m) * c) : 0.f);
  }
  const float lse = logf(s);
  // q (log q - log p), the scale taken with q: what is left of a mask of the lowest value stays finite
  const float each = s == 0.f ? inf : e.q * (e.log_q + lse) - (e.q * scale) * (e.z - m);
  const float part = wave_sum(there && !(e.q == 0.f) ? each : 0.f);
  const float listed = wave_sum(e.q);
  DistillResult r{part, 0.f, m, lse, listed};
  float over = 0.f;
  if constexpr (REST) {
    const float left = fmaxf(1.f - listed, 0.f);
    r.total += left;
    if (left > 0.f) {
      if (!(o.s == 0.f)) {
        r.loss += left * (logf(left) - ((o.m - m) * scale + logf(o.s) - lse));
        over = left / o.s;
      } else if (left > 1e-6f) {  // less is the rounding of a sum that is 1: nothing is left on either side
        r.loss += inf;
      }
    }
  }
  r.f = s == 0.f ? 0.f : r.total * down / s - over;
  if (bad) r.loss = r.f = r.lse = __builtin_nanf("");
  return r;
}

template <typename T>
__device__ __forceinline__ void patch_listed(const DistillArgs& g, T* out, const Entry& e, float scaled, float total,
                                             float m, float lse) {
  if (e.id < 0 || !e.first) return;
  const float p = expf((e.z - m) * g.scale - lse);
  out[e.id] = (T)(lse == -__builtin_inff() ? 0.f : scaled * (total * p - e.q_token));
}

// Loss, and with `grad` the gradient too, one block a row: the logits are read once for the sums and
// once more (from a cache) for the gradient.
template <typename T, bool REST>
__global__ __launch_bounds__(64 * kWaves) void distill_kernel(DistillArgs g, uint32_t bitmap_mask) {
  constexpr int NT = 64 * kWaves, N = RowTypes<T>::n;
  extern __shared__ uint32_t bitmap[];
  __shared__ float parts[kWaves][3];
  __shared__ int listed[64];
  __shared__ float result[5];
  const int64_t row = block_row();
  if (row >= g.rows) return;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const T* z = static_cast<const T*>(g.logits) + row * g.stride;
  const float c = g.scale * kLog2e;
  const Cut<T> cut(z, g.vocab);
  const DistillRow<T, REST> r{z, cut, g.vocab, g.entries, bitmap_mask, (uint32_t)cut.nvec <= bitmap_mask + 1,
                              reinterpret_cast<const uint8_t*>(bitmap), listed};
  bool bad = false;
  Entry e{};
  if (wave == 0) e = entry_of<T, REST>(g, z, row, lane, bad);
  if constexpr (REST) {
    for (uint32_t i = threadIdx.x; i <= bitmap_mask / 4; i += NT) bitmap[i] = 0;
    __syncthreads();
    if (wave == 0) {
      listed[lane] = (int)e.id;
      const int d = (int)e.id - cut.head;
      if (e.id >= 0 && d >= 0 && d / N < cut.nvec) {
        const uint32_t at = (d / N) & bitmap_mask;
        atomicOr(&bitmap[at / 4], 1u << (at % 4 * 8 + d % N));
      }
    }
    __syncthreads();
  }
  Online o;
  for (int i = threadIdx.x; i < cut.nvec; i += NT) {
    Wide<T> x = widen<T>(load_packed(z + cut.start(i)));
    if constexpr (REST) {
      const uint32_t b = r.marks(i);
      if (b) {
#pragma unroll
        for (int k = 0; k < N; ++k)
          if (b >> k & 1) x[k] = -__builtin_inff();
      }
    }
    float hi = x[0];
#pragma unroll
    for (int k = 1; k < N; ++k) hi = fmaxf(hi, x[k]);
    if (hi > o.m) o.rise(hi, c);
#pragma unroll
    for (int k = 0; k < N; ++k) o.s += exp2_hw((x[k] - o.m) * c);
  }
  if ((int)threadIdx.x < cut.edges) {
    const int at = cut.edge(threadIdx.x);
    if (!REST || !r.is_listed(at)) {
      const float x = (float)z[at];
      if (x > o.m) o.rise(x, c);
      o.s += exp2_hw((x - o.m) * c);
    }
  }
  o = block_join<kWaves>(o, c, parts);
  if (wave == 0) {
    const DistillResult d = distill_finish<REST>(e, o, g.scale, bad);
    if (lane == 0) {
      if (g.loss) g.loss[row] = d.loss;
      if (g.stats) g.stats[row] = make_float4(o.m, d.f, d.m, d.lse);
      result[0] = d.f;
      result[1] = d.m;
      result[2] = d.lse;
      result[3] = d.total;
    }
  }
  if (!g.grad) return;
  __syncthreads();
  T* out = static_cast<T*>(g.grad) + row * g.grad_stride;
  const float scaled = g.scale * g.grad_loss[row], f = result[0] * scaled;
  auto one = [&](float x) { return exp2_hw((x - o.m) * c) * f; };
  for (int i = threadIdx.x; i < cut.nvec; i += NT) {
    Wide<T> x = widen<T>(load_packed(z + cut.start(i)));
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = one(x[k]);
    store_packed(out + cut.start(i), narrow<T>(x));
  }
  if ((int)threadIdx.x < cut.edges) {
    const int at = cut.edge(threadIdx.x);
    out[at] = (T)one((float)z[at]);
  }
  __syncthreads();
  if (wave == 0) patch_listed(g, out, e, scaled, result[3], result[1], result[2]);
}

template <typename T, bool REST>
__global__ __launch_bounds__(64 * kWaves) void distill_grad_kernel(DistillArgs g) {
  constexpr int NT = 64 * kWaves, N = RowTypes<T>::n;
  const int64_t row = block_row();
  if (row >= g.rows) return;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const T* z = static_cast<const T*>(g.logits) + row * g.stride;
  T* out = static_cast<T*>(g.grad) + row * g.grad_stride;
  const float c = g.scale * kLog2e;
  const Cut<T> cut(z, g.vocab);
  const float4 st = g.stats[row];
  const float scaled = g.scale * g.grad_loss[row], f = st.y * scaled, m = st.x;
  bool bad = false;
  Entry e{};
  float total = 0.f;
  if (wave == 0) {
    e = entry_of<T, REST>(g, z, row, lane, bad);
    total = wave_sum(e.q);
    if (REST) total += fmaxf(1.f - total, 0.f);
  }
  __syncthreads();  // in place: the entries' logits are read before anything is written
  auto one = [&](float x) { return exp2_hw((x - m) * c) * f; };
  for (int i = threadIdx.x; i < cut.nvec; i += NT) {
    Wide<T> x = widen<T>(load_packed(z + cut.start(i)));
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = one(x[k]);
    store_packed(out + cut.start(i), narrow<T>(x));
  }
  if ((int)threadIdx.x < cut.edges) {
    const int at = cut.edge(threadIdx.x);
    out[at] = (T)one((float)z[at]);
  }
  __syncthreads();
  if (wave == 0) patch_listed(g, out, e, scaled, total, st.z, st.w);
}

}  // namespace

int row_parts(int64_t rows, int64_t vocab) {
  int64_t parts = (kBlocksWanted + rows - 1) / rows;
  if (parts > vocab / kPartLeast) parts = vocab / kPartLeast;
  return parts < 1 ? 1 : parts > kPartsMost ? kPartsMost : (int)parts;
}

hipError_t launch_logprobs(const LogprobArgs& g, int dtype, hipStream_t stream) {
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (g.vocab / RowTypes<T>::n <= 256)
      HVDX_LAUNCH((logprobs_kernel<T, 1>), row_grid(g.rows * g.parts), dim3(64), 0, stream, g);
    else
      HVDX_LAUNCH((logprobs_kernel<T, kWaves>), row_grid(g.rows * g.parts), dim3(64 * kWaves), 0, stream, g);
  });
  return hipGetLastError();
}

hipError_t launch_logprobs_join(const LogprobArgs& g, int dtype, hipStream_t stream) {
  by_type(dtype, [&](auto t) {
    HVDX_LAUNCH(logprobs_join_kernel<decltype(t)>, row_grid(g.rows), dim3(64 * kWaves), 0, stream, g);
  });
  return hipGetLastError();
}

hipError_t launch_logprobs_grad(const LogprobGradArgs& g, int dtype, hipStream_t stream) {
  by_type(dtype, [&](auto t) {
    HVDX_LAUNCH(logprobs_grad_kernel<decltype(t)>, row_grid(g.rows), dim3(64 * kWaves), 0, stream, g);
  });
  return hipGetLastError();
}

hipError_t launch_distill(const DistillArgs& g, int dtype, hipStream_t stream) {
  const int64_t vectors = g.vocab / (dtype == HVDX_FLOAT32 ? 4 : 8) + 1;
  uint32_t bytes = 64;
  while (bytes < vectors && bytes < (uint32_t)kBitmapMost) bytes *= 2;
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (g.rest)
      HVDX_LAUNCH((distill_kernel<T, true>), row_grid(g.rows), dim3(64 * kWaves), bytes, stream, g, bytes - 1);
    else
      HVDX_LAUNCH((distill_kernel<T, false>), row_grid(g.rows), dim3(64 * kWaves), 0, stream, g, 0u);
  });
  return hipGetLastError();
}

hipError_t launch_distill_grad(const DistillArgs& g, int dtype, hipStream_t stream) {
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    if (g.rest) HVDX_LAUNCH((distill_grad_kernel<T, true>), row_grid(g.rows), dim3(64 * kWaves), 0, stream, g);
    else HVDX_LAUNCH((distill_grad_kernel<T, false>), row_grid(g.rows), dim3(64 * kWaves), 0, stream, g);
  });
  return hipGetLastError();
}

}  // namespace hvdx
