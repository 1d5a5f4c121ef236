// The residual connection between two blocks with the norms on either side, and its gradient.
//
// Forward, a row: r_y = (mean y^2 + eps)^{-1/2}, u = y r_y w_post, x' = x + s gate u,
// r_x = (mean x'^2 + eps)^{-1/2}, h = x' r_x w.  x' is normalised before it is rounded to its type.
// Backward, with xh = x' r_x and yh = y r_y:
//   dX = dx' + r_x (dh w - xh mean(dh w xh)),  dw = sum over rows of dh xh,
//   dgate = sum over the rows that share it of s u dX,  du = s gate dX,
//   dw_post = sum over rows of du yh,  dy = r_y (du w_post - yh mean(du w_post yh)).
// Sums, statistics and the weights' gradients are in binary32.  Bound: memory; a row stays in
// registers between its reads and its writes.  A thread keeps the same columns for every row of its
// block, so that the sums over rows stay in registers too; blocks write theirs to the
// workspace, and a second launch adds those in a fixed order.
#include <type_traits>

#include "rows.hpp"

namespace hvdx {
namespace {

template <typename T>
__device__ __forceinline__ Wide<T> load_some(const T* p, int count) {  // elements past `count` are 0
  if (count >= RowTypes<T>::n) return widen<T>(load_packed(p));
  Wide<T> v = 0.f;
#pragma unroll
  for (int k = 0; k < RowTypes<T>::n; ++k)
    if (k < count) v[k] = (float)p[k];
  return v;
}
template <typename T>
__device__ __forceinline__ void store_some(T* p, Wide<T> v, int count) {
  if (count >= RowTypes<T>::n) {
    store_packed(p, narrow<T>(v));
    return;
  }
#pragma unroll
  for (int k = 0; k < RowTypes<T>::n; ++k)
    if (k < count) p[k] = (T)v[k];
}
// As many binary32 values as the rows' type has in 16 bytes.
template <typename T>
__device__ __forceinline__ Wide<T> load_floats(const float* p, int count) {
  Wide<T> v = 0.f;
  constexpr int n = RowTypes<T>::n;
  if (count >= n) {
#pragma unroll
    for (int k = 0; k < n; k += 4) {
      const auto q = load_packed(p + k);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[k + i] = q[i];
    }
    return v;
  }
#pragma unroll
  for (int k = 0; k < n; ++k)
    if (k < count) v[k] = p[k];
  return v;
}
template <typename T>
__device__ __forceinline__ void store_floats(float* p, Wide<T> v, int count) {
#pragma unroll
  for (int k = 0; k < RowTypes<T>::n; ++k)
    if (k < count) p[k] = v[k];
}
template <typename T>
__device__ __forceinline__ Wide<T> load_gate(const void* gate, int f32, int64_t at, int count) {
  return f32 ? load_floats<T>(static_cast<const float*>(gate) + at, count)
             : load_some<T>(static_cast<const T*>(gate) + at, count);
}

template <typename T>
__device__ __forceinline__ float dot(Wide<T> a, Wide<T> b, float sum) {
#pragma unroll
  for (int k = 0; k < RowTypes<T>::n; ++k) sum = fmaf(a[k], b[k], sum);
  return sum;
}

// The sum over the block, in every thread.  Two calls in a row need W floats of `lds` each of their own:
// the second one's barrier stands between the first one's reads and the third one's writes.
template <int W>
__device__ __forceinline__ float block_sum(float x, float* lds) {
  x = wave_sum(x);
  if constexpr (W > 1) {
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) x += lds[w];
  }
  return x;
}

template <typename T, int W, int NV>
__global__ __launch_bounds__(64 * W) void norm_kernel(NormArgs g) {
  constexpr int N = RowTypes<T>::n, NT = 64 * W;
  __shared__ float lds[2][W];
  const int64_t row = block_row();
  if (row >= g.rows) return;
  const T* x = static_cast<const T*>(g.x) + row * g.x_stride;
  const float mean = 1.f / (float)g.dim;
  Wide<T> v[NV], u[NV];
  int count[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = ((int)threadIdx.x + i * NT) * N;
    count[i] = g.dim - at;
    v[i] = load_some(x + at, count[i]);
    if (g.y) u[i] = load_some(static_cast<const T*>(g.y) + row * g.y_stride + at, count[i]);
  }
  if (g.y) {
    float ry = 1.f;
    if (g.post) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) sum = dot<T>(u[i], u[i], sum);
      ry = 1.f / sqrtf(block_sum<W>(sum, lds[0]) * mean + g.eps);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int at = ((int)threadIdx.x + i * NT) * N;
      if (g.post) u[i] *= ry * load_floats<T>(g.post + at, count[i]);
      if (g.gate) u[i] *= load_gate<T>(g.gate, g.gate_f32, row / g.gate_rows * g.dim + at, count[i]);
      v[i] += g.scale * u[i];
      if (g.x_out) store_some(static_cast<T*>(g.x_out) + row * g.dim + at, v[i], count[i]);
    }
    if (g.stats && threadIdx.x == 0) g.stats[row].x = ry;
  } else if (g.stats && threadIdx.x == 0) {
    g.stats[row].x = 1.f;
  }
  if (!g.h_out && !g.stats) return;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) sum = dot<T>(v[i], v[i], sum);
  const float rx = 1.f / sqrtf(block_sum<W>(sum, lds[1]) * mean + g.eps);
  if (g.stats && threadIdx.x == 0) g.stats[row].y = rx;
  if (!g.h_out) return;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = ((int)threadIdx.x + i * NT) * N;
    Wide<T> h = v[i] * rx;
    if (g.weight) h *= load_floats<T>(g.weight + at, count[i]);
    store_some(static_cast<T*>(g.h_out) + row * g.dim + at, h, count[i]);
  }
}

template <typename T, int W, int NV>
__global__ __launch_bounds__(64 * W) void norm_grad_kernel(NormGradArgs g) {
  constexpr int N = RowTypes<T>::n, NT = 64 * W;
  __shared__ float lds[2][W];
  const int64_t block = block_row();
  const NormPlan& p = g.plan;
  if (block >= p.blocks) return;
  const float mean = 1.f / (float)g.dim;
  int turn = 0;
  Wide<T> dweight[NV], dpost[NV], dgate[NV];
  int count[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    dweight[i] = dpost[i] = 0.f;
    count[i] = g.dim - ((int)threadIdx.x + i * NT) * N;
  }
  const int64_t group0 = p.segments > 1 ? block / p.segments : block * p.per_block;
  int64_t group1 = p.segments > 1 ? group0 + 1 : group0 + p.per_block;
  if (group1 > p.groups) group1 = p.groups;
  for (int64_t group = group0; group < group1; ++group) {
    const int64_t first = group * p.span;
    const int64_t from = first + (p.segments > 1 ? block % p.segments * p.seg_rows : 0);
    int64_t to = from + p.seg_rows;
    if (to > first + p.span) to = first + p.span;
#pragma unroll
    for (int i = 0; i < NV; ++i) dgate[i] = 0.f;
    for (int64_t row = from; row < to; ++row) {
      const float2 r = g.stats[row];
      Wide<T> d[NV], a[NV], b[NV];
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int at = ((int)threadIdx.x + i * NT) * N;
        d[i] = 0.f;
        if (g.dx) d[i] = load_some(static_cast<const T*>(g.dx) + row * g.dx_stride + at, count[i]);
        if (g.dh) {
          a[i] = r.y * load_some(static_cast<const T*>(g.x) + row * g.x_stride + at, count[i]);
          b[i] = load_some(static_cast<const T*>(g.dh) + row * g.dh_stride + at, count[i]);
          dweight[i] += b[i] * a[i];
          if (g.weight) b[i] *= load_floats<T>(g.weight + at, count[i]);
          sum = dot<T>(a[i], b[i], sum);
        }
      }
      if (g.dh) {
        sum = block_sum<W>(sum, lds[turn ^= 1]) * mean;
#pragma unroll
        for (int i = 0; i < NV; ++i) d[i] += r.y * (b[i] - a[i] * sum);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int at = ((int)threadIdx.x + i * NT) * N;
        if (g.grad_x) store_some(static_cast<T*>(g.grad_x) + row * g.dim + at, d[i], count[i]);
      }
      if (!g.y) continue;
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int at = ((int)threadIdx.x + i * NT) * N;
        a[i] = load_some(static_cast<const T*>(g.y) + row * g.y_stride + at, count[i]);
        if (g.post) a[i] *= r.x;
        d[i] *= g.scale;
        Wide<T> post = 1.f;
        if (g.post) post = load_floats<T>(g.post + at, count[i]);
        if (g.gate) {
          dgate[i] += d[i] * a[i] * post;
          d[i] *= load_gate<T>(g.gate, g.gate_f32, group * g.dim + at, count[i]);
        }
        if (g.post) {
          dpost[i] += d[i] * a[i];
          d[i] *= post;
          sum = dot<T>(d[i], a[i], sum);
        }
      }
      if (g.post) sum = block_sum<W>(sum, lds[turn ^= 1]) * mean;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int at = ((int)threadIdx.x + i * NT) * N;
        if (g.post) d[i] = r.x * (d[i] - a[i] * sum);
        if (g.grad_y) store_some(static_cast<T*>(g.grad_y) + row * g.dim + at, d[i], count[i]);
      }
    }
    if (g.grad_gate) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int at = ((int)threadIdx.x + i * NT) * N;
        if (p.segments > 1) store_floats<T>(g.partial + (2 * p.blocks + block) * g.dim + at, dgate[i], count[i]);
        else if (g.gate_f32) store_floats<T>(static_cast<float*>(g.grad_gate) + group * g.dim + at, dgate[i], count[i]);
        else store_some(static_cast<T*>(g.grad_gate) + group * g.dim + at, dgate[i], count[i]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int at = ((int)threadIdx.x + i * NT) * N;
    if (g.grad_weight) store_floats<T>(g.partial + block * g.dim + at, dweight[i], count[i]);
    if (g.grad_post) store_floats<T>(g.partial + (p.blocks + block) * g.dim + at, dpost[i], count[i]);
  }
}

// The blocks' sums added in a fixed order: blockIdx.y 0 the weights', 1 the post norm's, 2 + group a
// group's vector of the gate.
template <typename G>
__global__ __launch_bounds__(256) void norm_sums_kernel(NormGradArgs g) {
  __shared__ float lds[4][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, column = (int)blockIdx.x * 64 + lane;
  const int64_t which = blockIdx.y, group = which - 2;
  if (which == 0 ? !g.grad_weight : which == 1 && !g.grad_post) return;
  const int64_t count = which < 2 ? g.plan.blocks : g.plan.segments;
  const float* p = g.partial + (which < 2 ? which * count : 2 * g.plan.blocks + group * count) * g.dim + column;
  float sum = 0.f;
  if (column < g.dim)
    for (int64_t k = wave; k < count; k += 4) sum += p[k * g.dim];
  lds[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || column >= g.dim) return;
  sum = (lds[0][lane] + lds[1][lane]) + (lds[2][lane] + lds[3][lane]);
  if (which == 0) g.grad_weight[column] = sum;
  else if (which == 1) g.grad_post[column] = sum;
  else static_cast<G*>(g.grad_gate)[group * g.dim + column] = (G)sum;
}

// The threads and vectors each that hold a row of `dim` elements.
template <typename T, typename F>
void by_dim(int dim, F f) {
  const int vectors = (dim + RowTypes<T>::n - 1) / RowTypes<T>::n;
  using std::integral_constant;
#define HVDX_SHAPE(w, nv) f(integral_constant<int, w>{}, integral_constant<int, nv>{})
  if (vectors <= 64) HVDX_SHAPE(1, 1);
  else if (vectors <= 128) HVDX_SHAPE(1, 2);
  else if (vectors <= 256) HVDX_SHAPE(4, 1);
  else if (vectors <= 512) HVDX_SHAPE(4, 2);
  else if (vectors <= 1024) HVDX_SHAPE(16, 1);
  else if (vectors <= 2048) HVDX_SHAPE(16, 2);
  else if (vectors <= 4096) HVDX_SHAPE(16, 4);
  else if constexpr (sizeof(T) == 4) HVDX_SHAPE(16, 8);
#undef HVDX_SHAPE
}
static_assert(HVDX_MAX_NORM_DIM <= 64 * 16 * 8 * 4 && HVDX_MAX_NORM_DIM <= 64 * 16 * 4 * 8);

}  // namespace

hipError_t launch_norm(const NormArgs& g, int dtype, hipStream_t stream) {
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    by_dim<T>(g.dim, [&](auto w, auto nv) {
      HVDX_LAUNCH((norm_kernel<T, w(), nv()>), row_grid(g.rows), dim3(64 * w()), 0, stream, g);
    });
  });
  return hipGetLastError();
}

NormPlan norm_plan(int64_t rows, int64_t gate_rows) {
  constexpr int64_t kBlocks = 512;
  NormPlan p{};
  p.span = gate_rows ? gate_rows : rows;
  p.groups = rows / p.span;
  p.segments = 1;
  if (p.groups < kBlocks) p.segments = (kBlocks + p.groups - 1) / p.groups;
  if (p.segments > p.span) p.segments = p.span;
  p.seg_rows = (p.span + p.segments - 1) / p.segments;
  p.segments = (p.span + p.seg_rows - 1) / p.seg_rows;
  p.per_block = p.segments > 1 ? 1 : (p.groups + kBlocks - 1) / kBlocks;
  p.blocks = p.segments > 1 ? p.groups * p.segments : (p.groups + p.per_block - 1) / p.per_block;
  return p;
}

hipError_t launch_norm_grad(const NormGradArgs& g, int dtype, hipStream_t stream) {
  by_type(dtype, [&](auto t) {
    using T = decltype(t);
    by_dim<T>(g.dim, [&](auto w, auto nv) {
      HVDX_LAUNCH((norm_grad_kernel<T, w(), nv()>), row_grid(g.plan.blocks), dim3(64 * w()), 0, stream, g);
    });
  });
  return hipGetLastError();
}

hipError_t launch_norm_grad_sums(const NormGradArgs& g, int dtype, hipStream_t stream) {
  const int64_t gates = g.grad_gate && g.plan.segments > 1 ? g.plan.groups : 0;  // fewer than norm_plan's blocks
  const dim3 grid((unsigned)(g.dim + 63) / 64, (unsigned)(2 + gates));
  by_type(g.gate_f32 ? HVDX_FLOAT32 : dtype, [&](auto t) {
    HVDX_LAUNCH(norm_sums_kernel<decltype(t)>, grid, dim3(256), 0, stream, g);
  });
  return hipGetLastError();
}

}  // namespace hvdx
