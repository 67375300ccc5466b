// Layer norm over the rows of a matrix, and its backward pass with the sums of the weight's and the bias's gradient.
//
//   y = h w + b,  h = (x - mean) rstd,  rstd = 1 / sqrt(var + eps)
//   dx = rstd (u - mean(u) - h mean(u h)),  u = dy w,     dw = sum over rows of dy h,  db = sum over rows of dy
//
// One pass over memory in either direction: a row stays in the registers of one group of threads (a warp, or a CTA), each of which owns the
// same columns in every row that its group takes, so that the weights are loaded once and the sums of dw and db stay in registers
// too; the groups' sums are then added by a second kernel, in a fixed order.  The variance is taken from the centred values, in
// a second reduction, not from the squares.  All arithmetic is in fp32; y and dx are rounded to their type once.
// Rows of more than kNormCols columns do not fit the registers: CTAs then read them again from L2.
#include <algorithm>

#include "atomo_ops.cuh"

namespace atomo {
namespace {

constexpr int kGroupMax = 512;                                   // threads per row, at most
constexpr int kGroupCols = 16;                                   // columns per thread, at most
constexpr int kNormCols = kGroupMax * kGroupCols;
constexpr int kWarpsPerCta = 8;                                  // rows side by side where a warp takes a row
constexpr int kBackCtas = 148 * 4;                               // partial rows of dw and db, at most

struct Weight { const void* p; int type; };
__device__ __forceinline__ float weight_at(const Weight& w, int64_t i, float none) {
  if (!w.p) return none;
  if (w.type == ATOMO_TYPE_F32) return reinterpret_cast<const float*>(w.p)[i];
  if (w.type == ATOMO_TYPE_BF16) return to_float(reinterpret_cast<const __nv_bfloat16*>(w.p)[i]);
  return to_float(reinterpret_cast<const __half*>(w.p)[i]);
}

// sums of R values over a group: a warp, or all warps of the CTA (which meet once; s: R x 32 floats that nobody reads any more)
template <int R, bool WARP>
__device__ __forceinline__ void group_sum(float (&v)[R], float* s) {
#pragma unroll
  for (int r = 0; r < R; ++r) v[r] = warp_sum(v[r]);
  if constexpr (!WARP) {
    const int warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
      for (int r = 0; r < R; ++r) s[r * 32 + (threadIdx.x >> 5)] = v[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float t = 0.0f;
      for (int w = 0; w < warps; ++w) t += s[r * 32 + w];
      v[r] = t;
    }
  }
}

// Columns of a thread: PACKS pieces of VEC neighbouring ones, a group's width apart.  R rows at a time.
template <typename T, int VEC, int PACKS, int R, bool WARP>
__global__ void __launch_bounds__(WARP ? kWarpsPerCta * 32 : kGroupMax) ln_forward_kernel(const T* x, int64_t rows, int cols, int64_t ld, Weight weight, Weight bias,
                                                                                         float eps, T* y, int64_t ld_y, float* __restrict__ mean, float* __restrict__ rstd) {
  __shared__ float s_sum[2][R * 32];
  const int width = WARP ? 32 : blockDim.x, lane = WARP ? threadIdx.x & 31 : threadIdx.x;
  const int64_t groups = WARP ? (int64_t)gridDim.x * kWarpsPerCta : gridDim.x;
  const int64_t group = WARP ? (int64_t)blockIdx.x * kWarpsPerCta + (threadIdx.x >> 5) : blockIdx.x;
  const float inv = 1.0f / (float)cols;
  float w[PACKS][VEC], b[PACKS][VEC];
#pragma unroll
  for (int k = 0; k < PACKS; ++k) {
    const int c = (k * width + lane) * VEC;
#pragma unroll
    for (int j = 0; j < VEC; ++j) { w[k][j] = c < cols ? weight_at(weight, c + j, 1.0f) : 0.0f; b[k][j] = c < cols ? weight_at(bias, c + j, 0.0f) : 0.0f; }
  }
  for (int64_t r0 = group * R; r0 < rows; r0 += groups * R) {
    Pack<T, VEC> raw[R][PACKS];
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int k = 0; k < PACKS; ++k) {
        const int c = (k * width + lane) * VEC;
        if (r0 + r < rows && c < cols) raw[r][k] = load_pack<T, VEC>(x + (r0 + r) * ld + c);
        else {
#pragma unroll
          for (int j = 0; j < VEC; ++j) raw[r][k].v[j] = from_float<T>(0.0f);
        }
      }
    }
    float mu[R], var[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mu[r] = 0.0f;
#pragma unroll
      for (int k = 0; k < PACKS; ++k) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) mu[r] += to_float(raw[r][k].v[j]);
      }
    }
    group_sum<R, WARP>(mu, s_sum[0]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mu[r] *= inv; var[r] = 0.0f;
#pragma unroll
      for (int k = 0; k < PACKS; ++k) {
        if ((k * width + lane) * VEC < cols) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) { const float d = to_float(raw[r][k].v[j]) - mu[r]; var[r] = fmaf(d, d, var[r]); }
        }
      }
    }
    group_sum<R, WARP>(var, s_sum[1]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r0 + r >= rows) break;
      const float rs = 1.0f / sqrtf(var[r] * inv + eps);
#pragma unroll
      for (int k = 0; k < PACKS; ++k) {
        const int c = (k * width + lane) * VEC;
        if (c < cols) {
          Pack<T, VEC> o;
#pragma unroll
          for (int j = 0; j < VEC; ++j) o.v[j] = from_float<T>(fmaf((to_float(raw[r][k].v[j]) - mu[r]) * rs, w[k][j], b[k][j]));
          store_pack<T, VEC>(y + (r0 + r) * ld_y + c, o);
        }
      }
      if (lane == 0) { mean[r0 + r] = mu[r]; rstd[r0 + r] = rs; }
    }
  }
}

template <typename T, int VEC, int PACKS, int R, bool WARP>
__global__ void __launch_bounds__(WARP ? kWarpsPerCta * 32 : kGroupMax) ln_backward_kernel(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, int64_t rows, int cols,
                                                                                          Weight weight, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                                                          T* dx, int64_t ld_dx, float* __restrict__ parts) {
  __shared__ float s_sum[2][2 * R * 32];
  extern __shared__ float s_cols[];                              // WARP: [warps][cols], twice
  const int width = WARP ? 32 : blockDim.x, lane = WARP ? threadIdx.x & 31 : threadIdx.x;
  const int64_t groups = WARP ? (int64_t)gridDim.x * kWarpsPerCta : gridDim.x;
  const int64_t group = WARP ? (int64_t)blockIdx.x * kWarpsPerCta + (threadIdx.x >> 5) : blockIdx.x;
  const float inv = 1.0f / (float)cols;
  float w[PACKS][VEC], dw[PACKS][VEC], db[PACKS][VEC];
#pragma unroll
  for (int k = 0; k < PACKS; ++k) {
    const int c = (k * width + lane) * VEC;
#pragma unroll
    for (int j = 0; j < VEC; ++j) { w[k][j] = c < cols ? weight_at(weight, c + j, 1.0f) : 0.0f; dw[k][j] = 0.0f; db[k][j] = 0.0f; }
  }
  int turn = 0;
  for (int64_t r0 = group * R; r0 < rows; r0 += groups * R, turn ^= 1) {
    Pack<T, VEC> px[R][PACKS], pd[R][PACKS];
    float mu[R], rs[R], s[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool in = r0 + r < rows;
#pragma unroll
      for (int k = 0; k < PACKS; ++k) {
        const int c = (k * width + lane) * VEC;
        if (in && c < cols) { px[r][k] = load_pack<T, VEC>(x + (r0 + r) * ld_x + c); pd[r][k] = load_pack<T, VEC>(dy + (r0 + r) * ld_dy + c); }
        else {
#pragma unroll
          for (int j = 0; j < VEC; ++j) { px[r][k].v[j] = from_float<T>(0.0f); pd[r][k].v[j] = from_float<T>(0.0f); }
        }
      }
      mu[r] = in ? mean[r0 + r] : 0.0f; rs[r] = in ? rstd[r0 + r] : 0.0f;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[2 * r] = 0.0f; s[2 * r + 1] = 0.0f;
#pragma unroll
      for (int k = 0; k < PACKS; ++k) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float d = to_float(pd[r][k].v[j]), hat = (to_float(px[r][k].v[j]) - mu[r]) * rs[r], u = d * w[k][j];
          s[2 * r] += u; s[2 * r + 1] = fmaf(u, hat, s[2 * r + 1]);
          dw[k][j] = fmaf(d, hat, dw[k][j]); db[k][j] += d;
        }
      }
    }
    group_sum<2 * R, WARP>(s, s_sum[turn]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r0 + r >= rows) break;
      const float m1 = s[2 * r] * inv, m2 = s[2 * r + 1] * inv;
#pragma unroll
      for (int k = 0; k < PACKS; ++k) {
        const int c = (k * width + lane) * VEC;
        if (c < cols) {
          Pack<T, VEC> o;
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const float hat = (to_float(px[r][k].v[j]) - mu[r]) * rs[r], u = to_float(pd[r][k].v[j]) * w[k][j];
            o.v[j] = from_float<T>(rs[r] * (u - m1 - hat * m2));
          }
          store_pack<T, VEC>(dx + (r0 + r) * ld_dx + c, o);
        }
      }
    }
  }
  // this CTA's rows of partial sums: dw, then db
  float* part_w = parts + (int64_t)blockIdx.x * cols;
  float* part_b = parts + ((int64_t)gridDim.x + blockIdx.x) * cols;
  if constexpr (WARP) {
    float* mine = s_cols + (threadIdx.x >> 5) * 2 * cols;
#pragma unroll
    for (int k = 0; k < PACKS; ++k) {
      const int c = (k * width + lane) * VEC;
      if (c < cols) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) { mine[c + j] = dw[k][j]; mine[cols + c + j] = db[k][j]; }
      }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * cols; c += blockDim.x) {
      float t = 0.0f;
#pragma unroll
      for (int v = 0; v < kWarpsPerCta; ++v) t += s_cols[v * 2 * cols + c];
      if (c < cols) part_w[c] = t; else part_b[c - cols] = t;
    }
  } else {
#pragma unroll
    for (int k = 0; k < PACKS; ++k) {
      const int c = (k * width + lane) * VEC;
      if (c < cols) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) { part_w[c + j] = dw[k][j]; part_b[c + j] = db[k][j]; }
      }
    }
  }
}

// sums of the partial rows: 32 columns per CTA, sixteen rows side by side
constexpr int kJoinRows = 16;
__global__ void __launch_bounds__(32 * kJoinRows) ln_join_kernel(const float* __restrict__ parts, int n, int cols, float* __restrict__ dweight, float* __restrict__ dbias) {
  __shared__ float s[kJoinRows][33];
  wait_for_previous();
  const int c = blockIdx.x * 32 + threadIdx.x;
  float* out = blockIdx.y == 0 ? dweight : dbias;
  float t = 0.0f;
  if (out && c < cols) {
    const float* p = parts + (int64_t)blockIdx.y * n * cols + c;
#pragma unroll 8
    for (int i = threadIdx.y; i < n; i += kJoinRows) t += p[(int64_t)i * cols];
  }
  s[threadIdx.y][threadIdx.x] = t;
  __syncthreads();
  if (threadIdx.y == 0 && out && c < cols) {
    t = 0.0f;
#pragma unroll
    for (int i = 0; i < kJoinRows; ++i) t += s[i][threadIdx.x];
    out[c] = t;
  }
}

// ---- rows longer than the registers hold ----------------------------------------------------------
constexpr int kLongThreads = 1024;
template <typename T>
__global__ void __launch_bounds__(kLongThreads) ln_forward_long_kernel(const T* x, int cols, int64_t ld, Weight weight, Weight bias, float eps,
                                                                       T* y, int64_t ld_y, float* __restrict__ mean, float* __restrict__ rstd) {
  __shared__ float s_sum[2][32];
  const int64_t row = blockIdx.x;
  const T* p = x + row * ld;
  float v[1] = {0.0f};
  for (int c = threadIdx.x; c < cols; c += kLongThreads) v[0] += to_float(p[c]);
  group_sum<1, false>(v, s_sum[0]);
  const float mu = v[0] / (float)cols;
  v[0] = 0.0f;
  for (int c = threadIdx.x; c < cols; c += kLongThreads) { const float d = to_float(p[c]) - mu; v[0] = fmaf(d, d, v[0]); }
  group_sum<1, false>(v, s_sum[1]);
  const float rs = 1.0f / sqrtf(v[0] / (float)cols + eps);
  for (int c = threadIdx.x; c < cols; c += kLongThreads)
    y[row * ld_y + c] = from_float<T>(fmaf((to_float(p[c]) - mu) * rs, weight_at(weight, c, 1.0f), weight_at(bias, c, 0.0f)));
  if (threadIdx.x == 0) { mean[row] = mu; rstd[row] = rs; }
}

template <typename T>
__global__ void __launch_bounds__(kLongThreads) ln_backward_long_kernel(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, int cols, Weight weight,
                                                                        const float* __restrict__ mean, const float* __restrict__ rstd, T* dx, int64_t ld_dx) {
  __shared__ float s_sum[2 * 32];
  const int64_t row = blockIdx.x;
  const float mu = mean[row], rs = rstd[row];
  float s[2] = {0.0f, 0.0f};
  for (int c = threadIdx.x; c < cols; c += kLongThreads) {
    const float u = to_float(dy[row * ld_dy + c]) * weight_at(weight, c, 1.0f), hat = (to_float(x[row * ld_x + c]) - mu) * rs;
    s[0] += u; s[1] = fmaf(u, hat, s[1]);
  }
  group_sum<2, false>(s, s_sum);
  const float m1 = s[0] / (float)cols, m2 = s[1] / (float)cols;
  for (int c = threadIdx.x; c < cols; c += kLongThreads) {
    const float u = to_float(dy[row * ld_dy + c]) * weight_at(weight, c, 1.0f), hat = (to_float(x[row * ld_x + c]) - mu) * rs;
    dx[row * ld_dx + c] = from_float<T>(rs * (u - m1 - hat * m2));
  }
}
// partial sums of dw and db: a CTA takes 256 columns of every gridDim.y-th row
template <typename T>
__global__ void __launch_bounds__(256) ln_columns_kernel(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, int64_t rows, int cols,
                                                         const float* __restrict__ mean, const float* __restrict__ rstd, float* __restrict__ parts) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  float w = 0.0f, b = 0.0f;
#pragma unroll 4
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
    const float d = to_float(dy[r * ld_dy + c]);
    w = fmaf(d, (to_float(x[r * ld_x + c]) - mean[r]) * rstd[r], w); b += d;
  }
  parts[(int64_t)blockIdx.y * cols + c] = w;
  parts[((int64_t)gridDim.y + blockIdx.y) * cols + c] = b;
}

// ---- choice of form -------------------------------------------------------------------------------
bool fits16(const void* p, int64_t ld, int64_t cols, int size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld * size) % 16 == 0 && (cols * size) % 16 == 0;
}
int sm_ctas(const void* kernel, int threads, size_t smem) {      // CTAs of a full GPU
  int per = 1;
  if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, threads, smem) != cudaSuccess) { cudaGetLastError(); per = 1; }
  return 148 * std::max(per, 1);
}

template <typename T, int VEC, int PACKS, int R>
cudaError_t forward_form(const NormForward& a, cudaStream_t st) {
  const Weight w{a.weight, a.weight_type}, b{a.bias, a.weight_type};
  if (a.cols <= 32 * VEC * PACKS) {
    static const int full = sm_ctas((const void*)ln_forward_kernel<T, VEC, PACKS, R, true>, kWarpsPerCta * 32, 0);
    const int grid = (int)std::min<int64_t>((a.rows + kWarpsPerCta * R - 1) / (kWarpsPerCta * R), full);
    ln_forward_kernel<T, VEC, PACKS, R, true><<<grid, kWarpsPerCta * 32, 0, st>>>((const T*)a.x, a.rows, (int)a.cols, a.ld, w, b, a.eps, (T*)a.y, a.ld_y, a.mean, a.rstd);
  } else {
    const int threads = (int)((a.cols + 32 * VEC * PACKS - 1) / (32 * VEC * PACKS)) * 32;
    const int grid = (int)std::min<int64_t>((a.rows + R - 1) / R, 148 * std::max(1, 1024 / threads));
    ln_forward_kernel<T, VEC, PACKS, R, false><<<grid, threads, 0, st>>>((const T*)a.x, a.rows, (int)a.cols, a.ld, w, b, a.eps, (T*)a.y, a.ld_y, a.mean, a.rstd);
  }
  return cudaGetLastError();
}
template <typename T>
cudaError_t forward_type(const NormForward& a, cudaStream_t st) {
  if (a.cols > kNormCols) {
    ln_forward_long_kernel<T><<<(unsigned)a.rows, kLongThreads, 0, st>>>((const T*)a.x, (int)a.cols, a.ld, Weight{a.weight, a.weight_type}, Weight{a.bias, a.weight_type}, a.eps,
                                                                        (T*)a.y, a.ld_y, a.mean, a.rstd);
    return cudaGetLastError();
  }
  constexpr int kVec = 16 / (int)sizeof(T);
  if (fits16(a.x, a.ld, a.cols, sizeof(T)) && fits16(a.y, a.ld_y, a.cols, sizeof(T))) {
    if (a.cols <= kGroupMax * kVec) return forward_form<T, kVec, 1, 2>(a, st);
    return forward_form<T, kVec, kGroupCols / kVec, 1>(a, st);
  }
  if (a.cols <= kGroupMax * 4) return forward_form<T, 1, 4, 2>(a, st);
  return forward_form<T, 1, kGroupCols, 1>(a, st);
}

int back_ctas(int64_t rows, int64_t per) { return (int)std::min<int64_t>((rows + per - 1) / per, kBackCtas); }

template <typename T>
cudaError_t backward_join(const NormBackward& a, int n, cudaStream_t st) {
  if (!a.dweight && !a.dbias) return cudaSuccess;
  return launch_after(ln_join_kernel, dim3((unsigned)((a.cols + 31) / 32), 2), dim3(32, kJoinRows), 0, st, a.ws, n, (int)a.cols, a.dweight, a.dbias);
}
template <typename T, int VEC, int PACKS, int R>
cudaError_t backward_form(const NormBackward& a, cudaStream_t st) {
  const Weight w{a.weight, a.weight_type};
  int grid;
  if (a.cols <= 32 * VEC * PACKS) {
    grid = back_ctas(a.rows, kWarpsPerCta * R);
    ln_backward_kernel<T, VEC, PACKS, R, true><<<grid, kWarpsPerCta * 32, kWarpsPerCta * 2 * a.cols * 4, st>>>((const T*)a.dy, a.ld_dy, (const T*)a.x, a.ld_x, a.rows, (int)a.cols, w, a.mean, a.rstd,
                                                                                                        (T*)a.dx, a.ld_dx, a.ws);
  } else {
    const int threads = (int)((a.cols + 32 * VEC * PACKS - 1) / (32 * VEC * PACKS)) * 32;
    grid = std::min(back_ctas(a.rows, R), 148 * std::max(1, 512 / threads));
    ln_backward_kernel<T, VEC, PACKS, R, false><<<grid, threads, 0, st>>>((const T*)a.dy, a.ld_dy, (const T*)a.x, a.ld_x, a.rows, (int)a.cols, w, a.mean, a.rstd, (T*)a.dx, a.ld_dx, a.ws);
  }
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : backward_join<T>(a, grid, st);
}
template <typename T>
cudaError_t backward_type(const NormBackward& a, cudaStream_t st) {
  if (a.rows == 0) return backward_join<T>(a, 0, st);
  if (a.cols > kNormCols) {
    const Weight w{a.weight, a.weight_type};
    const int split = back_ctas(a.rows, 32);                     // first, since dx may lie where dy or x does
    ln_columns_kernel<T><<<dim3((unsigned)((a.cols + 255) / 256), split), 256, 0, st>>>((const T*)a.dy, a.ld_dy, (const T*)a.x, a.ld_x, a.rows, (int)a.cols, a.mean, a.rstd, a.ws);
    ln_backward_long_kernel<T><<<(unsigned)a.rows, kLongThreads, 0, st>>>((const T*)a.dy, a.ld_dy, (const T*)a.x, a.ld_x, (int)a.cols, w, a.mean, a.rstd, (T*)a.dx, a.ld_dx);
    const cudaError_t e = cudaGetLastError();
    return e != cudaSuccess ? e : backward_join<T>(a, split, st);
  }
  constexpr int kVec = 16 / (int)sizeof(T);
  if (fits16(a.x, a.ld_x, a.cols, sizeof(T)) && fits16(a.dy, a.ld_dy, a.cols, sizeof(T)) && fits16(a.dx, a.ld_dx, a.cols, sizeof(T))) {
    if (a.cols <= kGroupMax * kVec) return backward_form<T, kVec, 1, 2>(a, st);
    return backward_form<T, kVec, kGroupCols / kVec, 1>(a, st);
  }
  if (a.cols <= kGroupMax * 4) return backward_form<T, 1, 4, 2>(a, st);
  return backward_form<T, 1, kGroupCols, 1>(a, st);
}

}  // namespace

int launch_layer_norm(const NormForward& a, cudaStream_t st) {
  if (a.rows == 0) return (int)cudaSuccess;
  if (a.type == ATOMO_TYPE_F32) return (int)forward_type<float>(a, st);
  if (a.type == ATOMO_TYPE_BF16) return (int)forward_type<__nv_bfloat16>(a, st);
  return (int)forward_type<__half>(a, st);
}

uint64_t layer_norm_workspace(int64_t rows, int64_t cols) { return (uint64_t)std::min<int64_t>(rows, kBackCtas) * 2 * cols * 4; }

int launch_layer_norm_backward(const NormBackward& a, cudaStream_t st) {
  if (a.type == ATOMO_TYPE_F32) return (int)backward_type<float>(a, st);
  if (a.type == ATOMO_TYPE_BF16) return (int)backward_type<__nv_bfloat16>(a, st);
  return (int)backward_type<__half>(a, st);
}

}  // namespace atomo
