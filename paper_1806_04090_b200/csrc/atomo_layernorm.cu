// Layer norm over the rows of a matrix, and its backward pass with the sums of the weight's and the bias's gradient.
//
//   y = h w + b,  h = (x - mean) rstd,  rstd = 1 / sqrt(var + eps)
//   dx = rstd (u - mean(u) - h mean(u h)),  u = dy w,     dw = sum over rows of dy h,  db = sum over rows of dy
//
// One pass over memory in either direction: a row stays on chip with one group of threads (a warp, or a CTA), each of which owns the
// same columns in every row that its group takes, so that the weights are loaded once and the sums of dw and db stay in registers
// too; the groups' sums are then added by a second kernel, in a fixed order.  The rows to come are copied to shared memory meanwhile, by the threads that
// will use them, so that copies in flight take no registers and are waited for by their own thread alone.  A thread has up to 32 columns, two at a time in packed
// fp32: what a row costs every warp (shuffles, the exchange among warps) outweighs the arithmetic where a thread has few, and instruction issue then bounds
// the kernels instead of memory (2048 bf16 columns, 8 per thread: 33 instructions per element forward, 82 us for 32768 rows).
//   The variance is taken from the values centred on the warp's mean, and the warps' are combined as M2 = sum of M2_w + n_w (mean_w - mean)^2, which takes
// one exchange and loses nothing where the mean is far from zero.  All arithmetic is in fp32; y and dx are rounded to their type once.
// Rows of more than kNormCols columns do not fit: CTAs then read them again from L2.
#include <algorithm>

#include "atomo_ops.cuh"

namespace atomo {
namespace {

constexpr int kGroupMax = 512;                                   // threads per row, at most
constexpr int kNormCols = kGroupMax * 32;
constexpr int kWarpsPerCta = 8;                                  // rows side by side where a warp takes a row
constexpr int kBackCtas = 148 * 4;                               // partial rows of dw and db, at most
#ifndef FST
#define FST 4
#endif
#ifndef BST
#define BST 3
#endif
// By the bytes of a row that a thread has: rows per step; steps whose rows are in shared memory or on the way there (512 threads with 128 bytes of x and of dy:
// 128 KB a step)
__host__ __device__ constexpr int rows_per_step(int bytes) { return bytes <= 32 ? 2 : 1; }
__host__ __device__ constexpr int forward_stages(int bytes) { return bytes <= 64 ? FST : 2; }
__host__ __device__ constexpr int backward_stages(int bytes) { return bytes <= 64 ? BST : 1; }

struct Weight { const void* p; int type; };
__device__ __forceinline__ float weight_at(const Weight& w, int64_t i, float none) {
  if (!w.p) return none;
  if (w.type == ATOMO_TYPE_F32) return reinterpret_cast<const float*>(w.p)[i];
  if (w.type == ATOMO_TYPE_BF16) return to_float(reinterpret_cast<const __nv_bfloat16*>(w.p)[i]);
  return to_float(reinterpret_cast<const __half*>(w.p)[i]);
}

// ---- pairs of values ----
__device__ __forceinline__ uint64_t both(float x) { return pack2(x, x); }
__device__ __forceinline__ float halves(uint64_t v) { float a, b; unpack2(v, a, b); return a + b; }

// sum over the lanes that differ in the bits below `span`, a power of two
__device__ __forceinline__ float span_sum(float v, int span) {
  for (int o = 1; o < span; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ int warp_span() {                     // warps of the CTA, rounded up to a power of two
  int span = 1;
  while (span < (int)(blockDim.x >> 5)) span <<= 1;
  return span;
}
__device__ __forceinline__ float one_over_root(float x) {        // to about one unit in the last place
  const float r = rsqrtf(x);
  return fmaf(r * 0.5f, fmaf(-x * r, r, 1.0f), r);
}

// A thread's packs of the rows that come next: STAGES steps of ROWS rows (of N arrays: x, or x and dy), in shared memory.  16- and 4-byte packs are copied
// asynchronously; 2-byte ones are loaded.
template <typename T, int VEC, int PACKS, int ROWS, int STAGES>
struct RowRing {
  static constexpr int kBytes = VEC * (int)sizeof(T);
  static constexpr bool kAsync = kBytes == 16 || kBytes == 4;
  static constexpr uint32_t kAll = PACKS == 32 ? 0xffffffffu : (1u << (PACKS & 31)) - 1u;
  Pack<T, VEC>* slot;                  // of this thread
  __device__ __forceinline__ Pack<T, VEC>* at(int stage, int row, int k) const { return slot + ((stage * ROWS + row) * PACKS + k) * blockDim.x; }
  __device__ __forceinline__ void put(int stage, int row, int k, const T* p) {
    if constexpr (kAsync) copy_async<kBytes>(at(stage, row, k), p); else *at(stage, row, k) = load_pack<T, VEC>(p);
  }
  __device__ __forceinline__ void close() { if constexpr (kAsync) asm volatile("cp.async.commit_group;" ::: "memory"); }
  __device__ __forceinline__ void wait() { if constexpr (kAsync) asm volatile("cp.async.wait_group %0;" :: "n"(STAGES - 1) : "memory"); }
  // the thread's columns of a row, as pairs; zeros where it has none (in: a bit per pack)
  __device__ __forceinline__ void get(int stage, int row, uint32_t in, uint64_t (&v)[VEC * PACKS / 2]) const {
    if (in == kAll) {
#pragma unroll
      for (int k = 0; k < PACKS; k += VEC > 1 ? 1 : 2) {
        if constexpr (VEC > 1) {
          const Pack<T, VEC> raw = *at(stage, row, k);
#pragma unroll
          for (int j = 0; j < VEC; j += 2) v[(k * VEC + j) / 2] = pair_of(raw.v + j);
        } else v[k / 2] = pack2(to_float(at(stage, row, k)->v[0]), to_float(at(stage, row, k + 1)->v[0]));
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC * PACKS / 2; ++e) v[e] = 0;
#pragma unroll
      for (int k = 0; k < PACKS; k += VEC > 1 ? 1 : 2) {
        if (!(in >> k & 1u)) break;                               // (the packs that a thread has are its first ones)
        if constexpr (VEC > 1) {
          const Pack<T, VEC> raw = *at(stage, row, k);
#pragma unroll
          for (int j = 0; j < VEC; j += 2) v[(k * VEC + j) / 2] = pair_of(raw.v + j);
        } else v[k / 2] = pack2(to_float(at(stage, row, k)->v[0]), in >> (k + 1) & 1u ? to_float(at(stage, row, k + 1)->v[0]) : 0.0f);
      }
    }
  }
};
template <typename T, int VEC, int PACKS>
__device__ __forceinline__ void put_pairs(T* row, int width, int lane, uint32_t in, const uint64_t (&v)[VEC * PACKS / 2]) {
  if constexpr (VEC > 1) {
#pragma unroll
    for (int k = 0; k < PACKS; ++k) {
      if (in >> k & 1u) {
        Pack<T, VEC> o;
#pragma unroll
        for (int j = 0; j < VEC; j += 2) pair_to(o.v + j, v[(k * VEC + j) / 2]);
        store_pack<T, VEC>(row + (k * width + lane) * VEC, o);
      }
    }
  } else {
#pragma unroll
    for (int k = 0; k < PACKS; k += 2) {
      float a, b;
      unpack2(v[k / 2], a, b);
      if (in >> k & 1u) row[k * width + lane] = from_float<T>(a);
      if (in >> (k + 1) & 1u) row[(k + 1) * width + lane] = from_float<T>(b);
    }
  }
}
// the same into a row of fp32 values of any alignment
template <int VEC, int PACKS>
__device__ __forceinline__ void put_columns(float* row, int width, int lane, uint32_t in, const uint64_t (&v)[VEC * PACKS / 2]) {
#pragma unroll
  for (int e = 0; e < VEC * PACKS; e += 2) {
    float f[2];
    unpack2(v[e / 2], f[0], f[1]);
#pragma unroll
    for (int i = 0; i < 2; ++i) if (in >> ((e + i) / VEC) & 1u) row[((e + i) / VEC * width + lane) * VEC + (e + i) % VEC] = f[i];
  }
}
// the thread's columns of the weight (or of what stands in for it where there is none)
template <int VEC, int PACKS>
__device__ __forceinline__ void get_weight(const Weight& w, int width, int lane, uint32_t in, float none, uint64_t (&v)[VEC * PACKS / 2]) {
  float f[VEC * PACKS];
#pragma unroll
  for (int k = 0; k < PACKS; ++k) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) f[k * VEC + j] = in >> k & 1u ? weight_at(w, (k * width + lane) * VEC + j, none) : 0.0f;
  }
#pragma unroll
  for (int e = 0; e < VEC * PACKS / 2; ++e) v[e] = pack2(f[2 * e], f[2 * e + 1]);
}

// Columns of a thread: PACKS pieces of VEC neighbouring ones, a group's width apart; with 32 the weights are read anew for every row.
template <typename T, int VEC, int PACKS, bool WARP>
__global__ void __launch_bounds__(WARP ? kWarpsPerCta * 32 : kGroupMax) ln_forward_kernel(const T* x, int64_t rows, int cols, int64_t ld, Weight weight, Weight bias,
                                                                                         float eps, T* y, int64_t ld_y, float* __restrict__ mean, float* __restrict__ rstd) {
  constexpr int E = VEC * PACKS, R = rows_per_step(E * sizeof(T)), kStages = forward_stages(E * sizeof(T));
  constexpr bool kKeep = E < 32;
  extern __shared__ uint4 s_ring[];
  __shared__ float2 s_sum[2][R][16];
  __shared__ float s_count[16];
  const int width = WARP ? 32 : blockDim.x, lane = WARP ? threadIdx.x & 31 : threadIdx.x, warps = blockDim.x >> 5;
  const int64_t groups = WARP ? (int64_t)gridDim.x * kWarpsPerCta : gridDim.x;
  const int64_t group = WARP ? (int64_t)blockIdx.x * kWarpsPerCta + (threadIdx.x >> 5) : blockIdx.x;
  const float inv = 1.0f / (float)cols;
  uint32_t in = 0;                                               // packs that lie inside the row
#pragma unroll
  for (int k = 0; k < PACKS; ++k) if ((k * width + lane) * VEC < cols) in |= 1u << k;
  const bool full = in == RowRing<T, VEC, PACKS, R, kStages>::kAll;
  RowRing<T, VEC, PACKS, R, kStages> ring{reinterpret_cast<Pack<T, VEC>*>(s_ring) + threadIdx.x};
  const T* from = x + group * R * ld + lane * VEC;               // the next row to fetch
  int64_t fetched = group * R;
  auto fetch = [&](int stage) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int k = 0; k < PACKS; ++k) if (fetched + r < rows && (in >> k & 1u)) ring.put(stage, r, k, from + r * ld + k * width * VEC);
    }
    ring.close();
    from += groups * R * ld; fetched += groups * R;
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) fetch(i);
  uint64_t w[E / 2], b[E / 2];
  if constexpr (kKeep) { get_weight<VEC, PACKS>(weight, width, lane, in, 1.0f, w); get_weight<VEC, PACKS>(bias, width, lane, in, 0.0f, b); }
  const float count = warp_sum((float)(__popc(in) * VEC)), inv_count = 1.0f / count;       // columns of this warp
  const int span = WARP ? 1 : warp_span(), mate = threadIdx.x & (span - 1);
  const bool other = mate < warps;
  float mate_count = 0.0f, mate_inv = 0.0f;                      // columns of the warp whose sums this lane takes
  if constexpr (!WARP) {
    if ((threadIdx.x & 31) == 0) s_count[threadIdx.x >> 5] = count;
    __syncthreads();
    if (other) { mate_count = s_count[mate]; mate_inv = 1.0f / mate_count; }
  }
  int stage = 0, turn = 0;
  for (int64_t r0 = group * R; r0 < rows; r0 += groups * R, turn ^= 1) {
    fetch(stage == 0 ? kStages - 1 : stage - 1);
    ring.wait();
    uint64_t v[R][E / 2];
    float mu[R], var[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r0 + r < rows) ring.get(stage, r, in, v[r]);
      else {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) v[r][e] = 0;
      }
      uint64_t t = v[r][0];
#pragma unroll
      for (int e = 1; e < E / 2; ++e) t = add2(t, v[r][e]);
      mu[r] = halves(t);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) mu[r] = warp_sum(mu[r]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint64_t centre = both(-mu[r] * inv_count);
      uint64_t t = 0;
      if (full) {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) { const uint64_t d = add2(v[r][e], centre); t = fma2(d, d, t); }
        var[r] = halves(t);
      } else {
        var[r] = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          float p, q;
          unpack2(add2(v[r][e / 2], centre), p, q);
          const float d = in >> (e / VEC) & 1u ? (e & 1 ? q : p) : 0.0f;
          var[r] = fmaf(d, d, var[r]);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) var[r] = warp_sum(var[r]);
    if constexpr (!WARP) {
      if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) s_sum[turn][r][threadIdx.x >> 5] = make_float2(mu[r], var[r]);
      }
      __syncthreads();
#pragma unroll
      for (int r = 0; r < R; ++r) {                               // a lane per warp
        const float2 q = other ? s_sum[turn][r][mate] : make_float2(0.0f, 0.0f);
        mu[r] = span_sum(q.x, span);
        const float d = fmaf(-mu[r], inv, q.x * mate_inv);
        var[r] = span_sum(fmaf(mate_count * d, d, q.y), span);
      }
    }
    if constexpr (!kKeep) { get_weight<VEC, PACKS>(weight, width, lane, in, 1.0f, w); get_weight<VEC, PACKS>(bias, width, lane, in, 0.0f, b); }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r0 + r < rows) {
        const float m = mu[r] * inv, rs = one_over_root(fmaf(var[r], inv, eps));
        const uint64_t centre = both(-m), scale = both(rs);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) v[r][e] = fma2(mul2(add2(v[r][e], centre), scale), w[e], b[e]);
        put_pairs<T, VEC, PACKS>(y + (r0 + r) * ld_y, width, lane, in, v[r]);
        if (lane == 0) { mean[r0 + r] = m; rstd[r0 + r] = rs; }
      }
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;
  }
}

template <typename T, int VEC, int PACKS, bool WARP>
__global__ void __launch_bounds__(WARP ? kWarpsPerCta * 32 : kGroupMax) ln_backward_kernel(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, int64_t rows, int cols,
                                                                                          Weight weight, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                                                          T* dx, int64_t ld_dx, float* __restrict__ parts) {
  constexpr int E = VEC * PACKS, R = rows_per_step(E * sizeof(T)), kStages = backward_stages(E * sizeof(T));
  constexpr bool kKeep = E < 32;
  extern __shared__ uint4 s_ring[];                              // WARP: afterwards [warps][2][cols] floats
  __shared__ float2 s_sum[2][R][16];
  const int width = WARP ? 32 : blockDim.x, lane = WARP ? threadIdx.x & 31 : threadIdx.x;
  const int64_t groups = WARP ? (int64_t)gridDim.x * kWarpsPerCta : gridDim.x;
  const int64_t group = WARP ? (int64_t)blockIdx.x * kWarpsPerCta + (threadIdx.x >> 5) : blockIdx.x;
  const float inv = 1.0f / (float)cols;
  uint32_t in = 0;                                               // packs that lie inside the row
#pragma unroll
  for (int k = 0; k < PACKS; ++k) if ((k * width + lane) * VEC < cols) in |= 1u << k;
  RowRing<T, VEC, PACKS, 2 * R, kStages> ring{reinterpret_cast<Pack<T, VEC>*>(s_ring) + threadIdx.x};
  const T *from_x = x + group * R * ld_x + lane * VEC, *from_dy = dy + group * R * ld_dy + lane * VEC;       // the next row to fetch
  int64_t fetched = group * R;
  auto fetch = [&](int stage) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int k = 0; k < PACKS; ++k) {
        if (fetched + r < rows && (in >> k & 1u)) {
          ring.put(stage, 2 * r, k, from_x + r * ld_x + k * width * VEC);
          ring.put(stage, 2 * r + 1, k, from_dy + r * ld_dy + k * width * VEC);
        }
      }
    }
    ring.close();
    from_x += groups * R * ld_x; from_dy += groups * R * ld_dy; fetched += groups * R;
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) fetch(i);
  uint64_t w[E / 2], dw[E / 2], db[E / 2];
  if constexpr (kKeep) get_weight<VEC, PACKS>(weight, width, lane, in, 1.0f, w);
#pragma unroll
  for (int e = 0; e < E / 2; ++e) { dw[e] = 0; db[e] = 0; }
  const int span = WARP ? 1 : warp_span(), mate = threadIdx.x & (span - 1);
  const bool other = mate < (int)(blockDim.x >> 5);
  int stage = 0, turn = 0;
  float next_mu[R], next_rs[R];
  auto stats = [&](int64_t r0) {
#pragma unroll
    for (int r = 0; r < R; ++r) { next_mu[r] = r0 + r < rows ? mean[r0 + r] : 0.0f; next_rs[r] = r0 + r < rows ? rstd[r0 + r] : 0.0f; }
  };
  stats(group * R);
  for (int64_t r0 = group * R; r0 < rows; r0 += groups * R, turn ^= 1) {
    float mu[R], rs[R];
    float2 s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) { mu[r] = next_mu[r]; rs[r] = next_rs[r]; }
    stats(r0 + groups * R);
    fetch(stage == 0 ? kStages - 1 : stage - 1);
    ring.wait();
    if constexpr (!kKeep) get_weight<VEC, PACKS>(weight, width, lane, in, 1.0f, w);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] = make_float2(0.0f, 0.0f);
      if (r0 + r >= rows) continue;
      uint64_t h[E / 2], d[E / 2], s1 = 0, s2 = 0;
      ring.get(stage, 2 * r, in, h); ring.get(stage, 2 * r + 1, in, d);            // (a column without a value has d = 0 and counts for nothing)
      const uint64_t centre = both(-mu[r]), scale = both(rs[r]);
#pragma unroll
      for (int e = 0; e < E / 2; ++e) {
        const uint64_t hat = mul2(add2(h[e], centre), scale), u = mul2(d[e], w[e]);
        s1 = add2(s1, u); s2 = fma2(u, hat, s2);
        dw[e] = fma2(d[e], hat, dw[e]); db[e] = add2(db[e], d[e]);
      }
      s[r] = make_float2(halves(s1), halves(s2));
    }
#pragma unroll
    for (int r = 0; r < R; ++r) { s[r].x = warp_sum(s[r].x); s[r].y = warp_sum(s[r].y); }
    if constexpr (!WARP) {
      if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) s_sum[turn][r][threadIdx.x >> 5] = s[r];
      }
      __syncthreads();
#pragma unroll
      for (int r = 0; r < R; ++r) {                               // a lane per warp
        const float2 q = other ? s_sum[turn][r][mate] : make_float2(0.0f, 0.0f);
        s[r] = make_float2(span_sum(q.x, span), span_sum(q.y, span));
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r0 + r < rows) {
        // rs (u - m1 - hat m2)
        const uint64_t centre = both(-mu[r]), scale = both(rs[r]), m1 = both(-rs[r] * (s[r].x * inv)), m2 = both(-rs[r] * (s[r].y * inv));
        uint64_t h[E / 2], d[E / 2];
        ring.get(stage, 2 * r, in, h); ring.get(stage, 2 * r + 1, in, d);          // again, rather than kept in registers
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          const uint64_t hat = mul2(add2(h[e], centre), scale), u = mul2(d[e], w[e]);
          d[e] = fma2(hat, m2, fma2(u, scale, m1));
        }
        put_pairs<T, VEC, PACKS>(dx + (r0 + r) * ld_dx, width, lane, in, d);
      }
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;
  }
  // this CTA's rows of partial sums: dw, then db
  float* part_w = parts + (int64_t)blockIdx.x * cols;
  float* part_b = parts + ((int64_t)gridDim.x + blockIdx.x) * cols;
  if constexpr (WARP) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();                                             // the ring is no longer read
    float* s_cols = reinterpret_cast<float*>(s_ring);
    float* mine = s_cols + (threadIdx.x >> 5) * 2 * cols;
    put_columns<VEC, PACKS>(mine, width, lane, in, dw);
    put_columns<VEC, PACKS>(mine + cols, width, lane, in, db);
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * cols; c += blockDim.x) {
      float t = 0.0f;
#pragma unroll
      for (int v = 0; v < kWarpsPerCta; ++v) t += s_cols[v * 2 * cols + c];
      if (c < cols) part_w[c] = t; else part_b[c - cols] = t;
    }
  } else {
    put_columns<VEC, PACKS>(part_w, width, lane, in, dw);
    put_columns<VEC, PACKS>(part_b, width, lane, in, db);
  }
}

// sums of the partial rows: 32 columns per CTA, 32 rows side by side
constexpr int kJoinRows = 32;
__global__ void __launch_bounds__(32 * kJoinRows) ln_join_kernel(const float* __restrict__ parts, int n, int cols, float* __restrict__ dweight, float* __restrict__ dbias) {
  __shared__ float s[kJoinRows][33];
  wait_for_previous();
  const int c = blockIdx.x * 32 + threadIdx.x;
  float* out = blockIdx.y == 0 ? dweight : dbias;
  float t = 0.0f;
  if (out && c < cols) {
    const float* p = parts + (int64_t)blockIdx.y * n * cols + c;
#pragma unroll 10
    for (int i = threadIdx.y; i < n; i += kJoinRows) t += p[(int64_t)i * cols];
  }
  s[threadIdx.y][threadIdx.x] = t;
  __syncthreads();
  // the 32 sums of a column by a warp
  t = warp_sum(s[threadIdx.x][threadIdx.y]);
  const int d = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && out && d < cols) out[d] = t;
}

// ---- rows longer than the registers hold ----------------------------------------------------------
constexpr int kLongThreads = 1024;
// sums of R values over the CTA (which meets once; s: R x 32 floats that nobody reads any more)
template <int R>
__device__ __forceinline__ void long_sum(float (&v)[R], float* s) {
#pragma unroll
  for (int r = 0; r < R; ++r) { v[r] = warp_sum(v[r]); if ((threadIdx.x & 31) == 0) s[r * 32 + (threadIdx.x >> 5)] = v[r]; }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) v[r] = warp_sum(s[r * 32 + (threadIdx.x & 31)]);
}
template <typename T>
__global__ void __launch_bounds__(kLongThreads) ln_forward_long_kernel(const T* x, int cols, int64_t ld, Weight weight, Weight bias, float eps,
                                                                       T* y, int64_t ld_y, float* __restrict__ mean, float* __restrict__ rstd) {
  __shared__ float s_sum[2][32];
  const int64_t row = blockIdx.x;
  const T* p = x + row * ld;
  float v[1] = {0.0f};
  for (int c = threadIdx.x; c < cols; c += kLongThreads) v[0] += to_float(p[c]);
  long_sum<1>(v, s_sum[0]);
  const float mu = v[0] / (float)cols;
  v[0] = 0.0f;
  for (int c = threadIdx.x; c < cols; c += kLongThreads) { const float d = to_float(p[c]) - mu; v[0] = fmaf(d, d, v[0]); }
  long_sum<1>(v, s_sum[1]);
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
  long_sum<2>(s, s_sum);
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
// bytes that a thread moves in one piece: 16 where base, leading dimension and length allow it, else 4, else a value
int pack_bytes(const void* p, int64_t ld, int64_t cols, int size) {
  for (int bytes = 16; bytes > size; bytes = bytes == 16 ? 4 : size)
    if (reinterpret_cast<uintptr_t>(p) % bytes == 0 && (ld * size) % bytes == 0 && (cols * size) % bytes == 0) return bytes;
  return size;
}
template <int VEC, int PACKS> struct Form { static constexpr int kVec = VEC, kPacks = PACKS; };
// Columns per thread: one pack where a warp then holds the row, else 16 (a warp up to 512 columns, CTAs of up to 512 threads from there), else 32.
template <typename T, int VEC, typename F> cudaError_t by_packs(int64_t cols, F f) {
  constexpr int kFew = VEC >= 4 ? VEC : 4;
  if (cols <= 32 * kFew) return f(Form<VEC, kFew / VEC>{});
  return cols <= kGroupMax * 16 ? f(Form<VEC, 16 / VEC>{}) : f(Form<VEC, 32 / VEC>{});
}
template <typename T, typename F> cudaError_t by_form(int bytes, int64_t cols, F f) {
  if (bytes == 16) return by_packs<T, 16 / (int)sizeof(T)>(cols, f);
  if constexpr (sizeof(T) == 2) { if (bytes == 4) return by_packs<T, 2>(cols, f); }
  return by_packs<T, 1>(cols, f);
}
// CTAs of a kernel that the GPU holds at a time, asked for once per number of warps (`known`: 0 before that)
int resident(const void* kernel, int threads, size_t smem, int (&known)[17]) {
  int& n = known[threads / 32];
  if (n == 0) {
    int per = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, threads, smem) != cudaSuccess) cudaGetLastError();
    n = 148 * std::max(per, 1);
  }
  return n;
}

template <typename T, int VEC, int PACKS>
cudaError_t forward_form(const NormForward& a, cudaStream_t st) {
  constexpr int kBytes = VEC * PACKS * (int)sizeof(T), R = rows_per_step(kBytes);
  const Weight w{a.weight, a.weight_type}, b{a.bias, a.weight_type};
  const bool warp = a.cols <= 32 * VEC * PACKS;
  const int threads = warp ? kWarpsPerCta * 32 : (int)((a.cols + 32 * VEC * PACKS - 1) / (32 * VEC * PACKS)) * 32;
  const int64_t step = warp ? kWarpsPerCta * R : R;
  const size_t smem = (size_t)forward_stages(kBytes) * R * threads * kBytes;
  static int known[2][17];
  const void* kernel = warp ? (const void*)ln_forward_kernel<T, VEC, PACKS, true> : (const void*)ln_forward_kernel<T, VEC, PACKS, false>;
  const int grid = (int)std::min<int64_t>((a.rows + step - 1) / step, resident(kernel, threads, smem, known[warp]));
  if (warp) ln_forward_kernel<T, VEC, PACKS, true><<<grid, threads, smem, st>>>((const T*)a.x, a.rows, (int)a.cols, a.ld, w, b, a.eps, (T*)a.y, a.ld_y, a.mean, a.rstd);
  else ln_forward_kernel<T, VEC, PACKS, false><<<grid, threads, smem, st>>>((const T*)a.x, a.rows, (int)a.cols, a.ld, w, b, a.eps, (T*)a.y, a.ld_y, a.mean, a.rstd);
  return cudaGetLastError();
}
template <typename T>
cudaError_t forward_type(const NormForward& a, cudaStream_t st) {
  if (a.cols > kNormCols) {
    ln_forward_long_kernel<T><<<(unsigned)a.rows, kLongThreads, 0, st>>>((const T*)a.x, (int)a.cols, a.ld, Weight{a.weight, a.weight_type}, Weight{a.bias, a.weight_type}, a.eps,
                                                                        (T*)a.y, a.ld_y, a.mean, a.rstd);
    return cudaGetLastError();
  }
  const int bytes = std::min(pack_bytes(a.x, a.ld, a.cols, sizeof(T)), pack_bytes(a.y, a.ld_y, a.cols, sizeof(T)));
  return by_form<T>(bytes, a.cols, [&](auto f) { return forward_form<T, decltype(f)::kVec, decltype(f)::kPacks>(a, st); });
}

int back_ctas(int64_t rows, int64_t per) { return (int)std::min<int64_t>((rows + per - 1) / per, kBackCtas); }

cudaError_t backward_join(const NormBackward& a, int n, cudaStream_t st) {
  if (!a.dweight && !a.dbias) return cudaSuccess;
  return launch_after(ln_join_kernel, dim3((unsigned)((a.cols + 31) / 32), 2), dim3(32, kJoinRows), 0, st, a.ws, n, (int)a.cols, a.dweight, a.dbias);
}
template <typename T, int VEC, int PACKS>
cudaError_t backward_form(const NormBackward& a, cudaStream_t st) {
  constexpr int kBytes = VEC * PACKS * (int)sizeof(T), R = rows_per_step(kBytes);
  const Weight w{a.weight, a.weight_type};
  const bool warp = a.cols <= 32 * VEC * PACKS;
  const int threads = warp ? kWarpsPerCta * 32 : (int)((a.cols + 32 * VEC * PACKS - 1) / (32 * VEC * PACKS)) * 32;
  const int64_t step = warp ? kWarpsPerCta * R : R;
  const size_t ring = (size_t)backward_stages(kBytes) * 2 * R * threads * kBytes;
  const size_t smem = warp ? std::max<size_t>(ring, (size_t)kWarpsPerCta * 2 * a.cols * 4) : ring;
  static int known[2][17];
  const void* kernel = warp ? (const void*)ln_backward_kernel<T, VEC, PACKS, true> : (const void*)ln_backward_kernel<T, VEC, PACKS, false>;
  const int grid = (int)std::min<int64_t>(back_ctas(a.rows, step), warp ? 148 * 2 : resident(kernel, threads, smem, known[warp]));
  if (warp) ln_backward_kernel<T, VEC, PACKS, true><<<grid, threads, smem, st>>>((const T*)a.dy, a.ld_dy, (const T*)a.x, a.ld_x, a.rows, (int)a.cols, w, a.mean, a.rstd, (T*)a.dx, a.ld_dx, a.ws);
  else ln_backward_kernel<T, VEC, PACKS, false><<<grid, threads, smem, st>>>((const T*)a.dy, a.ld_dy, (const T*)a.x, a.ld_x, a.rows, (int)a.cols, w, a.mean, a.rstd, (T*)a.dx, a.ld_dx, a.ws);
  const cudaError_t e = cudaGetLastError();
  return e != cudaSuccess ? e : backward_join(a, grid, st);
}
template <typename T>
cudaError_t backward_type(const NormBackward& a, cudaStream_t st) {
  if (a.rows == 0) return backward_join(a, 0, st);
  if (a.cols > kNormCols) {
    const Weight w{a.weight, a.weight_type};
    const int split = back_ctas(a.rows, 32);                     // first, since dx may lie where dy or x does
    ln_columns_kernel<T><<<dim3((unsigned)((a.cols + 255) / 256), split), 256, 0, st>>>((const T*)a.dy, a.ld_dy, (const T*)a.x, a.ld_x, a.rows, (int)a.cols, a.mean, a.rstd, a.ws);
    ln_backward_long_kernel<T><<<(unsigned)a.rows, kLongThreads, 0, st>>>((const T*)a.dy, a.ld_dy, (const T*)a.x, a.ld_x, (int)a.cols, w, a.mean, a.rstd, (T*)a.dx, a.ld_dx);
    const cudaError_t e = cudaGetLastError();
    return e != cudaSuccess ? e : backward_join(a, split, st);
  }
  const int bytes = std::min({pack_bytes(a.x, a.ld_x, a.cols, sizeof(T)), pack_bytes(a.dy, a.ld_dy, a.cols, sizeof(T)), pack_bytes(a.dx, a.ld_dx, a.cols, sizeof(T))});
  return by_form<T>(bytes, a.cols, [&](auto f) { return backward_form<T, decltype(f)::kVec, decltype(f)::kPacks>(a, st); });
}

}  // namespace

int layer_norm_configure() {
  cudaError_t e = cudaSuccess;
  auto each = [&](auto t) {
    using T = decltype(t);
    for (int bytes : {16, 4, (int)sizeof(T)})
      for (int64_t cols : {1, kGroupMax * 16, kNormCols})
        by_form<T>(bytes, cols, [&](auto f) {
          constexpr int VEC = decltype(f)::kVec, PACKS = decltype(f)::kPacks;
          auto room = [&](auto kernel) { if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024); };
          room(ln_forward_kernel<T, VEC, PACKS, true>); room(ln_forward_kernel<T, VEC, PACKS, false>);
          room(ln_backward_kernel<T, VEC, PACKS, true>); room(ln_backward_kernel<T, VEC, PACKS, false>);
          return e;
        });
  };
  each(float()); each(__nv_bfloat16()); each(__half());
  return (int)e;
}

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
