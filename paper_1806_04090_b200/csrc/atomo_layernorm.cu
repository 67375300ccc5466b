// Layer norm over the rows of a matrix, and its backward pass with the sums of the weight's and the bias's gradient.
//
//   y = h w + b,  h = (x - mean) rstd,  rstd = 1 / sqrt(var + eps)
//   dx = rstd (u - mean(u) - h mean(u h)),  u = dy w,     dw = sum over rows of dy h,  db = sum over rows of dy
//
// One pass over memory in either direction: a row stays on chip with one group of threads (a warp, or a CTA), each of which owns the
// same columns in every row that its group takes, so that the weights are loaded once and the sums of dw and db stay in registers
// too; the groups' sums are then added by a second kernel (of a few rows: inside a cluster), in a fixed order.  The rows to come are copied to shared memory meanwhile, by the threads that
// will use them, so that copies in flight take no registers and are waited for by their own thread alone; rows that are not aligned are copied in whole 16 bytes
// all the same and shared by the group.  A thread has up to 16 columns, two at a time in packed
// fp32: what a row costs every warp (shuffles, the exchange among warps) outweighs the arithmetic where a thread has few, and instruction issue then bounds
// the kernels instead of memory (2048 bf16 columns, 8 per thread: 33 instructions per element forward, 82 us for 32768 rows; as it is, 14 and 51 us, 5.3 TB/s,
// backward 23 and 82 us, 4.9 TB/s, of which the join is 4).
//   The variance is taken from the values centred on the warp's mean, and the warps' are combined as M2 = sum of M2_w + n_w (mean_w - mean)^2, which takes
// one exchange and loses nothing where the mean is far from zero.  All arithmetic is in fp32; y and dx are rounded to their type once.
// Rows of more than kNormCols columns do not fit: CTAs then read them again from L2.
#include <algorithm>
#include <atomic>

#include "atomo_ops.cuh"

namespace atomo {
namespace {

constexpr int kGroupMax = 512;                                   // threads per row, at most
constexpr int kNormCols = kGroupMax * 16;
constexpr int kCtaThreads = 256;                                 // of a CTA with several groups side by side
constexpr int kBackCtas = 148 * 4;                               // partial rows of dw and db, at most
constexpr int kMates = 8;                                        // CTAs of a cluster that adds them itself, at most
// By the bytes of a row that a thread has (up to 64): rows per step; steps whose rows are in shared memory or on the way there
constexpr int kForwardStages = 4, kBackwardStages = 3;
__host__ __device__ constexpr int rows_per_step(int bytes) { return bytes <= 32 ? 2 : 1; }

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

// sum over the lanes that differ in the bits below `span`, a power of two up to CTA / 32
template <int CTA> __device__ __forceinline__ float span_sum(float v, int span) {
#pragma unroll
  for (int o = 1; o < CTA / 32; o <<= 1) if (o < span) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// the threads of a group meet (barrier 0 is the whole CTA's)
__device__ __forceinline__ void meet(int group, int width) {
  if (width == 32) __syncwarp();
  else asm volatile("bar.sync %0, %1;" :: "r"(group + 1), "r"(width) : "memory");
}
// this thread's place: the group in its CTA, the thread in its group, the warp whose sums it takes in an exchange (if there is one)
struct Place {
  int width, group, lane, span, mate; bool other;
  __device__ __forceinline__ explicit Place(int width) : width(width), group(threadIdx.x / width), lane(threadIdx.x - group * width), span(1) {
    while (span * 32 < width) span <<= 1;
    const int at = threadIdx.x & (span - 1);
    other = at * 32 < width;
    mate = group * (width >> 5) + at;
  }
};
__device__ __forceinline__ void cluster_meet() { asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float4 remote_values(const float* p, int rank) {
  uint32_t a = (uint32_t)__cvta_generic_to_shared(p);
  float4 v;
  asm("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(a) : "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ float one_over_root(float x) {        // to about one unit in the last place; of zero Inf, of Inf zero
  const float r = rsqrtf(x), e = fmaf(-x * r, r, 1.0f);
  return e == e ? fmaf(r * 0.5f, e, r) : r;
}

// The rows that come next: STAGES steps of ROWS rows (x, or x and dy by turns) in shared memory, for a group of `width` threads of which this is `lane`.
// Aligned rows: a thread copies its own packs (of 16 bytes) and waits for nobody else's.  CTA: threads, at most.
template <typename T, int VEC, int PACKS, int ROWS, int STAGES, int CTA>
struct OwnRing {
  static constexpr bool kShared = false;
  static constexpr uint32_t kAll = (1u << PACKS) - 1u;
  Pack<T, VEC>* slot; int hop, at; uint32_t in;                  // hop: values between two packs of a thread
  __device__ __forceinline__ OwnRing(uint4* smem, int, int width, int lane, int, uint32_t in)
      : slot(reinterpret_cast<Pack<T, VEC>*>(smem) + threadIdx.x), hop(width * VEC), at(lane * VEC), in(in) {}
  static size_t bytes(int, int) { return (size_t)STAGES * ROWS * PACKS * CTA * 16; }
  __device__ __forceinline__ void put(int stage, int row, const T* p, const T*, const T*) {
    p += at;
    Pack<T, VEC>* to = slot + stage * (ROWS * PACKS * CTA);
#pragma unroll
    for (int k = 0; k < PACKS; ++k) if (in >> k & 1u) copy_async<16>(to + (row * PACKS + k) * CTA, p + k * hop);
  }
  __device__ __forceinline__ Pack<T, VEC> pack(int stage, int row, int k, uint32_t) const { return slot[stage * (ROWS * PACKS * CTA) + (row * PACKS + k) * CTA]; }
};
// Other rows: the group copies the 16 bytes that hold them, as far as they lie within the matrix (its first and last value are given), and all of it waits.
template <typename T, int VEC, int PACKS, int ROWS, int STAGES, int CTA>
struct SharedRing {
  static constexpr bool kShared = true;
  static constexpr uint32_t kAll = (1u << PACKS) - 1u;
  uint8_t* base; int width, lane, cols, pitch;
  static __host__ __device__ __forceinline__ int row_pitch(int cols) { return ((cols * (int)sizeof(T) + 15) / 16 + 1) * 16; }
  __device__ __forceinline__ SharedRing(uint4* smem, int group, int width, int lane, int cols, uint32_t)
      : width(width), lane(lane), cols(cols), pitch(row_pitch(cols)) { base = reinterpret_cast<uint8_t*>(smem) + (size_t)group * STAGES * ROWS * pitch; }
  static size_t bytes(int groups, int cols) { return (size_t)groups * STAGES * ROWS * row_pitch(cols); }
  __device__ __forceinline__ uint8_t* row_at(int stage, int row) const { return base + (stage * ROWS + row) * pitch; }
  __device__ __forceinline__ void put(int stage, int row, const T* p, const T* first, const T* last) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15, lo = reinterpret_cast<uintptr_t>(first), hi = reinterpret_cast<uintptr_t>(last + 1);
    const int n = (int)((reinterpret_cast<uintptr_t>(p + cols) - a + 15) >> 4);
    uint8_t* to = row_at(stage, row);
    for (int i = lane; i < n; i += width) {
      const uintptr_t from = a + (uintptr_t)i * 16;
      if (from >= lo && from + 16 <= hi) copy_async<16>(to + i * 16, reinterpret_cast<const void*>(from));
      else {
#pragma unroll
        for (int j = 0; j < 16; j += (int)sizeof(T))
          if (from + j >= lo && from + j < hi) *reinterpret_cast<T*>(to + i * 16 + j) = *reinterpret_cast<const T*>(from + j);
      }
    }
  }
  __device__ __forceinline__ Pack<T, VEC> pack(int stage, int row, int k, uint32_t low) const {
    return *reinterpret_cast<const Pack<T, VEC>*>(row_at(stage, row) + (low & 15u) + (k * width + lane) * VEC * (int)sizeof(T));
  }
};
template <typename T, int VEC, int PACKS, int ROWS, int STAGES, int CTA>
using Ring = typename std::conditional<VEC * sizeof(T) == 16, OwnRing<T, VEC, PACKS, ROWS, STAGES, CTA>, SharedRing<T, VEC, PACKS, ROWS, STAGES, CTA>>::type;

// the thread's columns of a row (the low bits of whose address in global memory are given), as pairs; zeros where it has none (in: a bit per pack)
__device__ __forceinline__ uint32_t low_of(const void* p) { return (uint32_t)reinterpret_cast<uintptr_t>(p); }
template <typename T, int VEC, int PACKS, typename R>
__device__ __forceinline__ void get_pairs(const R& ring, int stage, int row, uint32_t low, uint32_t in, uint64_t (&v)[VEC * PACKS / 2]) {
  if (in == R::kAll) {
#pragma unroll
    for (int k = 0; k < PACKS; k += VEC > 1 ? 1 : 2) {
      if constexpr (VEC > 1) {
        const Pack<T, VEC> raw = ring.pack(stage, row, k, low);
#pragma unroll
        for (int j = 0; j < VEC; j += 2) v[(k * VEC + j) / 2] = pair_of(raw.v + j);
      } else v[k / 2] = pack2(to_float(ring.pack(stage, row, k, low).v[0]), to_float(ring.pack(stage, row, k + 1, low).v[0]));
    }
  } else {
#pragma unroll
    for (int e = 0; e < VEC * PACKS / 2; ++e) v[e] = 0;
#pragma unroll
    for (int k = 0; k < PACKS; k += VEC > 1 ? 1 : 2) {
      if (!(in >> k & 1u)) break;                                 // (the packs that a thread has are its first ones)
      if constexpr (VEC > 1) {
        const Pack<T, VEC> raw = ring.pack(stage, row, k, low);
#pragma unroll
        for (int j = 0; j < VEC; j += 2) v[(k * VEC + j) / 2] = pair_of(raw.v + j);
      } else v[k / 2] = pack2(to_float(ring.pack(stage, row, k, low).v[0]), in >> (k + 1) & 1u ? to_float(ring.pack(stage, row, k + 1, low).v[0]) : 0.0f);
    }
  }
}
__device__ __forceinline__ void close_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" :: "n"(LEFT) : "memory"); }
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

// Columns of a thread: PACKS pieces of VEC neighbouring ones, a group's width apart.
template <typename T, int VEC, int PACKS, int CTA>
__global__ void __launch_bounds__(CTA, 512 / CTA) ln_forward_kernel(int group_width, const T* x, int64_t rows, int cols, int64_t ld, Weight weight, Weight bias,
                                                               float eps, T* y, int64_t ld_y, float* __restrict__ mean, float* __restrict__ rstd) {
  constexpr int E = VEC * PACKS, R = rows_per_step(E * sizeof(T)), kStages = kForwardStages;
  extern __shared__ uint4 s_ring[];
  __shared__ float2 s_sum[2][R][16];
  __shared__ float s_count[16];
  const Place at(group_width);
  const int width = at.width, lane = at.lane, beside = blockDim.x / width;
  const int ahead = gridDim.x * beside * R, first = ((int)blockIdx.x * beside + at.group) * R;        // rows between two steps; the first one
  const float inv = 1.0f / (float)cols;
  uint32_t in = 0;                                               // packs that lie inside the row
#pragma unroll
  for (int k = 0; k < PACKS; ++k) if ((k * width + lane) * VEC < cols) in |= 1u << k;
  using Rows = Ring<T, VEC, PACKS, R, kStages, CTA>;
  const bool full = in == Rows::kAll;
  Rows ring(s_ring, at.group, width, lane, cols, in);
  const int64_t step = ahead * ld, step_y = ahead * ld_y;
  const T *from = x + first * ld, *last = x + (rows - 1) * ld + cols - 1;          // the next rows to fetch; the matrix's last value
  int left = (int)rows - first;                                  // rows from there on
  auto fetch = [&](int stage) {
#pragma unroll
    for (int r = 0; r < R; ++r) if (r < left) ring.put(stage, r, from + r * ld, x, last);
    close_copies();
    from += step; left -= ahead;
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) fetch(i);
  uint64_t w[E / 2], b[E / 2];
  get_weight<VEC, PACKS>(weight, width, lane, in, 1.0f, w);
  get_weight<VEC, PACKS>(bias, width, lane, in, 0.0f, b);
  const float count = warp_sum((float)(__popc(in) * VEC)), inv_count = 1.0f / count;       // columns of this warp
  float mate_count = 0.0f, mate_inv = 0.0f;                      // columns of the warp whose sums this lane takes
  if ((threadIdx.x & 31) == 0) s_count[threadIdx.x >> 5] = count;
  __syncthreads();
  if (at.other) { mate_count = s_count[at.mate]; mate_inv = 1.0f / mate_count; }
  int stage = 0, turn = 0;
  uint32_t low = low_of(x + first * ld);
  T* to = y + first * ld_y;
  for (int r0 = first; r0 < (int)rows; r0 += ahead, turn ^= 1) {
    if constexpr (Rows::kShared) { wait_copies<kStages - 2>(); meet(at.group, width); }       // the copies of the whole group; nobody reads the step before any more
    fetch(stage == 0 ? kStages - 1 : stage - 1);
    if constexpr (!Rows::kShared) wait_copies<kStages - 1>();
    uint64_t v[R][E / 2];
    float mu[R], var[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r0 + r < (int)rows) get_pairs<T, VEC, PACKS>(ring, stage, r, low + r * (uint32_t)ld * (uint32_t)sizeof(T), in, v[r]);
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
    if (width > 32) {
      if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) s_sum[turn][r][threadIdx.x >> 5] = make_float2(mu[r], var[r]);
      }
      meet(at.group, width);
#pragma unroll
      for (int r = 0; r < R; ++r) {                               // a lane per warp
        const float2 q = at.other ? s_sum[turn][r][at.mate] : make_float2(0.0f, 0.0f);
        mu[r] = span_sum<CTA>(q.x, at.span);
        const float d = fmaf(-mu[r], inv, q.x * mate_inv);
        var[r] = span_sum<CTA>(fmaf(mate_count * d, d, q.y), at.span);
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r0 + r < (int)rows) {
        const float m = mu[r] * inv, rs = one_over_root(fmaf(var[r], inv, eps));
        const uint64_t centre = both(-m), scale = both(rs);
#pragma unroll
        for (int e = 0; e < E / 2; ++e) v[r][e] = fma2(mul2(add2(v[r][e], centre), scale), w[e], b[e]);
        put_pairs<T, VEC, PACKS>(to + r * ld_y, width, lane, in, v[r]);
        if (lane == 0) { mean[r0 + r] = m; rstd[r0 + r] = rs; }
      }
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;
    low += (uint32_t)step * (uint32_t)sizeof(T); to += step_y;
  }
}

template <typename T, int VEC, int PACKS, int CTA>
__global__ void __launch_bounds__(CTA, 512 / CTA) ln_backward_kernel(int group_width, const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, int64_t rows, int cols,
                                                                Weight weight, const float* __restrict__ mean, const float* __restrict__ rstd,
                                                                T* dx, int64_t ld_dx, float* __restrict__ parts_w, float* __restrict__ parts_b, int mates) {
  constexpr int E = VEC * PACKS, R = rows_per_step(E * sizeof(T)), kStages = kBackwardStages;
  extern __shared__ uint4 s_ring[];                              // afterwards, of several groups: [groups][2][cols] floats
  __shared__ float2 s_sum[2][R][16];
  const Place at(group_width);
  const int width = at.width, lane = at.lane, beside = blockDim.x / width;
  const int ahead = gridDim.x * beside * R, first = ((int)blockIdx.x * beside + at.group) * R;        // rows between two steps; the first one
  const float inv = 1.0f / (float)cols;
  uint32_t in = 0;                                               // packs that lie inside the row
#pragma unroll
  for (int k = 0; k < PACKS; ++k) if ((k * width + lane) * VEC < cols) in |= 1u << k;
  using Rows = Ring<T, VEC, PACKS, 2 * R, kStages, CTA>;
  Rows ring(s_ring, at.group, width, lane, cols, in);
  const int64_t step_x = ahead * ld_x, step_dy = ahead * ld_dy, step_dx = ahead * ld_dx;
  const T *from_x = x + first * ld_x, *from_dy = dy + first * ld_dy;               // the next rows to fetch
  const T *last_x = x + (rows - 1) * ld_x + cols - 1, *last_dy = dy + (rows - 1) * ld_dy + cols - 1;
  int left = (int)rows - first;                                  // rows from there on
  auto fetch = [&](int stage) {
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (r < left) { ring.put(stage, 2 * r, from_x + r * ld_x, x, last_x); ring.put(stage, 2 * r + 1, from_dy + r * ld_dy, dy, last_dy); }
    close_copies();
    from_x += step_x; from_dy += step_dy; left -= ahead;
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) fetch(i);
  uint64_t w[E / 2], dw[E / 2], db[E / 2];
  get_weight<VEC, PACKS>(weight, width, lane, in, 1.0f, w);
#pragma unroll
  for (int e = 0; e < E / 2; ++e) { dw[e] = 0; db[e] = 0; }
  int stage = 0, turn = 0;
  float next_mu[R], next_rs[R];
  auto stats = [&](int r0) {
#pragma unroll
    for (int r = 0; r < R; ++r) { next_mu[r] = r0 + r < (int)rows ? mean[r0 + r] : 0.0f; next_rs[r] = r0 + r < (int)rows ? rstd[r0 + r] : 0.0f; }
  };
  stats(first);
  uint32_t low_x = low_of(x + first * ld_x), low_dy = low_of(dy + first * ld_dy);
  T* to = dx + first * ld_dx;
  for (int r0 = first; r0 < (int)rows; r0 += ahead, turn ^= 1) {
    float mu[R], rs[R];
    float2 s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) { mu[r] = next_mu[r]; rs[r] = next_rs[r]; }
    stats(r0 + ahead);
    if constexpr (Rows::kShared) { wait_copies<kStages - 2>(); meet(at.group, width); }
    fetch(stage == 0 ? kStages - 1 : stage - 1);
    if constexpr (!Rows::kShared) wait_copies<kStages - 1>();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      s[r] = make_float2(0.0f, 0.0f);
      if (r0 + r >= (int)rows) continue;
      uint64_t h[E / 2], d[E / 2], s1 = 0, s2 = 0;
      get_pairs<T, VEC, PACKS>(ring, stage, 2 * r, low_x + r * (uint32_t)ld_x * (uint32_t)sizeof(T), in, h);
      get_pairs<T, VEC, PACKS>(ring, stage, 2 * r + 1, low_dy + r * (uint32_t)ld_dy * (uint32_t)sizeof(T), in, d);            // (a column without a value has d = 0 and counts for nothing)
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
    if (width > 32) {
      if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) s_sum[turn][r][threadIdx.x >> 5] = s[r];
      }
      meet(at.group, width);
#pragma unroll
      for (int r = 0; r < R; ++r) {                               // a lane per warp
        const float2 q = at.other ? s_sum[turn][r][at.mate] : make_float2(0.0f, 0.0f);
        s[r] = make_float2(span_sum<CTA>(q.x, at.span), span_sum<CTA>(q.y, at.span));
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r0 + r < (int)rows) {
        // rs (u - m1 - hat m2)
        const uint64_t centre = both(-mu[r]), scale = both(rs[r]), m1 = both(-rs[r] * (s[r].x * inv)), m2 = both(-rs[r] * (s[r].y * inv));
        uint64_t h[E / 2], d[E / 2];
        get_pairs<T, VEC, PACKS>(ring, stage, 2 * r, low_x + r * (uint32_t)ld_x * (uint32_t)sizeof(T), in, h);
        get_pairs<T, VEC, PACKS>(ring, stage, 2 * r + 1, low_dy + r * (uint32_t)ld_dy * (uint32_t)sizeof(T), in, d);          // again, rather than kept in registers
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          const uint64_t hat = mul2(add2(h[e], centre), scale), u = mul2(d[e], w[e]);
          d[e] = fma2(hat, m2, fma2(u, scale, m1));
        }
        put_pairs<T, VEC, PACKS>(to + r * ld_dx, width, lane, in, d);
      }
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;
    low_x += (uint32_t)step_x * (uint32_t)sizeof(T); low_dy += (uint32_t)step_dy * (uint32_t)sizeof(T); to += step_dx;
  }
  // the columns' sums.  Of one CTA, or of a cluster of `mates` that adds them through distributed shared memory: the results; else this CTA's rows of partial sums
  const int64_t row = mates > 1 ? 0 : (int64_t)blockIdx.x * cols;
  float* part_w = parts_w ? parts_w + row : nullptr;             // (null: a result that is not asked for)
  float* part_b = parts_b ? parts_b + row : nullptr;
  if (beside > 1 || mates > 1) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();                                             // the ring is no longer read
    float* s_cols = reinterpret_cast<float*>(s_ring);
    float* mine = s_cols + at.group * 2 * cols;
    put_columns<VEC, PACKS>(mine, width, lane, in, dw);
    put_columns<VEC, PACKS>(mine + cols, width, lane, in, db);
    __syncthreads();
    auto put = [&](int c, float t) {
      float* part = c < cols ? part_w : part_b;
      if (part) part[c < cols ? c : c - cols] = t;
    };
    if (beside > 1) {
      for (int c = threadIdx.x; c < 2 * cols; c += blockDim.x) {
        float t = 0.0f;
        for (int v = 0; v < beside; ++v) t += s_cols[v * 2 * cols + c];
        if (mates > 1) s_cols[c] = t; else put(c, t);
      }
    }
    if (mates > 1) {
      cluster_meet();
      for (int c = (blockIdx.x * blockDim.x + threadIdx.x) * 4; c < 2 * cols; c += mates * blockDim.x * 4) {
        float4 v[kMates];
#pragma unroll
        for (int k = 0; k < kMates; ++k) if (k < mates) v[k] = remote_values(s_cols + c, k);          // (all on their way at a time)
        float4 t = v[0];
#pragma unroll
        for (int k = 1; k < kMates; ++k) if (k < mates) { t.x += v[k].x; t.y += v[k].y; t.z += v[k].z; t.w += v[k].w; }
        const float f[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) if (c + e < 2 * cols) put(c + e, f[e]);
      }
      cluster_meet();                                            // nobody leaves while its shared memory is read
    }
  } else {
    if (part_w) put_columns<VEC, PACKS>(part_w, width, lane, in, dw);
    if (part_b) put_columns<VEC, PACKS>(part_b, width, lane, in, db);
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
constexpr int kLongThreads = 512;
// sums of R values over the CTA (which meets once; s: R x 32 floats that nobody reads any more)
template <int R>
__device__ __forceinline__ void long_sum(float (&v)[R], float* s) {
#pragma unroll
  for (int r = 0; r < R; ++r) { v[r] = warp_sum(v[r]); if ((threadIdx.x & 31) == 0) s[r * 32 + (threadIdx.x >> 5)] = v[r]; }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) v[r] = warp_sum((threadIdx.x & 31) < kLongThreads / 32 ? s[r * 32 + (threadIdx.x & 31)] : 0.0f);
}
// (VEC columns at a time: 16 bytes where the rows allow it)
template <typename T, int VEC>
__global__ void __launch_bounds__(kLongThreads) ln_forward_long_kernel(const T* x, int cols, int64_t ld, Weight weight, Weight bias, float eps, T* y, int64_t ld_y, float* mean, float* rstd) {
  __shared__ float s_sum[2][32];
  const int64_t row = blockIdx.x;
  const T* p = x + row * ld;
  float v[1] = {0.0f};
#pragma unroll 4
  for (int c = threadIdx.x * VEC; c < cols; c += kLongThreads * VEC) {
    const Pack<T, VEC> q = load_pack<T, VEC>(p + c);
#pragma unroll
    for (int j = 0; j < VEC; ++j) v[0] += to_float(q.v[j]);
  }
  long_sum<1>(v, s_sum[0]);
  const float mu = v[0] / (float)cols;
  v[0] = 0.0f;
#pragma unroll 4
  for (int c = threadIdx.x * VEC; c < cols; c += kLongThreads * VEC) {
    const Pack<T, VEC> q = load_pack<T, VEC>(p + c);
#pragma unroll
    for (int j = 0; j < VEC; ++j) { const float d = to_float(q.v[j]) - mu; v[0] = fmaf(d, d, v[0]); }
  }
  long_sum<1>(v, s_sum[1]);
  const float rs = one_over_root(v[0] / (float)cols + eps);
#pragma unroll 2
  for (int c = threadIdx.x * VEC; c < cols; c += kLongThreads * VEC) {
    Pack<T, VEC> q = load_pack<T, VEC>(p + c);
#pragma unroll
    for (int j = 0; j < VEC; ++j) q.v[j] = from_float<T>(fmaf((to_float(q.v[j]) - mu) * rs, weight_at(weight, c + j, 1.0f), weight_at(bias, c + j, 0.0f)));
    store_pack<T, VEC>(y + row * ld_y + c, q);
  }
  if (threadIdx.x == 0) { mean[row] = mu; rstd[row] = rs; }
}

template <typename T, int VEC>
__global__ void __launch_bounds__(kLongThreads) ln_backward_long_kernel(const T* dy, int64_t ld_dy, const T* x, int64_t ld_x, int cols, Weight weight, const float* mean, const float* rstd,
                                                                        T* dx, int64_t ld_dx) {
  __shared__ float s_sum[2 * 32];
  const int64_t row = blockIdx.x;
  const float mu = mean[row], rs = rstd[row];
  float s[2] = {0.0f, 0.0f};
#pragma unroll 2
  for (int c = threadIdx.x * VEC; c < cols; c += kLongThreads * VEC) {
    const Pack<T, VEC> d = load_pack<T, VEC>(dy + row * ld_dy + c), q = load_pack<T, VEC>(x + row * ld_x + c);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const float u = to_float(d.v[j]) * weight_at(weight, c + j, 1.0f), hat = (to_float(q.v[j]) - mu) * rs;
      s[0] += u; s[1] = fmaf(u, hat, s[1]);
    }
  }
  long_sum<2>(s, s_sum);
  const float m1 = s[0] / (float)cols, m2 = s[1] / (float)cols;
#pragma unroll 2
  for (int c = threadIdx.x * VEC; c < cols; c += kLongThreads * VEC) {
    Pack<T, VEC> d = load_pack<T, VEC>(dy + row * ld_dy + c);
    const Pack<T, VEC> q = load_pack<T, VEC>(x + row * ld_x + c);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const float u = to_float(d.v[j]) * weight_at(weight, c + j, 1.0f), hat = (to_float(q.v[j]) - mu) * rs;
      d.v[j] = from_float<T>(rs * (u - m1 - hat * m2));
    }
    store_pack<T, VEC>(dx + row * ld_dx + c, d);
  }
}
constexpr int kLongRows = 32;                                    // of a partial sum, at least
// partial sums of dw and db: a CTA takes 256 VEC columns of every gridDim.y-th row
template <typename T, int VEC>
__global__ void __launch_bounds__(256) ln_columns_kernel(const T* __restrict__ dy, int64_t ld_dy, const T* __restrict__ x, int64_t ld_x, int64_t rows, int cols,
                                                         const float* __restrict__ mean, const float* __restrict__ rstd, float* __restrict__ parts) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * VEC;
  if (c >= cols) return;
  float w[VEC], b[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) { w[j] = 0.0f; b[j] = 0.0f; }
#pragma unroll 4
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
    const Pack<T, VEC> d = load_pack<T, VEC>(dy + r * ld_dy + c), q = load_pack<T, VEC>(x + r * ld_x + c);
    const float mu = mean[r], rs = rstd[r];
#pragma unroll
    for (int j = 0; j < VEC; ++j) { w[j] = fmaf(to_float(d.v[j]), (to_float(q.v[j]) - mu) * rs, w[j]); b[j] += to_float(d.v[j]); }
  }
#pragma unroll
  for (int j = 0; j < VEC; ++j) { parts[(int64_t)blockIdx.y * cols + c + j] = w[j]; parts[((int64_t)gridDim.y + blockIdx.y) * cols + c + j] = b[j]; }
}

// ---- choice of form -------------------------------------------------------------------------------
// bytes that a thread moves in one piece: 16 where base, leading dimension and length allow it, else 4, else a value
int pack_bytes(const void* p, int64_t ld, int64_t cols, int size) {
  for (int bytes = 16; bytes > size; bytes = bytes == 16 ? 4 : size)
    if (reinterpret_cast<uintptr_t>(p) % bytes == 0 && (ld * size) % bytes == 0 && (cols * size) % bytes == 0) return bytes;
  return size;
}
template <int VEC, int PACKS> struct Form { static constexpr int kVec = VEC, kPacks = PACKS; };
// Columns per thread: one pack where a warp then holds the row, else 16 (a warp up to 512 columns, CTAs of up to 512 threads from there).
template <typename T, int VEC, typename F> cudaError_t by_packs(int64_t cols, F f) {
  constexpr int kFew = VEC >= 4 ? VEC : 4;
  if (cols <= 32 * kFew) return f(Form<VEC, kFew / VEC>{});
  return f(Form<VEC, 16 / VEC>{});
}
template <typename T, typename F> cudaError_t by_form(int bytes, int64_t cols, F f) {
  if (bytes == 16) return by_packs<T, 16 / (int)sizeof(T)>(cols, f);
  if constexpr (sizeof(T) == 2) { if (bytes == 4) return by_packs<T, 2>(cols, f); }
  return by_packs<T, 1>(cols, f);
}
// CTAs of a kernel that the GPU holds at a time.  What its registers allow is asked for once per number of warps (`known`: 0 before that); then what shared
// memory does, 227 KB of it with 1 KB for each CTA and what it has besides the ring.
int resident(const void* kernel, int threads, size_t smem, std::atomic<int> (&known)[17]) {
  int n = known[threads / 32].load(std::memory_order_relaxed);
  if (n == 0) {
    int per = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, threads, 0) != cudaSuccess) cudaGetLastError();
    n = std::max(per, 1);
    known[threads / 32].store(n, std::memory_order_relaxed);
  }
  return 148 * std::max(1, std::min(n, (int)(227 * 1024 / (smem + 2048))));
}

// threads of a group (the same whatever the type: 16 columns each, or a warp), of a CTA
struct Shape { int width, threads; };
Shape shape_of(int64_t cols) {
  const int width = (int)((cols + 511) / 512) * 32;
  return Shape{width, width <= kCtaThreads ? kCtaThreads / width * width : width};
}
// A backward pass in one launch, by a cluster whose CTAs add the columns' sums themselves: while each takes about a step (narrow rows: four).  Without the second
// launch and the workspace a call takes 3.7 us less of the host; kernels, us, one | two launches: 250 x 64 bf16 4.9 | 4.3, 32 x 1023 fp32 8.0 | 7.8, 8 x 4096 fp32 5.9 | 6.4,
// 8 x 8192 bf16 10 | 21 (there by one CTA, four steps); more rows: 250 x 512 fp32 8.4 | 5.4, 128 x 1023 fp32 16 | 8.
bool one_launch(int64_t rows, int64_t cols) {
  if (cols > kNormCols) return false;
  const Shape s = shape_of(cols);
  return rows <= (int64_t)kMates * (cols <= 128 ? 4 : 1) * (s.threads / s.width);
}

template <typename T, int VEC, int PACKS, int CTA>
cudaError_t forward_cta(const NormForward& a, Shape s, cudaStream_t st) {
  constexpr int R = rows_per_step(VEC * PACKS * (int)sizeof(T));
  const int64_t step = (int64_t)s.threads / s.width * R;         // rows of a CTA's step
  const size_t smem = Ring<T, VEC, PACKS, R, kForwardStages, CTA>::bytes(s.threads / s.width, (int)a.cols);
  static std::atomic<int> known[17];
  const int grid = (int)std::min<int64_t>((a.rows + step - 1) / step, resident((const void*)ln_forward_kernel<T, VEC, PACKS, CTA>, s.threads, smem, known));
  ln_forward_kernel<T, VEC, PACKS, CTA><<<grid, s.threads, smem, st>>>(s.width, (const T*)a.x, a.rows, (int)a.cols, a.ld, Weight{a.weight, a.weight_type}, Weight{a.bias, a.weight_type}, a.eps,
                                                                       (T*)a.y, a.ld_y, a.mean, a.rstd);
  return cudaGetLastError();
}
template <typename T, int VEC, int PACKS>
cudaError_t forward_form(const NormForward& a, cudaStream_t st) {
  const Shape s = shape_of(a.cols);
  if constexpr (VEC * PACKS == 16) { if (s.threads > kCtaThreads) return forward_cta<T, VEC, PACKS, kGroupMax>(a, s, st); }
  return forward_cta<T, VEC, PACKS, kCtaThreads>(a, s, st);
}
template <typename T>
cudaError_t forward_type(const NormForward& a, cudaStream_t st) {
  const int bytes = std::min(pack_bytes(a.x, a.ld, a.cols, sizeof(T)), pack_bytes(a.y, a.ld_y, a.cols, sizeof(T)));
  if (a.cols > kNormCols) {
    auto launch = [&](auto kernel) {
      kernel<<<(unsigned)a.rows, kLongThreads, 0, st>>>((const T*)a.x, (int)a.cols, a.ld, Weight{a.weight, a.weight_type}, Weight{a.bias, a.weight_type}, a.eps, (T*)a.y, a.ld_y, a.mean, a.rstd);
    };
    if (bytes == 16) launch(ln_forward_long_kernel<T, 16 / sizeof(T)>); else launch(ln_forward_long_kernel<T, 1>);
    return cudaGetLastError();
  }
  return by_form<T>(bytes, a.cols, [&](auto f) { return forward_form<T, decltype(f)::kVec, decltype(f)::kPacks>(a, st); });
}

int back_ctas(int64_t rows, int64_t per) { return (int)std::min<int64_t>((rows + per - 1) / per, kBackCtas); }

cudaError_t backward_join(const NormBackward& a, int n, cudaStream_t st) {
  if (!a.dweight && !a.dbias) return cudaSuccess;
  return launch_after(ln_join_kernel, dim3((unsigned)((a.cols + 31) / 32), 2), dim3(32, kJoinRows), 0, st, a.ws, n, (int)a.cols, a.dweight, a.dbias);
}
template <typename T, int VEC, int PACKS, int CTA>
cudaError_t backward_cta(const NormBackward& a, Shape s, cudaStream_t st) {
  constexpr int R = rows_per_step(VEC * PACKS * (int)sizeof(T));
  const int beside = s.threads / s.width;
  const size_t smem = std::max<size_t>(Ring<T, VEC, PACKS, 2 * R, kBackwardStages, CTA>::bytes(beside, (int)a.cols), (size_t)beside * 2 * a.cols * 4 + 16);       // (sums are read four at a time)
  static std::atomic<int> known[17];
  auto launch = [&](int grid, int mates, float* w, float* b) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = mates; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid); cfg.blockDim = dim3(s.threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cfg.attrs = attr; cfg.numAttrs = mates > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, ln_backward_kernel<T, VEC, PACKS, CTA>, s.width, (const T*)a.dy, a.ld_dy, (const T*)a.x, a.ld_x, a.rows, (int)a.cols,
                              Weight{a.weight, a.weight_type}, a.mean, a.rstd, (T*)a.dx, a.ld_dx, w, b, mates);
  };
  if (one_launch(a.rows, a.cols)) {
    const int mates = (int)std::min<int64_t>((a.rows + beside * R - 1) / (beside * R), kMates);
    return launch(mates, mates, a.dweight, a.dbias);
  }
  const int grid = std::min(back_ctas(a.rows, (int64_t)beside * R), resident((const void*)ln_backward_kernel<T, VEC, PACKS, CTA>, s.threads, smem, known));
  const cudaError_t e = launch(grid, 1, a.ws, a.ws + (int64_t)grid * a.cols);
  return e != cudaSuccess ? e : backward_join(a, grid, st);
}
template <typename T, int VEC, int PACKS>
cudaError_t backward_form(const NormBackward& a, cudaStream_t st) {
  const Shape s = shape_of(a.cols);
  if constexpr (VEC * PACKS == 16) { if (s.threads > kCtaThreads) return backward_cta<T, VEC, PACKS, kGroupMax>(a, s, st); }
  return backward_cta<T, VEC, PACKS, kCtaThreads>(a, s, st);
}
template <typename T>
cudaError_t backward_type(const NormBackward& a, cudaStream_t st) {
  if (a.rows == 0) return backward_join(a, 0, st);
  const int bytes = std::min({pack_bytes(a.x, a.ld_x, a.cols, sizeof(T)), pack_bytes(a.dy, a.ld_dy, a.cols, sizeof(T)), pack_bytes(a.dx, a.ld_dx, a.cols, sizeof(T))});
  if (a.cols > kNormCols) {
    const int split = back_ctas(a.rows, kLongRows);              // first, since dx may lie where dy or x does
    auto launch = [&](auto columns, auto kernel, int vec) {
      columns<<<dim3((unsigned)((a.cols + 256 * vec - 1) / (256 * vec)), split), 256, 0, st>>>((const T*)a.dy, a.ld_dy, (const T*)a.x, a.ld_x, a.rows, (int)a.cols, a.mean, a.rstd, a.ws);
      kernel<<<(unsigned)a.rows, kLongThreads, 0, st>>>((const T*)a.dy, a.ld_dy, (const T*)a.x, a.ld_x, (int)a.cols, Weight{a.weight, a.weight_type}, a.mean, a.rstd, (T*)a.dx, a.ld_dx);
    };
    if (bytes == 16) launch(ln_columns_kernel<T, 16 / sizeof(T)>, ln_backward_long_kernel<T, 16 / sizeof(T)>, 16 / (int)sizeof(T));
    else launch(ln_columns_kernel<T, 1>, ln_backward_long_kernel<T, 1>, 1);
    const cudaError_t e = cudaGetLastError();
    return e != cudaSuccess ? e : backward_join(a, split, st);
  }
  return by_form<T>(bytes, a.cols, [&](auto f) { return backward_form<T, decltype(f)::kVec, decltype(f)::kPacks>(a, st); });
}

}  // namespace

int layer_norm_configure() {
  cudaError_t e = cudaSuccess;
  auto each = [&](auto t) {
    using T = decltype(t);
    for (int bytes : {16, 4, (int)sizeof(T)})
      for (int64_t cols : {1, kNormCols})
        by_form<T>(bytes, cols, [&](auto f) {
          constexpr int VEC = decltype(f)::kVec, PACKS = decltype(f)::kPacks;
          auto room = [&](auto kernel) { if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024); };
          room(ln_forward_kernel<T, VEC, PACKS, kCtaThreads>); room(ln_backward_kernel<T, VEC, PACKS, kCtaThreads>);
          if constexpr (VEC * PACKS == 16) { room(ln_forward_kernel<T, VEC, PACKS, kGroupMax>); room(ln_backward_kernel<T, VEC, PACKS, kGroupMax>); }
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

uint64_t layer_norm_workspace(int64_t rows, int64_t cols) {
  if (one_launch(rows, cols)) return 0;
  const int parts = cols > kNormCols ? back_ctas(rows, kLongRows) : (int)std::min<int64_t>(rows, kBackCtas);
  return (uint64_t)parts * 2 * cols * 4;
}

int launch_layer_norm_backward(const NormBackward& a, cudaStream_t st) {
  if (a.type == ATOMO_TYPE_F32) return (int)backward_type<float>(a, st);
  if (a.type == ATOMO_TYPE_BF16) return (int)backward_type<__nv_bfloat16>(a, st);
  return (int)backward_type<__half>(a, st);
}

}  // namespace atomo
