// The parameter update behind the gradient exchange: global norm of a list of gradients, AdamW over a list of parameters.
//
// Both are one pass over memory.  The tensors of a call travel as kernel arguments (up to 32 KB of them), so that a call needs no table
// in device memory; a CTA finds the tensor of its chunk by bisection over the tensors' first chunks.
#include <algorithm>

#include "atomo_ops.cuh"

namespace atomo {
namespace {

// =================================== norm ========================================================
// sqrt(sum g^2).  Squares are summed in fp32 over the 16 or 32 values that a thread has in registers and in fp64 from there on.  Where
// such a sum is not well inside the range of fp32 (values around 1e19 or 1e-14 and beyond, all of them zero, NaN or Inf) it is
// formed again in fp64 from the registers: the norm neither overflows nor loses small gradients.  (It is right to 17 half-units: up to 32 fused sums
// in fp32, halved by the root, and the result's own rounding.)
// 133M fp32 values (534 MB): 83 us, 6.4 TB/s, what a copy reaches.  Up to 1 MB goes through one cluster of up to eight CTAs: one launch, 4 us.
constexpr int kNormThreads = 256, kNormLoads = 4;
constexpr int kNormChunk = kNormThreads * kNormLoads * 16;     // bytes per step of a CTA
constexpr int kNormCluster = 8;

struct NormTensor { const uint8_t* data; int64_t n; uint32_t chunk0; int32_t type; };   // chunk0: first chunk in the launch
template <int N> struct NormBatch {
  NormTensor t[N];
  int n; uint32_t chunks; int slot0;
  double max_norm; double* slots; float* out;
};

__device__ __forceinline__ void square_pair(uint32_t w, int type, float& a, float& b) {
  if (type == ATOMO_TYPE_BF16) { a = __uint_as_float(w << 16); b = __uint_as_float(w & 0xffff0000u); }
  else { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w)); a = f.x; b = f.y; }
}
__device__ __forceinline__ bool sum_holds(float s) { return s > 1.0e-27f && s < 1.0e37f; }

__device__ __forceinline__ double norm_value(const NormTensor& t, int64_t i) {
  if (t.type == ATOMO_TYPE_F32) return (double)reinterpret_cast<const float*>(t.data)[i];
  if (t.type == ATOMO_TYPE_BF16) return (double)to_float(reinterpret_cast<const __nv_bfloat16*>(t.data)[i]);
  return (double)to_float(reinterpret_cast<const __half*>(t.data)[i]);
}

// squares of what a thread holds of one chunk; zeros count for nothing
__device__ __forceinline__ double norm_chunk(const uint4 (&r)[kNormLoads], int type) {
  float s = 0.0f;
  if (type == ATOMO_TYPE_F32) {
#pragma unroll
    for (int j = 0; j < kNormLoads; ++j) {
      const float* f = reinterpret_cast<const float*>(&r[j]);
#pragma unroll
      for (int k = 0; k < 4; ++k) s = fmaf(f[k], f[k], s);
    }
  } else {
#pragma unroll
    for (int j = 0; j < kNormLoads; ++j) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(&r[j]);
#pragma unroll
      for (int k = 0; k < 4; ++k) { float a, b; square_pair(w[k], type, a, b); s = fmaf(a, a, s); s = fmaf(b, b, s); }
    }
  }
  if (sum_holds(s)) return (double)s;
  double d = 0.0;
#pragma unroll
  for (int j = 0; j < kNormLoads; ++j) {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&r[j]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float a = __uint_as_float(w[k]), b = 0.0f;
      if (type != ATOMO_TYPE_F32) square_pair(w[k], type, a, b);
      d = fma((double)a, (double)a, d); d = fma((double)b, (double)b, d);
    }
  }
  return d;
}

__device__ __forceinline__ void norm_finish(double sum, double max_norm, float* out) {
  const double norm = sqrt(sum);
  out[0] = (float)norm;
  // a norm that is not finite gives a factor that is none: atomo_adamw then leaves the parameters as they are
  out[1] = norm <= 1.7e308 ? (float)fmin(1.0, max_norm / (norm + 1e-6)) : __int_as_float(0x7fc00000);
}

__device__ __forceinline__ double block_sum(double v, double* s_warp) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
  if (threadIdx.x < 32) {
    t = threadIdx.x < (blockDim.x >> 5) ? s_warp[threadIdx.x] : 0.0;
    t = warp_sum(t);
  }
  return t;                                                      // valid in warp 0
}

// A CTA takes a contiguous run of the launch's chunks.  ONE: the launch is one cluster, whose first CTA adds the others' sums through
// distributed shared memory; else the sums go to slots that norm_join_kernel adds.
template <int N, bool ONE>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(const __grid_constant__ NormBatch<N> B) {
  __shared__ double s_warp[kNormThreads / 32];
  __shared__ double s_ctas[kNormCluster];
  if constexpr (ONE) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");       // this CTA runs: its shared memory may be written to
  const uint32_t per = (B.chunks + gridDim.x - 1) / gridDim.x;
  const uint32_t first = blockIdx.x * per, last = min(first + per, B.chunks);
  double acc = 0.0;
  if (first < last) {
    int lo = 0, hi = B.n - 1;                                    // the last tensor that starts at or before `first`
    while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (B.t[mid].chunk0 <= first) lo = mid; else hi = mid - 1; }
    NormTensor t = B.t[lo];
    uint32_t end = lo + 1 < B.n ? B.t[lo + 1].chunk0 : B.chunks;
    for (uint32_t c = first; c < last; ++c) {
      if (c >= end) { ++lo; t = B.t[lo]; end = lo + 1 < B.n ? B.t[lo + 1].chunk0 : B.chunks; }
      const int size = type_bytes(t.type);
      // the values before the first 16-byte boundary and behind the last one are taken one by one, by the tensor's first chunk
      const int64_t head = min(t.n, (int64_t)(((16u - (uint32_t)(reinterpret_cast<uintptr_t>(t.data) & 15u)) & 15u) / size));
      const int64_t packs = (t.n - head) * size / 16, tail = t.n - head - packs * (16 / size);
      const uint8_t* body = t.data + head * size;
      const int64_t at = (int64_t)(c - t.chunk0) * (kNormThreads * kNormLoads) + threadIdx.x;
      uint4 r[kNormLoads];
#pragma unroll
      for (int j = 0; j < kNormLoads; ++j) {
        const int64_t i = at + j * kNormThreads;
        r[j] = i < packs ? *reinterpret_cast<const uint4*>(body + i * 16) : make_uint4(0u, 0u, 0u, 0u);
      }
      acc += norm_chunk(r, t.type);
      if (c == t.chunk0 && threadIdx.x < head + tail) {
        const double x = norm_value(t, threadIdx.x < head ? threadIdx.x : t.n - tail + (threadIdx.x - head));
        acc = fma(x, x, acc);
      }
    }
  }
  const double sum = block_sum(acc, s_warp);
  if constexpr (ONE) {
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (threadIdx.x == 0) {
      uint32_t remote, local = (uint32_t)__cvta_generic_to_shared(&s_ctas[blockIdx.x]);
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(0));
      asm volatile("st.shared::cluster.f64 [%0], %1;" :: "r"(remote), "d"(sum) : "memory");
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      double all = 0.0;
      for (uint32_t k = 0; k < gridDim.x; ++k) all += s_ctas[k];
      norm_finish(all, B.max_norm, B.out);
    }
  } else {
    if (threadIdx.x == 0) B.slots[B.slot0 + blockIdx.x] = sum;
  }
}

__global__ void __launch_bounds__(kNormThreads) norm_join_kernel(const double* __restrict__ slots, int n, double max_norm, float* __restrict__ out) {
  __shared__ double s_warp[kNormThreads / 32];
  wait_for_previous();
  double acc = 0.0;
  for (int i = threadIdx.x; i < n; i += kNormThreads) acc += slots[i];
  const double sum = block_sum(acc, s_warp);
  if (threadIdx.x == 0) norm_finish(sum, max_norm, out);
}

uint64_t norm_chunks(const atomo_tensor& t) {                   // upper bound that the kernel's own split never exceeds
  return std::max<uint64_t>(1, ((uint64_t)t.n * type_bytes(t.type) + kNormChunk - 1) / kNormChunk);
}

template <int N>
cudaError_t norm_launch(NormBatch<N>& B, int grid, bool one, cudaStream_t st) {
  if (!one) { norm_kernel<N, false><<<grid, kNormThreads, 0, st>>>(B); return cudaGetLastError(); }
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = grid; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid); cfg.blockDim = dim3(kNormThreads); cfg.stream = st;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, norm_kernel<N, true>, B);
}

template <int N>
cudaError_t norm_batch(const atomo_tensor* g, const int* index, int n, int grid, bool one, int slot0, double max_norm, float* out, double* slots, cudaStream_t st) {
  NormBatch<N> B;
  uint64_t at = 0;
  for (int i = 0; i < n; ++i) {
    const atomo_tensor& t = g[index[i]];
    B.t[i] = NormTensor{static_cast<const uint8_t*>(t.data), t.n, (uint32_t)at, t.type};
    at += norm_chunks(t);
  }
  B.n = n; B.chunks = (uint32_t)at; B.slot0 = slot0; B.max_norm = max_norm; B.slots = slots; B.out = out;
  return norm_launch<N>(B, grid, one, st);
}

__global__ void norm_empty_kernel(double max_norm, float* out) { norm_finish(0.0, max_norm, out); }

}  // namespace

namespace {
constexpr int kNormMost = 1024;                                  // tensors of a launch, 24 bytes each: 24 KB of kernel arguments
struct NormPlan { int tensors = 0; uint64_t chunks = 0; bool one = false; };   // one: few enough chunks for one cluster
NormPlan norm_plan(const atomo_tensor* grads, int n) {
  NormPlan p;
  for (int i = 0; i < n; ++i) if (grads[i].n > 0) { ++p.tensors; p.chunks += norm_chunks(grads[i]); }
  p.one = p.tensors <= kNormMost && p.chunks <= 8 * kNormCluster;
  return p;
}
}  // namespace

int grad_norm_slots(const atomo_tensor* grads, int n) { return norm_plan(grads, n).one ? 0 : kNormSlots; }

int launch_grad_norm(const atomo_tensor* grads, int n, double max_norm, float* out, double* slots, cudaStream_t st) {
  constexpr int kMost = kNormMost;
  const NormPlan plan = norm_plan(grads, n);
  const int m = plan.tensors;
  if (m == 0) { norm_empty_kernel<<<1, 1, 0, st>>>(max_norm, out); return (int)cudaGetLastError(); }
  std::vector<int> index;
  index.reserve(m);
  for (int i = 0; i < n; ++i) if (grads[i].n > 0) index.push_back(i);
  if (plan.one) {
    const int grid = (int)std::min<uint64_t>(plan.chunks, kNormCluster);
    if (m <= 8) return (int)norm_batch<8>(grads, index.data(), m, grid, true, 0, max_norm, out, slots, st);
    if (m <= 128) return (int)norm_batch<128>(grads, index.data(), m, grid, true, 0, max_norm, out, slots, st);
    return (int)norm_batch<kMost>(grads, index.data(), m, grid, true, 0, max_norm, out, slots, st);
  }
  const int launches = (m + kMost - 1) / kMost;
  int used = 0;
  for (int l = 0; l < launches; ++l) {
    const int i0 = l * kMost, count = std::min(kMost, m - i0);
    uint64_t part = 0;
    for (int i = i0; i < i0 + count; ++i) part += norm_chunks(grads[index[i]]);
    // the slots are shared out evenly: a call of more than kNormSlots * kMost tensors is refused before it gets here
    const int grid = (int)std::min<uint64_t>(part, (uint64_t)kNormSlots / launches);
    const cudaError_t e = count <= 8 ? norm_batch<8>(grads, &index[i0], count, grid, false, used, max_norm, out, slots, st)
                        : count <= 128 ? norm_batch<128>(grads, &index[i0], count, grid, false, used, max_norm, out, slots, st)
                                       : norm_batch<kMost>(grads, &index[i0], count, grid, false, used, max_norm, out, slots, st);
    if (e != cudaSuccess) return (int)e;
    used += grid;
  }
  return (int)launch_after(norm_join_kernel, dim3(1), dim3(kNormThreads), 0, st, slots, used, max_norm, out);
}

namespace {

// =================================== AdamW =======================================================
// m = b1 m + (1 - b1) c g,  v = b2 v + (1 - b2) (c g)^2,  p = p - lr wd p - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps),
// all in fp32, the moments' products and sums each rounded once, in the order written here with (1 - b2) (c g) first: a state in 8 bits is what such a
// moment rounds to, so that an element's codes do not depend on its address, and any other program gets them from the same formula.  c is read from device memory.  A CTA takes kAdamChunk neighbouring elements of a tensor, a thread several groups of
// neighbouring ones, all loads first.  Chunks that lie inside an aligned tensor go through adam_inside, compiled for the types (with 8-bit states
// instruction issue bounds the kernel as much as memory does); a tensor's last chunk, tensors of other alignment, other pairs of types and a very small eps through
// adam_any (25.6M fp32 elements, back to back, us, inside | any: fp32 states 109 | 110, 8-bit states 68 | 129).
constexpr int kAdamThreads = 256, kAdamChunk = 2048;
constexpr int kStateBlock = ATOMO_STATE_BLOCK;

struct AdamTensor {
  void* p; const void* g; void* m; void* v; uint8_t* ms; uint8_t* vs; float* master;
  int64_t n; float decay; int32_t type; uint32_t index, vec;     // vec: every array may be moved in whole groups
};
template <int N> struct AdamBatch {
  AdamTensor t[N];
  uint32_t chunk0[N];
  int n; AdamHyper h;
};

// the gradient's factor; false where its norm was not finite: then nothing is updated
__device__ __forceinline__ bool adam_factor(const AdamHyper& h, float& c) {
  c = h.scale ? h.scale[1] : 1.0f;
  return fabsf(c) <= 3.4028235e38f;
}
__device__ __forceinline__ float root(float x) { float r; asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }

__device__ __forceinline__ void adam_element(const AdamHyper& h, float c, float decay, float g, float& p, float& m, float& v) {
  g = __fmul_rn(g, c);
  m = __fadd_rn(__fmul_rn(h.beta1, m), __fmul_rn(h.one_minus_beta1, g));
  v = __fadd_rn(__fmul_rn(h.beta2, v), __fmul_rn(__fmul_rn(h.one_minus_beta2, g), g));
  const float d = fmaf(root(v), h.inv_root_bias2, h.eps);
  p = fmaf(-h.step_size, __fdividef(m, d), fmaf(decay, p, p));
}

// The same for pairs of elements, on packed fp32, without the care for subnormal numbers that root and quotient take: a second moment below 2^-126
// counts as zero.  Its root, below 2^-63, is multiplied by inv_root_bias2 before eps is added: beside an eps of kEpsPairs inv_root_bias2 or more that is less
// than 2^-25 of the sum, half of half a unit.  Calls with a smaller eps go through adam_element.
constexpr float kEpsPairs = 1.0f / (1ull << 38);                 // 3.6e-12
struct AdamPairs { uint64_t c, one, b1, r1, b2, r2, inv, eps, decay, step; };
__device__ __forceinline__ AdamPairs adam_pairs(const AdamHyper& h, float c, float decay) {
  auto both = [](float x) { return pack2(x, x); };
  return AdamPairs{both(c), both(h.one), both(h.beta1), both(h.one_minus_beta1), both(h.beta2), both(h.one_minus_beta2), both(h.inv_root_bias2), both(h.eps), both(decay), both(-h.step_size)};
}
__device__ __forceinline__ void adam_pair(const AdamPairs& k, const float* g, float* p, float* m, float* v) {
  const uint64_t g2 = mul2(pack2(g[0], g[1]), k.c), p2 = pack2(p[0], p[1]);
  // (The sums are fused ones of a product with a one that the compiler does not know: it fuses a packed product and a packed sum, be they written as such or
  // with a zero between them, and the product is then not rounded.  8-bit states of 25.6M elements back to back: 66.2 us fused, 67.7 so.)
  const uint64_t m2 = fma2(k.one, mul2(k.b1, pack2(m[0], m[1])), mul2(k.r1, g2));
  const uint64_t v2 = fma2(k.one, mul2(k.b2, pack2(v[0], v[1])), mul2(mul2(k.r2, g2), g2));
  unpack2(m2, m[0], m[1]); unpack2(v2, v[0], v[1]);
  float s0, s1;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(s0) : "f"(v[0]));
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(s1) : "f"(v[1]));
  unpack2(fma2(pack2(s0, s1), k.inv, k.eps), s0, s1);
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(s0));
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(s1));
  unpack2(fma2(k.step, mul2(m2, pack2(s0, s1)), fma2(k.decay, p2, p2)), p[0], p[1]);
}

// ---- states in 8 bits: e4m3 codes times a power of two for each 32 neighbouring elements, kept as its exponent byte ----
__device__ __forceinline__ float state_scale(uint32_t byte) { return __uint_as_float(byte > 0u ? byte << 23 : 0x00400000u); }
__device__ __forceinline__ void state_decode(uint32_t codes, float s, float* x) {
  uint32_t lo, hi;
  asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(codes));
  const float2 a = __half22float2(*reinterpret_cast<__half2*>(&lo)), b = __half22float2(*reinterpret_cast<__half2*>(&hi));
  const uint64_t s2 = pack2(s, s);
  unpack2(mul2(pack2(a.x, a.y), s2), x[0], x[1]); unpack2(mul2(pack2(b.x, b.y), s2), x[2], x[3]);
}
// The power of two brings the block's largest finite magnitude into [224, 448), so that rounding it up stays within e4m3.  The magnitude
// times 2^-120 has e4m3's exponent in the exponent field of fp32, subnormal numbers included, so that its code is bits 27 to 20;
// 16 random bits added below them round up with the probability of what is cut off (to 2^-16 of a step).  All of it four bits
// further up leaves the code in the top byte.
// ABOVE_ZERO: a value above zero is never rounded to zero (a second moment of zero beside a first moment that is not would make a
// step of any size).  What is not finite becomes NaN.
// PER neighbouring elements per thread; the high (HIGH) or low 16 bits of their random words.
template <int PER, bool ABOVE_ZERO, bool HIGH>
__device__ __forceinline__ void state_encode(const float (&x)[PER], const uint32_t (&random)[PER], uint32_t (&codes)[PER / 4], uint32_t& byte) {
  constexpr uint32_t kMask = ABOVE_ZERO ? 0xffffffffu : 0x7fffffffu;          // (a second moment has no sign)
  float y[PER], factor;
  uint32_t top = 0u;
#pragma unroll
  for (int j = 0; j < PER; ++j) { y[j] = __uint_as_float(__float_as_uint(x[j]) & kMask); top = max(top, __float_as_uint(y[j])); }
#pragma unroll
  for (int o = 1; o < kStateBlock / PER; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  // up to here one factor does (an exponent byte of at most 133): beyond, values of 2^14 and more, and those that are not finite
  const bool plain = __all_sync(0xffffffffu, top < 0x46e00000u);
  if (plain) {
    byte = (uint32_t)max((int)((top + 0x200000u) >> 23) - 8, 0);
    factor = __uint_as_float((134u - byte) << 23);
  } else {
    top = 0u;
#pragma unroll
    for (int j = 0; j < PER; ++j) { const uint32_t a = __float_as_uint(y[j]); if (a < 0x7f800000u) top = max(top, a); }
#pragma unroll
    for (int o = 1; o < kStateBlock / PER; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    byte = (uint32_t)max((int)((top + 0x200000u) >> 23) - 8, 0);
    factor = __uint_as_float(7u << 23);                          // 2^-120
#pragma unroll
    for (int j = 0; j < PER; ++j) y[j] = __fmul_rn(y[j], __uint_as_float((254u - byte) << 23));
  }
  // (No product by `*` here: nvcc 12.9.86 takes the bits of one for zero where they are shifted and added as below, which a kernel of these lines alone
  // shows; of a packed product, of __fmul_rn and of mul.rn.f32 they are right.  The packed one takes half the instructions.)
  uint32_t t[PER], least = 0xffffffffu;
  const uint64_t factors = pack2(factor, factor);
#pragma unroll
  for (int j = 0; j < PER; j += 2) {
    float a, b;
    unpack2(mul2(pack2(y[j], y[j + 1]), factors), a, b);
    t[j] = __float_as_uint(a) * 16u + __byte_perm(random[j], 0u, HIGH ? 0x4324 : 0x4104);                  // the 16 bits in bytes 1 and 2
    t[j + 1] = __float_as_uint(b) * 16u + __byte_perm(random[j + 1], 0u, HIGH ? 0x4324 : 0x4104);
    least = min(least, min(t[j], t[j + 1]));
  }
  if (!plain) {
#pragma unroll
    for (int j = 0; j < PER; ++j) if ((__float_as_uint(x[j]) & 0x7fffffffu) >= 0x7f800000u) t[j] = 0x7f000000u;
  }
  if (ABOVE_ZERO && least < 1u << 24) {
#pragma unroll
    for (int j = 0; j < PER; ++j) t[j] = x[j] > 0.0f ? max(t[j], 1u << 24) : t[j];
  }
#pragma unroll
  for (int q = 0; q < PER / 4; ++q) {
    const uint32_t a = __byte_perm(t[4 * q], t[4 * q + 1], 0x0073), b = __byte_perm(t[4 * q + 2], t[4 * q + 3], 0x0073);
    codes[q] = __byte_perm(a, b, 0x5410);
    if (!ABOVE_ZERO) {                                           // signs
      const uint32_t sa = __byte_perm(__float_as_uint(x[4 * q]), __float_as_uint(x[4 * q + 1]), 0x0073);
      const uint32_t sb = __byte_perm(__float_as_uint(x[4 * q + 2]), __float_as_uint(x[4 * q + 3]), 0x0073);
      codes[q] |= __byte_perm(sa, sb, 0x5410) & 0x80808080u;
    }
  }
}
__device__ __forceinline__ uint4 state_words(const AdamHyper& h, uint32_t tensor, int64_t e) {
  const uint64_t block = (uint64_t)e >> 2;
  return philox4x32_10(make_uint4((uint32_t)block, (uint32_t)(block >> 32) | 0x80000000u, tensor, h.step & 0x7fffffffu), h.key);
}

// ---- any alignment and any types, four elements at a time ----
// four elements of `size` bytes each as they lie in memory, in the low words of r; `count` of them exist
__device__ __forceinline__ uint4 load_raw4(const void* base, int size, int64_t e, int count, bool vec) {
  uint4 r = make_uint4(0u, 0u, 0u, 0u);
  const uint8_t* p = static_cast<const uint8_t*>(base) + e * size;
  if (vec && count >= 4) {
    if (size == 4) r = *reinterpret_cast<const uint4*>(p);
    else if (size == 2) { const uint2 q = *reinterpret_cast<const uint2*>(p); r.x = q.x; r.y = q.y; }
    else r.x = *reinterpret_cast<const uint32_t*>(p);
    return r;
  }
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (j < count) {
      if (size == 4) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
      else if (size == 2) w[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j & 1));
      else w[0] |= (uint32_t)p[j] << (8 * j);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_raw4(void* base, int size, int64_t e, int count, bool vec, uint4 r) {
  uint8_t* p = static_cast<uint8_t*>(base) + e * size;
  if (vec && count >= 4) {
    if (size == 4) *reinterpret_cast<uint4*>(p) = r;
    else if (size == 2) *reinterpret_cast<uint2*>(p) = make_uint2(r.x, r.y);
    else *reinterpret_cast<uint32_t*>(p) = r.x;
    return;
  }
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (j < count) {
      if (size == 4) reinterpret_cast<uint32_t*>(p)[j] = w[j];
      else if (size == 2) reinterpret_cast<uint16_t*>(p)[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
      else p[j] = (uint8_t)(w[0] >> (8 * j));
    }
  }
}
__device__ __forceinline__ void unpack4(uint4 r, int type, float (&x)[4]) {
  if (type == ATOMO_TYPE_F32) { x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w); }
  else if (type == ATOMO_TYPE_BF16) {
    x[0] = __uint_as_float(r.x << 16); x[1] = __uint_as_float(r.x & 0xffff0000u);
    x[2] = __uint_as_float(r.y << 16); x[3] = __uint_as_float(r.y & 0xffff0000u);
  } else {
    const float2 a = __half22float2(*reinterpret_cast<__half2*>(&r.x)), b = __half22float2(*reinterpret_cast<__half2*>(&r.y));
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
  }
}
// to the nearest value of the type, ties to even
__device__ __forceinline__ uint4 pack4(const float (&x)[4], int type) {
  uint4 r = make_uint4(0u, 0u, 0u, 0u);
  if (type == ATOMO_TYPE_F32) r = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  else if (type == ATOMO_TYPE_BF16) {
    __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    r.x = *reinterpret_cast<uint32_t*>(&a); r.y = *reinterpret_cast<uint32_t*>(&b);
  } else {
    __half2 a = __floats2half2_rn(x[0], x[1]), b = __floats2half2_rn(x[2], x[3]);
    r.x = *reinterpret_cast<uint32_t*>(&a); r.y = *reinterpret_cast<uint32_t*>(&b);
  }
  return r;
}

template <int BITS>
__device__ __noinline__ void adam_any(const AdamTensor& t, const AdamHyper& h, int64_t first) {
  float c;
  if (!adam_factor(h, c)) return;
  constexpr int kSize = BITS / 8;                                // bytes of a state
  const bool vec = t.vec != 0u, has_master = t.master != nullptr;
  const int psize = type_bytes(t.type);
  const float decay = -h.lr * t.decay;
#pragma unroll 2
  for (int u = 0; u < kAdamChunk / (kAdamThreads * 4); ++u) {
    const int64_t e = first + (u * kAdamThreads + threadIdx.x) * 4;
    const int count = (int)max((int64_t)0, min((int64_t)4, t.n - e));
    const uint4 rg = load_raw4(t.g, type_bytes(h.grad_type), e, count, vec);
    const uint4 rp = has_master ? load_raw4(t.master, 4, e, count, vec) : load_raw4(t.p, psize, e, count, vec);
    const uint4 rm = load_raw4(t.m, kSize, e, count, vec), rv = load_raw4(t.v, kSize, e, count, vec);
    float p[4], g[4], m[4], v[4];
    unpack4(rg, h.grad_type, g);
    unpack4(rp, has_master ? (int)ATOMO_TYPE_F32 : t.type, p);
    if constexpr (BITS == 8) {
      const uint32_t bm = count > 0 ? t.ms[e / kStateBlock] : 0u, bv = count > 0 ? t.vs[e / kStateBlock] : 0u;
      state_decode(rm.x, state_scale(bm), m); state_decode(rv.x, state_scale(bv), v);
    } else { unpack4(rm, ATOMO_TYPE_F32, m); unpack4(rv, ATOMO_TYPE_F32, v); }
#pragma unroll
    for (int j = 0; j < 4; ++j) adam_element(h, c, decay, g[j], p[j], m[j], v[j]);
    if constexpr (BITS == 8) {
      const uint4 w = state_words(h, t.index, e);
      const uint32_t random[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) if (j >= count) { m[j] = 0.0f; v[j] = 0.0f; }
      uint32_t new_m, new_v, cm[1], cv[1];
      state_encode<4, false, false>(m, random, cm, new_m);
      state_encode<4, true, true>(v, random, cv, new_v);
      if (count > 0) {
        store_raw4(t.m, 1, e, count, vec, make_uint4(cm[0], 0u, 0u, 0u));
        store_raw4(t.v, 1, e, count, vec, make_uint4(cv[0], 0u, 0u, 0u));
        if (e % kStateBlock == 0) { t.ms[e / kStateBlock] = (uint8_t)new_m; t.vs[e / kStateBlock] = (uint8_t)new_v; }
      }
    } else {
      store_raw4(t.m, 4, e, count, vec, pack4(m, ATOMO_TYPE_F32));
      store_raw4(t.v, 4, e, count, vec, pack4(v, ATOMO_TYPE_F32));
    }
    if (has_master) store_raw4(t.master, 4, e, count, vec, pack4(p, ATOMO_TYPE_F32));
    store_raw4(t.p, psize, e, count, vec, pack4(p, t.type));
  }
}

// ---- a chunk inside an aligned tensor ----
// (Eight fp32 values in one piece, 32 bytes aligned: two of 16 touch each sector twice, 78 against 74 us with 8-bit states of 25.6M elements.)
template <typename T, int PER> __device__ __forceinline__ void load_group(const T* p, float (&x)[PER]) {
  if constexpr (sizeof(T) == 4 && PER == 8) {
    asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "l"(p) : "memory");
    return;
  }
  constexpr int kVec = 16 / (int)sizeof(T) < PER ? 16 / (int)sizeof(T) : PER;
#pragma unroll
  for (int k = 0; k < PER; k += kVec) {
    const Pack<T, kVec> r = load_pack<T, kVec>(p + k);
#pragma unroll
    for (int j = 0; j < kVec; ++j) x[k + j] = to_float(r.v[j]);
  }
}
template <typename T, int PER> __device__ __forceinline__ void store_group(T* p, const float (&x)[PER]) {
  if constexpr (sizeof(T) == 4 && PER == 8) {
    asm volatile("st.global.v8.f32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};"
                 :: "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]), "l"(p) : "memory");
    return;
  }
  constexpr int kVec = 16 / (int)sizeof(T) < PER ? 16 / (int)sizeof(T) : PER;
#pragma unroll
  for (int k = 0; k < PER; k += kVec) {
    Pack<T, kVec> r;
#pragma unroll
    for (int j = 0; j < kVec; ++j) r.v[j] = from_float<T>(x[k + j]);
    store_pack<T, kVec>(p + k, r);
  }
}

// Elements per group: with 8-bit states eight, so that four lanes share a block.
template <int BITS, typename P, typename G, bool MASTER>
__device__ __forceinline__ void adam_inside(const AdamTensor& t, const AdamHyper& h, int64_t first) {
  constexpr int PER = BITS == 8 ? 8 : 4, kGroups = kAdamChunk / (kAdamThreads * PER);
  P* tp = static_cast<P*>(t.p) + first + threadIdx.x * PER;
  float* tw = t.master + first + threadIdx.x * PER;
  const G* tg = static_cast<const G*>(t.g) + first + threadIdx.x * PER;
  float p[kGroups][PER], g[kGroups][PER];
  if constexpr (BITS == 32) {
    float* tm = static_cast<float*>(t.m) + first + threadIdx.x * PER;
    float* tv = static_cast<float*>(t.v) + first + threadIdx.x * PER;
    float m[kGroups][PER], v[kGroups][PER];
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      constexpr int kStep = kAdamThreads * PER;
      load_group<G, PER>(tg + u * kStep, g[u]);
      if constexpr (MASTER) load_group<float, PER>(tw + u * kStep, p[u]); else load_group<P, PER>(tp + u * kStep, p[u]);
      load_group<float, PER>(tm + u * kStep, m[u]);
      load_group<float, PER>(tv + u * kStep, v[u]);
    }
    float c;
    if (!adam_factor(h, c)) return;
    const AdamPairs k = adam_pairs(h, c, -h.lr * t.decay);
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      constexpr int kStep = kAdamThreads * PER;
#pragma unroll
      for (int j = 0; j < PER; j += 2) adam_pair(k, g[u] + j, p[u] + j, m[u] + j, v[u] + j);
      store_group<float, PER>(tm + u * kStep, m[u]);
      store_group<float, PER>(tv + u * kStep, v[u]);
      if constexpr (MASTER) store_group<float, PER>(tw + u * kStep, p[u]);
      store_group<P, PER>(tp + u * kStep, p[u]);
    }
  } else {
    uint8_t* tm = static_cast<uint8_t*>(t.m) + first + threadIdx.x * PER;
    uint8_t* tv = static_cast<uint8_t*>(t.v) + first + threadIdx.x * PER;
    uint8_t* sm = t.ms + first / kStateBlock + threadIdx.x * PER / kStateBlock;
    uint8_t* sv = t.vs + first / kStateBlock + threadIdx.x * PER / kStateBlock;
    uint2 rm[kGroups], rv[kGroups];
    uint32_t bm[kGroups], bv[kGroups];
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      constexpr int kStep = kAdamThreads * PER;
      rm[u] = *reinterpret_cast<const uint2*>(tm + u * kStep); rv[u] = *reinterpret_cast<const uint2*>(tv + u * kStep);
      bm[u] = sm[u * kStep / kStateBlock]; bv[u] = sv[u * kStep / kStateBlock];
      load_group<G, PER>(tg + u * kStep, g[u]);
      if constexpr (MASTER) load_group<float, PER>(tw + u * kStep, p[u]); else load_group<P, PER>(tp + u * kStep, p[u]);
    }
    float c;
    if (!adam_factor(h, c)) return;
    const AdamPairs k = adam_pairs(h, c, -h.lr * t.decay);
#pragma unroll
    for (int u = 0; u < kGroups; ++u) {
      constexpr int kStep = kAdamThreads * PER;
      float m[PER], v[PER];
      const float fm = state_scale(bm[u]), fv = state_scale(bv[u]);
      state_decode(rm[u].x, fm, m); state_decode(rm[u].y, fm, m + 4);
      state_decode(rv[u].x, fv, v); state_decode(rv[u].y, fv, v + 4);
#pragma unroll
      for (int j = 0; j < PER; j += 2) adam_pair(k, g[u] + j, p[u] + j, m + j, v + j);
      if constexpr (MASTER) store_group<float, PER>(tw + u * kStep, p[u]);
      store_group<P, PER>(tp + u * kStep, p[u]);
      const int64_t e = first + (u * kAdamThreads + threadIdx.x) * PER;
      const uint4 w0 = state_words(h, t.index, e), w1 = state_words(h, t.index, e + 4);
      const uint32_t random[PER] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
      uint32_t new_m, new_v, cm[2], cv[2];
      state_encode<PER, false, false>(m, random, cm, new_m);
      state_encode<PER, true, true>(v, random, cv, new_v);
      *reinterpret_cast<uint2*>(tm + u * kStep) = make_uint2(cm[0], cm[1]);
      *reinterpret_cast<uint2*>(tv + u * kStep) = make_uint2(cv[0], cv[1]);
      if (threadIdx.x % (kStateBlock / PER) == 0) { sm[u * kStep / kStateBlock] = (uint8_t)new_m; sv[u * kStep / kStateBlock] = (uint8_t)new_v; }
    }
  }
}

// Chunks of 2048 elements and five CTAs per SM, us (8-bit states, 25.6M elements | fp32 states, 11M | fp32 states and master copy, 133M): 74 | 51 | 550;
// of 4096 and three per SM: 78 | 53 | 553; of 4096 and four: 90 | 53 | 562; of 2048 and six: 83 | 51 | 553.  The update by pairs took the instructions per
// element with 8-bit states from 65 to 53, its moments rounded operation by operation to 54 (issue slots 62 % busy).  Memory bounds all three: 413, 308 and 3738 MB, 5.6, 6.0 and 6.8 TB/s.
template <int N, int BITS>
__global__ void __launch_bounds__(kAdamThreads, 5) adamw_kernel(const __grid_constant__ AdamBatch<N> B) {
  int lo = 0, hi = B.n - 1;                                      // the last tensor that starts at or before this chunk
  while (lo < hi) { const int mid = (lo + hi + 1) >> 1; if (B.chunk0[mid] <= blockIdx.x) lo = mid; else hi = mid - 1; }
  const AdamTensor& t = B.t[lo];
  const AdamHyper& h = B.h;
  const int64_t first = (int64_t)(blockIdx.x - B.chunk0[lo]) * kAdamChunk;
  if (t.vec && first + kAdamChunk <= t.n && h.eps >= kEpsPairs * h.inv_root_bias2) {
    const bool same = h.grad_type == t.type, wide = h.grad_type == ATOMO_TYPE_F32, master = t.master != nullptr;
    if (t.type == ATOMO_TYPE_F32) {
      if (!master && wide) return adam_inside<BITS, float, float, false>(t, h, first);
    } else if (t.type == ATOMO_TYPE_BF16) {
      if (master && wide) return adam_inside<BITS, __nv_bfloat16, float, true>(t, h, first);
      if (master && same) return adam_inside<BITS, __nv_bfloat16, __nv_bfloat16, true>(t, h, first);
      if (!master && wide) return adam_inside<BITS, __nv_bfloat16, float, false>(t, h, first);
      if (!master && same) return adam_inside<BITS, __nv_bfloat16, __nv_bfloat16, false>(t, h, first);
    } else {
      if (master && wide) return adam_inside<BITS, __half, float, true>(t, h, first);
      if (master && same) return adam_inside<BITS, __half, __half, true>(t, h, first);
      if (!master && wide) return adam_inside<BITS, __half, float, false>(t, h, first);
      if (!master && same) return adam_inside<BITS, __half, __half, false>(t, h, first);
    }
  }
  adam_any<BITS>(t, h, first);
}

bool apart(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

template <int N>
cudaError_t adamw_batch(const atomo_adamw_tensor* ts, const void* const* grads, const int* index, int n, int bits, const AdamHyper& h, cudaStream_t st) {
  AdamBatch<N> B;
  uint64_t at = 0;
  const int ssize = bits / 8;
  for (int i = 0; i < n; ++i) {
    const atomo_adamw_tensor& t = ts[index[i]];
    const void* g = grads[index[i]];
    const int wide = ssize == 1 ? 8 : 4;                         // elements of a group
    const bool vec = apart(t.param, wide * type_bytes(t.type)) && apart(g, wide * type_bytes(h.grad_type)) && apart(t.exp_avg, wide * ssize) && apart(t.exp_avg_sq, wide * ssize) &&
                     apart(t.master, wide * 4);
    B.t[i] = AdamTensor{t.param, g, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale, t.exp_avg_sq_scale, t.master, t.n, t.weight_decay, t.type, (uint32_t)index[i], vec};
    B.chunk0[i] = (uint32_t)at;
    at += (uint64_t)((t.n + kAdamChunk - 1) / kAdamChunk);
  }
  B.n = n; B.h = h;
  if (bits == 8) adamw_kernel<N, 8><<<(unsigned)at, kAdamThreads, 0, st>>>(B);
  else adamw_kernel<N, 32><<<(unsigned)at, kAdamThreads, 0, st>>>(B);
  return cudaGetLastError();
}

}  // namespace

int launch_adamw(const atomo_adamw_tensor* tensors, const void* const* grads, int n, int bits, const AdamHyper& h, cudaStream_t st) {
  constexpr int kMost = 380;                                     // 84 bytes each: just under 32 KB of kernel arguments
  constexpr uint64_t kMostChunks = 0x7fffffffull;                // CTAs of a launch
  std::vector<int> index;
  index.reserve(n);
  for (int i = 0; i < n; ++i) if (tensors[i].n > 0) index.push_back(i);
  for (int i0 = 0; i0 < (int)index.size();) {
    int count = 0;
    uint64_t chunks = 0;
    while (i0 + count < (int)index.size() && count < kMost) {
      const uint64_t c = (uint64_t)((tensors[index[i0 + count]].n + kAdamChunk - 1) / kAdamChunk);
      if (count > 0 && chunks + c > kMostChunks) break;
      chunks += c; ++count;
    }
    const cudaError_t e = count <= 8 ? adamw_batch<8>(tensors, grads, &index[i0], count, bits, h, st)
                        : count <= 64 ? adamw_batch<64>(tensors, grads, &index[i0], count, bits, h, st)
                                      : adamw_batch<kMost>(tensors, grads, &index[i0], count, bits, h, st);
    if (e != cudaSuccess) return (int)e;
    i0 += count;
  }
  return (int)cudaSuccess;
}

}  // namespace atomo
