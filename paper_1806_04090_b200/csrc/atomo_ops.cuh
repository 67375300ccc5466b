// Descriptors and launchers of the operators on either side of the gradient exchange (gradient norm, AdamW, embedding, layer norm),
// and what their kernels share: values of three types in 32-bit arithmetic, launches that overlap their predecessor's end.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <string.h>

#include <type_traits>
#include <vector>

#include "atomo_common.cuh"

namespace atomo {

__host__ __device__ __forceinline__ int type_bytes(int type) { return type == ATOMO_TYPE_F32 ? 4 : 2; }

// ---- values ---------------------------------------------------------------------------------------
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }

// V neighbouring values, moved in one piece
template <typename T, int V> struct alignas(V * sizeof(T)) Pack { T v[V]; };
template <typename T, int V> __device__ __forceinline__ Pack<T, V> load_pack(const T* p) { return *reinterpret_cast<const Pack<T, V>*>(p); }
template <typename T, int V> __device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& x) { *reinterpret_cast<Pack<T, V>*>(p) = x; }

// two neighbouring values as a pair of fp32, and back
template <typename T> __device__ __forceinline__ uint64_t pair_of(const T* p) {
  if constexpr (sizeof(T) == 4) return pack2(p[0], p[1]);
  else {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
    if constexpr (std::is_same<T, __nv_bfloat16>::value) return pack2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    return pack2(f.x, f.y);
  }
}
template <typename T> __device__ __forceinline__ void pair_to(T* p, uint64_t v) {
  float a, b;
  unpack2(v, a, b);
  if constexpr (sizeof(T) == 4) { p[0] = a; p[1] = b; }
  else if constexpr (std::is_same<T, __nv_bfloat16>::value) *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(a, b);
  else *reinterpret_cast<__half2*>(p) = __floats2half2_rn(a, b);
}

// a copy of BYTES bytes (16 or 4) from global to shared memory that the thread waits for with cp.async.wait_group
template <int BYTES> __device__ __forceinline__ void copy_async(void* shared, const void* global) {
  const uint32_t s = (uint32_t)__cvta_generic_to_shared(shared);
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(s), "l"(global) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" :: "r"(s), "l"(global), "n"(BYTES) : "memory");
}

// ---- launches -------------------------------------------------------------------------------------
// A kernel launched with launch_after() may start while the kernel before it in the stream ends; it calls wait_for_previous() in every
// thread before it touches memory.
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
template <typename... P, typename... A>
cudaError_t launch_after(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, A... args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cfg.attrs = attr; cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// ---- gradient norm (atomo_step.cu) ----------------------------------------------------------------
constexpr int kNormSlots = 148 * 8;     // partial sums of a call, at most
int grad_norm_slots(const atomo_tensor* grads, int n);                           // how many a call needs: 0 where one cluster does it all
int launch_grad_norm(const atomo_tensor* grads, int n, double max_norm, float* out, double* slots, cudaStream_t st);   // cudaError_t

// ---- AdamW (atomo_step.cu) ------------------------------------------------------------------------
struct AdamHyper {
  float beta1, one_minus_beta1, beta2, one_minus_beta2;
  float one = 1.0f;                           // a one that the kernels' compiler does not know
  float lr, step_size, inv_root_bias2, eps;   // step_size = lr / (1 - beta1^t), inv_root_bias2 = 1 / sqrt(1 - beta2^t)
  const float* scale;                         // DEVICE: {norm, factor of the gradient}, or null
  uint32_t step; int32_t grad_type;
  PhiloxRoundKeys key;
};
int launch_adamw(const atomo_adamw_tensor* tensors, const void* const* grads, int n, int bits, const AdamHyper& h, cudaStream_t st);   // cudaError_t

// ---- embedding (atomo_embedding.cu) ---------------------------------------------------------------
constexpr int kEmbChunk = 32;           // sorted tokens that are summed by one group of threads
constexpr int kSortClusters = 5;        // clusters of 1, 2, .. 16 CTAs
struct SortRoom { int clusters[kSortClusters] = {}; };           // of each size, how many the GPU holds side by side
struct EmbLookup {
  const void* table; int type; int64_t rows, cols, ld;
  const void* ids; int id_bytes; int64_t n;
  float scale; void* out; int64_t ld_out; int32_t* status;
};
struct EmbBackward {
  const void* ids; int id_bytes; int64_t n;
  const void* grad; int type; int64_t ld, rows, cols;
  float scale; int64_t padding;         // id whose tokens are left out, or -1
  float* out; int64_t ld_out; int accumulate; int32_t* status;
  uint8_t* ws;
  SortRoom room;
};
int embedding_configure(SortRoom* room);                                         // shared memory, cluster sizes of the current device; cudaError_t
int launch_embedding(const EmbLookup& a, cudaStream_t st);                       // cudaError_t
uint64_t embedding_workspace(int64_t n, int64_t cols);
int launch_embedding_backward(const EmbBackward& a, cudaStream_t st);            // cudaError_t

// ---- layer norm (atomo_layernorm.cu) --------------------------------------------------------------
struct NormForward {
  const void* x; int type; int64_t rows, cols, ld;
  const void *weight, *bias; int weight_type; float eps;
  void* y; int64_t ld_y; float *mean, *rstd;
};
struct NormBackward {
  const void *dy, *x; int type; int64_t rows, cols, ld_dy, ld_x;
  const void* weight; int weight_type; const float *mean, *rstd;
  void* dx; int64_t ld_dx; float *dweight, *dbias;
  float* ws;
};
int layer_norm_configure();                                                      // shared memory; cudaError_t
int launch_layer_norm(const NormForward& a, cudaStream_t st);                    // cudaError_t
uint64_t layer_norm_workspace(int64_t rows, int64_t cols);
int launch_layer_norm_backward(const NormBackward& a, cudaStream_t st);          // cudaError_t

}  // namespace atomo
