// Embedding lookup, and the gradient of the table by sorted tokens.
//
//   out[t] = s table[id[t]],   dtable[v] = s sum_{t : id[t] = v} dout[t]
//
// The gradient's sums run in the order of the tokens, so that the same call gives the same bits each time (a payload that is encoded
// from it does too), which sums by atomics would not.  Four kernels:
//   emb_sort_kernel   stable radix sort of (id, token), eight bits a pass, by the CTAs of one cluster: they exchange their histograms
//                     through distributed shared memory and their items through L2, with the hardware cluster barrier between; a tile's items are put in
//                     order in shared memory first, so that they leave in runs.  It also lists the long runs of equal ids.
//   emb_zero_kernel   writes the rows without tokens, beside the sort: a CTA looks through the ids for those of its own rows, so that it needs no sort.
//   emb_sum_kernel    chunks of kEmbChunk neighbouring sorted tokens, so that a frequent token's run is split among CTAs.  A run that ends in the chunk it
//                     starts in, or in the next one, is summed by the former and goes to its row; a longer one leaves one part per chunk in the workspace.
//   emb_join_kernel   adds the parts of the longer runs, in order.
// What bounds it is memory: dout is read once, the table's gradient written once.  64k tokens of 2048 bf16 columns, 32000 rows, 530 MB in all: sort 25 us beside
// the zero rows' 39, sums 64 (6.1 TB/s), join 14.
// Short lists go through emb_direct_kernel, which does all of it: a CTA has every so-manieth row of the table (frequent ids often lie side by side) and some
// columns, finds the tokens of its rows among all ids, sorts them in shared memory and sums them; and it has a stretch of rows in which it writes those without
// tokens.  A launch instead of four, and no wait between them.
#include <algorithm>

#include "atomo_ops.cuh"

namespace atomo {
namespace {

constexpr int kEmbThreads = 256;
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortItems = 8, kSortTile = kSortThreads * kSortItems;
constexpr int kSortClusterMax = 16;

struct Ids { const void* p; int wide; };                         // wide: 64-bit
__device__ __forceinline__ int64_t load_id(const Ids& ids, int64_t t) {
  return ids.wide ? reinterpret_cast<const int64_t*>(ids.p)[t] : (int64_t) reinterpret_cast<const int32_t*>(ids.p)[t];
}
__device__ __forceinline__ void raise_word(int32_t* status) { if (status) atomicCAS(status, (int32_t)ATOMO_OK, (int32_t)ATOMO_ERR_INVALID_ARG); }

// Threads of a CTA: cx along a row (VEC columns each), cy rows; `slabs` CTAs share a row
struct EmbShape { int cx, cy, slabs; };
EmbShape emb_shape(int64_t cols, int vec) {
  const int64_t packs = (cols + vec - 1) / vec;
  EmbShape s;
  if (packs <= kEmbThreads / 2) {
    s.cx = 8;                                                    // at most 32 rows, whose chunks' items take 25 KB of shared memory
    while (s.cx < packs) s.cx += s.cx < 32 ? s.cx : 32;           // (warps that are full as far as can be)
    s.cy = kEmbThreads / s.cx; s.slabs = 1;
  } else {
    s.slabs = (int)((packs + kEmbThreads - 1) / kEmbThreads);
    s.cx = (int)(((packs + s.slabs - 1) / s.slabs + 31) / 32 * 32); s.cy = 1;
  }
  return s;
}

// ---- lookup ---------------------------------------------------------------------------------------
// A CTA goes on to other tokens, whose ids it fetches while the rows are under way; what it writes is not kept in L2 for long, so that the rows of frequent
// tokens stay.  64k tokens of 2048 bf16, us, CTAs per SM x tokens at a time: 5 x 2 57, 6 x 2 59 (the order of 4 x 2, 4 x 3, 3 x 4, 8 x 2 behind them: 64 to 72); one
// CTA per two tokens, many more than fit: 84; without the streaming stores 72 at best.
// A thread has one pack of 16 bytes of a row, or four smaller ones (what a token costs it, 60 instructions, is shared by them).
constexpr int kLookCtas = 5, kLookTokens = 2;
template <typename T, int VEC> __host__ __device__ constexpr int look_packs() { return VEC * sizeof(T) == 16 ? 1 : 4; }
template <typename T, int VEC>
__device__ __forceinline__ void scale_pack(Pack<T, VEC>& x, float scale) {
  if constexpr (VEC > 1) {
    const uint64_t both = pack2(scale, scale);
#pragma unroll
    for (int j = 0; j < VEC; j += 2) pair_to(x.v + j, mul2(pair_of(x.v + j), both));
  } else x.v[0] = from_float<T>(to_float(x.v[0]) * scale);
}
template <typename T, int VEC, int U>
__global__ void __launch_bounds__(kEmbThreads, kLookCtas) emb_lookup_kernel(const T* __restrict__ table, int64_t rows, int64_t cols, int64_t ld, Ids ids, int64_t n,
                                                                 float scale, T* __restrict__ out, int64_t ld_out, int32_t* status) {
  constexpr int P = look_packs<T, VEC>();
  const int64_t col = ((int64_t)blockIdx.y * P * blockDim.x + threadIdx.x) * VEC, step = (int64_t)gridDim.x * U * blockDim.y;
  const int hop = blockDim.x * VEC;                              // between a thread's packs
  if (col >= cols) return;
  int64_t id[U], t0 = (int64_t)blockIdx.x * U * blockDim.y + threadIdx.y;
#pragma unroll
  for (int u = 0; u < U; ++u) { const int64_t t = t0 + (int64_t)u * blockDim.y; id[u] = t < n ? load_id(ids, t) : -1; }
  for (; t0 < n; t0 += step) {
    Pack<T, VEC> x[U][P];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool valid = id[u] >= 0 && id[u] < rows;
      if (!valid && col == 0 && t0 + (int64_t)u * blockDim.y < n) raise_word(status);
      const T* from = table + id[u] * ld + col;
#pragma unroll
      for (int p = 0; p < P; ++p) {
        if (valid && col + p * hop < cols) x[u][p] = load_pack<T, VEC>(from + p * hop);
        else {
#pragma unroll
          for (int j = 0; j < VEC; ++j) x[u][p].v[j] = from_float<T>(0.0f);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) { const int64_t t = t0 + step + (int64_t)u * blockDim.y; id[u] = t < n ? load_id(ids, t) : -1; }      // the next ones, meanwhile
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t t = t0 + (int64_t)u * blockDim.y;
      if (t < n) {
        T* to = out + t * ld_out + col;
#pragma unroll
        for (int p = 0; p < P; ++p) {
          if (col + p * hop < cols) {
            scale_pack(x[u][p], scale);
            if constexpr (VEC * sizeof(T) == 16) __stcs(reinterpret_cast<uint4*>(to), *reinterpret_cast<uint4*>(&x[u][p]));
            else store_pack<T, VEC>(to + p * hop, x[u][p]);
          }
        }
      }
    }
  }
}

// ---- sort -----------------------------------------------------------------------------------------
struct SortArgs {
  Ids ids; int64_t n, rows, padding;
  uint64_t* items[2];                   // id << 32 | token; the sorted ones end in [passes & 1]
  uint32_t* runs;                       // [0] number of long runs, then the chunks that they start in
  int32_t* status;
  int passes, bits;
  int64_t segment;                      // tokens of a CTA
  uint32_t ctas;                        // CTAs: one cluster
  int beside;                           // the next kernel in the stream runs beside this one
};
// rows without tokens
struct ZeroArgs { Ids ids; int64_t n, rows, padding, cols; float* out; int64_t ld_out; int vec_out, wide_ids; };
constexpr int kZeroThreads = 1024;

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote_u32(const uint32_t* local, uint32_t rank) {
  uint32_t a = (uint32_t)__cvta_generic_to_shared(local), r, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(r) : "memory");
  return v;
}

__device__ __forceinline__ void put_remote(uint64_t* local, uint32_t rank, uint64_t x) {
  uint32_t a = (uint32_t)__cvta_generic_to_shared(local), r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("st.shared::cluster.u64 [%0], %1;" :: "r"(r), "l"(x) : "memory");
}

// a token as a sort item: ids that have no row, and the padding id, come last
__device__ __forceinline__ uint64_t sort_item(const SortArgs& a, int64_t t) {
  const int64_t id = load_id(a.ids, t);
  const bool ok = id >= 0 && id < a.rows;
  if (!ok) raise_word(a.status);
  return (uint64_t)(ok && id != a.padding ? (uint32_t)id : (uint32_t)a.rows) << 32 | (uint32_t)t;
}

// a run is long if it goes on behind the chunk that follows the one it starts in
__device__ __forceinline__ uint32_t item_id(const uint64_t* items, int64_t i) { return (uint32_t)(items[i] >> 32); }

// a row, by a warp
__device__ __forceinline__ void zero_row(float* p, int64_t cols, int vec) {
  int64_t c = threadIdx.x & 31;
  if (vec) {
    for (; c < cols / 4; c += 32) reinterpret_cast<float4*>(p)[c] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    c = cols / 4 * 4 + (threadIdx.x & 31);
  }
  for (; c < cols; c += 32) p[c] = 0.0f;
}
// A range of rows per CTA.  It follows the sort in the stream, runs beside it (on the other SMs: a CTA that sorts takes all registers of its own) and ends after it.
__global__ void __launch_bounds__(kZeroThreads, 2) emb_zero_kernel(const __grid_constant__ ZeroArgs a) {
  constexpr int kFlags = 32768;
  __shared__ uint8_t s_seen[kFlags];
  const int64_t per = (a.rows + gridDim.x - 1) / gridDim.x, begin = (int64_t)blockIdx.x * per, end = min(begin + per, a.rows);
  for (int64_t r0 = begin; r0 < end; r0 += kFlags) {
    const int count = (int)min((int64_t)kFlags, end - r0);
    for (int i = threadIdx.x; i < count; i += kZeroThreads) s_seen[i] = 0;
    __syncthreads();
    auto see = [&](int64_t id) { if (id >= r0 && id < r0 + count && id != a.padding) s_seen[id - r0] = 1; };
    int64_t done = 0;                                            // ids 16 bytes at a time, as far as they lie so
    if (a.wide_ids) {
      const int each = a.ids.wide ? 2 : 4;
      const int64_t quads = a.n / each;
#pragma unroll 8
      for (int64_t q = threadIdx.x; q < quads; q += kZeroThreads) {
        const int4 v = reinterpret_cast<const int4*>(a.ids.p)[q];
        if (a.ids.wide) { see((int64_t)v.y << 32 | (uint32_t)v.x); see((int64_t)v.w << 32 | (uint32_t)v.z); }
        else { see(v.x); see(v.y); see(v.z); see(v.w); }
      }
      done = quads * each;
    }
    for (int64_t t = done + threadIdx.x; t < a.n; t += kZeroThreads) see(load_id(a.ids, t));
    __syncthreads();
    for (int r = threadIdx.x >> 5; r < count; r += kZeroThreads / 32) if (!s_seen[r]) zero_row(a.out + (r0 + r) * a.ld_out, a.cols, a.vec_out);
    __syncthreads();
  }
  wait_for_previous();                   // so that what follows this kernel follows the sort too
}

// ONE: a CTA's segment fits one tile: its items stay in registers between ranking and writing, and between passes in the shared memory of the CTAs that
// rank them next.  Longer lists go through L2, a tile at a time.  (Lanes with equal digits are found by eight votes: the match instruction took
// 1.3 k cycles per item and warp of a CTA of 32.)
template <bool ONE>
__global__ void __launch_bounds__(kSortThreads, 1) emb_sort_kernel(const __grid_constant__ SortArgs a) {
  extern __shared__ uint64_t s_items[];                          // [kSortTile] the tile in order; ONE: [kSortTile] what the next pass ranks
  uint64_t* s_next = s_items + kSortTile;
  __shared__ __align__(16) uint16_t s_warp[kSortWarps][256];     // a digit's items per warp, then before the warp
  __shared__ uint32_t s_hist[256], s_base[256], s_tile[256], s_first[256], s_scan[2][8];   // s_first: of a digit in the ordered tile
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t begin = min((int64_t)blockIdx.x * a.segment, a.n), end = min(begin + a.segment, a.n);
  if (a.beside) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0 && tid == 0) a.runs[0] = 0;
  uint64_t item[kSortItems];
  uint32_t rank[kSortItems];
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = 32 + pass * a.bits;
    const uint32_t mask = (1u << a.bits) - 1u;
    const uint64_t* src = a.items[pass & 1];
    uint64_t* dst = a.items[(pass + 1) & 1];
    const bool last = pass + 1 == a.passes;
    // items of a tile: warp by warp, each 32 x `per` of them in order
    auto load_tile = [&](int64_t t0) {
      const int per = (int)((min((int64_t)kSortTile, end - t0) + kSortThreads - 1) / kSortThreads);
#pragma unroll
      for (int j = 0; j < kSortItems; ++j) {
        if (j < per) {
          const int64_t t = t0 + (int64_t)warp * 32 * per + j * 32 + lane;
          item[j] = t < end ? (pass == 0 ? sort_item(a, t) : ONE ? s_next[t - begin] : src[t]) : 0u;
        }
      }
      return per;
    };
    // rank of every item among those of its digit in its warp; s_warp = items of a digit in the warps before, s_tile = in the tile
    auto rank_tile = [&](int64_t t0, int per) {
      reinterpret_cast<uint4*>(s_warp[warp])[lane] = make_uint4(0u, 0u, 0u, 0u);
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kSortItems; ++j) {
        if (j < per) {
          const bool valid = t0 + (int64_t)warp * 32 * per + j * 32 + lane < end;
          const uint32_t digit = (uint32_t)(item[j] >> shift) & mask;
          uint32_t peers = __ballot_sync(0xffffffffu, valid);              // lanes with the same digit
#pragma unroll
          for (int b = 0; b < 8; ++b) {
            const uint32_t set = __ballot_sync(0xffffffffu, digit >> b & 1u);
            peers &= digit >> b & 1u ? set : ~set;
          }
          const uint32_t below = __popc(peers & ((1u << lane) - 1u));
          uint32_t before = 0u;
          if (valid) before = s_warp[warp][digit];
          __syncwarp();
          if (valid && below == 0u) s_warp[warp][digit] = (uint16_t)(before + __popc(peers));
          __syncwarp();
          rank[j] = before + below;
        }
      }
      __syncthreads();
      if (tid < 256) {
        uint32_t run = 0;
#pragma unroll 16
        for (int w = 0; w < kSortWarps; ++w) { const uint32_t c = s_warp[w][tid]; s_warp[w][tid] = (uint16_t)run; run += c; }
        s_tile[tid] = run;
      }
    };
    // exclusive sums over the 256 digits of v, by the first 256 threads; all threads meet
    auto scan = [&](uint32_t v, uint32_t* s) {
      uint32_t x = v;
      if (tid < 256) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t y = __shfl_up_sync(0xffffffffu, x, o); if (lane >= o) x += y; }
        if (lane == 31) s[warp] = x;
      }
      __syncthreads();
      if (tid < 256) for (int w = 0; w < warp; ++w) x += s[w];
      return x - v;
    };
    // the tile in order into shared memory, from there in runs to its places (s_base: the digit's first)
    auto write_tile = [&](int64_t t0, int per) {
      const uint32_t first = scan(tid < 256 ? s_tile[tid] : 0u, s_scan[0]);
      if (tid < 256) s_first[tid] = first;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kSortItems; ++j) {
        if (j < per && t0 + (int64_t)warp * 32 * per + j * 32 + lane < end) {
          const uint32_t digit = (uint32_t)(item[j] >> shift) & mask;
          s_items[s_first[digit] + s_warp[warp][digit] + rank[j]] = item[j];
        }
      }
      __syncthreads();
      const int count = (int)min((int64_t)kSortTile, end - t0);
#pragma unroll
      for (int j = 0; j < kSortItems; ++j) {
        const int i = j * kSortThreads + tid;
        if (i < count) {
          const uint64_t x = s_items[i];
          const uint32_t digit = (uint32_t)(x >> shift) & mask;
          const uint32_t at = s_base[digit] + (i - s_first[digit]);
          if (ONE && !last) {
            const uint32_t cta = at / (uint32_t)a.segment;
            put_remote(s_next + (at - cta * (uint32_t)a.segment), cta, x);
          } else dst[at] = x;
        }
      }
    };
    int per = 0;
    if (tid < 256) s_hist[tid] = 0u;
    if constexpr (ONE) {
      if (begin < end) { per = load_tile(begin); rank_tile(begin, per); if (tid < 256) s_hist[tid] = s_tile[tid]; }
    } else {
      for (int64_t t0 = begin; t0 < end; t0 += kSortTile) {
        per = load_tile(t0); rank_tile(t0, per);
        if (tid < 256) s_hist[tid] += s_tile[tid];
        __syncthreads();
      }
    }
    cluster_sync();
    // first place of this CTA's items of a digit: all items of smaller digits, and those of this one in the CTAs before
    uint32_t below = 0, total = 0;
    if (tid < 256) {
#pragma unroll
      for (uint32_t b = 0; b < kSortClusterMax; ++b) {
        if (b < a.ctas) { const uint32_t c = remote_u32(&s_hist[tid], b); if (b < blockIdx.x) below += c; total += c; }
      }
    }
    const uint32_t smaller = scan(total, s_scan[1]);
    if (tid < 256) s_base[tid] = smaller + below;
    if constexpr (ONE) {
      if (begin < end) write_tile(begin, per);
    } else {
      __syncthreads();
      for (int64_t t0 = begin; t0 < end; t0 += kSortTile) {
        per = load_tile(t0); rank_tile(t0, per);
        __syncthreads();
        write_tile(t0, per);
        __syncthreads();
        if (tid < 256) s_base[tid] += s_tile[tid];
        __syncthreads();
      }
    }
    cluster_sync();
  }
  // the long runs, by the chunk that they start in
  const uint64_t* items = a.items[a.passes & 1];
  const int64_t chunks = (a.n + kEmbChunk - 1) / kEmbChunk;
  for (int64_t c = (int64_t)blockIdx.x * kSortThreads + tid; c + 2 < chunks; c += (int64_t)a.ctas * kSortThreads) {
    const uint32_t k = item_id(items, (c + 1) * kEmbChunk - 1);
    if (k < (uint32_t)a.rows && item_id(items, (c + 2) * kEmbChunk) == k && (c == 0 || item_id(items, c * kEmbChunk - 1) != k)) a.runs[1 + atomicAdd(&a.runs[0], 1u)] = (uint32_t)c;
  }
}

// ---- sums -----------------------------------------------------------------------------------------
struct SumArgs {
  const uint64_t* items; const uint32_t* runs;
  int64_t n, chunks, rows, cols;
  const void* dout; int64_t ld;
  float scale; int accumulate;
  float* out; int64_t ld_out;
  float* parts; int64_t ld_part;       // [chunks][2][ld_part]: the part of a long run that came over the chunk's start, of one that goes over its end
  int vec_out;                         // out may be moved 16 bytes at a time
};

// V columns of a row of the gradient
template <int V>
__device__ __forceinline__ void put_row(const SumArgs& a, float* p, const float (&x)[V]) {
  if (V % 4 == 0 && a.vec_out) {
#pragma unroll
    for (int j = 0; j + 3 < V; j += 4) {
      float4 y = make_float4(a.scale * x[j], a.scale * x[j + 1], a.scale * x[j + 2], a.scale * x[j + 3]);
      if (a.accumulate) { const float4 o = *reinterpret_cast<const float4*>(p + j); y.x += o.x; y.y += o.y; y.z += o.z; y.w += o.w; }
      *reinterpret_cast<float4*>(p + j) = y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) p[j] = a.accumulate ? p[j] + a.scale * x[j] : a.scale * x[j];
  }
}

// A thread's packs of the gradient's rows on their way: AHEAD rows, each thread's own, so that it waits for nobody else's.  They are copied to shared memory
// asynchronously, which takes no registers; a 16-bit value with the whole word that it lies in.
// (Sums of 30000 tokens of 1023 bf16 columns, us: one value per thread, loaded and stored, 103; four values per thread, copied in their words, 55.  10033 tokens of
// 1155 fp32 columns: 27 and 20.)
template <typename T, int VEC, int AHEAD>
struct RowQueue {
  static constexpr int kBytes = VEC * (int)sizeof(T), kCell = kBytes < 4 ? 4 : kBytes;
  static constexpr int kPacks = look_packs<T, VEC>(), kPitch = kEmbThreads * kCell;    // of a thread; bytes between two of its cells
  static constexpr size_t kSize = (size_t)AHEAD * kPacks * kPitch;
  uint8_t* slot;
  __device__ __forceinline__ uint8_t* cell(int turn, int k) const { return slot + turn * (kPacks * kPitch) + k * kPitch; }
  // edge: the word may lie outside the matrix
  __device__ __forceinline__ void put(int turn, int k, const T* p, bool edge) {
    if constexpr (kBytes >= 4) copy_async<kBytes>(cell(turn, k), p);
    else {
      const uintptr_t at = reinterpret_cast<uintptr_t>(p);
      if (edge) *reinterpret_cast<T*>(cell(turn, k) + (at & 2)) = *p;
      else copy_async<4>(cell(turn, k), reinterpret_cast<const void*>(at & ~(uintptr_t)3));
    }
  }
  __device__ __forceinline__ void close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" :: "n"(AHEAD - 1) : "memory"); }
  // low: of the pack's address in global memory
  __device__ __forceinline__ Pack<T, VEC> get(int turn, int k, uint32_t low) const {
    return *reinterpret_cast<const Pack<T, VEC>*>(cell(turn, k) + (kBytes < 4 ? low & 2u : 0u));
  }
};

constexpr int kEmbAhead = 12, kWindow = 3 * kEmbChunk + 2;
template <typename T, int VEC>
__global__ void __launch_bounds__(kEmbThreads, 4) emb_sum_kernel(const __grid_constant__ SumArgs a) {
  extern __shared__ uint4 s_raw[];     // [kEmbAhead][threads] packs or words, then [cy][kWindow] items
  wait_for_previous();
  const int tid = threadIdx.y * blockDim.x + threadIdx.x, threads = blockDim.x * blockDim.y;
  using Queue = RowQueue<T, VEC, kEmbAhead>;
  constexpr int P = Queue::kPacks;
  const int col = (blockIdx.y * P * blockDim.x + threadIdx.x) * VEC, hop = blockDim.x * VEC, cols = (int)a.cols;       // hop: between a thread's packs
  bool in[P];                                                    // the packs that lie inside the row
#pragma unroll
  for (int k = 0; k < P; ++k) in[k] = col + k * hop < cols;
  uint64_t* s_items = reinterpret_cast<uint64_t*>(reinterpret_cast<uint8_t*>(s_raw) + Queue::kSize);
  for (int i = tid; i < (int)blockDim.y * kWindow; i += threads) {
    const int64_t at = ((int64_t)blockIdx.x * blockDim.y + i / kWindow - 1) * kEmbChunk + i % kWindow - 1;
    s_items[i] = at >= 0 && at < a.n ? a.items[at] : ~0ull;
  }
  __syncthreads();
  const int64_t chunk = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (chunk >= a.chunks || !in[0]) return;
  const int64_t first = chunk * kEmbChunk;
  const uint64_t* items = s_items + threadIdx.y * kWindow + kEmbChunk + 1;      // of this chunk; a chunk and one token before, two chunks behind
  auto id_at = [&](int i) { return (uint32_t)(items[i] >> 32); };
  int begin = 0, end = (int)min((int64_t)kEmbChunk, a.n - first);
  // the run at the chunk's start: skipped if the chunk before sums it, else a part; the one at its end: followed into the next chunk, or a part
  const uint32_t head = id_at(0), tail = id_at(end - 1);
  const bool head_part = id_at(-1) == head;
  bool tail_part = false;
  if (head_part && id_at(kEmbChunk) != head && id_at(-kEmbChunk - 1) != head) {
    while (begin < end && id_at(begin) == head) ++begin;
  }
  if (end == kEmbChunk && tail < (uint32_t)a.rows && id_at(kEmbChunk) == tail && !(head_part && head == tail)) {
    tail_part = id_at(2 * kEmbChunk) == tail;
    if (!tail_part) while (end < 2 * kEmbChunk && id_at(end) == tail) ++end;
  }
  while (begin < end && id_at(end - 1) >= (uint32_t)a.rows) --end;             // tokens that are left out come last
  if (begin >= end) return;
  const T* dout = static_cast<const T*>(a.dout) + col;
  Queue queue{reinterpret_cast<uint8_t*>(s_raw) + tid * Queue::kCell};
  auto fetch = [&](int i, int turn) {
    const uint32_t token = (uint32_t)items[i];
    const T* row = dout + (int64_t)token * a.ld;
    const bool edge = token == 0u || token == (uint32_t)(a.n - 1);
#pragma unroll
    for (int k = 0; k < P; ++k) if (in[k]) queue.put(turn, k, row + k * hop, edge);
  };
#pragma unroll
  for (int i = 0; i < kEmbAhead - 1; ++i) {
    if (begin + i < end) fetch(begin + i, i);
    queue.close();
  }
  float acc[P][VEC];
  auto clear = [&] {
#pragma unroll
    for (int k = 0; k < P; ++k) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[k][j] = 0.0f;
    }
  };
  clear();
  uint32_t run = id_at(begin);
  bool part = head_part && begin == 0;
  auto flush = [&](int slot) {
#pragma unroll
    for (int k = 0; k < P; ++k) {
      if (!in[k]) continue;
      if (slot >= 0) {
        float* p = a.parts + (chunk * 2 + slot) * a.ld_part + col + k * hop;
#pragma unroll
        for (int j = 0; j < VEC; ++j) p[j] = acc[k][j];
      } else put_row<VEC>(a, a.out + (int64_t)run * a.ld_out + col + k * hop, acc[k]);
    }
  };
  int turn = 0;
  for (int i = begin; i < end; ++i) {
    if (i + kEmbAhead - 1 < end) fetch(i + kEmbAhead - 1, turn == 0 ? kEmbAhead - 1 : turn - 1);
    queue.close();
    queue.wait();
    const uint32_t id = id_at(i);
    if (id != run) {
      flush(part ? 0 : -1);
      run = id; part = false;
      clear();
    }
    const uint32_t low = (uint32_t)reinterpret_cast<uintptr_t>(dout) + (uint32_t)items[i] * (uint32_t)a.ld * (uint32_t)sizeof(T);      // (of all packs: the hop is a multiple of four bytes)
#pragma unroll
    for (int k = 0; k < P; ++k) {
      const Pack<T, VEC> x = queue.get(turn, k, low);
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[k][j] += to_float(x.v[j]);
    }
    turn = turn + 1 == kEmbAhead ? 0 : turn + 1;
  }
  flush(part ? 0 : tail_part ? 1 : -1);
}

// A CTA adds the parts of one long run for 128 columns: eight slices of the run's chunks, then the slices.  A thread copies ten parts at a time to shared memory
// asynchronously (of loads to registers the compiler kept one under way: 20 k cycles for a run of 294 chunks, 21 us in all).
constexpr int kJoinSlices = 8, kJoinAhead = 10;
__global__ void __launch_bounds__(32 * kJoinSlices) emb_join_kernel(const __grid_constant__ SumArgs a) {
  __shared__ float4 s_part[kJoinSlices][32], s_ahead[kJoinAhead][kJoinSlices][32];
  wait_for_previous();
  const int64_t slabs = (a.cols + 127) / 128, units = (int64_t)a.runs[0] * slabs;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t c0 = a.runs[1 + unit / slabs], col = (unit % slabs) * 128 + threadIdx.x * 4;
    const uint32_t k = item_id(a.items, (c0 + 1) * kEmbChunk - 1);
    int64_t count = 1;                                            // the chunks that have a part: those that start with this id (the ids ascend)
    for (;;) {
      const int64_t c = c0 + count + threadIdx.y * 32 + threadIdx.x;
      const int more = __syncthreads_count(c < a.chunks && item_id(a.items, c * kEmbChunk) == k);
      count += more;
      if (more < 32 * kJoinSlices) break;
    }
    const int64_t per = (count + kJoinSlices - 1) / kJoinSlices;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (col < a.cols) {
      const int64_t i1 = min(count, (threadIdx.y + 1) * per);
      const float* p = a.parts + c0 * 2 * a.ld_part + col;       // slot 1 of the first chunk, slot 0 of the others
      for (int64_t i = threadIdx.y * per; i < i1; i += kJoinAhead) {
        const int n = (int)min((int64_t)kJoinAhead, i1 - i);
        for (int u = 0; u < n; ++u) copy_async<16>(&s_ahead[u][threadIdx.y][threadIdx.x], p + ((i + u) * 2 + (i + u == 0)) * a.ld_part);
        asm volatile("cp.async.wait_all;" ::: "memory");
        for (int u = 0; u < n; ++u) { const float4 x = s_ahead[u][threadIdx.y][threadIdx.x]; acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w; }
      }
    }
    s_part[threadIdx.y][threadIdx.x] = acc;
    __syncthreads();
    if (threadIdx.y == 0 && col < a.cols) {
      float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < kJoinSlices; ++s) { const float4 v = s_part[s][threadIdx.x]; x[0] += v.x; x[1] += v.y; x[2] += v.z; x[3] += v.w; }
      float* p = a.out + (int64_t)k * a.ld_out + col;
      if (col + 3 < a.cols) put_row<4>(a, p, x);
      else {
#pragma unroll
        for (int j = 0; j < 3; ++j) if (col + j < a.cols) { const float y[1] = {x[j]}; put_row<1>(a, p + j, y); }
      }
    }
    __syncthreads();
  }
}

// ---- short lists, in one launch -------------------------------------------------------------------
constexpr int kDirectThreads = 512, kDirectWarps = kDirectThreads / 32, kDirectBits = 12, kDirectMost = 1 << kDirectBits;   // tokens at most
constexpr int kDirectRows = 8192;                                // rows of a CTA's stretch, at most
struct DirectArgs {
  Ids ids; int n, padded; int64_t rows, cols, padding;           // padded: a power of two that holds n
  const void* dout; int64_t ld;
  float scale; int accumulate;
  float* out; int64_t ld_out; int vec_out;
  int32_t* status; int per;                                      // rows of a CTA's stretch
};
template <typename T, int VEC> struct DirectShape {              // columns of a CTA: 32 lanes, at least four columns each
  static constexpr int kPacks = VEC >= 4 ? 1 : 4 / VEC, kCols = 32 * VEC * kPacks;
};

template <typename T, int VEC>
__global__ void __launch_bounds__(kDirectThreads, 2) emb_direct_kernel(const __grid_constant__ DirectArgs a) {
  constexpr int PACKS = DirectShape<T, VEC>::kPacks, COLS = DirectShape<T, VEC>::kCols, kAhead = VEC * sizeof(T) == 16 && sizeof(T) == 2 ? 4 : 8;
  extern __shared__ __align__(16) uint32_t s_keys[];             // [padded] row << kDirectBits | token; then [2][warps][COLS] parts of runs, a flag per row
  float* s_part = reinterpret_cast<float*>(s_keys + a.padded);
  uint8_t* s_seen = reinterpret_cast<uint8_t*>(s_part + 2 * kDirectWarps * COLS);
  __shared__ int s_count, s_row[2][kDirectWarps + 1];            // rows of the parts, -1: none
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t c0 = (int64_t)blockIdx.y * COLS;
  const uint32_t hop = gridDim.x;                                // between two rows of this CTA, the first of which is blockIdx.x
  const int64_t z0 = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * a.per;
  const int rows = a.accumulate ? 0 : (int)max((int64_t)0, min((int64_t)a.per, a.rows - z0));     // of its stretch
  auto row_at = [&](int i) { return a.out + ((int64_t)i * hop + blockIdx.x) * a.ld_out + c0; };
  for (int i = tid; i < (rows + 3) / 4; i += kDirectThreads) reinterpret_cast<uint32_t*>(s_seen)[i] = 0u;
  if (tid == 0) s_count = 0;
  if (tid <= kDirectWarps) s_row[0][tid] = s_row[1][tid] = -1;
  __syncthreads();
  // the tokens of these rows, in any order
  int64_t id[kDirectMost / kDirectThreads];
#pragma unroll
  for (int i = 0; i < kDirectMost / kDirectThreads; ++i) { const int t = i * kDirectThreads + tid; id[i] = t < a.n ? load_id(a.ids, t) : -1; }
#pragma unroll
  for (int i = 0; i < kDirectMost / kDirectThreads; ++i) {
    const int t = i * kDirectThreads + tid;
    if (i * kDirectThreads >= a.n) break;
    const bool valid = id[i] >= 0 && id[i] < a.rows;
    if (t < a.n && !valid && blockIdx.x == 0 && blockIdx.y == 0) raise_word(a.status);
    const uint32_t row = (uint32_t)id[i] / hop;
    const bool taken = valid && id[i] != a.padding, mine = taken && (uint32_t)id[i] - row * hop == blockIdx.x;
    const uint32_t ballot = __ballot_sync(0xffffffffu, mine);
    if (ballot != 0u) {
      int at = 0;
      if (lane == 0) at = atomicAdd(&s_count, __popc(ballot));
      at = __shfl_sync(0xffffffffu, at, 0);
      if (mine) s_keys[at + __popc(ballot & ((1u << lane) - 1u))] = row << kDirectBits | (uint32_t)t;
    }
    if (taken && id[i] >= z0 && id[i] < z0 + rows) s_seen[id[i] - z0] = 1;
  }
  __syncthreads();
  // all keys differ, so that any way to sort them gives the same order: rows, and in a row the tokens, ascending.  Up to 256 a thread counts the keys below
  // its own; more are sorted in a network.
  const int count = s_count;
  if (count <= 256) {
    uint32_t mine = 0;
    int below = 0;
    const int quads = (count + 3) / 4;
    if (tid >= count && tid < quads * 4) s_keys[tid] = 0xffffffffu;
    __syncthreads();
    if (tid < count) {
      mine = s_keys[tid];
      for (int q = 0; q < quads; ++q) {
        const uint4 k = reinterpret_cast<const uint4*>(s_keys)[q];
        below += (k.x < mine) + (k.y < mine) + (k.z < mine) + (k.w < mine);
      }
    }
    __syncthreads();
    if (tid < count) s_keys[below] = mine;
    __syncthreads();
  } else {
    int size = 512;
    while (size < count) size <<= 1;
    for (int i = count + tid; i < size; i += kDirectThreads) s_keys[i] = 0xffffffffu;
    __syncthreads();
    for (int k = 2; k <= size; k <<= 1) {
      for (int j = k >> 1; j > 0; j >>= 1) {
        for (int p = tid; p < size / 2; p += kDirectThreads) {
          const int i = 2 * p - (p & (j - 1)), l = i + j;
          const uint32_t x = s_keys[i], y = s_keys[l];
          if ((x > y) == ((i & k) == 0)) { s_keys[i] = y; s_keys[l] = x; }
        }
        __syncthreads();
      }
    }
  }
  // a warp sums a stretch of the sorted tokens; runs that go over its ends leave parts
  const T* dout = static_cast<const T*>(a.dout) + c0;
  auto inside = [&](int p) { return c0 + (p * 32 + lane) * VEC < a.cols; };
  float acc[PACKS][VEC];
  auto clear = [&] {
#pragma unroll
    for (int p = 0; p < PACKS; ++p) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[p][j] = 0.0f;
    }
  };
  const SumArgs put{nullptr, nullptr, 0, 0, a.rows, a.cols, nullptr, 0, a.scale, a.accumulate, a.out, a.ld_out, nullptr, 0, a.vec_out};
  const int stretch = (count + kDirectWarps - 1) / kDirectWarps, begin = min(warp * stretch, count), end = min(begin + stretch, count);
  if (begin < end) {
    int run = (int)(s_keys[begin] >> kDirectBits);
    bool part = begin > 0 && (int)(s_keys[begin - 1] >> kDirectBits) == run;
    auto flush = [&](int slot) {
      if (slot >= 0) {
        if (lane == 0) s_row[slot][warp] = run;
#pragma unroll
        for (int p = 0; p < PACKS; ++p) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) s_part[(slot * kDirectWarps + warp) * COLS + (p * 32 + lane) * VEC + j] = acc[p][j];
        }
      } else {
#pragma unroll
        for (int p = 0; p < PACKS; ++p) if (inside(p)) put_row<VEC>(put, row_at(run) + (p * 32 + lane) * VEC, acc[p]);
      }
    };
    clear();
    for (int i0 = begin; i0 < end; i0 += kAhead) {
      Pack<T, VEC> x[kAhead][PACKS];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int64_t token = i0 + u < end ? (int64_t)(s_keys[i0 + u] & (kDirectMost - 1)) : 0;
#pragma unroll
        for (int p = 0; p < PACKS; ++p) if (i0 + u < end && inside(p)) x[u][p] = load_pack<T, VEC>(dout + token * a.ld + (p * 32 + lane) * VEC);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (i0 + u < end) {
          const int row = (int)(s_keys[i0 + u] >> kDirectBits);
          if (row != run) { flush(part ? 0 : -1); run = row; part = false; clear(); }
#pragma unroll
          for (int p = 0; p < PACKS; ++p) {
            if (inside(p)) {
#pragma unroll
              for (int j = 0; j < VEC; ++j) acc[p][j] += to_float(x[u][p].v[j]);
            }
          }
        }
      }
    }
    flush(part ? 0 : end < count && (int)(s_keys[end] >> kDirectBits) == run ? 1 : -1);
  }
  // (last: before the sums, whose loads then wait behind these stores, the whole took a tenth longer)
  for (int r = warp; r < rows; r += kDirectWarps) if (!s_seen[r]) zero_row(a.out + (z0 + r) * a.ld_out, a.cols, a.vec_out);
  // the runs that went over: their parts in order, a thread per column
  __syncthreads();
  if (tid < COLS && c0 + tid < a.cols) {
    float sum[1] = {0.0f};
    for (int w = 0; w < kDirectWarps; ++w) {
      const int over = s_row[0][w];
      if (over >= 0) {
        sum[0] += s_part[w * COLS + tid];
        if (s_row[0][w + 1] != over) put_row<1>(put, row_at(over) + tid, sum);
      }
      if (s_row[1][w] >= 0) sum[0] = s_part[(kDirectWarps + w) * COLS + tid];
    }
  }
}

// columns that a thread moves in one piece: 16 bytes where base, leading dimension and length allow it, for 16-bit types also 4 bytes
int emb_vec(const void* base, int64_t ld, int64_t cols, int size) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(base);
  for (int bytes = 16; bytes > size; bytes = bytes == 16 ? 4 : size)
    if (p % bytes == 0 && (ld * size) % bytes == 0 && (cols * size) % bytes == 0) return bytes / size;
  return 1;
}

template <typename T, int VEC>
cudaError_t lookup_typed(const EmbLookup& a, cudaStream_t st) {
  const EmbShape s = emb_shape(a.cols, VEC * look_packs<T, VEC>());
  const dim3 block(s.cx, s.cy);
  // several tokens at a time from where so many fewer threads still fill the GPU
  const bool many = a.n * s.slabs * s.cx / kLookTokens >= 148 * 2048;
  const int64_t per = (int64_t)s.cy * (many ? kLookTokens : 1);
  const dim3 grid((unsigned)std::min<int64_t>((a.n + per - 1) / per, many ? std::max(1, 148 * kLookCtas / s.slabs) : (int64_t)1 << 30), s.slabs);
  const Ids ids{a.ids, a.id_bytes == 8};
  if (many) emb_lookup_kernel<T, VEC, kLookTokens><<<grid, block, 0, st>>>((const T*)a.table, a.rows, a.cols, a.ld, ids, a.n, a.scale, (T*)a.out, a.ld_out, a.status);
  else emb_lookup_kernel<T, VEC, 1><<<grid, block, 0, st>>>((const T*)a.table, a.rows, a.cols, a.ld, ids, a.n, a.scale, (T*)a.out, a.ld_out, a.status);
  return cudaGetLastError();
}
template <typename T>
cudaError_t lookup_type(const EmbLookup& a, cudaStream_t st) {
  const int vec = std::min(emb_vec(a.table, a.ld, a.cols, sizeof(T)), emb_vec(a.out, a.ld_out, a.cols, sizeof(T)));
  if (vec == 16 / (int)sizeof(T)) return lookup_typed<T, 16 / sizeof(T)>(a, st);
  if constexpr (sizeof(T) == 2) { if (vec == 2) return lookup_typed<T, 2>(a, st); }
  return lookup_typed<T, 1>(a, st);
}

struct EmbLayout { uint64_t items[2], runs, parts, bytes; int64_t chunks, ld_part; };
EmbLayout emb_layout(int64_t n, int64_t cols) {
  EmbLayout l{};
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t p = at; at = align_up(at + bytes, 256); return p; };
  l.chunks = (n + kEmbChunk - 1) / kEmbChunk;
  l.ld_part = (cols + 3) / 4 * 4;
  for (int i = 0; i < 2; ++i) l.items[i] = take((uint64_t)n * 8);
  l.runs = take((uint64_t)(l.chunks + 1) * 4);
  l.parts = take((uint64_t)l.chunks * 2 * l.ld_part * 4);
  l.bytes = at;
  return l;
}

struct SortLaunch {
  cudaLaunchAttribute attr[1];
  cudaLaunchConfig_t cfg = {};
  SortLaunch(int cluster, size_t smem, cudaStream_t st) {
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(cluster); cfg.blockDim = dim3(kSortThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st; cfg.attrs = attr; cfg.numAttrs = 1;
  }
  SortLaunch(const SortLaunch&) = delete;
};

template <typename T, int VEC>
cudaError_t sum_typed(SumArgs& a, cudaStream_t st) {
  using Queue = RowQueue<T, VEC, kEmbAhead>;
  const EmbShape s = emb_shape(a.cols, VEC * Queue::kPacks);
  const size_t smem = Queue::kSize + (size_t)s.cy * kWindow * 8;
  return launch_after(emb_sum_kernel<T, VEC>, dim3((unsigned)((a.chunks + s.cy - 1) / s.cy), s.slabs), dim3(s.cx, s.cy), smem, st, a);
}
template <typename T>
cudaError_t sum_type(SumArgs& a, cudaStream_t st) {
  const int vec = emb_vec(a.dout, a.ld, a.cols, sizeof(T));
  if (vec == 16 / (int)sizeof(T)) return sum_typed<T, 16 / sizeof(T)>(a, st);
  if constexpr (sizeof(T) == 2) { if (vec == 2) return sum_typed<T, 2>(a, st); }
  return sum_typed<T, 1>(a, st);
}

}  // namespace

namespace {
template <typename T, int VEC>
cudaError_t direct_typed(DirectArgs& a, cudaStream_t st) {
  constexpr int COLS = DirectShape<T, VEC>::kCols;
  const int slabs = (int)((a.cols + COLS - 1) / COLS);
  // two CTAs per SM; more where their stretches would get too long, or their rows' numbers not fit the keys
  int64_t ctas = std::max<int64_t>(1, std::min<int64_t>(a.rows, 2 * 148 / slabs));
  ctas = std::max({ctas, (a.rows + (int64_t)slabs * kDirectRows - 1) / ((int64_t)slabs * kDirectRows), (a.rows >> (32 - kDirectBits)) + 1});
  a.per = (int)((a.rows + ctas * slabs - 1) / (ctas * slabs));
  a.padded = 512;                                                // (the network's size, where it is used)
  while (a.padded < a.n) a.padded <<= 1;
  const size_t smem = (size_t)a.padded * 4 + (size_t)2 * kDirectWarps * COLS * 4 + (a.per + 3) / 4 * 4;
  emb_direct_kernel<T, VEC><<<dim3((unsigned)ctas, slabs), kDirectThreads, smem, st>>>(a);
  return cudaGetLastError();
}
template <typename T>
cudaError_t direct_type(DirectArgs& a, cudaStream_t st) {
  const int vec = emb_vec(a.dout, a.ld, a.cols, sizeof(T));
  if (vec == 16 / (int)sizeof(T)) return direct_typed<T, 16 / sizeof(T)>(a, st);
  if constexpr (sizeof(T) == 2) { if (vec == 2) return direct_typed<T, 2>(a, st); }
  return direct_typed<T, 1>(a, st);
}
}  // namespace

int embedding_configure(SortRoom* room) {
  cudaError_t e = cudaFuncSetAttribute(emb_sort_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortTile * 16);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(emb_sort_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortTile * 8);
  // up to 48 KB of packs in flight and 25 KB of items
  auto sum = [&](auto kernel) { if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 80 * 1024); };
  sum(emb_sum_kernel<float, 4>); sum(emb_sum_kernel<float, 1>);
  sum(emb_sum_kernel<__nv_bfloat16, 8>); sum(emb_sum_kernel<__nv_bfloat16, 2>); sum(emb_sum_kernel<__nv_bfloat16, 1>);
  sum(emb_sum_kernel<__half, 8>); sum(emb_sum_kernel<__half, 2>); sum(emb_sum_kernel<__half, 1>);
  // 16 KB of keys, 32 KB of parts and 8 KB of flags
  auto direct = [&](auto kernel) { if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 57 * 1024); };
  direct(emb_direct_kernel<float, 4>); direct(emb_direct_kernel<float, 1>);
  direct(emb_direct_kernel<__nv_bfloat16, 8>); direct(emb_direct_kernel<__nv_bfloat16, 2>); direct(emb_direct_kernel<__nv_bfloat16, 1>);
  direct(emb_direct_kernel<__half, 8>); direct(emb_direct_kernel<__half, 2>); direct(emb_direct_kernel<__half, 1>);
  if (e != cudaSuccess) return (int)e;
  const bool wide = cudaFuncSetAttribute(emb_sort_kernel<true>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                    cudaFuncSetAttribute(emb_sort_kernel<false>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
  for (int lg = 0; lg < kSortClusters; ++lg) {
    int clusters = 0;
    const SortLaunch l(1 << lg, kSortTile * 16, nullptr);
    if ((lg < 4 || wide) && cudaOccupancyMaxActiveClusters(&clusters, emb_sort_kernel<true>, &l.cfg) != cudaSuccess) clusters = 0;
    room->clusters[lg] = clusters;
  }
  cudaGetLastError();
  return 0;
}

int launch_embedding(const EmbLookup& a, cudaStream_t st) {
  if (a.n == 0) return (int)cudaSuccess;
  if (a.type == ATOMO_TYPE_F32) return (int)lookup_type<float>(a, st);
  if (a.type == ATOMO_TYPE_BF16) return (int)lookup_type<__nv_bfloat16>(a, st);
  return (int)lookup_type<__half>(a, st);
}

// One launch, or four.  Kernels alone, us, one | four (tokens x rows x columns, fp32): 256 x 21294 x 38 6 | 19, 1000 x 5000 x 64 6 | 24, 1000 x 32000 x 1024 27 | 34,
// 2000 x 32000 x 2048 56 | 57, 3000 x 32000 x 1024 36 | 36, 4000 x 16000 x 1024 28 | 27, 4000 x 50000 x 512 32 | 30, 4001 x 10007 x 515 22 | 25, 4000 x 32000 x 2048
// 66 | 59 (bf16 alike): a frequent id's tokens wait for one CTA, the longer the more there are and the wider they are.  The rule knows neither the rows, which move the
// crossing (4000 x 50000 x 512 takes the one launch, 2 us slower), nor the ids' distribution (these are Zipf's).  One launch spares the host 13 us a call.
static bool one_launch(int64_t n, int64_t cols) { return n <= 2048 || (n <= kDirectMost && n * cols <= 5 << 19); }
uint64_t embedding_workspace(int64_t n, int64_t cols) { return one_launch(n, cols) ? 0 : emb_layout(n, cols).bytes; }

int launch_embedding_backward(const EmbBackward& b, cudaStream_t st) {
  if (b.n == 0 && b.accumulate) return (int)cudaSuccess;
  const int vec_out = reinterpret_cast<uintptr_t>(b.out) % 16 == 0 && b.ld_out % 4 == 0;
  if (one_launch(b.n, b.cols)) {
    DirectArgs d{};
    d.ids = Ids{b.ids, b.id_bytes == 8}; d.n = (int)b.n; d.rows = b.rows; d.cols = b.cols; d.padding = b.padding; d.dout = b.grad; d.ld = b.ld;
    d.scale = b.scale; d.accumulate = b.accumulate; d.out = b.out; d.ld_out = b.ld_out; d.vec_out = vec_out; d.status = b.status;
    return (int)(b.type == ATOMO_TYPE_F32 ? direct_type<float>(d, st) : b.type == ATOMO_TYPE_BF16 ? direct_type<__nv_bfloat16>(d, st) : direct_type<__half>(d, st));
  }
  const EmbLayout l = emb_layout(b.n, b.cols);
  cudaError_t e = cudaSuccess;
  SortArgs s{};
  s.ids = Ids{b.ids, b.id_bytes == 8}; s.n = b.n; s.rows = b.rows; s.padding = b.padding; s.status = b.status;
  for (int i = 0; i < 2; ++i) s.items[i] = reinterpret_cast<uint64_t*>(b.ws + l.items[i]);
  s.runs = reinterpret_cast<uint32_t*>(b.ws + l.runs);
  int bits = 1;
  while ((b.rows >> bits) != 0) ++bits;                          // ids as sort keys are 0 .. rows
  s.passes = (bits + 7) / 8; s.bits = (bits + s.passes - 1) / s.passes;
  // a token per thread up to the cluster's size
  int lg = 0;
  while (lg + 1 < kSortClusters && ((int64_t)kSortThreads << lg) < b.n && b.room.clusters[lg + 1] > 0) ++lg;
  const int ctas = 1 << lg;
  s.ctas = (uint32_t)ctas;
  s.segment = (b.n + ctas - 1) / ctas;
  s.beside = !b.accumulate;
  const size_t smem = s.segment <= kSortTile ? kSortTile * 16 : kSortTile * 8;
  const SortLaunch launch(ctas, smem, st);
  e = s.segment <= kSortTile ? cudaLaunchKernelEx(&launch.cfg, emb_sort_kernel<true>, s) : cudaLaunchKernelEx(&launch.cfg, emb_sort_kernel<false>, s);
  if (e == cudaSuccess && s.beside) {    // a CTA on each of the other SMs, fewer where one would have less than 16 KB to write
    const ZeroArgs z{s.ids, b.n, b.rows, b.padding, b.cols, b.out, b.ld_out, vec_out, reinterpret_cast<uintptr_t>(b.ids) % 16 == 0};
    e = launch_after(emb_zero_kernel, dim3((unsigned)std::min<int64_t>(148 - ctas, std::max<int64_t>(1, b.rows * b.cols / 4096))), dim3(kZeroThreads), 0, st, z);
  }
  if (e != cudaSuccess) return (int)e;
  SumArgs a{};
  a.items = s.items[s.passes & 1]; a.runs = s.runs;
  a.n = b.n; a.chunks = l.chunks; a.rows = b.rows; a.cols = b.cols;
  a.dout = b.grad; a.ld = b.ld; a.scale = b.scale; a.accumulate = b.accumulate; a.out = b.out; a.ld_out = b.ld_out; a.vec_out = vec_out;
  a.parts = reinterpret_cast<float*>(b.ws + l.parts); a.ld_part = l.ld_part;
  e = b.type == ATOMO_TYPE_F32 ? sum_type<float>(a, st) : b.type == ATOMO_TYPE_BF16 ? sum_type<__nv_bfloat16>(a, st) : sum_type<__half>(a, st);
  if (e != cudaSuccess) return (int)e;
  const int64_t units = (l.chunks / 2) * ((b.cols + 127) / 128);
  return (int)launch_after(emb_join_kernel, dim3((unsigned)std::min<int64_t>(units, 148 * 8)), dim3(32, kJoinSlices), 0, st, a);
}

}  // namespace atomo
