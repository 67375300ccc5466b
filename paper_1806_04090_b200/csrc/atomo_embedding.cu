// Embedding lookup, and the gradient of the table by sorted tokens.
//
//   out[t] = s table[id[t]],   dtable[v] = s sum_{t : id[t] = v} dout[t]
//
// The gradient's sums run in the order of the tokens, so that the same call gives the same bits each time (a payload that is encoded
// from it does too), which sums by atomics would not.  Three kernels:
//   emb_sort_kernel   stable radix sort of (id, token), eight bits a pass, by the CTAs of one cluster: they exchange their histograms
//                     through distributed shared memory and their items through L2, with the hardware cluster barrier between.  It also
//                     marks the rows that have tokens and lists the runs of equal ids that go over the end of a chunk.
//   emb_sum_kernel    chunks of kEmbChunk neighbouring sorted tokens, so that a frequent token's run is split among CTAs: the sum of a run that lies
//                     within a chunk goes to its row, the parts of longer ones to the workspace; other CTAs write the rows without tokens.
//   emb_join_kernel   adds the parts of the longer runs, in order.
// What bounds it is memory: dout is read once, the table's gradient written once.
#include <algorithm>

#include "atomo_ops.cuh"

namespace atomo {
namespace {

constexpr int kEmbThreads = 256;
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortItems = 8, kSortTile = kSortThreads * kSortItems;
constexpr int kSortCluster = 8;

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
    s.cx = 4;                                                    // at most 64 rows, whose chunks' entries take 16 KB of shared memory
    while (s.cx < packs) s.cx <<= 1;
    s.cy = kEmbThreads / s.cx; s.slabs = 1;
  } else {
    s.slabs = (int)((packs + kEmbThreads - 1) / kEmbThreads);
    s.cx = (int)(((packs + s.slabs - 1) / s.slabs + 31) / 32 * 32); s.cy = 1;
  }
  return s;
}

// ---- lookup ---------------------------------------------------------------------------------------
template <typename T, int VEC, int U>
__global__ void __launch_bounds__(kEmbThreads) emb_lookup_kernel(const T* __restrict__ table, int64_t rows, int64_t cols, int64_t ld, Ids ids, int64_t n,
                                                                 float scale, T* __restrict__ out, int64_t ld_out, int32_t* status) {
  const int64_t col = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * VEC;
  const int64_t t0 = (int64_t)blockIdx.x * U * blockDim.y + threadIdx.y;
  int64_t id[U];
#pragma unroll
  for (int u = 0; u < U; ++u) { const int64_t t = t0 + (int64_t)u * blockDim.y; id[u] = t < n ? load_id(ids, t) : -1; }
  if (col >= cols) return;
  Pack<T, VEC> x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (id[u] >= 0 && id[u] < rows) x[u] = load_pack<T, VEC>(table + id[u] * ld + col);
    else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) x[u].v[j] = from_float<T>(0.0f);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t t = t0 + (int64_t)u * blockDim.y;
    if (t >= n) break;
    if ((id[u] < 0 || id[u] >= rows) && col == 0) raise_word(status);
#pragma unroll
    for (int j = 0; j < VEC; ++j) x[u].v[j] = from_float<T>(to_float(x[u].v[j]) * scale);
    store_pack<T, VEC>(out + t * ld_out + col, x[u]);
  }
}

// ---- sort -----------------------------------------------------------------------------------------
struct SortArgs {
  Ids ids; int64_t n, rows, padding;
  uint32_t *keys[2], *toks[2];          // the sorted pairs end in [passes & 1]
  uint8_t* touched;                     // [rows] rows that have tokens
  uint32_t* runs;                       // [0] number of runs that go over a chunk's end, then the chunks that they start in
  int32_t* status;
  int passes, bits;
  int64_t segment;                      // tokens of a CTA
};

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote_u32(const uint32_t* local, uint32_t rank) {
  uint32_t a = (uint32_t)__cvta_generic_to_shared(local), r, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(r) : "memory");
  return v;
}

// an id as a sort key: ids that have no row, and the padding id, come last
__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, int64_t t) {
  const int64_t id = load_id(a.ids, t);
  const bool ok = id >= 0 && id < a.rows;
  if (!ok) raise_word(a.status);
  return ok && id != a.padding ? (uint32_t)id : (uint32_t)a.rows;
}

// ONE: a CTA's segment fits one tile, whose ranks stay in registers
template <bool ONE>
__global__ void __launch_bounds__(kSortThreads, 1) emb_sort_kernel(SortArgs a) {
  __shared__ uint16_t s_warp[kSortWarps][256];                   // a digit's items per warp, then before the warp
  __shared__ uint32_t s_hist[256], s_base[256], s_tile[256], s_scan[8];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t begin = min((int64_t)blockIdx.x * a.segment, a.n), end = min(begin + a.segment, a.n);
  for (int64_t i = (int64_t)blockIdx.x * kSortThreads + tid; i < a.rows; i += (int64_t)gridDim.x * kSortThreads) a.touched[i] = 0;
  if (blockIdx.x == 0 && tid == 0) a.runs[0] = 0;
  uint32_t key[kSortItems], tok[kSortItems], rank[kSortItems];
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * a.bits;
    const uint32_t mask = (1u << a.bits) - 1u;
    const uint32_t* src_k = a.keys[pass & 1];
    const uint32_t* src_t = a.toks[pass & 1];
    uint32_t* dst_k = a.keys[(pass + 1) & 1];
    uint32_t* dst_t = a.toks[(pass + 1) & 1];
    // items of a tile: warp by warp, each 32 x `items` of them in order
    auto load_tile = [&](int64_t t0) {
      const int items = (int)((min((int64_t)kSortTile, end - t0) + kSortThreads - 1) / kSortThreads);
#pragma unroll
      for (int j = 0; j < kSortItems; ++j) {
        if (j >= items) break;
        const int64_t t = t0 + (int64_t)warp * 32 * items + j * 32 + lane;
        tok[j] = 0xffffffffu; key[j] = 0u;
        if (t < end) { key[j] = pass == 0 ? sort_key(a, t) : src_k[t]; tok[j] = pass == 0 ? (uint32_t)t : src_t[t]; }
      }
      return items;
    };
    // rank of every item among those of its digit in its warp; s_warp = items of a digit in the warps before, s_tile = in the tile
    auto rank_tile = [&](int64_t t0, int items) {
      uint4* row = reinterpret_cast<uint4*>(s_warp[warp]);
      row[lane] = make_uint4(0u, 0u, 0u, 0u);
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kSortItems; ++j) {
        if (j >= items) break;
        const bool valid = t0 + (int64_t)warp * 32 * items + j * 32 + lane < end;
        const uint32_t digit = valid ? (key[j] >> shift) & mask : 0xffffffffu;
        const uint32_t peers = __match_any_sync(0xffffffffu, digit);
        const uint32_t below = __popc(peers & ((1u << lane) - 1u));
        uint32_t before = 0u;
        if (valid) before = s_warp[warp][digit];
        __syncwarp();
        if (valid && below == 0u) s_warp[warp][digit] = (uint16_t)(before + __popc(peers));
        __syncwarp();
        rank[j] = before + below;
      }
      __syncthreads();
      if (tid < 256) {
        uint32_t run = 0;
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) { const uint32_t c = s_warp[w][tid]; s_warp[w][tid] = (uint16_t)run; run += c; }
        s_tile[tid] = run;
      }
      __syncthreads();
    };
    auto scatter_tile = [&](int64_t t0, int items) {
#pragma unroll
      for (int j = 0; j < kSortItems; ++j) {
        if (j >= items) break;
        if (t0 + (int64_t)warp * 32 * items + j * 32 + lane < end) {
          const uint32_t digit = (key[j] >> shift) & mask;
          const uint32_t at = s_base[digit] + s_warp[warp][digit] + rank[j];
          dst_k[at] = key[j]; dst_t[at] = tok[j];
          if (pass + 1 == a.passes && key[j] < (uint32_t)a.rows) a.touched[key[j]] = 1;
        }
      }
    };
    int items = 0;
    if (tid < 256) s_hist[tid] = 0u;
    if constexpr (ONE) {
      if (begin < end) { items = load_tile(begin); rank_tile(begin, items); if (tid < 256) s_hist[tid] = s_tile[tid]; }
    } else {
      for (int64_t t0 = begin; t0 < end; t0 += kSortTile) {
        items = load_tile(t0); rank_tile(t0, items);
        if (tid < 256) s_hist[tid] += s_tile[tid];
      }
    }
    cluster_sync();
    // first place of this CTA's items of a digit: all items of smaller digits, and those of this one in the CTAs before
    uint32_t below = 0, total = 0, scan = 0;
    if (tid < 256) {
      for (uint32_t b = 0; b < gridDim.x; ++b) { const uint32_t c = remote_u32(&s_hist[tid], b); if (b < blockIdx.x) below += c; total += c; }
      scan = total;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) { const uint32_t v = __shfl_up_sync(0xffffffffu, scan, o); if (lane >= o) scan += v; }
      if (lane == 31) s_scan[warp] = scan;
    }
    __syncthreads();
    if (tid < 256) {
      uint32_t before = 0;
      for (int w = 0; w < warp; ++w) before += s_scan[w];
      s_base[tid] = before + scan - total + below;
    }
    __syncthreads();
    if constexpr (ONE) {
      if (begin < end) scatter_tile(begin, items);
    } else {
      for (int64_t t0 = begin; t0 < end; t0 += kSortTile) {
        items = load_tile(t0); rank_tile(t0, items);
        scatter_tile(t0, items);
        __syncthreads();
        if (tid < 256) s_base[tid] += s_tile[tid];
        __syncthreads();
      }
    }
    cluster_sync();
  }
  // runs that go over the end of the chunk that they start in
  const uint32_t* keys = a.keys[a.passes & 1];
  const int64_t chunks = (a.n + kEmbChunk - 1) / kEmbChunk;
  for (int64_t c = (int64_t)blockIdx.x * kSortThreads + tid; c + 1 < chunks; c += (int64_t)gridDim.x * kSortThreads) {
    const uint32_t k = keys[c * kEmbChunk + kEmbChunk - 1];
    if (k < (uint32_t)a.rows && keys[(c + 1) * kEmbChunk] == k && (c == 0 || keys[c * kEmbChunk - 1] != k)) a.runs[1 + atomicAdd(&a.runs[0], 1u)] = (uint32_t)c;
  }
}

// ---- sums -----------------------------------------------------------------------------------------
struct SumArgs {
  const uint32_t *keys, *toks; const uint8_t* touched; const uint32_t* runs;
  int64_t n, chunks, rows, cols;
  const void* dout; int64_t ld;
  float scale; int accumulate;
  float* out; int64_t ld_out;
  float* parts; int64_t ld_part;       // [chunks][2][ld_part]: the part of a run that came over the chunk's start, of one that goes over its end
  int64_t sum_ctas;                    // CTAs (along x) that sum; the others write rows without tokens
  int zero_rows;                       // rows of one of those
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

template <typename T, int VEC>
__global__ void __launch_bounds__(kEmbThreads) emb_sum_kernel(SumArgs a) {
  constexpr int kAhead = 8;
  extern __shared__ uint32_t s_chunk[];                           // [cy][2][kEmbChunk] keys, tokens
  wait_for_previous();
  const int tid = threadIdx.y * blockDim.x + threadIdx.x, threads = blockDim.x * blockDim.y;
  const int64_t col = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * VEC;
  if ((int64_t)blockIdx.x >= a.sum_ctas) {
    const int64_t r0 = ((int64_t)blockIdx.x - a.sum_ctas) * a.zero_rows;
    if (col >= a.cols) return;
    for (int64_t r = r0 + threadIdx.y; r < min(r0 + a.zero_rows, a.rows); r += blockDim.y) {
      if (a.n > 0 && a.touched[r]) continue;
      float* p = a.out + r * a.ld_out + col;
      if (VEC % 4 == 0 && a.vec_out) {
#pragma unroll
        for (int j = 0; j < VEC; j += 4) *reinterpret_cast<float4*>(p + j) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) p[j] = 0.0f;
      }
    }
    return;
  }
  for (int i = tid; i < (int)blockDim.y * kEmbChunk; i += threads) {
    const int64_t at = (int64_t)blockIdx.x * blockDim.y * kEmbChunk + i;
    const int y = i / kEmbChunk, k = i % kEmbChunk;
    s_chunk[(y * 2) * kEmbChunk + k] = at < a.n ? a.keys[at] : 0xffffffffu;
    s_chunk[(y * 2 + 1) * kEmbChunk + k] = at < a.n ? a.toks[at] : 0u;
  }
  __syncthreads();
  const int64_t chunk = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (chunk >= a.chunks || col >= a.cols) return;
  const int64_t first = chunk * kEmbChunk;
  const int count = (int)min((int64_t)kEmbChunk, a.n - first);
  const uint32_t* keys = s_chunk + threadIdx.y * 2 * kEmbChunk;
  const uint32_t* toks = keys + kEmbChunk;
  const uint32_t before = first > 0 ? a.keys[first - 1] : 0xffffffffu, behind = first + count < a.n ? a.keys[first + count] : 0xffffffffu;
  const T* dout = static_cast<const T*>(a.dout) + col;
  float acc[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) acc[j] = 0.0f;
  uint32_t run = keys[0];
  bool came_over = run == before;
  auto flush = [&](bool goes_over) {
    if (run < (uint32_t)a.rows) {
      if (came_over || goes_over) {
        float* p = a.parts + (chunk * 2 + (came_over ? 0 : 1)) * a.ld_part + col;
#pragma unroll
        for (int j = 0; j < VEC; ++j) p[j] = acc[j];
      } else put_row<VEC>(a, a.out + (int64_t)run * a.ld_out + col, acc);
    }
  };
  for (int i0 = 0; i0 < count; i0 += kAhead) {
    Pack<T, VEC> x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (i0 + u < count && keys[i0 + u] < (uint32_t)a.rows) x[u] = load_pack<T, VEC>(dout + (int64_t)toks[i0 + u] * a.ld);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (i0 + u >= count) break;
      const uint32_t k = keys[i0 + u];
      if (k != run) {
        flush(false);
        run = k; came_over = false;
#pragma unroll
        for (int j = 0; j < VEC; ++j) acc[j] = 0.0f;
      }
      if (k < (uint32_t)a.rows) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) acc[j] += to_float(x[u].v[j]);
      }
    }
  }
  flush(run == behind);
}

// A CTA adds the parts of one run for 128 columns: eight slices of the run's chunks, then the slices.
constexpr int kJoinSlices = 8;
__global__ void __launch_bounds__(32 * kJoinSlices) emb_join_kernel(SumArgs a) {
  __shared__ float4 s_part[kJoinSlices][32];
  __shared__ int64_t s_last;
  wait_for_previous();
  const int64_t slabs = (a.cols + 127) / 128, units = (int64_t)a.runs[0] * slabs;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int64_t c0 = a.runs[1 + unit / slabs], col = (unit % slabs) * 128 + threadIdx.x * 4;
    const uint32_t k = a.keys[c0 * kEmbChunk + kEmbChunk - 1];
    if (threadIdx.x == 0 && threadIdx.y == 0) {                   // last chunk that starts with this id: the keys ascend
      int64_t lo = c0 + 1, hi = a.chunks - 1;
      while (lo < hi) { const int64_t mid = (lo + hi + 1) >> 1; if (a.keys[mid * kEmbChunk] == k) lo = mid; else hi = mid - 1; }
      s_last = lo;
    }
    __syncthreads();
    const int64_t count = s_last - c0 + 1, per = (count + kJoinSlices - 1) / kJoinSlices;
    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (col < a.cols) {
      const int64_t i1 = min(count, (threadIdx.y + 1) * per);
#pragma unroll 4
      for (int64_t i = threadIdx.y * per; i < i1; ++i) {
        const float4 x = *reinterpret_cast<const float4*>(a.parts + ((c0 + i) * 2 + (i == 0 ? 1 : 0)) * a.ld_part + col);
        acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
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
      else for (int64_t j = 0; col + j < a.cols; ++j) { const float y[1] = {x[j]}; put_row<1>(a, p + j, y); }
    }
    __syncthreads();
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
  const EmbShape s = emb_shape(a.cols, VEC);
  const dim3 block(s.cx, s.cy);
  // four tokens per thread from where a quarter as many threads still fill the GPU
  const bool many = a.n * s.slabs * s.cx / 4 >= 148 * 2048;
  const int u = many ? 4 : 1;
  const dim3 grid((unsigned)((a.n + (int64_t)s.cy * u - 1) / ((int64_t)s.cy * u)), s.slabs);
  const Ids ids{a.ids, a.id_bytes == 8};
  if (many) emb_lookup_kernel<T, VEC, 4><<<grid, block, 0, st>>>((const T*)a.table, a.rows, a.cols, a.ld, ids, a.n, a.scale, (T*)a.out, a.ld_out, a.status);
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

struct EmbLayout { uint64_t keys[2], toks[2], touched, runs, parts, bytes; int64_t chunks, ld_part; };
EmbLayout emb_layout(int64_t n, int64_t rows, int64_t cols) {
  EmbLayout l{};
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t p = at; at = align_up(at + bytes, 256); return p; };
  l.chunks = (n + kEmbChunk - 1) / kEmbChunk;
  l.ld_part = (cols + 3) / 4 * 4;
  for (int i = 0; i < 2; ++i) { l.keys[i] = take((uint64_t)n * 4); l.toks[i] = take((uint64_t)n * 4); }
  l.touched = take((uint64_t)rows);
  l.runs = take((uint64_t)(l.chunks + 1) * 4);
  l.parts = take((uint64_t)l.chunks * 2 * l.ld_part * 4);
  l.bytes = at;
  return l;
}

template <typename T, int VEC>
cudaError_t sum_typed(SumArgs& a, cudaStream_t st) {
  const EmbShape s = emb_shape(a.cols, VEC);
  a.sum_ctas = (a.chunks + s.cy - 1) / s.cy;
  // rows of a CTA that writes zeros: about 64 KB of them
  a.zero_rows = (int)std::max<int64_t>(s.cy, std::min<int64_t>(1024, 65536 / (4 * std::min<int64_t>(a.cols, (int64_t)s.cx * VEC))));
  const int64_t zero_ctas = a.accumulate ? 0 : (a.rows + a.zero_rows - 1) / a.zero_rows;
  if (a.sum_ctas + zero_ctas == 0) return cudaSuccess;
  return launch_after(emb_sum_kernel<T, VEC>, dim3((unsigned)(a.sum_ctas + zero_ctas), s.slabs), dim3(s.cx, s.cy), (size_t)s.cy * 2 * kEmbChunk * 4, st, a);
}
template <typename T>
cudaError_t sum_type(SumArgs& a, cudaStream_t st) {
  const int vec = emb_vec(a.dout, a.ld, a.cols, sizeof(T));
  if (vec == 16 / (int)sizeof(T)) return sum_typed<T, 16 / sizeof(T)>(a, st);
  if constexpr (sizeof(T) == 2) { if (vec == 2) return sum_typed<T, 2>(a, st); }
  return sum_typed<T, 1>(a, st);
}

}  // namespace

int launch_embedding(const EmbLookup& a, cudaStream_t st) {
  if (a.n == 0) return (int)cudaSuccess;
  if (a.type == ATOMO_TYPE_F32) return (int)lookup_type<float>(a, st);
  if (a.type == ATOMO_TYPE_BF16) return (int)lookup_type<__nv_bfloat16>(a, st);
  return (int)lookup_type<__half>(a, st);
}

uint64_t embedding_workspace(int64_t n, int64_t rows, int64_t cols) { return emb_layout(n, rows, cols).bytes; }

int launch_embedding_backward(const EmbBackward& b, cudaStream_t st) {
  const EmbLayout l = emb_layout(b.n, b.rows, b.cols);
  SumArgs a{};
  a.n = b.n; a.chunks = l.chunks; a.rows = b.rows; a.cols = b.cols;
  a.dout = b.grad; a.ld = b.ld; a.scale = b.scale; a.accumulate = b.accumulate; a.out = b.out; a.ld_out = b.ld_out; a.ld_part = l.ld_part;
  a.vec_out = reinterpret_cast<uintptr_t>(b.out) % 16 == 0 && b.ld_out % 4 == 0;
  if (b.n > 0) {
    SortArgs s{};
    s.ids = Ids{b.ids, b.id_bytes == 8}; s.n = b.n; s.rows = b.rows; s.padding = b.padding; s.status = b.status;
    for (int i = 0; i < 2; ++i) { s.keys[i] = reinterpret_cast<uint32_t*>(b.ws + l.keys[i]); s.toks[i] = reinterpret_cast<uint32_t*>(b.ws + l.toks[i]); }
    s.touched = b.ws + l.touched;
    s.runs = reinterpret_cast<uint32_t*>(b.ws + l.runs);
    int bits = 1;
    while ((b.rows >> bits) != 0) ++bits;                        // keys are 0 .. rows
    s.passes = (bits + 7) / 8; s.bits = (bits + s.passes - 1) / s.passes;
    const int ctas = b.n <= kSortThreads ? 1 : kSortCluster;
    s.segment = (b.n + ctas - 1) / ctas;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas); cfg.blockDim = dim3(kSortThreads); cfg.stream = st; cfg.attrs = attr; cfg.numAttrs = 1;
    const cudaError_t e = s.segment <= kSortTile ? cudaLaunchKernelEx(&cfg, emb_sort_kernel<true>, s) : cudaLaunchKernelEx(&cfg, emb_sort_kernel<false>, s);
    if (e != cudaSuccess) return (int)e;
    a.keys = s.keys[s.passes & 1]; a.toks = s.toks[s.passes & 1]; a.touched = s.touched; a.runs = s.runs;
    a.parts = reinterpret_cast<float*>(b.ws + l.parts);
  }
  cudaError_t e = b.type == ATOMO_TYPE_F32 ? sum_type<float>(a, st) : b.type == ATOMO_TYPE_BF16 ? sum_type<__nv_bfloat16>(a, st) : sum_type<__half>(a, st);
  if (e != cudaSuccess || l.chunks < 2) return (int)e;
  const int64_t units = (l.chunks - 1) * ((b.cols + 127) / 128);
  return (int)launch_after(emb_join_kernel, dim3((unsigned)std::min<int64_t>(units, 148 * 4)), dim3(32, kJoinSlices), 0, st, a);
}

}  // namespace atomo
