// Token embedding: lookup with scaling, and its gradient by sorted tokens.
//
//   lookup    out[i] = s E[t_i]
//   gradient  dE[v] (+)= s sum_{i : t_i = v} dy[i]
//
// The gradient sorts (token, position) pairs with a stable radix sort and then walks the merge of
// two lists: the sorted entries and the ends of the table's rows.  Every warp takes an equal share of
// that merge for a slab of 256 columns, whatever the tokens are: a token that comes thousands of
// times is split over warps, and the rows that no token names are zeroed along the way.  A row that
// lies in several shares is added up from the shares' fp32 sums in a second small kernel, in order.
#include "lm_common.cuh"

#include <algorithm>
#include <cmath>
#include <new>

using namespace cd;
using namespace cd::lm;

namespace {

constexpr int kMaxBins = 512;     // digits of up to 9 bits
constexpr int kSortThreads = 256;
constexpr int kSortItems = 8;     // per thread
constexpr int kSortTile = kSortThreads * kSortItems;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSlab = 256;        // columns that a warp takes, 8 per lane
constexpr int kWalkThreads = 256;

}  // namespace

struct dion_embed_plan {
  int device = 0, num_sms = 0;
  int64_t vocab = 0, dim = 0, max_tokens = 0;
  void *ws = nullptr;
  uint32_t *key[2] = {}, *pos[2] = {};  // sorted back and forth
  uint32_t *hist = nullptr;             // [tiles][kMaxBins]
  float *head = nullptr, *tail = nullptr;  // [max_parts][slabs * kSlab]: sums of rows that begin or end outside a part
  int32_t *head_row = nullptr, *tail_row = nullptr;  // [max_parts]: the rows they belong to, -1: none
  int64_t max_parts = 0, slabs = 0;
};

namespace {

// ------------------------------------------------------------------------------- lookup ---
// A warp per token and slab of 256 columns; V elements per access.
template <class TE, class TO, int V>
__global__ void __launch_bounds__(256) lookup_kernel(const void *tokens, int32_t token_dtype, int64_t num_tokens,
                                                     const TE *table, int64_t ldt, int64_t vocab, int64_t dim,
                                                     int64_t slabs, float scale, TO *out, int64_t ldo) {
  chain_enter();
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5);
  const int64_t i = unit / slabs;
  if (i >= num_tokens) return;
  const int64_t c0 = (unit - i * slabs) * kSlab + lane * V;
  const int64_t t = load_index(tokens, token_dtype, i);
  const bool real = t >= 0 && t < vocab;
  float v[8 / V][V];
#pragma unroll
  for (int c = 0; c < 8 / V; ++c) {
#pragma unroll
    for (int e = 0; e < V; ++e) v[c][e] = 0.f;
    if (real && c0 + c * 32 * V < dim) load_vec<TE, V>(table + t * ldt + c0 + c * 32 * V, v[c]);
  }
#pragma unroll
  for (int c = 0; c < 8 / V; ++c) {
    if (c0 + c * 32 * V >= dim) break;
#pragma unroll
    for (int e = 0; e < V; ++e) v[c][e] = real ? v[c][e] * scale : 0.f;
    store_vec<TO, V>(out + i * ldo + c0 + c * 32 * V, v[c]);
  }
}

// --------------------------------------------------------------------------------- sort ---
// The key of a token outside the table is `vocab`: it sorts behind every row's entries.
__device__ __forceinline__ uint32_t token_key(const void *tokens, int32_t dtype, int64_t i, int64_t vocab) {
  const int64_t t = load_index(tokens, dtype, i);
  return (t >= 0 && t < vocab) ? (uint32_t)t : (uint32_t)vocab;
}

// Counts of each digit in each tile of kSortTile entries.  key == null: the first pass, from the tokens.
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const uint32_t *key, const void *tokens, int32_t dtype,
                                                                  int64_t vocab, int64_t n, int shift, int bits,
                                                                  uint32_t *hist) {
  __shared__ uint32_t count[kMaxBins];
  const int bins = 1 << bits;
  for (int b = threadIdx.x; b < bins; b += kSortThreads) count[b] = 0;
  chain_enter();
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
  for (int k = threadIdx.x; k < kSortTile; k += kSortThreads) {
    const int64_t i = base + k;
    if (i < n) atomicAdd(&count[((key ? key[i] : token_key(tokens, dtype, i, vocab)) >> shift) & (bins - 1)], 1u);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads) hist[(int64_t)blockIdx.x * kMaxBins + b] = count[b];
}

// Moves each entry to its place for one digit.  A tile's entries keep their order: warp w holds
// entries [w 256, (w + 1) 256) in rounds of 32, ranks within a round come from the lanes that share
// the digit, ranks across rounds and warps from per-warp counters.
__global__ void __launch_bounds__(kSortThreads) sort_move_kernel(const uint32_t *key, const uint32_t *pos, const void *tokens,
                                                                 int32_t dtype, int64_t vocab, int64_t n, int shift,
                                                                 int bits, const uint32_t *hist, int tiles,
                                                                 uint32_t *key_out, uint32_t *pos_out) {
  __shared__ uint32_t first[kMaxBins];              // where this tile's entries of a digit begin
  __shared__ uint32_t count[kSortWarps][kMaxBins];  // of each warp; then where the warp's entries begin
  __shared__ uint32_t warp_total[kSortWarps];
  const int bins = 1 << bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int b = threadIdx.x; b < kSortWarps * kMaxBins; b += kSortThreads) (&count[0][0])[b] = 0;
  chain_enter();
  __syncthreads();
  uint32_t k[kSortItems], p[kSortItems], rank[kSortItems];
  const int64_t base = (int64_t)blockIdx.x * kSortTile + warp * (32 * kSortItems) + lane;
#pragma unroll
  for (int r = 0; r < kSortItems; ++r) {
    const int64_t i = base + r * 32;
    const bool in = i < n;
    k[r] = in ? (key ? key[i] : token_key(tokens, dtype, i, vocab)) : 0u;
    p[r] = in ? (pos ? pos[i] : (uint32_t)i) : 0u;
    const uint32_t digit = in ? (k[r] >> shift) & (bins - 1) : (uint32_t)bins;  // entries past the end match each other only
    const uint32_t same = __match_any_sync(0xffffffffu, digit);
    const int leader = __ffs(same) - 1;
    uint32_t before = 0;
    if (in && lane == leader) {
      before = count[warp][digit];
      count[warp][digit] = before + __popc(same);
    }
    rank[r] = __shfl_sync(0xffffffffu, before, leader) + __popc(same & ((1u << lane) - 1));
    __syncwarp();
  }
  __syncthreads();
  // totals of the digits over all tiles, and over the tiles before this one; two digits per thread
  uint32_t total[2] = {0, 0}, mine[2] = {0, 0};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int b = threadIdx.x * 2 + h;
    if (b < bins) {
#pragma unroll 8
      for (int t = 0; t < tiles; ++t) {
        const uint32_t c = hist[(int64_t)t * kMaxBins + b];
        total[h] += c;
        if (t < (int)blockIdx.x) mine[h] += c;
      }
    }
  }
  uint32_t sum = total[0] + total[1], scan = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, scan, o);
    if (lane >= o) scan += x;
  }
  if (lane == 31) warp_total[warp] = scan;
  __syncthreads();
  uint32_t off = scan - sum;
  for (int w = 0; w < warp; ++w) off += warp_total[w];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int b = threadIdx.x * 2 + h;
    if (b < bins) first[b] = off + mine[h];
    off += total[h];
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kSortThreads) {
    uint32_t at = first[b];
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t c = count[w][b];
      count[w][b] = at;
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortItems; ++r) {
    if (base + r * 32 < n) {
      const uint32_t at = count[warp][(k[r] >> shift) & (bins - 1)] + rank[r];
      key_out[at] = k[r];
      pos_out[at] = p[r];
    }
  }
}

// --------------------------------------------------------------------------------- walk ---
struct Walk {
  const uint32_t *key, *pos;  // sorted entries
  int64_t n, vocab, dim, ldg, ldd, parts, slabs, share;
  float scale;
  float *head, *tail;
  int32_t *head_row, *tail_row;
};

// Entries of the first d items of the merge.  Entry j comes behind j entries and key[j] row ends, so
// its place is j + key[j]; when accumulating there are no row ends in the merge and it is j.
// Entries outside the table have places behind the last row end.
template <bool ACC>
__device__ __forceinline__ int64_t entries_before(const uint32_t *key, int64_t n, int64_t d) {
  if (ACC) return d < n ? d : n;
  const int lane = threadIdx.x & 31;
  int64_t lo = 0, hi = n < d ? n : d;  // the answer lies in [lo, hi]; 33-way search
  while (hi > lo) {
    const int64_t step = (hi - lo + 32) / 33;
    const int64_t j = lo + (lane + 1) * step - 1;  // probe: is entry j among the first d items?
    const bool in = j < hi && j + (int64_t)key[j] < d;
    const int hits = __popc(__ballot_sync(0xffffffffu, in));
    const int64_t l2 = lo + hits * step, h2 = lo + (hits + 1) * step - 1;
    lo = l2;
    hi = hits < 32 && h2 < hi ? h2 : hi;
  }
  return lo;
}

// One warp: a part of the merge, a slab of columns.
template <class TG, class TD, int V, bool ACC>
__global__ void __launch_bounds__(kWalkThreads) walk_kernel(const Walk w, const TG *grad, TD *dst) {
  chain_enter();
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * (kWalkThreads / 32) + (threadIdx.x >> 5);
  const int64_t part = unit / w.slabs, slab = unit - part * w.slabs;
  if (part >= w.parts) return;
  constexpr int C = 8 / V;
  const int64_t c0 = slab * kSlab + lane * V;
  const int64_t d0 = part * w.share, d1 = d0 + w.share;
  int64_t j = entries_before<ACC>(w.key, w.n, d0);
  const int64_t j1 = entries_before<ACC>(w.key, w.n, d1);
  float acc[C][V];
  auto clear = [&] {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < V; ++e) acc[c][e] = 0.f;
  };
  auto put_partial = [&](float *to) {
#pragma unroll
    for (int c = 0; c < C; ++c) store_vec<float, V>(to + (part * w.slabs + slab) * kSlab + c * 32 * V + lane * V, acc[c]);
  };
  auto put_row = [&](int64_t row) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (c0 + c * 32 * V >= w.dim) break;
      float v[V];
      TD *to = dst + row * w.ldd + c0 + c * 32 * V;
      if (ACC) load_vec<TD, V>(to, v);
#pragma unroll
      for (int e = 0; e < V; ++e) v[e] = ACC ? fmaf(w.scale, acc[c][e], v[e]) : w.scale * acc[c][e];
      store_vec<TD, V>(to, v);
    }
  };
  auto add = [&](int64_t at) {
    const TG *from = grad + (int64_t)w.pos[at] * w.ldg + c0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (c0 + c * 32 * V >= w.dim) break;
      float v[V];
      load_vec<TG, V>(from + c * 32 * V, v);
#pragma unroll
      for (int e = 0; e < V; ++e) acc[c][e] += v[e];
    }
  };
  clear();
  int64_t head_row = -1, tail_row = -1;
  if (ACC) {
    // rows end where the key changes; the part's last row goes on where the next entry has its key
    while (j < j1 && w.key[j] < w.vocab) {
      const int64_t row = w.key[j];
      const bool begun = j > 0 && w.key[j - 1] == row;
      while (j < j1 && w.key[j] == row) add(j++);
      if (j == j1 && j < w.n && w.key[j] == row) {
        put_partial(w.tail);
        tail_row = row;
      } else if (begun) {
        put_partial(w.head);
        head_row = row;
      } else {
        put_row(row);
      }
      clear();
    }
  } else {
    const int64_t i0 = d0 - j < w.vocab ? d0 - j : w.vocab, i1 = d1 - j1 < w.vocab ? d1 - j1 : w.vocab;
    const bool begun = j > 0 && i0 < w.vocab && w.key[j - 1] == i0;
    for (int64_t row = i0; row < i1; ++row) {
      while (j < j1 && w.key[j] == row) add(j++);
      if (row == i0 && begun) {
        put_partial(w.head);
        head_row = row;
      } else {
        put_row(row);
      }
      clear();
    }
    if (j < j1 && i1 < w.vocab) {
      while (j < j1) add(j++);
      put_partial(w.tail);
      tail_row = i1;
    }
  }
  if (slab == 0 && lane == 0) {
    w.head_row[part] = (int32_t)head_row;
    w.tail_row[part] = (int32_t)tail_row;
  }
}

// Rows that several parts have sums of: one block per part and slab; where the part ends such a row,
// the sums are added in the order of the parts and the row is written.
template <class TD, bool ACC>
__global__ void __launch_bounds__(kSlab) join_kernel(const Walk w, TD *dst) {
  chain_enter();
  const int64_t part = blockIdx.x / w.slabs, slab = blockIdx.x - part * w.slabs;
  const int64_t row = w.head_row[part];
  if (row < 0) return;
  int64_t from = part;
  while (from > 0 && w.tail_row[from - 1] == row) --from;
  const int64_t col = slab * kSlab + threadIdx.x;
  if (col >= w.dim) return;
  float sum = 0.f;
#pragma unroll 8
  for (int64_t q = from; q < part; ++q) sum += w.tail[(q * w.slabs + slab) * kSlab + threadIdx.x];
  sum += w.head[(part * w.slabs + slab) * kSlab + threadIdx.x];
  TD *to = dst + row * w.ldd + col;
  float v[1] = {0.f};
  if (ACC) load_vec<TD, 1>(to, v);
  v[0] = ACC ? fmaf(w.scale, sum, v[0]) : w.scale * sum;
  store_vec<TD, 1>(to, v);
}

// ----------------------------------------------------------------------------- dispatch ---
// Elements per access: the widest of 8, 4, 2, 1 that divides the rows and that both tensors' rows are
// aligned to (16 bytes at most).
int vector_width(int64_t dim, const void *a, int64_t lda, int32_t ta, const void *b, int64_t ldb, int32_t tb) {
  for (int v = 8; v > 1; v /= 2) {
    auto fits = [&](const void *p, int64_t ld, int32_t t) {
      const int64_t bytes = std::min<int64_t>(16, (int64_t)v * element_bytes(t));
      return aligned_to(p, bytes) && ld * element_bytes(t) % bytes == 0;
    };
    if (dim % v == 0 && fits(a, lda, ta) && fits(b, ldb, tb)) return v;
  }
  return 1;
}

template <class F>
cudaError_t with_width(int v, F &&f) {
  switch (v) {
    case 8: return f(std::integral_constant<int, 8>());
    case 4: return f(std::integral_constant<int, 4>());
    case 2: return f(std::integral_constant<int, 2>());
    default: return f(std::integral_constant<int, 1>());
  }
}

template <class F>
cudaError_t with_types(int32_t a, int32_t b, F &&f) {
  using BF = __nv_bfloat16;
  if (a == DION_DTYPE_FP32) return b == DION_DTYPE_FP32 ? f(float(), float()) : f(float(), BF());
  return b == DION_DTYPE_FP32 ? f(BF(), float()) : f(BF(), BF());
}

constexpr int64_t kSizeLimit = (int64_t)1 << 30;

dion_status check_rows(int64_t n, int64_t dim, const void *p, int32_t dtype, int64_t ld) {
  if (!is_dtype(dtype) || (n > 0 && !p) || ld < dim) return DION_ERR_INVALID_ARG;
  if (!aligned_to(p, element_bytes(dtype))) return DION_ERR_ALIGNMENT;
  return DION_OK;
}

dion_status check_tokens(int64_t n, const void *tokens, int32_t dtype) {
  if (n < 0 || !is_index(dtype) || (n > 0 && !tokens)) return DION_ERR_INVALID_ARG;
  if (n >= kSizeLimit) return DION_ERR_UNSUPPORTED;
  if (!aligned_to(tokens, dtype == DION_INDEX_INT64 ? 8 : 4)) return DION_ERR_ALIGNMENT;
  return DION_OK;
}

}  // namespace

extern "C" {

dion_status dion_embed_plan_create(int64_t vocab, int64_t dim, int64_t max_tokens, dion_embed_plan **out) {
  if (!out) return DION_ERR_INVALID_ARG;
  *out = nullptr;
  if (vocab < 1 || dim < 1 || max_tokens < 0) return DION_ERR_INVALID_ARG;
  if (vocab >= kSizeLimit || dim >= kSizeLimit || max_tokens >= kSizeLimit) return DION_ERR_UNSUPPORTED;
  dion_embed_plan *p = new (std::nothrow) dion_embed_plan();
  if (!p) return DION_ERR_CUDA;
  p->vocab = vocab, p->dim = dim, p->max_tokens = max_tokens;
  p->slabs = (dim + kSlab - 1) / kSlab;
  if (cudaGetDevice(&p->device) != cudaSuccess ||
      cudaDeviceGetAttribute(&p->num_sms, cudaDevAttrMultiProcessorCount, p->device) != cudaSuccess) {
    delete p;
    return DION_ERR_CUDA;
  }
  // one wave of the walk at 4 blocks per SM
  p->max_parts = std::max<int64_t>(1, (int64_t)p->num_sms * 4 * (kWalkThreads / 32) / p->slabs);
  const int64_t tiles = (max_tokens + kSortTile - 1) / kSortTile;
  size_t off = 0;
  auto region = [&](size_t bytes) {
    const size_t at = off;
    off += (bytes + 255) & ~(size_t)255;
    return at;
  };
  const size_t o_key0 = region(4 * max_tokens), o_key1 = region(4 * max_tokens);
  const size_t o_pos0 = region(4 * max_tokens), o_pos1 = region(4 * max_tokens);
  const size_t o_hist = region(4 * tiles * kMaxBins);
  const size_t sums = 4 * (size_t)p->max_parts * p->slabs * kSlab;
  const size_t o_head = region(sums), o_tail = region(sums);
  const size_t o_hrow = region(4 * p->max_parts), o_trow = region(4 * p->max_parts);
  if (cudaMalloc(&p->ws, off) != cudaSuccess) {
    cudaGetLastError();
    delete p;
    return DION_ERR_CUDA;
  }
  char *b = static_cast<char *>(p->ws);
  p->key[0] = reinterpret_cast<uint32_t *>(b + o_key0), p->key[1] = reinterpret_cast<uint32_t *>(b + o_key1);
  p->pos[0] = reinterpret_cast<uint32_t *>(b + o_pos0), p->pos[1] = reinterpret_cast<uint32_t *>(b + o_pos1);
  p->hist = reinterpret_cast<uint32_t *>(b + o_hist);
  p->head = reinterpret_cast<float *>(b + o_head), p->tail = reinterpret_cast<float *>(b + o_tail);
  p->head_row = reinterpret_cast<int32_t *>(b + o_hrow), p->tail_row = reinterpret_cast<int32_t *>(b + o_trow);
  *out = p;
  return DION_OK;
}

dion_status dion_embed_lookup(dion_embed_plan *p, const void *tokens, int32_t token_dtype, int64_t num_tokens,
                              const void *table, int32_t table_dtype, int64_t ldt, float scale, void *out,
                              int32_t out_dtype, int64_t ldo, void *stream) {
  if (!p || !std::isfinite(scale) || !table) return DION_ERR_INVALID_ARG;
  dion_status st = check_tokens(num_tokens, tokens, token_dtype);
  if (st == DION_OK) st = check_rows(num_tokens, p->dim, table, table_dtype, ldt);
  if (st == DION_OK) st = check_rows(num_tokens, p->dim, out, out_dtype, ldo);
  if (st != DION_OK) return st;
  if (num_tokens == 0) return DION_OK;
  const int64_t blocks = (num_tokens * p->slabs + 7) / 8;
  if (blocks > INT32_MAX) return DION_ERR_UNSUPPORTED;
  OnDevice on(p->device);
  if (!on.ok) return DION_ERR_CUDA;
  const int width = vector_width(p->dim, table, ldt, table_dtype, out, ldo, out_dtype);
  const cudaError_t e = with_types(table_dtype, out_dtype, [&](auto te, auto to) {
    using TE = decltype(te);
    using TO = decltype(to);
    return with_width(width, [&](auto v) {
      return launch(lookup_kernel<TE, TO, decltype(v)::value>, blocks, 256, 0, static_cast<cudaStream_t>(stream), 1, tokens,
                    token_dtype, num_tokens, static_cast<const TE *>(table), ldt, p->vocab, p->dim, p->slabs, scale,
                    static_cast<TO *>(out), ldo);
    });
  });
  return e == cudaSuccess ? DION_OK : DION_ERR_CUDA;
}

dion_status dion_embed_gradient(dion_embed_plan *p, const void *tokens, int32_t token_dtype, int64_t num_tokens,
                                const void *grad, int32_t grad_dtype, int64_t ldg, float scale, void *table_grad,
                                int32_t table_grad_dtype, int64_t ldd, int32_t accumulate, void *stream) {
  if (!p || !std::isfinite(scale) || !table_grad) return DION_ERR_INVALID_ARG;
  dion_status st = check_tokens(num_tokens, tokens, token_dtype);
  if (st == DION_OK && num_tokens > p->max_tokens) st = DION_ERR_INVALID_ARG;
  if (st == DION_OK) st = check_rows(num_tokens, p->dim, grad, grad_dtype, ldg);
  if (st == DION_OK) st = check_rows(p->vocab, p->dim, table_grad, table_grad_dtype, ldd);
  if (st != DION_OK) return st;
  if (num_tokens == 0 && accumulate) return DION_OK;
  OnDevice on(p->device);
  if (!on.ok) return DION_ERR_CUDA;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;

  // sort: as few digits of at most 9 bits as the largest key (vocab) needs
  int bits = 1;
  while (((int64_t)1 << bits) <= p->vocab) ++bits;
  const int passes = (bits + 8) / 9, digit = (bits + passes - 1) / passes;
  const int tiles = (int)((num_tokens + kSortTile - 1) / kSortTile);
  int at = 0;
  for (int pass = 0; pass < passes && tiles > 0 && e == cudaSuccess; ++pass) {
    const uint32_t *key = pass ? p->key[at] : nullptr, *pos = pass ? p->pos[at] : nullptr;
    const int shift = pass * digit, next = 1 - at;
    e = launch(sort_count_kernel, tiles, kSortThreads, 0, s, 1, key, tokens, token_dtype, p->vocab, num_tokens, shift, digit,
               p->hist);
    if (e == cudaSuccess)
      e = launch(sort_move_kernel, tiles, kSortThreads, 0, s, 1, key, pos, tokens, token_dtype, p->vocab, num_tokens, shift,
                 digit, p->hist, tiles, p->key[next], p->pos[next]);
    at = next;
  }
  if (e != cudaSuccess) return DION_ERR_CUDA;

  Walk w{};
  w.key = p->key[at], w.pos = p->pos[at];
  w.n = num_tokens, w.vocab = p->vocab, w.dim = p->dim, w.ldg = ldg, w.ldd = ldd, w.slabs = p->slabs, w.scale = scale;
  w.head = p->head, w.tail = p->tail, w.head_row = p->head_row, w.tail_row = p->tail_row;
  const int64_t items = num_tokens + (accumulate ? 0 : p->vocab);
  w.share = std::max<int64_t>(8, (items + p->max_parts - 1) / p->max_parts);
  w.parts = (items + w.share - 1) / w.share;
  const int64_t blocks = (w.parts * w.slabs + kWalkThreads / 32 - 1) / (kWalkThreads / 32);
  const int width = vector_width(p->dim, grad, ldg, grad_dtype, table_grad, ldd, table_grad_dtype);
  e = with_types(grad_dtype, table_grad_dtype, [&](auto tg, auto td) {
    using TG = decltype(tg);
    using TD = decltype(td);
    const TG *g = static_cast<const TG *>(grad);
    TD *d = static_cast<TD *>(table_grad);
    cudaError_t r = with_width(width, [&](auto v) {
      constexpr int V = decltype(v)::value;
      return accumulate ? launch(walk_kernel<TG, TD, V, true>, blocks, kWalkThreads, 0, s, 1, w, g, d)
                        : launch(walk_kernel<TG, TD, V, false>, blocks, kWalkThreads, 0, s, 1, w, g, d);
    });
    if (r != cudaSuccess) return r;
    return accumulate ? launch(join_kernel<TD, true>, w.parts * w.slabs, kSlab, 0, s, 1, w, d)
                      : launch(join_kernel<TD, false>, w.parts * w.slabs, kSlab, 0, s, 1, w, d);
  });
  return e == cudaSuccess ? DION_OK : DION_ERR_CUDA;
}

void dion_embed_plan_destroy(dion_embed_plan *p) {
  if (!p) return;
  OnDevice on(p->device);
  cudaDeviceSynchronize();
  cudaFree(p->ws);
  delete p;
}

}  // extern "C"
