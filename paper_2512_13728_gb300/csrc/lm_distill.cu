// Distillation from a teacher's top logits: loss, and loss with gradient.
//
// Per row, with c = log2(e):  q_j = 2^((z_j - m) c / T) / s_T,  s_T = sum_j 2^((z_j - m) c / T),  m = max z,
// and the same with T = 1 for the hard labels.  One pass holds the running m, s_T and s_1.  The gradient
// needs the row again: a row (or, for long ones, its part) stays in shared memory between the two uses,
// so the logits are read once and the gradient is written once.  A cluster of blocks shares a row that
// is too long for one block, or rows that are too few to fill the GPU.
#include "lm_common.cuh"

#include <algorithm>
#include <cmath>
#include <cooperative_groups.h>

using namespace cd;
using namespace cd::lm;
namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kPartBytes = 200 * 1024;  // of a row in one block's shared memory
constexpr int kMaxCluster = 8;

struct Args {
  dion_distill d;
  float *loss;
  void *grad;
  int64_t ldg;
  int32_t cluster, part;  // blocks per row, chunks of 16 bytes per block
};

struct Stats {  // running maximum and sums of one set of logits
  float m, st, s1;
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The reference point of an exponential: the maximum, or 0 for a set without finite logits.
__device__ __forceinline__ float anchor(float m) { return m == -INFINITY ? 0.f : m; }

template <bool SOFT, bool HARD>
__device__ __forceinline__ Stats merge(const Stats &a, const Stats &b, float ct, float c1) {
  Stats r;
  r.m = fmaxf(a.m, b.m);
  const float at = anchor(r.m);
  r.st = r.s1 = 0.f;
  if (SOFT) r.st = a.st * exp2f((a.m - at) * ct) + b.st * exp2f((b.m - at) * ct);
  if (HARD) r.s1 = a.s1 * exp2f((a.m - at) * c1) + b.s1 * exp2f((b.m - at) * c1);
  return r;
}

// Adds the logits of G chunks to the statistics.
template <class T, int G, bool SOFT, bool HARD>
__device__ __forceinline__ void take(const float (&v)[G][16 / sizeof(T)], Stats &s, float ct, float c1) {
  constexpr int N = 16 / sizeof(T);
  float m = s.m;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int e = 0; e < N; ++e) m = fmaxf(m, v[g][e]);
  if (m > s.m) {
    if (SOFT) s.st *= exp2_fast((s.m - m) * ct);
    if (HARD) s.s1 *= exp2_fast((s.m - m) * c1);
    s.m = m;
  }
  const float at = anchor(s.m);
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if (SOFT) s.st += exp2_fast((v[g][e] - at) * ct);
      if (HARD) s.s1 += exp2_fast((v[g][e] - at) * c1);
    }
}

__device__ __forceinline__ void copy_16(void *smem, const void *global) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(smem))),
               "l"(global)
               : "memory");
}

template <class T>
__device__ __forceinline__ float load_one(const T *p) {
  float v[1];
  load_vec<T, 1>(p, v);
  return v[0];
}

__device__ __forceinline__ float load_any(const void *p, int32_t dtype, int64_t i) {
  return dtype == DION_DTYPE_FP32 ? static_cast<const float *>(p)[i] : load_one(static_cast<const __nv_bfloat16 *>(p) + i);
}

// One row per cluster.  GRAD: with the gradient.  SOFT, HARD: which terms the loss has.
template <class T, bool GRAD, bool SOFT, bool HARD>
__global__ void __launch_bounds__(kThreads) distill_kernel(const Args A) {
  constexpr int N = 16 / sizeof(T);
  extern __shared__ uint4 smem[];
  __shared__ Stats warp_stats[kWarps], block_stats, row_stats;
  __shared__ float red[kWarps], red2[kWarps];
  __shared__ int any;
  const dion_distill &d = A.d;
  const int top = SOFT ? (int)d.top : 0, entries = top + (HARD ? 1 : 0);
  uint4 *chunks = smem;  // GRAD: the block's part of the row
  int32_t *col = reinterpret_cast<int32_t *>(smem + (GRAD ? A.part : 0));  // [entries]: column, -1: absent
  float *share = reinterpret_cast<float *>(col + entries);                 // what the entry takes off its column's gradient
  float *zval = share + entries;                                           // its logit
  float *log_p = zval + entries;                                           // its teacher's log-probability
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  chain_enter();
  const int rank = (int)(blockIdx.x % (unsigned)A.cluster);
  const int64_t row = blockIdx.x / (unsigned)A.cluster;
  const T *z = static_cast<const T *>(d.logits) + row * d.ld;
  T *g = static_cast<T *>(A.grad) + (GRAD ? row * A.ldg : 0);
  const float w = d.weights ? d.weights[row] : 1.f;
  const int lead = (int)(reinterpret_cast<uintptr_t>(z) % 16 / sizeof(T));  // elements before the row in its first chunk
  const int64_t all = (lead + d.vocab + N - 1) / N;                         // chunks of the row
  const int64_t c_lo = (int64_t)rank * A.part, c_hi = c_lo + A.part < all ? c_lo + A.part : all;
  const uint4 *zc = reinterpret_cast<const uint4 *>(z - lead);
  // whether the gradient's rows sit at the same place within 16 bytes, so that whole chunks are stored
  const bool same_place = GRAD && (int)(reinterpret_cast<uintptr_t>(g) % 16 / sizeof(T)) == lead;

  if (w == 0.f) {  // the same for every block of the cluster
    if (rank == 0 && tid == 0) A.loss[row] = 0.f;
    if (GRAD) {
      for (int64_t c = c_lo + tid; c < c_hi; c += kThreads) {
        const int64_t j = c * N - lead;
        if (same_place && j >= 0 && j + N <= d.vocab)
          *reinterpret_cast<uint4 *>(g + j) = make_uint4(0, 0, 0, 0);
        else
          for (int e = 0; e < N; ++e)
            if (j + e >= 0 && j + e < d.vocab) g[j + e] = T(0.f);
      }
    }
    return;
  }

  // start the row's part on its way; a chunk at an end of the row that is not wholly its own is put
  // together from single elements, with -infinity around them
  const float inv_t = 1.f / d.temperature, ct = kLog2e * inv_t, c1 = kLog2e;
  auto edge = [&](int64_t c, float(&v)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const int64_t j = c * N - lead + e;
      v[e] = j >= 0 && j < d.vocab ? load_one(z + j) : -INFINITY;
    }
  };
  auto whole = [&](int64_t c) { return c * N >= lead && (c + 1) * N <= lead + d.vocab; };
  if (GRAD) {
    for (int64_t c = c_lo + tid; c < c_hi; c += kThreads) {
      if (whole(c)) {
        copy_16(&chunks[c - c_lo], &zc[c]);
      } else {
        float v[N];
        edge(c, v);
        store_vec<T, N>(reinterpret_cast<T *>(&chunks[c - c_lo]), v);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }

  // the teacher's entries, while the row is on its way: columns, logits, p
  if (tid == 0) any = 0;
  __syncthreads();
  float t_max = -INFINITY;
  if (SOFT) {
    for (int k = tid; k < top; k += kThreads) {
      const int64_t id = load_index(d.ids, d.id_dtype, row * d.ld_ids + k);
      const float t = load_any(d.teacher, d.teacher_dtype, row * d.ld_teacher + k);
      const bool there = id >= 0 && id < d.vocab && t != -INFINITY;
      col[k] = there ? (int32_t)id : -1;
      share[k] = t;
      zval[k] = there ? load_one(z + id) : 0.f;
      if (there) any = 1;
      if (there) t_max = t > t_max || t != t ? t : t_max;  // NaN stays
    }
  }
  if (HARD && tid == 0) {
    const int64_t y = load_index(d.labels, d.label_dtype, row);
    const bool there = y >= 0 && y < d.vocab;
    col[top] = there ? (int32_t)y : -1;
    share[top] = there ? w * d.hard : 0.f;
    zval[top] = there ? load_one(z + y) : 0.f;
  }
  bool soft_row = false;
  if (SOFT) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float x = __shfl_xor_sync(0xffffffffu, t_max, o);
      t_max = x > t_max || x != x ? x : t_max;
    }
    if (lane == 0) red[warp] = t_max;
    __syncthreads();
    soft_row = any != 0;
    for (int k = 0; k < kWarps; ++k) t_max = red[k] > t_max || red[k] != red[k] ? red[k] : t_max;
    float sum = 0.f;
    for (int k = tid; k < top; k += kThreads)
      if (col[k] >= 0) sum += expf((share[k] - t_max) * inv_t);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) red2[warp] = sum;
    __syncthreads();
    sum = 0.f;
    for (int k = 0; k < kWarps; ++k) sum += red2[k];
    const float log_sum = logf(sum);
    for (int k = tid; k < top; k += kThreads) {
      float p = 0.f;
      if (col[k] >= 0) {
        log_p[k] = (share[k] - t_max) * inv_t - log_sum;
        p = expf(log_p[k]);
      }
      share[k] = w * (1.f - d.hard) * d.temperature * p;
    }
  }

  // statistics of the block's part
  Stats s{-INFINITY, 0.f, 0.f};
  if (GRAD) {
    asm volatile("cp.async.wait_all;" ::: "memory");  // each thread reads only what it copied itself
    int64_t c = c_lo + tid;
    for (; c + 3 * kThreads < c_hi; c += 4 * kThreads) {
      float v[4][N];
#pragma unroll
      for (int u = 0; u < 4; ++u) load_vec<T, N>(reinterpret_cast<const T *>(&chunks[c - c_lo + u * kThreads]), v[u]);
      take<T, 4, SOFT, HARD>(v, s, ct, c1);
    }
    for (; c < c_hi; c += kThreads) {
      float v[1][N];
      load_vec<T, N>(reinterpret_cast<const T *>(&chunks[c - c_lo]), v[0]);
      take<T, 1, SOFT, HARD>(v, s, ct, c1);
    }
  } else {
    int64_t c = c_lo + tid;
    for (; c + 3 * kThreads < c_hi; c += 4 * kThreads) {
      float v[4][N];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t cu = c + u * kThreads;
        if (whole(cu))
          load_vec<T, N>(reinterpret_cast<const T *>(&zc[cu]), v[u]);
        else
          edge(cu, v[u]);
      }
      take<T, 4, SOFT, HARD>(v, s, ct, c1);
    }
    for (; c < c_hi; c += kThreads) {
      float v[1][N];
      if (whole(c))
        load_vec<T, N>(reinterpret_cast<const T *>(&zc[c]), v[0]);
      else
        edge(c, v[0]);
      take<T, 1, SOFT, HARD>(v, s, ct, c1);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Stats x;
    x.m = __shfl_xor_sync(0xffffffffu, s.m, o);
    x.st = __shfl_xor_sync(0xffffffffu, s.st, o);
    x.s1 = __shfl_xor_sync(0xffffffffu, s.s1, o);
    s = merge<SOFT, HARD>(s, x, ct, c1);
  }
  if (lane == 0) warp_stats[warp] = s;
  __syncthreads();
  if (tid == 0) {
    for (int k = 1; k < kWarps; ++k) s = merge<SOFT, HARD>(s, warp_stats[k], ct, c1);
    block_stats = row_stats = s;
  }
  if (A.cluster > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();  // every block has its statistics (and the logits of its entries)
    if (tid == 0) {
      Stats r = *cluster.map_shared_rank(&block_stats, 0);
      for (int b = 1; b < A.cluster; ++b) r = merge<SOFT, HARD>(r, *cluster.map_shared_rank(&block_stats, b), ct, c1);
      row_stats = r;
    }
    cluster.sync();  // the statistics were read; no block may leave before
  } else {
    __syncthreads();
  }
  s = row_stats;
  const float at = anchor(s.m);

  if (rank == 0 && warp == 0) {
    float loss = 0.f;
    if (SOFT && soft_row) {
      const float log_st = logf(s.st);
      for (int k = lane; k < top; k += 32) {
        if (col[k] < 0) continue;
        const float p = expf(log_p[k]);
        if (!(p <= 0.f)) loss += p * (log_p[k] - ((zval[k] - at) * inv_t - log_st));
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, o);
      loss *= (1.f - d.hard) * d.temperature * d.temperature;
    }
    if (HARD && col[top] >= 0) loss += d.hard * (logf(s.s1) - (zval[top] - at));
    if (lane == 0) A.loss[row] = w * loss;
  }
  if (!GRAD) return;

  // gradient without the teacher's and the label's own parts
  const float kt = SOFT && soft_row ? w * (1.f - d.hard) * d.temperature / s.st : 0.f;
  const float k1 = HARD && col[top] >= 0 ? w * d.hard / s.s1 : 0.f;
  auto base = [&](float x) {
    float r = 0.f;
    if (SOFT) r = soft_row ? kt * exp2_fast((x - at) * ct) : 0.f;
    if (HARD) r += col[top] >= 0 ? k1 * exp2_fast((x - at) * c1) : 0.f;
    return r;
  };
  for (int64_t c = c_lo + tid; c < c_hi; c += kThreads) {
    float v[N];
    load_vec<T, N>(reinterpret_cast<const T *>(&chunks[c - c_lo]), v);
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = base(v[e]);
    const int64_t j = c * N - lead;
    if (same_place && j >= 0 && j + N <= d.vocab) {
      store_vec<T, N>(g + j, v);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e)
        if (j + e >= 0 && j + e < d.vocab) {
          const float one[1] = {v[e]};
          store_vec<T, 1>(g + j + e, one);
        }
    }
  }
  __syncthreads();  // the entries' columns are written over what was written above
  const int64_t j_lo = c_lo * N - lead, j_hi = c_hi * N - lead;
  for (int k = tid; k < entries; k += kThreads) {
    const int32_t j = col[k];
    if (j < j_lo || j >= j_hi || j < 0) continue;
    float off = 0.f;  // of every entry with this column; the first of them writes
    bool first = true;
    for (int i = 0; i < entries; ++i) {
      if (col[i] != j) continue;
      if (i < k) first = false;
      off += share[i];
    }
    if (!first) continue;
    const float one[1] = {base(zval[k]) - off};
    store_vec<T, 1>(g + j, one);
  }
}

dion_status check(const dion_distill *d, float *loss) {
  if (!d || d->rows < 0 || d->vocab < 1 || d->top < 0 || !is_dtype(d->dtype) || !(d->temperature > 0.f) ||
      !std::isfinite(d->temperature) || !(d->hard >= 0.f && d->hard <= 1.f))
    return DION_ERR_INVALID_ARG;
  if (d->top > DION_DISTILL_MAX_TOP || d->vocab > DION_DISTILL_MAX_VOCAB || d->rows > ((int64_t)1 << 30) / kMaxCluster)
    return DION_ERR_UNSUPPORTED;
  const bool soft = d->hard < 1.f, hard = d->hard > 0.f;
  if (d->rows == 0) return DION_OK;
  if (!d->logits || !loss || d->ld < d->vocab) return DION_ERR_INVALID_ARG;
  if (soft && (!is_index(d->id_dtype) || !is_dtype(d->teacher_dtype))) return DION_ERR_INVALID_ARG;
  if (soft && d->top > 0 && (!d->ids || !d->teacher || d->ld_ids < d->top || d->ld_teacher < d->top)) return DION_ERR_INVALID_ARG;
  if (hard && (!d->labels || !is_index(d->label_dtype))) return DION_ERR_INVALID_ARG;
  auto index_bytes = [](int32_t t) { return t == DION_INDEX_INT64 ? 8 : 4; };
  if (!aligned_to(d->logits, element_bytes(d->dtype)) || !aligned_to(loss, 4) || !aligned_to(d->weights, 4) ||
      (soft && (!aligned_to(d->ids, index_bytes(d->id_dtype)) || !aligned_to(d->teacher, element_bytes(d->teacher_dtype)))) ||
      (hard && !aligned_to(d->labels, index_bytes(d->label_dtype))))
    return DION_ERR_ALIGNMENT;
  return DION_OK;
}

template <class T, bool GRAD>
cudaError_t run(const Args &A, size_t smem, cudaStream_t s) {
  const bool soft = A.d.hard < 1.f, hard = A.d.hard > 0.f;
  auto kernel = soft ? hard ? distill_kernel<T, GRAD, true, true> : distill_kernel<T, GRAD, true, false>
                     : distill_kernel<T, GRAD, false, true>;
  const cudaError_t e = allow_dynamic_smem(kernel, smem);
  if (e != cudaSuccess) return e;
  return launch(kernel, A.d.rows * A.cluster, kThreads, smem, s, A.cluster, A);
}

dion_status enqueue(const dion_distill *d, float *loss, void *grad, int64_t ldg, bool with_grad, void *stream) {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return DION_ERR_CUDA;
  Args A{};
  A.d = *d, A.loss = loss, A.grad = grad, A.ldg = ldg;
  const int64_t bytes = d->vocab * element_bytes(d->dtype), chunks = bytes / 16 + 2;  // the most a row can touch
  A.cluster = 1;
  while (A.cluster < kMaxCluster && ((with_grad && chunks * 16 > (int64_t)kPartBytes * A.cluster) ||
                                     (d->rows * A.cluster * 2 <= sms && chunks / A.cluster > 2 * kThreads)))
    A.cluster *= 2;
  A.part = (int32_t)((chunks + A.cluster - 1) / A.cluster);
  const size_t entries = (d->hard < 1.f ? (size_t)d->top : 0) + (d->hard > 0.f ? 1 : 0);
  const size_t smem = (with_grad ? (size_t)A.part * 16 : 0) + entries * 16;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = d->dtype == DION_DTYPE_FP32
                            ? with_grad ? run<float, true>(A, smem, s) : run<float, false>(A, smem, s)
                            : with_grad ? run<__nv_bfloat16, true>(A, smem, s) : run<__nv_bfloat16, false>(A, smem, s);
  return e == cudaSuccess ? DION_OK : DION_ERR_CUDA;
}

}  // namespace

extern "C" {

dion_status dion_distill_loss(const dion_distill *d, float *loss, void *stream) {
  const dion_status st = check(d, loss);
  if (st != DION_OK || d->rows == 0) return st;
  return enqueue(d, loss, nullptr, 0, false, stream);
}

dion_status dion_distill_loss_grad(const dion_distill *d, float *loss, void *grad, int64_t ldg, void *stream) {
  const dion_status st = check(d, loss);
  if (st != DION_OK || d->rows == 0) return st;
  if (!grad || ldg < d->vocab) return DION_ERR_INVALID_ARG;
  if (!aligned_to(grad, element_bytes(d->dtype))) return DION_ERR_ALIGNMENT;
  return enqueue(d, loss, grad, ldg, true, stream);
}

}  // extern "C"
