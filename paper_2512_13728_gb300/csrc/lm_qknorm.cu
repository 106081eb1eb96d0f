// Norm and rotation of queries and keys, forward and backward.
//
// For a head x in R^D with weights w:  r = 1 / sqrt(mean(x^2) + eps),  n = r x,  u = w n, and the pairs
// (a, b) of u's first `rotary` elements turned by angle_j:  y = R u.  Backward, from g = dL/dy:
//   gu = R^T g,   dw = sum over heads and tokens of gu n,   dx = r (w gu - n mean(w gu n)).
//
// A group of lanes holds a head as D / 2 pairs (the elements that pass are paired across their own
// halves, with angle 0), so a rotation never leaves a lane; the mean is a shuffle sum over the group.
// A group takes several heads of one token and computes the token's sines and cosines once.
#include "lm_common.cuh"

#include <algorithm>
#include <cmath>
#include <new>

using namespace cd;
using namespace cd::lm;

namespace {
constexpr int kMaxHeadDim = 256;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
}  // namespace

struct dion_qknorm_plan {
  int device = 0, num_sms = 0;
  int32_t head_dim = 0, rotary = 0, interleaved = 0;
  float eps = 0.f;
  void *ws = nullptr;
  uint64_t *turn = nullptr;     // [rotary / 2]: turns per position as a fraction of 2^64
  float *partial = nullptr;     // [max_blocks][2][head_dim]: a block's sums of dwq, dwk
  uint32_t *finished = nullptr; // blocks that have written theirs
  int64_t max_blocks = 0;
};

namespace {

struct Heads {
  void *p;
  int64_t sb, st, sh;
};

struct Args {
  int64_t batch, tokens, tasks;  // tasks = batch * tokens * split
  int32_t hq, hk, split;         // a token's heads are dealt to `split` groups
  int32_t dim, half;             // half = rotary / 2
  int32_t chunks, group;         // chunks of V pairs per head, lanes per head
  float eps;
  const void *pos;
  int64_t pos_sb;
  int32_t pos_dtype;
  const uint64_t *turn;
  Heads q, k, gq, gk, oq, ok;
  const float *wq, *wk;
  float *dwq, *dwk;
  float *partial;
  uint32_t *finished;
};

// Where pair u of a head sits: its first element, and the distance to the second.  Pairs at and beyond
// `half` are the elements that pass.
template <bool INTER>
__device__ __forceinline__ void pair_place(int u, int dim, int half, int &at, int &apart) {
  if (INTER) {
    at = 2 * u, apart = 1;
  } else if (u < half) {
    at = u, apart = half;
  } else {
    at = half + u, apart = dim / 2 - half;
  }
}

// A lane's V pairs (a, b) of one chunk; V divides half and dim / 2 - half unless interleaved.
template <class T, int V, bool INTER>
__device__ __forceinline__ void load_pairs(const T *x, int u, int dim, int half, float (&a)[V], float (&b)[V]) {
  int at, apart;
  pair_place<INTER>(u, dim, half, at, apart);
  if (INTER) {
    float lo[V], hi[V];
    load_vec<T, V>(x + at, lo);
    load_vec<T, V>(x + at + V, hi);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      a[e] = 2 * e < V ? lo[(2 * e) % V] : hi[(2 * e) % V];
      b[e] = 2 * e + 1 < V ? lo[(2 * e + 1) % V] : hi[(2 * e + 1) % V];
    }
  } else {
    load_vec<T, V>(x + at, a);
    load_vec<T, V>(x + at + apart, b);
  }
}
template <class T, int V, bool INTER>
__device__ __forceinline__ void store_pairs(T *x, int u, int dim, int half, const float (&a)[V], const float (&b)[V]) {
  int at, apart;
  pair_place<INTER>(u, dim, half, at, apart);
  if (INTER) {
    float lo[V], hi[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      lo[e] = e & 1 ? b[e / 2] : a[e / 2];
      hi[e] = (V + e) & 1 ? b[(V + e) / 2] : a[(V + e) / 2];
    }
    store_vec<T, V>(x + at, lo);
    store_vec<T, V>(x + at + V, hi);
  } else {
    store_vec<T, V>(x + at, a);
    store_vec<T, V>(x + at + apart, b);
  }
}

// Sum over the lanes of a group (a power of two, aligned).
__device__ __forceinline__ float group_sum(float v, int group) {
  for (int o = group >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// cos and sin of a token's angle for pair u.  position * turn wraps modulo one turn exactly; the top 32
// bits, as a signed fraction of half a turn, are within 2^-32 of it, and fp32's rounding of that is
// 2^-25 of half a turn at most.
__device__ __forceinline__ void pair_angle(const Args &A, int64_t position, int u, float &c, float &s) {
  c = 1.f, s = 0.f;
  if (u < A.half) {
    const int32_t part = (int32_t)(((uint64_t)position * A.turn[u]) >> 32);
    sincospif((float)part * 0x1p-31f, &s, &c);
  }
}

// What a group works on: a token and its first head; heads h, h + split, ... of q, then of k.
struct Task {
  int64_t b, t;
  int32_t head;
  int64_t position;
};
__device__ __forceinline__ Task task_of(const Args &A, int64_t i) {
  Task k;
  const int64_t token = i / A.split;
  k.head = (int32_t)(i - token * A.split);
  k.b = token / A.tokens;
  k.t = token - k.b * A.tokens;
  k.position = A.pos ? load_index(A.pos, A.pos_dtype, k.b * A.pos_sb + k.t) : k.t;
  return k;
}
template <class T>
__device__ __forceinline__ T *head_of(const Heads &H, const Task &k, int h) {
  return static_cast<T *>(H.p) + k.b * H.sb + k.t * H.st + h * H.sh;
}

// ------------------------------------------------------------------------------ forward ---
// NC chunks of V pairs per lane, `group` lanes apart.
template <class T, int V, int NC, bool INTER>
__global__ void __launch_bounds__(kThreads) forward_kernel(const Args A) {
  chain_enter();
  const int lane = threadIdx.x & 31, in_group = lane & (A.group - 1);
  const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / A.group;
  const bool live = i < A.tasks;  // the shuffles need every lane
  const Task k = task_of(A, live ? i : 0);
  float c[NC][V], s[NC][V];
#pragma unroll
  for (int n = 0; n < NC; ++n)
#pragma unroll
    for (int e = 0; e < V; ++e) pair_angle(A, k.position, (in_group + n * A.group) * V + e, c[n][e], s[n][e]);
  const float inv_dim = 1.f / (float)A.dim;
  const int heads = A.hq + A.hk;
  for (int h0 = 0; h0 < heads; h0 += A.split) {  // the same count for every group
    const int h = h0 + k.head;
    const bool on = live && h < heads, is_q = h < A.hq;
    const T *x = head_of<const T>(is_q ? A.q : A.k, k, is_q ? h : h - A.hq);
    float a[NC][V], b[NC][V], sum = 0.f;
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const int u = (in_group + n * A.group) * V;
      if (on && 2 * u < A.dim) {
        load_pairs<T, V, INTER>(x, u, A.dim, A.half, a[n], b[n]);
#pragma unroll
        for (int e = 0; e < V; ++e) sum = fmaf(a[n][e], a[n][e], fmaf(b[n][e], b[n][e], sum));
      }
    }
    const float r = rsqrtf(group_sum(sum, A.group) * inv_dim + A.eps);
    if (!on) continue;
    const float *w = is_q ? A.wq : A.wk;
    T *y = head_of<T>(is_q ? A.oq : A.ok, k, is_q ? h : h - A.hq);
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const int u = (in_group + n * A.group) * V;
      if (2 * u >= A.dim) continue;
      float wa[V], wb[V];
#pragma unroll
      for (int e = 0; e < V; ++e) wa[e] = wb[e] = 1.f;
      if (w)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          int at, apart;
          pair_place<INTER>(u + e, A.dim, A.half, at, apart);
          wa[e] = w[at], wb[e] = w[at + apart];
        }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float ua = a[n][e] * r * wa[e], ub = b[n][e] * r * wb[e];
        a[n][e] = ua * c[n][e] - ub * s[n][e];
        b[n][e] = ub * c[n][e] + ua * s[n][e];
      }
      store_pairs<T, V, INTER>(y, u, A.dim, A.half, a[n], b[n]);
    }
  }
}

// ----------------------------------------------------------------------------- backward ---
template <class T, int V, int NC, bool INTER>
__global__ void __launch_bounds__(kThreads) backward_kernel(const Args A) {
  __shared__ float red[kWarps][2 * kMaxHeadDim];
  __shared__ bool last;
  chain_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in_group = lane & (A.group - 1);
  const int64_t per_block = kThreads / A.group, stride = per_block * gridDim.x;
  const int64_t first = (int64_t)blockIdx.x * per_block + threadIdx.x / A.group;
  const int64_t rounds = (A.tasks + stride - 1) / stride;
  const float inv_dim = 1.f / (float)A.dim;
  const int heads = A.hq + A.hk;
  float dqa[NC][V], dqb[NC][V], dka[NC][V], dkb[NC][V];  // this lane's sums of dwq, dwk
#pragma unroll
  for (int n = 0; n < NC; ++n)
#pragma unroll
    for (int e = 0; e < V; ++e) dqa[n][e] = dqb[n][e] = dka[n][e] = dkb[n][e] = 0.f;
  for (int64_t round = 0; round < rounds; ++round) {
    const int64_t i = first + round * stride;
    const bool live = i < A.tasks;
    const Task k = task_of(A, live ? i : 0);
    float c[NC][V], s[NC][V];
#pragma unroll
    for (int n = 0; n < NC; ++n)
#pragma unroll
      for (int e = 0; e < V; ++e) pair_angle(A, k.position, (in_group + n * A.group) * V + e, c[n][e], s[n][e]);
    for (int h0 = 0; h0 < heads; h0 += A.split) {
      const int h = h0 + k.head;
      const bool on = live && h < heads, is_q = h < A.hq;
      const int hh = is_q ? h : h - A.hq;
      const T *x = head_of<const T>(is_q ? A.q : A.k, k, hh);
      const T *g = head_of<const T>(is_q ? A.gq : A.gk, k, hh);
      const float *w = is_q ? A.wq : A.wk;
      float a[NC][V], b[NC][V], ga[NC][V], gb[NC][V], sum = 0.f, dot = 0.f;
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        const int u = (in_group + n * A.group) * V;
        if (on && 2 * u < A.dim) {
          load_pairs<T, V, INTER>(x, u, A.dim, A.half, a[n], b[n]);
          load_pairs<T, V, INTER>(g, u, A.dim, A.half, ga[n], gb[n]);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            int at, apart;
            pair_place<INTER>(u + e, A.dim, A.half, at, apart);
            const float wa = w ? w[at] : 1.f, wb = w ? w[at + apart] : 1.f;
            const float ra = ga[n][e] * c[n][e] + gb[n][e] * s[n][e], rb = gb[n][e] * c[n][e] - ga[n][e] * s[n][e];
            ga[n][e] = ra, gb[n][e] = rb;
            sum = fmaf(a[n][e], a[n][e], fmaf(b[n][e], b[n][e], sum));
            dot = fmaf(ra * wa, a[n][e], fmaf(rb * wb, b[n][e], dot));
          }
        }
      }
      const float r = rsqrtf(group_sum(sum, A.group) * inv_dim + A.eps);
      dot = group_sum(dot, A.group) * inv_dim * r * r;  // n mean(w gu n) = x r * r * mean(w gu x)
      if (!on) continue;
      T *y = head_of<T>(is_q ? A.oq : A.ok, k, hh);
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        const int u = (in_group + n * A.group) * V;
        if (2 * u >= A.dim) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          int at, apart;
          pair_place<INTER>(u + e, A.dim, A.half, at, apart);
          const float wa = w ? w[at] : 1.f, wb = w ? w[at + apart] : 1.f;
          const float da = ga[n][e] * a[n][e] * r, db = gb[n][e] * b[n][e] * r;
          if (is_q)
            dqa[n][e] += da, dqb[n][e] += db;
          else
            dka[n][e] += da, dkb[n][e] += db;
          a[n][e] = r * (wa * ga[n][e] - a[n][e] * dot);
          b[n][e] = r * (wb * gb[n][e] - b[n][e] * dot);
        }
        store_pairs<T, V, INTER>(y, u, A.dim, A.half, a[n], b[n]);
      }
    }
  }
  if (!A.dwq && !A.dwk) return;
  // the block's sums of dw: over the groups of a warp, then over the warps, then over the blocks, each
  // in a fixed order; the last block to finish adds up the blocks
#pragma unroll
  for (int n = 0; n < NC; ++n)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float v[4] = {dqa[n][e], dqb[n][e], dka[n][e], dkb[n][e]};
#pragma unroll
      for (int m = 0; m < 4; ++m)
        for (int o = A.group; o < 32; o <<= 1) v[m] += __shfl_xor_sync(0xffffffffu, v[m], o);
      const int u = (in_group + n * A.group) * V + e;
      if (lane < A.group && 2 * u < A.dim) {
        int at, apart;
        pair_place<INTER>(u, A.dim, A.half, at, apart);
        red[warp][at] = v[0], red[warp][at + apart] = v[1];
        red[warp][A.dim + at] = v[2], red[warp][A.dim + at + apart] = v[3];
      }
    }
  __syncthreads();
  for (int d = threadIdx.x; d < 2 * A.dim; d += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) v += red[w][d];
    A.partial[(int64_t)blockIdx.x * 2 * A.dim + d] = v;
  }
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(A.finished, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  for (int d = threadIdx.x; d < 2 * A.dim; d += kThreads) {
    float v = 0.f;
#pragma unroll 8
    for (int blk = 0; blk < (int)gridDim.x; ++blk) v += __ldcg(&A.partial[(int64_t)blk * 2 * A.dim + d]);
    float *to = d < A.dim ? A.dwq : A.dwk;
    if (to) to[d < A.dim ? d : d - A.dim] = v;
  }
  if (threadIdx.x == 0) *A.finished = 0;  // for the next call
}

// ----------------------------------------------------------------------------- dispatch ---
dion_status check_heads(const dion_heads *h, int32_t heads, int32_t dtype) {
  if (heads == 0) return DION_OK;
  if (!h || !h->data) return DION_ERR_INVALID_ARG;
  return aligned_to(h->data, element_bytes(dtype)) ? DION_OK : DION_ERR_ALIGNMENT;
}

Heads heads_of(const dion_heads *h) {
  return h ? Heads{h->data, h->batch_stride, h->token_stride, h->head_stride} : Heads{nullptr, 0, 0, 0};
}

// Pairs per access: the widest that divides the rotated and the passing pairs and that every
// tensor is aligned to.
int pair_width(const dion_qknorm_plan *p, const dion_qk_shape *s, const Heads *h, int n) {
  const int es = element_bytes(s->dtype);
  for (int v = 16 / es; v > 1; v /= 2) {
    bool fits = p->head_dim / 2 % v == 0 && (p->interleaved || p->rotary / 2 % v == 0);
    for (int i = 0; i < n; ++i)
      fits = fits && (!h[i].p || (aligned_to(h[i].p, v * es) && h[i].sb % v == 0 && h[i].st % v == 0 && h[i].sh % v == 0));
    if (fits) return v;
  }
  return 1;
}

dion_status check_shape(const dion_qknorm_plan *p, const dion_qk_shape *s) {
  if (!p || !s || s->batch < 0 || s->tokens < 0 || s->heads < 0 || s->kv_heads < 0 || s->heads + (int64_t)s->kv_heads < 1 ||
      !is_dtype(s->dtype))
    return DION_ERR_INVALID_ARG;
  if (s->positions && !is_index(s->position_dtype)) return DION_ERR_INVALID_ARG;
  if (s->positions && !aligned_to(s->positions, s->position_dtype == DION_INDEX_INT64 ? 8 : 4)) return DION_ERR_ALIGNMENT;
  const int64_t limit = (int64_t)1 << 40, per = ((int64_t)s->heads + s->kv_heads) * p->head_dim;
  if (s->batch > 0 && s->tokens > 0 && (per > limit || s->batch > limit / per || s->tokens > limit / per / s->batch))
    return DION_ERR_UNSUPPORTED;
  return DION_OK;
}

Args make_args(const dion_qknorm_plan *p, const dion_qk_shape *s, int v, int nc) {
  Args A{};
  A.batch = s->batch, A.tokens = s->tokens, A.hq = s->heads, A.hk = s->kv_heads;
  A.dim = p->head_dim, A.half = p->rotary / 2, A.eps = p->eps;
  A.pos = s->positions, A.pos_sb = s->position_batch_stride, A.pos_dtype = s->position_dtype;
  A.turn = p->turn, A.partial = p->partial, A.finished = p->finished;
  A.chunks = p->head_dim / 2 / v;
  A.group = 1;
  while (A.group * nc < A.chunks) A.group *= 2;
  return A;
}

// Heads per group: enough groups to fill the GPU first, then up to 8 heads of a token for each group,
// which share its sines and cosines.
void split_heads(Args &A, int num_sms) {
  const int heads = A.hq + A.hk;
  const int64_t tokens = A.batch * A.tokens, want = (int64_t)num_sms * 1024 / A.group;
  int64_t split = (heads + 7) / 8;
  if (tokens * split < want) split = std::min<int64_t>(heads, (want + tokens - 1) / tokens);
  A.split = (int32_t)split;
  A.tasks = tokens * split;
}

template <class T, bool INTER, class F>
cudaError_t with_width(int v, F &&f) {
  if constexpr (sizeof(T) == 2)
    if (v == 8) return f(T(), std::integral_constant<int, 8>(), std::integral_constant<int, 1>(), std::integral_constant<bool, INTER>());
  if (v == 4) return f(T(), std::integral_constant<int, 4>(), std::integral_constant<int, 1>(), std::integral_constant<bool, INTER>());
  if (v == 2) return f(T(), std::integral_constant<int, 2>(), std::integral_constant<int, 2>(), std::integral_constant<bool, INTER>());
  return f(T(), std::integral_constant<int, 1>(), std::integral_constant<int, 4>(), std::integral_constant<bool, INTER>());
}
template <class F>
cudaError_t with_kernel(int32_t dtype, int v, bool inter, F &&f) {
  if (dtype == DION_DTYPE_FP32) return inter ? with_width<float, true>(v, f) : with_width<float, false>(v, f);
  return inter ? with_width<__nv_bfloat16, true>(v, f) : with_width<__nv_bfloat16, false>(v, f);
}
int chunks_per_lane(int v) { return v >= 4 ? 1 : 4 / v; }

}  // namespace

extern "C" {

dion_status dion_qknorm_plan_create(int32_t head_dim, int32_t rotary_dim, int32_t interleaved, double theta,
                                    const double *inv_freq, float eps, dion_qknorm_plan **out) {
  if (!out) return DION_ERR_INVALID_ARG;
  *out = nullptr;
  if (head_dim < 2 || head_dim % 2 || rotary_dim < 0 || rotary_dim % 2 || rotary_dim > head_dim || !(eps >= 0.f) ||
      !std::isfinite(eps) || (!inv_freq && !(theta > 0.0 && std::isfinite(theta))))
    return DION_ERR_INVALID_ARG;
  if (head_dim > kMaxHeadDim) return DION_ERR_UNSUPPORTED;
  uint64_t turn[kMaxHeadDim / 2] = {};
  for (int j = 0; j < rotary_dim / 2; ++j) {
    const double f = inv_freq ? inv_freq[j] : std::pow(theta, -2.0 * j / rotary_dim);
    if (!std::isfinite(f)) return DION_ERR_INVALID_ARG;
    double t = f / 6.283185307179586476925;  // turns per position
    t -= std::floor(t);
    t = std::ldexp(t, 64);
    turn[j] = t >= 0x1p64 ? 0 : (uint64_t)t;
  }
  dion_qknorm_plan *p = new (std::nothrow) dion_qknorm_plan();
  if (!p) return DION_ERR_CUDA;
  p->head_dim = head_dim, p->rotary = rotary_dim, p->interleaved = interleaved != 0, p->eps = eps;
  cudaError_t e = cudaGetDevice(&p->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&p->num_sms, cudaDevAttrMultiProcessorCount, p->device);
  p->max_blocks = 2 * (int64_t)p->num_sms;
  const size_t o_partial = sizeof(turn), o_done = o_partial + sizeof(float) * 2 * head_dim * p->max_blocks;
  if (e == cudaSuccess) e = cudaMalloc(&p->ws, o_done + 16);
  if (e == cudaSuccess) {
    char *b = static_cast<char *>(p->ws);
    p->turn = reinterpret_cast<uint64_t *>(b);
    p->partial = reinterpret_cast<float *>(b + o_partial);
    p->finished = reinterpret_cast<uint32_t *>(b + o_done);
    e = cudaMemcpy(p->turn, turn, sizeof(turn), cudaMemcpyHostToDevice);
    if (e == cudaSuccess) e = cudaMemset(p->finished, 0, 16);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
  }
  if (e != cudaSuccess) {
    cudaGetLastError();
    cudaFree(p->ws);
    delete p;
    return DION_ERR_CUDA;
  }
  *out = p;
  return DION_OK;
}

dion_status dion_qknorm_forward(dion_qknorm_plan *p, const dion_qk_shape *s, const dion_heads *q, const dion_heads *k,
                                const float *wq, const float *wk, const dion_heads *q_out, const dion_heads *k_out,
                                void *stream) {
  dion_status st = check_shape(p, s);
  if (st != DION_OK) return st;
  if (s->batch == 0 || s->tokens == 0) return DION_OK;
  st = check_heads(q, s->heads, s->dtype);
  if (st == DION_OK) st = check_heads(k, s->kv_heads, s->dtype);
  if (st == DION_OK) st = check_heads(q_out, s->heads, s->dtype);
  if (st == DION_OK) st = check_heads(k_out, s->kv_heads, s->dtype);
  if (st != DION_OK) return st;
  if (!aligned_to(wq, 4) || !aligned_to(wk, 4)) return DION_ERR_ALIGNMENT;
  OnDevice on(p->device);
  if (!on.ok) return DION_ERR_CUDA;
  const Heads h[4] = {heads_of(s->heads ? q : nullptr), heads_of(s->kv_heads ? k : nullptr),
                      heads_of(s->heads ? q_out : nullptr), heads_of(s->kv_heads ? k_out : nullptr)};
  const int v = pair_width(p, s, h, 4);
  Args A = make_args(p, s, v, chunks_per_lane(v));
  A.q = h[0], A.k = h[1], A.oq = h[2], A.ok = h[3], A.wq = wq, A.wk = wk;
  split_heads(A, p->num_sms);
  const int64_t blocks = (A.tasks * A.group + kThreads - 1) / kThreads;
  if (blocks > INT32_MAX) return DION_ERR_UNSUPPORTED;
  const cudaError_t e = with_kernel(s->dtype, v, p->interleaved, [&](auto t, auto V, auto NC, auto I) {
    return launch(forward_kernel<decltype(t), decltype(V)::value, decltype(NC)::value, decltype(I)::value>, blocks, kThreads,
                  0, static_cast<cudaStream_t>(stream), 1, A);
  });
  return e == cudaSuccess ? DION_OK : DION_ERR_CUDA;
}

dion_status dion_qknorm_backward(dion_qknorm_plan *p, const dion_qk_shape *s, const dion_heads *gq, const dion_heads *gk,
                                 const dion_heads *q, const dion_heads *k, const float *wq, const float *wk,
                                 const dion_heads *dq, const dion_heads *dk, float *dwq, float *dwk, void *stream) {
  dion_status st = check_shape(p, s);
  if (st != DION_OK) return st;
  if (!aligned_to(wq, 4) || !aligned_to(wk, 4) || !aligned_to(dwq, 4) || !aligned_to(dwk, 4)) return DION_ERR_ALIGNMENT;
  const cudaStream_t cs = static_cast<cudaStream_t>(stream);
  OnDevice on(p->device);
  if (!on.ok) return DION_ERR_CUDA;
  if (s->batch == 0 || s->tokens == 0) {  // sums of nothing
    if (dwq && cudaMemsetAsync(dwq, 0, sizeof(float) * p->head_dim, cs) != cudaSuccess) return DION_ERR_CUDA;
    if (dwk && cudaMemsetAsync(dwk, 0, sizeof(float) * p->head_dim, cs) != cudaSuccess) return DION_ERR_CUDA;
    return DION_OK;
  }
  const dion_heads *in[6] = {gq, gk, q, k, dq, dk};
  Heads h[6];
  for (int i = 0; i < 6; ++i) {
    const int32_t n = i % 2 ? s->kv_heads : s->heads;
    st = check_heads(in[i], n, s->dtype);
    if (st != DION_OK) return st;
    h[i] = heads_of(n ? in[i] : nullptr);
  }
  const int v = pair_width(p, s, h, 6);
  Args A = make_args(p, s, v, chunks_per_lane(v));
  A.gq = h[0], A.gk = h[1], A.q = h[2], A.k = h[3], A.oq = h[4], A.ok = h[5];
  A.wq = wq, A.wk = wk, A.dwq = dwq, A.dwk = dwk;
  split_heads(A, p->num_sms);
  const int64_t blocks = std::min(p->max_blocks, (A.tasks * A.group + kThreads - 1) / kThreads);
  const cudaError_t e = with_kernel(s->dtype, v, p->interleaved, [&](auto t, auto V, auto NC, auto I) {
    return launch(backward_kernel<decltype(t), decltype(V)::value, decltype(NC)::value, decltype(I)::value>, blocks, kThreads,
                  0, cs, 1, A);
  });
  return e == cudaSuccess ? DION_OK : DION_ERR_CUDA;
}

void dion_qknorm_plan_destroy(dion_qknorm_plan *p) {
  if (!p) return;
  OnDevice on(p->device);
  cudaDeviceSynchronize();
  cudaFree(p->ws);
  delete p;
}

}  // extern "C"
