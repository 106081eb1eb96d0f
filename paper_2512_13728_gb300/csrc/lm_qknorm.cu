// Norm and rotation of queries and keys, forward and backward.
//
// For a head x in R^D with weights w:  r = 1 / sqrt(mean(x^2) + eps),  n = r x,  u = w n, and the pairs
// (a, b) of u's first `rotary` elements turned by angle_j:  y = R u.  Backward, from g = dL/dy:
//   gu = R^T g,   dw = sum over heads and tokens of gu n,   dx = r (w gu - n mean(w gu n)).
//
// A group of lanes holds a head as D / 2 pairs (the elements that pass are paired across their own
// halves, with angle 0), so a rotation never leaves a lane; the mean is a shuffle sum over the group.
// A warp takes one token at a time: its sines and cosines are computed once by the warp's lanes, and
// several heads per group are loaded before the first is used.
#include "lm_common.cuh"

#include <algorithm>
#include <cmath>
#include <new>

using namespace cd;
using namespace cd::lm;

namespace {
constexpr int kMaxHeadDim = 256;
constexpr int kMaxPairs = kMaxHeadDim / 2;
constexpr int kMaxHeads = 2048;  // of q, of k
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
#ifndef FU
#define FU 4
#define FB 1
#define BU 2
#define BB 2
#endif
constexpr int kForwardHeads = FU;   // heads that a group has in flight
constexpr int kBackwardHeads = BU;
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
  int64_t batch, tokens;  // sequences, tokens of each
  int64_t tasks;          // forward: tokens of all sequences * parts
  int32_t hq, hk;
  int32_t q_batches, batches;  // batches of heads (one kind each) of q, of q and k
  int32_t parts;               // warps that share a token's batches
  int32_t dim, half;           // half = rotary / 2
  int32_t group;               // lanes per head
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

// A lane's pairs of a head: NC chunks of V, `group` lanes apart; V divides half and dim / 2 - half unless
// interleaved, when a chunk's pairs are 2 V neighbouring elements.
template <class T, int V, int NC, bool INTER>
struct HeadPairs {
  Raw<T, V> lo[NC], hi[NC];
  __device__ __forceinline__ void load(const T *x, bool on, int in_group, const Args &A) {
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const int u = (in_group + n * A.group) * V;
#pragma unroll
      for (uint32_t &w : lo[n].w) w = 0;
#pragma unroll
      for (uint32_t &w : hi[n].w) w = 0;
      if (on && 2 * u < A.dim) {
        int at, apart;
        pair_place<INTER>(u, A.dim, A.half, at, apart);
        lo[n].load(x + at);
        hi[n].load(x + at + (INTER ? V : apart));
      }
    }
  }
  __device__ __forceinline__ float a(int n, int e) const {
    if (!INTER) return lo[n].at(e);
    return 2 * e < V ? lo[n].at((2 * e) % V) : hi[n].at((2 * e) % V);
  }
  __device__ __forceinline__ float b(int n, int e) const {
    if (!INTER) return hi[n].at(e);
    return 2 * e + 1 < V ? lo[n].at((2 * e + 1) % V) : hi[n].at((2 * e + 1) % V);
  }
};
template <class T, int V, bool INTER>
__device__ __forceinline__ void store_pairs(T *x, int u, const Args &A, const float (&a)[V], const float (&b)[V]) {
  int at, apart;
  pair_place<INTER>(u, A.dim, A.half, at, apart);
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

// Sines and cosines of a token's pairs into the warp's shared memory.  position * turn wraps modulo one
// turn exactly; the top 32 bits, as a signed fraction of half a turn, are within 2^-31 of it, and
// fp32's rounding of that is 2^-25 of half a turn at most.
__device__ __forceinline__ void token_angles(const Args &A, int64_t position, float *cs, float *sn) {
  __syncwarp();  // the last token's were read
  for (int u = threadIdx.x & 31; u < A.dim / 2; u += 32) {
    float c = 1.f, s = 0.f;
    if (u < A.half) {
      const int32_t part = (int32_t)(((uint64_t)position * A.turn[u]) >> 32);
      sincospif((float)part * 0x1p-31f, &s, &c);
    }
    cs[u] = c, sn[u] = s;
  }
  __syncwarp();
}

// The weights of both kinds by pairs, in shared memory: [kind][first or second of the pair][pair].
template <bool INTER>
__device__ __forceinline__ void stage_weights(const Args &A, float (&w)[2][2][kMaxPairs]) {
  for (int i = threadIdx.x; i < 2 * A.dim; i += kThreads) {
    const int kind = i / A.dim, r = i - kind * A.dim, second = r >= A.dim / 2, u = r - second * (A.dim / 2);
    int at, apart;
    pair_place<INTER>(u, A.dim, A.half, at, apart);
    const float *from = kind ? A.wk : A.wq;
    w[kind][second][u] = from ? from[at + second * apart] : 1.f;
  }
  __syncthreads();
}

// V neighbouring floats of shared memory for each of a lane's chunks.
template <int V, int NC>
__device__ __forceinline__ void read_pairs(const float *from, int in_group, const Args &A, float (&v)[NC][V]) {
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    const int u = (in_group + n * A.group) * V;
    const float *at = from + (2 * u < A.dim ? u : 0);
    if constexpr (V == 8) {  // two accesses: shared memory has none of 32 bytes
      const float4 x = *reinterpret_cast<const float4 *>(at), y = *reinterpret_cast<const float4 *>(at + 4);
      v[n][0] = x.x, v[n][1] = x.y, v[n][2] = x.z, v[n][3] = x.w, v[n][4] = y.x, v[n][5] = y.y, v[n][6] = y.z, v[n][7] = y.w;
    } else {
      load_vec<float, V>(at, v[n]);
    }
  }
}

struct Token {
  int64_t b, t;
  __device__ __forceinline__ Token(const Args &A, int64_t i) {
    if (i <= 0x7fffffff && A.tokens <= 0x7fffffff) {  // a 64-bit division costs more than a head
      b = (uint32_t)i / (uint32_t)A.tokens;
    } else {
      b = i / A.tokens;
    }
    t = i - b * A.tokens;
  }
  __device__ __forceinline__ int64_t position(const Args &A) const {
    return A.pos ? load_index(A.pos, A.pos_dtype, b * A.pos_sb + t) : t;
  }
  template <class T>
  __device__ __forceinline__ T *heads(const Heads &H) const {
    return static_cast<T *>(H.p) + b * H.sb + t * H.st;
  }
};

// ------------------------------------------------------------------------------ forward ---
template <class T, int V, int NC, bool INTER>
__global__ void __launch_bounds__(kThreads, FB) forward_kernel(const __grid_constant__ Args A) {
  constexpr int U = kForwardHeads;
  __shared__ __align__(16) float w[2][2][kMaxPairs], angles[kWarps][2][kMaxPairs];
  chain_enter();
  stage_weights<INTER>(A, w);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in_group = lane & (A.group - 1), groups = 32 / A.group;
  const int64_t task = (int64_t)blockIdx.x * kWarps + warp;
  if (task >= A.tasks) return;
  const int64_t i = task <= 0x7fffffff ? (int64_t)((uint32_t)task / (uint32_t)A.parts) : task / A.parts;
  const Token tok(A, i);
  const int64_t position = tok.position(A);
  const float inv_dim = 1.f / (float)A.dim;
  bool angles_ready = false;
  for (int batch = (int)(task - i * A.parts); batch < A.batches; batch += A.parts) {
    const int kind = batch >= A.q_batches;
    const int heads = kind ? A.hk : A.hq, h0 = (batch - (kind ? A.q_batches : 0)) * U * groups + lane / A.group;
    const Heads &X = kind ? A.k : A.q, &Y = kind ? A.ok : A.oq;
    const T *x = tok.heads<const T>(X);
    T *y = tok.heads<T>(Y);
    HeadPairs<T, V, NC, INTER> p[U];
#pragma unroll
    for (int k = 0; k < U; ++k) p[k].load(x + (h0 + k * groups) * X.sh, h0 + k * groups < heads, in_group, A);
    if (!angles_ready) token_angles(A, position, angles[warp][0], angles[warp][1]);
    angles_ready = true;
    float c[NC][V], s[NC][V], wa[NC][V], wb[NC][V];
    read_pairs<V, NC>(angles[warp][0], in_group, A, c);
    read_pairs<V, NC>(angles[warp][1], in_group, A, s);
    read_pairs<V, NC>(w[kind][0], in_group, A, wa);
    read_pairs<V, NC>(w[kind][1], in_group, A, wb);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if ((batch - (kind ? A.q_batches : 0)) * U * groups + k * groups >= heads) break;  // the same for the whole warp
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < NC; ++n)
#pragma unroll
        for (int e = 0; e < V; ++e) sum = fmaf(p[k].a(n, e), p[k].a(n, e), fmaf(p[k].b(n, e), p[k].b(n, e), sum));
      const float r = rsqrtf(group_sum(sum, A.group) * inv_dim + A.eps);
      const int h = h0 + k * groups;
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        const int u = (in_group + n * A.group) * V;
        if (h >= heads || 2 * u >= A.dim) continue;
        float a[V], b[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float ua = p[k].a(n, e) * r * wa[n][e], ub = p[k].b(n, e) * r * wb[n][e];
          a[e] = ua * c[n][e] - ub * s[n][e];
          b[e] = ub * c[n][e] + ua * s[n][e];
        }
        store_pairs<T, V, INTER>(y + h * Y.sh, u, A, a, b);
      }
    }
  }
}

// ----------------------------------------------------------------------------- backward ---
// A warp keeps to one batch of heads and goes over tokens, so that its sums of dw stay in registers.
template <class T, int V, int NC, bool INTER>
__global__ void __launch_bounds__(kThreads, BB) backward_kernel(const __grid_constant__ Args A) {
  constexpr int U = kBackwardHeads;
  __shared__ __align__(16) float w[2][2][kMaxPairs], angles[kWarps][2][kMaxPairs], red[kWarps][2 * kMaxHeadDim];
  __shared__ bool last;
  chain_enter();
  stage_weights<INTER>(A, w);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in_group = lane & (A.group - 1), groups = 32 / A.group;
  const int64_t all = A.batch * A.tokens;
  const int unit = blockIdx.x * kWarps + warp, batch = unit % A.batches;
  const int64_t first = unit / A.batches, stride = ((int64_t)gridDim.x * kWarps - batch + A.batches - 1) / A.batches;
  const int kind = batch >= A.q_batches;
  const int heads = kind ? A.hk : A.hq, h_first = (batch - (kind ? A.q_batches : 0)) * U * groups, h0 = h_first + lane / A.group;
  const Heads &X = kind ? A.k : A.q, &G = kind ? A.gk : A.gq, &Y = kind ? A.ok : A.oq;
  const float inv_dim = 1.f / (float)A.dim;
  float wa[NC][V], wb[NC][V], da[NC][V], db[NC][V];  // weights, and this lane's sums of their gradients
  read_pairs<V, NC>(w[kind][0], in_group, A, wa);
  read_pairs<V, NC>(w[kind][1], in_group, A, wb);
#pragma unroll
  for (int n = 0; n < NC; ++n)
#pragma unroll
    for (int e = 0; e < V; ++e) da[n][e] = db[n][e] = 0.f;
  for (int64_t i = first; i < all; i += stride) {
    const Token tok(A, i);
    const T *x = tok.heads<const T>(X), *g = tok.heads<const T>(G);
    T *y = tok.heads<T>(Y);
    HeadPairs<T, V, NC, INTER> p[U], q[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const bool on = h0 + k * groups < heads;
      p[k].load(x + (h0 + k * groups) * X.sh, on, in_group, A);
      q[k].load(g + (h0 + k * groups) * G.sh, on, in_group, A);
    }
    token_angles(A, tok.position(A), angles[warp][0], angles[warp][1]);
    float c[NC][V], s[NC][V];
    read_pairs<V, NC>(angles[warp][0], in_group, A, c);
    read_pairs<V, NC>(angles[warp][1], in_group, A, s);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (h_first + k * groups >= heads) break;  // the same for the whole warp
      float ga[NC][V], gb[NC][V], sum = 0.f, dot = 0.f;
#pragma unroll
      for (int n = 0; n < NC; ++n)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float a = p[k].a(n, e), b = p[k].b(n, e), oa = q[k].a(n, e), ob = q[k].b(n, e);
          ga[n][e] = oa * c[n][e] + ob * s[n][e];
          gb[n][e] = ob * c[n][e] - oa * s[n][e];
          sum = fmaf(a, a, fmaf(b, b, sum));
          dot = fmaf(ga[n][e] * wa[n][e], a, fmaf(gb[n][e] * wb[n][e], b, dot));
        }
      sum = group_sum(sum, A.group);
      dot = group_sum(dot, A.group);
      const float r = rsqrtf(sum * inv_dim + A.eps);
      const float back = dot * inv_dim * r * r * r;  // dx = r w gu - x r^3 mean(w gu x)
      const int h = h0 + k * groups;
#pragma unroll
      for (int n = 0; n < NC; ++n) {
        const int u = (in_group + n * A.group) * V;
        if (h >= heads || 2 * u >= A.dim) continue;
        float oa[V], ob[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float a = p[k].a(n, e), b = p[k].b(n, e), ra = r * ga[n][e], rb = r * gb[n][e];
          da[n][e] = fmaf(ra, a, da[n][e]), db[n][e] = fmaf(rb, b, db[n][e]);
          oa[e] = ra * wa[n][e] - a * back;
          ob[e] = rb * wb[n][e] - b * back;
        }
        store_pairs<T, V, INTER>(y + h * Y.sh, u, A, oa, ob);
      }
    }
  }
  if (!A.dwq && !A.dwk) return;
  // the block's sums of dw: over the groups of a warp, then over the warps, then over the blocks, each
  // in a fixed order; the last block to finish adds up the blocks
  for (int d = lane; d < 2 * A.dim; d += 32) red[warp][d] = 0.f;
  __syncwarp();
#pragma unroll
  for (int n = 0; n < NC; ++n)
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float va = da[n][e], vb = db[n][e];
      for (int o = A.group; o < 32; o <<= 1) {
        va += __shfl_xor_sync(0xffffffffu, va, o);
        vb += __shfl_xor_sync(0xffffffffu, vb, o);
      }
      const int u = (in_group + n * A.group) * V + e;
      if (lane < A.group && 2 * u < A.dim) {
        int at, apart;
        pair_place<INTER>(u, A.dim, A.half, at, apart);
        red[warp][kind * A.dim + at] = va, red[warp][kind * A.dim + at + apart] = vb;
      }
    }
  __syncthreads();
  for (int d = threadIdx.x; d < 2 * A.dim; d += kThreads) {
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) v += red[k][d];
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
  if (s->heads > kMaxHeads || s->kv_heads > kMaxHeads) return DION_ERR_UNSUPPORTED;
  if (s->positions && !aligned_to(s->positions, s->position_dtype == DION_INDEX_INT64 ? 8 : 4)) return DION_ERR_ALIGNMENT;
  const int64_t limit = (int64_t)1 << 40, per = ((int64_t)s->heads + s->kv_heads) * p->head_dim;
  if (s->batch > 0 && s->tokens > 0 && (per > limit || s->batch > limit / per || s->tokens > limit / per / s->batch))
    return DION_ERR_UNSUPPORTED;
  return DION_OK;
}

Args make_args(const dion_qknorm_plan *p, const dion_qk_shape *s, int v, int nc, int heads_in_flight) {
  Args A{};
  A.batch = s->batch, A.tokens = s->tokens, A.hq = s->heads, A.hk = s->kv_heads;
  A.dim = p->head_dim, A.half = p->rotary / 2, A.eps = p->eps;
  A.pos = s->positions, A.pos_sb = s->position_batch_stride, A.pos_dtype = s->position_dtype;
  A.turn = p->turn, A.partial = p->partial, A.finished = p->finished;
  A.group = 1;
  while (A.group * nc * v < p->head_dim / 2) A.group *= 2;
  const int per = heads_in_flight * (32 / A.group);
  A.q_batches = (int32_t)(((int64_t)A.hq + per - 1) / per);
  A.batches = A.q_batches + (int32_t)(((int64_t)A.hk + per - 1) / per);
  return A;
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
  // two resident blocks per SM, and a warp for every batch of the most heads that a call may have
  p->max_blocks = std::max<int64_t>(2 * (int64_t)p->num_sms, 2 * kMaxHeads / kBackwardHeads / kWarps);
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
  Args A = make_args(p, s, v, chunks_per_lane(v), kForwardHeads);
  A.q = h[0], A.k = h[1], A.oq = h[2], A.ok = h[3], A.wq = wq, A.wk = wk;
  // a warp per token, or more where the tokens do not give every SM its 16 warps
  const int64_t all = s->batch * s->tokens;
  A.parts = (int32_t)std::min<int64_t>(A.batches, ((int64_t)p->num_sms * 16 + all - 1) / all);
  A.tasks = all * A.parts;
  const int64_t blocks = (A.tasks + kWarps - 1) / kWarps;
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
  Args A = make_args(p, s, v, chunks_per_lane(v), kBackwardHeads);
  A.gq = h[0], A.gk = h[1], A.q = h[2], A.k = h[3], A.oq = h[4], A.ok = h[5];
  A.wq = wq, A.wk = wk, A.dwq = dwq, A.dwk = dwk;
  const int64_t units = s->batch * s->tokens * A.batches;
  const int64_t blocks = std::max<int64_t>(std::min(p->max_blocks, (units + kWarps - 1) / kWarps),
                                           (A.batches + kWarps - 1) / kWarps);  // a warp for every batch of heads
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
