// Norm and rotation of queries and keys, forward and backward.
//
// For a head x in R^D with weights w:  r = 1 / sqrt(mean(x^2) + eps),  n = r x,  u = w n, and the pairs
// (a, b) of u's first `rotary` elements turned by angle_j:  y = R u.  Backward, from g = dL/dy:
//   gu = R^T g,   dw = sum over heads and tokens of gu n,   dx = r (w gu - n mean(w gu n)).
//
// A group of lanes holds a head as D / 2 pairs (the elements that pass are paired across their own
// halves, with angle 0), so a rotation never leaves a lane; the mean is a shuffle sum over the group.
// A warp keeps to one kind and a few of its heads and goes over tokens (blocks of tokens, where the heads of
// one do not fill a warp): it computes a token's sines and cosines once, and holds the weights and the
// sums of their gradients in registers.  What it reads runs ahead of it through a ring of asynchronous
// copies in shared memory, of which every lane reads only what it copied itself.
#include "lm_common.cuh"
#include "tc_common.cuh"

#include <algorithm>
#include <cmath>
#include <new>
#include <numeric>

using namespace cd;
using namespace cd::lm;

namespace {
constexpr int kMaxHeadDim = 256;
constexpr int kMaxPairs = kMaxHeadDim / 2;
constexpr int kMaxHeads = 2048;  // of q, of k
constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kRing = 4;      // steps (a head per group of lanes) on their way
constexpr int kMaxSteps = 8;  // of a token, for a warp
// Blocks per SM, by the pairs that a lane holds: eight of them take 96 registers forward, 158 backward.
constexpr int forward_blocks(int pairs) { return pairs == 8 ? 5 : 6; }
constexpr int backward_blocks(int pairs) { return pairs == 8 ? 3 : 4; }
}  // namespace

struct dion_qknorm_plan {
  int device = 0, num_sms = 0;
  int32_t head_dim = 0, rotary = 0, interleaved = 0;
  float eps = 0.f;
  void *ws = nullptr;
  uint64_t *turn = nullptr;     // [rotary / 2]: turns per position as a fraction of 2^64
  float *partial = nullptr;     // [max_blocks][2][head_dim]: a block's sums of dwq, dwk
  int64_t max_blocks = 0;       // of the backward kernel
};

namespace {

struct Heads {
  void *p;
  int64_t sb, st, sh;
};

// Division by a number that the host knows: n < 2^31 by d in a multiplication, an addition and a shift
// (Granlund and Montgomery, 1994).
struct FastDiv {
  uint32_t d, m, l;
  static FastDiv of(uint32_t d) {
    uint32_t l = 0;
    while (((uint64_t)1 << l) < d) ++l;
    return {d, (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << l) - d)) / d + 1), l};
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, m) + n) >> l; }
};

constexpr int kMaxBlockTokens = 16;

// q or k.  Head h of token j of a block is unit j heads + h; a step is as many units as a warp has groups.
struct Kind {
  int32_t heads, tokens;  // tokens of a block
  int32_t steps, blocks;  // steps of a block, blocks in all
  int32_t weight;         // warps that a step counts for, among those of both kinds
  FastDiv by_heads;
};

struct Args {
  int32_t all;  // tokens of all sequences
  FastDiv by_tokens, by_pairs;
  Kind kind[2];
  int32_t steps;      // of a block, what a warp takes (a batch) at most
  int32_t dim, half;  // half = rotary / 2
  int32_t group;      // lanes per head
  bool multi;         // whether blocks have several tokens
  float eps;
  const void *pos;
  int64_t pos_sb;
  int32_t pos_dtype;
  const uint64_t *turn;
  Heads q, k, gq, gk, oq, ok;
  const float *wq, *wk;
  float *partial;  // null: no gradient of the weights
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

// A lane's pairs of a head are NC chunks of V, `group` lanes apart; V divides half and dim / 2 - half unless
// interleaved, when a chunk's pairs are 2 V neighbouring elements.  In memory and in the ring a chunk is
// two pieces of V elements (the pairs' firsts and seconds, or its two halves).
template <class T_, int V, int NC, bool INTER_>
struct Lane {
  using T = T_;
  static constexpr bool INTER = INTER_;
  static constexpr int kWidth = V, kPairs = NC * V, kPacks = kPairs / 2;
  static constexpr int kAngles = kPairs * 32;  // of the tokens of a block: as many as the warp's lanes hold pairs
  static constexpr int kPiece = V * (int)sizeof(T);   // bytes
  static constexpr int kStep = 2 * NC * 32 * kPiece;  // of a warp's ring, a step of one tensor
  int at[NC], apart[NC];  // the pieces' first elements in a head: at, at + apart
  bool has[NC];
  __device__ __forceinline__ Lane(const Args &A) {
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const int u = first_pair(A, n);
      has[n] = 2 * u < A.dim;
      at[n] = apart[n] = 0;
      if (has[n]) pair_place<INTER>(u, A.dim, A.half, at[n], apart[n]);
      if (INTER) apart[n] = V;
    }
  }
  static __device__ __forceinline__ int first_pair(const Args &A, int n) {
    return ((threadIdx.x & (A.group - 1)) + n * A.group) * V;
  }
  // starts the copies of a head into a step of the ring; zeros where there is no head or chunk
  __device__ __forceinline__ void copy(const Args &A, const T *x, bool on, char *step) const {
    char *to = step + (threadIdx.x & 31) * kPiece;
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const bool real = on && has[n];
#pragma unroll
      for (int h = 0; h < 2; ++h, to += 32 * kPiece) {
        const T *from = x + at[n] + h * apart[n];
        if constexpr (kPiece == 16)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(to)), "l"(from), "r"(real ? 16 : 0) : "memory");
        else if constexpr (kPiece >= 4)
          asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(tc::smem_u32(to)), "l"(from), "n"(kPiece),
                       "r"(real ? kPiece : 0)
                       : "memory");
        else
          *reinterpret_cast<T *>(to) = real ? *from : T(0.f);
      }
    }
  }
  // a step's pairs, packed in twos: firsts and seconds
  __device__ __forceinline__ void read(const Args &A, const char *step, uint64_t (&a)[kPacks], uint64_t (&b)[kPacks]) const {
    const char *from = step + (threadIdx.x & 31) * kPiece;
    float x[2][kPairs];
#pragma unroll
    for (int n = 0; n < NC; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        Raw<T, V> raw;
        raw.load(reinterpret_cast<const T *>(from + (2 * n + h) * 32 * kPiece));
#pragma unroll
        for (int e = 0; e < V; ++e) {
          if (INTER)  // element h V + e of the chunk's 2 V
            x[(h * V + e) & 1][n * V + (h * V + e) / 2] = raw.at(e);
          else
            x[h][n * V + e] = raw.at(e);
        }
      }
#pragma unroll
    for (int i = 0; i < kPacks; ++i) a[i] = pack2(x[0][2 * i], x[0][2 * i + 1]), b[i] = pack2(x[1][2 * i], x[1][2 * i + 1]);
  }
  __device__ __forceinline__ void store(const Args &A, T *y, bool on, const uint64_t (&a)[kPacks], const uint64_t (&b)[kPacks],
                                        char *step) const {
    if (!on) return;
    float x[2][kPairs];
#pragma unroll
    for (int i = 0; i < kPacks; ++i) unpack2(a[i], x[0][2 * i], x[0][2 * i + 1]), unpack2(b[i], x[1][2 * i], x[1][2 * i + 1]);
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      if (!has[n]) continue;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[V];
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] = INTER ? x[(h * V + e) & 1][n * V + (h * V + e) / 2] : x[h][n * V + e];
        store_vec<T, V>(y + at[n] + h * apart[n], v);
      }
    }
  }
  // the lane's values of an array of pairs in shared memory
  __device__ __forceinline__ void read_pairs(const float *from, const Args &A, uint64_t (&v)[kPacks]) const {
    float x[kPairs];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      const float *p = from + (has[n] ? first_pair(A, n) : 0);
#pragma unroll
      for (int e = 0; e < V; e += V < 4 ? V : 4) {
        float y[V < 4 ? V : 4];
        load_vec<float, (V < 4 ? V : 4)>(p + e, y);
#pragma unroll
        for (int k = 0; k < (V < 4 ? V : 4); ++k) x[n * V + e + k] = y[k];
      }
    }
#pragma unroll
    for (int i = 0; i < kPacks; ++i) v[i] = pack2(x[2 * i], x[2 * i + 1]);
  }
};

// Pairs whose firsts or seconds are aligned to two elements at most (a rotated part of 2 x 19 elements),
// in heads that are whole 16-byte pieces: heads are copied and written in pieces, through the ring's
// step, from which a lane picks its pairs one by one.  (16384 tokens of 8 + 4 heads of 256 in bf16, 102
// rotated: 73 us; with accesses of one element to global memory 98 us.)
template <class T_>
struct StagedLane : Lane<T_, 1, 4, false> {
  using Base = Lane<T_, 1, 4, false>;
  using T = T_;
  using Base::at, Base::apart, Base::has, Base::kPacks, Base::kPairs;
  __device__ __forceinline__ StagedLane(const Args &A) : Base(A) {}
  static __device__ __forceinline__ int head_bytes(const Args &A) { return A.dim * (int)sizeof(T); }
  static __device__ __forceinline__ T *head_of(const Args &A, char *step) {
    return reinterpret_cast<T *>(step + (threadIdx.x & 31) / A.group * head_bytes(A));
  }
  __device__ __forceinline__ void copy(const Args &A, const T *x, bool on, char *step) const {
    char *head = reinterpret_cast<char *>(head_of(A, step));
    for (int p = 16 * (threadIdx.x & (A.group - 1)); p < head_bytes(A); p += 16 * A.group)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(tc::smem_u32(head + p)),
                   "l"(reinterpret_cast<const char *>(x) + p), "r"(on ? 16 : 0)
                   : "memory");
  }
  __device__ __forceinline__ void read(const Args &A, char *step, uint64_t (&a)[kPacks], uint64_t (&b)[kPacks]) const {
    __syncwarp();  // each lane has waited for its own copies
    const T *head = head_of(A, step);
    float x[2][kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        Raw<T, 1> raw;
        raw.w[0] = 0;
        if (has[i]) raw.load(head + at[i] + h * apart[i]);
        x[h][i] = raw.at(0);
      }
#pragma unroll
    for (int i = 0; i < kPacks; ++i) a[i] = pack2(x[0][2 * i], x[0][2 * i + 1]), b[i] = pack2(x[1][2 * i], x[1][2 * i + 1]);
  }
  __device__ __forceinline__ void store(const Args &A, T *y, bool on, const uint64_t (&a)[kPacks], const uint64_t (&b)[kPacks],
                                        char *step) const {
    __syncwarp();  // the step is read
    T *head = head_of(A, step);
    if (on) {
      float x[2][kPairs];
#pragma unroll
      for (int i = 0; i < kPacks; ++i) unpack2(a[i], x[0][2 * i], x[0][2 * i + 1]), unpack2(b[i], x[1][2 * i], x[1][2 * i + 1]);
#pragma unroll
      for (int i = 0; i < kPairs; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float v[1] = {x[h][i]};
          if (has[i]) store_vec<T, 1>(head + at[i] + h * apart[i], v);
        }
    }
    __syncwarp();
    if (on)
      for (int p = 16 * (threadIdx.x & (A.group - 1)); p < head_bytes(A); p += 16 * A.group)
        *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(y) + p) =
            *reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(head) + p);
  }
};

// Sum over the lanes of a group (a power of two, aligned).
__device__ __forceinline__ float group_sum(float v, int group) {
  for (int o = group >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
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

// What a warp goes over: a batch of a kind's steps, and every stride-th block of tokens.  A batch of n steps
// has n `weight` of every kind[0].steps kind[0].weight + kind[1].steps kind[1].weight warps, so that all have
// the same work.
// MULTI: whether blocks have several tokens.
template <bool MULTI>
struct Unit {
  int kind, first_step, steps, heads, tokens, blocks, block, stride;
  int groups, unit;  // of a step: its units, this lane's of the batch's first
  FastDiv by_heads;
  __device__ __forceinline__ Unit(const Args &A, int id) {
    const int q_slots = A.kind[0].steps * A.kind[0].weight, cycle = q_slots + A.kind[1].steps * A.kind[1].weight;
    const int slot = id % cycle;
    kind = slot >= q_slots;
    const Kind &K = A.kind[kind];
    heads = K.heads, tokens = K.tokens, blocks = K.blocks, by_heads = K.by_heads;
    const int begin = kind ? q_slots : 0, in_kind = slot - begin;
    first_step = in_kind / K.weight / A.steps * A.steps;
    steps = min(A.steps, K.steps - first_step);
    groups = 32 / A.group, unit = first_step * groups + (threadIdx.x & 31) / A.group;
    const int before = first_step * K.weight, share = steps * K.weight;
    block = id / cycle * share + in_kind - before;
    const int warps = (int)gridDim.x * kWarps, left = warps % cycle - begin - before;
    stride = warps / cycle * share + max(0, min(left, share));
  }
};

// A block of tokens and a step of it, and this lane's head in it; runs ahead of the work (the copies) or
// with it.
template <bool MULTI>
struct Cursor {
  int block, step, seq;  // seq: blocks so far
  int in_block, h;       // the head's token in the block, the head
  int b, t;              // its sequence, its token there
  bool real;
  __device__ __forceinline__ Cursor(const Args &A, const Unit<MULTI> &U) : block(U.block), step(0), seq(0) { place(A, U); }
  __device__ __forceinline__ void place(const Args &A, const Unit<MULTI> &U) {
    const int unit = U.unit + step * U.groups;
    in_block = MULTI ? (int)U.by_heads.div(unit) : 0;
    h = unit - in_block * U.heads;
    unsigned token = MULTI ? (unsigned)block * U.tokens + in_block : block;
    real = h < U.heads;
    if (MULTI) {
      real = in_block < U.tokens && token < (unsigned)A.all;
      if (!real) in_block = h = token = 0;
    }
    b = (int)A.by_tokens.div(token), t = (int)token - b * (int)A.by_tokens.d;
  }
  __device__ __forceinline__ bool on(const Unit<MULTI> &U) const { return block < U.blocks; }
  // the next step; true where the head is no longer in the same token
  __device__ __forceinline__ bool next(const Args &A, const Unit<MULTI> &U) {
    if (++step < U.steps) {
      if (MULTI) {
        place(A, U);
        return true;
      }
      h += U.groups;
      real = h < U.heads;
      return false;
    }
    step = 0, ++seq;
    block = U.stride < U.blocks - block ? block + U.stride : U.blocks;
    if (block < U.blocks) place(A, U);
    return true;
  }
  template <class T>
  __device__ __forceinline__ T *head(const Heads &H) const {
    return static_cast<T *>(H.p) + b * H.sb + t * H.st + h * H.sh;
  }
};

// The positions of the blocks on their way: a lane per token copies them with the block's first step.
template <int S, bool MULTI>
struct Positions {
  int64_t slot[S][MULTI ? kMaxBlockTokens : 1];
  __device__ __forceinline__ void copy(const Args &A, const Unit<MULTI> &U, const Cursor<MULTI> &c) {
    const int lane = threadIdx.x & 31;
    if (!A.pos || c.step != 0 || lane >= (MULTI ? U.tokens : 1)) return;
    int b = c.b, t = c.t;
    if (MULTI) {
      const unsigned token = (unsigned)c.block * U.tokens + lane;
      if (token >= (unsigned)A.all) return;
      b = (int)A.by_tokens.div(token), t = (int)token - b * (int)A.by_tokens.d;
    }
    int64_t *to = &slot[c.seq % S][lane];
    const int64_t i = b * A.pos_sb + t;
    if (A.pos_dtype == DION_INDEX_INT64)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(tc::smem_u32(to)), "l"(static_cast<const int64_t *>(A.pos) + i)
                   : "memory");
    else
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(tc::smem_u32(to)), "l"(static_cast<const int32_t *>(A.pos) + i)
                   : "memory");
  }
  __device__ __forceinline__ int64_t of(const Args &A, int seq, int in_block) const {
    const int64_t *from = &slot[seq % S][in_block];
    return A.pos_dtype == DION_INDEX_INT64 ? *from : (int64_t)*reinterpret_cast<const int32_t *>(from);
  }
};

// Sines and cosines of the pairs of a block's tokens into the warp's shared memory, [token][pair].  position *
// turn wraps modulo one turn exactly; the top 32 bits, as a signed fraction of half a turn, are within
// 2^-31 of it, and fp32's rounding of that is 2^-25 of half a turn at most.
template <int S, bool MULTI>
__device__ __forceinline__ void block_angles(const Args &A, const Unit<MULTI> &U, const Cursor<MULTI> &at,
                                             const Positions<S, MULTI> &positions, float *cs, float *sn) {
  __syncwarp();  // the last block's were read; this one's positions are there for every lane
  const int pairs = A.dim / 2;
  const int64_t only = MULTI ? 0 : A.pos ? positions.of(A, at.seq, 0) : at.t;
  for (int i = threadIdx.x & 31; i < (MULTI ? U.tokens : 1) * pairs; i += 32) {
    const int j = MULTI ? (int)A.by_pairs.div(i) : 0, u = i - j * pairs;
    const unsigned token = MULTI ? (unsigned)at.block * U.tokens + j : at.block;
    float c = 1.f, s = 0.f;
    if (u < A.half && token < (unsigned)A.all) {
      const int64_t position = !MULTI ? only : A.pos ? positions.of(A, at.seq, j) : token - A.by_tokens.div(token) * A.by_tokens.d;
      const int32_t part = (int32_t)(((uint64_t)position * A.turn[u]) >> 32);
      sincospif((float)part * 0x1p-31f, &s, &c);
    }
    cs[i] = c, sn[i] = s;
  }
  __syncwarp();
}

__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// ------------------------------------------------------------------------------ forward ---
// Reads and writes each head once; bound by memory, close behind by instructions: 32 x 1024 tokens of 16 + 16 heads
// of 128 in bf16 87 us, 6.2 TB/s.  A lane's 16 elements take four packed products each way for the rotation
// with the weights multiplied into the sines and cosines once a token.  Heads of other widths leave lanes
// of a group idle (80 elements: 5 of 8) and are bound by instructions: 6 x 6081 tokens of 4 + 2 heads of 80 in
// 39 us, 1.8 TB/s.  One token of 16 sequences: 4.3 us of the GPU's time.
template <class L, bool MULTI>
__global__ void __launch_bounds__(kThreads, forward_blocks(L::kPairs)) forward_kernel(const __grid_constant__ Args A) {
  using T = typename L::T;
  constexpr int S = kRing, P = L::kPacks;
  __shared__ __align__(16) float w[2][2][kMaxPairs], angles[kWarps][2][MULTI ? L::kAngles : kMaxPairs];
  __shared__ __align__(16) char ring[kWarps][S][L::kStep];
  __shared__ Positions<S, MULTI> positions[kWarps];
  chain_enter();
  const int warp = threadIdx.x >> 5;
  const Unit<MULTI> U(A, blockIdx.x * kWarps + warp);
  const Heads &X = U.kind ? A.k : A.q, &Y = U.kind ? A.ok : A.oq;
  const L mine(A);
  const int64_t x_step = U.groups * X.sh, y_step = U.groups * Y.sh;
  Cursor<MULTI> ahead(A, U), at(A, U);
  const T *from = ahead.template head<const T>(X);
  T *to = at.template head<T>(Y);
  int filled = 0, used = 0;  // places of the ring
  auto fill = [&] {
    if (ahead.on(U)) {
      mine.copy(A, from, ahead.real, ring[warp][filled]);
      positions[warp].copy(A, U, ahead);
      if (ahead.next(A, U))
        from = ahead.template head<const T>(X);
      else
        from += x_step;
    }
    commit_copies();
    filled = filled + 1 == S ? 0 : filled + 1;
  };
#pragma unroll
  for (int k = 0; k < S - 1; ++k) fill();
  stage_weights<L::INTER>(A, w);  // while the first steps are on their way
  const float inv_dim = 1.f / (float)A.dim;
  uint64_t ac[P], bs[P], bc[P], as[P];  // of a token: wa cos, -wb sin, wb cos, wa sin
  while (at.on(U)) {
    wait_copies<S - 2>();
    if (at.step == 0) block_angles(A, U, at, positions[warp], angles[warp][0], angles[warp][1]);
    if (at.step == 0 || MULTI) {
      const int first = at.in_block * (A.dim / 2);
      uint64_t c[P], s[P], wa[P], wb[P];
      mine.read_pairs(angles[warp][0] + first, A, c);
      mine.read_pairs(angles[warp][1] + first, A, s);
      mine.read_pairs(w[U.kind][0], A, wa);
      mine.read_pairs(w[U.kind][1], A, wb);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        ac[i] = mul2(wa[i], c[i]), as[i] = mul2(wa[i], s[i]), bc[i] = mul2(wb[i], c[i]);
        bs[i] = mul2(mul2(wb[i], s[i]), pack2(-1.f, -1.f));
      }
    }
    uint64_t a[P], b[P], sum2 = 0, sum2b = 0;
    mine.read(A, ring[warp][used], a, b);
#pragma unroll
    for (int i = 0; i < P; ++i) sum2 = fma2(a[i], a[i], sum2), sum2b = fma2(b[i], b[i], sum2b);
    float sum, more;
    unpack2(add2(sum2, sum2b), sum, more);
    const float r = rsqrtf(group_sum(sum + more, A.group) * inv_dim + A.eps);
    const uint64_t r2 = pack2(r, r);
    uint64_t ya[P], yb[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      ya[i] = mul2(r2, fma2(b[i], bs[i], mul2(a[i], ac[i])));
      yb[i] = mul2(r2, fma2(a[i], as[i], mul2(b[i], bc[i])));
    }
    mine.store(A, to, at.real, ya, yb, ring[warp][used]);
    used = used + 1 == S ? 0 : used + 1;
    if (at.next(A, U))
      to = at.template head<T>(Y);
    else
      to += y_step;
    fill();
  }
}

// ----------------------------------------------------------------------------- backward ---
// Reads x and g once, writes dx once, and adds up dw in registers over all of a warp's tokens: the weights'
// gradient costs no memory but a block's sums at the end.  Two means per head (of x^2 and of w gu x) share one
// round of shuffles.  Bound by memory: 32 x 1024 tokens of 16 + 16 heads of 128 in bf16 134 us with the sums of
// dw, 6.0 TB/s; a few thousand tokens by their latency (3 x 701 of 12 + 12 heads of 64 in fp32: 9.5 us, and 4.0
// for the sums).
template <class L, bool MULTI>
__global__ void __launch_bounds__(kThreads, backward_blocks(L::kPairs)) backward_kernel(const __grid_constant__ Args A) {
  using T = typename L::T;
  constexpr int S = kRing, P = L::kPacks;
  __shared__ __align__(16) float w[2][2][kMaxPairs], angles[kWarps][2][MULTI ? L::kAngles : kMaxPairs];
  __shared__ __align__(16) char ring[kWarps][S][2][L::kStep];
  __shared__ Positions<S, MULTI> positions[kWarps];
  chain_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Unit<MULTI> U(A, blockIdx.x * kWarps + warp);
  const Heads &X = U.kind ? A.k : A.q, &G = U.kind ? A.gk : A.gq, &Y = U.kind ? A.ok : A.oq;
  const L mine(A);
  const int64_t x_step = U.groups * X.sh, g_step = U.groups * G.sh, y_step = U.groups * Y.sh;
  Cursor<MULTI> ahead(A, U), at(A, U);
  const T *from = ahead.template head<const T>(X), *from_g = ahead.template head<const T>(G);
  T *to = at.template head<T>(Y);
  int filled = 0, used = 0;
  auto fill = [&] {
    if (ahead.on(U)) {
      mine.copy(A, from, ahead.real, ring[warp][filled][0]);
      mine.copy(A, from_g, ahead.real, ring[warp][filled][1]);
      positions[warp].copy(A, U, ahead);
      if (ahead.next(A, U))
        from = ahead.template head<const T>(X), from_g = ahead.template head<const T>(G);
      else
        from += x_step, from_g += g_step;
    }
    commit_copies();
    filled = filled + 1 == S ? 0 : filled + 1;
  };
#pragma unroll
  for (int k = 0; k < S - 1; ++k) fill();
  stage_weights<L::INTER>(A, w);  // while the first steps are on their way
  const float inv_dim = 1.f / (float)A.dim;
  uint64_t c[P], s[P], ns[P], wa[P], wb[P], da[P], db[P];  // ns = -s; da, db: this lane's sums of dw
  mine.read_pairs(w[U.kind][0], A, wa);
  mine.read_pairs(w[U.kind][1], A, wb);
#pragma unroll
  for (int i = 0; i < P; ++i) da[i] = db[i] = 0;
  while (at.on(U)) {
    wait_copies<S - 2>();
    if (at.step == 0) block_angles(A, U, at, positions[warp], angles[warp][0], angles[warp][1]);
    if (at.step == 0 || MULTI) {
      const int first = at.in_block * (A.dim / 2);
      mine.read_pairs(angles[warp][0] + first, A, c);
      mine.read_pairs(angles[warp][1] + first, A, s);
#pragma unroll
      for (int i = 0; i < P; ++i) ns[i] = mul2(s[i], pack2(-1.f, -1.f));
    }
    uint64_t a[P], b[P], ga[P], gb[P], sum2 = 0, sum2b = 0, dot2 = 0, dot2b = 0;
    mine.read(A, ring[warp][used][0], a, b);
    mine.read(A, ring[warp][used][1], ga, gb);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const uint64_t oa = ga[i], ob = gb[i];
      ga[i] = fma2(ob, s[i], mul2(oa, c[i]));
      gb[i] = fma2(oa, ns[i], mul2(ob, c[i]));
      sum2 = fma2(a[i], a[i], sum2), sum2b = fma2(b[i], b[i], sum2b);
      dot2 = fma2(mul2(ga[i], wa[i]), a[i], dot2), dot2b = fma2(mul2(gb[i], wb[i]), b[i], dot2b);
    }
    float sum, dot, more;
    unpack2(add2(sum2, sum2b), sum, more);
    sum += more;
    unpack2(add2(dot2, dot2b), dot, more);
    dot += more;
    for (int o = A.group >> 1; o > 0; o >>= 1) {
      sum += __shfl_xor_sync(0xffffffffu, sum, o);
      dot += __shfl_xor_sync(0xffffffffu, dot, o);
    }
    const float r = rsqrtf(sum * inv_dim + A.eps);
    const float back = -dot * inv_dim * r * r * r;  // dx = r w gu - x r^3 mean(w gu x)
    const uint64_t r2 = pack2(r, r), back2 = pack2(back, back);
    if (at.real) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const uint64_t ra = mul2(r2, ga[i]), rb = mul2(r2, gb[i]);
        da[i] = fma2(ra, a[i], da[i]), db[i] = fma2(rb, b[i], db[i]);
        a[i] = fma2(ra, wa[i], mul2(a[i], back2));
        b[i] = fma2(rb, wb[i], mul2(b[i], back2));
      }
    }
    mine.store(A, to, at.real, a, b, ring[warp][used][0]);
    used = used + 1 == S ? 0 : used + 1;
    if (at.next(A, U))
      to = at.template head<T>(Y);
    else
      to += y_step;
    fill();
  }
  if (!A.partial) return;
  // the block's sums of dw, over the groups of a warp, then over the warps, in the angles' place
  __syncwarp();
  constexpr int kRed = sizeof(angles[0]) / sizeof(float);
  float *red = &angles[0][0][0];  // [kWarps][dim] of the warp's kind
  for (int d = lane; d < A.dim; d += 32) red[warp * kRed + d] = 0.f;
  __syncwarp();
#pragma unroll
  for (int i = 0; i < L::kPairs; ++i) {
    float v[4];
    unpack2(da[i / 2], v[0], v[1]);
    unpack2(db[i / 2], v[2], v[3]);
    float va = v[i & 1], vb = v[2 + (i & 1)];
    for (int o = A.group; o < 32; o <<= 1) {
      va += __shfl_xor_sync(0xffffffffu, va, o);
      vb += __shfl_xor_sync(0xffffffffu, vb, o);
    }
    if (lane < A.group && mine.has[i / L::kWidth]) {
      int place, apart;
      pair_place<L::INTER>(L::first_pair(A, i / L::kWidth) + i % L::kWidth, A.dim, A.half, place, apart);
      red[warp * kRed + place] = va, red[warp * kRed + place + apart] = vb;
    }
  }
  __syncthreads();
  const int q_slots = A.kind[0].steps * A.kind[0].weight, cycle = q_slots + A.kind[1].steps * A.kind[1].weight;
  for (int d = threadIdx.x; d < 2 * A.dim; d += kThreads) {
    const int kind = d >= A.dim;
    float v = 0.f;
    for (int k = 0; k < kWarps; ++k)
      if ((((int)blockIdx.x * kWarps + k) % cycle >= q_slots) == (kind != 0)) v += red[k * kRed + d - kind * A.dim];
    A.partial[(int64_t)blockIdx.x * 2 * A.dim + d] = v;
  }
}

// dw from the blocks' sums: a block per 32 columns, whose warps take the rows in turn; fixed order.  Bound by
// latency: 456 blocks' sums of 2 x 128 in 4 us.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads) sum_weights_kernel(const float *partial, int blocks, int dim, float *dwq, float *dwk) {
  __shared__ float red[kSumThreads / 32][33];
  chain_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (d < 2 * dim)
#pragma unroll 8
    for (int b = warp; b < blocks; b += kSumThreads / 32) v += partial[(int64_t)b * 2 * dim + d];
  red[warp][lane] = v;
  __syncthreads();
  v = red[lane][warp];  // lane l: the sum of warp l for column `warp`
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const int col = blockIdx.x * 32 + warp;
  if (lane != 0 || col >= 2 * dim) return;
  float *to = col < dim ? dwq : dwk;
  if (to) to[col < dim ? col : col - dim] = v;
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
  if (s->batch > 0 && s->tokens > INT32_MAX / s->batch) return DION_ERR_UNSUPPORTED;
  return DION_OK;
}

// Instructions per token in blocks of n tokens, for `heads` heads of which a warp takes `groups` at a time:
// about 170 for a step, 300 in the kernel where each step may be of other tokens, 50 for each 32 of the
// block's angles, 80 for the block.
double block_cost(int n, bool multi, int heads, int groups, int pairs) {
  const int steps = (n * heads + groups - 1) / groups;
  return (double)(steps * (multi ? 300 : 170) + (n * pairs + 31) / 32 * 50 + 80) / n;
}
// The tokens of a block with the least of them, up to `most`; each of `warps` warps is left one block at least.
int block_tokens(int heads, int groups, int pairs, int most, int64_t all, int64_t warps) {
  int best = 1;
  for (int n = 2; heads > 0 && n <= most && (all + n - 1) / n >= warps; ++n)
    if (block_cost(n, true, heads, groups, pairs) < block_cost(best, true, heads, groups, pairs)) best = n;
  return best;
}

// Args of a call whose kernel has `pairs` pairs per lane and `resident` blocks at a time, and the blocks that it
// takes.
Args make_args(const dion_qknorm_plan *p, const dion_qk_shape *s, int pairs, int64_t resident, int64_t *blocks) {
  Args A{};
  A.all = (int32_t)(s->batch * s->tokens);
  A.by_tokens = FastDiv::of((uint32_t)s->tokens), A.by_pairs = FastDiv::of((uint32_t)p->head_dim / 2);
  A.dim = p->head_dim, A.half = p->rotary / 2, A.eps = p->eps;
  A.pos = s->positions, A.pos_sb = s->position_batch_stride, A.pos_dtype = s->position_dtype;
  A.turn = p->turn;
  A.group = 1;
  while (A.group * pairs < p->head_dim / 2) A.group *= 2;
  const int groups = 32 / A.group, most = std::min(kMaxBlockTokens, pairs * 64 / p->head_dim);
  // blocks of several tokens, where both kinds together gain (71829 tokens of 3 + 3 heads of 96 in bf16: 91 us
  // token by token, 62 in blocks of four; 63915 tokens of 12 + 3 heads of 32: 67 and 38 us)
  int tokens[2];
  double single = 0, several = 0;
  for (int i = 0; i < 2; ++i) {
    const int heads = i ? s->kv_heads : s->heads, half = p->head_dim / 2;
    tokens[i] = block_tokens(heads, groups, half, most, A.all, resident * kWarps);
    if (heads == 0) continue;
    single += block_cost(1, false, heads, groups, half);
    several += block_cost(tokens[i], true, heads, groups, half);
  }
  const bool multi = A.multi = several < single;
  int64_t cycle = 0, work = 0;
  for (int i = 0; i < 2; ++i) {
    Kind &K = A.kind[i];
    K.heads = i ? s->kv_heads : s->heads;
    K.tokens = multi ? tokens[i] : 1;
    K.steps = (K.tokens * K.heads + groups - 1) / groups;
    K.blocks = (int32_t)(((int64_t)A.all + K.tokens - 1) / K.tokens);
    K.by_heads = FastDiv::of((uint32_t)std::max(K.heads, 1));
  }
  for (int i = 0; i < 2; ++i) {  // a step of this kind is done once for each of its blocks
    Kind &K = A.kind[i];
    K.weight = A.kind[1 - i].tokens / std::gcd(K.tokens, A.kind[1 - i].tokens);
    cycle += (int64_t)K.steps * K.weight, work += (int64_t)K.steps * K.blocks;
  }
  // a warp takes several steps of a block, which share its angles, as far as every warp has some
  A.steps = (int32_t)std::max<int64_t>(1, std::min<int64_t>(kMaxSteps, work / (resident * kWarps)));
  *blocks = (std::max(std::min(resident * kWarps, work), cycle) + kWarps - 1) / kWarps;
  return A;
}

// Whether every head of the tensors is whole 16-byte pieces.
bool heads_in_pieces(const dion_qknorm_plan *p, const dion_qk_shape *s, const Heads *h, int n) {
  const int es = element_bytes(s->dtype), v = 16 / es;
  bool fits = p->head_dim % v == 0;
  for (int i = 0; i < n; ++i)
    fits = fits && (!h[i].p || (aligned_to(h[i].p, 16) && h[i].sb % v == 0 && h[i].st % v == 0 && h[i].sh % v == 0));
  return fits;
}

// What a lane holds: `v` pairs per access, or staged.
template <class L>
struct Tag {
  using type = L;
};
template <class T, bool INTER, class F>
cudaError_t with_width(int v, bool staged, F &&f) {
  if constexpr (sizeof(T) == 2)
    if (v == 8) return f(Tag<Lane<T, 8, 1, INTER>>());
  if (v == 4) return f(Tag<Lane<T, 4, 1, INTER>>());
  if constexpr (!INTER)
    if (staged) return f(Tag<StagedLane<T>>());
  if (v == 2) return f(Tag<Lane<T, 2, 2, INTER>>());
  return f(Tag<Lane<T, 1, 4, INTER>>());
}
template <class F>
cudaError_t with_lane(int32_t dtype, int v, bool staged, bool inter, F &&f) {
  using BF = __nv_bfloat16;
  if (dtype == DION_DTYPE_FP32) return inter ? with_width<float, true>(v, staged, f) : with_width<float, false>(v, staged, f);
  return inter ? with_width<BF, true>(v, staged, f) : with_width<BF, false>(v, staged, f);
}

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
  // the resident blocks, or a warp for every step (times its weight) of the most heads that a call may have
  p->max_blocks = std::max<int64_t>((int64_t)p->num_sms * backward_blocks(4), 4 * kMaxHeads / kWarps);
  const size_t o_partial = sizeof(turn);
  if (e == cudaSuccess) e = cudaMalloc(&p->ws, o_partial + sizeof(float) * 2 * head_dim * p->max_blocks);
  if (e == cudaSuccess) {
    char *b = static_cast<char *>(p->ws);
    p->turn = reinterpret_cast<uint64_t *>(b);
    p->partial = reinterpret_cast<float *>(b + o_partial);
    e = cudaMemcpy(p->turn, turn, sizeof(turn), cudaMemcpyHostToDevice);
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
  int64_t blocks = 0;
  Args A = make_args(p, s, v == 8 ? 8 : 4, (int64_t)p->num_sms * forward_blocks(v == 8 ? 8 : 4), &blocks);
  A.q = h[0], A.k = h[1], A.oq = h[2], A.ok = h[3], A.wq = wq, A.wk = wk;
  const bool multi = A.multi;
  const cudaError_t e = with_lane(s->dtype, v, heads_in_pieces(p, s, h, 4), p->interleaved, [&](auto lane) {
    using L = typename decltype(lane)::type;
    return launch(multi ? forward_kernel<L, true> : forward_kernel<L, false>, blocks, kThreads, 0,
                  static_cast<cudaStream_t>(stream), 1, A);
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
  int64_t blocks = 0;
  Args A = make_args(p, s, v == 8 ? 8 : 4, (int64_t)p->num_sms * backward_blocks(v == 8 ? 8 : 4), &blocks);
  A.gq = h[0], A.gk = h[1], A.q = h[2], A.k = h[3], A.oq = h[4], A.ok = h[5];
  A.wq = wq, A.wk = wk, A.partial = dwq || dwk ? p->partial : nullptr;
  const bool multi = A.multi;
  cudaError_t e = with_lane(s->dtype, v, heads_in_pieces(p, s, h, 6), p->interleaved, [&](auto lane) {
    using L = typename decltype(lane)::type;
    return launch(multi ? backward_kernel<L, true> : backward_kernel<L, false>, blocks, kThreads, 0, cs, 1, A);
  });
  if (e == cudaSuccess && A.partial)
    e = launch(sum_weights_kernel, (2 * p->head_dim + 31) / 32, kSumThreads, 0, cs, 1, p->partial, (int)blocks, p->head_dim, dwq,
               dwk);
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
