// Softmax cross entropy of node states against a vocabulary, in pieces of the vocabulary, with its
// gradient; the [n, V] logits are never in memory:
//   z = X W^T,  lse_i = log sum_v exp(z_iv),  loss_i = lse_i - z_{i,t_i}
//   P = softmax(z) - onehot(t),  dX = diag(g) P W,  dW = P^T diag(g) X     (g: the loss's gradient)
//
// Three kinds of kernels:
//   k_xent_count, k_xent_rows   the labelled rows of X, gathered side by side (rows left out cost
//                               nothing after this and may hold anything), and the operands' 16-bit forms;
//                               a few microseconds, bytes and latency
//   k_xent_fwd (+ join)         128 x 256 tiles of z in tensor memory, sum of exponentials.  65537 rows x
//                               49999: 0.88 ms at H = 256, bound by the product (tensor pipe 92% active,
//                               0.87 ms at the measured peak); 0.63 ms at H = 64, in the epilogue, no unit
//                               of it full (special functions 59% of their rate, issue slots 52%): its 16
//                               warps work on one accumulator in step and wait for the special functions'
//                               queue together
//   k_xent_bwd (+ join)         128 x 128 tiles of z recomputed, P written back over z in tensor
//                               memory as the A operand of the second product; some CTAs with the rows
//                               of X staying (dX), the others with the rows of W (dW).  The same shape:
//                               4.0 ms at H = 256 for four products (3.5 at the measured peak; tensor
//                               pipe 78%), 1.56 ms at H = 64 (epilogue: issue slots 67%); with fp32
//                               gradients 6.6 ms and 2.66 (six products)
// A staying tile of 128 rows against one passing tile is a unit; the units of a launch, staying tile
// by staying tile, are cut into as many equal runs as there are SMs, so one row or a hundred thousand
// fill the card alike.  A staying tile whose units fall to several CTAs leaves partial results, which
// the join adds in the order of the CTAs.  The number of labelled rows is known on the device only:
// every kernel derives its runs from it.
//
// Number formats ("forms") of the operands:
//   bf16           X and W as they are; P rounded to bf16 (bf16 gradients, whose own rounding is as large)
//   fp16, 1 term   bf16 X and W with fp32 gradients: scaled by a power of two, they are exact in
//                  fp16 (down to 2^-29 of the largest), and P, as the sum of two fp16 terms, keeps 21 bits;
//                  fp16 and bf16 operands cannot be mixed in one product
//   fp16, 2 terms  fp32 X and W, each the sum of two fp16 terms (22 bits, down to 2^-17 of the largest,
//                  below that off by 2^-39 of it at most); products of the two low terms (2^-22) are left out
// The largest is that of a row of X, and that of all of W.  X's exponents go with the rows' statistics (as
// W's could not: a row of X is a thread's in the forward, a row of W a column, whose factor would have to
// be read for each of its logits); one exponent for all of X lost other rows' bits to one large row.
// The tensor core truncates when it adds to its fp32 accumulator.  Measured: a step of 16 products loses
// 0.2-0.45 x 2^-24 of the accumulator where signs are mixed, 3.4 x 2^-24 where all are of one sign, always
// towards zero, so that a sum of N steps of one sign ends up 1.7 N x 2^-24 low.  A gradient in fp32 leaves
// tensor memory every kDrainSteps steps and is added up in registers (low by 2^-18 at most: 2.8e-6
// measured); one in bf16 leaves it every kLongSteps steps and is added up in the CTA's partial result
// (2^-12, an eighth of bf16's half gap; 65537 rows x 49999: 2% longer at H = 256 than without, no difference
// at H <= 192; 1024 steps took 5%).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>
#include <numeric>

#include "gemm_tc.h"
#include "kernels.h"
#include "tc_util.cuh"
#include "token.h"

namespace bg {

using namespace tc;

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kDrainSteps = 64, kLongSteps = 2048;

enum Form { kBf16 = 0, kF16x1 = 1, kF16x2 = 2 };

// ------------------------------------------------------------------------------ workspace
inline size_t al(size_t x) { return (x + 255) & ~(size_t)255; }

// CTAs of a tile kernel at most: one on each SM of a GB300.  The workspace has partial results for so many,
// whatever device a call runs on.
constexpr int kMaxCtas = 152;
constexpr int kMaxRowBlocks = 2048;
constexpr int kTableBlocks = 608;  // at most, of the table's amax and conversion
constexpr int64_t kDirectRows = 32768;

// Rows of one block of k_xent_count / k_xent_rows: few, so that many blocks share the copying, while
// there are at most kMaxRowBlocks blocks (each adds up the counts of those before it).
inline int64_t rows_per_block(int64_t n) {
  return n <= 64LL * 1024 ? 64 : 256 * ((n + 256LL * kMaxRowBlocks - 1) / (256LL * kMaxRowBlocks));
}

struct Ws {
  int64_t rb, nb, cap, vcap;  // rows a block, blocks, X rows and W rows rounded up to whole tiles
  size_t head, counts, amax, xexp, row, stat, hit, x, w, full, part, total;
};

Ws layout(int form, int64_t n, int H, int V, int backward, int ctas) {
  Ws w{};
  w.rb = rows_per_block(n);
  w.nb = std::max<int64_t>(1, (n + w.rb - 1) / w.rb);
  w.cap = (n + 127) / 128 * 128;
  w.vcap = ((int64_t)V + 127) / 128 * 128;
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += al(bytes);
    return at;
  };
  const int terms = form == kF16x2 ? 2 : 1;
  w.head = take(16);
  w.counts = take((size_t)w.nb * 4);
  w.amax = take((size_t)(w.nb + kTableBlocks) * 4);
  w.xexp = take(form == kBf16 ? 0 : (size_t)n);
  w.row = take((size_t)w.cap * 4);
  w.stat = take((size_t)w.cap * 16);
  w.hit = take((size_t)w.cap * 4);
  w.x = take((size_t)terms * w.cap * H * 2);
  w.w = take(form == kBf16 ? 0 : (size_t)terms * w.vcap * H * 2);
  w.full = take(backward ? 0 : (size_t)w.cap * 32);
  w.part = take(backward ? (size_t)ctas * 2 * 128 * H * 4 : (size_t)ctas * 2 * 512 * 8);
  w.total = o;
  return w;
}

// Statistics of the gathered rows ("slots"), in blocks of 64, so that one copy brings a tile's: -lse (bf16
// form: times log2 e), dloss (fp16 forms: times 2^e, e the exponent of the row's largest element, which X's
// terms lack), the target, and what the row's logits are multiplied by to undo the operands' scales.
enum { kNlse = 0, kG = 64, kTgt = 128, kDs = 192 };
constexpr int kNoTarget = -2;  // target of a row that counts and has none (-1: no row)
__host__ __device__ __forceinline__ int64_t stat_at(int64_t slot) { return slot / 64 * 256 + slot % 64; }

// ------------------------------------------------------------------------------ rows
struct RowArgs {
  int form, x_bf16, backward, grad_bf16, clear_dx;
  int soft;            // rows have no target of their own
  float inv_tau, tau;  // the logits' and the weights' factor (1: plain cross entropy)
  int direct;  // k_xent_rows counts by itself: k_xent_count did not run
  int tb;      // blocks that work on the table
  int64_t n, rb, nb, cap, vcap;
  int H, V;
  const void* X;
  const void* W;
  const int32_t* target;
  const float* lse_in;
  const float* dloss;
  int* head;  // number of labelled rows; exponents of the scales of W and of the weights (fp16 forms)
  int* counts;
  uint32_t* amax;  // [nb] of dloss 2^e, [tb] of W: bits of the largest finite magnitude
  int8_t* xexp;    // [n] exponent e of each labelled row's largest finite element
  int32_t* row;
  float* stat;
  uint16_t* x;
  uint16_t* w;
  float* loss;
  float* lse_out;
  void* dX;
  int* status;
};

__device__ __forceinline__ void load8f(const void* p, int bf16, int64_t at, float* v) {
  if (bf16) {
    const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + at);
    const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(u[j] << 16);
      v[2 * j + 1] = __uint_as_float(u[j] & 0xFFFF0000u);
    }
  } else {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    const float4 a = q[0], b = q[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}

__device__ __forceinline__ uint32_t amax8(const float* v, uint32_t m) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t b = __float_as_uint(v[j]) & 0x7FFFFFFFu;
    if (b < 0x7F800000u) m = max(m, b);
  }
  return m;
}

// The maxima over the block of two values at once (sm [16]).
__device__ __forceinline__ void block_max2(uint32_t& a, uint32_t& b, uint32_t* sm) {
  a = __reduce_max_sync(0xffffffffu, a);
  b = __reduce_max_sync(0xffffffffu, b);
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0) sm[warp] = a, sm[8 + warp] = b;
  __syncthreads();
  for (int i = 0; i < 8; ++i) {
    a = max(a, sm[i]);
    b = max(b, sm[8 + i]);
  }
}

// Exponent of the number with these bits, -100 at least.
__device__ __forceinline__ int exp_of(uint32_t bits) { return max((int)(bits >> 23) - 127, -100); }
// Exponent k such that values of magnitude up to the one with these bits, times 2^k, are below 2^15.
__device__ __forceinline__ int shift_of(uint32_t bits) { return 14 - exp_of(bits); }
__device__ __forceinline__ float pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// Labelled rows of each block of rb rows and, for the fp16 forms, the exponent of each one's largest finite
// element, the largest magnitude of their weights (dloss 2^e) and of W.  X has a scale a row: one large row
// does not cost the others their bits.
__global__ void __launch_bounds__(256) k_xent_count(RowArgs a) {
  __shared__ uint32_t sm[16];
  __shared__ uint32_t top[256];
  __shared__ int sums[8];
  grid_dep_launch();
  grid_dep_wait();
  const int lanes = a.H / 8, tid = threadIdx.x;
  uint32_t mg = 0, mw = 0;
  if ((int64_t)blockIdx.x >= a.nb) {
    const int b = blockIdx.x - (int)a.nb;
    const int64_t chunks = (int64_t)a.V * lanes;
#pragma unroll 4
    for (int64_t i = (int64_t)b * 256 + tid; i < chunks; i += (int64_t)a.tb * 256) {
      float v[8];
      load8f(a.W, a.x_bf16, i * 8, v);
      mw = amax8(v, mw);
    }
    block_max2(mg, mw, sm);
    if (tid == 0) a.amax[a.nb + b] = mw;
    return;
  }
  const int64_t r0 = blockIdx.x * a.rb, r1 = min(a.n, r0 + a.rb);
  // a row is `lanes` threads; those of them that are in this warp
  const int rows = 256 / lanes, r = tid / lanes, q = tid % lanes;
  const int w0 = max(r * lanes, tid & ~31), w1 = min((r + 1) * lanes, (tid | 31) + 1);
  const unsigned mates = (0xffffffffu >> (32 - (w1 - w0))) << (w0 & 31);
  int c = 0;
  for (int64_t g0 = r0; g0 < r1; g0 += 256) {
    if (a.form != kBf16) {
      __syncthreads();
      top[tid] = 0;
      __syncthreads();
      if (r < rows)
#pragma unroll 4
        for (int k = r; k < 256 && g0 + k < r1; k += rows) {
          const int t = a.target[g0 + k];
          if (t < 0 || t >= a.V) continue;
          float v[8];
          load8f(a.X, a.x_bf16, (g0 + k) * a.H + q * 8, v);
          const uint32_t m = __reduce_max_sync(mates, amax8(v, 0));
          if (tid == w0) atomicMax(&top[k], m);
        }
      __syncthreads();
    }
    const int64_t i = g0 + tid;
    const int t = i < r1 ? a.target[i] : -1;
    if (t < 0 || t >= a.V) continue;
    ++c;
    if (a.form == kBf16) continue;
    const int e = exp_of(top[tid]);
    a.xexp[i] = (int8_t)e;
    if (a.backward) {
      const uint32_t b = __float_as_uint(a.dloss[i] * a.tau * pow2(e)) & 0x7FFFFFFFu;
      if (b < 0x7F800000u) mg = max(mg, b);
    }
  }
  __syncwarp();
  c = __reduce_add_sync(0xffffffffu, c);
  if ((tid & 31) == 0) sums[tid >> 5] = c;
  block_max2(mg, mw, sm);  // (and the barrier that the sums need)
  if (tid == 0) {
    int s = 0;
    for (int i = 0; i < 8; ++i) s += sums[i];
    a.counts[blockIdx.x] = s;
    a.amax[blockIdx.x] = mg;
  }
}

// 8 elements to the form's terms: plane t of `dst` starts at t * plane.
__device__ __forceinline__ void put8(uint16_t* dst, int64_t plane, int64_t at, int form, float scale,
                                     const float* v) {
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float x = v[2 * j] * scale, y = v[2 * j + 1] * scale;
    const __half2 h = __floats2half2_rn(x, y);
    hi[j] = *reinterpret_cast<const uint32_t*>(&h);
    const float2 f = __half22float2(h);
    const __half2 l = __floats2half2_rn(x - f.x, y - f.y);
    lo[j] = *reinterpret_cast<const uint32_t*>(&l);
  }
  *reinterpret_cast<uint4*>(dst + at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  if (form == kF16x2)
    *reinterpret_cast<uint4*>(dst + plane + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
}

// The labelled rows, side by side in their order: X in the form's terms, the row each came from, its
// target and, for the gradient, its lse and g; the outputs of the rows left out.  The last block adds
// empty rows up to a whole tile (zeros, -lse = -inf: every probability 0) and the number of rows.  The
// blocks from nb on convert W.
__global__ void __launch_bounds__(256) k_xent_rows(RowArgs a) {
  __shared__ int wsum[8];
  __shared__ uint32_t sm[16];
  __shared__ int64_t from[256];  // row of each slot of the group at hand
  __shared__ float up[256];      // and the scale of its elements
  grid_dep_launch();
  grid_dep_wait();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int lanes = a.H / 8, rows = 256 / lanes, rr = tid / lanes, q = tid % lanes;
  const bool table = (int64_t)blockIdx.x >= a.nb;
  uint32_t mg = 0, mw = 0;
  int before = 0;  // labelled rows of the blocks before this one
  if (!table) {
    if (a.direct) {
      const int4* t4 = reinterpret_cast<const int4*>(a.target);
#pragma unroll 8
      for (int i = tid; i < (int)(blockIdx.x * a.rb / 4); i += 256) {
        const int4 t = t4[i];
        before += (t.x >= 0 && t.x < a.V) + (t.y >= 0 && t.y < a.V) + (t.z >= 0 && t.z < a.V) +
                  (t.w >= 0 && t.w < a.V);
      }
    } else {
#pragma unroll 4
      for (int64_t i = tid; i < (int64_t)blockIdx.x; i += 256) before += a.counts[i];
    }
    before = __reduce_add_sync(0xffffffffu, before);
    if (lane == 0) wsum[warp] = before;
  }
  if (a.form != kBf16) {
#pragma unroll 4
    for (int64_t i = tid; i < a.nb; i += 256) mg = max(mg, a.amax[i]);
    for (int i = tid; i < a.tb; i += 256) mw = max(mw, a.amax[a.nb + i]);
  }
  block_max2(mg, mw, sm);
  if (table) {
    const int b = blockIdx.x - (int)a.nb;
    const float scale = pow2(shift_of(mw));
    const int64_t chunks = (int64_t)a.V * lanes, all = a.vcap * lanes;
#pragma unroll 4
    for (int64_t i = (int64_t)b * 256 + tid; i < all; i += (int64_t)a.tb * 256) {
      float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (i < chunks) load8f(a.W, a.x_bf16, i * 8, v);
      put8(a.w, a.vcap * a.H, i * 8, a.form, scale, v);
    }
    return;
  }
  int64_t base = 0;
  for (int i = 0; i < 8; ++i) base += wsum[i];
  const int64_t r0 = blockIdx.x * a.rb, r1 = min(a.n, r0 + a.rb);
  for (int64_t g0 = r0; g0 < r1; g0 += 256) {
    const int64_t i = g0 + tid;
    int t = i < r1 ? a.target[i] : -1;
    if (t >= a.V) {
      if (atomicCAS(a.status, 0, 2) == 0) atomicExch(a.status + 1, kSiteXentTarget);
      t = -1;
    }
    const unsigned ballot = __ballot_sync(0xffffffffu, t >= 0);
    __syncthreads();
    if (lane == 0) wsum[warp] = __popc(ballot);
    __syncthreads();
    int before = 0, count = 0;
    for (int w = 0; w < 8; ++w) {
      before += w < warp ? wsum[w] : 0;
      count += wsum[w];
    }
    if (t >= 0) {
      const int k = before + __popc(ballot & ((1u << lane) - 1));
      const int64_t slot = base + k;
      from[k] = i;
      a.row[slot] = (int32_t)i;
      float* st = a.stat + stat_at(slot);
      st[kTgt] = __int_as_float(a.soft ? kNoTarget : t);
      int e = 0;
      if (a.form != kBf16) {
        e = a.xexp[i];
        up[k] = pow2(14 - e);
        st[kDs] = pow2(max(-126, min(127, e - 14 - shift_of(mw)))) * a.inv_tau;
      }
      if (a.backward) {
        const float lse = safe_lse(a.lse_in[i]);
        st[kNlse] = a.form == kBf16 ? -lse * kLog2e : -lse;
        st[kG] = a.dloss[i] * a.tau * pow2(e);
      }
    } else if (i < r1 && !a.backward) {
      a.loss[i] = 0.f;
      a.lse_out[i] = 0.f;
    }
    __syncthreads();
    if (rr < rows) {
      for (int k = rr; k < count; k += rows) {
        const int64_t src = from[k] * a.H + q * 8, dst = (base + k) * a.H + q * 8;
        if (a.form == kBf16) {
          *reinterpret_cast<uint4*>(a.x + dst) =
              *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.X) + src);
        } else {
          float v[8];
          load8f(a.X, a.x_bf16, src, v);
          put8(a.x, a.cap * a.H, dst, a.form, up[k], v);
        }
      }
      if (a.clear_dx)
        for (int k = rr; k < 256 && g0 + k < r1; k += rows) {
          const int tk = a.target[g0 + k];
          if (tk >= 0 && tk < a.V) continue;
          const int64_t at = (g0 + k) * a.H + q * 8;
          const uint4 zero = make_uint4(0, 0, 0, 0);
          if (a.grad_bf16) {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.dX) + at) = zero;
          } else {
            uint4* p = reinterpret_cast<uint4*>(static_cast<float*>(a.dX) + at);
            p[0] = zero;
            p[1] = zero;
          }
        }
    }
    base += count;
  }
  if ((int64_t)blockIdx.x == a.nb - 1) {
    const int64_t end = (base + 127) / 128 * 128;
    if (tid == 0) {
      a.head[0] = (int)base;
      if (a.form != kBf16) {
        a.head[1] = shift_of(mw);
        a.head[2] = shift_of(mg);
      }
    }
    for (int64_t s = base + tid; s < end; s += 256) {
      a.row[s] = -1;
      float* st = a.stat + stat_at(s);
      st[kTgt] = __int_as_float(-1);
      st[kDs] = 1.f;
      if (a.backward) {
        st[kNlse] = -INFINITY;
        st[kG] = 0.f;
      }
    }
    if (rr < rows)
      for (int64_t s = base + rr; s < end; s += rows) {
        const uint4 zero = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(a.x + s * a.H + q * 8) = zero;
        if (a.form == kF16x2) *reinterpret_cast<uint4*>(a.x + (a.cap + s) * a.H + q * 8) = zero;
      }
  }
}

// ------------------------------------------------------------------------------ units
// Unit u = t * ct + j is staying tile t against passing tile j; CTA c takes [begin(c), begin(c + 1)).
// Where a tile has few units (kWholeUnits), the runs are of whole tiles: nothing is left to join, and
// the launch that would do it is saved.
// With fewer units than CTAs the last CTAs take none, so that those between a tile's first and last
// all have a part of it.
constexpr int kWholeUnits = 4;
struct Units {
  int64_t ct, U;
  int G;  // CTAs that take units
  int step, nt;
  bool tiles;  // runs are of whole staying tiles
  __device__ Units(int64_t rt, int64_t ct_, int ctas, bool tiles_, int step_ = 1)
      : ct(ct_), U(rt * ct_), G((int)min((int64_t)ctas, tiles_ ? rt : rt * ct_)), step(step_),
        nt((int)rt), tiles(tiles_) {}
  // The rows that staying tile t stands for: tile t * step mod nt (step prime to nt).  Tiles of
  // frequent tokens, whose units take up to half as long again, then do not all fall to one CTA.
  __device__ int tile(int t) const { return step == 1 ? t : (int)((uint32_t)t * (uint64_t)(uint32_t)step % (uint32_t)nt); }
  // (divided in 32 bits where that holds the operands, several times faster)
  static __device__ int64_t div(int64_t x, int64_t y) {
    return ((uint64_t)x | (uint64_t)y) >> 32 ? x / y : (int64_t)((uint32_t)x / (uint32_t)y);
  }
  __device__ int64_t begin(int c) const {
    return c >= G ? U : tiles ? div((int64_t)nt * c, G) * ct : div(U * c, G);
  }
  // the staying tile of unit u
  __device__ int64_t tile_of(int64_t u) const { return div(u, ct); }
  // staying and passing tile of the next unit of a run
  struct Walk {
    int t, j;
    bool starts, ends;  // the unit is the first (last) of its staying tile in this run
    int64_t left;
    int ct;
    __device__ Walk(const Units& u, int c) : ct((int)u.ct) {
      const int64_t u0 = u.begin(c);
      left = u.begin(c + 1) - u0;
      t = left > 0 ? (int)u.tile_of(u0) : 0;
      j = left > 0 ? (int)(u0 - (int64_t)t * u.ct) : 0;
      starts = true;
      ends = left == 1 || j + 1 == ct;
    }
    __device__ bool more() const { return left > 0; }
    __device__ void next() {
      --left;
      starts = ends;
      if (++j == ct) j = 0, ++t;
      ends = left == 1 || j + 1 == ct;
    }
  };
  // the last CTA with units before `end` (runs that share tiles)
  __device__ int last_before(int64_t end) const { return (int)div(end * G + U - 1, U) - 1; }
  // whether CTA c has all units of tile t
  __device__ bool whole(int c, int64_t t) const { return begin(c) <= t * ct && t * ct + ct <= begin(c + 1); }
  // which of its two partial results CTA c keeps of tile t, one it shares with others
  __device__ int slot(int c, int64_t t) const { return t == tile_of(begin(c)) ? 0 : 1; }
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// mbar_wait without a call, bounded as that is: a kernel that moves registers between warpgroups
// (setmaxnreg) cannot be allocated with a function call in it.
__device__ __forceinline__ bool mbar_wait_inline(uint64_t* bar, uint32_t parity, int* status, int site,
                                                 volatile int* abort, uint32_t backoff_ns = 0) {
  for (uint32_t i = 0; i < kSpinLimit; ++i) {
    if (mbar_try(bar, parity)) return true;
    if ((i & 1023u) == 1023u && *abort) return false;
    if (backoff_ns) __nanosleep(backoff_ns);
  }
  if (atomicCAS(status, 0, 1) == 0) atomicExch(status + 1, site);
  *abort = 1;
  return false;
}

// The same for whole warps, with a branch that is known to be the same for all lanes.
__device__ __forceinline__ bool mbar_wait_warp(uint64_t* bar, uint32_t parity, int* status, int site,
                                               volatile int* abort, uint32_t backoff_ns = 0) {
  for (uint32_t i = 0; i < kSpinLimit; ++i) {
    if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
    if ((i & 1023u) == 1023u && __any_sync(0xffffffffu, *abort)) return false;
    if (backoff_ns) __nanosleep(backoff_ns);
  }
  if (atomicCAS(status, 0, 1) == 0) atomicExch(status + 1, site);
  *abort = 1;
  return false;
}

// two fp32 at a time
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint64_t pack2u(uint32_t a, uint32_t b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t x, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

__device__ __forceinline__ uint32_t tmem_ld1(uint32_t taddr) {
  uint32_t r;
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr));
  return r;
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
// Fragments of 16 lanes: a thread has, of every 8 columns, columns 2 (l % 4) and + 1 in rows l / 4 and
// + 8 (.16x256b); stores of packed pairs: of every 4 columns, column l % 4 in those rows (.16x128b).
__device__ __forceinline__ void tmem_ld_frag32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_frag16(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
                 "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st_frag8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.16x128b.x2.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3])
               : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// Shared-memory descriptor of an MN-major operand with the 128-byte swizzle: rows of 64 elements along
// N, one row a K index, 8-row groups 1024 bytes apart (stride byte offset), the next 64 elements of
// N at `lbo` bytes (leading byte offset).
__device__ __forceinline__ uint64_t desc_sw128_mnmajor(uint32_t start, uint32_t lbo) {
  uint64_t d = 0;
  d |= (uint64_t)((start >> 4) & 0x3FFFu);
  d |= (uint64_t)((lbo >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// kind::f16 instruction descriptor, M = 128; b_mn: B is MN-major.
__device__ __forceinline__ uint32_t idesc16(int bf16, int N, int b_mn) {
  return (bf16 ? idesc_bf16_f32(128, N) : idesc_f16_f32(128, N)) | (uint32_t)b_mn << 16;
}

constexpr int kFwdThreads = 576;  // 16 epilogue warps, a TMA warp, an MMA warp
// The backward has 16 epilogue warps, a TMA warp, an MMA warp for each product and an idle warp, so that
// registers can move between whole warpgroups: of 640 x 96 at launch, 512 x 104 go to the epilogue (up to
// 64 gradient sums a thread) and 128 x 64 stay.
constexpr int kBwdThreads = 640;
constexpr int kMaxStages = 6;

// ------------------------------------------------------------------------------ forward
struct FwdArgs {
  int H, V;
  int direct;  // X is the caller's, all n rows of it
  int tiles;   // runs of whole tiles
  float c;     // bf16 form: log2 e / tau, what logits are multiplied by
  float tau2;  // soft targets: tau^2
  const float* inner;  // [n] soft targets: what loss / tau^2 - lse is; else NULL
  int64_t n, cap, vcap;
  const int* head;
  const int32_t* target;  // direct: the caller's
  const int32_t* row;
  const float* stat;
  float* hit;    // [cap] logit of the target
  float2* full;  // [4][cap] reference and sum of each quarter of the columns
  float2* part;  // [G][2][4][128] the same of tiles shared by CTAs
  float* loss;
  float* lse;
  int* status;
};

__device__ __forceinline__ int64_t fwd_rows(const FwdArgs& a) { return a.direct ? a.n : a.head[0]; }

// Target of slot s, -1 where there is none.
__device__ __forceinline__ int fwd_target(const FwdArgs& a, int64_t s) {
  if (!a.direct) return __float_as_int(a.stat[stat_at(s) + kTgt]);
  int t = s < a.n ? a.target[s] : -1;
  if (a.inner) return t < 0 ? -1 : kNoTarget;
  if (t >= a.V) {
    if (atomicCAS(a.status, 0, 2) == 0) atomicExch(a.status + 1, kSiteXentTarget);
    t = -1;
  }
  return t;
}

// lse and loss of slot s from the reference `top` (in units of kLog2e z) and the sum l to it.
__device__ __forceinline__ void fwd_finish(const FwdArgs& a, int64_t s, int tgt, float top, float l) {
  const int64_t i = a.direct ? s : a.row[s];
  if (i < 0 || i >= a.n) return;
  float v = 0.f, loss = 0.f;
  if (tgt != -1) {
    // (top + log2 l) / c with c = kLog2e as it was rounded, 1 / c in two parts, so that the only error
    // that counts is the result's own rounding
    constexpr float inv = (float)(1.0 / (double)kLog2e), rest = (float)(1.0 / (double)kLog2e - (double)inv);
    // (a sum of 0: the reference, rounded up, lies 2^7 or more above the largest logit, which it then
    // stands for to the last bit of fp32)
    const float log_l = l == 0.f ? 0.f : log2f(l);
    const float hi = top * inv, lo = fmaf(top, inv, -hi) + fmaf(top, rest, log_l * inv);
    v = hi + lo;
    loss = a.inner ? ((hi + a.inner[i]) + lo) * a.tau2 : (hi - a.hit[s]) + lo;
  }
  a.lse[i] = v;
  a.loss[i] = loss;
}

// z tiles of 128 rows x 256 columns.  X's tile stays in shared memory, W passes through a ring in
// pieces of 256 rows x 64 elements, two accumulators of 256 columns fill tensor memory.
template <int HC, int T>
struct FCfg {
  static constexpr int A_BYTES = T * HC * 16384;
  static constexpr int PIECE = 32768;
  static constexpr int ROOM = (232448 - 2048 - A_BYTES) / PIECE;
  static constexpr int ST = ROOM < 6 ? ROOM : 6;
  static constexpr int NP = T == 1 ? HC : 3 * HC;  // 64-element pieces of the product
  static constexpr int SMEM = A_BYTES + ST * PIECE + 2048;
  static_assert(ST >= 2 && SMEM <= 232448, "shared memory");
};

struct FwdBars {
  uint64_t a_full, a_empty, full[6], empty[6], s_full[2], s_empty[2], q_full[2], drain;
  uint32_t tmem;
  int abort;
};

// Sum of exp2(c z - m) over 32 columns.
__device__ __forceinline__ float sum32(const uint32_t* v, float c, float m) {
  const uint64_t c2 = pack2(c, c), m2 = pack2(-m, -m);
  uint64_t s[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 32; j += 4)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float a, b;
      unpack2(fma2(pack2u(v[j + 2 * k], v[j + 2 * k + 1]), c2, m2), a, b);
      s[k] = add2(s[k], pack2(ex2(a), ex2(b)));
    }
  float a, b;
  unpack2(add2(s[0], s[1]), a, b);
  return a + b;
}

// Largest of 32 columns.
__device__ __forceinline__ float max32(const uint32_t* v) {
  float top[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) top[k] = __uint_as_float(v[k]);
#pragma unroll
  for (int j = 4; j < 32; ++j) top[j & 3] = fmaxf(top[j & 3], __uint_as_float(v[j]));
  return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}

template <int HC, int T>
__global__ void __launch_bounds__(kFwdThreads, 1)
    k_xent_fwd(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW,
               const __grid_constant__ FwdArgs a) {
  using C = FCfg<HC, T>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  uint8_t* ring = smem + C::A_BYTES;
  FwdBars* bars = reinterpret_cast<FwdBars*>(ring + C::ST * C::PIECE);
  volatile int* abort = &bars->abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(&bars->a_full, 1);
    mbar_init(&bars->a_empty, 1);
    for (int s = 0; s < C::ST; ++s) {
      mbar_init(&bars->full[s], 1);
      mbar_init(&bars->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&bars->s_full[b], 1);
      mbar_init(&bars->s_empty[b], 16);
      mbar_init(&bars->q_full[b], 16);
    }
    mbar_init(&bars->drain, 1);
    bars->abort = 0;
    fence_mbar_init();
  }
  if (warp == 17) {
    tmem_alloc(&bars->tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_dep_launch();
  grid_dep_wait();
  const uint32_t tmem = bars->tmem;
  const Units un((fwd_rows(a) + 127) / 128, (a.V + 255) / 256, gridDim.x, a.tiles);
  Units::Walk w(un, blockIdx.x);

  if (warp == 16) {
    if (lane == 0) {
      tma_prefetch_desc(&tmX);
      tma_prefetch_desc(&tmW);
      uint32_t it = 0, seg = 0;
      bool ok = true;
      for (; w.more() && ok; w.next()) {
        if (w.starts) {
          ok = seg == 0 || mbar_wait(&bars->a_empty, (seg - 1) & 1, a.status, 701, abort, 32);
          if (!ok) break;
          mbar_expect_tx(&bars->a_full, C::A_BYTES);
          for (int p = 0; p < T * HC; ++p)
            tma_load_2d(smem + p * 16384, &tmX, &bars->a_full, p % HC * 64,
                        (int)((p / HC) * a.cap) + w.t * 128);
          ++seg;
        }
        for (int p = 0; p < C::NP && ok; ++p, ++it) {
          const int s = it % C::ST;
          ok = mbar_wait(&bars->empty[s], ((it / C::ST) & 1) ^ 1, a.status, 702, abort, 32);
          if (!ok) break;
          mbar_expect_tx(&bars->full[s], C::PIECE);
          tma_load_2d(ring + s * C::PIECE, &tmW, &bars->full[s], p % HC * 64,
                      (int)(T == 2 && p < HC ? a.vcap : 0) + w.j * 256);
        }
      }
      if (*abort) {  // copies in flight land before the block leaves
        for (uint32_t k = 0; seg && k < (1u << 22) && !mbar_try(&bars->a_full, (seg - 1) & 1); ++k) {
        }
        for (uint32_t q = it > C::ST ? it - C::ST : 0; q < it; ++q)
          for (uint32_t k = 0; k < (1u << 22) && !mbar_try(&bars->full[q % C::ST], (q / C::ST) & 1); ++k) {
          }
      }
    }
  } else if (warp == 17) {
    const bool leader = elect_one_sync();
    const uint32_t idesc = idesc16(T == 1, 256, 0);
    const uint64_t A = desc_sw128_kmajor(smem_u32(smem)), R = desc_sw128_kmajor(smem_u32(ring));
    uint32_t it = 0, seg = 0, n = 0;
    bool ok = true;
    for (; w.more() && ok; w.next(), ++n) {
      if (w.starts) {
        ok = mbar_wait(&bars->a_full, seg & 1, a.status, 703, abort);
        ++seg;
      }
      const int b = n & 1;
      ok = ok && mbar_wait(&bars->s_empty[b], ((n >> 1) & 1) ^ 1, a.status, 704, abort);
      for (int p = 0; p < C::NP && ok; ++p, ++it) {
        const int s = it % C::ST;
        ok = mbar_wait(&bars->full[s], (it / C::ST) & 1, a.status, 705, abort);
        if (!ok) break;
        tc_fence_after();
        // two terms: high x low, low x high, then high x high, so that the accumulator is small
        // (and loses little) in the first two thirds
        const int ab = T == 2 && p >= HC && p < 2 * HC ? p : p % HC;
        // past H the pieces hold zeros; a step is 32 bytes, 2 in a descriptor's units
        const uint64_t ad = A + ab * (16384 >> 4), bd = R + s * (C::PIECE >> 4);
        if (leader) {
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_ss(tmem + b * 256, ad + kk * 2, bd + kk * 2, idesc, p > 0 || kk > 0);
        }
        if (leader) tc_commit(&bars->empty[s]);
        __syncwarp();
      }
      if (ok && leader) {
        tc_commit(&bars->s_full[b]);
        if (w.ends) tc_commit(&bars->a_empty);
      }
      __syncwarp();
    }
    if (leader) tc_commit(&bars->drain);
    __syncwarp();
    for (uint32_t k = 0; k < (1u << 24) && !mbar_try(&bars->drain, 0); ++k) {
    }
  } else {
    // a thread is a row; each warpgroup has 64 columns of a tile
    const int q = warp & 3, wg = warp >> 2, r = q * 32 + lane;
    float ds = 1.f, c = a.c;  // z ds is the logit, z c the same in base 2 (over tau)
    const uint32_t base = tmem + ((uint32_t)(q * 32) << 16) + wg * 64;
    float m = -3.0e38f, l = 0.f;
    int tgt = -1;
    uint32_t n = 0, finished = 0;
    for (; w.more(); w.next(), ++n) {
      if (w.starts) {
        tgt = fwd_target(a, (int64_t)w.t * 128 + r);
        if (T == 2) {
          ds = a.stat[stat_at((int64_t)w.t * 128 + r) + kDs];
          c = kLog2e * ds;
        }
      }
      const int b = n & 1;
      const bool ok = mbar_wait(&bars->s_full[b], (n >> 1) & 1, a.status, 706, abort, 20);
      tc_fence_after();
      const int w0 = w.j * 256 + wg * 64, at = tgt - w0;
      const bool here = tgt >= 0 && at >= 0 && at < 64, check = w.starts || w0 + 64 > a.V;
      // the targets' logits, a column at a time (a warp leaves as a whole)
      unsigned hits = __ballot_sync(0xffffffffu, here || !ok);
      if (hits && __any_sync(0xffffffffu, !ok)) break;
      while (hits) {
        const int col = __shfl_sync(0xffffffffu, at, __ffs(hits) - 1);
        const float z = __uint_as_float(tmem_ld1(base + b * 256 + col));
        tmem_wait_ld();
        if (here && at == col) a.hit[w.t * 128 + r] = T == 2 ? z * ds : z;
        hits &= ~__ballot_sync(0xffffffffu, here && at == col);
      }
      // l = sum exp2(c z - m).  m need not be the running maximum, only near it: it is the maximum of
      // the row's first columns, and moves up when a sum passes 2^40 (so nothing overflows,
      // and what an early m made too large keeps all its bits).  This takes the maximum out of the
      // common path.  That path has one branch, the same for the whole warp, with all that is rare behind
      // it, and 32 columns at hand: with 64, and the targets found by comparing every column, 65537
      // rows x 49999 took 0.64 instead of 0.62 ms at H = 64, 0.68 instead of 0.61 at H = 128.
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t v[32];
        tmem_ld32(base + b * 256 + 32 * half, v);
        tmem_wait_ld();
        if (half) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars->s_empty[b]);
        }
        float sum = sum32(v, c, m);  // (of no use, and not used, where a tile starts)
        if (__any_sync(0xffffffffu, check || !(sum <= 0x1p40f))) {
          const bool start = w.starts && !half;
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (w0 + 32 * half + i >= a.V) v[i] = 0xFF800000u;
          if (start) {
            m = -3.0e38f;
            l = 0.f;
          }
          // (rounded up: of logits beyond 2^31, whose products with c are rounded by more than 2^7, the terms
          // may vanish but not overflow)
          const float top = start || !(sum <= 0x1p40f) ? fmaxf(m, __fmul_ru(max32(v), c)) : m;
          l *= ex2(m - top);
          m = top;
          sum = sum32(v, c, m);
        }
        l += sum;
      }
      if (w.ends) {
        // the sum's reference is m itself, so that fwd_finish undoes exactly what was done here
        const int64_t slot = (int64_t)w.t * 128 + r;
        if (un.whole(blockIdx.x, w.t)) {
          // The first warpgroup waits for all four quarters.  Tiles take turns at two barriers, and a warp
          // arrives for a tile only once all warps have for the one before: nothing else keeps the other
          // warpgroups, which do not wait here, from arriving for the next tile in a slow warp's place (a
          // tile may be a single unit, and the accumulator is free before its sum is done).
          auto quarters = [&](uint32_t tile) {
            return __all_sync(0xffffffffu, mbar_wait(&bars->q_full[tile & 1], (tile >> 1) & 1, a.status, 707, abort,
                                                     32));
          };
          if (finished > 0 && !quarters(finished - 1)) break;
          a.full[wg * a.cap + slot] = make_float2(m, l);
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars->q_full[finished & 1]);
          if (wg == 0) {
            if (!quarters(finished)) break;
            float2 p[4];
            for (int k = 0; k < 4; ++k) p[k] = a.full[k * a.cap + slot];
            const float top = fmaxf(fmaxf(p[0].x, p[1].x), fmaxf(p[2].x, p[3].x));
            float sum = 0.f;
            for (int k = 0; k < 4; ++k) sum += p[k].y * ex2(p[k].x - top);
            fwd_finish(a, slot, tgt, top, sum);
          }
          ++finished;
        } else {
          a.part[(((int64_t)blockIdx.x * 2 + un.slot(blockIdx.x, w.t)) * 4 + wg) * 128 + r] =
              make_float2(m, l);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 17) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Rows of the tiles that several CTAs have parts of.  Block c takes the tile that CTA c is the first to
// begin inside of, 8 of its rows a block; a row is 2 threads', or a warp's where it has parts of many CTAs.
__global__ void __launch_bounds__(256) k_xent_join(const __grid_constant__ FwdArgs a) {
  grid_dep_launch();
  grid_dep_wait();
  const int64_t rows = fwd_rows(a);
  const Units un((rows + 127) / 128, (a.V + 255) / 256, gridDim.x, a.tiles);
  const int c = blockIdx.x;
  if (c >= un.G || c == 0) return;
  const int64_t begin = un.begin(c), t = un.tile_of(begin), first = t * un.ct, end = first + un.ct;
  if (begin == first || un.begin(c - 1) > first) return;  // none, or an earlier CTA begins inside it too
  const int last = un.last_before(end);
  // CTA c - 1 has the first part (in its second place unless the tile is its first), the others begin
  // with this tile
  const float2* head = a.part + ((int64_t)(c - 1) * 2 + un.slot(c - 1, t)) * 512;
  const float2* tail = a.part + (int64_t)c * 1024;
  const int n = 4 * (last - c + 2), lanes = n > 16 ? 32 : 2;
  const int q = threadIdx.x / lanes;
  if (q < 8) {
    const int r = blockIdx.y * 8 + q;
    const int64_t s = t * 128 + r;
    if (s >= rows) return;  // (a whole group of lanes)
    float m = -3.0e38f, l = 0.f;
    for (int i = threadIdx.x % lanes; i < n; i += lanes) {
      const float2 p = i < 4 ? head[i * 128 + r] : tail[(int64_t)(i / 4 - 1) * 1024 + (i & 3) * 128 + r];
      const float mn = fmaxf(m, p.x);
      l = l * ex2(m - mn) + p.y * ex2(p.x - mn);
      m = mn;
    }
    const unsigned group = lanes == 32 ? 0xffffffffu : 3u << (threadIdx.x & 30);
    float top = m;
    for (int o = lanes / 2; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(group, top, o));
    l *= ex2(m - top);
    for (int o = lanes / 2; o; o >>= 1) l += __shfl_xor_sync(group, l, o);
    if (threadIdx.x % lanes == 0) {
      const int64_t i = a.direct ? s : 0;
      const int tgt = a.direct ? (a.target[i] < a.V ? a.target[i] : -1) : 0;
      fwd_finish(a, s, tgt, top, l);
    }
  }
}

// ------------------------------------------------------------------------------ backward
struct BwdArgs {
  int H, V, accumulate, out_bf16;
  int split;  // CTAs that compute dX; the others compute dW
  int tiles;  // runs of whole tiles
  int step;   // of the order of dW's tiles
  float l2e;  // bf16 form: log2 e / tau
  float tau;
  const float* add_x;  // bf16 gradients: added before they are rounded (or NULL)
  const float* add_w;
  int64_t cap, vcap;
  const int* head;
  const int32_t* row;
  const float* stat;
  const float* dloss;
  void* dX;
  void* dW;
  float* part;  // [G][2][128 x H], see part_at
  int* status;
};

// Place of columns c .. c + 3 (c a multiple of 4) of row r in a partial result: a warp, a lane a row,
// reads and writes 512 bytes in a row.
__device__ __forceinline__ int part_at(int r, int c) { return c * 128 + r * 4; }

// One unit: z = S B^T (S the staying tile, B the passing one), P from z, G += P B.  B serves both
// products: as its rows lie (K-major) in the first, transposed (MN-major) in the second.
//
// A passing tile has 128 rows, and 64 with two terms at H > 128, where 128 would not fit.  Tensor memory
// holds G and as many units' z as fit beside it.  The two products are issued by a warp each: with one
// warp, G of a unit that is ready would wait behind the next unit's z, and that for its load (measured
// at H = 256 with two ring stages: 3660 cycles a unit instead of the 2048 that the products take).
template <int HC, int FORM>
struct BCfg {
  static constexpr int T = FORM == kF16x2 ? 2 : 1;   // terms of S and B
  static constexpr int PT = FORM == kBf16 ? 1 : 2;   // terms of P
  static constexpr bool KEEP = FORM != kBf16;        // G is added up in registers
  static constexpr int NB = HC > 2 && T == 2 ? 64 : 128;  // passing rows of a unit
  static constexpr int CW = NB / 4;                  // columns of z of a thread
  // of which it works on so many at a time: fewer where it also holds up to 64 sums
  static constexpr int PW = KEEP && HC > 2 ? 16 : CW;
  // The epilogue keeps what targets cost in a path of its own (APART), and waits with a branch that is
  // known to be the same for the whole warp (UNIFORM).  us of dX and dW, without either -> with both: 65537 x
  // 49999 with fp32 gradients, H = 64 2700 -> 2605, H = 128 3320 -> 3270; fp32 inputs, 20000 x 32000 at
  // H = 128 1204 -> 1140; bf16 gradients, H = 256 3950 -> 3910.  With bf16 gradients the path apart takes
  // back at H = 64 what the branch gains (1690 -> 1550 with the branch alone, 1686 with both).  At H = 128,
  // where the two products take the tensor cores as long as each other and the epilogue is not what is
  // waited for, either costs (1970 -> 2120).  At H = 192 the branch gains (3120 -> 3000) and the path apart
  // makes no difference (fp32 forms: neither does).
  static constexpr bool APART = KEEP || HC > 2;
  static constexpr bool UNIFORM = KEEP || HC != 2;
  static constexpr int S_BYTES = T * HC * 16384;
  static constexpr int BOX = NB * 128;  // 64 elements of each passing row
  static constexpr int B_BYTES = T * HC * BOX;
  static constexpr int STATS = 4 * NB * 4;  // of passing X rows
  static constexpr int ROOM = (232448 - 2048 - S_BYTES) / (B_BYTES + 2048);
  static constexpr int ST = ROOM < kMaxStages ? ROOM : kMaxStages;
  static constexpr int SMEM = S_BYTES + ST * (B_BYTES + 2048) + 2048;
  static constexpr int GCOLS = HC * 64;
  static constexpr int ZROOM = (512 - GCOLS) / NB;
  static constexpr int ZB = ZROOM < 4 ? ZROOM : 4;   // units' z in tensor memory
  static constexpr int STEPS = NB / 16 * (T == 2 ? 3 : PT);  // accumulating steps of a unit
  static constexpr int DRAIN = (KEEP ? kDrainSteps : kLongSteps) / STEPS;  // units before G leaves TMEM
  static_assert(ST >= 1 && SMEM <= 232448, "shared memory");
  static_assert(ZB >= 2, "tensor memory");
  static_assert(DRAIN >= 1, "drain interval");
};

struct BwdBars {
  uint64_t s_full, s_empty, full[kMaxStages], empty[kMaxStages], z_full[4], z_empty[4], p_full[4], g_full, g_empty, drain_z, drain_g;
  uint32_t tmem;
  int abort;
};

// A place in a ring of N and the parity of its turn.
template <int N>
struct Turn {
  int i = 0;
  uint32_t parity = 0;
  __device__ __forceinline__ void next() {
    if (++i == N) i = 0, parity ^= 1;
  }
};

// Targets among a warp's values, and columns past the vocabulary, take extra work.  Whether there are any is
// asked within the one path (kEither), or first, for a path without (kUsual) and one with that work
// (kRare): see BCfg::APART.
enum { kEither, kUsual, kRare };

// Whether a passing row of X has its target among the 32 staying rows of W from `first`: the whole warp's
// answer from a row a lane.
__device__ __forceinline__ bool hit_row(const float* stat, int i, int first) {
  const int at = __float_as_int(stat[kTgt + i]) - first;
  return __any_sync(0xffffffffu, at >= 0 && at < 32);
}

// P of N columns of a row (a thread's) from their logits, for dX: descale and nlse = -lse of the row, hit =
// its target's place among the columns, of which the first `valid` exist.
template <int FORM, int N, int PATH>
__device__ __forceinline__ void probs_row(uint32_t* v, float log2e, float descale, float up, float nlse, int hit,
                                          int valid) {
  const uint64_t l2e = pack2(log2e, log2e), ds = pack2(descale, descale), up2 = pack2(up, up);
  const uint64_t nl = pack2(nlse, nlse);
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    uint64_t x = pack2u(v[i], v[i + 1]);
    x = FORM == kBf16 ? fma2(x, l2e, nl) : fma2(fma2(x, ds, nl), l2e, up2);
    float a, b;
    unpack2(x, a, b);
    v[i] = __float_as_uint(ex2(a));
    v[i + 1] = __float_as_uint(ex2(b));
  }
  if (PATH == kRare || (PATH == kEither && __any_sync(0xffffffffu, (hit >= 0 && hit < N) || valid < N))) {
    const float one = FORM == kBf16 ? 1.f : 32768.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i == hit) v[i] = __float_as_uint(__uint_as_float(v[i]) - one);
      if (i >= valid) v[i] = 0;
    }
  }
}

// The same for dW, whose statistics (scale, -lse, g, target of the passing X rows) go by column.  Were a
// thread a row here too, it would read every column's: at 32 columns a warp 16 shared-memory loads of
// 512 bytes, more than the SM can deliver in the time of the products (measured: 1.8 x the time of the
// dX kernel at H = 64).  So tensor memory is read in fragments in which a thread has two neighbouring
// columns of every 8, in rows l / 4, + 8, + 16, + 24 of its warp's 32 (l = lane): a quarter of the
// loads.  v[16 h + 4 g + 2 a + b]: row 16 h + 8 a + l / 4, column 8 g + 2 (l % 4) + b.
template <int FORM, int N, int PATH>
__device__ __forceinline__ void probs_col(uint32_t* v, float log2e, float up, const float* stat, int mine) {
  const uint64_t l2e = pack2(log2e, log2e), up2 = pack2(up, up);
  const int lane = threadIdx.x & 31, c = 2 * (lane & 3);
  const bool hits = PATH == kEither && hit_row(stat, lane & (N - 1), mine - lane / 4);
#pragma unroll
  for (int g = 0; g < N / 8; ++g) {
    const uint64_t nl = *reinterpret_cast<const uint64_t*>(stat + kNlse + 8 * g + c);
    const uint64_t g2 = *reinterpret_cast<const uint64_t*>(stat + kG + 8 * g + c);
    const uint64_t ds = FORM == kBf16 ? 0 : *reinterpret_cast<const uint64_t*>(stat + kDs + 8 * g + c);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t* p = v + (k >> 1) * (N / 2) + 4 * g + 2 * (k & 1);
      uint64_t x = pack2u(p[0], p[1]);
      x = FORM == kBf16 ? fma2(x, l2e, nl) : fma2(fma2(x, ds, nl), l2e, up2);
      float a, b;
      unpack2(x, a, b);
      unpack2(mul2(pack2(ex2(a), ex2(b)), g2), a, b);
      p[0] = __float_as_uint(a);
      p[1] = __float_as_uint(b);
    }
  }
  if (PATH == kRare || (PATH == kEither && hits)) {
    // all columns, without branches (skipping groups of 8 without a hit took longer)
    const float upg = FORM == kBf16 ? -1.f : -ex2(up);
#pragma unroll
    for (int g = 0; g < N / 8; ++g) {
      const int2 tt = *reinterpret_cast<const int2*>(stat + kTgt + 8 * g + c);
      const float2 gg = *reinterpret_cast<const float2*>(stat + kG + 8 * g + c);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t* p = v + (k >> 1) * (N / 2) + 4 * g + 2 * (k & 1);
        const int row = mine + 16 * (k >> 1) + 8 * (k & 1);
        if (tt.x == row) p[0] = __float_as_uint(fmaf(gg.x, upg, __uint_as_float(p[0])));
        if (tt.y == row) p[1] = __float_as_uint(fmaf(gg.y, upg, __uint_as_float(p[1])));
      }
    }
  }
}

// Two neighbouring values of P as the form's terms.
template <int FORM>
__device__ __forceinline__ void terms(uint32_t a, uint32_t b, uint32_t& hi, uint32_t& lo) {
  const float x = __uint_as_float(a), y = __uint_as_float(b);
  if (FORM == kBf16) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(x, y);
    hi = *reinterpret_cast<const uint32_t*>(&p);
  } else {
    // the high term by cutting the mantissa to fp16's 11 bits, so that the rest is exact and nothing has to
    // be converted back
    const uint32_t hx = a & 0xFFFFE000u, hy = b & 0xFFFFE000u;
    const __half2 p = __floats2half2_rn(__uint_as_float(hx), __uint_as_float(hy));
    hi = *reinterpret_cast<const uint32_t*>(&p);
    const __half2 l = __floats2half2_rn(x - __uint_as_float(hx), y - __uint_as_float(hy));
    lo = *reinterpret_cast<const uint32_t*>(&l);
  }
}

// A warp's part of a unit: P over z in tensor memory (columns from `at`).
template <int HC, int FORM, bool DW, int PATH>
__device__ __forceinline__ void z_to_p(uint32_t at, float log2e, float descale, float up, const float* stat, int mine,
                                       float nlse, int hit, int valid) {
  using C = BCfg<HC, FORM>;
  constexpr int N = PATH == kRare ? 16 : C::PW;  // (short: its time matters little)
#pragma unroll(PATH == kRare ? 1 : 16)
  for (int pc = 0; pc < C::CW; pc += N) {
    uint32_t v[N];
    if (DW) {
      // (N / 2 registers for each half of the warp's rows)
      if (N == 32) {
        tmem_ld_frag32(at + pc, v);
        tmem_ld_frag32(at + pc + (16u << 16), v + 16);
      } else {
        tmem_ld_frag16(at + pc, v);
        tmem_ld_frag16(at + pc + (16u << 16), v + 8);
      }
      tmem_wait_ld();
      probs_col<FORM, N, PATH>(v, log2e, up, stat + pc, mine);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < N; c += 16) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t* p = v + h * (N / 2) + c / 2 + 2 * i;
            terms<FORM>(p[0], p[1], hi[i], lo[i]);
          }
          tmem_st_frag8(at + pc + (h * 16u << 16) + c, hi);
          if (FORM != kBf16) tmem_st_frag8(at + pc + (h * 16u << 16) + c + 8, lo);
        }
    } else {
      if (N == 32)
        tmem_ld32(at + pc, v);
      else
        tmem_ld16(at + pc, v);
      tmem_wait_ld();
      probs_row<FORM, N, PATH>(v, log2e, descale, up, nlse, hit - pc, valid - pc);
#pragma unroll
      for (int c = 0; c < N; c += 16) {
        uint32_t hi[8], lo[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) terms<FORM>(v[c + 2 * i], v[c + 2 * i + 1], hi[i], lo[i]);
        tmem_st8(at + pc + c, hi);
        if (FORM != kBf16) tmem_st8(at + pc + c + 8, lo);
      }
    }
  }
}

// v += the 16 columns of a row of a partial result that begin at p.
__device__ __forceinline__ void add16(const float* p, uint32_t* v) {
#pragma unroll
  for (int i = 0; i < 16; i += 4) {
    const float4 x = *reinterpret_cast<const float4*>(p + part_at(0, i));
    v[i] = __float_as_uint(__uint_as_float(v[i]) + x.x);
    v[i + 1] = __float_as_uint(__uint_as_float(v[i + 1]) + x.y);
    v[i + 2] = __float_as_uint(__uint_as_float(v[i + 2]) + x.z);
    v[i + 3] = __float_as_uint(__uint_as_float(v[i + 3]) + x.w);
  }
}

// The epilogue warps of k_xent_bwd: P from z, and G to its destination.
template <int HC, int FORM, bool DW>
__device__ __forceinline__ void bwd_epilogue(const BwdArgs& a, const Units& un, int cta, uint32_t tmem,
                                             const uint8_t* stats, BwdBars* bars) {
  using C = BCfg<HC, FORM>;
  volatile int* abort = &bars->abort;
  const uint32_t zbuf = tmem + C::GCOLS;
  Units::Walk w(un, cta);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // a thread is a row; its warpgroup has CW columns of each unit and GQ columns of G
  const int q = warp & 3, wg = warp >> 2, r = q * 32 + lane;
  constexpr int GQ = HC * 16;
  const int c0 = wg * C::CW;
  const uint32_t quarter = (uint32_t)(q * 32) << 16;
  // P is scaled by 2^up: probabilities to 2^15 for dX, times the weights to 2^15 for dW
  const int up = FORM == kBf16 ? 0 : DW ? a.head[2] : 15;
  float acc[C::KEEP ? GQ : 1];
  uint32_t groups = 0;
  int in_group = 0;
  Turn<C::ST> s;
  Turn<C::ZB> b;
  bool fresh = true, pending = false, spilled = false, ok = true;
  float nlse = 0.f, descale = 1.f;
  int tgt = -1, first = 0;
  auto wait = [&](uint64_t* bar, uint32_t parity, int site, uint32_t backoff_ns) {
    return C::UNIFORM ? mbar_wait_warp(bar, parity, a.status, site, abort, backoff_ns)
                      : __all_sync(0xffffffffu, mbar_wait_inline(bar, parity, a.status, site, abort, backoff_ns)) != 0;
  };
  // takes the finished group of G: adds it to the registers
  auto collect = [&]() {
    if (!wait(&bars->g_full, groups & 1, 717, 32)) return false;
    ++groups;
    tc_fence_after();
    if (C::KEEP) {
#pragma unroll
      for (int c = 0; c < GQ; c += 16) {
        uint32_t v[16];
        tmem_ld16(tmem + quarter + wg * GQ + c, v);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 16; ++i)
          acc[C::KEEP ? c + i : 0] = fresh ? __uint_as_float(v[i])
                                           : acc[C::KEEP ? c + i : 0] + __uint_as_float(v[i]);
      }
      fresh = false;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->g_empty);
    }
    return true;
  };
  for (; w.more() && ok; w.next(), s.next(), b.next()) {
    if (DW && w.starts) first = un.tile(w.t) * 128;
    if (!DW && w.starts) {
      const float* st = a.stat + stat_at(w.t * 128 + r);
      nlse = st[kNlse];
      tgt = __float_as_int(st[kTgt]);
      if (FORM != kBf16) descale = st[kDs];
    }
    ok = wait(&bars->z_full[b.i], b.parity, 718, 20);
    if (!ok) break;
    tc_fence_after();
    const uint32_t at = zbuf + quarter + b.i * C::NB + c0;
    const float* st = reinterpret_cast<const float*>(stats + s.i * 2048) + stat_at(c0);
    const int w0 = w.j * C::NB + c0, hit = tgt < 0 ? -1 : tgt - w0, mine = first + q * 32 + lane / 4;
    bool rare = true;
    if (C::APART)
      rare = DW ? hit_row(st, lane & (C::CW - 1), first + q * 32)
                : __any_sync(0xffffffffu, (hit >= 0 && hit < C::CW) || w0 + C::CW > a.V);
    if (rare)
      z_to_p<HC, FORM, DW, C::APART ? kRare : kEither>(at, FORM == kBf16 ? a.l2e : kLog2e, descale, (float)up, st, mine, nlse, hit, a.V - w0);
    else
      z_to_p<HC, FORM, DW, kUsual>(at, FORM == kBf16 ? a.l2e : kLog2e, descale, (float)up, st, mine, nlse, hit, a.V - w0);
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(&bars->p_full[b.i]);
    if (pending) {
      ok = collect();
      pending = false;
      if (!ok) break;
    }
    const bool close = ++in_group == C::DRAIN || w.ends;
    if (close) {
      in_group = 0;
      pending = C::KEEP && !w.ends;
    }
    if (!(C::KEEP ? w.ends : close)) continue;
    ok = collect();
    if (!ok) break;
    fresh = true;
    // the tile's result: finished where this CTA had all its units, else for the join; of a long sum, what
    // there is of it so far goes to the same place as what is left to the join, and is added there
    const bool whole = w.ends && un.whole(cta, w.t);
    int64_t orow = (DW ? first : w.t * 128) + r;
    float s1 = 1.f, s2 = 1.f, s3 = 1.f;
    if (DW) {
      if (orow >= a.V) orow = -1;
      if (FORM != kBf16) s1 = pow2(-up), s2 = pow2(-14);  // (X's elements are times 2^14, once 2^e is undone)
    } else {
      orow = a.row[orow];
      s3 = orow < 0 ? 0.f : a.dloss[orow] * a.tau;
      if (FORM != kBf16) s1 = pow2(-15), s2 = pow2(-a.head[1]);
    }
    float* pt = a.part + ((int64_t)blockIdx.x * 2 + un.slot(cta, w.t)) * 128 * a.H;
#pragma unroll(C::KEEP ? 4 : 1)
    for (int c = 0; c < GQ; c += 16) {
      const int col = wg * GQ + c;
      uint32_t v[16];
      if (C::KEEP) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(acc[C::KEEP ? c + i : 0]);
      } else if (col < a.H) {
        tmem_ld16(tmem + quarter + col, v);
        tmem_wait_ld();
        if (spilled) add16(pt + part_at(r, col), v);
      }
      if (col >= a.H) continue;
      float* x = reinterpret_cast<float*>(v);
      if (!whole) {
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<float4*>(pt + part_at(r, col + i)) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
        continue;
      }
      if (orow < 0) continue;
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = x[i] * s1 * s2 * s3;
      if (a.out_bf16) {
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(DW ? a.dW : a.dX) + orow * a.H + col;
        const float* add = DW ? a.add_w : a.add_x;
        if (add) {
          add += orow * a.H + col;
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const float4 p = *reinterpret_cast<const float4*>(add + i);
            x[i] += p.x;
            x[i + 1] += p.y;
            x[i + 2] += p.z;
            x[i + 3] += p.w;
          }
        }
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
          __nv_bfloat162 h[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) h[k] = __floats2bfloat162_rn(x[i + 2 * k], x[i + 2 * k + 1]);
          *reinterpret_cast<uint4*>(o + i) = *reinterpret_cast<const uint4*>(h);
        }
      } else {
        float* o = static_cast<float*>(DW ? a.dW : a.dX) + orow * a.H + col;
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          float4 h = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
          if (a.accumulate) {
            const float4 p = *reinterpret_cast<const float4*>(o + i);
            h = make_float4(h.x + p.x, h.y + p.y, h.z + p.z, h.w + p.w);
          }
          *reinterpret_cast<float4*>(o + i) = h;
        }
      }
    }
    if (!C::KEEP) {
      spilled = !w.ends;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->g_empty);
    }
  }
}

// The first a.split CTAs compute dX (X stays), the others dW (W stays): the two have as many units.
template <int HC, int FORM>
__global__ void __launch_bounds__(kBwdThreads, 1)
    k_xent_bwd(const __grid_constant__ CUtensorMap tmXs, const __grid_constant__ CUtensorMap tmXp,
               const __grid_constant__ CUtensorMap tmWs, const __grid_constant__ CUtensorMap tmWp,
               const __grid_constant__ BwdArgs a) {
  using C = BCfg<HC, FORM>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~uintptr_t(1023));
  uint8_t* ring = smem + C::S_BYTES;
  uint8_t* stats = ring + C::ST * C::B_BYTES;  // 2048 bytes a stage
  BwdBars* bars = reinterpret_cast<BwdBars*>(stats + C::ST * 2048);
  volatile int* abort = &bars->abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(&bars->s_full, 1);
    mbar_init(&bars->s_empty, 1);
    for (int s = 0; s < C::ST; ++s) {
      mbar_init(&bars->full[s], 1);
      mbar_init(&bars->empty[s], 1);
    }
    for (int b = 0; b < C::ZB; ++b) {
      mbar_init(&bars->z_full[b], 1);
      mbar_init(&bars->z_empty[b], 1);
      mbar_init(&bars->p_full[b], 16);
    }
    mbar_init(&bars->g_full, 1);
    mbar_init(&bars->g_empty, 16);
    mbar_init(&bars->drain_z, 1);
    mbar_init(&bars->drain_g, 1);
    bars->abort = 0;
    fence_mbar_init();
  }
  if (warp == 17) {
    tmem_alloc(&bars->tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_dep_launch();
  grid_dep_wait();
  const uint32_t tmem = bars->tmem, zbuf = tmem + C::GCOLS;
  const int64_t rows = a.head[0];
  const bool dw = (int)blockIdx.x >= a.split;
  const int cta = blockIdx.x - (dw ? a.split : 0);
  const Units un(dw ? (a.V + 127) / 128 : (rows + 127) / 128,
                 dw ? (rows + C::NB - 1) / C::NB : (a.V + C::NB - 1) / C::NB,
                 dw ? gridDim.x - a.split : a.split, a.tiles, dw ? a.step : 1);

  if (warp == 16) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (lane == 0) {
      Units::Walk w(un, cta);
      const CUtensorMap* tmS = dw ? &tmWs : &tmXs;
      const CUtensorMap* tmB = dw ? &tmXp : &tmWp;
      const int splane = (int)(dw ? a.vcap : a.cap), pplane = (int)(dw ? a.cap : a.vcap);
      tma_prefetch_desc(tmS);
      tma_prefetch_desc(tmB);
      uint32_t it = 0, seg = 0;
      Turn<C::ST> s;
      bool ok = true;
      for (; w.more() && ok; w.next(), s.next(), ++it) {
        if (w.starts) {
          ok = seg == 0 || mbar_wait_inline(&bars->s_empty, (seg - 1) & 1, a.status, 711, abort, 32);
          if (!ok) break;
          mbar_expect_tx(&bars->s_full, C::S_BYTES);
          for (int p = 0; p < C::T * HC; ++p)
            tma_load_2d(smem + p * 16384, tmS, &bars->s_full, p % HC * 64,
                        p / HC * splane + un.tile(w.t) * 128);
          ++seg;
        }
        ok = mbar_wait_inline(&bars->empty[s.i], s.parity ^ 1, a.status, 712, abort, 32);
        if (!ok) break;
        mbar_expect_tx(&bars->full[s.i], C::B_BYTES + (dw ? C::STATS : 0));
        for (int p = 0; p < C::T * HC; ++p)
          tma_load_2d(ring + s.i * C::B_BYTES + p * C::BOX, tmB, &bars->full[s.i], p % HC * 64,
                      p / HC * pplane + w.j * C::NB);
        if (dw) {
          uint8_t* d = stats + s.i * 2048;
          const int64_t at = (int64_t)w.j * C::NB;
          bulk_load(d, a.stat + stat_at(at), C::STATS, &bars->full[s.i]);
        }
      }
      if (*abort) {  // copies in flight land before the block leaves
        for (uint32_t k = 0; seg && k < (1u << 22) && !mbar_try(&bars->s_full, (seg - 1) & 1); ++k) {
        }
        for (uint32_t q = it > C::ST ? it - C::ST : 0; q < it; ++q)
          for (uint32_t k = 0; k < (1u << 22) && !mbar_try(&bars->full[q % C::ST], (q / C::ST) & 1); ++k) {
          }
      }
    }
  } else if (warp == 17) {
    // z = S B^T, as many units ahead as tensor memory and the ring hold
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    Units::Walk w(un, cta);
    const bool leader = elect_one_sync();
    const uint32_t iz = idesc16(FORM == kBf16, C::NB, 0);
    // a descriptor's address field is in 16 bytes
    const uint64_t S = desc_sw128_kmajor(smem_u32(smem)), R = desc_sw128_kmajor(smem_u32(ring));
    uint32_t seg = 0;
    Turn<C::ST> s;
    Turn<C::ZB> b;
    bool ok = true;
    for (; w.more() && ok; w.next(), s.next(), b.next()) {
      if (w.starts) {
        ok = mbar_wait_inline(&bars->s_full, seg & 1, a.status, 715, abort);
        ++seg;
      }
      ok = ok && mbar_wait_inline(&bars->z_empty[b.i], b.parity ^ 1, a.status, 719, abort);
      ok = ok && mbar_wait_inline(&bars->full[s.i], s.parity, a.status, 716, abort);
      tc_fence_after();
      const uint64_t B = R + s.i * (C::B_BYTES >> 4);
      const uint32_t d = zbuf + b.i * C::NB;
      // past H both operands hold zeros; two terms: low x high and high x low first, while the
      // accumulator is small
      constexpr int n = C::T == 2 ? 3 : 1;
      if (leader && ok) {
#pragma unroll
        for (int pr = 0; pr < n; ++pr) {
          const uint64_t as = S + (n == 3 && pr == 0 ? HC * (16384 >> 4) : 0);
          const uint64_t bs = B + (n == 3 && pr == 1 ? HC * (C::BOX >> 4) : 0);
#pragma unroll
          for (int k = 0; k < HC * 4; ++k)
            mma_ss(d, as + (k >> 2) * (16384 >> 4) + (k & 3) * 2,
                   bs + (k >> 2) * (C::BOX >> 4) + (k & 3) * 2, iz, pr > 0 || k > 0);
        }
        tc_commit(&bars->z_full[b.i]);
        if (w.ends) tc_commit(&bars->s_empty);
      }
      ok = __all_sync(0xffffffffu, ok);  // (as a whole)
    }
    if (leader) tc_commit(&bars->drain_z);
    __syncwarp();
    for (uint32_t k = 0; k < (1u << 24) && !mbar_try(&bars->drain_z, 0); ++k) {
    }
  } else if (warp == 18) {
    // G (+)= P B, small products first
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    Units::Walk w(un, cta);
    const bool leader = elect_one_sync();
    const uint32_t ig = idesc16(FORM == kBf16, a.H, 1);
    const uint64_t R = desc_sw128_mnmajor(smem_u32(ring), C::BOX);
    uint32_t groups = 0;
    int in_group = 0;
    Turn<C::ST> s;
    Turn<C::ZB> b;
    bool ok = true;
    for (; w.more() && ok; w.next(), s.next(), b.next()) {
      ok = mbar_wait_inline(&bars->p_full[b.i], b.parity, a.status, 713, abort);
      if (ok && in_group == 0 && groups > 0)
        ok = mbar_wait_inline(&bars->g_empty, (groups - 1) & 1, a.status, 714, abort);
      tc_fence_after();
      const uint64_t B = R + s.i * (C::B_BYTES >> 4);
      const uint32_t p = zbuf + b.i * C::NB;
      constexpr int n = C::T == 2 ? 3 : C::PT;
      const bool close = ++in_group == C::DRAIN || w.ends;
      if (leader && ok) {
#pragma unroll
        for (int pr = 0; pr < n; ++pr) {
          // 16 columns of z hold 16 of P: 8 columns of the high terms, 8 of the low ones
          const uint32_t pa = p + (C::PT == 2 && pr == 0 ? 8 : 0);
          const uint64_t bs = B + (n == 3 && pr == 1 ? HC * (C::BOX >> 4) : 0);
#pragma unroll
          for (int k = 0; k < C::NB / 16; ++k)
            mma_ts(tmem, pa + k * 16, bs + k * (2048 >> 4), ig,
                   in_group > 1 || pr > 0 || k > 0);
        }
        tc_commit(&bars->empty[s.i]);
        tc_commit(&bars->z_empty[b.i]);
        if (close) tc_commit(&bars->g_full);
      }
      if (close) {
        ++groups;
        in_group = 0;
      }
      ok = __all_sync(0xffffffffu, ok);  // (as a whole)
    }
    if (leader) tc_commit(&bars->drain_g);
    __syncwarp();
    for (uint32_t k = 0; k < (1u << 24) && !mbar_try(&bars->drain_g, 0); ++k) {
    }
  } else if (warp > 18) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    if (dw && un.ct == 0 && !a.accumulate) {  // no labelled rows
      const int64_t n16 = (int64_t)a.V * a.H / (a.out_bf16 ? 8 : 4), ctas = gridDim.x - a.split;
      for (int64_t i = (int64_t)cta * 512 + threadIdx.x; i < n16; i += ctas * 512)
        static_cast<uint4*>(a.dW)[i] = make_uint4(0, 0, 0, 0);
    }
    if (dw)
      bwd_epilogue<HC, FORM, true>(a, un, cta, tmem, stats, bars);
    else
      bwd_epilogue<HC, FORM, false>(a, un, cta, tmem, stats, bars);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 17) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Tiles that several CTAs have parts of: the sum of the parts in the order of the CTAs.  Block row c
// takes the tile that CTA c is the first to begin inside of, 32 rows x 32 columns a block (with a
// whole tile's rows a block, tiles of many parts took twice as long).
__global__ void __launch_bounds__(256)
    k_xent_bwd_join(const __grid_constant__ BwdArgs a, int form, int nb) {
  grid_dep_launch();
  grid_dep_wait();
  const int64_t rows = a.head[0];
  const bool dw = (int)blockIdx.x >= a.split;
  const int c = blockIdx.x - (dw ? a.split : 0), ctas = dw ? gridDim.x - a.split : a.split;
  const Units un(dw ? (a.V + 127) / 128 : (rows + 127) / 128,
                 dw ? (rows + nb - 1) / nb : (a.V + nb - 1) / nb, ctas, a.tiles, dw ? a.step : 1);
  void* out = dw ? a.dW : a.dX;
  if (c >= un.G || c == 0) return;
  const int64_t begin = un.begin(c), t = un.tile_of(begin), first = t * un.ct, end = first + un.ct;
  if (begin == first) return;
  const int64_t prev = un.begin(c - 1);
  if (prev > first) return;  // an earlier CTA begins inside the tile too
  const int hb = a.H / 32, col = (int)(blockIdx.y % hb) * 32 + (threadIdx.x >> 5) * 4;
  const int r = (int)(blockIdx.y / hb) * 32 + (threadIdx.x & 31);
  // CTA c - 1 has the first part (in its second place unless the tile is its first), the others begin
  // with this tile
  const int64_t stride = 128LL * a.H;
  const float* part = a.part + (int64_t)(blockIdx.x - c) * 2 * stride + part_at(r, col);
  const float* head = part + ((int64_t)(c - 1) * 2 + (un.tile_of(prev) == t ? 0 : 1)) * stride;
  float4 x = *reinterpret_cast<const float4*>(head);
  const int last = un.last_before(end);
#pragma unroll 8
  for (int k = c; k <= last; ++k) {
    const float4 p = *reinterpret_cast<const float4*>(part + (int64_t)k * 2 * stride);
    x = make_float4(x.x + p.x, x.y + p.y, x.z + p.z, x.w + p.w);
  }
  float s1 = 1.f, s2 = 1.f;
  if (form != kBf16) {
    s1 = pow2(dw ? -a.head[2] : -15);
    s2 = pow2(dw ? -14 : -a.head[1]);
  }
  int64_t orow = (int64_t)un.tile((int)t) * 128 + r;
  float s3 = 1.f;
  if (dw) {
    if (orow >= a.V) return;
  } else {
    orow = a.row[orow];
    if (orow < 0) return;
    s3 = a.dloss[orow] * a.tau;
  }
  x = make_float4(x.x * s1 * s2 * s3, x.y * s1 * s2 * s3, x.z * s1 * s2 * s3, x.w * s1 * s2 * s3);
  if (a.out_bf16) {
    if (const float* add = dw ? a.add_w : a.add_x) {
      const float4 p = *reinterpret_cast<const float4*>(add + orow * a.H + col);
      x = make_float4(x.x + p.x, x.y + p.y, x.z + p.z, x.w + p.w);
    }
    __nv_bfloat162 w[2] = {__floats2bfloat162_rn(x.x, x.y), __floats2bfloat162_rn(x.z, x.w)};
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(out) + orow * a.H + col) =
        *reinterpret_cast<const uint2*>(w);
  } else {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(out) + orow * a.H + col);
    if (a.accumulate) {
      const float4 p = *o;
      x = make_float4(x.x + p.x, x.y + p.y, x.z + p.z, x.w + p.w);
    }
    *o = x;
  }
}

// ------------------------------------------------------------------------------ host
struct Call {
  int form, H, V, ctas;
  int64_t n;
  Ws w;
  char* base;
  cudaStream_t st;
  template <typename P>
  P* at(size_t off) const { return reinterpret_cast<P*>(base + off); }
};

// Count, gather and convert: fills everything the tile kernels read.
cudaError_t prepare(const XentArgs& a, Call& c, RowArgs r) {
  r.form = c.form;
  r.x_bf16 = a.bf16;
  r.n = a.n;
  r.rb = c.w.rb;
  r.nb = c.w.nb;
  r.cap = c.w.cap;
  r.vcap = c.w.vcap;
  r.H = a.H;
  r.V = a.V;
  r.X = a.X;
  r.W = a.W;
  r.target = a.target;
  r.head = c.at<int>(c.w.head);
  r.counts = c.at<int>(c.w.counts);
  r.amax = c.at<uint32_t>(c.w.amax);
  r.xexp = c.at<int8_t>(c.w.xexp);
  r.row = c.at<int32_t>(c.w.row);
  r.stat = c.at<float>(c.w.stat);
  r.x = c.at<uint16_t>(c.w.x);
  r.w = c.at<uint16_t>(c.w.w);
  r.status = a.status;
  r.soft = a.soft != nullptr;
  r.tau = a.soft ? a.soft->tau : 1.f;
  r.inv_tau = 1.f / r.tau;
  // Up to kDirectRows rows, each block of k_xent_rows counts the rows before its own (at most 128 KB of
  // targets, from L2) in less time than a launch takes; the fp16 forms need the magnitudes first anyway.
  r.direct = c.form == kBf16 && a.n <= kDirectRows;
  // of the table, 256 times 8 elements a block and pass
  r.tb = c.form == kBf16 ? 0
                         : (int)std::min<int64_t>(kTableBlocks, ((int64_t)a.V * (a.H / 8) + 255) / 256);
  cudaError_t e;
  if (!r.direct) {
    e = launch_pdl(k_xent_count, dim3((unsigned)c.w.nb + r.tb), dim3(256), 0, c.st, r);
    if (e != cudaSuccess) return e;
    note_launch();
  }
  e = launch_pdl(k_xent_rows, dim3((unsigned)c.w.nb + r.tb), dim3(256), 0, c.st, r);
  if (e != cudaSuccess) return e;
  note_launch();
  return cudaSuccess;
}

// Tensor maps over the gathered rows of X and over W (as it is, or its converted planes).
bool map_x(const Call& c, CUtensorMap* m, int box) {
  const int64_t rows = (c.form == kF16x2 ? 2 : 1) * c.w.cap;
  return make_map_ld(m, c.base + c.w.x, rows, c.H, c.H, box);
}
bool map_w(const Call& c, const void* W, CUtensorMap* m, int box) {
  if (c.form == kBf16) return make_map_ld(m, W, c.V, c.H, c.H, box);
  return make_map_ld(m, c.base + c.w.w, (c.form == kF16x2 ? 2 : 1) * c.w.vcap, c.H, c.H, box);
}

template <int HC, int T>
cudaError_t run_fwd(const Call& c, const XentArgs& x, const FwdArgs& f) {
  using C = FCfg<HC, T>;
  CUtensorMap mx, mw;
  if (!(f.direct ? make_map_ld(&mx, x.X, c.n, c.H, c.H, 128) : map_x(c, &mx, 128)) ||
      !map_w(c, x.W, &mw, 256))
    return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  cudaError_t e = allow_smem(k_xent_fwd<HC, T>, C::SMEM, done);
  if (e != cudaSuccess) return e;
  return launch_pdl(k_xent_fwd<HC, T>, dim3(c.ctas), dim3(kFwdThreads), C::SMEM, c.st, mx, mw, f);
}

template <int HC, int FORM>
cudaError_t run_bwd(const Call& c, const void* W, const BwdArgs& b) {
  using C = BCfg<HC, FORM>;
  CUtensorMap xs, xp, ws, wp;
  if (!map_x(c, &xs, 128) || !map_w(c, W, &ws, 128)) return cudaErrorInvalidValue;
  xp = xs;
  wp = ws;
  if (C::NB != 128 && (!map_x(c, &xp, C::NB) || !map_w(c, W, &wp, C::NB))) return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  cudaError_t e = allow_smem(k_xent_bwd<HC, FORM>, C::SMEM, done);
  if (e != cudaSuccess) return e;
  e = launch_pdl(k_xent_bwd<HC, FORM>, dim3(c.ctas), dim3(kBwdThreads), C::SMEM, c.st, xs, xp, ws, wp,
                 b);
  if (e != cudaSuccess) return e;
  note_launch();
  if (b.tiles) return cudaSuccess;
  e = launch_pdl(k_xent_bwd_join, dim3(c.ctas, c.H / 32 * 4), dim3(256), 0, c.st, b, FORM, C::NB);
  if (e != cudaSuccess) return e;
  note_launch();
  return cudaSuccess;
}

template <int FORM>
cudaError_t run_bwd_h(const Call& c, const void* W, const BwdArgs& b) {
  switch ((c.H + 63) / 64) {
    case 1: return run_bwd<1, FORM>(c, W, b);
    case 2: return run_bwd<2, FORM>(c, W, b);
    case 3: return run_bwd<3, FORM>(c, W, b);
    default: return run_bwd<4, FORM>(c, W, b);
  }
}

int form_of(int bf16, int backward, int grad_bf16) {
  return !bf16 ? kF16x2 : backward && !grad_bf16 ? kF16x1 : kBf16;
}

// SMs of the current device (asked once a device; the calls may come from several threads).
cudaError_t device_sms(int* sms) {
  static std::atomic<int> known[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  *sms = dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0;
  if (*sms > 0) return cudaSuccess;
  e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess && dev < 64) known[dev].store(*sms, std::memory_order_relaxed);
  return e;
}

cudaError_t make_call(const XentArgs& a, int form, int backward, cudaStream_t st, Call* call) {
  Call& c = *call;
  int sms = 0;
  const cudaError_t e = device_sms(&sms);
  if (e != cudaSuccess) return e;
  c.form = form;
  c.H = a.H;
  c.V = a.V;
  c.n = a.n;
  c.ctas = xent_ctas(sms);
  c.w = layout(form, a.n, a.H, a.V, backward, c.ctas);
  c.base = static_cast<char*>(a.ws);
  c.st = st;
  return cudaSuccess;
}

}  // namespace

// At least 2: a backward call that computes dX and dW has CTAs for each (none waits for another, so that
// they need not run at the same time).
int xent_ctas(int sms) { return std::max(2, std::min(sms, kMaxCtas)); }

size_t xent_ws_bytes(int bf16, int64_t n, int H, int V, int backward) {
  return layout(form_of(bf16, backward, 0), n, H, V, backward, kMaxCtas).total;
}

size_t xent_ws_used(int bf16, int64_t n, int H, int V, int backward, int grad_bf16, int sms) {
  return layout(form_of(bf16, backward, grad_bf16), n, H, V, backward, xent_ctas(sms)).total;
}

cudaError_t xent_fwd(const XentArgs& a, float* loss, float* lse, cudaStream_t st) {
  if (a.n == 0) return cudaSuccess;
  Call c;
  cudaError_t e = make_call(a, form_of(a.bf16, 0, 0), 0, st, &c);
  if (e != cudaSuccess) return e;
  FwdArgs f{};
  f.H = a.H;
  f.V = a.V;
  f.n = a.n;
  f.cap = c.w.cap;
  f.vcap = c.w.vcap;
  f.head = c.at<int>(c.w.head);
  f.target = a.target;
  f.row = c.at<int32_t>(c.w.row);
  f.stat = c.at<float>(c.w.stat);
  f.hit = c.at<float>(c.w.hit);
  f.full = c.at<float2>(c.w.full);
  f.part = c.at<float2>(c.w.part);
  f.loss = loss;
  f.lse = lse;
  f.status = a.status;
  f.c = a.soft ? kLog2e * (1.f / a.soft->tau) : kLog2e;
  f.tau2 = a.soft ? a.soft->tau * a.soft->tau : 1.f;
  f.inner = a.soft ? a.soft->inner : nullptr;
  // A row's logits depend on no other row, so bf16 rows need no gathering to be right; up to two units
  // a CTA it would only take longer (one row against 32000 x 128: 17 us with it, 13 without).
  const int64_t ct = ((int64_t)a.V + 255) / 256, units = c.w.cap / 128 * ct;
  f.direct = a.bf16 && units <= 2 * c.ctas;
  f.tiles = ct <= kWholeUnits;
  if (!f.direct) {
    RowArgs r{};
    r.loss = loss;
    r.lse_out = lse;
    e = prepare(a, c, r);
    if (e != cudaSuccess) return e;
  }
  switch ((a.H + 63) / 64 * 2 + (a.bf16 ? 0 : 1)) {
    case 2: e = run_fwd<1, 1>(c, a, f); break;
    case 3: e = run_fwd<1, 2>(c, a, f); break;
    case 4: e = run_fwd<2, 1>(c, a, f); break;
    case 5: e = run_fwd<2, 2>(c, a, f); break;
    case 6: e = run_fwd<3, 1>(c, a, f); break;
    case 7: e = run_fwd<3, 2>(c, a, f); break;
    case 8: e = run_fwd<4, 1>(c, a, f); break;
    default: e = run_fwd<4, 2>(c, a, f); break;
  }
  if (e != cudaSuccess) return e;
  note_launch();
  if (f.tiles) return cudaSuccess;
  e = launch_pdl(k_xent_join, dim3(c.ctas, 16), dim3(256), 0, st, f);
  if (e != cudaSuccess) return e;
  note_launch();
  return cudaSuccess;
}

cudaError_t xent_bwd(const XentArgs& a, const float* lse, const float* dloss, int grad_bf16,
                     void* dX, void* dW, int accumulate, cudaStream_t st) {
  if (a.n == 0) {
    if (!dW || accumulate) return cudaSuccess;
    return cudaMemsetAsync(dW, 0, (size_t)a.V * a.H * (grad_bf16 ? 2 : 4), st);
  }
  const int form = form_of(a.bf16, 1, grad_bf16);
  Call c;
  cudaError_t e = make_call(a, form, 1, st, &c);
  if (e != cudaSuccess) return e;
  RowArgs r{};
  r.backward = 1;
  r.grad_bf16 = grad_bf16;
  r.clear_dx = dX && !accumulate;
  r.lse_in = lse;
  r.dloss = dloss;
  r.dX = dX;
  e = prepare(a, c, r);
  if (e != cudaSuccess) return e;
  BwdArgs b{};
  b.H = a.H;
  b.V = a.V;
  b.accumulate = accumulate;
  b.head = c.at<int>(c.w.head);
  b.row = c.at<int32_t>(c.w.row);
  b.stat = c.at<float>(c.w.stat);
  b.dloss = dloss;
  b.part = c.at<float>(c.w.part);
  b.status = a.status;
  b.l2e = a.soft ? kLog2e * (1.f / a.soft->tau) : kLog2e;
  b.tau = a.soft ? a.soft->tau : 1.f;
  b.add_x = a.soft ? a.soft->add_x : nullptr;
  b.add_w = a.soft ? a.soft->add_w : nullptr;
  b.out_bf16 = grad_bf16;
  // a unit of dW takes 2-20% longer (column statistics, frequent tokens): 72 of 152 CTAs for dX
  b.split = !dW ? c.ctas : !dX ? 0 : std::max(1, c.ctas * 9 / 19);
  b.tiles = (!dX || a.V <= kWholeUnits * 128) && (!dW || a.n <= kWholeUnits * 128);
  const int tiles = (int)(c.w.vcap / 128);
  b.step = std::max(1, (int)(tiles * 0.618));
  while (std::gcd(b.step, tiles) != 1) ++b.step;
  b.cap = c.w.cap;
  b.vcap = c.w.vcap;
  b.dX = dX;
  b.dW = dW;
  if (form == kBf16) return run_bwd_h<kBf16>(c, a.W, b);
  if (form == kF16x1) return run_bwd_h<kF16x1>(c, a.W, b);
  return run_bwd_h<kF16x2>(c, a.W, b);
}

}  // namespace bg
