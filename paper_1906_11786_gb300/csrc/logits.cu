// Logits of states against a vocabulary: Z = X W^T, every one of them written.
//
// A tile is 128 tokens x up to 256 rows of X (128 with two terms at H > 128), computed transposed: the tokens are
// the rows of tensor memory, so that a lane has a token and a row of Z is side by side in a warpgroup, whatever
// its length and alignment.  The tile of X stays in shared memory while W passes through a ring in pieces of 128
// rows x 64 elements; CTAs take runs of tiles of W against one tile of X.
//
// Bound by the writing of Z: 16383 x 49999 x 256 bf16 to fp32 573 us (3.28 GB; 5.8 TB/s, floor 489), H = 64 526; to
// bf16 435 and 321 (floor 245; there by the way through shared memory, 128 lanes x 16 rows a barrier).  fp32 X and
// W: 650 us at H = 64, 740 at 128, 1170 at 256 (three products, operands from shared memory at its full rate with
// 128 rows a tile).  One row x 32000 x 128: 6.7 us, a launch.
//
// bf16 X and W enter the product as they are.  fp32 ones enter as two fp16 terms each (22 bits, down to
// 2^-17 of the largest magnitude in the row; each row of X and of W has a power of two of its own, undone in
// the epilogue), three products, the two small ones first, while the accumulator is small and loses little.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>

#include "answer.h"
#include "gemm_tc.h"
#include "kernels.h"
#include "tc_util.cuh"
#include "token.h"

namespace bg {

using namespace tc;

namespace {

constexpr int kEpilogue = 16;  // warps of the epilogue, four warpgroups; then a TMA warp and an MMA warp
constexpr int kThreads = (kEpilogue + 2) * 32;
constexpr int kMaxStages = 8;

inline size_t al(size_t x) { return (x + 255) & ~(size_t)255; }

// Workspace of the fp32 form: the terms' planes (rows rounded up to whole tiles) and the rows' exponents.
struct Ws {
  int64_t cap, vcap;
  size_t x, w, xe, we, total;
};
Ws layout(int bf16, int64_t n, int H, int V) {
  Ws w{};
  if (bf16) return w;
  w.cap = (n + 127) / 128 * 128;
  w.vcap = ((int64_t)V + 127) / 128 * 128;
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t at = o;
    o += al(bytes);
    return at;
  };
  w.x = take((size_t)2 * w.cap * H * 2);
  w.w = take((size_t)2 * w.vcap * H * 2);
  w.xe = take((size_t)(w.cap + 128) * 4);  // (whole tiles of 256 rows)
  w.we = take((size_t)w.vcap * 4);
  w.total = o;
  return w;
}

__device__ __forceinline__ float pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// Two fp16 terms of each row of X and W, times 2^(14 - e), e the exponent of the row's largest finite
// element.  A row is `lanes` = H / 8 threads out of a power of two of them.
struct SplitArgs {
  const float* src[2];
  uint16_t* dst[2];
  float* xs;    // scales of the rows of X
  int32_t* we;  // exponents of those of W
  int64_t rows[2], plane[2];
  int H, width;
};
__global__ void __launch_bounds__(256) k_logits_split(SplitArgs a) {
  grid_dep_launch();
  grid_dep_wait();
  const int lanes = a.H / 8, q = threadIdx.x & (a.width - 1), per = 256 / a.width;
  int64_t row = (int64_t)blockIdx.x * per + threadIdx.x / a.width;
  const int which = row >= a.rows[0];
  if (which) row -= a.rows[0];
  const bool in = row < a.rows[which] && q < lanes;
  float v[8];
  uint32_t top = 0;
  if (in) {
    const float4* p = reinterpret_cast<const float4*>(a.src[which] + row * a.H) + 2 * q;
    const float4 x = p[0], y = p[1];
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t b = __float_as_uint(v[j]) & 0x7FFFFFFFu;
      if (b < 0x7F800000u) top = max(top, b);
    }
  }
  for (int o = a.width / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (!in) return;
  const int e = max((int)(top >> 23) - 127, -100);
  const float up = pow2(14 - e);
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float x = v[2 * j] * up, y = v[2 * j + 1] * up;
    const __half2 h = __floats2half2_rn(x, y);
    hi[j] = *reinterpret_cast<const uint32_t*>(&h);
    const float2 f = __half22float2(h);
    const __half2 l = __floats2half2_rn(x - f.x, y - f.y);
    lo[j] = *reinterpret_cast<const uint32_t*>(&l);
  }
  uint16_t* d = a.dst[which] + row * a.H + q * 8;
  *reinterpret_cast<uint4*>(d) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  *reinterpret_cast<uint4*>(d + a.plane[which] * a.H) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  if (q == 0) {
    if (which == 0)
      a.xs[row] = pow2(e - 14);
    else
      a.we[row] = e - 14;
  }
}

// A few rows of X in fp32, without terms: a row of W is `width` threads of 8 elements (H / 8 rounded up to a power
// of two), read once for all of them, and what bounds it.  32000 x 128: 4 rows 9 us without terms, 5 rows 15 with
// their pass over W (49999 x 256: 22 and 36, 4001 x 64: 6 and 8; one row 6, 10 and 6).
constexpr int kFew = 4;
template <typename O>
__global__ void __launch_bounds__(256)
    k_logits_few(int n, int H, int V, int width, const float* __restrict__ X, const float* __restrict__ W, int64_t ldz,
                 O* __restrict__ Z) {
  grid_dep_launch();
  grid_dep_wait();
  const int lane = threadIdx.x & (width - 1), at = lane * 8;
  const bool in = at < H;
  float x[kFew][8];
#pragma unroll
  for (int r = 0; r < kFew; ++r)
#pragma unroll
    for (int j = 0; j < 8; ++j) x[r][j] = in && r < n ? X[r * H + at + j] : 0.f;
  const int step = gridDim.x * (256 / width);
  // (whole warps: the sums go over lanes)
  for (int v0 = blockIdx.x * (256 / width) + (threadIdx.x & ~31) / width; v0 < V; v0 += step) {
    const int v = v0 + (threadIdx.x & 31) / width;
    float w[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (in && v < V) {
      const float4* p = reinterpret_cast<const float4*>(W + (int64_t)v * H + at);
      const float4 a = __ldg(p), b = __ldg(p + 1);
      w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
      w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
    float mine = 0.f;
#pragma unroll
    for (int r = 0; r < kFew; ++r) {
      if (r >= n) break;
      float z = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) z = fmaf(x[r][j], w[j], z);
      for (int o = width / 2; o; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
      if (lane == r) mine = z;  // (four threads at least)
    }
    // An infinite element makes a logit NaN, as the terms do (of an infinite one the second is NaN): which kernel a
    // number of rows takes is not seen in its logits.  (Finite elements whose sum overflows stay infinite there too.)
    if (__any_sync(0xffffffffu, !(fabsf(mine) < INFINITY))) {
      unsigned bad = 0;  // bit r: row r of X with this row of W
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (!(fabsf(w[j]) < INFINITY)) bad = ~0u;
#pragma unroll
        for (int r = 0; r < kFew; ++r)
          if (!(fabsf(x[r][j]) < INFINITY)) bad |= 1u << r;
      }
      for (int o = width / 2; o; o >>= 1) bad |= __shfl_xor_sync(0xffffffffu, bad, o);
      if (lane < kFew && (bad >> lane & 1u)) mine = NAN;
    }
    if (lane < n && v < V) Z[lane * ldz + v] = (O)mine;
  }
}

template <int HC, int T, typename O>
struct Cfg {
  static constexpr int RN = T == 1 || HC <= 2 ? 256 : 128;  // rows of X of a tile
  static constexpr int XPIECE = RN * 128;                   // 64 elements of each
  static constexpr int X_BYTES = T * HC * XPIECE;
  // Staging of results on their way from a lane a token to a lane 16 bytes of a row, SR rows of a warpgroup.
  static constexpr int S = 32 / (int)sizeof(O), E = 16 / (int)sizeof(O);  // elements of a sector, of 16 bytes
  static constexpr int STEP = 128 - S;  // tokens from tile to tile
  static constexpr int SR = T == 2 && HC == 4 ? 8 : 16;
  static constexpr int ROUND = kEpilogue / 4 * SR;  // rows of all warpgroups
  static constexpr int STRIDE = 128 + S;  // elements of a staged row
  static constexpr int BUF = SR * STRIDE * (int)sizeof(O);
  static constexpr int STAGING = kEpilogue / 4 * BUF;
  static constexpr int PIECE = 16384;
  static constexpr int ROOM = (232448 - 2048 - X_BYTES - STAGING) / PIECE;
  static constexpr int ST = ROOM < kMaxStages ? ROOM : kMaxStages;
  static constexpr int SMEM = X_BYTES + ST * PIECE + STAGING + 2048;
  // The pieces of the high terms of a tile of W are used twice: they stay in the ring where they fit beside one
  // more (16383 rows x 49999 x 256 with fewer stages, loaded twice: 1270 instead of 1170 us).
  static constexpr bool KEPT = T == 2 && ST > HC;
  static constexpr int PIECES = T == 1 || KEPT ? T * HC : 3 * HC;  // of a tile of W that are loaded
  static_assert(ST >= 3 && SMEM <= 232448, "shared memory");
};

struct Bars {
  uint64_t x_full, x_empty, full[kMaxStages], empty[kMaxStages], d_full[2], d_empty[2], drain;
  uint32_t tmem;
  int abort;
};

struct Args {
  int V, vt;  // vt: tiles of W
  int64_t n, units, cap, vcap, ldz;
  const float* xs;
  const int32_t* we;
  int* status;
};

// Unit u is tile u / vt of X against tile u % vt of W; CTA c takes a run of them.
struct Walk {
  int64_t u, end;
  int64_t rt;
  int v, vt;
  bool fresh;  // first unit of its tile of X
  __device__ Walk(const Args& a) : vt(a.vt) {
    u = a.units * blockIdx.x / gridDim.x;
    end = a.units * (blockIdx.x + 1) / gridDim.x;
    rt = u / vt;
    v = (int)(u - rt * vt);
    fresh = true;
  }
  __device__ bool more() const { return u < end; }
  __device__ bool last_of_tile() const { return u + 1 == end || v + 1 == vt; }
  __device__ void next() {
    ++u;
    fresh = false;
    if (++v == vt) v = 0, ++rt, fresh = true;
  }
};

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
                 "=r"(r[7])
               : "r"(taddr));
}

// A warpgroup's way of SR rows of a tile to memory.
//
// A row of Z begins anywhere in a 32-byte sector, and a sector that is written in parts costs HBM twice (16383
// rows x 49999 fp32: 1240 us when each warp wrote its 32 tokens of a row at once, 611 where rows were aligned).
// So tiles overlap by a sector: of a tile's 128 tokens each row writes the STEP of them that fill whole sectors,
// wherever those begin in this row.  A staged row has its tokens at columns o .. o + 127, o the first one's
// place in its sector, so that sectors begin at multiples of S and 16 aligned bytes are a lane's.  STEP and the
// rows from one turn to the next are multiples of S: a place in the staging has the same o all along, and all
// addresses but one are made once.  (As bulk copies of a row each the same writes took 750-990 us.)
template <typename C, int T, typename O>
struct Writer {
  static constexpr int LPR = 128 / C::E, RPI = 32 / LPR, N = C::SR / (4 * RPI);  // lanes of a row; rows of a warp
  const Args& a;
  O* Z;
  O* buf;  // of this warpgroup
  int wg, q, lane;
  uint32_t put[C::SR];  // where this lane's token goes in the staged rows
  int64_t to[N];        // bytes from the first row's token t0 to this lane's parts of rows
  uint32_t get[N];

  __device__ __forceinline__ int offset(const O* p) const {
    return (int)((reinterpret_cast<uintptr_t>(p) & 31) / sizeof(O));
  }
  __device__ __forceinline__ Writer(const Args& a_, O* Z_, O* buf_, int wg_, int q_, int lane_)
      : a(a_), Z(Z_), buf(buf_), wg(wg_), q(q_), lane(lane_) {
    const O* first = Z + (int64_t)wg * C::SR * a.ldz;
    const int step = (int)(a.ldz & (C::S - 1)), o0 = offset(first), l = lane % LPR;
#pragma unroll
    for (int j = 0; j < C::SR; ++j)
      put[j] = smem_u32(buf + j * C::STRIDE + q * 32 + lane + ((o0 + j * step) & (C::S - 1)));
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int j = q * RPI + lane / LPR + 4 * RPI * k, o = (o0 + j * step) & (C::S - 1);
      const int col = (o ? C::S : 0) + l * C::E;  // of the row's whole sectors
      to[k] = ((int64_t)j * a.ldz + col - o) * (int)sizeof(O);
      get[k] = smem_u32(buf + j * C::STRIDE + min(col, 128 + C::S - C::E));
    }
  }
  __device__ __forceinline__ void sync() const { asm volatile("bar.sync %0, 128;" ::"r"(1 + wg) : "memory"); }
  __device__ __forceinline__ void stage(uint32_t at, float z, float) const {
    asm volatile("st.shared.f32 [%0], %1;" ::"r"(at), "f"(z) : "memory");
  }
  __device__ __forceinline__ void stage(uint32_t at, float z, __nv_bfloat16) const {
    const __nv_bfloat16 h = __float2bfloat16(z);
    asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"(*reinterpret_cast<const unsigned short*>(&h)) : "memory");
  }
  // d: rows c .. c + SR - 1 of the tile that begins at row0 and token t0, from this lane's token
  // (fp32 form: xs their rows' scales, up and up2 the token's)
  __device__ __forceinline__ void write(const uint32_t* d, const float* xs, int64_t row0, int rows, int c, int t0,
                                        float up, float up2, bool dead) {
    float z[C::SR];
#pragma unroll
    for (int j = 0; j < C::SR; ++j) z[j] = __uint_as_float(d[j]);
    if constexpr (T == 2) {
#pragma unroll
      for (int j = 0; j < C::SR; ++j) z[j] = z[j] * up * xs[j];
      if (__any_sync(0xffffffffu, up2 != 1.f)) {
#pragma unroll
        for (int j = 0; j < C::SR; ++j) z[j] *= up2;
      }
    }
    sync();  // the rows before these have been read
#pragma unroll
    for (int j = 0; j < C::SR; ++j) stage(put[j], z[j], O());
    sync();
    if (dead) return;
    char* first = reinterpret_cast<char*>(Z + (row0 + c) * a.ldz + t0);
    if (t0 > 0 && t0 + 128 < a.V) {
      uint4 x[N];
#pragma unroll
      for (int k = 0; k < N; ++k)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(x[k].x), "=r"(x[k].y), "=r"(x[k].z), "=r"(x[k].w)
                     : "r"(get[k]));
      const int left = lane % LPR < C::STEP / C::E ? rows - c - q * RPI - lane / LPR : 0;
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (left > 4 * RPI * k) __stcs(reinterpret_cast<uint4*>(first + to[k]), x[k]);
    } else {
      // the row's first and last tiles: also the tokens before the first whole sector, and all that are left
      for (int j = q; j < C::SR && c + j < rows; j += 4) {
        O* row = reinterpret_cast<O*>(first) + (int64_t)j * a.ldz;
        const int o = offset(row), cs = o ? C::S : 0;
        const int lo = t0 > 0 ? cs : o, hi = t0 + 128 >= a.V ? o + a.V - t0 : cs + C::STEP;
        for (int k = lo + lane; k < hi; k += 32) row[k - o] = buf[j * C::STRIDE + k];
      }
    }
  }
};

template <int HC, int T, typename O>
__global__ void __launch_bounds__(kThreads, 1)
    k_logits(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW,
             const __grid_constant__ Args a, O* Z) {
  using C = Cfg<HC, T, O>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem =
      reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = smem + C::X_BYTES;
  uint8_t* staging = ring + C::ST * C::PIECE;
  Bars* bars = reinterpret_cast<Bars*>(staging + C::STAGING);
  volatile int* abort = &bars->abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(&bars->x_full, 1);
    mbar_init(&bars->x_empty, 1);
    for (int s = 0; s < C::ST; ++s) {
      mbar_init(&bars->full[s], 1);
      mbar_init(&bars->empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&bars->d_full[b], 1);
      mbar_init(&bars->d_empty[b], kEpilogue);
    }
    mbar_init(&bars->drain, 1);
    bars->abort = 0;
    fence_mbar_init();
  }
  if (warp == kEpilogue + 1) {
    tmem_alloc(&bars->tmem, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_dep_launch();
  grid_dep_wait();
  const uint32_t tmem = bars->tmem;
  Walk w(a);

  if (warp == kEpilogue) {
    if (lane == 0) {
      tma_prefetch_desc(&tmX);
      tma_prefetch_desc(&tmW);
      uint32_t it = 0, seg = 0;
      bool ok = true;
      for (; w.more() && ok; w.next()) {
        if (w.fresh) {
          ok = seg == 0 || mbar_wait(&bars->x_empty, (seg - 1) & 1, a.status, 721, abort, 32);
          if (!ok) break;
          mbar_expect_tx(&bars->x_full, C::X_BYTES);
          for (int p = 0; p < T * HC; ++p)
            tma_load_2d(smem + p * C::XPIECE, &tmX, &bars->x_full, p % HC * 64,
                        (int)(p / HC * a.cap + w.rt * C::RN));
          ++seg;
        }
        // two terms: the low one's pieces, then the high one's (twice where the ring does not keep them)
        for (int p = 0; p < C::PIECES && ok; ++p, ++it) {
          const int s = it % C::ST;
          ok = mbar_wait(&bars->empty[s], ((it / C::ST) & 1) ^ 1, a.status, 722, abort, 32);
          if (!ok) break;
          mbar_expect_tx(&bars->full[s], C::PIECE);
          tma_load_2d(ring + s * C::PIECE, &tmW, &bars->full[s], p % HC * 64,
                      (int)(T == 2 && p < HC ? a.vcap : 0) + w.v * C::STEP);
        }
      }
      if (*abort) {  // copies in flight land before the block leaves
        for (uint32_t k = 0; seg && k < (1u << 22) && !mbar_try(&bars->x_full, (seg - 1) & 1); ++k) {
        }
        for (uint32_t q = it > C::ST ? it - C::ST : 0; q < it; ++q)
          for (uint32_t k = 0; k < (1u << 22) && !mbar_try(&bars->full[q % C::ST], (q / C::ST) & 1); ++k) {
          }
      }
    }
  } else if (warp == kEpilogue + 1) {
    const bool leader = elect_one_sync();
    const uint64_t X = desc_sw128_kmajor(smem_u32(smem)), R = desc_sw128_kmajor(smem_u32(ring));
    uint32_t it = 0, seg = 0, k = 0;
    bool ok = true;
    for (; w.more() && ok; w.next(), ++k) {
      if (w.fresh) {
        ok = mbar_wait(&bars->x_full, seg & 1, a.status, 723, abort);
        ++seg;
      }
      const int b = k & 1;
      ok = ok && mbar_wait(&bars->d_empty[b], ((k >> 1) & 1) ^ 1, a.status, 724, abort);
      const int rows = (int)min((int64_t)C::RN, a.n - w.rt * C::RN), N = (rows + 15) & ~15;
      const uint32_t idesc = T == 1 ? idesc_bf16_f32(128, N) : idesc_f16_f32(128, N);
      // piece p of W (in ring stage s) by the term of X that begins at piece xp
      auto product = [&](int s, int xp, bool more) {
        const uint64_t ad = R + s * (C::PIECE >> 4), bd = X + (uint64_t)xp * (C::XPIECE >> 4);
        if (leader) {
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            mma_ss(tmem + b * 256, ad + kk * 2, bd + kk * 2, idesc, more || kk > 0);
        }
      };
      // (past H the pieces hold zeros)
      for (int p = 0; p < C::PIECES && ok; ++p) {
        const uint32_t i = it + p;
        ok = mbar_wait(&bars->full[i % C::ST], (i / C::ST) & 1, a.status, 725, abort);
        if (!ok) break;
        tc_fence_after();
        // low x high, then high x low; the high terms' pieces stay for high x high
        product(i % C::ST, p < T * HC ? p : p - T * HC, p > 0);
        if (leader && (!C::KEPT || p < HC)) tc_commit(&bars->empty[i % C::ST]);
        __syncwarp();
      }
      if (C::KEPT && ok)
        for (int p = 0; p < HC; ++p) {
          const uint32_t i = it + HC + p;
          product(i % C::ST, p, true);
          if (leader) tc_commit(&bars->empty[i % C::ST]);
          __syncwarp();
        }
      it += C::PIECES;
      if (ok && leader) {
        tc_commit(&bars->d_full[b]);
        if (w.last_of_tile()) tc_commit(&bars->x_empty);
      }
      __syncwarp();
    }
    if (leader) tc_commit(&bars->drain);
    __syncwarp();
    for (uint32_t q = 0; q < (1u << 24) && !mbar_try(&bars->drain, 0); ++q) {
    }
  } else {
    const int q = warp & 3, wg = warp >> 2;
    const uint32_t base = tmem + ((uint32_t)(q * 32) << 16);
    Writer<C, T, O> out(a, Z, reinterpret_cast<O*>(staging + wg * C::BUF), wg, q, lane);
    uint32_t k = 0;
    bool dead = false;  // a wait gave up: the warpgroup's barriers are met all the same, nothing is written
    for (; w.more(); w.next(), ++k) {
      const int b = k & 1, t0 = w.v * C::STEP, v = t0 + q * 32 + lane;
      const int64_t row0 = w.rt * C::RN;
      const int rows = (int)min((int64_t)C::RN, a.n - row0);
      // a token's scale in two parts: with the row's between them nothing overflows that the logit does not
      const int we = T == 2 && v < a.V ? a.we[v] : 0, we1 = min(we, 60);
      const float up = pow2(we1), up2 = pow2(we - we1);
      dead = dead || !mbar_wait(&bars->d_full[b], (k >> 1) & 1, a.status, 726, abort, 20);
      dead = __any_sync(0xffffffffu, dead);
      tc_fence_after();
      auto fetch = [&](int c, uint32_t* d) {
        if (C::SR == 16)
          tmem_ld16(base + b * 256 + c, d);
        else
          tmem_ld8(base + b * 256 + c, d);
        tmem_wait_ld();
      };
      for (int c = wg * C::SR; c < rows; c += C::ROUND) {
        uint32_t d[C::SR];
        float xs[T == 2 ? C::SR : 4];
        if constexpr (T == 2) {  // (the scales' array is as long as whole tiles are)
#pragma unroll
          for (int j = 0; j < C::SR; j += 4)
            *reinterpret_cast<float4*>(xs + j) = __ldg(reinterpret_cast<const float4*>(a.xs + row0 + c + j));
        }
        fetch(c, d);
        if (c + C::ROUND >= rows) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars->d_empty[b]);
        }
        out.write(d, xs, row0, rows, c, t0, up, up2, dead);
      }
      if (wg * C::SR >= rows) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars->d_empty[b]);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kEpilogue + 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int HC, int T, typename O>
cudaError_t run(const LogitsArgs& l, const Ws& ws, cudaStream_t st) {
  using C = Cfg<HC, T, O>;
  char* base = static_cast<char*>(l.ws);
  CUtensorMap mx, mw;
  const bool ok = T == 1 ? make_map_ld(&mx, l.X, l.n, l.H, l.H, C::RN) && make_map_ld(&mw, l.W, l.V, l.H, l.H, 128)
                         : make_map_ld(&mx, base + ws.x, 2 * ws.cap, l.H, l.H, C::RN) &&
                               make_map_ld(&mw, base + ws.w, 2 * ws.vcap, l.H, l.H, 128);
  if (!ok) return cudaErrorInvalidValue;
  static std::atomic<uint64_t> done{0};
  cudaError_t e = allow_smem(k_logits<HC, T, O>, C::SMEM, done);
  if (e != cudaSuccess) return e;
  Args a{};
  a.V = l.V;
  a.vt = l.V <= 128 ? 1 : (l.V - 128 + C::STEP - 1) / C::STEP + 1;
  a.n = l.n;
  a.units = (l.n + C::RN - 1) / C::RN * a.vt;
  a.cap = ws.cap;
  a.vcap = ws.vcap;
  a.ldz = l.ldz;
  a.xs = reinterpret_cast<const float*>(base + ws.xe);
  a.we = reinterpret_cast<const int32_t*>(base + ws.we);
  a.status = l.status;
  const int ctas = (int)std::min<int64_t>(gemm_tn_num_sms(), a.units);
  e = launch_pdl(k_logits<HC, T, O>, dim3(ctas), dim3(kThreads), C::SMEM, st, mx, mw, a, static_cast<O*>(l.Z));
  if (e == cudaSuccess) note_launch();
  return e;
}

template <int T, typename O>
cudaError_t run_h(const LogitsArgs& l, const Ws& ws, cudaStream_t st) {
  switch ((l.H + 63) / 64) {
    case 1: return run<1, T, O>(l, ws, st);
    case 2: return run<2, T, O>(l, ws, st);
    case 3: return run<3, T, O>(l, ws, st);
    default: return run<4, T, O>(l, ws, st);
  }
}

}  // namespace

size_t logits_ws_bytes(int bf16, int64_t n, int H, int V) { return n <= kFew ? 0 : layout(bf16, n, H, V).total; }

cudaError_t logits_fwd(const LogitsArgs& l, cudaStream_t st) {
  if (l.n == 0) return cudaSuccess;
  const Ws ws = layout(l.bf16, l.n, l.H, l.V);
  if (l.bf16)
    return l.out_bf16 ? run_h<1, __nv_bfloat16>(l, ws, st) : run_h<1, float>(l, ws, st);
  const int width = l.H / 8 <= 4 ? 4 : l.H / 8 <= 8 ? 8 : l.H / 8 <= 16 ? 16 : 32;
  if (l.n <= kFew) {
    // rows of W that are a block's at a time, eight blocks an SM
    const int per = 256 / width;
    const dim3 grid((unsigned)std::min<int64_t>((l.V + per - 1) / per, 152 * 8));
    const float *X = static_cast<const float*>(l.X), *W = static_cast<const float*>(l.W);
    const cudaError_t e =
        l.out_bf16 ? launch_pdl(k_logits_few<__nv_bfloat16>, grid, dim3(256), 0, st, (int)l.n, l.H, l.V, width, X, W,
                                l.ldz, static_cast<__nv_bfloat16*>(l.Z))
                   : launch_pdl(k_logits_few<float>, grid, dim3(256), 0, st, (int)l.n, l.H, l.V, width, X, W, l.ldz,
                                static_cast<float*>(l.Z));
    if (e == cudaSuccess) note_launch();
    return e;
  }
  SplitArgs s{};
  char* base = static_cast<char*>(l.ws);
  s.src[0] = static_cast<const float*>(l.X);
  s.src[1] = static_cast<const float*>(l.W);
  s.dst[0] = reinterpret_cast<uint16_t*>(base + ws.x);
  s.dst[1] = reinterpret_cast<uint16_t*>(base + ws.w);
  s.xs = reinterpret_cast<float*>(base + ws.xe);
  s.we = reinterpret_cast<int32_t*>(base + ws.we);
  s.rows[0] = l.n;
  s.rows[1] = l.V;
  s.plane[0] = ws.cap;
  s.plane[1] = ws.vcap;
  s.H = l.H;
  s.width = width;
  const int per = 256 / s.width;
  cudaError_t e = launch_pdl(k_logits_split, dim3((unsigned)((l.n + l.V + per - 1) / per)), dim3(256), 0, st, s);
  if (e != cudaSuccess) return e;
  note_launch();
  return l.out_bf16 ? run_h<2, __nv_bfloat16>(l, ws, st) : run_h<2, float>(l, ws, st);
}

}  // namespace bg
