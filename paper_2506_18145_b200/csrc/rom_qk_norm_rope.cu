// RMS norm of every head of q and k and its rotation by the row's position, in one pass, and the backward of both.
//
// Eight lanes (fewer or more by the head's width) own a head of one row: each holds two runs of eight places, the two halves of eight pairs in the rotated part,
// sixteen adjacent places behind it.  The angle pos * inv_freq is formed in two numbers of 64 bits and reduced to a turn before it is rounded: an fp32 product is off by 0.06 at a position
// of a million.  A block takes the sines and cosines of its rows once, into shared memory; a group of lanes folds them and the weights into two factors a place for the
// heads of a row that it works on, with several heads' loads in flight.
//
// Memory bounds both: everything is read and written once, at 88 to 91 % of a copy's rate for 0.5 and 0.8 GB of bf16 (95 and 141 us a pass).  The backward needs twice the bytes in
// flight for that, so it copies heads ahead into shared memory.  One row takes 2 us on the device.
#include <math.h>

#include "rom_serve.cuh"

namespace rom {
namespace {

constexpr int QK_THREADS = 256;

struct QkArgs {
  const void *q, *k;            // inputs of the forward
  const void *gq, *gk;          // backward: gradients of its outputs (contiguous)
  void *yq, *yk;                // what the call writes
  long long ldq, ldk, ldyq, ldyk;
  const float *w_q, *w_k;
  const int32_t* pos;
  const float* inv_freq;
  float* part;                  // backward: [blocks][d_head] sums of dn xhat, the blocks of q first
  int rows, nq, nk, d, rot, interleaved;
  float eps;
};

// Eight adjacent elements as four pairs.
template <typename T>
__device__ __forceinline__ void pairs_of(const Raw8<T>& raw, float2 (&v)[4]) {
  float x[8];
  raw.get(x);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = make_float2(x[2 * e], x[2 * e + 1]);
}
template <typename T>
__device__ __forceinline__ void store_pairs(T* p, const float2 (&v)[4]) {
  const float x[8] = {v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
  Raw8<T>::store(p, x);
}
// 16 bytes from memory into the lane's own place in shared memory, and back.
__device__ __forceinline__ void copy16(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// A lane's places: runs at oa and ob.  Where a run does not exist its loads go to run a (or to the head's first) and count as zeros.
struct QkLane {
  int oa, ob;
  bool has_a, has_b, turns;
  __device__ __forceinline__ QkLane(int l, const QkArgs& p) {
    turns = 16 * l < p.rot;
    const bool apart = turns && !p.interleaved;
    oa = apart ? 8 * l : 16 * l;
    ob = apart ? p.rot / 2 + 8 * l : 16 * l + 8;
    has_a = oa < p.d;
    has_b = ob < p.d;
    if (!has_a) oa = 0;
    if (!has_b) ob = oa;
  }
};
// 1 / 2 pi, rounded to 64 bits, and what that left
constexpr double INV_2PI = 0.15915494309189535, INV_2PI_LO = -9.839338337591243e-18;
// cos and sin of rows [row0, row0 + n) of a block, [n][rot / 2].
__device__ __forceinline__ void block_angles(const QkArgs& p, int row0, int n, float2* cs) {
  const int half = p.rot / 2;
  for (int i = threadIdx.x; i < n * half; i += QK_THREADS) {
    const int r = i / half, e = i - r * half;
    // the product's 55 bits and 1 / 2 pi as two numbers each: with one, an angle of 2^31 was 4e-7 off, eight units of fp32
    const double pos = (double)__ldg(p.pos + row0 + r), freq = (double)__ldg(p.inv_freq + e), a = pos * freq, a_lo = fma(pos, freq, -a);
    const double t = a * INV_2PI, t_lo = fma(a, INV_2PI, -t) + fma(a, INV_2PI_LO, a_lo * INV_2PI);
    float s, c;
    sincospif(2.0f * (float)((t - rint(t)) + t_lo), &s, &c);
    cs[i] = make_float2(c, s);
  }
}
// The lane's eight pairs of a row: cosines and sines (1 and 0 where nothing is turned).
__device__ __forceinline__ void lane_angles(const QkLane& at, int l, const float2* cs, float (&c)[8], float (&s)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float2 v = at.turns ? cs[8 * l + e] : make_float2(1.0f, 0.0f);
    c[e] = v.x;
    s[e] = v.y;
  }
}
// Sum over a group of LANES lanes; all lanes of the warp call it.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int m = LANES / 2; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}
__device__ __forceinline__ void load_weights(const float* w, const QkLane& at, float2 (&wa)[4], float2 (&wb)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    wa[e] = w ? make_float2(__ldg(w + at.oa + 2 * e), __ldg(w + at.oa + 2 * e + 1)) : both(1.0f);
    wb[e] = w ? make_float2(__ldg(w + at.ob + 2 * e), __ldg(w + at.ob + 2 * e + 1)) : both(1.0f);
  }
}
// What the lane multiplies a run's places with: y = x f + other g, other being the pair's second member, in the other run or (INTER: interleaved) beside it.  Where nothing is
// turned g is 0.
struct Factors { float2 fa[4], ga[4], fb[4], gb[4]; };
template <bool INTER>
__device__ __forceinline__ void factors(Factors& f, const float2 (&wa)[4], const float2 (&wb)[4], const float (&c)[8], const float (&s)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (INTER) {
      f.fa[e] = __fmul2_rn(wa[e], both(c[e]));
      f.ga[e] = make_float2(-wa[e].y * s[e], wa[e].x * s[e]);
      f.fb[e] = __fmul2_rn(wb[e], both(c[4 + e]));
      f.gb[e] = make_float2(-wb[e].y * s[4 + e], wb[e].x * s[4 + e]);
    } else {
      const float2 c2 = make_float2(c[2 * e], c[2 * e + 1]), s2 = make_float2(s[2 * e], s[2 * e + 1]);
      f.fa[e] = __fmul2_rn(wa[e], c2);
      f.ga[e] = __fmul2_rn(wb[e], make_float2(-s2.x, -s2.y));
      f.fb[e] = __fmul2_rn(wb[e], c2);
      f.gb[e] = __fmul2_rn(wa[e], s2);
    }
  }
}

// A block has `rows_b` rows and the splits [blockIdx.y splits_b, ..) of their heads; a split is up to `per` heads of q or of k, and a group of LANES lanes takes one of a row at
// a time.  Groups of a warp run in step (their sums are warp shuffles): what lies beyond an end is computed from the last valid place and not stored.
template <typename T, int LANES, bool INTER>
__global__ void __launch_bounds__(QK_THREADS, 2) qk_norm_rope_kernel(QkArgs p, int rows_b, int splits_b, int per) {
  constexpr int GROUPS = QK_THREADS / LANES, U = sizeof(T) == 2 ? 4 : 2;
  extern __shared__ float2 cs[];
  const int l = threadIdx.x % LANES, row0 = blockIdx.x * rows_b, n_rows = min(rows_b, p.rows - row0);
  const int splits_q = (p.nq + per - 1) / per, splits = splits_q + (p.nk + per - 1) / per, s0 = blockIdx.y * splits_b, ns = min(splits_b, splits - s0);
  const QkLane at(l, p);
  const float inv_d = 1.0f / (float)p.d;
  pdl_sync();
  if (p.rot) block_angles(p, row0, n_rows, cs);
  __syncthreads();
  const int items = n_rows * ns;
  for (int i0 = threadIdx.x / 32 * (32 / LANES); i0 < items; i0 += GROUPS) {
    const int i = i0 + (threadIdx.x & 31) / LANES, item = min(i, items - 1), r = item / ns, split = s0 + item - r * ns;
    const bool is_k = split >= splits_q;
    const int h0 = (is_k ? split - splits_q : split) * per, n = min(per, (is_k ? p.nk : p.nq) - h0), stored = i < items ? n : 0;
    const long long row = row0 + r;
    const T* x = (is_k ? static_cast<const T*>(p.k) + row * p.ldk : static_cast<const T*>(p.q) + row * p.ldq) + (size_t)h0 * p.d;
    T* y = (is_k ? static_cast<T*>(p.yk) + row * p.ldyk : static_cast<T*>(p.yq) + row * p.ldyq) + (size_t)h0 * p.d;
    Factors f;
    {
      float c[8], s[8];
      float2 wa[4], wb[4];
      lane_angles(at, l, cs + r * (p.rot / 2), c, s);
      load_weights(is_k ? p.w_k : p.w_q, at, wa, wb);
      factors<INTER>(f, wa, wb, c, s);
    }
    const int most = __reduce_max_sync(0xffffffffu, n);      // of the warp's groups
    for (int h = 0; h < most; h += U) {
      Raw8<T> ra[U], rb[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const T* from = x + min(h + u, n - 1) * p.d;
        ra[u].load(from + at.oa);
        rb[u].load(from + at.ob);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float2 a[4], b[4], sa = both(0.0f), sb = both(0.0f);
        pairs_of(ra[u], a);
        pairs_of(rb[u], b);
#pragma unroll
        for (int e = 0; e < 4; ++e) { sa = __ffma2_rn(a[e], a[e], sa); sb = __ffma2_rn(b[e], b[e], sb); }
        const float ss = (at.has_a ? sa.x + sa.y : 0.0f) + (at.has_b ? sb.x + sb.y : 0.0f);
        const float2 r2 = both(rsqrtf(fmaf(lanes_sum<LANES>(ss), inv_d, p.eps)));
        float2 ya[4], yb[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 oa = INTER ? make_float2(a[e].y, a[e].x) : b[e], ob = INTER ? make_float2(b[e].y, b[e].x) : a[e];
          ya[e] = __fmul2_rn(__ffma2_rn(oa, f.ga[e], __fmul2_rn(a[e], f.fa[e])), r2);
          yb[e] = __fmul2_rn(__ffma2_rn(ob, f.gb[e], __fmul2_rn(b[e], f.fb[e])), r2);
        }
        T* to = y + (h + u) * p.d;
        if (h + u < stored && at.has_a) store_pairs(to + at.oa, ya);
        if (h + u < stored && at.has_b) store_pairs(to + at.ob, yb);
      }
    }
  }
}

// The backward: rows in tiles of `rows_b`, walked by a fixed number of blocks; dw is summed per lane, then over the block's groups in order, and the blocks' sums by
// qk_sum_weights: the same from run to run.  A block works on the heads of q or on those of k (the blocks behind the first blocks_q): one set
// of weights and sums in registers.
// A lane copies what it needs of the next heads into places of its own in shared memory (AHEAD heads, of x and dy): in registers they left none for the arithmetic, and one
// head ahead was half of what memory takes to answer.
template <typename T> struct QkBwd {
  static constexpr int PIECES = 4 * sizeof(T) / 2, AHEAD = sizeof(T) == 2 ? 4 : 2, STAGE = PIECES * QK_THREADS * 16;      // 16-byte pieces of a head and lane: runs a, b of x, a, b of dy
};
template <typename T, int LANES, bool INTER>
__global__ void __launch_bounds__(QK_THREADS, 2) qk_norm_rope_bwd_kernel(QkArgs p, int rows_q, int rows_k, int per, int blocks_q) {
  constexpr int GROUPS = QK_THREADS / LANES;
  using B = QkBwd<T>;
  extern __shared__ __align__(16) unsigned char bwd_smem[];      // heads ahead, afterwards the sums [GROUPS][d]; then cos and sin [rows_b][rot / 2]
  float2* cs = reinterpret_cast<float2*>(bwd_smem + B::AHEAD * B::STAGE);
  const uint32_t place = (uint32_t)__cvta_generic_to_shared(bwd_smem) + threadIdx.x * 16;
  const bool is_k = (int)blockIdx.x >= blocks_q;
  const int block = is_k ? blockIdx.x - blocks_q : blockIdx.x, blocks = is_k ? gridDim.x - blocks_q : blocks_q;
  const int l = threadIdx.x % LANES, heads = is_k ? p.nk : p.nq, splits = (heads + per - 1) / per;
  const QkLane at(l, p);
  pdl_sync();
  const long long ldx = is_k ? p.ldk : p.ldq, ldy = is_k ? p.ldyk : p.ldyq;
  const T *xs = static_cast<const T*>(is_k ? p.k : p.q), *gs = static_cast<const T*>(is_k ? p.gk : p.gq);
  T* ys = static_cast<T*>(is_k ? p.yk : p.yq);
  float2 wa[4], wb[4], sa[4], sb[4];
  load_weights(is_k ? p.w_k : p.w_q, at, wa, wb);
#pragma unroll
  for (int e = 0; e < 4; ++e) sa[e] = sb[e] = both(0.0f);
  const float inv_d = 1.0f / (float)p.d;
  const int rows_b = is_k ? rows_k : rows_q;
  for (int row0 = block * rows_b; row0 < p.rows; row0 += blocks * rows_b) {
    const int n_rows = min(rows_b, p.rows - row0), items = n_rows * splits;
    __syncthreads();
    if (p.rot) block_angles(p, row0, n_rows, cs);
    __syncthreads();
    for (int i0 = threadIdx.x / 32 * (32 / LANES); i0 < items; i0 += GROUPS) {
      const int i = i0 + (threadIdx.x & 31) / LANES, item = min(i, items - 1), r = item / splits, h0 = (item - r * splits) * per, n = min(per, heads - h0), stored = i < items ? n : 0;
      const long long row = row0 + r;
      float c[8], s[8];                // (the rotation back: sines taken negative below)
      lane_angles(at, l, cs + r * (p.rot / 2), c, s);
      const T *x = xs + row * ldx + (size_t)h0 * p.d, *g = gs + (row * heads + h0) * p.d;
      T* y = ys + row * ldy + (size_t)h0 * p.d;
      // dn, the rotation back of dy
      auto back = [&](const float2 (&va)[4], const float2 (&vb)[4], float2 (&da)[4], float2 (&db)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (INTER) {
            da[e] = __ffma2_rn(make_float2(va[e].y, va[e].x), make_float2(s[e], -s[e]), __fmul2_rn(va[e], both(c[e])));
            db[e] = __ffma2_rn(make_float2(vb[e].y, vb[e].x), make_float2(s[4 + e], -s[4 + e]), __fmul2_rn(vb[e], both(c[4 + e])));
          } else {
            const float2 c2 = make_float2(c[2 * e], c[2 * e + 1]), s2 = make_float2(s[2 * e], s[2 * e + 1]);
            da[e] = __ffma2_rn(vb[e], s2, __fmul2_rn(va[e], c2));
            db[e] = __ffma2_rn(va[e], make_float2(-s2.x, -s2.y), __fmul2_rn(vb[e], c2));
          }
        }
      };
      const int most = __reduce_max_sync(0xffffffffu, n);      // of the warp's groups
      auto ask = [&](int h) {          // (an empty group behind the last head: the count of groups is the same)
        if (h < most) {
          const int off = min(h, n - 1) * p.d;
          const T* from[4] = {x + off + at.oa, x + off + at.ob, g + off + at.oa, g + off + at.ob};
          const uint32_t to = place + (h % B::AHEAD) * B::STAGE;
#pragma unroll
          for (int q = 0; q < B::PIECES; ++q) copy16(to + q * (QK_THREADS * 16), from[q / (B::PIECES / 4)] + q % (B::PIECES / 4) * (16 / sizeof(T)));
        }
        copies_commit();
      };
#pragma unroll
      for (int h = 0; h < B::AHEAD - 1; ++h) ask(h);
      for (int h = 0; h < most; ++h) {
        ask(h + B::AHEAD - 1);
        copies_wait<B::AHEAD - 1>();
        const uint32_t here = place + (h % B::AHEAD) * B::STAGE;
        // eight values of a run, unpacked where they are used: once for the sums, once for the result
        auto run = [&](int which, float2 (&v)[4]) {
          if constexpr (sizeof(T) == 2) {
            Raw8<T> raw;
            raw.q = lds16(here + which * (QK_THREADS * 16));
            pairs_of(raw, v);
          } else {
            const uint4 lo = lds16(here + 2 * which * (QK_THREADS * 16)), hi = lds16(here + (2 * which + 1) * (QK_THREADS * 16));
            v[0] = make_float2(__uint_as_float(lo.x), __uint_as_float(lo.y));
            v[1] = make_float2(__uint_as_float(lo.z), __uint_as_float(lo.w));
            v[2] = make_float2(__uint_as_float(hi.x), __uint_as_float(hi.y));
            v[3] = make_float2(__uint_as_float(hi.z), __uint_as_float(hi.w));
          }
        };
        float ss, dot;
        {
          float2 a[4], b[4], va[4], vb[4], da[4], db[4], qa = both(0.0f), qb = both(0.0f), ta = both(0.0f), tb = both(0.0f);
          run(0, a);
          run(1, b);
          run(2, va);
          run(3, vb);
          back(va, vb, da, db);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            qa = __ffma2_rn(a[e], a[e], qa);
            qb = __ffma2_rn(b[e], b[e], qb);
            ta = __ffma2_rn(__fmul2_rn(a[e], da[e]), wa[e], ta);
            tb = __ffma2_rn(__fmul2_rn(b[e], db[e]), wb[e], tb);
          }
          ss = (at.has_a ? qa.x + qa.y : 0.0f) + (at.has_b ? qb.x + qb.y : 0.0f);
          dot = (at.has_a ? ta.x + ta.y : 0.0f) + (at.has_b ? tb.x + tb.y : 0.0f);
        }
        const float r1 = rsqrtf(fmaf(lanes_sum<LANES>(ss), inv_d, p.eps));
        const float m = lanes_sum<LANES>(dot) * inv_d * r1 * r1;      // mean(dn w xhat) r
        if (h < stored) {
          float2 a[4], b[4], va[4], vb[4], da[4], db[4];
          run(0, a);
          run(1, b);
          run(2, va);
          run(3, vb);
          back(va, vb, da, db);
          T* to = y + h * p.d;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            sa[e] = __ffma2_rn(__fmul2_rn(a[e], da[e]), both(r1), sa[e]);
            sb[e] = __ffma2_rn(__fmul2_rn(b[e], db[e]), both(r1), sb[e]);
            a[e] = __fmul2_rn(both(r1), __ffma2_rn(a[e], both(-m), __fmul2_rn(da[e], wa[e])));
            b[e] = __fmul2_rn(both(r1), __ffma2_rn(b[e], both(-m), __fmul2_rn(db[e], wb[e])));
          }
          if (at.has_a) store_pairs(to + at.oa, a);
          if (at.has_b) store_pairs(to + at.ob, b);
        }
      }
    }
  }
  copies_wait<0>();
  __syncthreads();
  float* sums = reinterpret_cast<float*>(bwd_smem);
  float* mine = sums + (size_t)(threadIdx.x / LANES) * p.d;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (at.has_a) { mine[at.oa + 2 * e] = sa[e].x; mine[at.oa + 2 * e + 1] = sa[e].y; }
    if (at.has_b) { mine[at.ob + 2 * e] = sb[e].x; mine[at.ob + 2 * e + 1] = sb[e].y; }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.d; i += QK_THREADS) {
    float s = 0.0f;
    for (int g = 0; g < GROUPS; ++g) s += sums[(size_t)g * p.d + i];
    p.part[(size_t)blockIdx.x * p.d + i] = s;
  }
}
// One warp a column: lanes take the blocks' sums in turn, in 64 bits, and meet in a fixed order.
__global__ void __launch_bounds__(QK_THREADS) qk_sum_weights(const float* part, int blocks_q, int blocks, int d, float* dw_q, float* dw_k) {
  pdl_sync();
  const int i = blockIdx.x * (QK_THREADS / 32) + threadIdx.x / 32, lane = threadIdx.x & 31;
  if (i >= 2 * d) return;
  const int first = i < d ? 0 : blocks_q, end = i < d ? blocks_q : blocks, col = i < d ? i : i - d;
  double s = 0.0;
  for (int b = first + lane; b < end; b += 32) s += (double)part[(size_t)b * d + col];
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
  float* to = i < d ? dw_q : dw_k;
  if (lane == 0 && to) to[col] = (float)s;
}

int check_qk(const rom_qk_config* c, int rows) {
  if (!c || rows < 0 || c->n_q_heads < 1 || c->n_k_heads < 1 || c->d_head < 1 || c->rot_dim < 0 || c->rot_dim > c->d_head) return ROM_ERR_INVALID_ARG;
  if ((c->dtype != ROM_F32 && c->dtype != ROM_BF16) || c->interleaved < 0 || c->interleaved > 1 || !(c->eps > 0.0f) || !isfinite(c->eps)) return ROM_ERR_INVALID_ARG;
  if (c->d_head % 8 != 0 || c->d_head > 256 || c->rot_dim % 16 != 0 || c->n_q_heads > 1024 || c->n_k_heads > 1024 || rows >= 1 << 30) return ROM_ERR_UNSUPPORTED;
  return ROM_OK;
}
int lanes_of(int d) { int n = 1; while (16 * n < d) n *= 2; return n; }
// Heads a group takes of a row: its factors cost about as much as two heads, so up to sixteen, as long as the groups fill the SMs (two blocks each) twice.
int heads_per_group(int rows, int heads, int lanes) {
  int per = 16;
  while (per > 1 && (per / 2 >= heads || (long long)rows * heads / per < 148LL * 4 * (QK_THREADS / lanes))) per /= 2;
  return per;
}
// Rows of a block: one split for every group.
int rows_per_block(int splits, int lanes) {
  const int n = QK_THREADS / lanes / splits;
  return n < 1 ? 1 : n < 32 ? n : 32;
}
constexpr int kBwdBlocks = 296;      // of q and k together, two to an SM, where each has several tiles; twice as many of one tile each
template <typename F>
cudaError_t by_lanes(int lanes, F&& go) {
  switch (lanes) {
    case 1: return go(std::integral_constant<int, 1>());
    case 2: return go(std::integral_constant<int, 2>());
    case 4: return go(std::integral_constant<int, 4>());
    case 8: return go(std::integral_constant<int, 8>());
    default: return go(std::integral_constant<int, 16>());
  }
}
template <typename T>
cudaError_t launch_forward(const rom_qk_config& c, const QkArgs& p, cudaStream_t st) {
  return by_lanes(lanes_of(c.d_head), [&](auto n) {
    constexpr int LANES = decltype(n)::value;
    const int per = heads_per_group(p.rows, p.nq + p.nk, LANES), splits = (p.nq + per - 1) / per + (p.nk + per - 1) / per, rows_b = rows_per_block(splits, LANES);
    const int splits_b = rows_b > 1 || per > 1 || splits < QK_THREADS / LANES ? splits : QK_THREADS / LANES;      // few rows of many heads: a row on several blocks
    const size_t smem = sizeof(float2) * (size_t)rows_b * (p.rot / 2);           // at most 32 rows of 128 pairs
    count_launch();
    return launch_k(p.interleaved ? qk_norm_rope_kernel<T, LANES, true> : qk_norm_rope_kernel<T, LANES, false>, dim3((p.rows + rows_b - 1) / rows_b, (splits + splits_b - 1) / splits_b),
                    QK_THREADS, smem, st, p, rows_b, splits_b, per);
  });
}
template <typename T>
cudaError_t launch_backward(const rom_qk_config& c, const QkArgs& p, float* dw_q, float* dw_k, cudaStream_t st) {
  const int lanes = lanes_of(c.d_head), per = heads_per_group(p.rows, p.nq + p.nk, lanes);
  const int splits_q = (p.nq + per - 1) / per, splits_k = (p.nk + per - 1) / per, rows_q = rows_per_block(splits_q, lanes), rows_k = rows_per_block(splits_k, lanes);
  int blocks_q = (p.rows + rows_q - 1) / rows_q, blocks_k = (p.rows + rows_k - 1) / rows_k;      // tiles
  if (blocks_q + blocks_k > 2 * kBwdBlocks) {      // blocks by their share of the heads
    const int want = kBwdBlocks * p.nq / (p.nq + p.nk), n = want < 1 ? 1 : want >= kBwdBlocks ? kBwdBlocks - 1 : want;
    blocks_q = blocks_q < n ? blocks_q : n;
    blocks_k = blocks_k < kBwdBlocks - n ? blocks_k : kBwdBlocks - n;
  }
  blocks_q = blocks_q < 1 ? 1 : blocks_q;
  blocks_k = blocks_k < 1 ? 1 : blocks_k;
  const int blocks = blocks_q + blocks_k, rows_b = rows_q > rows_k ? rows_q : rows_k;
  const cudaError_t e = by_lanes(lanes, [&](auto n) {
    constexpr int LANES = decltype(n)::value;
    // 64 KB of heads ahead (the sums, at most 16 KB, lie over them: a group's lanes hold more than half as many places as d, or all) and at most 32 rows of 128 pairs
    constexpr int ahead = QkBwd<T>::AHEAD * QkBwd<T>::STAGE, most = ahead + 32 * 128 * (int)sizeof(float2);
    auto kern = p.interleaved ? qk_norm_rope_bwd_kernel<T, LANES, true> : qk_norm_rope_bwd_kernel<T, LANES, false>;
    const cudaError_t set = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (set != cudaSuccess) return set;
    count_launch();
    return launch_k(kern, dim3(blocks), QK_THREADS, ahead + sizeof(float2) * (size_t)rows_b * (p.rot / 2), st, p, rows_q, rows_k, per, blocks_q);
  });
  if (e != cudaSuccess || (!dw_q && !dw_k)) return e;
  count_launch();
  return launch_k(qk_sum_weights, dim3((2 * p.d + QK_THREADS / 32 - 1) / (QK_THREADS / 32)), QK_THREADS, 0, st, (const float*)p.part, blocks_q, blocks, p.d, dw_q, dw_k);
}

// Output rows that are their input's (same address and pitch) or begin elsewhere.
bool in_place_ok(const void* in, int64_t ld_in, const void* out, int64_t ld_out) { return in != out || ld_in == ld_out; }

}  // namespace
}  // namespace rom

using namespace rom;

extern "C" {

int rom_qk_norm_rope(const rom_qk_config* cfg, int32_t rows, const void* q, int64_t ldq, const void* k, int64_t ldk, const float* w_q, const float* w_k, const int32_t* pos,
                     const float* inv_freq, void* q_out, int64_t ldq_out, void* k_out, int64_t ldk_out, void* stream) {
  int rc = check_qk(cfg, rows);
  if (rc != ROM_OK) return rc;
  if (rows == 0) return ROM_OK;
  const rom_qk_config& c = *cfg;
  const size_t esz = c.dtype == ROM_BF16 ? 2 : 4;
  const int wq = c.n_q_heads * c.d_head, wk = c.n_k_heads * c.d_head;
  if (!q || !k || !q_out || !k_out || (c.rot_dim > 0 && (!pos || !inv_freq))) return ROM_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || !aligned4(w_q) || !aligned4(w_k) || !aligned4(pos) || !aligned4(inv_freq)) return ROM_ERR_INVALID_ARG;
  if (!pitch_ok(ldq, wq, esz) || !pitch_ok(ldk, wk, esz) || !pitch_ok(ldq_out, wq, esz) || !pitch_ok(ldk_out, wk, esz)) return ROM_ERR_INVALID_ARG;
  if (!in_place_ok(q, ldq, q_out, ldq_out) || !in_place_ok(k, ldk, k_out, ldk_out) || q_out == k_out || q_out == k || k_out == q) return ROM_ERR_INVALID_ARG;
  if ((rc = check_device()) != ROM_OK) return rc;
  LaunchCounter::count = 0;
  QkArgs p{q, k, nullptr, nullptr, q_out, k_out, ldq, ldk, ldq_out, ldk_out, w_q, w_k, pos, inv_freq, nullptr, rows, c.n_q_heads, c.n_k_heads, c.d_head, c.rot_dim, c.interleaved, c.eps};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return (c.dtype == ROM_BF16 ? launch_forward<__nv_bfloat16>(c, p, st) : launch_forward<float>(c, p, st)) == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

int rom_qk_norm_rope_backward_workspace_size(const rom_qk_config* cfg, int32_t rows, size_t* bytes) {
  const int rc = check_qk(cfg, rows);
  if (rc != ROM_OK) return rc;
  if (!bytes) return ROM_ERR_INVALID_ARG;
  *bytes = sizeof(float) * (size_t)cfg->d_head * 2 * kBwdBlocks;
  return ROM_OK;
}

int rom_qk_norm_rope_backward(const rom_qk_config* cfg, int32_t rows, const void* dq_out, const void* dk_out, const void* q, int64_t ldq, const void* k, int64_t ldk,
                              const float* w_q, const float* w_k, const int32_t* pos, const float* inv_freq, void* dq, int64_t lddq, void* dk, int64_t lddk, float* dw_q,
                              float* dw_k, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_qk(cfg, rows);
  if (rc != ROM_OK) return rc;
  const rom_qk_config& c = *cfg;
  const size_t esz = c.dtype == ROM_BF16 ? 2 : 4;
  const int wq = c.n_q_heads * c.d_head, wk = c.n_k_heads * c.d_head;
  if (!w_q != !dw_q || !w_k != !dw_k || !aligned4(dw_q) || !aligned4(dw_k) || !ws || !aligned16(ws)) return ROM_ERR_INVALID_ARG;
  if (rows > 0) {
    if (!dq_out || !dk_out || !q || !k || !dq || !dk || (c.rot_dim > 0 && (!pos || !inv_freq))) return ROM_ERR_INVALID_ARG;
    const void* ptrs[] = {dq_out, dk_out, q, k, dq, dk};
    for (const void* a : ptrs)
      if (!aligned16(a)) return ROM_ERR_INVALID_ARG;
    if (!aligned4(w_q) || !aligned4(w_k) || !aligned4(pos) || !aligned4(inv_freq)) return ROM_ERR_INVALID_ARG;
    if (!pitch_ok(ldq, wq, esz) || !pitch_ok(ldk, wk, esz) || !pitch_ok(lddq, wq, esz) || !pitch_ok(lddk, wk, esz)) return ROM_ERR_INVALID_ARG;
    for (const void* a : {dq_out, dk_out, q, k})
      if (a == dq || a == dk) return ROM_ERR_INVALID_ARG;
    if (dq == dk) return ROM_ERR_INVALID_ARG;
  }
  if (ws_bytes < sizeof(float) * (size_t)c.d_head * 2 * kBwdBlocks) return ROM_ERR_WORKSPACE;
  if ((rc = check_device()) != ROM_OK) return rc;
  LaunchCounter::count = 0;
  QkArgs p{q, k, dq_out, dk_out, dq, dk, ldq, ldk, lddq, lddk, w_q, w_k, pos, inv_freq, static_cast<float*>(ws), rows, c.n_q_heads, c.n_k_heads, c.d_head, c.rot_dim, c.interleaved, c.eps};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return (c.dtype == ROM_BF16 ? launch_backward<__nv_bfloat16>(c, p, dw_q, dw_k, st) : launch_backward<float>(c, p, dw_q, dw_k, st)) == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

}  // extern "C"
