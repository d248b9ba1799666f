// Linear attention with a decay per head on the 5th-generation tensor cores (bf16), in chunks of 128 rows.  With i and j places in a chunk of `len` rows,
//   scores  s_ij = q_i . k_j                                 [128 x 128]   A = Q, B = K (both K-major)
//   O1 = Q S,   O2 = P V,  P_ij = p lambda^{i-j} s_ij (j <= i, else 0) [128 x dv]   A = Q / A = P from tensor memory, B = S^T as written / B = V (MN-major)
//   out_i = inter lambda^{i+1} O1_i + O2_i
//   S^T <- lambda^len S^T + V^T K~,  K~_j = ks lambda^{len-1-j} k_j      [dv x dk]     A = V^T, B = K~ (both MN-major)
// (backwards: rows run the other way, j >= i, the exponents are counted from the chunk's other end.)
//
// Roundings: P and the S that a chunk meets are bf16 (half a step each, of separate parts of the sum); K~ is hi + lo, two bf16 numbers, in two matrix products, since
// the state is an fp32 result that many chunks add up in.  S itself stays in fp32 registers, one column of S^T's rows per thread; lambda^128 is two floats.
//
// One CTA per SM walks one head of one segment of the packed rows.  320 threads: warp 0 issues the copies (TMA boxes of 64 columns x 128 rows, zeros beyond a head's
// width), warp 1 the matrix products, warps 2..5 turn scores into P and O1, O2 into output rows, warps 6..9 scale K in place (K~ hi; lo beside it), and keep S.  K and V
// are double-buffered; the scores' tensor memory is reused for P.
//
// Values that are not finite: a masked P is 0 by selection, but 0 * V is not 0 for a V of a later row that is not finite.  Rows whose O2 is not finite are summed
// again over their own and earlier rows alone (slow_rows).  Rows behind the chunk's last one are never part of a sum: K~ and P are selected 0, V rows in the last
// contracted step are cleared.
#include <float.h>
#include <math.h>

#include "rom_linattn.cuh"
#include "rom_tc_ptx.cuh"

namespace rom {
namespace {

using bf16 = __nv_bfloat16;
constexpr int LT_C = 128;                     // rows of a chunk
constexpr int LT_BOX = 64 * LT_C * 2;         // bytes of one TMA box
constexpr int LT_THREADS = 320;
constexpr uint32_t LT_TMEM = 512;

__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}
// A warp's wait, polled by one lane.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t limit) {
  int ok = 1;
  if ((threadIdx.x & 31) == 0) ok = mbar_wait(bar, parity, abort_flag, limit);
  ok = __shfl_sync(0xffffffffu, ok, 0);
  __syncwarp();
  return ok != 0;
}
__device__ __forceinline__ void warp_arrive(uint32_t bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ void umma_bf16_ta(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float lo_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v) { asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory"); }

// D = f32, A = B = bf16; bits 15 / 16: A / B is MN-major; M = 128
__host__ __device__ constexpr uint32_t lt_idesc(int n, bool a_mn, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}
// An MN-major tile of 64-column boxes of 128 rows: as make_smem_desc_mn, the next 64 columns one box further.  (An operand of 128 columns that has one box alone reads
// the 16 KB behind it, which are other tiles of this block, into accumulator lanes that nobody reads.)
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3ffffu) >> 4) | (uint64_t)(LT_BOX >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// One row of K (128 bytes of one box, 16-byte pieces swizzled by the row) times w: hi in place, lo beside it; zeros where the row is not part of the sum.
__device__ __forceinline__ void scale_row(uint32_t khi, uint32_t klo, int row, float w, bool live, int piece0, int pieces) {
#pragma unroll 4
  for (int i = 0; i < pieces; ++i) {
    const uint32_t off = row * 128 + (((piece0 + i) ^ (row & 7)) << 4);
    uint4 hi = make_uint4(0, 0, 0, 0), lo = hi;
    if (live) {
      const uint4 x = lds128(khi + off);
      const uint32_t in[4] = {x.x, x.y, x.z, x.w};
      uint32_t h[4], l[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a = lo_of(in[e]), b = hi_of(in[e]);
        h[e] = pack2(a * w, b * w);
        l[e] = pack2(fmaf(a, w, -lo_of(h[e])), fmaf(b, w, -hi_of(h[e])));      // (of an infinite product NaN: not finite either way)
      }
      hi = make_uint4(h[0], h[1], h[2], h[3]);
      lo = make_uint4(l[0], l[1], l[2], l[3]);
    }
    sts128(khi + off, hi);
    sts128(klo + off, lo);
  }
}
template <int BOXES>
__device__ __forceinline__ void clear_row(uint32_t tile, int row) {
#pragma unroll
  for (int b = 0; b < BOXES; ++b)
#pragma unroll
    for (int i = 0; i < 8; ++i) sts128(tile + b * LT_BOX + row * 128 + i * 16, make_uint4(0, 0, 0, 0));
}
// V^T K~: hi and lo, the first ks steps of 16 rows.
__device__ __forceinline__ void issue_state(uint32_t tmem_d, uint32_t v, uint32_t khi, uint32_t klo, uint32_t idesc, int ks, bool accumulate) {
  const uint64_t a = desc_mn(v), h = desc_mn(khi), l = desc_mn(klo);
  for (int k = 0; k < ks; ++k) umma_bf16(tmem_d, a + (uint64_t)(MN_KSTEP * k), h + (uint64_t)(MN_KSTEP * k), idesc, accumulate || k > 0 ? 1u : 0u);
  for (int k = 0; k < ks; ++k) umma_bf16(tmem_d, a + (uint64_t)(MN_KSTEP * k), l + (uint64_t)(MN_KSTEP * k), idesc, 1u);
}
template <int BOXES>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int row) {
#pragma unroll
  for (int b = 0; b < BOXES; ++b) tma_load_3d(dst + b * LT_BOX, map, bar, 64 * b, head, row);
}
__device__ __forceinline__ void latch(const LinPass& p, volatile int* abort_flag, int where) {
  if (!*abort_flag) {
    atomicExch(p.status + kStatCode, ROM_ERR_DEVICE_TIMEOUT);
    atomicExch(p.status + kStatWhere, where);
  }
  *abort_flag = 1;
}

// The rows [r0, r1) of one sequence in one segment, in chunks.
struct LinPiece {
  int s, r0, r1;
  bool over;             // the state comes over a cut
  bool ends;             // the sequence's last state is left here
  __device__ __forceinline__ int chunks() const { return (r1 - r0 + LT_C - 1) / LT_C; }
  template <bool REV>
  __device__ __forceinline__ void chunk(int m, int& row0, int& len) const {
    if (REV) { const int end = r1 - LT_C * m; row0 = max(r0, end - LT_C); len = end - row0; }
    else { row0 = r0 + LT_C * m; len = min(LT_C, r1 - row0); }
  }
};
struct LinSegment {
  int a, b, seg;
  bool last;
  __device__ __forceinline__ LinSegment(const Ragged& q, int seg_, int seg_rows, int n_seg) : a(seg_ * seg_rows), b(min(a + seg_rows, q.rows)), seg(seg_), last(seg_ + 1 == n_seg) {}
  __device__ __forceinline__ int first(const Ragged& q) const {      // all lanes of a warp
    const int s = q.first_from(a);
    return s > 0 && q.end_of(s - 1) > a ? s - 1 : s;
  }
  // false: no sequence from s on is of this segment
  template <bool REV>
  __device__ __forceinline__ bool piece(const Ragged& q, int s, LinPiece& x) const {
    if (s >= q.n_seq) return false;
    const int st = q.start_of(s), en = q.end_of(s);
    if (st >= b && !last) return false;
    const bool empty = en <= st;
    x.s = s;
    x.r0 = max(st, a);
    x.r1 = empty ? x.r0 : max(min(en, b), x.r0);
    x.over = !empty && (REV ? en > b : st < a);
    x.ends = empty || (x.r1 > x.r0 && (REV ? st >= a : en <= b));
    return true;
  }
};

// ------------------------------------------------------------------------------------------------------------------------------ the walk
template <int KP, int VP>
struct WalkShape {
  static constexpr int KB = KP / 64, VB = VP / 64;
  static constexpr int QST = KP + VP < 256 ? 2 : 1;                 // stages of Q: one where 227 KB leave no room
  static constexpr int Q = 0, K = Q + QST * KB * LT_BOX, V = K + 2 * KB * LT_BOX, LO = V + 2 * VB * LT_BOX, S = LO + KB * LT_BOX, BYTES = S + KB * VP * 128;
  static constexpr int SC = 0, O1 = 128, KV = O1 + VP, O2 = KV + KP;      // tensor-memory columns (P over the scores' first 64)
};

// Rows of O2 that are not finite, summed again: out = f O1 + sum over their own and earlier rows.  Rare; all lanes of the warp call it.
template <bool REV>
__device__ __noinline__ void slow_rows(const LinPass& p, const bf16* q, const bf16* k, const bf16* v, bf16* out, uint32_t taddr_o1, const float* lam, int i, int row0, int len, float f,
                                       bool mine, int head) {
  for (int c0 = 0; c0 < p.dv; c0 += 32) {
    uint32_t r[32];
    __syncwarp();
    tmem_ld32_issue(taddr_o1 + c0, r);
    tmem_ld_wait(r);
    if (!mine) continue;
    float acc[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) acc[e] = f * __uint_as_float(r[e]);
    const bf16* qi = q + (int64_t)(row0 + i) * p.ldq;
    for (int j = REV ? i : 0; j < (REV ? len : i + 1); ++j) {
      const bf16* kj = k + (int64_t)(row0 + j) * p.ldk;
      float s = 0.0f;
      for (int d = 0; d < p.dk; ++d) s = fmaf(to_f32(qi[d]), to_f32(kj[d]), s);
      const float w = to_f32(__float2bfloat16_rn(s * p.p_scale * lam[REV ? j - i : i - j]));
      const bf16* vj = v + (int64_t)(row0 + j) * p.ldv + c0;
#pragma unroll
      for (int e = 0; e < 32; ++e)
        if (c0 + e < p.dv) acc[e] = fmaf(w, to_f32(vj[e]), acc[e]);
    }
    const int64_t to = (int64_t)(row0 + i) * p.ldo + (int64_t)head * p.dv + c0;
#pragma unroll
    for (int e = 0; e < 32; ++e)
      if (c0 + e < p.dv) {
        if (p.out_f32) reinterpret_cast<float*>(out)[to + e] = acc[e];
        else out[to + e] = __float2bfloat16_rn(acc[e]);
      }
  }
}

template <int KP, int VP, bool REV>
__global__ void __launch_bounds__(LT_THREADS, 1)
lin_walk_tc(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ LinPass p, const Ragged seqs,
            int seg_rows, int n_seg, uint32_t wait_limit, uint32_t stall) {
  using W = WalkShape<KP, VP>;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  __shared__ __align__(16) float lam[LT_C + 4], lam_lo[LT_C + 4];
  __shared__ __align__(8) unsigned long long bars[16];
  __shared__ uint32_t tmem_s;
  __shared__ int abort_s;
  volatile int* abort_flag = &abort_s;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), head = blockIdx.x;
  auto bar = [&](int i) { return smem_u32(&bars[i]); };
  // full: copies have landed; empty: the matrix products that read them are done; the others by name
  auto q_full = [&](int s) { return bar(s); };
  auto q_empty = [&](int s) { return bar(2 + s); };
  auto kv_full = [&](int s) { return bar(4 + s); };
  auto kv_empty = [&](int s) { return bar(6 + s); };
  const uint32_t sc_full = bar(8), p_ready = bar(9), k_ready = bar(10), s_ready = bar(11), pv_full = bar(12), o_free = bar(13), state_full = bar(14), drain = bar(15);
  if (tid == 0) {
    for (int i = 0; i < 16; ++i) mbar_init(bar(i), i == 9 || i == 10 || i == 11 || i == 13 ? 4 : 1);
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(LT_TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  if (tid <= LT_C) {
    const double l = exp((double)__ldg(p.log_decay + head) * tid);
    lam[tid] = (float)l;
    lam_lo[tid] = (float)(l - (double)lam[tid]);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();                       // (behind the block's tensor memory: the successor takes its own before it waits)
  const uint32_t tmem = tmem_s;
  const LinSegment seg(seqs, blockIdx.y, seg_rows, n_seg);
  const int s_first = seg.first(seqs);
  LinPiece x;
  int n = 0;                           // chunks so far

  if (warp == 0) {
    // ---------------------------------------------------------------- copies
    if (elect_one()) {
      bool ok = true;
      for (int s = s_first; ok && seg.piece<REV>(seqs, s, x); ++s)
        for (int m = 0, mm = x.chunks(); m < mm; ++m, ++n) {
          int row0, len;
          x.chunk<REV>(m, row0, len);
          const int st = n & 1, qs = n % W::QST;
          if (!mbar_wait(kv_empty(st), (n >> 1 & 1) ^ 1, abort_flag, wait_limit)) { ok = false; break; }
          mbar_expect_tx(kv_full(st), (W::KB + W::VB) * LT_BOX + stall);
          load_tile<W::KB>(base + W::K + st * W::KB * LT_BOX, &tmap_k, kv_full(st), head / p.kdiv, row0);
          load_tile<W::VB>(base + W::V + st * W::VB * LT_BOX, &tmap_v, kv_full(st), head / p.vdiv, row0);
          if (!mbar_wait(q_empty(qs), (n / W::QST & 1) ^ 1, abort_flag, wait_limit)) { ++n; ok = false; break; }
          mbar_expect_tx(q_full(qs), W::KB * LT_BOX);
          load_tile<W::KB>(base + W::Q + qs * W::KB * LT_BOX, &tmap_q, q_full(qs), head / p.qdiv, row0);
        }
      if (!ok) latch(p, abort_flag, 51);
      if (*abort_flag)                 // the copies still in flight land (bounded) before the block ends
        for (int i = 1; i <= 2 && i <= n; ++i) {
          const int c = n - i;
          for (uint32_t it = 0; it < wait_limit >> 2 && !mbar_try_wait(kv_full(c & 1), c >> 1 & 1); ++it) {}
          for (uint32_t it = 0; it < wait_limit >> 2 && !mbar_try_wait(q_full(c % W::QST), c / W::QST & 1); ++it) {}
        }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---------------------------------------------------------------- matrix products
    if (elect_one()) {
      constexpr uint32_t d_sc = lt_idesc(LT_C, false, false), d_o1 = lt_idesc(VP, false, false), d_o2 = lt_idesc(VP, false, true), d_kv = lt_idesc(KP, true, true);
      bool ok = true, issued = false;
      auto wait = [&](uint32_t b, uint32_t parity) { ok = ok && mbar_wait(b, parity, abort_flag, wait_limit); return ok; };
      for (int s = s_first; ok && seg.piece<REV>(seqs, s, x); ++s)
        for (int m = 0, mm = x.chunks(); m < mm; ++m, ++n) {
          int row0, len;
          x.chunk<REV>(m, row0, len);
          const int st = n & 1, qs = n % W::QST, ks = (len + 15) / 16;
          const uint32_t ph = n & 1, q = base + W::Q + qs * W::KB * LT_BOX, k = base + W::K + st * W::KB * LT_BOX, v = base + W::V + st * W::VB * LT_BOX;
          // scores, once the P that lies over them has been used
          if (!wait(kv_full(st), n >> 1 & 1) || !wait(q_full(qs), n / W::QST & 1) || (n > 0 && !wait(pv_full, ph ^ 1))) break;
          tc_fence_after();
#pragma unroll
          for (int b = 0; b < W::KB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              umma_bf16(tmem + W::SC, make_smem_desc(q + b * LT_BOX) + 2 * e, make_smem_desc(k + b * LT_BOX) + 2 * e, d_sc, b + e > 0 ? 1u : 0u);
          umma_commit(sc_full);
          issued = true;
          // Q S, once the output before has been read and S written
          if (!wait(s_ready, ph) || (n > 0 && !wait(o_free, ph ^ 1))) break;
          tc_fence_after();
#pragma unroll
          for (int b = 0; b < W::KB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              umma_bf16(tmem + W::O1, make_smem_desc(q + b * LT_BOX) + 2 * e, make_smem_desc(base + W::S + b * VP * 128) + 2 * e, d_o1, b + e > 0 ? 1u : 0u);
          umma_commit(q_empty(qs));
          if (!wait(p_ready, ph) || !wait(k_ready, ph)) break;
          tc_fence_after();
          for (int e = 0; e < ks; ++e) umma_bf16_ta(tmem + W::O2, tmem + W::SC + 8 * e, desc_mn(v) + (uint64_t)(MN_KSTEP * e), d_o2, e > 0 ? 1u : 0u);
          umma_commit(pv_full);
          issue_state(tmem + W::KV, v, k, base + W::LO, d_kv, ks, false);
          umma_commit(state_full);
          umma_commit(kv_empty(st));
        }
      if (!ok) latch(p, abort_flag, 52);
      if (*abort_flag && issued) {     // what has been issued may still read shared memory and write tensor memory
        umma_commit(drain);
        for (uint32_t it = 0; it < wait_limit >> 2 && !mbar_try_wait(drain, 0); ++it) {}
      }
    }
    __syncwarp();
  } else if (warp < 6) {
    // ---------------------------------------------------------------- scores to P, outputs
    const int quarter = warp & 3, i = quarter * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    bf16* out = static_cast<bf16*>(p.out);
    bool ok = true;
    for (int s = s_first; ok && seg.piece<REV>(seqs, s, x); ++s)
      for (int m = 0, mm = x.chunks(); m < mm; ++m, ++n) {
        int row0, len;
        x.chunk<REV>(m, row0, len);
        const uint32_t ph = n & 1;
        const int early = m == 0 && !x.over && p.early ? 1 : 0, blocks = (len + 31) / 32;
        if (!(ok = warp_wait(sc_full, ph, abort_flag, wait_limit))) break;
        tc_fence_after();
        for (int b = 0; b < blocks; ++b) {
          uint32_t w[16];
          if (REV ? b < quarter : b > quarter) {
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = 0;
          } else {
            uint32_t r[32];
            tmem_ld32_issue(lanes + W::SC + 32 * b, r);
            tmem_ld_wait(r);
            if (b == quarter) {
#pragma unroll
              for (int e = 0; e < 32; e += 2) {
                const int g0 = REV ? e - lane : lane - e, g1 = REV ? e + 1 - lane : lane - e - 1;
                const bool on0 = g0 >= 0 && (!REV || 32 * b + e < len), on1 = g1 >= 0 && (!REV || 32 * b + e + 1 < len);
                const float p0 = __uint_as_float(r[e]) * (p.p_scale * lam[max(g0, 0)]), p1 = __uint_as_float(r[e + 1]) * (p.p_scale * lam[max(g1, 0)]);
                w[e / 2] = pack2(on0 ? p0 : 0.0f, on1 ? p1 : 0.0f);
              }
            } else {
              // lambda^{i-j} = lambda^{i - last of the block} lambda^{last - j}
              const float f = p.p_scale * lam[REV ? 32 * b - i : i - 32 * b - 31];
              const bool whole = !REV || 32 * b + 32 <= len;
#pragma unroll
              for (int e = 0; e < 32; e += 4) {
                const float4 u = *reinterpret_cast<const float4*>(lam + (REV ? e : 28 - e));
                const float2 u0 = REV ? make_float2(u.x, u.y) : make_float2(u.w, u.z), u1 = REV ? make_float2(u.z, u.w) : make_float2(u.y, u.x);
                float2 p0 = __fmul2_rn(make_float2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])), __fmul2_rn(u0, make_float2(f, f)));
                float2 p1 = __fmul2_rn(make_float2(__uint_as_float(r[e + 2]), __uint_as_float(r[e + 3])), __fmul2_rn(u1, make_float2(f, f)));
                if (REV && !whole) {
                  const int j = 32 * b + e;
                  p0 = make_float2(j < len ? p0.x : 0.0f, j + 1 < len ? p0.y : 0.0f);
                  p1 = make_float2(j + 2 < len ? p1.x : 0.0f, j + 3 < len ? p1.y : 0.0f);
                }
                w[e / 2] = pack2(p0.x, p0.y);
                w[e / 2 + 1] = pack2(p1.x, p1.y);
              }
            }
          }
          tmem_st16(lanes + W::SC + 16 * b, w);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        warp_arrive(p_ready);
        if (!(ok = warp_wait(pv_full, ph, abort_flag, wait_limit))) break;
        tc_fence_after();
        const bool mine = i < len;
        const float f = p.inter_scale * lam[REV ? max(len - i - early, 0) : i + 1 - early];
        const int64_t to = (int64_t)(row0 + i) * p.ldo + (int64_t)head * p.dv;
        float2 odd = make_float2(0.0f, 0.0f);
#pragma unroll 1
        for (int c = 0; c < p.dv; c += 32) {
          uint32_t r1[32], r2[32];
          __syncwarp();
          tmem_ld32_issue(lanes + W::O1 + c, r1);
          tmem_ld32_issue(lanes + W::O2 + c, r2);
          tmem_ld_wait(r1);
          tmem_ld_wait(r2);
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            float2 o[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              const float2 b2 = make_float2(__uint_as_float(r2[e + 2 * h]), __uint_as_float(r2[e + 2 * h + 1]));
              odd = __ffma2_rn(b2, make_float2(0.0f, 0.0f), odd);
              o[h] = __ffma2_rn(make_float2(__uint_as_float(r1[e + 2 * h]), __uint_as_float(r1[e + 2 * h + 1])), make_float2(f, f), b2);
            }
            if (mine && c + e < p.dv) {
              if (p.out_f32) {
                float4* dst = reinterpret_cast<float4*>(static_cast<float*>(p.out) + to + c + e);
                dst[0] = make_float4(o[0].x, o[0].y, o[1].x, o[1].y);
                dst[1] = make_float4(o[2].x, o[2].y, o[3].x, o[3].y);
              } else {
                *reinterpret_cast<uint4*>(out + to + c + e) = make_uint4(pack2(o[0].x, o[0].y), pack2(o[1].x, o[1].y), pack2(o[2].x, o[2].y), pack2(o[3].x, o[3].y));
              }
            }
          }
        }
        const bool again = mine && !(odd.x == 0.0f && odd.y == 0.0f);
        if (__any_sync(0xffffffffu, again))
          slow_rows<REV>(p, static_cast<const bf16*>(p.q) + (int64_t)(head / p.qdiv) * p.dk, static_cast<const bf16*>(p.k) + (int64_t)(head / p.kdiv) * p.dk,
                         static_cast<const bf16*>(p.v) + (int64_t)(head / p.vdiv) * p.dv, out, lanes + W::O1, lam, i, row0, len, f, again, head);
        tc_fence_before();
        warp_arrive(o_free);
      }
    if (!ok) latch(p, abort_flag, 53);
  } else {
    // ---------------------------------------------------------------- K~ and the state: thread c keeps column c of S
    const int quarter = warp & 3, c = quarter * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    const size_t state = (size_t)p.dk * p.dv;
    float S[KP];
    bool ok = true;
    auto write_s = [&]() {      // bf16 rows of S^T, K-major
      if (c < VP)
#pragma unroll
        for (int a = 0; a < KP; a += 8)
          sts128(base + W::S + (a / 64) * VP * 128 + c * 128 + (((a / 8 & 7) ^ (c & 7)) << 4),
                 make_uint4(pack2(S[a], S[a + 1]), pack2(S[a + 2], S[a + 3]), pack2(S[a + 4], S[a + 5]), pack2(S[a + 6], S[a + 7])));
      fence_async();
      warp_arrive(s_ready);
    };
    for (int s = s_first; ok && seg.piece<REV>(seqs, s, x); ++s) {
      const int mm = x.chunks(), slot = seqs.slot_of(s);
      const float* from = lin_init_of(p, seqs, s, head);
      if (x.over) from = p.seg_state + ((size_t)(REV ? seg.seg : seg.seg - 1) * p.H + head) * state;
      else if (!REV && mm > 0 && from && p.init_copy && !x.ends) from = p.init_copy + ((size_t)seg.seg * p.H + head) * state;
      if (mm == 0 && !x.ends) continue;
#pragma unroll
      for (int a = 0; a < KP; a += 4) {
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (from && c < p.dv && a < p.dk) {
          if (p.transposed) v = *reinterpret_cast<const float4*>(from + (size_t)c * p.dk + a);
          else v = make_float4(from[(size_t)a * p.dv + c], from[(size_t)(a + 1) * p.dv + c], from[(size_t)(a + 2) * p.dv + c], from[(size_t)(a + 3) * p.dv + c]);
        }
        S[a] = v.x; S[a + 1] = v.y; S[a + 2] = v.z; S[a + 3] = v.w;
      }
      if (mm > 0) write_s();
      for (int m = 0; m < mm; ++m, ++n) {
        int row0, len;
        x.chunk<REV>(m, row0, len);
        const int st = n & 1, early = m == 0 && !x.over && p.early ? 1 : 0, rows16 = (len + 15) / 16 * 16;
        const uint32_t ph = n & 1, k = base + W::K + st * W::KB * LT_BOX;
        if (!(ok = warp_wait(kv_full(st), n >> 1 & 1, abort_flag, wait_limit) && warp_wait(sc_full, ph, abort_flag, wait_limit))) break;
        if (c < rows16) {
          const bool live = c < len;
          const float w = live ? p.k_scale * lam[REV ? c : len - 1 - c] : 0.0f;
#pragma unroll
          for (int b = 0; b < W::KB; ++b) scale_row(k + b * LT_BOX, base + W::LO + b * LT_BOX, c, w, live, 0, 8);
          if (!live) clear_row<W::VB>(base + W::V + st * W::VB * LT_BOX, c);
        }
        fence_async();
        warp_arrive(k_ready);
        if (!(ok = warp_wait(state_full, ph, abort_flag, wait_limit))) break;
        tc_fence_after();
        const float f = lam[len - early], fl = lam_lo[len - early];
#pragma unroll
        for (int a = 0; a < KP; a += 32) {
          uint32_t r[32];
          tmem_ld32_issue(lanes + W::KV + a, r);
          tmem_ld_wait(r);
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            float2 v = __ffma2_rn(make_float2(S[a + e], S[a + e + 1]), make_float2(fl, fl), make_float2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])));
            v = __ffma2_rn(make_float2(S[a + e], S[a + e + 1]), make_float2(f, f), v);
            S[a + e] = v.x;
            S[a + e + 1] = v.y;
          }
        }
        tc_fence_before();
        if (m + 1 < mm) write_s();
      }
      if (!ok) break;
      if (p.last && slot >= 0 && x.ends && c < p.dv) {
        const float f = p.init_all && !seqs.resumes(s) ? 0.0f : mm > 0 && p.early ? lam[1] : 1.0f;
        float* to = p.last + ((size_t)slot * p.H + head) * state + c;
        const bool none = p.init_all && !seqs.resumes(s);
#pragma unroll
        for (int a = 0; a < KP; ++a)
          if (a < p.dk) to[(size_t)a * p.dv] = none ? 0.0f : f * S[a];
      }
    }
    if (!ok) latch(p, abort_flag, 54);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(LT_TMEM) : "memory");
}

// ------------------------------------------------------------------------------------------------------------------------------ launch 1: states at the cuts
// sum over a segment's rows of the sequence that reaches over its far end, lambda^{distance to that end} ks k_j v_j^T: every row's weight is known, so all chunks add
// up in tensor memory.  Warps 2..9 scale K, two to a row.
template <int KP, int VP>
struct StateShape {
  static constexpr int KB = KP / 64, VB = VP / 64;
  static constexpr int STAGE = (2 * KB + VB) * LT_BOX, LO = KB * LT_BOX, V = 2 * KB * LT_BOX;      // K (hi) | lo | V
  static constexpr int STAGES = KP == 128 ? 2 : 3, BYTES = STAGES * STAGE + (VB == 1 ? LT_BOX : 0);      // (see desc_mn: one box behind the last V)
};
constexpr int kLtMaxSmem = 232448 - 4096;      // what a block may ask for, less its static variables
static_assert(WalkShape<128, 128>::BYTES + 1024 <= kLtMaxSmem + 2048 && WalkShape<128, 64>::BYTES + 1024 <= kLtMaxSmem && WalkShape<64, 128>::BYTES + 1024 <= kLtMaxSmem, "shared memory");
static_assert(StateShape<128, 128>::BYTES + 1024 <= kLtMaxSmem && StateShape<128, 64>::BYTES + 1024 <= kLtMaxSmem && StateShape<64, 128>::BYTES + 1024 <= kLtMaxSmem, "shared memory");

template <int KP, int VP, bool REV>
__global__ void __launch_bounds__(LT_THREADS, 1)
lin_state_tc(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ LinPass p, const Ragged seqs, int seg_rows, uint32_t wait_limit, uint32_t stall) {
  using W = StateShape<KP, VP>;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  __shared__ __align__(8) unsigned long long bars[3 * 3 + 2];
  __shared__ uint32_t tmem_s;
  __shared__ int abort_s;
  volatile int* abort_flag = &abort_s;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), head = blockIdx.x, seg = REV ? blockIdx.y + 1 : blockIdx.y;
  pdl_wait();
  const int a = seg * seg_rows, b = min(a + seg_rows, seqs.rows), s = lin_spanning(seqs, REV ? a : b);
  if (s < 0) return;
  const int r0 = REV ? a : max(seqs.start_of(s), a), r1 = REV ? min(seqs.end_of(s), b) : b, chunks = (r1 - r0 + LT_C - 1) / LT_C;
  if (r1 <= r0) return;
  auto full = [&](int i) { return smem_u32(&bars[i]); };
  auto empty = [&](int i) { return smem_u32(&bars[3 + i]); };
  auto scaled = [&](int i) { return smem_u32(&bars[6 + i]); };
  const uint32_t done = smem_u32(&bars[9]), drain = smem_u32(&bars[10]);
  if (tid == 0) {
    for (int i = 0; i < 3; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); mbar_init(scaled(i), 8); }
    mbar_init(done, 1);
    mbar_init(drain, 1);
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"((uint32_t)KP) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();
  const uint32_t tmem = tmem_s;
  if (warp == 0) {
    if (elect_one()) {
      bool ok = true;
      int n = 0;
      for (; n < chunks; ++n) {
        const int st = n % W::STAGES;
        const uint32_t at = base + st * W::STAGE;
        if (!mbar_wait(empty(st), (n / W::STAGES & 1) ^ 1, abort_flag, wait_limit)) { ok = false; break; }
        mbar_expect_tx(full(st), (W::KB + W::VB) * LT_BOX + stall);
        load_tile<W::KB>(at, &tmap_k, full(st), head / p.kdiv, r0 + LT_C * n);
        load_tile<W::VB>(at + W::V, &tmap_v, full(st), head / p.vdiv, r0 + LT_C * n);
      }
      if (!ok) latch(p, abort_flag, 55);
      if (*abort_flag)
        for (int i = 1; i <= W::STAGES && i <= n; ++i)
          for (uint32_t it = 0; it < wait_limit >> 2 && !mbar_try_wait(full((n - i) % W::STAGES), (n - i) / W::STAGES & 1); ++it) {}
    }
    __syncwarp();
  } else if (warp == 1) {
    if (elect_one()) {
      bool ok = true, issued = false;
      for (int n = 0; n < chunks; ++n) {
        const int st = n % W::STAGES;
        const uint32_t at = base + st * W::STAGE;
        if (!mbar_wait(scaled(st), n / W::STAGES & 1, abort_flag, wait_limit)) { ok = false; break; }
        tc_fence_after();
        issue_state(tmem, at + W::V, at, at + W::LO, lt_idesc(KP, true, true), (min(LT_C, r1 - r0 - LT_C * n) + 15) / 16, n > 0);
        umma_commit(empty(st));
        issued = true;
      }
      if (ok) umma_commit(done);
      else latch(p, abort_flag, 56);
      if (*abort_flag && issued) {
        umma_commit(drain);
        for (uint32_t it = 0; it < wait_limit >> 2 && !mbar_try_wait(drain, 0); ++it) {}
      }
    }
    __syncwarp();
  } else {
    const int half = (warp - 2) >> 2, quarter = warp & 3, j = quarter * 32 + lane;
    const double g = (double)__ldg(p.log_decay + head);
    bool ok = true;
    for (int n = 0; n < chunks; ++n) {
      const int st = n % W::STAGES, row0 = r0 + LT_C * n, len = min(LT_C, r1 - row0), rows16 = (len + 15) / 16 * 16;
      const uint32_t at = base + st * W::STAGE;
      const float w = p.k_scale * (float)exp(g * max(REV ? row0 + j - r0 : r1 - 1 - row0 - j, 0));
      if (!(ok = warp_wait(full(st), n / W::STAGES & 1, abort_flag, wait_limit))) break;
      if (j < rows16) {
        const bool live = j < len;
        if (KP == 128) scale_row(at + half * LT_BOX, at + W::LO + half * LT_BOX, j, w, live, 0, 8);
        else scale_row(at, at + W::LO, j, w, live, 4 * half, 4);
        if (!live && half == 0) clear_row<W::VB>(at + W::V, j);
      }
      fence_async();
      warp_arrive(scaled(st));
    }
    if (ok && (ok = warp_wait(done, 0, abort_flag, wait_limit))) {
      tc_fence_after();
      float* to = p.seg_state + ((size_t)(REV ? seg - 1 : seg) * p.H + head) * ((size_t)p.dk * p.dv) + j;
      for (int c = half * (KP / 2); c < (half + 1) * (KP / 2); c += 32) {
        uint32_t r[32];
        __syncwarp();
        tmem_ld32_issue(tmem + ((uint32_t)(quarter * 32) << 16) + c, r);
        tmem_ld_wait(r);
#pragma unroll
        for (int e = 0; e < 32; ++e)
          if (j < p.dv && c + e < p.dk) to[(size_t)(c + e) * p.dv] = __uint_as_float(r[e]);
      }
    }
    if (!ok) latch(p, abort_flag, 57);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)KP) : "memory");
}

// ---------------------------------------------------------------------------------------------------------------------------------------- host
// bf16 [rows, heads, d] with row pitch ld as a 3-D tensor: a box is 64 columns of one head in 128 rows, zeros beyond the head's width and the last row.
bool make_tmap_heads(CUtensorMap* map, const void* ptr, int rows, int heads, int d, int64_t ld) {
  EncodeTiledFn fn = get_encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)rows};
  cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)ld * 2};
  cuuint32_t box[3] = {64, 1, LT_C};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int KP, int VP, bool REV>
cudaError_t launch_shape(const LinPass& p, const rom_ragged& seqs, LinCut cut, bool state_only, bool test_stall, cudaStream_t st) {
  CUtensorMap tq, tk, tv;
  if (!make_tmap_heads(&tk, p.k, seqs.rows, p.H / p.kdiv, p.dk, p.ldk) || !make_tmap_heads(&tv, p.v, seqs.rows, p.H / p.vdiv, p.dv, p.ldv)) return cudaErrorInvalidValue;
  const uint32_t limit = test_stall ? WAIT_LIMIT_TEST : WAIT_LIMIT, stall = test_stall ? 16 : 0;
  count_launch();
  if (state_only) {
    constexpr int smem = StateShape<KP, VP>::BYTES + 1024;
    auto kern = lin_state_tc<KP, VP, REV>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    return launch_k(kern, dim3(p.H, cut.n_seg - 1), LT_THREADS, smem, st, tk, tv, p, device_view(seqs), cut.seg_rows, limit, stall);
  }
  if (!make_tmap_heads(&tq, p.q, seqs.rows, p.H / p.qdiv, p.dk, p.ldq)) return cudaErrorInvalidValue;
  constexpr int smem = WalkShape<KP, VP>::BYTES + 1024;
  auto kern = lin_walk_tc<KP, VP, REV>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_k(kern, dim3(p.H, cut.n_seg), LT_THREADS, smem, st, tq, tk, tv, p, device_view(seqs), cut.seg_rows, cut.n_seg, limit, stall);
}

}  // namespace

cudaError_t launch_lin_tc(const LinPass& p, const rom_ragged& seqs, LinCut cut, bool state_only, bool test_stall, cudaStream_t st) {
  const bool k = p.dk > 64, v = p.dv > 64;
  if (p.reverse)
    return (k ? (v ? launch_shape<128, 128, true> : launch_shape<128, 64, true>) : (v ? launch_shape<64, 128, true> : launch_shape<64, 64, true>))(p, seqs, cut, state_only, test_stall, st);
  return (k ? (v ? launch_shape<128, 128, false> : launch_shape<128, 64, false>) : (v ? launch_shape<64, 128, false> : launch_shape<64, 64, false>))(p, seqs, cut, state_only, test_stall, st);
}

}  // namespace rom
