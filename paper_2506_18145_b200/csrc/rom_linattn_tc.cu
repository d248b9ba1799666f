// Linear attention with a decay per head on the 5th-generation tensor cores (bf16), in chunks of 128 rows.  With i and j places in a chunk of `len` rows,
//   scores  s_ij = q_i . k_j                                 [128 x 128]   A = Q, B = K (both K-major)
//   O1 = Q S,   O2 = P V,  P_ij = p lambda^{i-j} s_ij (j <= i, else 0) [128 x dv]   A = Q / A = P from tensor memory, B = S^T as written / B = V (MN-major)
//   out_i = inter lambda^{i+1} O1_i + O2_i
//   S^T <- lambda^len S^T + V^T K~,  K~_j = ks lambda^{len-1-j} k_j      [dv x dk]     A = V^T, B = K~ (both MN-major)
// (backwards: rows run the other way, j >= i, the exponents are counted from the chunk's other end.)
//
// Roundings: P and the S that a chunk meets are the sum of two bf16 numbers each, in two matrix products, which leaves out less than 2^-15 of a number: as one bf16 number each
// they made outputs 2.35e-3 of their norm off 64 bits, where the outputs' own rounding makes 1.66e-3.  K~ is the sum of three bf16 numbers, in three matrix products: all 24 bits of
// the fp32 product, since the state is an fp32 result that many chunks add up in (two left 4.9e-6 of its norm where fp32 sums leave 2e-7; 16384 rows of 32 heads of
// 128 take 211 us with three, 199 with two).
// Two where the state is no result but only read in two parts by dq or dk.  S itself stays in fp32 registers, one column of S^T's rows per thread; lambda^128 is two floats.
//
// One CTA per SM walks one run of chunks.  640 threads: warp 0 issues the copies (TMA boxes of 64 columns x 128 rows, zeros beyond a head's
// width), warp 1 the matrix products, warps 4..11 turn scores into P and O1, O2 into output rows, warps 12..19 scale K in place (K~'s first part; the others beside it), and keep S; two
// warps share each 32-lane quarter of tensor memory and take half of the columns each.  The scores' tensor memory is reused for P.
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
constexpr int LT_WALK_THREADS = 640, LT_SCALERS = 16, LT_STATE_THREADS = 64 + 32 * LT_SCALERS;
// Registers of the walk's threads: 640 x 96 at launch; the copies' and products' warps give theirs to those that make P and keep S: 128 x 48 + 256 x 104 + 256 x 112 =
// 640 x 96.
constexpr int LT_FEW = 48, LT_P = 104, LT_MANY = 112;
template <int N> __device__ __forceinline__ void registers_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void registers_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
constexpr uint32_t LT_TMEM = 512;

__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}
// A warp's wait; the outcome is the same in all lanes.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t limit) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, limit));
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
__device__ __forceinline__ void tmem_ld16_issue(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
                 "=r"(r[14]), "=r"(r[15])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld16_wait(uint32_t (&r)[16]) {      // (the registers pass through: nothing that reads them moves ahead)
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]),
                 "+r"(r[14]), "+r"(r[15])
               :: "memory");
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
// An MN-major tile of 64-column boxes: as make_smem_desc_mn, the next 64 columns one box further.  (An operand of 128 columns that has one box alone reads
// the box behind it, which is other tiles of this block, into accumulator lanes that nobody reads.)
template <int BOX>
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3ffffu) >> 4) | (uint64_t)(BOX >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

__device__ __forceinline__ float ld_state(const float* p) { float v; asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p)); return v; }
__device__ __forceinline__ float4 ld_state4(const float* p) {
  float4 v;
  asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p));
  return v;
}
// The upper halves of two fp32 numbers: bf16 numbers cut off, so that what is left of a number is exact, and 24 bits are three of them.
__device__ __forceinline__ uint32_t uppers(float2 x) { return __byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x7632); }
__device__ __forceinline__ float2 less_upper(float2 x) {
  return __ffma2_rn(make_float2(hi_of(__float_as_uint(x.x)), hi_of(__float_as_uint(x.y))), make_float2(-1.0f, -1.0f), x);      // (of an infinite number NaN: not finite either way)
}
// Two numbers as the sums of two bf16 numbers each.
__device__ __forceinline__ void halves(float2 x, uint32_t& first, uint32_t& second) {
  const float2 rest = less_upper(x);
  first = uppers(x);
  second = pack2(rest.x, rest.y);
}
// Part of one row of K (16-byte pieces of a 128-byte row of one box, swizzled by the row) times w: the first bf16 part in place, the second beside it, and the third where all of
// the product's bits are asked for; zeros where the row is not part of the sum.  Some pieces at a time: one after the other, a piece's load, conversions and stores took 230 cycles.
template <int AT_ONCE, bool THIRD>
__device__ __forceinline__ void scale_row(uint32_t khi, uint32_t klo, uint32_t kll, int row, float w, bool live, int piece0, int pieces) {
  const float2 ww = make_float2(w, w);
#pragma unroll 1
  for (int i = 0; i < pieces; i += AT_ONCE) {
    uint4 x[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      x[u] = lds128(khi + row * 128 + (((piece0 + i + u) ^ (row & 7)) << 4));
      if (!live) x[u] = make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const uint32_t off = row * 128 + (((piece0 + i + u) ^ (row & 7)) << 4), in[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
      uint32_t h[4], l[4], ll[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 y = __fmul2_rn(make_float2(lo_of(in[e]), hi_of(in[e])), ww), rest = less_upper(y);
        h[e] = uppers(y);
        if (THIRD) { l[e] = uppers(rest); ll[e] = uppers(less_upper(rest)); }
        else l[e] = pack2(rest.x, rest.y);
      }
      sts128(khi + off, make_uint4(h[0], h[1], h[2], h[3]));
      sts128(klo + off, make_uint4(l[0], l[1], l[2], l[3]));
      if (THIRD) sts128(kll + off, make_uint4(ll[0], ll[1], ll[2], ll[3]));
    }
  }
}
__device__ __forceinline__ void clear_row(uint32_t box, int row) {
#pragma unroll
  for (int i = 0; i < 8; ++i) sts128(box + row * 128 + i * 16, make_uint4(0, 0, 0, 0));
}
// A lane holds N 16-byte pieces of its row (128 or 64 bytes); they are exchanged among N lanes so that a store instruction of the warp writes 32 / N whole runs.
// Straight from the lanes it would touch 32 rows with 16 bytes each: many times the accesses of the LSU, which the loads and stores of K~ and S share (an output
// tile took 5200 cycles, everything beside it twice its time).  row_at: the lane's first row (N (lane / N)) and piece; rows: valid rows from there on.
template <int N>
__device__ __forceinline__ void store_rows(char* row_at, int64_t pitch, int rows, bool piece_ok, uint32_t (&w)[4 * N], int lane) {
#pragma unroll
  for (int m = 1; m < N; m *= 2) {
    const bool up = (lane & m) != 0;
#pragma unroll
    for (int q = 0; q < N; ++q) {
      if (q & m) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t a = w[4 * q + e], b = w[4 * (q | m) + e], got = __shfl_xor_sync(0xffffffffu, up ? a : b, m);
        w[4 * q + e] = up ? got : a;
        w[4 * (q | m) + e] = up ? b : got;
      }
    }
  }
#pragma unroll
  for (int t = 0; t < N; ++t)
    if (piece_ok && t < rows) *reinterpret_cast<uint4*>(row_at + t * pitch) = make_uint4(w[4 * t], w[4 * t + 1], w[4 * t + 2], w[4 * t + 3]);
}
// V^T K~ of a chunk: the first ks steps of 16 rows, the smallest parts first (the accumulator drops what is below its last bit at every step).
template <int BOX, bool THIRD>
__device__ __forceinline__ void issue_state(uint32_t tmem_d, uint32_t v, uint32_t khi, uint32_t klo, uint32_t kll, uint32_t idesc, int ks) {
  const uint64_t a = desc_mn<BOX>(v), h = desc_mn<BOX>(khi), l = desc_mn<BOX>(klo), ll = desc_mn<BOX>(kll);
  if (THIRD)
    for (int k = 0; k < ks; ++k) umma_bf16(tmem_d, a + (uint64_t)(MN_KSTEP * k), ll + (uint64_t)(MN_KSTEP * k), idesc, k > 0 ? 1u : 0u);
  for (int k = 0; k < ks; ++k) umma_bf16(tmem_d, a + (uint64_t)(MN_KSTEP * k), l + (uint64_t)(MN_KSTEP * k), idesc, THIRD || k > 0 ? 1u : 0u);
  for (int k = 0; k < ks; ++k) umma_bf16(tmem_d, a + (uint64_t)(MN_KSTEP * k), h + (uint64_t)(MN_KSTEP * k), idesc, 1u);
}
template <int BOXES>
__device__ __forceinline__ void prefetch_tile(const CUtensorMap* map, int head, int row) {
#pragma unroll
  for (int b = 0; b < BOXES; ++b)
    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(map), "r"(64 * b), "r"(head), "r"(row) : "memory");
}
template <int BOXES, int BOX = LT_BOX>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* map, uint32_t bar, int head, int row) {
#pragma unroll
  for (int b = 0; b < BOXES; ++b) tma_load_3d(dst + b * BOX, map, bar, 64 * b, head, row);
}
__device__ __forceinline__ void latch(const LinPass& p, volatile int* abort_flag, int where) {
  if (!*abort_flag) {
    atomicExch(p.status + kStatCode, ROM_ERR_DEVICE_TIMEOUT);
    atomicExch(p.status + kStatWhere, where);
  }
  *abort_flag = 1;
}

// The rows [r0, r1) of one sequence in one run, in chunks.
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
// The pieces of a run's rows of one head.
__device__ __forceinline__ int first_piece(const LinItem& it, const Ragged& q) {      // all lanes of a warp
  const int s = q.first_from(it.a);
  return s > 0 && q.end_of(s - 1) > it.a ? s - 1 : s;
}
template <bool REV>
__device__ __forceinline__ bool get_piece(const LinItem& it, const Ragged& q, bool skip_single, int s, LinPiece& x) {      // false: no sequence from s on has to do with these rows
  if (s >= q.n_seq) return false;
  const int st = q.start_of(s), en = q.end_of(s);
  if (st >= it.b && !it.last) return false;
  const bool empty = en <= st, skip = skip_single && en - st == 1;
  x.s = s;
  x.r0 = max(st, it.a);
  x.r1 = empty || skip ? x.r0 : max(min(en, it.b), x.r0);
  x.over = !empty && (REV ? en > it.b : st < it.a);
  x.ends = empty || (x.r1 > x.r0 && (REV ? st >= it.a : en <= it.b));
  return true;
}

// ------------------------------------------------------------------------------------------------------------------------------ the walk
// A wait that gives up ends the waits of its warp, not its loop: the warps that meet at named barriers (each role's eight) all come to every one of
// them, and only the results are left out.
__host__ __device__ constexpr int more(int a, int b) { return a > b ? a : b; }
template <int KP, int VP>
struct WalkShape {
  static constexpr int KB = KP / 64, VB = VP / 64;
  // stages, as many as 227 KB hold: a copy takes up to 2 us when memory is busy, a chunk of two heads' widths of 64 half of that
  // (Q, and at 128 x 128 V, with one stage: Q S and V^T K~ end well before their next operands are used, and these come from L2: no slower than two of V)
  static constexpr int KST = KP == 128 ? 2 : VP == 128 ? 3 : 4, QST = KP == 128 || VP == 128 ? 1 : 2, VST = KP == 128 && VP == 128 ? 1 : KST;
  static constexpr int Q = 0, K = Q + QST * KB * LT_BOX, V = K + KST * KB * LT_BOX, LO = V + VST * VB * LT_BOX, LL = LO + KB * LT_BOX, S = LL + KB * LT_BOX, S_BYTES = KB * VP * 128;
  // the second part of S; at 128 x 128 it has no room of its own, and lies where K~'s third part comes once Q S has read it
  static constexpr bool S2_IN_LL = KP == 128 && VP == 128;
  static constexpr int S2 = S2_IN_LL ? LL : S + S_BYTES, BYTES = S + (S2_IN_LL ? 1 : 2) * S_BYTES;
  static constexpr int BARS = 2 * (QST + KST + VST) + 9;
  static constexpr int SC = 0, O1 = 128, KV = O1 + VP, O2 = KV + KP;      // tensor-memory columns (P over the scores: of every 16 columns the first parts in 8, the second in 8)
};

// Rows of O2 that are not finite, summed again over their own and earlier rows, where what the state gives is finite (else the result is not, either way: a value that is not
// finite costs its own chunk alone).  Rare; all lanes of the warp come here.
template <bool REV>
__device__ __noinline__ void slow_rows(const LinPass& p, int head, uint32_t taddr_o1, uint32_t taddr_o2, const float* lam, int i, int row0, int len, float f, bool mine, int c_from, int c_to) {
#pragma unroll 1
  for (int c0 = c_from; c0 < c_to; c0 += 16) {
    uint32_t r[16], r2[16];
    __syncwarp();
    tmem_ld16_issue(taddr_o1 + c0, r);
    tmem_ld16_issue(taddr_o2 + c0, r2);
    tmem_ld16_wait(r);
    tmem_ld16_wait(r2);
    bool need = false;
#pragma unroll
    for (int e = 0; e < 16; ++e) need |= !(fabsf(__uint_as_float(r2[e])) <= FLT_MAX) && fabsf(f * __uint_as_float(r[e])) <= FLT_MAX;
    if (!mine || !need) continue;
    float acc[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
    const bf16* qi = static_cast<const bf16*>(p.q) + (int64_t)(row0 + i) * p.ldq + (head / p.qdiv) * p.dk;
#pragma unroll 1
    for (int j = REV ? i : 0; j < (REV ? len : i + 1); ++j) {
      const bf16* kj = static_cast<const bf16*>(p.k) + (int64_t)(row0 + j) * p.ldk + (head / p.kdiv) * p.dk;
      float s = 0.0f;
#pragma unroll 1
      for (int d = 0; d < p.dk; ++d) s = fmaf(to_f32(qi[d]), to_f32(kj[d]), s);
      const float w = s * (p.p_scale * lam[REV ? j - i : i - j]);
      const bf16* vj = static_cast<const bf16*>(p.v) + (int64_t)(row0 + j) * p.ldv + (head / p.vdiv) * p.dv + c0;
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (c0 + e < p.dv) acc[e] = fmaf(w, to_f32(vj[e]), acc[e]);
    }
    const int64_t to = (int64_t)(row0 + i) * p.ldo + (int64_t)head * p.dv + c0;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (c0 + e < p.dv) {
        const float o = fmaf(f, __uint_as_float(r[e]), acc[e]);
        if (p.out_f32) static_cast<float*>(p.out)[to + e] = o;
        else static_cast<bf16*>(p.out)[to + e] = __float2bfloat16_rn(o);
      }
  }
}

struct WalkArgs { CUtensorMap q, k, v; LinPass p; };
template <int BARS>
struct WalkShared {
  // powers of lambda: of the warps that make P (on the diagonal times p, behind 32 zeros), of those that keep S, with what each lost to fp32
  float p_lam[kLinPowers], p_diag[64], s_lam[kLinPowers], s_lo[kLinPowers];
  unsigned long long bars[BARS];
  uint32_t tmem;
  int abort;
};
template <int KP, int VP, bool REV, bool THIRD, int BARS>
__device__ __forceinline__ void walk(const WalkArgs& args, WalkShared<BARS>& sh, const uint32_t base, const Ragged& seqs, const LinCut& cut, uint32_t wait_limit, uint32_t stall) {
  using W = WalkShape<KP, VP>;
  const LinPass& p = args.p;
  const CUtensorMap &tmap_q = args.q, &tmap_k = args.k, &tmap_v = args.v;
  float *const p_diag = sh.p_diag, *const s_lam = sh.s_lam, *const s_lo = sh.s_lo;
  unsigned long long* const bars = sh.bars;
  uint32_t& tmem_s = sh.tmem;
  int& abort_s = sh.abort;
  volatile int* abort_flag = &abort_s;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), run = blockIdx.x;
  auto bar = [&](int i) { return smem_u32(&bars[i]); };
  // full: copies have landed; empty: the matrix products that read them are done; the others by name
  constexpr int BK = 2 * W::QST, BV = BK + 2 * W::KST, B1 = BV + 2 * W::VST;
  static_assert(W::BARS <= BARS, "barriers");
  auto q_full = [&](int s) { return bar(s); };
  auto q_empty = [&](int s) { return bar(W::QST + s); };
  auto k_full = [&](int s) { return bar(BK + s); };
  auto k_empty = [&](int s) { return bar(BK + W::KST + s); };
  auto v_full = [&](int s) { return bar(BV + s); };
  auto v_empty = [&](int s) { return bar(BV + W::VST + s); };
  const uint32_t sc_full = bar(B1), pv_full = bar(B1 + 1), state_full = bar(B1 + 2), drain = bar(B1 + 3), p_ready = bar(B1 + 4), k_ready = bar(B1 + 5), s_ready = bar(B1 + 6), o_free = bar(B1 + 7), s2_read = bar(B1 + 8);
  constexpr bool S2_LEAVES = W::S2_IN_LL && THIRD;      // K~'s third part waits for Q S to have read S's second
  if (tid == 0) {
    for (int i = 0; i < W::BARS; ++i) mbar_init(bar(i), i >= B1 + 4 && i < B1 + 8 ? 8 : 1);
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(LT_TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid < 32) p_diag[tid] = 0.0f;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_s;
  // Here the launch before may still run (launch 2, or the powers): inputs and the sequences' tables are older than it.  What it writes (states, powers) is read, and what
  // it may read or what its own predecessors may write (pools, outputs) is written, by warps that have waited for it.
  LinItem it(cut, run);
  LinPiece x;
  int n = 0;                           // chunks so far

  // Rows of the last quarter (backwards: the first) have four blocks of scores to turn into P, those of the first one: the copies' and products' warps poll on the
  // schedulers of the light quarters.
  constexpr int COPIES = REV ? 3 : 0, PRODUCTS = REV ? 2 : 1;
  // (setmaxnreg inside each role's branch: behind a join the compiler would hold every role to the fewest)
  if (warp == COPIES) {
    registers_down<LT_FEW>();
    // ---------------------------------------------------------------- copies
    const bool leader = elect_one();
    bool ok = true;
    while (it.next(cut, seqs)) {
      const int head = it.head, s_first = first_piece(it, seqs);
      if (leader)
      for (int s = s_first; ok && get_piece<REV>(it, seqs, p.skip_single, s, x); ++s) {
        if (!x.over && x.r1 > x.r0) {  // the state that the piece starts from, into L2 while the pieces before are walked
          const float* from = lin_init_of(p, seqs, s, head);
          if (from) asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"((uint32_t)(p.dk * p.dv * sizeof(float))) : "memory");
        }
        for (int m = 0, mm = x.chunks(); m < mm; ++m, ++n) {
          int row0, len;
          x.chunk<REV>(m, row0, len);
          const int ks = n % W::KST, qs = n % W::QST, vs = n % W::VST;
          if (n == 1) pdl_wait();      // (the first chunk's copies need not wait for the launch before, but no bounded wait may count its time)
          if (!mbar_wait(k_empty(ks), (n / W::KST & 1) ^ 1, abort_flag, wait_limit)) { ok = false; break; }
          mbar_expect_tx(k_full(ks), W::KB * LT_BOX + stall);
          load_tile<W::KB>(base + W::K + ks * W::KB * LT_BOX, &tmap_k, k_full(ks), head / p.kdiv, row0);
          // one stage of Q: it is asked for when Q S of the chunk before is done, 4000 cycles from memory where the chunk has 2500 left; from L2 1500
          if (W::QST == 1) prefetch_tile<W::KB>(&tmap_q, head / p.qdiv, row0);
          if (W::VST == 1) prefetch_tile<W::VB>(&tmap_v, head / p.vdiv, row0);
          if (!mbar_wait(q_empty(qs), (n / W::QST & 1) ^ 1, abort_flag, wait_limit)) { ++n; ok = false; break; }
          mbar_expect_tx(q_full(qs), W::KB * LT_BOX);
          load_tile<W::KB>(base + W::Q + qs * W::KB * LT_BOX, &tmap_q, q_full(qs), head / p.qdiv, row0);
          if (!mbar_wait(v_empty(vs), (n / W::VST & 1) ^ 1, abort_flag, wait_limit)) { ++n; ok = false; break; }
          mbar_expect_tx(v_full(vs), W::VB * LT_BOX);
          load_tile<W::VB>(base + W::V + vs * W::VB * LT_BOX, &tmap_v, v_full(vs), head / p.vdiv, row0);
        }
      }
      __syncwarp();
    }
    if (leader) {
      if (!ok) latch(p, abort_flag, 51);
      if (*abort_flag)                 // the copies still in flight land (bounded) before the block ends
        for (int i = 1; i <= W::KST && i <= n; ++i) {
          const int c = n - i;
          for (uint32_t it = 0; it < wait_limit >> 2 && !mbar_try_wait(k_full(c % W::KST), c / W::KST & 1); ++it) {}
          for (uint32_t it = 0; it < wait_limit >> 2 && !mbar_try_wait(q_full(c % W::QST), c / W::QST & 1); ++it) {}
          for (uint32_t it = 0; it < wait_limit >> 2 && !mbar_try_wait(v_full(c % W::VST), c / W::VST & 1); ++it) {}
        }
    }
    __syncwarp();
  } else if (warp == PRODUCTS) {
    registers_down<LT_FEW>();
    // ---------------------------------------------------------------- matrix products
    const bool leader = elect_one();
    bool ok = true, issued = false;
    pdl_wait();
    while (it.next(cut, seqs)) {
      const int s_first = first_piece(it, seqs);
      constexpr uint32_t d_sc = lt_idesc(LT_C, false, false), d_o1 = lt_idesc(VP, false, false), d_o2 = lt_idesc(VP, false, true), d_kv = lt_idesc(KP, true, true);
      auto wait = [&](uint32_t b, uint32_t parity) { ok = ok && mbar_wait(b, parity, abort_flag, wait_limit); return ok; };
      if (leader)
      for (int s = s_first; ok && get_piece<REV>(it, seqs, p.skip_single, s, x); ++s)
        for (int m = 0, mm = x.chunks(); m < mm; ++m, ++n) {
          int row0, len;
          x.chunk<REV>(m, row0, len);
          const int st = n % W::KST, qs = n % W::QST, vs = n % W::VST, ks = (len + 15) / 16;
          const uint32_t ph = n & 1, q = base + W::Q + qs * W::KB * LT_BOX, k = base + W::K + st * W::KB * LT_BOX, v = base + W::V + vs * W::VB * LT_BOX;
          // scores, once the P that lies over them has been used
          if (!wait(k_full(st), n / W::KST & 1) || !wait(q_full(qs), n / W::QST & 1) || (n > 0 && !wait(pv_full, ph ^ 1))) break;
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
              umma_bf16(tmem + W::O1, make_smem_desc(q + b * LT_BOX) + 2 * e, make_smem_desc(base + W::S2 + b * VP * 128) + 2 * e, d_o1, b + e > 0 ? 1u : 0u);
          if (S2_LEAVES) umma_commit(s2_read);
#pragma unroll
          for (int b = 0; b < W::KB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              umma_bf16(tmem + W::O1, make_smem_desc(q + b * LT_BOX) + 2 * e, make_smem_desc(base + W::S + b * VP * 128) + 2 * e, d_o1, 1u);
          umma_commit(q_empty(qs));
          // P V while K~ is made, but where that clears rows of V
          if (!wait(v_full(vs), n / W::VST & 1) || !wait(p_ready, ph) || ((len & 15) != 0 && !wait(k_ready, ph))) break;
          tc_fence_after();
          for (int e = 0; e < ks; ++e) umma_bf16_ta(tmem + W::O2, tmem + W::SC + 16 * e + 8, desc_mn<LT_BOX>(v) + (uint64_t)(MN_KSTEP * e), d_o2, e > 0 ? 1u : 0u);
          for (int e = 0; e < ks; ++e) umma_bf16_ta(tmem + W::O2, tmem + W::SC + 16 * e, desc_mn<LT_BOX>(v) + (uint64_t)(MN_KSTEP * e), d_o2, 1u);
          umma_commit(pv_full);
          if (!wait(k_ready, ph)) break;
          tc_fence_after();
          issue_state<LT_BOX, THIRD>(tmem + W::KV, v, k, base + W::LO, base + W::LL, d_kv, ks);
          umma_commit(state_full);
          umma_commit(k_empty(st));
          umma_commit(v_empty(vs));
        }
      __syncwarp();
    }
    if (leader) {
      if (!ok) latch(p, abort_flag, 52);
      if (*abort_flag && issued) {     // what has been issued may still read shared memory and write tensor memory
        umma_commit(drain);
        for (uint32_t it = 0; it < wait_limit >> 2 && !mbar_try_wait(drain, 0); ++it) {}
      }
    }
    __syncwarp();
  } else if (warp >= 4 && warp < 12) {
    // ---------------------------------------------------------------- scores to P, outputs
    const int quarter = warp & 3, half = (warp - 4) >> 2, i = quarter * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    bf16* out = static_cast<bf16*>(p.out);
    registers_up<LT_P>();
    const float* lam = sh.p_lam;
    pdl_wait();
    bool ok = true;
    while (it.next(cut, seqs)) {
    const int head = it.head, s_first = first_piece(it, seqs);
    asm volatile("bar.sync 5, 256;" ::: "memory");      // (all of these warps are done with the powers of the head before)
    if (const int e = tid - 128; e < kLinPowers) {
      const float l = __ldcg(p.powers + (size_t)head * 2 * kLinPowers + e);
      sh.p_lam[e] = l;
      if (e < 32) p_diag[32 + e] = p.p_scale * l;
    }
    asm volatile("bar.sync 5, 256;" ::: "memory");
    for (int s = s_first; get_piece<REV>(it, seqs, p.skip_single, s, x); ++s)
      for (int m = 0, mm = x.chunks(); m < mm; ++m, ++n) {
        int row0, len;
        x.chunk<REV>(m, row0, len);
        const uint32_t ph = n & 1;
        const int early = m == 0 && !x.over && p.early ? 1 : 0;
        ok = ok && warp_wait(sc_full, ph, abort_flag, wait_limit);
        tc_fence_after();
        // The quarter's two warps take every other 16 columns, and put P's first and second parts in the same columns, 8 each.  (Loops that are not unrolled, here, in the outputs and
        // over K's pieces: the roles' code together is more than the instruction cache holds, and unrolled 16384 rows of 32 heads of 128 took 232 us instead of 215, prompts with heads
        // of 64 120 instead of 98.)
#pragma unroll 1
        for (int b = half; b < (len + 15) / 16; b += 2) {
          uint32_t w[16];
          const int gap = 16 * b - 32 * quarter;      // of the columns from the quarter's first row
          if (REV ? gap < 0 : gap > 16) {
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = 0;
          } else {
            uint32_t r[16];
            tmem_ld16_issue(lanes + W::SC + 16 * b, r);
            tmem_ld16_wait(r);
            const bool diagonal = REV ? gap <= 16 : gap >= 0;
            // A masked score is times 0; where it is not finite, the row is summed again below.  In the last chunk, whose other rows are not the sequence's, they are
            // selected 0: forwards they are ahead of the diagonal, backwards in the last columns.
            if (len < LT_C && (REV ? 16 * b + 16 > len : diagonal)) {
#pragma unroll
              for (int e = 0; e < 16; ++e)
                if (REV ? 16 * b + e >= len : gap + e > lane) r[e] = 0;
            }
            // lambda^{i-j} in steps of eight places, lambda^{i - last of the eight} lambda^{last - j}.  On the diagonal the row's own eight have powers of their own, zeros behind it.
            float g[2];
            float2 d[4];
#pragma unroll
            for (int k = 0; k < 2; ++k)
              g[k] = diagonal ? p_diag[32 + (REV ? gap + 8 * k - lane : lane - gap - 8 * k - 7)] : p.p_scale * lam[REV ? 16 * b - i + 8 * k : i - 16 * b - 8 * k - 7];
            if (diagonal) {
              const float* l = p_diag + 32 + (REV ? -(lane & 7) : lane & 7);
#pragma unroll
              for (int e = 0; e < 4; ++e) d[e] = REV ? make_float2(l[2 * e], l[2 * e + 1]) : make_float2(l[-2 * e], l[-2 * e - 1]);
            }
            const float4 u0 = *reinterpret_cast<const float4*>(lam), u1 = *reinterpret_cast<const float4*>(lam + 4);
            const float2 u[4] = {REV ? make_float2(u0.x, u0.y) : make_float2(u1.w, u1.z), REV ? make_float2(u0.z, u0.w) : make_float2(u1.y, u1.x),
                                 REV ? make_float2(u1.x, u1.y) : make_float2(u0.w, u0.z), REV ? make_float2(u1.z, u1.w) : make_float2(u0.y, u0.x)};
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float2 f = __fmul2_rn(u[e], make_float2(g[k], g[k]));
                if (diagonal && gap + 8 * k == (lane & 24)) f = d[e];
                halves(__fmul2_rn(make_float2(__uint_as_float(r[8 * k + 2 * e]), __uint_as_float(r[8 * k + 2 * e + 1])), f), w[4 * k + e], w[8 + 4 * k + e]);
              }
          }
          tmem_st16(lanes + W::SC + 16 * b, w);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        warp_arrive(p_ready);
        ok = ok && warp_wait(pv_full, ph, abort_flag, wait_limit);
        tc_fence_after();
        const bool mine = i < len;
        const float f = p.inter_scale * lam[REV ? max(len - i - early, 0) : i + 1 - early];
        float2 odd = make_float2(0.0f, 0.0f);
        constexpr int PC = 4;
        const int c_from = half * (VP / 2), c_to = min(p.dv, c_from + VP / 2), first = quarter * 32 + lane / PC * PC, rows = ok ? len - first : 0;      // (rows that the lane stores)
        const int first8 = quarter * 32 + (lane & 24), rows8 = ok ? len - first8 : 0;
        // 16 columns: f O1 + O2, noting what is not finite
        auto columns = [&](int c, float2 (&o)[8]) {
          uint32_t r1[16], r2[16];
          __syncwarp();
          tmem_ld16_issue(lanes + W::O1 + c, r1);
          tmem_ld16_issue(lanes + W::O2 + c, r2);
          tmem_ld16_wait(r1);
          tmem_ld16_wait(r2);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 b2 = make_float2(__uint_as_float(r2[2 * e]), __uint_as_float(r2[2 * e + 1]));
            odd = __ffma2_rn(b2, make_float2(0.0f, 0.0f), odd);
            o[e] = __ffma2_rn(make_float2(__uint_as_float(r1[2 * e]), __uint_as_float(r1[2 * e + 1])), make_float2(f, f), b2);
          }
        };
        if (p.out_f32) {
#pragma unroll 1
          for (int c = c_from; c < c_to; c += 32) {
            uint32_t w[32];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              float2 o[8];
              columns(c + 16 * u, o);
#pragma unroll
              for (int e = 0; e < 8; ++e) { w[16 * u + 2 * e] = __float_as_uint(o[e].x); w[16 * u + 2 * e + 1] = __float_as_uint(o[e].y); }
            }
            const int col = c + 4 * (lane & 7);
            store_rows<8>(reinterpret_cast<char*>(static_cast<float*>(p.out) + (int64_t)(row0 + first8) * p.ldo + (int64_t)head * p.dv + col), p.ldo * 4, rows8, col < p.dv, w, lane);
          }
        } else
#pragma unroll 1
        for (int c1 = c_from; c1 < c_to; c1 += 32) {
          uint32_t w[4 * PC];
#pragma unroll
          for (int u = 0; u < PC / 2; ++u) {
            float2 o[8];
            columns(c1 + 16 * u, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) w[8 * u + e] = pack2(o[e].x, o[e].y);
          }
          const int col = c1 + 8 * (lane & (PC - 1));
          store_rows<PC>(reinterpret_cast<char*>(out + (int64_t)(row0 + first) * p.ldo + (int64_t)head * p.dv + col), p.ldo * 2, rows, col < p.dv, w, lane);
        }
        const bool again = ok && mine && !(odd.x == 0.0f && odd.y == 0.0f);
        if (__any_sync(0xffffffffu, again)) slow_rows<REV>(p, head, lanes + W::O1, lanes + W::O2, lam, i, row0, len, f, again, c_from, c_to);
        tc_fence_before();
        warp_arrive(o_free);
      }
    }
    if (!ok) latch(p, abort_flag, 53);
  } else if (warp >= 12) {
    registers_up<LT_MANY>();
    // ---------------------------------------------------------------- K~ and the state: two threads keep column c of S, half of its rows each
    constexpr int KH = KP / 2;
    const int quarter = warp & 3, half = (warp - 12) >> 2, c = quarter * 32 + lane, a0 = half * KH;
    const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16);
    const size_t state = (size_t)p.dk * p.dv;
    float S[KH];
    const float *lam = s_lam, *lam_lo = s_lo;
    pdl_wait();
    pdl_trigger();                     // (behind the block's tensor memory: the successor takes its own before it waits)
    bool ok = true;
    // Eight numbers of S^T's row c, K-major, in two parts.
    auto write_8 = [&](int a, float x0, float x1, float x2, float x3, float x4, float x5, float x6, float x7) {
      const uint32_t off = (KP == 128 ? half : 0) * VP * 128 + c * 128 + ((((KP == 128 ? 0 : 4 * half) + a / 8) ^ (c & 7)) << 4);
      uint4 h, l;
      halves(make_float2(x0, x1), h.x, l.x);
      halves(make_float2(x2, x3), h.y, l.y);
      halves(make_float2(x4, x5), h.z, l.z);
      halves(make_float2(x6, x7), h.w, l.w);
      sts128(base + W::S + off, h);
      sts128(base + W::S2 + off, l);
    };
    auto wrote_s = [&]() {
      fence_async();
      warp_arrive(s_ready);
    };
    while (it.next(cut, seqs)) {
    const int head = it.head, s_first = first_piece(it, seqs);
    asm volatile("bar.sync 6, 256;" ::: "memory");
    if (int e = tid - 384; e < kLinPowers) {
      s_lam[e] = __ldcg(p.powers + (size_t)head * 2 * kLinPowers + e);
      s_lo[e] = __ldcg(p.powers + (size_t)head * 2 * kLinPowers + kLinPowers + e);
    }
    asm volatile("bar.sync 6, 256;" ::: "memory");
    for (int s = s_first; get_piece<REV>(it, seqs, p.skip_single, s, x); ++s) {
      const int mm = x.chunks(), slot = seqs.slot_of(s);
      const float* from = lin_init_of(p, seqs, s, head);
      if (x.over) from = p.cut_state + (size_t)(REV ? run : run - 1) * state;
      else if (!REV && mm > 0 && from && p.init_copy && !x.ends) from = p.init_copy + (size_t)run * state;
      if (mm == 0 && !x.ends) continue;
      // (every load at a valid address and selected afterwards: one by one behind branches they took 10000 cycles)
      const bool mine = from != nullptr && c < p.dv;
      if (from) {
        const int col = min(c, p.dv - 1);
        if (p.transposed) {
          // rows of the memory are columns of S^T's rows: 32 rows x 16 columns at a time are read whole and change lanes through the (idle) space of K~'s second part
          float4 v[KH / 4];
#pragma unroll
          for (int g = 0; g < KH / 16; ++g)
#pragma unroll
            for (int u = 0; u < 4; ++u)
              v[4 * g + u] = ld_state4(from + (size_t)min(quarter * 32 + 8 * u + lane / 4, p.dv - 1) * p.dk + min(a0 + 16 * g + 4 * (lane & 3), p.dk - 4));
          const uint32_t mine_at = base + W::LO + (warp - 12) * 2048;
#pragma unroll
          for (int g = 0; g < KH / 16; ++g) {
            __syncwarp();
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const int row = 8 * u + lane / 4;
              const float4 x4 = v[4 * g + u];
              sts128(mine_at + row * 64 + (((lane & 3) ^ (row >> 1 & 3)) << 4), make_uint4(__float_as_uint(x4.x), __float_as_uint(x4.y), __float_as_uint(x4.z), __float_as_uint(x4.w)));
            }
            __syncwarp();
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const uint4 x4 = lds128(mine_at + lane * 64 + ((u ^ (lane >> 1 & 3)) << 4));
              S[16 * g + 4 * u] = __uint_as_float(x4.x); S[16 * g + 4 * u + 1] = __uint_as_float(x4.y);
              S[16 * g + 4 * u + 2] = __uint_as_float(x4.z); S[16 * g + 4 * u + 3] = __uint_as_float(x4.w);
            }
          }
          asm volatile("bar.sync 6, 256;" ::: "memory");      // (another warp's K~ would come into this one's place)
        } else {
#pragma unroll
          for (int a = 0; a < KH; ++a) S[a] = ld_state(from + (size_t)min(a0 + a, p.dk - 1) * p.dv + col);
        }
      }
#pragma unroll
      for (int a = 0; a < KH; ++a)
        if (!mine || a0 + a >= p.dk) S[a] = 0.0f;
      if (mm > 0) {
        if (c < VP)
#pragma unroll
          for (int a = 0; a < KH; a += 8) write_8(a, S[a], S[a + 1], S[a + 2], S[a + 3], S[a + 4], S[a + 5], S[a + 6], S[a + 7]);
        wrote_s();
      }
      for (int m = 0; m < mm; ++m, ++n) {
        int row0, len;
        x.chunk<REV>(m, row0, len);
        const int st = n % W::KST, vs = n % W::VST, early = m == 0 && !x.over && p.early ? 1 : 0, rows16 = (len + 15) / 16 * 16;
        const uint32_t ph = n & 1, k = base + W::K + st * W::KB * LT_BOX, box = KP == 128 ? half * LT_BOX : 0;
        // (the scores are made of this K: sc_full says that it has landed, but the copies' own barrier makes them visible)
        ok = ok && warp_wait(sc_full, ph, abort_flag, wait_limit) && warp_wait(k_full(st), n / W::KST & 1, abort_flag, wait_limit);
        if (rows16 > len) ok = ok && warp_wait(v_full(vs), n / W::VST & 1, abort_flag, wait_limit);
        if (S2_LEAVES) ok = ok && warp_wait(s2_read, ph, abort_flag, wait_limit);
        if (c < rows16) {
          const bool live = c < len;
          const float w = live ? p.k_scale * lam[REV ? c : len - 1 - c] : 0.0f;
          scale_row<2, THIRD>(k + box, base + W::LO + box, base + W::LL + box, c, w, live, KP == 128 ? 0 : 4 * half, KP == 128 ? 8 : 4);
          if (!live && half < W::VB) clear_row(base + W::V + (vs * W::VB + half) * LT_BOX, c);
        }
        fence_async();
        warp_arrive(k_ready);
        ok = ok && warp_wait(state_full, ph, abort_flag, wait_limit);
        tc_fence_after();
        const float f = lam[len - early], fl = lam_lo[len - early];
#pragma unroll
        for (int a = 0; a < KH; a += 16) {
          uint32_t r[16];
          tmem_ld16_issue(lanes + W::KV + a0 + a, r);
          tmem_ld16_wait(r);
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            float2 v = __ffma2_rn(make_float2(S[a + e], S[a + e + 1]), make_float2(fl, fl), make_float2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])));
            v = __ffma2_rn(make_float2(S[a + e], S[a + e + 1]), make_float2(f, f), v);
            S[a + e] = v.x;
            S[a + e + 1] = v.y;
          }
          if (c < VP && m + 1 < mm)      // (here and not behind the loop: all of S's parts at once are more registers than there are)
#pragma unroll
            for (int e = 0; e < 16; e += 8) write_8(a + e, S[a + e], S[a + e + 1], S[a + e + 2], S[a + e + 3], S[a + e + 4], S[a + e + 5], S[a + e + 6], S[a + e + 7]);
        }
        tc_fence_before();
        if (m + 1 < mm) wrote_s();
      }
      if (ok && p.last && slot >= 0 && x.ends && c < p.dv) {
        const bool none = lin_leaves_zeros(p, seqs, s);
        const float f = mm > 0 && p.early ? lam[1] : 1.0f;
        float* to = p.last + ((size_t)slot * p.H + head) * state + c;
#pragma unroll
        for (int a = 0; a < KH; a += 8)
          if (a0 + a < p.dk)
#pragma unroll
            for (int e = 0; e < 8; ++e) to[(size_t)(a0 + a + e) * p.dv] = none ? 0.0f : f * S[a + e];
      }
    }
    }
    if (!ok) latch(p, abort_flag, 54);
  } else {
    registers_down<LT_FEW>();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(LT_TMEM) : "memory");
}
__device__ __forceinline__ uint32_t aligned_base(unsigned char* raw) { return (smem_u32(raw) + 1023u) & ~1023u; }
// The forward's walk.
template <int KP, int VP>
__global__ void __launch_bounds__(LT_WALK_THREADS, 1)
lin_walk_tc(const __grid_constant__ WalkArgs args, const Ragged seqs, const LinCut cut, uint32_t wait_limit, uint32_t stall) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(16) WalkShared<WalkShape<KP, VP>::BARS> sh;
  walk<KP, VP, false, true>(args, sh, aligned_base(smem_raw), seqs, cut, wait_limit, stall);
}
// The backward's three: they read the same inputs and states and write different outputs, and a launch each would leave most SMs idle where sequences are few or short (two
// sequences of one row, 8 heads: 37 us in three launches, most of it their latency).
template <int KP, int VP>
__global__ void __launch_bounds__(LT_WALK_THREADS, 1)
lin_walk3_tc(const __grid_constant__ WalkArgs dq, const __grid_constant__ WalkArgs dv, const __grid_constant__ WalkArgs dk, const Ragged seqs, const LinCut cut, uint32_t wait_limit,
             uint32_t stall) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(16) WalkShared<more(WalkShape<KP, VP>::BARS, WalkShape<VP, KP>::BARS)> sh;
  const uint32_t base = aligned_base(smem_raw);
  if (blockIdx.y == 0) walk<KP, VP, true, true>(dv, sh, base, seqs, cut, wait_limit, stall);
  else if (blockIdx.y == 1) walk<VP, KP, true, false>(dk, sh, base, seqs, cut, wait_limit, stall);
  else walk<VP, KP, false, false>(dq, sh, base, seqs, cut, wait_limit, stall);
}

// ------------------------------------------------------------------------------------------------------------------------------ launch 1: states at the cuts
// sum over the rows between two cuts of the sequence that reaches over the far one, lambda^{distance to that cut} ks k_j v_j^T: every row's weight is known, so they
// add up in tensor memory, in steps of 64 rows: the first parts of K~ in one accumulator, the small ones in another, which the two products of V with K~'s first and second part
// fill as one of twice the width (in one accumulator for all of them the state was off by three times as much).  Every product of 16 rows drops what is below the accumulator's last bit,
// which is the same way each time: the error of one sum grows with its rows.  After 512 rows the sum moves to fp32 registers, which round to nearest, while the next 512 add up in
// another pair (32 heads without decay, runs of 4096 rows in one sum: the last state 3.8e-6 of its norm off, of 32768 rows 3.2e-5; so 4.4e-7 and 5.6e-7, for 3 us of a call of 217).
// Sixteen warps scale K, eight threads to a row (eight warps are as fast).  What bounds it: shared memory, 176 KB of copies, operands and K~ a step of 128 x 128, 1400 cycles of the
// 2000 that a step takes (the tensor pipe is busy for 41 % of them); from DRAM it asks for 4 TB/s.
template <int KP, int VP>
struct StateShape {
  static constexpr int KB = KP / 64, VB = VP / 64, ROWS = 64, BOX = 64 * ROWS * 2;
  static constexpr int STAGE = (3 * KB + VB) * BOX, LO = KB * BOX, LL = 2 * KB * BOX, V = 3 * KB * BOX;      // K (hi) | lo | the third part | V
  static constexpr int STAGES = 196608 / STAGE, BYTES = STAGES * STAGE + (VB == 1 ? BOX : 0);      // (see desc_mn: one box behind the last V)
};
constexpr int kLtMaxSmem = 232448 - 2048;      // what a block may ask for, less its static variables
static_assert(sizeof(WalkShared<WalkShape<64, 128>::BARS>) <= 2048, "shared memory");
static_assert(WalkShape<128, 128>::BYTES + 1024 <= kLtMaxSmem && WalkShape<128, 64>::BYTES + 1024 <= kLtMaxSmem && WalkShape<64, 128>::BYTES + 1024 <= kLtMaxSmem, "shared memory");
static_assert(WalkShape<64, 64>::BYTES + (int)sizeof(WalkShared<WalkShape<64, 64>::BARS>) + 1024 <= 232448, "shared memory");
static_assert(StateShape<128, 128>::BYTES + 1024 <= kLtMaxSmem && StateShape<128, 64>::BYTES + 1024 <= kLtMaxSmem && StateShape<64, 128>::BYTES + 1024 <= kLtMaxSmem, "shared memory");

struct StateArgs { CUtensorMap k, v; LinPass p; };
constexpr int LT_FOLD = 8;                    // steps of 64 rows in one sum
struct StateShared { unsigned long long bars[3 * 8 + 3]; uint32_t tmem; int abort; };
template <int KP, int VP, bool REV, bool THIRD>
__device__ __forceinline__ void cut_states(const StateArgs& args, StateShared& sh, const uint32_t base, const Ragged& seqs, const LinCut& cut, uint32_t wait_limit, uint32_t stall) {
  using W = StateShape<KP, VP>;
  const LinPass& p = args.p;
  const CUtensorMap &tmap_k = args.k, &tmap_v = args.v;
  unsigned long long* const bars = sh.bars;
  uint32_t& tmem_s = sh.tmem;
  int& abort_s = sh.abort;
  volatile int* abort_flag = &abort_s;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  // The launch before may still run.  It (the powers, or a walk of the backward pass before this one) writes no input and reads none of what this one writes (its
  // own predecessors, which may have, are complete); only the launches behind this one count on it being complete once this one is: every block waits before it ends.
  int head, r0, r1;
  if (!lin_cut_rows(cut, blockIdx.x + 1, REV, seqs, head, r0, r1)) { pdl_wait(); return; }
  const int chunks = (r1 - r0 + W::ROWS - 1) / W::ROWS;
  static_assert(W::STAGES <= 8, "barriers");
  // the rows that launch 3 begins with last: they are still in L2 when it comes
  auto step = [&](int n) { return REV ? n : chunks - 1 - n; };
  auto full = [&](int i) { return smem_u32(&bars[i]); };
  auto empty = [&](int i) { return smem_u32(&bars[8 + i]); };
  auto scaled = [&](int i) { return smem_u32(&bars[16 + i]); };
  auto done = [&](int sum) { return smem_u32(&bars[24 + (sum & 1)]); };
  const uint32_t drain = smem_u32(&bars[26]);
  if (tid == 0) {
    for (int i = 0; i < 8; ++i) { mbar_init(full(i), 1); mbar_init(empty(i), 1); mbar_init(scaled(i), LT_SCALERS); }
    mbar_init(done(0), 1);
    mbar_init(done(1), 1);
    mbar_init(drain, 1);
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"((uint32_t)(4 * KP)) : "memory");
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
        mbar_expect_tx(full(st), (W::KB + W::VB) * W::BOX + stall);
        load_tile<W::KB, W::BOX>(at, &tmap_k, full(st), head / p.kdiv, r0 + W::ROWS * step(n));
        load_tile<W::VB, W::BOX>(at + W::V, &tmap_v, full(st), head / p.vdiv, r0 + W::ROWS * step(n));
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
        const uint32_t sum = tmem + (n / LT_FOLD & 1) * 2 * KP;
        const uint64_t a = desc_mn<W::BOX>(at + W::V), hl = desc_mn<W::BOX>(at), ll = desc_mn<W::BOX>(at + W::LL);
        for (int k = 0, ks = (min(W::ROWS, r1 - r0 - W::ROWS * step(n)) + 15) / 16; k < ks; ++k) {
          umma_bf16(sum, a + (uint64_t)(MN_KSTEP * k), hl + (uint64_t)(MN_KSTEP * k), lt_idesc(2 * KP, true, true), n % LT_FOLD + k > 0 ? 1u : 0u);
          if (THIRD) umma_bf16(sum + KP, a + (uint64_t)(MN_KSTEP * k), ll + (uint64_t)(MN_KSTEP * k), lt_idesc(KP, true, true), 1u);
        }
        umma_commit(empty(st));
        if (n % LT_FOLD == LT_FOLD - 1 || n == chunks - 1) umma_commit(done(n / LT_FOLD));
        issued = true;
      }
      if (!ok) latch(p, abort_flag, 56);
      if (*abort_flag && issued) {
        umma_commit(drain);
        for (uint32_t it = 0; it < wait_limit >> 2 && !mbar_try_wait(drain, 0); ++it) {}
      }
    }
    __syncwarp();
  } else {
    constexpr int PARTS = LT_SCALERS / 2, COLS = KP * 4 / LT_SCALERS;      // threads to a row of K; columns of a warp at the end
    const int group = (warp - 2) >> 2, quarter = warp & 3, j = quarter * 32 + lane, row = (tid - 64) & 63, part = (tid - 64) >> 6;
    const double g2 = (double)__ldg(p.log_decay + head) * 1.4426950408889634;
    bool ok = true;
    float total[COLS];
#pragma unroll
    for (int e = 0; e < COLS; ++e) total[e] = 0.0f;
    auto fold = [&](int sum) {
      if (!(ok = ok && warp_wait(done(sum), sum >> 1 & 1, abort_flag, wait_limit))) return;
      tc_fence_after();
      const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16) + (sum & 1) * 2 * KP + group * COLS;
#pragma unroll
      for (int c = 0; c < COLS; c += 16) {
        uint32_t hi[16], lo[16];
        __syncwarp();
        tmem_ld16_issue(from + c, hi);
        tmem_ld16_issue(from + KP + c, lo);
        tmem_ld16_wait(hi);
        tmem_ld16_wait(lo);
#pragma unroll
        for (int e = 0; e < 16; ++e) total[c + e] += __uint_as_float(hi[e]) + __uint_as_float(lo[e]);
      }
      tc_fence_before();
    };
    int folded = 0;
    for (int n = 0; n < chunks && ok; ++n) {
      // the sum before, two steps late: its products are done.  (The pair is used again only once the warps have scaled a later step's keys.)
      if (n % LT_FOLD == 2 && n > LT_FOLD) fold(folded++);
      const int st = n % W::STAGES, row0 = r0 + W::ROWS * step(n), len = min(W::ROWS, r1 - row0), rows16 = (len + 15) / 16 * 16;
      const uint32_t at = base + st * W::STAGE;
      // lambda^{distance}: the exponent in 64 bits, its fraction alone through fp32
      const double t = fmax(g2 * max(REV ? row0 + row - r0 : r1 - 1 - row0 - row, 0), -400.0), whole = rint(t);
      const float w = p.k_scale * ldexpf(exp2f((float)(t - whole)), (int)whole);
      if (!(ok = ok && warp_wait(full(st), n / W::STAGES & 1, abort_flag, wait_limit))) break;
      if (row < rows16) {
        const bool live = row < len;
        constexpr int PIECES = KP / 8 / PARTS;
        const uint32_t box = PIECES * part / 8 * W::BOX;
        scale_row<PIECES, THIRD>(at + box, at + W::LO + box, at + W::LL + box, row, w, live, PIECES * part & 7, PIECES);
        if (!live && part < W::VB) clear_row(at + W::V + part * W::BOX, row);
      }
      fence_async();
      warp_arrive(scaled(st));
    }
    pdl_wait();
    while (folded <= (chunks - 1) / LT_FOLD) fold(folded++);
    if (ok && j < p.dv) {
      float* to = p.cut_state + (size_t)blockIdx.x * ((size_t)p.dk * p.dv) + j;
#pragma unroll
      for (int e = 0; e < COLS; ++e)
        if (group * COLS + e < p.dk) to[(size_t)(group * COLS + e) * p.dv] = total[e];
    }
    if (!ok) latch(p, abort_flag, 57);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)(4 * KP)) : "memory");
}
// blockIdx.y: the forward's states, the backward's.  WALKED: the first ones end in no result (the backward pass reads them), two parts do.
template <int KP, int VP, bool WALKED>
__global__ void __launch_bounds__(LT_STATE_THREADS, 1)
lin_state_tc(const __grid_constant__ StateArgs fwd, const __grid_constant__ StateArgs rev, const Ragged seqs, const LinCut cut, uint32_t wait_limit, uint32_t stall) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) StateShared sh;
  if (blockIdx.y == 0) cut_states<KP, VP, false, !WALKED>(fwd, sh, aligned_base(smem_raw), seqs, cut, wait_limit, stall);
  else cut_states<KP, VP, true, true>(rev, sh, aligned_base(smem_raw), seqs, cut, wait_limit, stall);
}

// ---------------------------------------------------------------------------------------------------------------------------------------- host
// bf16 [rows, heads, d] with row pitch ld as a 3-D tensor: a box is 64 columns of one head in box_rows rows, zeros beyond the head's width and the last row.
bool make_tmap_heads(CUtensorMap* map, const void* ptr, int rows, int heads, int d, int64_t ld, int box_rows) {
  EncodeTiledFn fn = get_encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)rows};
  cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)ld * 2};
  cuuint32_t box[3] = {64, 1, (cuuint32_t)box_rows};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool make_walk(WalkArgs& a, const LinPass& p, const rom_ragged& seqs) {
  a.p = p;
  return make_tmap_heads(&a.q, p.q, seqs.rows, p.H / p.qdiv, p.dk, p.ldq, LT_C) && make_tmap_heads(&a.k, p.k, seqs.rows, p.H / p.kdiv, p.dk, p.ldk, LT_C) &&
         make_tmap_heads(&a.v, p.v, seqs.rows, p.H / p.vdiv, p.dv, p.ldv, LT_C);
}
template <typename K>
cudaError_t allow_smem(K kern, int bytes) { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes); }

template <int KP, int VP>
cudaError_t launch_states_shape(const LinPass* p, int n, const rom_ragged& seqs, const LinCut& cut, uint32_t limit, uint32_t stall, cudaStream_t st) {
  constexpr int smem = StateShape<KP, VP>::BYTES + 1024, rows = StateShape<KP, VP>::ROWS;
  StateArgs a[2];
  for (int i = 0; i < n; ++i) {
    a[i].p = p[i];
    if (!make_tmap_heads(&a[i].k, p[i].k, seqs.rows, p[i].H / p[i].kdiv, p[i].dk, p[i].ldk, rows) || !make_tmap_heads(&a[i].v, p[i].v, seqs.rows, p[i].H / p[i].vdiv, p[i].dv, p[i].ldv, rows))
      return cudaErrorInvalidValue;
  }
  auto kern = n > 1 ? lin_state_tc<KP, VP, true> : lin_state_tc<KP, VP, false>;
  const cudaError_t e = allow_smem(kern, smem);
  if (e != cudaSuccess) return e;
  count_launch();
  return launch_k(kern, dim3(cut.blocks - 1, n), LT_STATE_THREADS, smem, st, a[0], a[n - 1], device_view(seqs), cut, limit, stall);
}
template <int KP, int VP>
cudaError_t launch_walks_shape(const LinPass* p, int n, const rom_ragged& seqs, const LinCut& cut, uint32_t limit, uint32_t stall, cudaStream_t st) {
  WalkArgs a[3];
  for (int i = 0; i < n; ++i)
    if (!make_walk(a[i], p[i], seqs)) return cudaErrorInvalidValue;
  count_launch();
  if (n == 1) {
    constexpr int smem = WalkShape<KP, VP>::BYTES + 1024;
    auto kern = lin_walk_tc<KP, VP>;
    const cudaError_t e = allow_smem(kern, smem);
    return e != cudaSuccess ? e : launch_k(kern, dim3(cut.blocks), LT_WALK_THREADS, smem, st, a[0], device_view(seqs), cut, limit, stall);
  }
  constexpr int smem = more(WalkShape<KP, VP>::BYTES, WalkShape<VP, KP>::BYTES) + 1024;
  auto kern = lin_walk3_tc<KP, VP>;
  const cudaError_t e = allow_smem(kern, smem);
  return e != cudaSuccess ? e : launch_k(kern, dim3(cut.blocks, 3), LT_WALK_THREADS, smem, st, a[0], a[1], a[2], device_view(seqs), cut, limit, stall);
}

}  // namespace

// By the model's d_k and d_v.
cudaError_t launch_lin_states_tc(const LinPass* p, int n, int dk, int dv, const rom_ragged& seqs, const LinCut& cut, bool test_stall, cudaStream_t st) {
  const uint32_t limit = test_stall ? WAIT_LIMIT_TEST : WAIT_LIMIT, stall = test_stall ? 16 : 0;
  return (dk > 64 ? (dv > 64 ? launch_states_shape<128, 128> : launch_states_shape<128, 64>) : (dv > 64 ? launch_states_shape<64, 128> : launch_states_shape<64, 64>))(p, n, seqs, cut, limit, stall, st);
}
cudaError_t launch_lin_walks_tc(const LinPass* p, int n, int dk, int dv, const rom_ragged& seqs, const LinCut& cut, bool test_stall, cudaStream_t st) {
  const uint32_t limit = test_stall ? WAIT_LIMIT_TEST : WAIT_LIMIT, stall = test_stall ? 16 : 0;
  return (dk > 64 ? (dv > 64 ? launch_walks_shape<128, 128> : launch_walks_shape<128, 64>) : (dv > 64 ? launch_walks_shape<64, 128> : launch_walks_shape<64, 64>))(p, n, seqs, cut, limit, stall, st);
}

}  // namespace rom
