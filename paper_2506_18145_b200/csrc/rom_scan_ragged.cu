// Selective scan over packed sequences (rom_scan_ragged): h_t = exp(Delta A) h_{t-1} + B-bar u_t, y_t = (C_t h_t + D u_t) SiLU(z_t), each sequence
// from its slot's state or from zeros.
//
// The packed rows are cut into chunks of equal length whatever sequences they hold, so that the work is even for any lengths and the
// host needs to know none of them.  A sequence that reaches over a chunk's end needs its state there: a first launch runs the last sequence of every
// such chunk alone, states only (h_end from the sequence's own start, or from zeros and then with the sum of Delta); in the second, which
// computes the outputs, a chunk that begins inside a sequence chains those: h <- exp(A sum Delta) h + h_end (exact: the recurrence is
// linear in h).  A sequence inside one chunk is walked once.  The first launch also sets aside the initial state of a sequence that
// reaches on, because the chunk with its end may write the slot (in place) before the chunk with its start has read it.
//
// A warp owns 32 channels of one chunk, a lane 4 states of 4 adjacent channels in packed pairs along the channels (the layout of
// rom_scan_warp.cu, where the reasons stand): eight rows are staged in shared memory, whatever sequences they belong to, while the next eight
// are in registers, and the initial states of the next four sequences are on their way to shared memory.
//
// bf16: what bounds it is one exponential per state update on the special-function unit, 4.65 T a second: the first launch keeps it 82 %
// busy, the second 70 % (23 prompts of 8186 x 2048; then the fp32 pipe and the latency of twelve warps).  fp32: decay() keeps fp32 accuracy, about ten operations more an update.
// Measured: one sequence of 16384 rows x 4096 channels 681 us (231 us of exponentials, once; they are evaluated twice here; rom_scan, in
// one launch for sequences of one length, takes 538), 23 prompts of 8186 x 2048 in Euler form 164 us (58),
// 64 prompts of 16384 x 2048 318 us, 512 one-row sequences x 4096 53 us (4.9 TB/s: states in and out), fp32 531 rows of 37
// sequences x 512 19.8 us.  A call whose sequences all hold a NaN from their first row on: 16384 x 4096 1294 us.
// Tried: a tile that ends with its sequence (512 one-row sequences 70 us, waiting for every one's rows), one initial state ahead, chunk starts moved to a
// sequence's start a third of a chunk away (fewer rows in the first launch, uneven chunks: no gain), one warp per sequence (16384 rows: 21 ms),
// an eighth of the exponentials, or a quarter of the first launch's, as polynomials on the fp32 pipe (2 % less where the work is most, up to 7 % more elsewhere).
#include <cmath>
#include <type_traits>

#include "rom_serve.cuh"

namespace rom {
namespace {

constexpr int RR = 8;             // rows per tile
constexpr int RWARPS = 4;         // warps per block
constexpr int NEXT = 4;           // sequences whose initial states are on their way

struct RaggedScan {
  Ragged s;
  const void* u; const float* delta; const float* A; const float* Bm; const float* Cm; long long ldb; const float* D;
  const void* z; long long ldz; const float* h_in; float* h_out; void* y; int De;
  int Lc, nch;                    // rows per chunk, chunks
  int bc16;                       // rows of B and C on 16-byte boundaries
  int early;                      // the first launch's blocks all run at once: the second's may take the room they leave (1 to 2 % of calls of a few thousand rows)
  float* h_end;                   // [nch, De, 16]: state at the end of a chunk that a sequence reaches over
  float* h_start;                 // [nch, De, 16]: initial state of the sequence that starts in the chunk and reaches on
  float* sum_delta;               // [nch, De]
};

struct RaggedTile {
  float4 dl[RR][8], u[RR][8];     // Delta, u (times Delta without zero-order hold) of 4 channels; group g of row r sits at g ^ r
  float4 b[RR][4], c[RR][4];
  float D[32];
  float4 y[RR][32];               // partial sums of 4 channels over one lane's states
  float4 h0[NEXT][4][32];         // initial states of the sequences to come: channel i of the lane
  int4 next[NEXT];                // those sequences: first row, row behind the last, slot to read, slot to write (-1: none)
};

__device__ __forceinline__ float2 pair(float v) { return make_float2(v, v); }

// bf16, zero-order hold: with w = -B u / A a step is h <- a (h - w) + w, of which 1 - a is taken of w.  a is up to 2^-22 off, so the input (1 - a) w is off by
// that over |Delta A|: below kSmallStep, where it could be more than 2^-10, and for an infinite w (inf - inf) a row of the warp's
// channels is run with 1 - a by itself.  16384 rows x 4096 channels: 927 us when all rows are, 681 when none is, 18 of them for the look at the rows
// (as many with packed or three-operand minima).
// (A growing state, Delta < 0, has no such steps.)
constexpr float kSmallStep = 1.0f / 4096.0f, kLargeInput = 0x1p62f;
// a = 2^t, d = 1 - a for t <= 0, within 2^-14 of itself: the larger of the first two terms of its power series, which stay below it, and 1 - a less
// the 2^-22 that a may be off, and its rounding, which does too.  Up to |t| of about 2^-6 it is the series, then the difference.
__device__ __forceinline__ void decay_of_small_steps(float2 t, float2& a, float2& d) {
  constexpr float ln2 = 0.6931471805599453f;
  const float2 ds = __fmul2_rn(__ffma2_rn(t, pair(-ln2 * ln2 / 2.0f), pair(-ln2)), t);
  a = make_float2(ex2_ftz(t.x), ex2_ftz(t.y));
  const float2 dl = __ffma2_rn(a, pair(-1.0f), pair(1.0f - 0x1.4p-22f));
  d = make_float2(fmaxf(ds.x, dl.x), fmaxf(ds.y, dl.y));
}
// Slot of lane l's partial sums of row r: conflict-free for a quarter-warp of writers (eight lanes, one row) and of readers (lanes 8 g + const, two rows).
__device__ __forceinline__ int y_slot(int l, int r) { return l ^ (2 * (l >> 3) + (r & 1)); }

// Sequences base .. base+31 by lane: first row (the end of the last one behind it), slot to read (-1: zeros), slot to write (-1: none).
struct SeqWindow {
  int base, start, in, out;
  __device__ __forceinline__ void load(const RaggedScan& p, int from) {
    base = from;
    const int i = from + (threadIdx.x & 31), n = p.s.n_seq;
    start = i <= n ? p.s.start_of(i) : p.s.rows;
    const int sl = i < n ? p.s.slot_of(i) : -1;
    in = sl >= 0 && p.h_in && p.s.resumes(i) ? sl : -1;
    out = p.h_out ? sl : -1;
  }
  // the window holds sequences i and i + 1 (all lanes call it alike)
  __device__ __forceinline__ void reach(const RaggedScan& p, int i) { if (i - base >= 31) load(p, i); }
  __device__ __forceinline__ int start_of(int i) const { return __shfl_sync(0xffffffffu, start, i - base); }
  __device__ __forceinline__ int end_of(int i) const { return __shfl_sync(0xffffffffu, start, i + 1 - base); }
  __device__ __forceinline__ int in_of(int i) const { return __shfl_sync(0xffffffffu, in, i - base); }
  __device__ __forceinline__ int out_of(int i) const { return __shfl_sync(0xffffffffu, out, i - base); }
};

// The chained states of a warp, h <- 2^(a sum Delta) h + h_end over the chunks [k0, k1), where the plain product has given a NaN: none of a chunk's decays may be
// zero where their product is, and an infinite state then stays infinite, as it does step by step; nor does a state of zero
// become one by a product past the largest number.  The chunk's largest Delta tells whether a decay is zero.
__device__ __noinline__ void chain_not_finite(const float* h_end, const float* sum_delta, const float* delta, const float* A, int Lc, int De, int c0, int q, int k0, int k1,
                                              float4* v) {
  for (int k = k0; k < k1; ++k)
#pragma unroll 1
    for (int i = 0; i < 4; ++i) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(A + (size_t)(c0 + i) * 16) + q);
      const float4 e = *reinterpret_cast<const float4*>(h_end + ((size_t)k * De + c0 + i) * 16 + 4 * q);
      const float sum = sum_delta[(size_t)k * De + c0 + i];
      auto lost = [&](float av, float h) { return av * kLog2eServe * sum < -126.0f && isinf(h); };
      float most = -INFINITY;
      if (lost(a.x, v[i].x) || lost(a.y, v[i].y) || lost(a.z, v[i].z) || lost(a.w, v[i].w))
#pragma unroll 8
        for (int r = 0; r < Lc; ++r) most = fmaxf(most, __ldg(delta + ((size_t)k * Lc + r) * De + c0 + i));
      auto next = [&](float av, float h, float end) {
        const float P = ex2_ftz(av * kLog2eServe * sum);
        return fmaf(lost(av, h) && av * kLog2eServe * most >= -126.0f ? __int_as_float(1) : fminf(P, 3.402823466e38f), h, end);
      };
      v[i] = make_float4(next(a.x, v[i].x, e.x), next(a.y, v[i].y, e.y), next(a.z, v[i].z, e.z), next(a.w, v[i].w, e.w));
    }
}

// STATE: the first launch.
template <typename T, bool ZOH, bool STATE>
__global__ void __launch_bounds__(RWARPS * 32, sizeof(T) == 2 ? 3 : 2)
scan_ragged_chunks(const RaggedScan p) {
  constexpr bool FINE = sizeof(T) == 4;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  // (behind the first launch the second reads what that one writes from the chained states on only)
  const bool second = !STATE && p.nch > 1;
  if (!second) pdl_wait();
  if (STATE && p.early) pdl_trigger();
  const int lane = threadIdx.x & 31, De = p.De, groups = De / 32;
  const int item = blockIdx.x * RWARPS + (threadIdx.x >> 5), chunk = item / groups, c_warp = (item % groups) * 32;
  if (chunk >= (STATE ? p.nch - 1 : p.nch)) return;
  RaggedTile& s = reinterpret_cast<RaggedTile*>(smem_raw)[threadIdx.x >> 5];
  const int r0 = chunk * p.Lc, r1 = min(r0 + p.Lc, p.s.rows);
  // ---- what this warp walks
  int t, hi, cur_end, next = 0, cur_out = -1, cur_in = -1, first_chunk = chunk;
  bool reach = false;
  SeqWindow w;
  if (STATE) {
    const int q = p.s.first_from(r1) - 1;      // the last sequence that starts before the chunk's end
    if (q < 0) return;
    const int first = p.s.start_of(q);
    if (p.s.end_of(q) <= r1) return;
    t = max(first, r0); hi = r1; cur_end = r1;
    if (first >= r0) cur_in = p.h_in && p.s.resumes(q) ? p.s.slot_of(q) : -1;
  } else {
    next = p.s.first_from(r0);
    reach = chunk > 0 && next > 0 && p.s.end_of(next - 1) > r0;
    hi = min(r1, p.s.start_of(p.s.n_seq));
    w.load(p, max(next - 1, 0));
    if (reach) {
      w.reach(p, next - 1);
      cur_end = w.end_of(next - 1); cur_out = w.out_of(next - 1);
      first_chunk = min(w.start_of(next - 1) / p.Lc, chunk - 1);      // (offsets that descend stay in bounds)
      t = r0;
    } else {
      w.reach(p, next);
      t = next < p.s.n_seq ? w.start_of(next) : r1;
      cur_end = t;
    }
  }

  // ---- compute role: channels c0 .. c0+3 (pairs), states 4q .. 4q+3
  const int q = lane & 3, cg = lane >> 2, c0 = c_warp + 4 * cg;
  float2 a2[4][2], kin[4][2], h[4][2], sdel[2];
  float av[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 a4 = __ldg(reinterpret_cast<const float4*>(p.A + (size_t)(c0 + i) * 16) + q);
    av[i][0] = a4.x; av[i][1] = a4.y; av[i][2] = a4.z; av[i][3] = a4.w;
  }
  auto set_state = [&](const float4 (&v)[4]) {
    const float hv[4][4] = {{v[0].x, v[0].y, v[0].z, v[0].w}, {v[1].x, v[1].y, v[1].z, v[1].w}, {v[2].x, v[2].y, v[2].z, v[2].w}, {v[3].x, v[3].y, v[3].z, v[3].w}};
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) h[n][j] = make_float2(hv[2 * j][n], hv[2 * j + 1][n]);
  };
  auto state_at = [&](int i) { return (size_t)(c0 + i) * 16 + 4 * q; };      // within one sequence's or chunk's [De, 16]
  auto put_state = [&](float* dst) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      *reinterpret_cast<float4*>(dst + state_at(2 * j)) = make_float4(h[0][j].x, h[1][j].x, h[2][j].x, h[3][j].x);
      *reinterpret_cast<float4*>(dst + state_at(2 * j + 1)) = make_float4(h[0][j].y, h[1][j].y, h[2][j].y, h[3][j].y);
    }
  };
  const float4 zero4 = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float a = FINE ? 1.0f : kLog2eServe, k = FINE ? 1.0f : -1.0f;
      a2[n][j] = make_float2(av[2 * j][n] * a, av[2 * j + 1][n] * a);
      kin[n][j] = make_float2(k / av[2 * j][n], k / av[2 * j + 1][n]);
    }
  // the smallest Delta whose steps are not small, whatever the channel and state
  constexpr bool CAREFUL = ZOH && !FINE;
  float d_small = 0.0f;
  if (CAREFUL) {
    float least = fabsf(av[0][0]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int n = 0; n < 4; ++n) least = fminf(least, fabsf(av[i][n]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
    d_small = kSmallStep / least;
  }
  if (second) pdl_wait();
  {
    float4 v[4] = {zero4, zero4, zero4, zero4};
    if (STATE) {
      if (cur_in >= 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = *reinterpret_cast<const float4*>(p.h_in + (size_t)cur_in * De * 16 + state_at(i));
          *reinterpret_cast<float4*>(p.h_start + (size_t)chunk * De * 16 + state_at(i)) = v[i];
        }
      }
    } else if (reach) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const float4*>(p.h_end + (size_t)first_chunk * De * 16 + state_at(i));
      for (int k0 = first_chunk + 1; k0 < chunk; k0 += 4) {      // four chunks' loads in flight; past the last one: the identity
        float4 d4[4], e4[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const bool in = k0 + k < chunk;
          d4[k] = in ? *reinterpret_cast<const float4*>(p.sum_delta + (size_t)(k0 + k) * De + c0) : zero4;
#pragma unroll
          for (int i = 0; i < 4; ++i) e4[k][i] = in ? *reinterpret_cast<const float4*>(p.h_end + (size_t)(k0 + k) * De * 16 + state_at(i)) : zero4;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float dk[4] = {d4[k].x, d4[k].y, d4[k].z, d4[k].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float al[4] = {av[i][0] * kLog2eServe, av[i][1] * kLog2eServe, av[i][2] * kLog2eServe, av[i][3] * kLog2eServe};
            v[i].x = fmaf(ex2_ftz(al[0] * dk[i]), v[i].x, e4[k][i].x);
            v[i].y = fmaf(ex2_ftz(al[1] * dk[i]), v[i].y, e4[k][i].y);
            v[i].z = fmaf(ex2_ftz(al[2] * dk[i]), v[i].z, e4[k][i].z);
            v[i].w = fmaf(ex2_ftz(al[3] * dk[i]), v[i].w, e4[k][i].w);
          }
        }
      }
      float any = 0.0f;                                          // (a NaN is there to the end)
#pragma unroll
      for (int i = 0; i < 4; ++i) any += (v[i].x + v[i].y) + (v[i].z + v[i].w);
      if (any != any) {
        float4 again[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) again[i] = *reinterpret_cast<const float4*>(p.h_end + (size_t)first_chunk * De * 16 + state_at(i));
        chain_not_finite(p.h_end, p.sum_delta, p.delta, p.A, p.Lc, De, c0, q, first_chunk + 1, chunk, again);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = again[i];
      }
    }
    set_state(v);
  }
  sdel[0] = make_float2(0.0f, 0.0f); sdel[1] = sdel[0];

  if (!STATE) {
    s.D[lane] = p.D ? __ldg(p.D + c_warp + lane) : 0.0f;
    // sequences without a row that lie in this chunk (the last chunk: behind the last row too): their state is the initial one
    for (int b = next; b < p.s.n_seq; b += 31) {
      w.load(p, b);
      const int after = __shfl_down_sync(0xffffffffu, w.start, 1);
      const bool mine = lane < 31 && b + lane < p.s.n_seq && (w.start < r1 || chunk == p.nch - 1);
      unsigned m = __ballot_sync(0xffffffffu, mine && after <= w.start && w.out >= 0);
      while (m) {
        const int i = b + __ffs(m) - 1, in = w.in_of(i), out = w.out_of(i);
        m &= m - 1;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          *reinterpret_cast<float4*>(p.h_out + (size_t)out * De * 16 + state_at(k)) =
              in >= 0 ? *reinterpret_cast<const float4*>(p.h_in + (size_t)in * De * 16 + state_at(k)) : zero4;
      }
      if (!__all_sync(0xffffffffu, mine || lane == 31)) break;
    }
    w.load(p, next);
  }
  // the next sequence with rows into place `at` of the ring, its initial state on the way to shared memory
  auto look_ahead = [&](int at) {
    int4 e = make_int4(0x7fffffff, 0x7fffffff, -1, -1);
    while (next < p.s.n_seq) {
      w.reach(p, next);
      const int first = w.start_of(next), end = w.end_of(next);
      if (end > first) {
        e = make_int4(first, end, w.in_of(next), w.out_of(next));
        ++next;
        break;
      }
      ++next;
    }
    if (e.z >= 0 && e.x < r1) {
      const float* src = e.y > r1 ? p.h_start + (size_t)chunk * De * 16 : p.h_in + (size_t)e.z * De * 16;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(&s.h0[at][i][lane])), "l"(src + state_at(i)) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    if (lane == 0) s.next[at] = e;
  };
  int head = 0;
  if (!STATE) {
#pragma unroll 1
    for (int i = 0; i < NEXT; ++i) look_ahead(i);
    __syncwarp();
  }

  // ---- loader / output role: row lt of every tile, channels lc .. lc+7 (four lanes per row: a quarter-warp touches two rows of global memory)
  const int lt = lane >> 2, l8 = lane & 3, lc = c_warp + 8 * l8;
  const T* __restrict__ up = static_cast<const T*>(p.u) + lc;
  const T* __restrict__ zp = STATE ? nullptr : static_cast<const T*>(p.z);
  const float* __restrict__ dp = p.delta + lc;
  Raw8<float> r_d;
  Raw8<T> r_u, r_z, cur_u, cur_z;
  float4 r_b, r_c;
  auto bc_row = [&](const float* v, size_t row) {
    const float* at = v + row * p.ldb + 4 * l8;
    return p.bc16 ? __ldg(reinterpret_cast<const float4*>(at)) : make_float4(__ldg(at), __ldg(at + 1), __ldg(at + 2), __ldg(at + 3));
  };
  auto fetch = [&](int t0, int m) {
    if (lt < m) {
      const size_t row = t0 + lt;
      r_d.load(dp + row * De);
      r_u.load(up + row * De);
      r_b = bc_row(p.Bm, row);
      if (!STATE) {
        r_c = bc_row(p.Cm, row);
        if (zp) r_z.load(zp + row * p.ldz + lc);
      }
    } else {                      // rows past the tile's end change nothing
      r_d.zero(); r_u.zero();
      r_b = zero4; r_c = zero4;
    }
  };
  bool running = STATE || reach;
  // the sequence that starts at the present row takes over
  auto enter = [&]() {
    if (running && cur_out >= 0) put_state(p.h_out + (size_t)cur_out * De * 16);
    const int4 e = s.next[head];
    asm volatile("cp.async.wait_group %0;" ::"n"(NEXT - 1) : "memory");
    float4 v[4] = {zero4, zero4, zero4, zero4};
    if (e.z >= 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = s.h0[head][i][lane];
    set_state(v);
    running = true; cur_end = e.y; cur_out = e.w;
    __syncwarp();
    look_ahead(head);
    __syncwarp();
    if (++head == NEXT) head = 0;
  };
  if (t < hi) fetch(t, min(RR, hi - t));
  while (t < hi) {
    const int m = min(RR, hi - t), t_next = t + m;
    unsigned careful = 0;         // four bits a row
    {
      float d[8], uu[8];
      r_d.get(d); r_u.get(uu);
      if (CAREFUL) {
        float least = d[0], most = fmaxf(fmaxf(fabsf(r_b.x), fabsf(r_b.y)), fmaxf(fabsf(r_b.z), fabsf(r_b.w)));
#pragma unroll
        for (int i = 0; i < 8; ++i) { least = fminf(least, d[i]); most = fmaxf(most, fabsf(uu[i])); }
        careful = __ballot_sync(0xffffffffu, lt < m && least >= 0.0f && (least < d_small || most >= kLargeInput));
      }
      if (!ZOH) {                 // B-bar = Delta B: the input enters as Delta u
#pragma unroll
        for (int i = 0; i < 8; ++i) uu[i] *= d[i];
      }
      s.dl[lt][(2 * l8) ^ lt] = make_float4(d[0], d[1], d[2], d[3]);
      s.dl[lt][(2 * l8 + 1) ^ lt] = make_float4(d[4], d[5], d[6], d[7]);
      s.u[lt][(2 * l8) ^ lt] = make_float4(uu[0], uu[1], uu[2], uu[3]);
      s.u[lt][(2 * l8 + 1) ^ lt] = make_float4(uu[4], uu[5], uu[6], uu[7]);
      s.b[lt][l8] = r_b;
      if (!STATE) { s.c[lt][l8] = r_c; cur_u = r_u; cur_z = r_z; }
    }
    __syncwarp();
    if (t_next < hi) fetch(t_next, min(RR, hi - t_next));
    if (!STATE && t >= cur_end) enter();
    // one row; its operands have been requested, those of row `ahead` are before this row's arithmetic: a load issued behind a row's exponentials
    // waits for all of them
    float4 nd = s.dl[0][cg], nu = s.u[0][cg], nb = s.b[0][q], nc = STATE ? zero4 : s.c[0][q];
    auto row = [&](int r, int ahead, auto careful_tag) {
      const float4 d4 = nd, u4 = nu, b4 = nb, c4 = nc;
      nd = s.dl[ahead][cg ^ ahead]; nu = s.u[ahead][cg ^ ahead]; nb = s.b[ahead][q];
      if (!STATE) nc = s.c[ahead][q];
      const float2 dl[2] = {make_float2(d4.x, d4.y), make_float2(d4.z, d4.w)}, uu[2] = {make_float2(u4.x, u4.y), make_float2(u4.z, u4.w)};
      const float bb[4] = {b4.x, b4.y, b4.z, b4.w}, cc[4] = {c4.x, c4.y, c4.z, c4.w};
      float2 acc[2];
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 x = __fmul2_rn(dl[j], a2[n][j]);
          const float2 uB = __fmul2_rn(uu[j], pair(bb[n]));
          if (FINE) {
            float2 a, e;
            decay(x, a, e);
            h[n][j] = __ffma2_rn(a, h[n][j], ZOH ? __fmul2_rn(e, __fmul2_rn(uB, kin[n][j])) : uB);
          } else if (decltype(careful_tag)::value) {
            float2 a, d;
            decay_of_small_steps(x, a, d);
            h[n][j] = __ffma2_rn(a, h[n][j], __fmul2_rn(d, __fmul2_rn(uB, kin[n][j])));
          } else {
            const float2 a = make_float2(ex2_ftz(x.x), ex2_ftz(x.y));
            if (ZOH) {            // w = -B u / A, h <- a (h - w) + w
              const float2 v = __fmul2_rn(uB, kin[n][j]);
              h[n][j] = __ffma2_rn(a, __ffma2_rn(v, pair(-1.0f), h[n][j]), v);
            } else {
              h[n][j] = __ffma2_rn(a, h[n][j], uB);
            }
          }
          if (!STATE) acc[j] = n == 0 ? __fmul2_rn(pair(cc[n]), h[n][j]) : __ffma2_rn(pair(cc[n]), h[n][j], acc[j]);
        }
      if (STATE) { sdel[0] = __fadd2_rn(sdel[0], dl[0]); sdel[1] = __fadd2_rn(sdel[1], dl[1]); }
      else s.y[r][y_slot(lane, r)] = make_float4(acc[0].x, acc[0].y, acc[1].x, acc[1].y);
    };
    constexpr int UF = FINE ? 2 : STATE ? 4 : RR, UC = 4;
    const bool whole = m == RR && (STATE || cur_end >= t_next);
    unsigned each = careful | careful >> 2;
    each = (each | each >> 1) & 0x11111111u;
    if (whole && !careful) {
#pragma unroll UF
      for (int r = 0; r < RR; ++r) row(r, min(r + 1, RR - 1), std::false_type{});
    } else if (CAREFUL && whole && each == 0x11111111u) {
#pragma unroll UC
      for (int r = 0; r < RR; ++r) row(r, min(r + 1, RR - 1), std::bool_constant<CAREFUL>{});
    } else {                      // the chunk's last rows, sequences that end here, rows that need care
#pragma unroll 1
      for (int r = 0; r < m; ++r) {
        if (!STATE && t + r >= cur_end) enter();
        if (CAREFUL && ((each >> (4 * r)) & 1u)) row(r, min(r + 1, RR - 1), std::bool_constant<CAREFUL>{});
        else row(r, min(r + 1, RR - 1), std::false_type{});
      }
    }
    __syncwarp();
    if (!STATE) {
      if (lt < m) {               // y = (sum over the four lanes + D u) * gate, rounded
        float o[8], uu[8], zz[8];
        cur_u.get(uu);
        if (zp) {
          cur_z.get(zz);
#pragma unroll
          for (int i = 0; i < 8; ++i) zz[i] = FINE ? silu_f(zz[i]) : silu_fast(zz[i]);
        }
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const int g4 = 8 * l8 + 4 * hf;
          const float4 x0 = s.y[lt][y_slot(g4, lt)], x1 = s.y[lt][y_slot(g4 + 1, lt)], x2 = s.y[lt][y_slot(g4 + 2, lt)], x3 = s.y[lt][y_slot(g4 + 3, lt)];
          const float4 D4 = reinterpret_cast<const float4*>(s.D)[2 * l8 + hf];
          float2 v0 = __fadd2_rn(__fadd2_rn(make_float2(x0.x, x0.y), make_float2(x1.x, x1.y)), __fadd2_rn(make_float2(x2.x, x2.y), make_float2(x3.x, x3.y)));
          float2 v1 = __fadd2_rn(__fadd2_rn(make_float2(x0.z, x0.w), make_float2(x1.z, x1.w)), __fadd2_rn(make_float2(x2.z, x2.w), make_float2(x3.z, x3.w)));
          v0 = __ffma2_rn(make_float2(D4.x, D4.y), make_float2(uu[4 * hf], uu[4 * hf + 1]), v0);
          v1 = __ffma2_rn(make_float2(D4.z, D4.w), make_float2(uu[4 * hf + 2], uu[4 * hf + 3]), v1);
          if (zp) {
            v0 = __fmul2_rn(v0, make_float2(zz[4 * hf], zz[4 * hf + 1]));
            v1 = __fmul2_rn(v1, make_float2(zz[4 * hf + 2], zz[4 * hf + 3]));
          }
          o[4 * hf] = v0.x; o[4 * hf + 1] = v0.y; o[4 * hf + 2] = v1.x; o[4 * hf + 3] = v1.y;
        }
        Raw8<T>::store(static_cast<T*>(p.y) + (size_t)(t + lt) * De + lc, o);
      }
      __syncwarp();
    }
    t = t_next;
  }
  if (STATE) {
    put_state(p.h_end + (size_t)chunk * De * 16);
    if (q == 0) *reinterpret_cast<float4*>(p.sum_delta + (size_t)chunk * De + c0) = make_float4(sdel[0].x, sdel[0].y, sdel[1].x, sdel[1].y);
  } else if (running && cur_end <= r1 && cur_out >= 0) {
    put_state(p.h_out + (size_t)cur_out * De * 16);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

// Rows of a chunk when there are n of them.
int chunk_rows(int rows, int n) { return n == 1 ? (rows > 0 ? rows : 1) : (int)align_up((size_t)(rows + n - 1) / n, RR); }
// Chunks that packed rows may be cut into.
int most_chunks(int De, int rows) {
  int n = 148 * 12 * 6 / (De / 32);
  if (n > 512) n = 512;
  if (n > rows / 8) n = rows / 8;
  return n > 1 ? n : 1;
}
// Chunks of the packed rows: the count with the smallest time by what the kernels were measured to take.  A block of four warps takes
// 155 / 235 / 330 ns a row with one / two / three of them on an SM, 128 / 188 / 255 ns states only; more than three come in rounds, of which the last
// may be of one or two.  fp32: two on an SM, about twice as long.  A warp takes 3 us before its first row, 0.1 us for every chunk that it chains,
// 0.4 us from one sequence to the next.  The first launch walks the rows of sequences that reach over a chunk's end, of one of length `mean` about
// mean (1 - exp(-Lc / mean)) on average over rounds, twice the mean at most where all blocks run at once.  A function of the sizes alone, so that workspace sizing and the launch agree.
int ragged_chunks(int De, int n_seq, int rows, bool fp32) {
  const double full[3] = {155.0, 235.0, 330.0}, state[3] = {128.0, 188.0, 255.0};
  const double mean = rows > 0 && n_seq > 0 ? (double)rows / n_seq : 1.0;
  const int most = fp32 ? 2 : 3;
  // blocks that each take fixed + rows_each * pace ns
  auto time = [&](double blocks, const double (&pace)[3], double rows_each, double fixed) {
    const double slow = fp32 ? 2.0 : 1.0;
    const int per_sm = (int)ceil(blocks / 148.0), last = per_sm % most;
    return per_sm / most * (fixed + rows_each * pace[most - 1] * slow) + (last ? fixed + rows_each * pace[last - 1] * slow : 0.0);
  };
  int best = 1;
  double best_t = 0.0;
  for (int n = 1; n <= most_chunks(De, rows); n += 1 + n / 16) {      // (a few us on the host at most)
    const double Lc = chunk_rows(rows, n), nch = rows > 0 ? ceil(rows / Lc) : 1.0;
    const double chained = mean < Lc ? 0.0 : mean / Lc < nch ? mean / Lc : nch;
    double t = time(nch * (De / 32) / RWARPS, full, Lc, 3000.0 + 100.0 * chained + 400.0 * Lc / mean);
    if (n > 1) {
      const double blocks = (nch - 1.0) * (De / 32) / RWARPS, longest = 2.0 * mean < Lc ? 2.0 * mean : Lc;
      t += time(blocks, state, blocks <= 148.0 * most ? longest : mean * (1.0 - exp(-Lc / mean)), 2000.0) + 3000.0;
    }
    if (n == 1 || t < best_t) { best = n; best_t = t; }
  }
  return best;
}
struct RaggedWs { int Lc, nch, early; size_t h_end, h_start, sum_delta, total; };
RaggedWs ragged_ws(const rom_config& c, int n_seq, int rows) {
  const int De = c.d_inner;
  RaggedWs l{};
  const int n = ragged_chunks(De, n_seq, rows, c.dtype == ROM_F32);
  l.Lc = chunk_rows(rows, n);
  l.nch = rows > 0 ? (rows + l.Lc - 1) / l.Lc : 1;
  l.early = (long long)l.nch * (De / 32) <= 148ll * RWARPS * (c.dtype == ROM_F32 ? 2 : 3);
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = align_up(o + bytes, 256); return at; };      // (within total: nch is most_chunks at most)
  const size_t keep = l.nch > 1 ? l.nch : 0;
  l.h_end = take(keep * De * 16 * sizeof(float));
  l.h_start = take(keep * De * 16 * sizeof(float));
  l.sum_delta = take(keep * De * sizeof(float));
  // What any number of sequences and rows up to these may take: a buffer for the largest batch does for all smaller ones, whose chunks may be more.
  const size_t most = most_chunks(De, rows);
  l.total = most > 1 ? 2 * align_up(most * De * 16 * sizeof(float), 256) + align_up(most * De * sizeof(float), 256) : 256;
  return l;
}

template <typename T, bool ZOH>
cudaError_t launch_scan_ragged(const RaggedScan& p, cudaStream_t st) {
  constexpr int smem = RWARPS * (int)sizeof(RaggedTile);
  cudaError_t e = cudaFuncSetAttribute(scan_ragged_chunks<T, ZOH, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(scan_ragged_chunks<T, ZOH, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const long long groups = p.De / 32;
  auto blocks = [&](long long chunks) { return dim3((unsigned)((chunks * groups + RWARPS - 1) / RWARPS)); };
  if (p.nch > 1) {
    if ((e = launch_k(scan_ragged_chunks<T, ZOH, true>, blocks(p.nch - 1), RWARPS * 32, smem, st, p)) != cudaSuccess) return e;
    count_launch();
  }
  count_launch();
  return launch_k(scan_ragged_chunks<T, ZOH, false>, blocks(p.nch), RWARPS * 32, smem, st, p);
}

}  // namespace
}  // namespace rom

using namespace rom;

extern "C" {

int rom_scan_ragged_workspace_size(const rom_config* cfg, int32_t n_seq, int32_t rows, size_t* bytes) {
  if (!bytes || n_seq < 0 || rows < 0) return ROM_ERR_INVALID_ARG;
  const int rc = check_config(cfg, 2);
  if (rc != ROM_OK) return rc;
  if (n_seq > kMaxRaggedSeqs || rows >= 1 << 30) return ROM_ERR_UNSUPPORTED;
  *bytes = ragged_ws(*cfg, n_seq, rows).total;
  return ROM_OK;
}

int rom_scan_ragged(const rom_config* cfg, const rom_ragged* seqs, const void* u, const float* delta, const float* A, const float* Bm,
                    const float* Cm, int64_t ld_bc, const float* D, const void* z, int64_t ldz, const float* h_in, float* h_out, void* y, void* ws,
                    size_t ws_bytes, void* stream) {
  int rc = check_config(cfg, 2);
  if (rc != ROM_OK) return rc;
  const rom_config& c = *cfg;
  if ((rc = check_ragged(seqs)) != ROM_OK) return rc;
  if (seqs->n_seq == 0) return ROM_OK;
  const size_t esz = c.dtype == ROM_BF16 ? 2 : 4;
  if (!A || !ws || (seqs->rows > 0 && (!u || !delta || !Bm || !Cm || !y))) return ROM_ERR_INVALID_ARG;
  if (ld_bc < c.d_state || (z && !pitch_ok(ldz, c.d_inner, esz))) return ROM_ERR_INVALID_ARG;
  const void* ptrs[] = {u, delta, A, z, y, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return ROM_ERR_INVALID_ARG;
  if (!aligned4(D) || !aligned4(Bm) || !aligned4(Cm)) return ROM_ERR_INVALID_ARG;
  if (!pools_ok(h_in, h_out, (size_t)seqs->n_slots * c.d_inner * c.d_state)) return ROM_ERR_INVALID_ARG;
  const RaggedWs lay = ragged_ws(c, seqs->n_seq, seqs->rows);
  if (ws_bytes < lay.total) return ROM_ERR_WORKSPACE;
  if ((rc = check_device()) != ROM_OK) return rc;
  LaunchCounter::count = 0;
  char* W = static_cast<char*>(ws);
  const int bc16 = aligned16(Bm) && aligned16(Cm) && ld_bc % 4 == 0;
  const RaggedScan p{device_view(*seqs), u, delta, A, Bm, Cm, ld_bc, D, z, ldz, h_in, h_out, y, c.d_inner, lay.Lc, lay.nch, bc16, lay.early,
                     reinterpret_cast<float*>(W + lay.h_end), reinterpret_cast<float*>(W + lay.h_start), reinterpret_cast<float*>(W + lay.sum_delta)};
  auto launch = c.dtype == ROM_BF16 ? (c.disc_mode == 0 ? launch_scan_ragged<__nv_bfloat16, true> : launch_scan_ragged<__nv_bfloat16, false>)
                                    : (c.disc_mode == 0 ? launch_scan_ragged<float, true> : launch_scan_ragged<float, false>);
  return launch(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

}  // extern "C"
