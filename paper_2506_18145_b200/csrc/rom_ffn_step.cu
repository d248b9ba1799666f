// FFN-MoE of the few tokens of a generation step (rom_ffn_moe_step): out_t = sum_k g_tk W_down,e (SiLU(W_gate,e x_t) * (W_up,e x_t)), e = topk_idx[t, k].
// Two launches: hidden rows g SiLU(gate) up of every assignment (token, slot), then the down projection with the sum over the slots in fp32.  In bf16
// a hidden row is kept as the sum of two bf16 numbers, high and low, 2^-16 off at most: rounded to one it added as much to the error as the output's own
// rounding (2.4e-3 of the outputs against 1.7e-3).  Both are columns of the same MMA, which takes as long for 32 columns as for 16.
//
// What bounds it: the chosen experts' weights, 6 d_model d_ff bytes each (bf16), read once.  rom_ffn_moe_forward takes five launches and pads every
// expert's tokens to 128 rows.  Here the weights are the M = 128 operand of tcgen05 and an expert's tokens (their halves) its 16, 32 or 64 columns: one CTA per SM
// walks (expert, weight rows, part of the contracted index) tiles; warp 0 keeps a ring of stages of 128 contracted elements full by TMA, warps 6..9
// put the tokens' rows beside them, warp 1 issues the MMAs, warps 2..5 take the accumulators (two, so that a tile's end runs beside the next tile).  The
// down projection, of few rows and a long contracted index, is cut along that index too: the parts go to the workspace and whoever brings
// a tile's last one adds them all, in the order of slots and parts, so that results do not depend on who came when.
// Measured (us a call, GB/s of the chosen experts' weights): one token of 2048 x 8192 25.9 (3890), 64 tokens with two of sixteen experts 262 (6140: 94 % of the
// measured copy), 16 tokens with two of eight 130 (6170), 8 tokens with one of eight of 1280 x 5120 43.3 (4760).  Small calls: about 10 us of launches, lists and
// first loads.  With 32 and more tokens an
// expert the MMAs bound it, and the down projection goes over its weights once for every 32 tokens: 64 tokens of one expert each of two 66 us (2.8 TB/s).  Tried: rings of half the size, so that both launches share the SMs and the second has its first weights when the first ends, no gain (the MMAs
// of short tiles bound it then); stages of 64 elements 264 and 29 us, of one 64-wide block a warp's turn each 0.37 us a stage.
//
// fp32: a warp has four weight rows and up to eight tokens, products over its lanes; the plain form for a small model in full precision.  Bound by the latency
// of the loads (activations from the L1 and L2 as often as weights): 5 tokens of 256 x 1024 9.6 us, 40 with two of sixteen of 512 x 2048 88 (2270 GB/s of weights).
// Tried: weights by cp.async three steps ahead through shared memory 79 to 85 for the second but 10.2 to 10.9 for the first and 5 to 14 % more at sixteen tokens an
// expert (less L1 for the activations); activations a step ahead 135; the down projection's weights asked for before the wait, 1 %.
#include <algorithm>
#include <type_traits>

#include "rom_serve.cuh"
#include "rom_tc_ptx.cuh"

namespace rom {
namespace {

typedef __nv_bfloat16 bf16;
constexpr int kFfnStepTokens = 64, kFfnStepAssign = kFfnStepTokens * kMaxK;
constexpr int kFfnMaxTiles = 1024;       // row tiles of the down projection
constexpr int kFfnMaxSplits = 16;

struct FfnStep {
  const void* x; const void* W_gu; const void* W_down; const int32_t* idx; const float* gates; void* out;
  void* hid;                // fp32: [B K, d_ff]; bf16: [B K, 2, d_ff], high and low halves
  int32_t* status;
  int T, K, E, Dm, F;
};

// Assignments by expert.  An expert's list is in ascending order, so that the order of every sum is fixed.
struct ByExpert {
  int off[kMaxE + 1];
  short list[kFfnStepAssign];
  signed char of[kFfnStepAssign];      // expert of an assignment, -1: none
  // all threads of the block; ends with a barrier
  __device__ __forceinline__ void build(const int32_t* idx, int A, int E) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    for (int a = threadIdx.x; a < A; a += blockDim.x) {
      const int e = __ldg(idx + a);
      of[a] = e >= 0 && e < E ? (signed char)e : (signed char)-1;
    }
    __syncthreads();
    for (int e = warp; e <= E; e += warps) {
      int n = 0;                       // assignments of the experts before e
      for (int a0 = 0; a0 < A; a0 += 32) n += __popc(__ballot_sync(0xffffffffu, a0 + lane < A && of[a0 + lane] >= 0 && of[a0 + lane] < e));
      if (lane == 0) off[e] = n;
      if (e == E) break;
      for (int a0 = 0; a0 < A; a0 += 32) {
        const unsigned m = __ballot_sync(0xffffffffu, a0 + lane < A && of[a0 + lane] == e);
        if ((m >> lane) & 1u) list[n + __popc(m & ((1u << lane) - 1u))] = (short)(a0 + lane);
        n += __popc(m);
      }
    }
    __syncthreads();
  }
  // the i-th expert that somebody chose, -1: there are fewer
  __device__ __forceinline__ int chosen(int i, int E) const {
    for (int e = 0; e < E; ++e)
      if (off[e + 1] > off[e] && i-- == 0) return e;
    return -1;
  }
};
// The status word of the call: cleared, or an expert index beyond the last one.
__device__ __forceinline__ void ffn_status(const FfnStep& p) {
  bool bad = false;
  for (int a = threadIdx.x; a < p.T * p.K; a += blockDim.x) bad |= __ldg(p.idx + a) >= p.E;
  bad = __syncthreads_or(bad);
  if (threadIdx.x < kStatusInts) p.status[threadIdx.x] = threadIdx.x == kStatCode && bad ? ROM_ERR_INVALID_ARG : 0;
}

// Sums of v[i], i < 32, over the lanes: lane i keeps the i-th.
__device__ __forceinline__ float sum_to_lane(float (&v)[32]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    const bool up = lane & s;
#pragma unroll
    for (int i = 0; i < s; ++i) {
      const float give = up ? v[i] : v[s + i], keep = up ? v[s + i] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, give, s);
    }
  }
  return v[0];
}

// ---------------------------------------------------------------------------------------------- fp32
// Four weight rows times up to eight rows of activations, elements [k0, k1), over the lanes of a warp; lane 8 r + j gets row r times activation j.
__device__ __forceinline__ float rows_4x8(const float* const (&w)[4], const float* const (&x)[8], int n, int k0, int k1) {
  constexpr int V = 4;
  const int lane = threadIdx.x & 31;
  float acc[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) acc[i] = 0.0f;
  V16<float> next[4];                  // the weights a round ahead
  int k = k0 + lane * V;
  if (k < k1)
#pragma unroll
    for (int r = 0; r < 4; ++r) next[r].load(w[r] + k);
  for (; k < k1; k += 32 * V) {
    float wv[4][V];
    float4 xq[8];
#pragma unroll
    for (int r = 0; r < 4; ++r) next[r].get(wv[r]);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) xq[j] = *reinterpret_cast<const float4*>(x[j] + k);
    if (k + 32 * V < k1)
#pragma unroll
      for (int r = 0; r < 4; ++r) next[r].load(w[r] + k + 32 * V);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= n) break;
      const float xv[V] = {xq[j].x, xq[j].y, xq[j].z, xq[j].w};
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[8 * r + j] = fmaf(wv[r][i], xv[i], acc[8 * r + j]);
    }
  }
  return sum_to_lane(acc);
}

// A warp has two hidden columns of one expert at a time.  Four blocks an SM for the loads' latency, though a few registers are spilled (three: 6 to 17 % longer).
constexpr int FR_UP_WARPS = 4;
__global__ void __launch_bounds__(FR_UP_WARPS * 32, 4)
ffn_step_up(const FfnStep p) {
  __shared__ ByExpert by;
  pdl_sync();
  if (blockIdx.x == 0 && blockIdx.y == 0) ffn_status(p);
  by.build(p.idx, p.T * p.K, p.E);
  const int lane = threadIdx.x & 31, j = lane & 7, e = by.chosen(blockIdx.y, p.E);
  if (e < 0) return;
  for (int f = (blockIdx.x * FR_UP_WARPS + (threadIdx.x >> 5)) * 2; f < p.F; f += gridDim.x * FR_UP_WARPS * 2) {
    const float* g = static_cast<const float*>(p.W_gu) + ((size_t)e * 2 * p.F + f) * p.Dm;
    const float* u = g + (size_t)p.F * p.Dm;
    const float* const w[4] = {g, g + p.Dm, u, u + p.Dm};
    for (int a0 = by.off[e]; a0 < by.off[e + 1]; a0 += 8) {
      const int n = min(8, by.off[e + 1] - a0);
      const float* x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = static_cast<const float*>(p.x) + (size_t)(by.list[a0 + min(i, n - 1)] / p.K) * p.Dm;
      const float v = rows_4x8(w, x, n, 0, p.Dm);
      const float up = __shfl_down_sync(0xffffffffu, v, 16);
      if (lane < 16 && j < n) {
        const int a = by.list[a0 + j];
        static_cast<float*>(p.hid)[(size_t)a * p.F + f + (lane >> 3)] = silu_f(v) * up * __ldg(p.gates + a);
      }
    }
  }
}
// A block has four rows of the output; its warps share the contracted index of every expert, two sets of them the experts, and add their sums at the
// end, in order.
constexpr int FR_PARTS = 8, FR_DOWN_WARPS = 2 * FR_PARTS;
__global__ void __launch_bounds__(FR_DOWN_WARPS * 32)
ffn_step_down(const FfnStep p) {
  __shared__ ByExpert by;
  __shared__ float sum[FR_DOWN_WARPS][kFfnStepTokens][4];
  by.build(p.idx, p.T * p.K, p.E);
  pdl_sync();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, d = blockIdx.x * 4;
  const int part = (p.F / 128 + FR_PARTS - 1) / FR_PARTS * 128, k0 = min(warp % FR_PARTS * part, p.F), k1 = min(k0 + part, p.F);
  float (*s)[4] = sum[warp];
  for (int t = lane; t < p.T * 4; t += 32) s[t >> 2][t & 3] = 0.0f;
  __syncwarp();
  int turn = warp / FR_PARTS;
  for (int e = 0; e < p.E && k0 < k1; ++e) {
    if (by.off[e] == by.off[e + 1] || (turn++ & 1)) continue;      // (every second chosen expert)
    const float* w0 = static_cast<const float*>(p.W_down) + ((size_t)e * p.Dm + d) * p.F;
    const float* const w[4] = {w0, w0 + p.F, w0 + 2 * (size_t)p.F, w0 + 3 * (size_t)p.F};
    for (int a0 = by.off[e]; a0 < by.off[e + 1]; a0 += 8) {
      const int n = min(8, by.off[e + 1] - a0);
      const float* x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = static_cast<const float*>(p.hid) + (size_t)by.list[a0 + min(i, n - 1)] * p.F;
      const float v = rows_4x8(w, x, n, k0, k1);
      for (int i = 0; i < n; ++i) {      // one at a time: two of them may be of one token
        if ((lane & 7) == i) s[by.list[a0 + i] / p.K][lane >> 3] += v;
        __syncwarp();
      }
    }
  }
  __syncthreads();
  for (int t = threadIdx.x; t < p.T * 4; t += FR_DOWN_WARPS * 32) {
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < FR_DOWN_WARPS; ++w) v += sum[w][t >> 2][t & 3];
    static_cast<float*>(p.out)[(size_t)(t >> 2) * p.Dm + d + (t & 3)] = v;
  }
}

cudaError_t launch_ffn_rows(const FfnStep& p, cudaStream_t st) {
  const int A = p.T * p.K;
  // (about eight blocks an SM at most: each makes its lists first)
  const int experts = A < p.E ? A : p.E, blocks = std::min(p.F / (2 * FR_UP_WARPS), std::max(148 * 8 / experts, 1));
  cudaError_t e = launch_k(ffn_step_up, dim3(blocks, experts), FR_UP_WARPS * 32, 0, st, p);
  if (e != cudaSuccess) return e;
  count_launch();
  e = launch_k(ffn_step_down, dim3(p.Dm / 4), FR_DOWN_WARPS * 32, 0, st, p);
  count_launch();
  return e;
}

// ---------------------------------------------------------------------------------------------- bf16: streamed weights
// Experts that T tokens with K choices each of E name, about.
int chosen_experts(int T, int K, int E) {
  double none = 1.0;
  for (int t = 0; t < T; ++t) none *= 1.0 - (double)K / E;
  const int n = (int)(E * (1.0 - none) + 0.5);
  return n < 1 ? 1 : n;
}
constexpr int kSizingSms = 148;      // (workspace sizing and the launch agree)
constexpr int FT_COLS = 64;                          // columns per pass at most
// Columns of a token: the down projection has the high and the low half of a hidden row, which add up to it within 2^-16, as two columns of the same MMA.
__host__ __device__ constexpr int ffn_per_token(bool up) { return up ? 1 : 2; }
constexpr int FT_MIN_STAGES = 4, FT_MAX_STAGES = 12;      // (a stage for each of the four warps that bring token rows)
constexpr int FT_KB = 2, FT_K = FT_KB * BLOCK_K;     // contracted elements per stage: two swizzled rows
constexpr int FT_SMEM = 208 * 1024;                  // operand ring
constexpr int FT_THREADS = 320;
// Bytes of a ring: its alignment, its stages, and what the MMA reads past the last one (always 128 rows from a tile's start).
constexpr int ffn_ring(int rows, int cols, int stages) {
  return 1024 + stages * FT_KB * (rows + cols) * 128 + std::max(128 * 128 - (rows + FT_KB * cols) * 128, 0);
}
constexpr int ffn_stages(int rows, int cols) {
  return std::min((FT_SMEM - ffn_ring(rows, cols, 0)) / (FT_KB * (rows + cols) * 128), FT_MAX_STAGES);
}
// Tokens of a stage: room for twice an expert's mean and eight more (down, where a token is two columns: half as much again and four more, at most 32);
// whoever has more than that many streams its weights again (from the L2 mostly), the others have deeper rings.  Down, 64 tokens of 2048 x 8192: with room for 64 tokens
// and twice the mean one of four experts each 88 us instead of 78, two of four 118 instead of 106, two of sixteen 259 instead of 255.
int ffn_tokens(int T, int K, int E, bool up) {
  const int mean = T * K / chosen_experts(T, K, E), want = std::min(T, up ? 2 * mean + 8 : mean + mean / 2 + 4);
  return want > 32 && up ? 64 : want > 16 ? 32 : 16;
}
// How the weights are cut into tiles: rows per tile and, of the down projection, parts of the contracted index.  The cheapest by the time that the
// fullest SM takes, in ns: rounds of tiles times stages of 60 ns and their bytes at 44 a ns (an SM's share of HBM), but at least 460 ns (eight MMAs of
// 128 rows, a good 100 cycles each however few their columns and valid rows), 1000 for a tile's end; parts of a sum that are written (100 bytes a ns) and read again (20).
struct FfnCut { int h, splits; };
FfnCut cut_tiles(int T, int K, int E, int rows_out, int Kd, bool up) {
  const long long n = chosen_experts(T, K, E), m = (T * K + n - 1) / n, kb = (Kd + FT_K - 1) / FT_K, per = up ? 2 : 1;
  const int per_token = ffn_per_token(up), cols = per_token * ffn_tokens(T, K, E, up);
  FfnCut best{8, 1};
  long long least = -1;
  for (int s = 1; s <= (up ? 1 : kFfnMaxSplits) && s <= kb; ++s)
    for (int h = up ? 64 : 128; h >= (up ? 8 : 32); h -= 8) {
      if (ffn_stages((int)per * h, cols) < FT_MIN_STAGES) continue;
      const long long rounds = (n * s * ((rows_out + h - 1) / h) + kSizingSms - 1) / kSizingSms;
      const long long stage = std::max(460ll, 60 + 2 * FT_K * (per * h + per_token * m) / 44), parts = up || (K == 1 && s == 1) ? 0 : 4 * m * h * rounds / 100 + 4ll * T * K * s * h / 20;
      const long long cost = rounds * ((kb + s - 1) / s * stage + 1000) + parts;
      if (least < 0 || cost < least) { least = cost; best.h = h; best.splits = s; }
    }
  return best;
}

struct FfnTc {
  const bf16* x; int ldx;                            // rows of activations: up: x of the token; down: hid of the assignment, two rows
  int Kd, w_rows, out_rows;                          // contracted length; weight rows per expert; rows of the product (up: pairs of them)
  const int32_t* idx; const float* gates;
  bf16* hid; float* part; bf16* out; int32_t* arrived; int32_t* status;
  int T, K, E;
  int h, tiles, splits, stages, tokens_cap;          // rows per tile, tiles per expert, parts of the contracted index, ring, tokens of a stage
  int direct;                                        // down: one expert and one part a token: written at once
  uint32_t stall;                                    // fault injection: bytes that a block's stages behind its first wait for in vain
};

// Whether a phase is over; does not wait.  A wait takes 200 to 250 cycles even then, as long as three MMAs: the producer and the issuer look at
// their next stage while they work on the present one.
__device__ __forceinline__ bool mbar_ready(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}
// A warp's wait, polled by one lane.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, uint32_t limit) {
  int ok = 1;
  if ((threadIdx.x & 31) == 0) ok = mbar_wait(bar, parity, abort_flag, limit);
  return __shfl_sync(0xffffffffu, ok, 0) != 0;
}
// FLIGHT: stages of token rows that each of the four warps has in flight besides the one it asks for: 4 FLIGHT + 1 stages at least, and one for each warp.
template <bool UP, int FLIGHT>
__global__ void __launch_bounds__(FT_THREADS, 1)
ffn_step_tc(const __grid_constant__ CUtensorMap tmap_w, const FfnTc p, uint32_t wait_limit) {
  constexpr int PT = ffn_per_token(UP);
  extern __shared__ __align__(128) unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  __shared__ ByExpert by;
  __shared__ int act[kMaxE], n_act_s, last_s;
  __shared__ __align__(16) float exch[16][132];      // up: 16 columns of 128 accumulator rows
  __shared__ __align__(8) unsigned long long bars[2 * FT_MAX_STAGES + 5];
  __shared__ uint32_t tmem_s;
  __shared__ int abort_s;
  volatile int* abort_flag = &abort_s;
  // (the warp's number from a shuffle and elect.sync tell the compiler that the roles' branches are uniform: with `lane == 0` the producer's and
  // the issuer's loops took 500 and 640 cycles a stage, whatever its size)
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), A = p.T * p.K;
  const bool leader = elect_one();
  auto full_bar = [&](int s) { return smem_u32(&bars[s]); };
  auto empty_bar = [&](int s) { return smem_u32(&bars[FT_MAX_STAGES + s]); };
  auto tfull_bar = [&](int a) { return smem_u32(&bars[2 * FT_MAX_STAGES + a]); };
  auto tempty_bar = [&](int a) { return smem_u32(&bars[2 * FT_MAX_STAGES + 2 + a]); };
  const uint32_t drain_bar = smem_u32(&bars[2 * FT_MAX_STAGES + 4]);

  if (tid == 0) {
    for (int s = 0; s < p.stages; ++s) { mbar_init(full_bar(s), 1 + 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 4); }
    mbar_init(drain_bar, 1);
    abort_s = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (tid == 32 * 9) asm volatile("prefetch.tensormap [%0];" ::"l"(&tmap_w) : "memory");
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_s)), "r"(2 * FT_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (UP) {                                          // (down: the choice of experts is older than the launch before)
    pdl_wait();
    if (warp == 1) pdl_trigger();                    // (the warp that has the block's tensor memory by now: the successor takes some before it waits)
  }
  by.build(p.idx, A, p.E);
  if (warp == 0) {                                   // the experts that somebody chose
    const bool lo = lane < p.E && by.off[lane + 1] > by.off[lane], hi = 32 + lane < p.E && by.off[33 + lane] > by.off[32 + lane];
    const unsigned ml = __ballot_sync(0xffffffffu, lo), mh = __ballot_sync(0xffffffffu, hi), below = (1u << lane) - 1u;
    if (lo) act[__popc(ml & below)] = lane;
    if (hi) act[__popc(ml) + __popc(mh & below)] = 32 + lane;
    if (lane == 0) n_act_s = __popc(ml) + __popc(mh);
  }
  if (UP && blockIdx.x == 0) {
    bool bad = false;
    for (int a = tid; a < A; a += FT_THREADS) bad |= __ldg(p.idx + a) >= p.E;
    bad = __syncthreads_or(bad);
    if (tid < kStatusInts) p.status[tid] = tid == kStatCode && bad ? ROM_ERR_INVALID_ARG : 0;
    for (int j = tid; j < kFfnMaxTiles; j += FT_THREADS) p.arrived[j] = 0;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_s;
  const int n_act = n_act_s, per_expert = p.tiles * p.splits, total = n_act * per_expert;
  const int num_kb = (p.Kd + FT_K - 1) / FT_K;
  const uint32_t w_bytes = (UP ? 2 : 1) * p.h * 128, x_bytes = PT * p.tokens_cap * 128, stage_bytes = FT_KB * (w_bytes + x_bytes);
  auto cols = [](int m) { return PT * m > 32 ? 64 : PT * m > 16 ? 32 : 16; };      // N of a pass over m tokens
  // item w: expert, first row, stages [kb0, kb0 + n) of the contracted index, walked from a start of the tile's own: in step all CTAs
  // would read the same columns of rows that are a power of two apart
  struct Item { int e, tile, part, kb0, n, rot; };
  auto item = [&](int w) {
    Item it;
    const int i = w / per_expert, r = w - i * per_expert;
    it.e = act[i];
    if (UP) {
      it.tile = r; it.part = 0; it.kb0 = 0; it.n = num_kb;
    } else {
      it.tile = r / p.splits; it.part = r - it.tile * p.splits;
      it.kb0 = num_kb * it.part / p.splits;
      it.n = num_kb * (it.part + 1) / p.splits - it.kb0;
    }
    it.rot = it.tile * 5 % it.n;
    return it;
  };
  auto k_of = [&](const Item& it, int q) { return (it.kb0 + (q + it.rot < it.n ? q + it.rot : q + it.rot - it.n)) * FT_K; };

  if (warp == 0) {
    // ---------------------------------------------------------------- TMA producer of the weights (nothing here depends on the launch before)
    if (leader) {
      int stage = 0, issued = 0; uint32_t phase = 0, tx = FT_KB * w_bytes;
      bool ok = true, ready = true;                  // ready: the next stage was free when it was looked at (all are at first)
      for (int w = blockIdx.x; w < total && ok; w += gridDim.x) {
        const Item it = item(w);
        const int row = it.e * p.w_rows + it.tile * p.h, m = by.off[it.e + 1] - by.off[it.e];
        for (int n0 = 0; n0 < m && ok; n0 += p.tokens_cap)
          for (int q = 0; q < it.n; ++q) {
            if (!ready && !mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, wait_limit)) { ok = false; break; }
            const int k0 = k_of(it, q), next = stage + 1 == p.stages ? 0 : stage + 1;
            const uint32_t dst = base + stage * stage_bytes;
            ready = mbar_ready(empty_bar(next), (next ? phase : phase ^ 1u) ^ 1u);
            mbar_expect_tx(full_bar(stage), tx);
            tx = FT_KB * w_bytes + p.stall;
#pragma unroll
            for (int b = 0; b < FT_KB; ++b) {
              tma_load_2d(dst + b * w_bytes, &tmap_w, full_bar(stage), k0 + b * BLOCK_K, row);
              if (UP) tma_load_2d(dst + b * w_bytes + p.h * 128, &tmap_w, full_bar(stage), k0 + b * BLOCK_K, row + p.out_rows);
            }
            ++issued;
            stage = next;
            if (!next) phase ^= 1u;
          }
      }
      if (!ok) {
        if (!*abort_flag) { atomicExch(p.status + kStatCode, ROM_ERR_DEVICE_TIMEOUT); atomicExch(p.status + kStatWhere, 4); }
        *abort_flag = 1;
      }
      if (*abort_flag) {                             // give the copies still in flight a bounded time to land before the CTA exits
        for (int i = 0; i < min(issued, p.stages); ++i) {
          if (--stage < 0) { stage = p.stages - 1; phase ^= 1u; }
          for (uint32_t k = 0; k < (wait_limit >> 2); ++k)
            if (mbar_try_wait(full_bar(stage), phase)) break;
        }
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMA issuer: weights are the M operand, tokens the N columns
    if (leader) {
      int stage = 0, acc = 0; uint32_t phase = 0, acc_phase = 0;
      bool ok = true, issued_any = false, ready = false;
      for (int w = blockIdx.x; w < total && ok; w += gridDim.x) {
        const Item it = item(w);
        const int m = by.off[it.e + 1] - by.off[it.e];
        for (int n0 = 0; n0 < m && ok; n0 += p.tokens_cap) {
          const int nc = cols(min(m - n0, p.tokens_cap));
          const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(nc >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
          if (!mbar_wait(tempty_bar(acc), acc_phase ^ 1u, abort_flag, wait_limit)) { ok = false; break; }
          tc_fence_after();
          for (int q = 0; q < it.n; ++q) {
            if (!ready && !mbar_wait(full_bar(stage), phase, abort_flag, wait_limit)) { ok = false; break; }
            tc_fence_after();
            const int next = stage + 1 == p.stages ? 0 : stage + 1;
            ready = mbar_ready(full_bar(next), next ? phase : phase ^ 1u);
            const int blocks = min(FT_KB, (p.Kd - k_of(it, q)) / BLOCK_K);
            for (int b = 0; b < blocks; ++b) {
              const uint64_t adesc = make_smem_desc(base + stage * stage_bytes + b * w_bytes), bdesc = make_smem_desc(base + stage * stage_bytes + FT_KB * w_bytes + b * x_bytes);
#pragma unroll
              for (int k = 0; k < BLOCK_K / UMMA_K; ++k)
                // few columns: into FT_COLS / nc accumulators in turns, so that an MMA does not wait for the one before
                umma_bf16(tmem_base + acc * FT_COLS + k * nc % FT_COLS, adesc + (uint64_t)(2 * k), bdesc + (uint64_t)(2 * k), idesc,
                          (q | b) != 0 || k * nc >= FT_COLS ? 1u : 0u);
            }
            umma_commit(empty_bar(stage));
            issued_any = true;
            stage = next;
            if (!next) phase ^= 1u;
          }
          if (!ok) break;
          umma_commit(tfull_bar(acc));
          if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
        }
      }
      if (!ok) {
        if (!*abort_flag) { atomicExch(p.status + kStatCode, ROM_ERR_DEVICE_TIMEOUT); atomicExch(p.status + kStatWhere, 5); }
        *abort_flag = 1;
      }
      if (*abort_flag && issued_any) {
        umma_commit(drain_bar);
        for (uint32_t k = 0; k < (wait_limit >> 2); ++k)
          if (mbar_try_wait(drain_bar, 0)) break;
      }
    }
  } else if (warp >= 6) {
    // ---------------------------------------------------------------- token rows, 16-byte pieces into the swizzled layout: a stage is one warp's,
    // the four warps take them in turns
    const int xw = warp - 6, lrow = lane >> 3, chunk = lane & 7;
    if (!UP) { pdl_wait(); pdl_trigger(); }
    int turn = 0, stage = 0, pub = xw, pending = 0; uint32_t phase = 0;      // turn: whose stage it is
    bool ok = true;
    auto publish = [&]() {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(full_bar(pub));
      if ((pub += 4) >= p.stages) pub -= p.stages;
      --pending;
    };
    for (int w = blockIdx.x; w < total && ok; w += gridDim.x) {
      const Item it = item(w);
      const int m_all = by.off[it.e + 1] - by.off[it.e];
      for (int n0 = 0; n0 < m_all && ok; n0 += p.tokens_cap) {
        const int m = min(m_all - n0, p.tokens_cap);
        const short* mine = by.list + by.off[it.e] + n0;
        for (int kb = 0; kb < it.n; ++kb) {
          if (turn == xw) {
            ok = warp_wait(empty_bar(stage), phase ^ 1u, abort_flag, wait_limit);
            if (!ok) break;
            const uint32_t dst = base + stage * stage_bytes + FT_KB * w_bytes;
            const int k0 = k_of(it, kb), blocks = min(FT_KB, (p.Kd - k0) / BLOCK_K);
            for (int i = lrow; i < PT * m; i += 4) { // (columns past the last token hold whatever the stage held: nobody reads their sums)
              // down: the high halves, then the low ones, each in half of the pass's columns
              const int a = mine[i / PT], r = UP ? i : (i >> 1) + (i & 1) * (cols(m) / 2);
              const bf16* src = p.x + (size_t)(UP ? a / p.K : 2 * a + (i & 1)) * p.ldx + k0 + chunk * 8;
              for (int b = 0; b < blocks; ++b)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + b * x_bytes + r * 128 + ((chunk ^ (r & 7)) << 4)), "l"(src + b * BLOCK_K) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (++pending > FLIGHT) {                // this warp's stage of FLIGHT copies ago has landed: publish it to the tensor cores
              asm volatile("cp.async.wait_group %0;" ::"n"(FLIGHT) : "memory");
              publish();
            }
          }
          turn = (turn + 1) & 3;
          if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
      }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    while (pending > 0) publish();
    if (!ok && lane == 0) {
      if (!*abort_flag) { atomicExch(p.status + kStatCode, ROM_ERR_DEVICE_TIMEOUT); atomicExch(p.status + kStatWhere, 7); }
      *abort_flag = 1;
    }
  } else {
    // ---------------------------------------------------------------- output: lane = weight row, column = token
    const int quarter = warp & 3, r_acc = quarter * 32 + lane, ct = tid - 64;      // ct: thread of the 128 here
    // (barriers and tensor-memory loads take whole warps: after branches by lane a warp is brought together first)
    auto together = [&]() { __syncwarp(); asm volatile("bar.sync 1, 128;" ::: "memory"); };
    auto all_warps = [&](bool mine) {
      int all;
      __syncwarp();
      asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 q, %1, 0;\n\tbar.red.and.pred p, 2, 128, q;\n\tselp.s32 %0, 1, 0, p;\n\t}" : "=r"(all) : "r"((int)mine) : "memory");
      return all != 0;
    };
    if (!UP) {
      pdl_wait();
      for (int t = blockIdx.x; t < p.T; t += gridDim.x) {      // tokens without an expert
        bool any = false;
        for (int k = 0; k < p.K; ++k) any |= by.of[t * p.K + k] >= 0;
        if (!any)
          for (int d = 8 * ct; d < p.out_rows; d += 8 * 128) *reinterpret_cast<uint4*>(p.out + (size_t)t * p.out_rows + d) = make_uint4(0, 0, 0, 0);
      }
    }
    int acc = 0; uint32_t acc_phase = 0;
    bool ok = true;
    for (int w = blockIdx.x; w < total && ok; w += gridDim.x) {
      const Item it = item(w);
      const int row0 = it.tile * p.h, rows = min(p.h, p.out_rows - row0), m_all = by.off[it.e + 1] - by.off[it.e];
      for (int n0 = 0; n0 < m_all && ok; n0 += p.tokens_cap) {
        const int m = min(m_all - n0, p.tokens_cap), nc = cols(m);
        const short* mine = by.list + by.off[it.e] + n0;
        ok = warp_wait(tfull_bar(acc), acc_phase, abort_flag, wait_limit);
        if (UP) ok = all_warps(ok);                  // (the four warps meet in the exchange below: they leave together)
        if (!ok) break;
        tc_fence_after();
        const uint32_t taddr = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)acc * FT_COLS;
        for (int c0 = 0; c0 < m; c0 += 32) {
          uint32_t r[32];
          __syncwarp();
          tmem_ld32_issue(taddr + c0, r);
          tmem_ld_wait(r);
          if (!UP || nc < FT_COLS) {                 // the sums of the turns and of the halves: columns 32 further on, then 16, then 8
            uint32_t r2[32];
            tmem_ld32_issue(taddr + 32, r2);
            tmem_ld_wait(r2);
            // (the last step down adds the halves: an infinite weight makes the low one's sum infinite of either sign or NaN)
            auto add = [&](uint32_t x, uint32_t y, bool halves) {
              const float u = __uint_as_float(x), v = __uint_as_float(y);
              return __float_as_uint(halves && isinf(u) ? u : u + v);
            };
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = add(r[j], r2[j], !UP && nc == 64);
            if (nc <= 16 * PT)
#pragma unroll
              for (int j = 0; j < 16; ++j) r[j] = add(r[j], r[16 + j], !UP && nc == 32);
            if (!UP && nc == 16)
#pragma unroll
              for (int j = 0; j < 8; ++j) r[j] = add(r[j], r[8 + j], true);
          }
          if (UP) {
#pragma unroll
            for (int jb = 0; jb < 32; jb += 16) {
              const int nn = min(16, m - c0 - jb);
              if (nn <= 0) break;
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (j < nn) exch[j][r_acc] = __uint_as_float(r[jb + j]);
              together();
              // gate rows are 0 .. h-1 of the accumulator, up rows h .. 2 h - 1: two hidden columns of one token a thread
              const int half = p.h / 2;
              for (int i = ct; i < nn * half; i += 128) {
                const int j = i / half, rr = (i % half) * 2;
                if (rr < rows) {
                  const int a = mine[c0 + jb + j];
                  const float2 g = *reinterpret_cast<const float2*>(&exch[j][rr]), u = *reinterpret_cast<const float2*>(&exch[j][p.h + rr]);
                  const float gate = __ldg(p.gates + a);
                  // high and low half; one that is not finite has no low half
                  const float v0 = silu_fast(g.x) * u.x * gate, v1 = silu_fast(g.y) * u.y * gate;
                  const __nv_bfloat162 hi = __floats2bfloat162_rn(v0, v1);
                  const float h0 = __low2float(hi), h1 = __high2float(hi);
                  bf16* to = p.hid + (size_t)a * 2 * p.out_rows + row0 + rr;
                  *reinterpret_cast<__nv_bfloat162*>(to) = hi;
                  *reinterpret_cast<__nv_bfloat162*>(to + p.out_rows) =
                      __floats2bfloat162_rn(isfinite(h0) ? v0 - h0 : 0.0f, isfinite(h1) ? v1 - h1 : 0.0f);
                }
              }
              together();
            }
          } else if (r_acc < rows) {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              if (c0 + j >= m) break;
              const int a = mine[c0 + j];
              if (p.direct) p.out[(size_t)a * p.out_rows + row0 + r_acc] = __float2bfloat16_rn(__uint_as_float(r[j]));
              else p.part[((size_t)it.part * A + a) * p.out_rows + row0 + r_acc] = __uint_as_float(r[j]);
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty_bar(acc));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      if (!UP && !p.direct) {
        // whoever brings the last part of these rows adds them all, in the order of slots and parts
        __threadfence();
        ok = all_warps(ok);
        if (!ok) break;
        if (ct == 0) last_s = atomicAdd(p.arrived + it.tile, 1) == n_act * p.splits - 1;
        together();
        const bool last = last_s != 0;
        if (last) {
          __threadfence();
          const int nv = rows / 4;
          const int outs = p.T * nv;
          auto add = [&](auto u_tag) {               // U outputs of a thread in flight
          constexpr int U = decltype(u_tag)::value;
          for (int i0 = 0; i0 < outs; i0 += 128 * U) {
            float4 v[U];
            int at[U], a0[U];                        // column and first assignment of an output
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const int i = min(i0 + 128 * u + ct, outs - 1), t = i / nv;
              at[u] = row0 + (i - t * nv) * 4;
              a0[u] = t * p.K;
              v[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
            for (int k = 0; k < p.K; ++k)
              for (int q = 0; q < p.splits; ++q) {
                float4 f[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                  if (i0 + 128 * u >= outs) break;   // (the same for all threads)
                  f[u] = by.of[a0[u] + k] >= 0 ? __ldcg(reinterpret_cast<const float4*>(p.part + ((size_t)q * A + a0[u] + k) * p.out_rows + at[u])) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                  if (i0 + 128 * u >= outs) break;
                  v[u].x += f[u].x; v[u].y += f[u].y; v[u].z += f[u].z; v[u].w += f[u].w;
                }
              }
#pragma unroll
            for (int u = 0; u < U; ++u) {
              if (i0 + 128 * u + ct >= outs) break;
              const __nv_bfloat162 lo = __floats2bfloat162_rn(v[u].x, v[u].y), hi = __floats2bfloat162_rn(v[u].z, v[u].w);
              *reinterpret_cast<uint2*>(p.out + (size_t)(a0[u] / p.K) * p.out_rows + at[u]) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
            }
          }
          };
          if (outs <= 256) add(std::integral_constant<int, 1>{});      // (a token or a few: 1 us less than with the longer code)
          else add(std::integral_constant<int, 4>{});
        }
        together();                                  // (last_s is read before it is written again)
      }
    }
    if (!ok && lane == 0) {
      if (!*abort_flag) { atomicExch(p.status + kStatCode, ROM_ERR_DEVICE_TIMEOUT); atomicExch(p.status + kStatWhere, 6); }
      *abort_flag = 1;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();                                    // (the leader comes from its own branch; before the barrier, for all warps, this cost 1 to 30 %)
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(2 * FT_COLS) : "memory");
  }
}

cudaError_t launch_ffn_tc(const FfnStep& s, const FfnCut& cd, float* part, int32_t* arrived, bool test_stall, cudaStream_t st) {
  int sms = 0;
  cudaError_t e = current_device_sm_count(&sms);
  if (e != cudaSuccess) return e;
  FfnTc p{};
  p.idx = s.idx; p.gates = s.gates; p.hid = static_cast<bf16*>(s.hid); p.part = part; p.out = static_cast<bf16*>(s.out); p.arrived = arrived; p.status = s.status;
  p.T = s.T; p.K = s.K; p.E = s.E; p.stall = test_stall ? 16 : 0;
  const FfnCut cu = cut_tiles(s.T, s.K, s.E, s.F, s.Dm, true);
  auto launch = [&](auto up_tag, const void* W) {
    constexpr bool up = decltype(up_tag)::value;
    p.tokens_cap = ffn_tokens(s.T, s.K, s.E, up);
    const int rows = (up ? 2 : 1) * p.h, cols = ffn_per_token(up) * p.tokens_cap;
    p.stages = ffn_stages(rows, cols);
    if (p.stages < FT_MIN_STAGES) return cudaErrorInvalidValue;      // (cut_tiles takes no such tile)
    CUtensorMap tw;
    if (!make_tmap(&tw, W, (uint64_t)s.E * p.w_rows, (uint64_t)p.Kd, (uint64_t)p.Kd, p.h)) return cudaErrorInvalidValue;
    auto kern = p.stages >= 9 ? ffn_step_tc<up, 1> : ffn_step_tc<up, 0>;
    cudaError_t rc = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, FT_SMEM);
    if (rc != cudaSuccess) return rc;
    count_launch();
    return launch_k(kern, dim3(sms), FT_THREADS, ffn_ring(rows, cols, p.stages), st, tw, p, p.stall ? WAIT_LIMIT_TEST : WAIT_LIMIT);
  };
  p.x = static_cast<const bf16*>(s.x); p.ldx = s.Dm; p.Kd = s.Dm; p.w_rows = 2 * s.F; p.out_rows = s.F;
  p.h = cu.h; p.tiles = (s.F + cu.h - 1) / cu.h; p.splits = 1;
  if ((e = launch(std::true_type{}, s.W_gu)) != cudaSuccess) return e;
  p.x = p.hid; p.ldx = s.F; p.Kd = s.F; p.w_rows = s.Dm; p.out_rows = s.Dm;
  p.h = cd.h; p.tiles = (s.Dm + cd.h - 1) / cd.h; p.splits = cd.splits; p.direct = s.K == 1 && cd.splits == 1;
  return launch(std::false_type{}, s.W_down);
}

int check_ffn_step(const rom_config* c, int d_ff) {
  if (!c) return ROM_ERR_INVALID_ARG;
  if (c->dtype != ROM_F32 && c->dtype != ROM_BF16) return ROM_ERR_INVALID_ARG;
  if (c->B < 1 || c->L < 1 || c->E < 1 || c->K < 1 || c->K > c->E || (c->flags & ~ROM_FLAG_TEST_STALL) != 0) return ROM_ERR_INVALID_ARG;
  if (c->E > kMaxE || c->K > kMaxK) return ROM_ERR_UNSUPPORTED;
  if (c->d_model < 64 || c->d_model % 64 != 0) return ROM_ERR_INVALID_ARG;
  if (d_ff < 128 || d_ff % 128 != 0) return d_ff < 1 ? ROM_ERR_INVALID_ARG : ROM_ERR_UNSUPPORTED;
  if ((int64_t)c->B * c->L > kFfnStepTokens) return ROM_ERR_UNSUPPORTED;
  if (c->d_model > 32 * kFfnMaxTiles || (int64_t)c->E * 2 * d_ff >= (int64_t)1 << 31 || (int64_t)c->E * c->d_model >= (int64_t)1 << 31) return ROM_ERR_UNSUPPORTED;
  return ROM_OK;
}
struct FfnStepWs { size_t status, arrived, hid, part, total; FfnCut down; };
FfnStepWs ffn_step_ws(const rom_config& c, int d_ff) {
  FfnStepWs l{};
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = align_up(o + bytes, 256); return at; };
  l.status = take(sizeof(int32_t) * kStatusInts);
  const bool tc = c.dtype == ROM_BF16;
  const size_t A = (size_t)c.B * c.L * c.K;
  l.arrived = take(tc ? sizeof(int32_t) * kFfnMaxTiles : 0);
  l.hid = take(4 * A * d_ff);      // (bf16: two halves)
  if (tc) l.down = cut_tiles(c.B * c.L, c.K, c.E, c.d_model, d_ff, false);
  // (as many parts as any number of tokens up to these may take: a buffer for the largest batch does for all smaller ones, which are cut into more)
  l.part = take(tc ? sizeof(float) * std::min(kFfnMaxSplits, (d_ff + FT_K - 1) / FT_K) * A * c.d_model : 0);
  l.total = o;
  return l;
}

}  // namespace
}  // namespace rom

using namespace rom;

extern "C" {

int rom_ffn_moe_step_workspace_size(const rom_config* cfg, int32_t d_ff, size_t* bytes) {
  if (!bytes) return ROM_ERR_INVALID_ARG;
  const int rc = check_ffn_step(cfg, d_ff);
  if (rc != ROM_OK) return rc;
  *bytes = ffn_step_ws(*cfg, d_ff).total;
  return ROM_OK;
}

int rom_ffn_moe_step(const rom_config* cfg, int32_t d_ff, const void* W_gu, const void* W_down, const void* x, const int32_t* topk_idx,
                     const float* gates, void* out, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_ffn_step(cfg, d_ff);
  if (rc != ROM_OK) return rc;
  if (!W_gu || !W_down || !x || !topk_idx || !gates || !out || !ws) return ROM_ERR_INVALID_ARG;
  const void* ptrs[] = {W_gu, W_down, x, out, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return ROM_ERR_INVALID_ARG;
  if (!aligned4(topk_idx) || !aligned4(gates)) return ROM_ERR_INVALID_ARG;
  const rom_config& c = *cfg;
  const FfnStepWs lay = ffn_step_ws(c, d_ff);
  if (ws_bytes < lay.total) return ROM_ERR_WORKSPACE;
  if ((rc = check_device()) != ROM_OK) return rc;
  LaunchCounter::count = 0;
  char* W = static_cast<char*>(ws);
  const FfnStep p{x, W_gu, W_down, topk_idx, gates, out, W + lay.hid, reinterpret_cast<int32_t*>(W + lay.status), c.B * c.L, c.K, c.E, c.d_model, d_ff};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = c.dtype == ROM_BF16 ? launch_ffn_tc(p, lay.down, reinterpret_cast<float*>(W + lay.part), reinterpret_cast<int32_t*>(W + lay.arrived), c.flags != 0, st)
                                            : launch_ffn_rows(p, st);
  return e == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

}  // extern "C"
