// FFN-MoE of the few tokens of a generation step (rom_ffn_moe_step): out_t = sum_k g_tk W_down,e (SiLU(W_gate,e x_t) * (W_up,e x_t)), e = topk_idx[t, k].
// Two launches: hidden rows g SiLU(gate) up of every assignment (token, slot), then the down projection with the sum over the slots.
// The weights of the chosen experts, read once, are what counts: 6 d_model d_ff bytes an expert (bf16).
#include "rom_serve.cuh"

namespace rom {
namespace {

constexpr int kFfnStepTokens = 64, kFfnStepAssign = kFfnStepTokens * kMaxK;

struct FfnStep {
  const void* x; const void* W_gu; const void* W_down; const int32_t* idx; const float* gates; void* out;
  void* hid;                // [B K, d_ff] storage type
  int32_t* status;
  int T, K, E, Dm, F;
};

// Assignments by expert.  An expert's list is in ascending order, so that the order of every sum is fixed.
struct ByExpert {
  int off[kMaxE + 1];
  short list[kFfnStepAssign];
  // all threads of the block; ends with a barrier
  __device__ __forceinline__ void build(const int32_t* idx, int A, int E) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    for (int e = warp; e < E; e += warps) {
      int n = 0;
      for (int a0 = 0; a0 < A; a0 += 32) n += __popc(__ballot_sync(0xffffffffu, a0 + lane < A && __ldg(idx + a0 + lane) == e));
      if (lane == 0) off[e + 1] = n;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      off[0] = 0;
      for (int e = 0; e < E; ++e) off[e + 1] += off[e];
    }
    __syncthreads();
    for (int e = warp; e < E; e += warps) {
      int n = off[e];
      if (n == off[e + 1]) continue;
      for (int a0 = 0; a0 < A; a0 += 32) {
        const unsigned m = __ballot_sync(0xffffffffu, a0 + lane < A && __ldg(idx + a0 + lane) == e);
        if ((m >> lane) & 1u) list[n + __popc(m & ((1u << lane) - 1u))] = (short)(a0 + lane);
        n += __popc(m);
      }
    }
    __syncthreads();
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

// Four weight rows times up to eight rows of activations, over the lanes of a warp; lane 8 r + j gets row r times activation j.
template <typename T>
__device__ __forceinline__ float rows_4x8(const T* const (&w)[4], const T* const (&x)[8], int n, int Kd) {
  constexpr int V = V16<T>::N;
  const int lane = threadIdx.x & 31;
  float acc[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) acc[i] = 0.0f;
  for (int k = lane * V; k < Kd; k += 32 * V) {
    V16<T> wq[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) wq[r].load(w[r] + k);
    float wv[4][V];
#pragma unroll
    for (int r = 0; r < 4; ++r) wq[r].get(wv[r]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= n) break;
      float xv[V];
      V16<T> xq;
      xq.q = *reinterpret_cast<const decltype(xq.q)*>(x[j] + k);
      xq.get(xv);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[8 * r + j] = fmaf(wv[r][i], xv[i], acc[8 * r + j]);
    }
  }
  return sum_to_lane(acc);
}

constexpr int FR_WARPS = 4;
template <typename T>
__global__ void __launch_bounds__(FR_WARPS * 32)
ffn_step_up(const FfnStep p) {
  __shared__ ByExpert by;
  pdl_sync();
  if (blockIdx.x == 0) ffn_status(p);
  by.build(p.idx, p.T * p.K, p.E);
  const int lane = threadIdx.x & 31, j = lane & 7;
  const int f = (blockIdx.x * FR_WARPS + (threadIdx.x >> 5)) * 2;      // a warp has two hidden columns of every expert
  for (int e = 0; e < p.E; ++e) {
    const T* g = static_cast<const T*>(p.W_gu) + ((size_t)e * 2 * p.F + f) * p.Dm;
    const T* u = g + (size_t)p.F * p.Dm;
    const T* const w[4] = {g, g + p.Dm, u, u + p.Dm};
    for (int a0 = by.off[e]; a0 < by.off[e + 1]; a0 += 8) {
      const int n = min(8, by.off[e + 1] - a0);
      const T* x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = static_cast<const T*>(p.x) + (size_t)(by.list[a0 + min(i, n - 1)] / p.K) * p.Dm;
      const float v = rows_4x8<T>(w, x, n, p.Dm);
      const float up = __shfl_down_sync(0xffffffffu, v, 16);
      if (lane < 16 && j < n) {
        const int a = by.list[a0 + j];
        static_cast<T*>(p.hid)[(size_t)a * p.F + f + (lane >> 3)] = from_f32<T>(silu_f(v) * up * __ldg(p.gates + a));
      }
    }
  }
}
template <typename T>
__global__ void __launch_bounds__(FR_WARPS * 32)
ffn_step_down(const FfnStep p) {
  __shared__ ByExpert by;
  __shared__ float sum[FR_WARPS][kFfnStepTokens][4];
  by.build(p.idx, p.T * p.K, p.E);
  pdl_sync();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int d = (blockIdx.x * FR_WARPS + warp) * 4;
  float (*s)[4] = sum[warp];
  for (int t = lane; t < p.T * 4; t += 32) s[t >> 2][t & 3] = 0.0f;
  __syncwarp();
  for (int e = 0; e < p.E; ++e) {
    const T* w0 = static_cast<const T*>(p.W_down) + ((size_t)e * p.Dm + d) * p.F;
    const T* const w[4] = {w0, w0 + p.F, w0 + 2 * (size_t)p.F, w0 + 3 * (size_t)p.F};
    for (int a0 = by.off[e]; a0 < by.off[e + 1]; a0 += 8) {
      const int n = min(8, by.off[e + 1] - a0);
      const T* x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = static_cast<const T*>(p.hid) + (size_t)by.list[a0 + min(i, n - 1)] * p.F;
      const float v = rows_4x8<T>(w, x, n, p.F);
      for (int i = 0; i < n; ++i) {      // one at a time: two of them may be of one token
        if ((lane & 7) == i) s[by.list[a0 + i] / p.K][lane >> 3] += v;
        __syncwarp();
      }
    }
  }
  for (int t = lane; t < p.T * 4; t += 32) static_cast<T*>(p.out)[(size_t)(t >> 2) * p.Dm + d + (t & 3)] = from_f32<T>(s[t >> 2][t & 3]);
}

template <typename T>
cudaError_t launch_ffn_rows(const FfnStep& p, cudaStream_t st) {
  cudaError_t e = launch_k(ffn_step_up<T>, dim3(p.F / (2 * FR_WARPS)), FR_WARPS * 32, 0, st, p);
  if (e != cudaSuccess) return e;
  count_launch();
  e = launch_k(ffn_step_down<T>, dim3(p.Dm / (4 * FR_WARPS)), FR_WARPS * 32, 0, st, p);
  count_launch();
  return e;
}

int check_ffn_step(const rom_config* c, int d_ff) {
  if (!c) return ROM_ERR_INVALID_ARG;
  if (c->dtype != ROM_F32 && c->dtype != ROM_BF16) return ROM_ERR_INVALID_ARG;
  if (c->B < 1 || c->L < 1 || c->E < 1 || c->K < 1 || c->K > c->E || c->flags != 0) return ROM_ERR_INVALID_ARG;
  if (c->E > kMaxE || c->K > kMaxK) return ROM_ERR_UNSUPPORTED;
  if (c->d_model < 64 || c->d_model % 64 != 0) return ROM_ERR_INVALID_ARG;
  if (d_ff < 128 || d_ff % 128 != 0) return d_ff < 1 ? ROM_ERR_INVALID_ARG : ROM_ERR_UNSUPPORTED;
  if ((int64_t)c->B * c->L > kFfnStepTokens) return ROM_ERR_UNSUPPORTED;
  return ROM_OK;
}
struct FfnStepWs { size_t status, hid, total; };
FfnStepWs ffn_step_ws(const rom_config& c, int d_ff) {
  FfnStepWs l{};
  size_t o = 0;
  auto take = [&](size_t bytes) { const size_t at = o; o = align_up(o + bytes, 256); return at; };
  l.status = take(sizeof(int32_t) * kStatusInts);
  l.hid = take((c.dtype == ROM_BF16 ? 2 : 4) * (size_t)c.B * c.L * c.K * d_ff);
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
  const cudaError_t e = c.dtype == ROM_BF16 ? launch_ffn_rows<__nv_bfloat16>(p, st) : launch_ffn_rows<float>(p, st);
  return e == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

}  // extern "C"
