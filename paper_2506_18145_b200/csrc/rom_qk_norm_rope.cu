// RMS norm of every head of q and k and its rotation by the row's position, in one pass, and the backward of both.
//
// Sixteen lanes (eight, four .. where heads are narrower) own a head of one row: each holds two runs of four places, the two halves of four pairs in the rotated
// part, eight adjacent places behind it.  The angle pos * inv_freq is formed in 64 bits and reduced to a turn before it is rounded: an fp32 product is off by
// 0.06 at a position of a million.  A lane takes the sine and cosine of its four pairs once for all heads it works on.
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
  float* part;                  // backward: [blocks][2][d_head] sums of dn xhat
  int rows, nq, nk, d, rot, interleaved;
  float eps;
};

// Four adjacent elements.
__device__ __forceinline__ void load4(const float* p, float (&v)[4]) { const float4 q = __ldg(reinterpret_cast<const float4*>(p)); v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w; }
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float (&v)[4]) {
  const uint2 q = __ldg(reinterpret_cast<const uint2*>(p));
  v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xffff0000u); v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xffff0000u);
}
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&v)[4]) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// The lane's places: runs at oa and ob; whether its pairs are rotated.
struct QkLane {
  int oa, ob;
  bool live, turns;
  __device__ __forceinline__ QkLane(int l, const QkArgs& p) {
    live = 8 * l < p.d;
    turns = 8 * l < p.rot;
    const bool apart = turns && !p.interleaved;
    oa = apart ? 4 * l : 8 * l;
    ob = apart ? p.rot / 2 + 4 * l : 8 * l + 4;
  }
};
__device__ __forceinline__ void angles(const QkArgs& p, int l, int row, float (&cs)[4], float (&sn)[4]) {
  const double at = (double)__ldg(p.pos + row) * 0.15915494309189535;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    double t = at * (double)__ldg(p.inv_freq + 4 * l + e);
    t -= rint(t);
    sincospif(2.0f * (float)t, &sn[e], &cs[e]);
  }
}
// (a, b) <- the pairs turned by the angles, forwards (way = 1) or back (-1)
__device__ __forceinline__ void turn(float (&a)[4], float (&b)[4], const float (&cs)[4], const float (&sn)[4], float way, bool interleaved) {
  if (!interleaved) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = a[e], y = b[e], s = way * sn[e];
      a[e] = x * cs[e] - y * s;
      b[e] = y * cs[e] + x * s;
    }
  } else {      // pairs 0, 1 lie in a, 2, 3 in b
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float x = a[2 * e], y = a[2 * e + 1], s = way * sn[e], u = b[2 * e], w = b[2 * e + 1], t = way * sn[2 + e];
      a[2 * e] = x * cs[e] - y * s;
      a[2 * e + 1] = y * cs[e] + x * s;
      b[2 * e] = u * cs[2 + e] - w * t;
      b[2 * e + 1] = w * cs[2 + e] + u * t;
    }
  }
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int m = LANES / 2; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}

// Groups of LANES lanes; a group works on `per` heads of one row, the heads of q first.
template <typename T, int LANES>
__global__ void __launch_bounds__(QK_THREADS) qk_norm_rope_kernel(QkArgs p, int per) {
  constexpr int GROUPS = QK_THREADS / LANES;
  const int l = threadIdx.x % LANES, heads = p.nq + p.nk, splits = (heads + per - 1) / per;
  const QkLane at(l, p);
  pdl_sync();
  const long long item = (long long)blockIdx.x * GROUPS + threadIdx.x / LANES;
  const bool mine = item < (long long)p.rows * splits;
  const int row = mine ? (int)(item / splits) : 0, h0 = mine ? (int)(item - (long long)row * splits) * per : 0;
  float wq[8], wk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = e < 4 ? at.oa + e : at.ob + e - 4;
    wq[e] = at.live && p.w_q ? __ldg(p.w_q + c) : 1.0f;
    wk[e] = at.live && p.w_k ? __ldg(p.w_k + c) : 1.0f;
  }
  float cs[4] = {}, sn[4] = {};
  if (mine && at.turns) angles(p, l, row, cs, sn);
  const int n = mine ? min(per, heads - h0) : 0;
  const float inv_d = 1.0f / (float)p.d;
#pragma unroll 4
  for (int i = 0; i < per; ++i) {      // (all lanes of the warp: the sums need them)
    const int h = h0 + i;
    const bool is_q = h < p.nq, on = i < n && at.live;
    const T* x = is_q ? static_cast<const T*>(p.q) + row * p.ldq + (long long)h * p.d : static_cast<const T*>(p.k) + row * p.ldk + (long long)(h - p.nq) * p.d;
    float a[4] = {}, b[4] = {};
    if (on) { load4(x + at.oa, a); load4(x + at.ob, b); }
    float ss = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) ss = fmaf(a[e], a[e], fmaf(b[e], b[e], ss));
    const float r = rsqrtf(fmaf(lanes_sum<LANES>(ss), inv_d, p.eps));
    if (on) {
#pragma unroll
      for (int e = 0; e < 4; ++e) { a[e] *= r * (is_q ? wq[e] : wk[e]); b[e] *= r * (is_q ? wq[4 + e] : wk[4 + e]); }
      if (at.turns) turn(a, b, cs, sn, 1.0f, p.interleaved);
      T* y = is_q ? static_cast<T*>(p.yq) + row * p.ldyq + (long long)h * p.d : static_cast<T*>(p.yk) + row * p.ldyk + (long long)(h - p.nq) * p.d;
      store4(y + at.oa, a);
      store4(y + at.ob, b);
    }
  }
}

// The backward: the same items, walked by a fixed number of blocks; dw is summed per lane, then over the block's groups in order, and the blocks' sums by
// qk_sum_weights: the same from run to run.
template <typename T, int LANES>
__global__ void __launch_bounds__(QK_THREADS) qk_norm_rope_bwd_kernel(QkArgs p, int per) {
  constexpr int GROUPS = QK_THREADS / LANES;
  extern __shared__ float sums[];      // [GROUPS][2][d]
  const int l = threadIdx.x % LANES, group = threadIdx.x / LANES, heads = p.nq + p.nk, splits = (heads + per - 1) / per;
  const QkLane at(l, p);
  pdl_sync();
  float wq[8], wk[8], sq[8] = {}, sk[8] = {};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int c = e < 4 ? at.oa + e : at.ob + e - 4;
    wq[e] = at.live && p.w_q ? __ldg(p.w_q + c) : 1.0f;
    wk[e] = at.live && p.w_k ? __ldg(p.w_k + c) : 1.0f;
  }
  const float inv_d = 1.0f / (float)p.d;
  const long long items = (long long)p.rows * splits;
  for (long long first = (long long)blockIdx.x * GROUPS; first < items; first += (long long)gridDim.x * GROUPS) {
    const long long item = first + group;
    const bool mine = item < items;
    const int row = mine ? (int)(item / splits) : 0, h0 = mine ? (int)(item - (long long)row * splits) * per : 0;
    float cs[4] = {}, sn[4] = {};
    if (mine && at.turns) angles(p, l, row, cs, sn);
    const int n = mine ? min(per, heads - h0) : 0;
#pragma unroll 2
    for (int i = 0; i < per; ++i) {
      const int h = h0 + i;
      const bool is_q = h < p.nq, on = i < n && at.live;
      const long long hh = is_q ? h : h - p.nq;
      const T* x = is_q ? static_cast<const T*>(p.q) + row * p.ldq + hh * p.d : static_cast<const T*>(p.k) + row * p.ldk + hh * p.d;
      const T* g = is_q ? static_cast<const T*>(p.gq) + ((long long)row * p.nq + hh) * p.d : static_cast<const T*>(p.gk) + ((long long)row * p.nk + hh) * p.d;
      float a[4] = {}, b[4] = {}, ga[4] = {}, gb[4] = {};
      if (on) { load4(x + at.oa, a); load4(x + at.ob, b); load4(g + at.oa, ga); load4(g + at.ob, gb); }
      if (at.turns) turn(ga, gb, cs, sn, -1.0f, p.interleaved);
      float ss = 0.0f, dot = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        ss = fmaf(a[e], a[e], fmaf(b[e], b[e], ss));
        dot = fmaf(a[e] * ga[e], is_q ? wq[e] : wk[e], fmaf(b[e] * gb[e], is_q ? wq[4 + e] : wk[4 + e], dot));
      }
      const float r = rsqrtf(fmaf(lanes_sum<LANES>(ss), inv_d, p.eps));
      const float m = lanes_sum<LANES>(dot) * inv_d * r * r;      // mean(dn w xhat) r
      if (on) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float ta = ga[e] * (a[e] * r), tb = gb[e] * (b[e] * r);
          if (is_q) { sq[e] += ta; sq[4 + e] += tb; } else { sk[e] += ta; sk[4 + e] += tb; }
          a[e] = r * (ga[e] * (is_q ? wq[e] : wk[e]) - a[e] * m);
          b[e] = r * (gb[e] * (is_q ? wq[4 + e] : wk[4 + e]) - b[e] * m);
        }
        T* y = is_q ? static_cast<T*>(p.yq) + row * p.ldyq + hh * p.d : static_cast<T*>(p.yk) + row * p.ldyk + hh * p.d;
        store4(y + at.oa, a);
        store4(y + at.ob, b);
      }
    }
  }
  if (at.live)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = e < 4 ? at.oa + e : at.ob + e - 4;
      sums[(size_t)group * 2 * p.d + c] = sq[e];
      sums[(size_t)group * 2 * p.d + p.d + c] = sk[e];
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * p.d; i += QK_THREADS) {
    float s = 0.0f;
    for (int g = 0; g < GROUPS; ++g) s += sums[(size_t)g * 2 * p.d + i];
    p.part[(size_t)blockIdx.x * 2 * p.d + i] = s;
  }
}
// One warp a column: lanes take the blocks' sums in turn, in 64 bits, and meet in a fixed order.
__global__ void __launch_bounds__(QK_THREADS) qk_sum_weights(const float* part, int blocks, int d, float* dw_q, float* dw_k) {
  pdl_sync();
  const int i = blockIdx.x * (QK_THREADS / 32) + threadIdx.x / 32, lane = threadIdx.x & 31;
  if (i >= 2 * d) return;
  double s = 0.0;
  for (int b = lane; b < blocks; b += 32) s += (double)part[(size_t)b * 2 * d + i];
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
  float* to = i < d ? dw_q : dw_k;
  if (lane == 0 && to) to[i < d ? i : i - d] = (float)s;
}

int check_qk(const rom_qk_config* c, int rows) {
  if (!c || rows < 0 || c->n_q_heads < 1 || c->n_k_heads < 1 || c->d_head < 1 || c->rot_dim < 0 || c->rot_dim > c->d_head) return ROM_ERR_INVALID_ARG;
  if ((c->dtype != ROM_F32 && c->dtype != ROM_BF16) || c->interleaved < 0 || c->interleaved > 1 || !(c->eps > 0.0f) || !isfinite(c->eps)) return ROM_ERR_INVALID_ARG;
  if (c->d_head % 8 != 0 || c->d_head > 256 || c->rot_dim % 16 != 0 || c->n_q_heads > 1024 || c->n_k_heads > 1024 || rows >= 1 << 30) return ROM_ERR_UNSUPPORTED;
  return ROM_OK;
}
int lanes_of(int d) { int n = 1; while (8 * n < d) n *= 2; return n; }
// Heads a group takes: one angle a row and lane costs about as much as two heads, so as many as leave the GPU two groups a lane slot; one where rows are few.
int heads_per_group(const rom_qk_config& c, int rows) {
  const long long all = (long long)rows * (c.n_q_heads + c.n_k_heads), slots = 148LL * 2048 / lanes_of(c.d_head);
  for (int per = 16; per > 1; per /= 2)
    if (all / per >= 2 * slots) return per;
  return 1;
}
constexpr int kBwdBlocks = 148 * 4;
int bwd_blocks(const rom_qk_config& c, int rows) {
  const int per = heads_per_group(c, rows), groups = QK_THREADS / lanes_of(c.d_head);
  const long long items = (long long)rows * ((c.n_q_heads + c.n_k_heads + per - 1) / per), n = (items + groups - 1) / groups;
  return (int)(n < kBwdBlocks ? (n < 1 ? 1 : n) : kBwdBlocks);
}
template <typename F>
cudaError_t by_lanes(int lanes, F&& go) {
  switch (lanes) {
    case 1: return go(std::integral_constant<int, 1>());
    case 2: return go(std::integral_constant<int, 2>());
    case 4: return go(std::integral_constant<int, 4>());
    case 8: return go(std::integral_constant<int, 8>());
    case 16: return go(std::integral_constant<int, 16>());
    default: return go(std::integral_constant<int, 32>());
  }
}
template <typename T>
cudaError_t launch_forward(const rom_qk_config& c, const QkArgs& p, cudaStream_t st) {
  return by_lanes(lanes_of(c.d_head), [&](auto n) {
    constexpr int LANES = decltype(n)::value;
    const int per = heads_per_group(c, p.rows), groups = QK_THREADS / LANES;
    const long long items = (long long)p.rows * ((p.nq + p.nk + per - 1) / per);
    count_launch();
    return launch_k(qk_norm_rope_kernel<T, LANES>, dim3((unsigned)((items + groups - 1) / groups)), QK_THREADS, 0, st, p, per);
  });
}
template <typename T>
cudaError_t launch_backward(const rom_qk_config& c, const QkArgs& p, float* dw_q, float* dw_k, cudaStream_t st) {
  const int blocks = bwd_blocks(c, p.rows);
  const cudaError_t e = by_lanes(lanes_of(c.d_head), [&](auto n) {
    constexpr int LANES = decltype(n)::value;
    const size_t smem = sizeof(float) * (QK_THREADS / LANES) * 2 * p.d;      // at most 32 KB: a group's lanes cover more than half of d / 8
    count_launch();
    return launch_k(qk_norm_rope_bwd_kernel<T, LANES>, dim3(blocks), QK_THREADS, smem, st, p, heads_per_group(c, p.rows));
  });
  if (e != cudaSuccess || (!dw_q && !dw_k)) return e;
  count_launch();
  return launch_k(qk_sum_weights, dim3((2 * p.d + QK_THREADS / 32 - 1) / (QK_THREADS / 32)), QK_THREADS, 0, st, (const float*)p.part, blocks, p.d, dw_q, dw_k);
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
  *bytes = sizeof(float) * 2 * (size_t)cfg->d_head * kBwdBlocks;
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
  if (ws_bytes < sizeof(float) * 2 * (size_t)c.d_head * kBwdBlocks) return ROM_ERR_WORKSPACE;
  if ((rc = check_device()) != ROM_OK) return rc;
  LaunchCounter::count = 0;
  QkArgs p{q, k, dq_out, dk_out, dq, dk, ldq, ldk, lddq, lddk, w_q, w_k, pos, inv_freq, static_cast<float*>(ws), rows, c.n_q_heads, c.n_k_heads, c.d_head, c.rot_dim, c.interleaved, c.eps};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return (c.dtype == ROM_BF16 ? launch_backward<__nv_bfloat16>(c, p, dw_q, dw_k, st) : launch_backward<float>(c, p, dw_q, dw_k, st)) == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

}  // extern "C"
