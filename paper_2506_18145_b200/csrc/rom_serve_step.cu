// One token of many sequences, their states in slots of a pool: the short conv on the slot's window, the recurrence on the slot's state.
// Both move states: 12 d_inner bytes in and out a token for the conv (four taps), 64 d_inner in and out for the scan; HBM bounds them from
// some tens of tokens on, the latency of two dependent loads (slot, then state) below.
// Measured at 4096 channels (bf16): 512 tokens conv 12.8 us (4.4 TB/s; 1.8 us of it a launch), scan 53.7 us (5.2 TB/s, 79 % of the measured copy; 50.8 replayed from a graph); 64 tokens 2.9 and
// 7.3 us; one token 1.8 and 1.9 us.  Scan, tried: blocks of eight warps 56 to 63 us, of four 52, of one 54; four tokens a warp 76; plain stores of
// the states 50.9 but 9.9 at 64 tokens.
#include "rom_serve.cuh"

namespace rom {
namespace {

// ---------------------------------------------------------------------------------------------- conv
// A thread has eight channels of one token: 16 (bf16) or 32 bytes of x, 32 of each window row.
template <typename T, int KC>
__global__ void __launch_bounds__(128)
conv_slot_step(const T* __restrict__ x, long long ldx, const T* __restrict__ w, const float* __restrict__ bias, const int32_t* __restrict__ slot,
               int n_slots, const float* win_in, float* win_out, T* __restrict__ y, int De, int B) {
  pdl_sync();
  const int g = blockIdx.x * 32 + (threadIdx.x & 31), b = blockIdx.y * 4 + (threadIdx.x >> 5);
  if (b >= B || g * 8 >= De) return;
  const int sl = slot ? __ldg(slot + b) : b;
  const int c = g * 8;
  Raw8<T> xq, wq[KC];
  xq.load(x + (size_t)b * ldx + c);
#pragma unroll
  for (int q = 0; q < KC; ++q) wq[q].load(w + (size_t)q * De + c);
  float u[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = bias ? __ldg(bias + c + i) : 0.0f;
  if (sl < 0 || sl >= n_slots) return;
  const size_t at = ((size_t)sl * (KC - 1)) * De + c;
  float v[KC][8], wv[8];
#pragma unroll
  for (int q = 0; q < KC - 1; ++q) {
    const float4 a = *reinterpret_cast<const float4*>(win_in + at + (size_t)q * De), d = *reinterpret_cast<const float4*>(win_in + at + (size_t)q * De + 4);
    v[q][0] = a.x; v[q][1] = a.y; v[q][2] = a.z; v[q][3] = a.w; v[q][4] = d.x; v[q][5] = d.y; v[q][6] = d.z; v[q][7] = d.w;
  }
  xq.get(v[KC - 1]);
#pragma unroll
  for (int q = 0; q < KC; ++q) {
    wq[q].get(wv);
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = fmaf(wv[i], v[q][i], u[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = sizeof(T) == 2 ? silu_fast(u[i]) : silu_f(u[i]);
  Raw8<T>::store(y + (size_t)b * De + c, u);
#pragma unroll
  for (int q = 0; q < KC - 1; ++q) {
    float* o = win_out + at + (size_t)q * De;
    *reinterpret_cast<float4*>(o) = make_float4(v[q + 1][0], v[q + 1][1], v[q + 1][2], v[q + 1][3]);
    *reinterpret_cast<float4*>(o + 4) = make_float4(v[q + 1][4], v[q + 1][5], v[q + 1][6], v[q + 1][7]);
  }
}

template <typename T>
cudaError_t launch_conv_slot_step(const rom_config& c, const void* x, int64_t ldx, const void* w, const float* bias, const int32_t* slot, int n_slots,
                                  const float* win_in, float* win_out, void* y, cudaStream_t st) {
  auto kern = c.d_conv == 2 ? conv_slot_step<T, 2> : c.d_conv == 3 ? conv_slot_step<T, 3> : conv_slot_step<T, 4>;
  count_launch();
  return launch_k(kern, dim3((c.d_inner / 8 + 31) / 32, (c.B + 3) / 4), 128, 0, st, (const T*)x, (long long)ldx, (const T*)w, bias, slot, n_slots, win_in,
                  win_out, (T*)y, c.d_inner, c.B);
}

// ---------------------------------------------------------------------------------------------- scan
// A warp has 32 channels of one token: four float4 of state a lane (states 4 t .. of channels 8 i + g, i < 4, lane = 4 g + t), so that states move
// as whole 512-byte rows.  u, Delta, z and y go by the lane's own channel 8 t + g: whole 64- or 128-byte rows too; the quad's lanes hand
// their u and Delta round and meet for the sums over states so that each ends with its own channel's.
// The two warps of a block share their channels, that is A; beyond some thousand blocks a warp has TOK tokens, whose states are requested
// together.
constexpr int SS_WARPS = 2, kSlotBlocks = 148 * 32;
template <typename T, bool ZOH, int TOK>
__global__ void __launch_bounds__(SS_WARPS * 32)
scan_slot_step(const T* __restrict__ u, const float* __restrict__ delta, const float* __restrict__ A, const float* __restrict__ Bm,
               const float* __restrict__ Cm, long long ldb, const float* __restrict__ D, const T* __restrict__ z, long long ldz,
               const int32_t* __restrict__ slot, int n_slots, const float* h_in, float* h_out, T* __restrict__ y, int De, int B) {
  pdl_sync();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int b0 = blockIdx.y * SS_WARPS * TOK + (threadIdx.x >> 5), c0 = blockIdx.x * 32, mine = c0 + 8 * t + g;
  int sl[TOK];
#pragma unroll
  for (int k = 0; k < TOK; ++k) {
    const int b = b0 + k * SS_WARPS;
    sl[k] = b >= B ? -1 : slot ? __ldg(slot + b) : b;
    if (sl[k] >= n_slots) sl[k] = -1;
  }
  float4 a4[4], h4[TOK][4], b4[TOK], c4[TOK];
  float uu[TOK], dl[TOK], zz[TOK];
#pragma unroll
  for (int i = 0; i < 4; ++i) a4[i] = __ldg(reinterpret_cast<const float4*>(A + (size_t)(c0 + 8 * i + g) * 16) + t);
  const float Dc = D ? __ldg(D + mine) : 0.0f;
#pragma unroll
  for (int k = 0; k < TOK; ++k) {
    const size_t b = min(b0 + k * SS_WARPS, B - 1), at = b * De + mine;
    uu[k] = to_f32(u[at]); dl[k] = __ldg(delta + at); zz[k] = z ? to_f32(z[b * ldz + mine]) : 0.0f;
    b4[k] = load4_any(Bm + b * ldb + 4 * t); c4[k] = load4_any(Cm + b * ldb + 4 * t);
  }
#pragma unroll
  for (int k = 0; k < TOK; ++k)
    if (sl[k] >= 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) h4[k][i] = *reinterpret_cast<const float4*>(h_in + ((size_t)sl[k] * De + c0 + 8 * i + g) * 16 + 4 * t);
#pragma unroll
  for (int k = 0; k < TOK; ++k) {
    if (sl[k] < 0) continue;
    const float bb[4] = {b4[k].x, b4[k].y, b4[k].z, b4[k].w}, cc[4] = {c4[k].x, c4[k].y, c4[k].z, c4[k].w};
    float part[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float ui = __shfl_sync(0xffffffffu, uu[k], (lane & 28) + i), di = __shfl_sync(0xffffffffu, dl[k], (lane & 28) + i);
      const float av[4] = {a4[i].x, a4[i].y, a4[i].z, a4[i].w};
      float hv[4] = {h4[k][i].x, h4[k][i].y, h4[k][i].z, h4[k][i].w}, p = 0.0f;
#pragma unroll
      for (int n = 0; n < 4; n += 2) {
        float2 a, e;
        decay(make_float2(di * av[n], di * av[n + 1]), a, e);
        hv[n] = fmaf(a.x, hv[n], (ZOH ? __fdividef(e.x, av[n]) : di) * (ui * bb[n]));
        hv[n + 1] = fmaf(a.y, hv[n + 1], (ZOH ? __fdividef(e.y, av[n + 1]) : di) * (ui * bb[n + 1]));
        p = fmaf(cc[n + 1], hv[n + 1], fmaf(cc[n], hv[n], p));
      }
      __stcs(reinterpret_cast<float4*>(h_out + ((size_t)sl[k] * De + c0 + 8 * i + g) * 16 + 4 * t), make_float4(hv[0], hv[1], hv[2], hv[3]));
      part[i] = p;
    }
    // sums over the quad: lane t keeps channel group t
    const bool hi = t & 2, odd = t & 1;
    const float s0 = (hi ? part[2] : part[0]) + __shfl_xor_sync(0xffffffffu, hi ? part[0] : part[2], 2);
    const float s1 = (hi ? part[3] : part[1]) + __shfl_xor_sync(0xffffffffu, hi ? part[1] : part[3], 2);
    float o = (odd ? s1 : s0) + __shfl_xor_sync(0xffffffffu, odd ? s0 : s1, 1);
    o = fmaf(Dc, uu[k], o);
    if (z) o *= sizeof(T) == 2 ? silu_fast(zz[k]) : silu_f(zz[k]);
    y[(size_t)(b0 + k * SS_WARPS) * De + mine] = from_f32<T>(o);
  }
}

template <typename T>
cudaError_t launch_scan_slot_step(const rom_config& c, const void* u, const float* delta, const float* A, const float* Bm, const float* Cm, int64_t ldb,
                                  const float* D, const void* z, int64_t ldz, const int32_t* slot, int n_slots, const float* h_in, float* h_out, void* y,
                                  cudaStream_t st) {
  const bool many = (long long)(c.d_inner / 32) * ((c.B + SS_WARPS - 1) / SS_WARPS) >= kSlotBlocks;
  auto kern = many ? (c.disc_mode == 0 ? scan_slot_step<T, true, 2> : scan_slot_step<T, false, 2>)
                   : (c.disc_mode == 0 ? scan_slot_step<T, true, 1> : scan_slot_step<T, false, 1>);
  const int per = SS_WARPS * (many ? 2 : 1);
  count_launch();
  return launch_k(kern, dim3(c.d_inner / 32, (c.B + per - 1) / per), SS_WARPS * 32, 0, st, (const T*)u, delta, A, Bm, Cm, (long long)ldb, D,
                  (const T*)z, (long long)ldz, slot, n_slots, h_in, h_out, (T*)y, c.d_inner, c.B);
}

int check_step(const rom_config* c) {
  const int rc = check_config(c, 2);
  if (rc != ROM_OK) return rc;
  return c->L == 1 ? ROM_OK : ROM_ERR_INVALID_ARG;
}

}  // namespace
}  // namespace rom

using namespace rom;

extern "C" {

int rom_conv_step(const rom_config* cfg, const void* x, int64_t ldx, const void* w_conv, const float* b_conv, const int32_t* slot, int32_t n_slots,
                  const float* win_in, float* win_out, void* y, void* stream) {
  int rc = check_step(cfg);
  if (rc != ROM_OK) return rc;
  const rom_config& c = *cfg;
  if (c.d_conv < 2 || c.d_conv > 4) return c.d_conv < 1 ? ROM_ERR_INVALID_ARG : ROM_ERR_UNSUPPORTED;
  const size_t esz = c.dtype == ROM_BF16 ? 2 : 4;
  if (!x || !w_conv || !win_in || !win_out || !y || n_slots < 0 || !pitch_ok(ldx, c.d_inner, esz)) return ROM_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(w_conv) || !aligned16(y) || !aligned4(b_conv) || !aligned4(slot)) return ROM_ERR_INVALID_ARG;
  if (!pools_ok(win_in, win_out, (size_t)n_slots * (c.d_conv - 1) * c.d_inner)) return ROM_ERR_INVALID_ARG;
  if ((rc = check_device()) != ROM_OK) return rc;
  LaunchCounter::count = 0;
  auto launch = c.dtype == ROM_BF16 ? launch_conv_slot_step<__nv_bfloat16> : launch_conv_slot_step<float>;
  return launch(c, x, ldx, w_conv, b_conv, slot, n_slots, win_in, win_out, y, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

int rom_scan_step(const rom_config* cfg, const void* u, const float* delta, const float* A, const float* Bm, const float* Cm, int64_t ld_bc,
                  const float* D, const void* z, int64_t ldz, const int32_t* slot, int32_t n_slots, const float* h_in, float* h_out, void* y,
                  void* stream) {
  int rc = check_step(cfg);
  if (rc != ROM_OK) return rc;
  const rom_config& c = *cfg;
  const size_t esz = c.dtype == ROM_BF16 ? 2 : 4;
  if (!u || !delta || !A || !Bm || !Cm || !h_in || !h_out || !y || n_slots < 0) return ROM_ERR_INVALID_ARG;
  if (ld_bc < c.d_state || (z && !pitch_ok(ldz, c.d_inner, esz))) return ROM_ERR_INVALID_ARG;
  const void* ptrs[] = {u, delta, A, z, y};
  for (const void* p : ptrs)
    if (!aligned16(p)) return ROM_ERR_INVALID_ARG;
  if (!aligned4(D) || !aligned4(Bm) || !aligned4(Cm) || !aligned4(slot)) return ROM_ERR_INVALID_ARG;
  if (!pools_ok(h_in, h_out, (size_t)n_slots * c.d_inner * c.d_state)) return ROM_ERR_INVALID_ARG;
  if ((rc = check_device()) != ROM_OK) return rc;
  LaunchCounter::count = 0;
  auto launch = c.dtype == ROM_BF16 ? launch_scan_slot_step<__nv_bfloat16> : launch_scan_slot_step<float>;
  return launch(c, u, delta, A, Bm, Cm, ld_bc, D, z, ldz, slot, n_slots, h_in, h_out, y, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

}  // extern "C"
