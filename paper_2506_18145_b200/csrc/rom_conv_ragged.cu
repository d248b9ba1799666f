// Causal depthwise conv + SiLU over packed sequences (rom_conv_ragged): y_t = SiLU(b + sum_j w_j x_{t-(k-1)+j}), windows carried in slots.
//
// HBM bounds it: every row is read and written once, 4 bytes a channel (bf16).  A warp has 256 channels (16 or 32 bytes a lane) of a tile of
// rows, which it walks with the window in registers, RB rows in flight; the rows before a tile are read again, from the L2 mostly.
//
// A tile takes the sequences that start in it and what reaches into it from before.  The first k-1 rows of a sequence need its old window, so they all
// belong to the tile in which it starts, even past the tile's end; the same thread then writes the new window.  Nobody else reads or
// writes the slot, so the pool may be updated in place.
#include "rom_serve.cuh"

namespace rom {
namespace {

constexpr int CR_WARPS = 4;

template <typename T, int KC>
struct ConvRows {
  static constexpr int RB = sizeof(T) == 2 ? 8 : 4;      // rows in flight
  const T* x; long long ldx; T* y; int De, c;
  float w[KC][8], bias[8], win[KC - 1][8];

  __device__ __forceinline__ void shift(const float (&v)[8]) {
#pragma unroll
    for (int q = 0; q + 1 < KC - 1; ++q)
#pragma unroll
      for (int i = 0; i < 8; ++i) win[q][i] = win[q + 1][i];
#pragma unroll
    for (int i = 0; i < 8; ++i) win[KC - 2][i] = v[i];
  }
  __device__ __forceinline__ void load_row(int r, float (&v)[8]) const {
    Raw8<T> q;
    q.load(x + (size_t)r * ldx + c);
    q.get(v);
  }
  // rows [a, b), the window holding the k-1 rows before a
  __device__ __forceinline__ void walk(int a, int b) {
    for (int r0 = a; r0 < b; r0 += RB) {
      Raw8<T> q[RB];
#pragma unroll
      for (int k = 0; k < RB; ++k)
        if (r0 + k < b) q[k].load(x + (size_t)(r0 + k) * ldx + c);
#pragma unroll
      for (int k = 0; k < RB; ++k)
        if (r0 + k < b) {
          float v[8], u[8];
          q[k].get(v);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            u[i] = bias[i];
#pragma unroll
            for (int j = 0; j < KC - 1; ++j) u[i] = fmaf(w[j][i], win[j][i], u[i]);
            u[i] = fmaf(w[KC - 1][i], v[i], u[i]);
            u[i] = sizeof(T) == 2 ? silu_fast(u[i]) : silu_f(u[i]);
          }
          Raw8<T>::store(y + (size_t)(r0 + k) * De + c, u);
          shift(v);
        }
    }
  }
};

template <typename T, int KC>
__global__ void __launch_bounds__(CR_WARPS * 32)
conv_ragged_kernel(const Ragged s, const T* __restrict__ x, long long ldx, const T* __restrict__ w, const float* __restrict__ bias,
                   const float* win_in, float* win_out, T* __restrict__ y, int De, int tile, int n_tiles) {
  pdl_sync();
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * CR_WARPS + (threadIdx.x >> 5);
  const int cb = (De / 8 + 31) / 32, ti = (int)(item / cb);
  if (ti >= n_tiles) return;
  const int c = ((int)(item % cb) * 32 + lane) * 8;
  const bool on = c < De;                                  // (a whole warp stays for the search)
  const int r0 = ti * tile, r1 = min(r0 + tile, s.rows);
  const int s0 = s.first_from(r0);
  if (!on) return;
  ConvRows<T, KC> cr;
  cr.x = x; cr.ldx = ldx; cr.y = y; cr.De = De; cr.c = c;
  {
    Raw8<T> q[KC];
#pragma unroll
    for (int j = 0; j < KC; ++j) q[j].load(w + (size_t)j * De + c);
#pragma unroll
    for (int j = 0; j < KC; ++j) q[j].get(cr.w[j]);
#pragma unroll
    for (int i = 0; i < 8; ++i) cr.bias[i] = bias ? __ldg(bias + c + i) : 0.0f;
  }
  if (s0 > 0) {                                            // what reaches into the tile: its rows from the k-1st on
    const int first = s.start_of(s0 - 1), a = max(r0, first + KC - 1), b = min(r1, s.end_of(s0 - 1));
    if (a < b) {
#pragma unroll
      for (int q = 0; q < KC - 1; ++q) cr.load_row(a - (KC - 1) + q, cr.win[q]);
      cr.walk(a, b);
    }
  }
  for (int i = s0; i < s.n_seq; ++i) {                     // what starts in it (the last tile: empty sequences behind the last row too)
    const int first = s.start_of(i), end = s.end_of(i);
    if (first >= r1 && !(r1 == s.rows && first == r1)) break;
    const int slot = s.slot_of(i);
    const size_t at = (size_t)max(slot, 0) * (KC - 1) * De + c;
    const bool old = win_in && slot >= 0 && s.resumes(i);
    float past[KC - 1][8];
#pragma unroll
    for (int q = 0; q < KC - 1; ++q)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 v = old ? *reinterpret_cast<const float4*>(win_in + at + (size_t)q * De + 4 * h) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        past[q][4 * h] = v.x; past[q][4 * h + 1] = v.y; past[q][4 * h + 2] = v.z; past[q][4 * h + 3] = v.w;
      }
    if (win_out && slot >= 0) {                            // entry q: row end - (k-1) + q, or that far into the old window
#pragma unroll
      for (int q = 0; q < KC - 1; ++q) {
        float v[8];
        const int r = end - (KC - 1) + q;
        if (r >= first) cr.load_row(r, v);
        else {
#pragma unroll
          for (int p = 0; p < KC - 1; ++p)
            if (p == r - first + KC - 1)
#pragma unroll
              for (int k = 0; k < 8; ++k) v[k] = past[p][k];
        }
        float* o = win_out + at + (size_t)q * De;
        *reinterpret_cast<float4*>(o) = make_float4(v[0], v[1], v[2], v[3]);
        *reinterpret_cast<float4*>(o + 4) = make_float4(v[4], v[5], v[6], v[7]);
      }
    }
#pragma unroll
    for (int q = 0; q < KC - 1; ++q)
#pragma unroll
      for (int k = 0; k < 8; ++k) cr.win[q][k] = past[q][k];
    cr.walk(first, min(end, max(r1, first + KC - 1)));
  }
}

template <typename T>
cudaError_t launch_conv_ragged(const rom_config& c, const Ragged& s, const void* x, int64_t ldx, const void* w, const float* bias, const float* win_in,
                               float* win_out, void* y, cudaStream_t st) {
  auto kern = c.d_conv == 2 ? conv_ragged_kernel<T, 2> : c.d_conv == 3 ? conv_ragged_kernel<T, 3> : conv_ragged_kernel<T, 4>;
  const int tile = 16;
  const long long cb = (c.d_inner / 8 + 31) / 32;
  const int n_tiles = s.rows > 0 ? (s.rows + tile - 1) / tile : 1;
  const long long blocks = (cb * n_tiles + CR_WARPS - 1) / CR_WARPS;
  if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
  count_launch();
  return launch_k(kern, dim3((unsigned)blocks), CR_WARPS * 32, 0, st, s, (const T*)x, (long long)ldx, (const T*)w, bias, win_in, win_out, (T*)y, c.d_inner, tile, n_tiles);
}

}  // namespace
}  // namespace rom

using namespace rom;

extern "C" int rom_conv_ragged(const rom_config* cfg, const rom_ragged* seqs, const void* x, int64_t ldx, const void* w_conv, const float* b_conv,
                               const float* win_in, float* win_out, void* y, void* stream) {
  int rc = check_config(cfg, 2);
  if (rc != ROM_OK) return rc;
  const rom_config& c = *cfg;
  if (c.d_conv < 2 || c.d_conv > 4) return c.d_conv < 1 ? ROM_ERR_INVALID_ARG : ROM_ERR_UNSUPPORTED;
  if ((rc = check_ragged(seqs)) != ROM_OK) return rc;
  if (seqs->n_seq == 0) return ROM_OK;
  const size_t esz = c.dtype == ROM_BF16 ? 2 : 4;
  if (!w_conv || (seqs->rows > 0 && (!x || !y)) || !pitch_ok(ldx, c.d_inner, esz)) return ROM_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(w_conv) || !aligned16(y) || !aligned4(b_conv)) return ROM_ERR_INVALID_ARG;
  if (!pools_ok(win_in, win_out, (size_t)seqs->n_slots * (c.d_conv - 1) * c.d_inner)) return ROM_ERR_INVALID_ARG;
  if ((rc = check_device()) != ROM_OK) return rc;
  LaunchCounter::count = 0;
  auto launch = c.dtype == ROM_BF16 ? launch_conv_ragged<__nv_bfloat16> : launch_conv_ragged<float>;
  return launch(c, device_view(*seqs), x, ldx, w_conv, b_conv, win_in, win_out, y, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}
