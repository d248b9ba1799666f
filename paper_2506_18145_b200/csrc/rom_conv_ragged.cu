// Causal depthwise conv + SiLU over packed sequences (rom_conv_ragged): y_t = SiLU(b + sum_j w_j x_{t-(k-1)+j}), windows carried in slots.
//
// HBM bounds it: every row is read and written once, 4 bytes a channel (bf16); the special-function unit is next (two operations a value).
// A warp has 256 (bf16) or 128 channels, 16 bytes a lane, of a tile of rows, which it walks with the window in registers, RB rows computed while
// the next RB are on their way; the rows before a tile are read again, from the L2 mostly.  The first rows are requested before the
// search for the tile's sequences, which takes two dependent loads.
//
// Measured: 16384 rows x 4096 channels (bf16) 55.4 us, 4.84 TB/s = 74 % of the measured copy (53.8 replayed from a graph); half its issue slots, 58 % of the special-function unit (profiles);
// 531 rows of 37 sequences x 512 (fp32) 4.3 us.  Tried: 8 bytes a lane 57 us, eight rows in flight 55 to 60, two 61, whole sequences a warp (serial).
//
// A tile takes the sequences that start in it and what reaches into it from before.  The first k-1 rows of a sequence need its old window, so they all
// belong to the tile in which it starts, even past the tile's end; the same thread then writes the new window.  Nobody else reads or
// writes the slot, so the pool may be updated in place.
#include "rom_serve.cuh"

namespace rom {
namespace {

constexpr int CR_WARPS = 4, CR_ROWS = 4;      // warps per block; rows in flight
constexpr int kConvWarps = 148 * 16;

// 16 bytes of a row as packed pairs
template <typename T>
__device__ __forceinline__ void unpack(const V16<T>& q, float2 (&v)[V16<T>::N / 2]) {
  float f[V16<T>::N];
  q.get(f);
#pragma unroll
  for (int i = 0; i < V16<T>::N / 2; ++i) v[i] = make_float2(f[2 * i], f[2 * i + 1]);
}

template <typename T, int KC>
struct ConvRows {
  static constexpr int P = V16<T>::N / 2;      // pairs a lane
  const T* x; long long ldx; T* y; int De, c;
  float2 w[KC][P], bias[P], win[KC - 1][P];

  __device__ __forceinline__ V16<T> load(int r) const {
    V16<T> q;
    q.load(x + (size_t)r * ldx + c);
    return q;
  }
  __device__ __forceinline__ void put(int r, const V16<T>& q) {
    float2 v[P];
    float o[2 * P];
    unpack(q, v);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      float2 u = bias[i];
#pragma unroll
      for (int j = 0; j < KC - 1; ++j) u = __ffma2_rn(w[j][i], win[j][i], u);
      u = __ffma2_rn(w[KC - 1][i], v[i], u);
      if (sizeof(T) == 2) {
        const float2 t = __fmul2_rn(u, make_float2(-1.4426950408889634f, -1.4426950408889634f));
        const float2 d = __fadd2_rn(make_float2(ex2_ftz(t.x), ex2_ftz(t.y)), make_float2(1.0f, 1.0f));
        u = __fmul2_rn(u, make_float2(rcp_ftz(d.x), rcp_ftz(d.y)));
      } else {
        u = make_float2(silu_f(u.x), silu_f(u.y));
      }
      o[2 * i] = u.x; o[2 * i + 1] = u.y;
#pragma unroll
      for (int j = 0; j + 1 < KC - 1; ++j) win[j][i] = win[j + 1][i];
      win[KC - 2][i] = v[i];
    }
    V16<T>::store(y + (size_t)r * De + c, o);
  }
  // rows [a, b), the window holding the k-1 rows before a, the first CR_ROWS rows requested
  __device__ __forceinline__ void walk(int a, int b, V16<T> (&q)[CR_ROWS]) {
    for (int r0 = a; r0 < b; r0 += CR_ROWS) {
      V16<T> cur[CR_ROWS];
#pragma unroll
      for (int k = 0; k < CR_ROWS; ++k) cur[k] = q[k];
      if (r0 + CR_ROWS < b)
#pragma unroll
        for (int k = 0; k < CR_ROWS; ++k) q[k] = load(min(r0 + CR_ROWS + k, b - 1));
#pragma unroll
      for (int k = 0; k < CR_ROWS; ++k)
        if (r0 + k < b) put(r0 + k, cur[k]);
    }
  }
};

template <typename T, int KC>
__global__ void __launch_bounds__(CR_WARPS * 32, 4)
conv_ragged_kernel(const Ragged s, const T* __restrict__ x, long long ldx, const T* __restrict__ w, const float* __restrict__ bias,
                   const float* win_in, float* win_out, T* __restrict__ y, int De, int tile, int n_tiles) {
  pdl_sync();
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * CR_WARPS + (threadIdx.x >> 5);
  constexpr int P = V16<T>::N / 2;
  const int cb = (De + 64 * P - 1) / (64 * P), ti = (int)(item / cb);
  if (ti >= n_tiles) return;
  const int c = ((int)(item % cb) * 32 + lane) * 2 * P;
  const bool on = c < De;                                  // (a whole warp stays for the search)
  const int r0 = ti * tile, r1 = min(r0 + tile, s.rows);
  ConvRows<T, KC> cr;
  cr.x = x; cr.ldx = ldx; cr.y = y; cr.De = De; cr.c = on ? c : 0;
  V16<T> q[CR_ROWS], halo[KC - 1], wq[KC];
  if (s.rows > 0) {
#pragma unroll
    for (int k = 0; k < KC - 1; ++k) halo[k] = cr.load(max(r0 - (KC - 1) + k, 0));
#pragma unroll
    for (int k = 0; k < CR_ROWS; ++k) q[k] = cr.load(min(r0 + k, s.rows - 1));      // (a sequence may go on past r1)
  }
#pragma unroll
  for (int j = 0; j < KC; ++j) wq[j].load(w + (size_t)j * De + cr.c);
#pragma unroll
  for (int i = 0; i < P; ++i) cr.bias[i] = bias ? make_float2(__ldg(bias + cr.c + 2 * i), __ldg(bias + cr.c + 2 * i + 1)) : make_float2(0.0f, 0.0f);
  const int s0 = s.first_from(r0);
  if (!on) return;
#pragma unroll
  for (int j = 0; j < KC; ++j) unpack(wq[j], cr.w[j]);
  for (int i = max(s0 - 1, 0); i < s.n_seq; ++i) {
    const int first = s.start_of(i), end = s.end_of(i);
    int from, stop;
    if (i < s0) {                                          // what reaches into the tile: its rows from the k-1st on
      from = max(r0, first + KC - 1); stop = min(r1, end);
      if (from >= stop) continue;
      if (from > r0)
#pragma unroll
        for (int k = 0; k < KC - 1; ++k) halo[k] = cr.load(from - (KC - 1) + k);
#pragma unroll
      for (int k = 0; k < KC - 1; ++k) unpack(halo[k], cr.win[k]);
    } else {                                               // what starts in it (the last tile: empty sequences behind the last row too)
      if (first >= r1 && !(r1 == s.rows && first == r1)) break;
      from = first; stop = min(end, max(r1, first + KC - 1));
      const int slot = s.slot_of(i);
      const size_t at = (size_t)max(slot, 0) * (KC - 1) * De + c;
      const bool old = win_in && slot >= 0 && s.resumes(i);
#pragma unroll
      for (int k = 0; k < KC - 1; ++k)
#pragma unroll
        for (int n = 0; n < P / 2; ++n) {
          const float4 p = old ? *reinterpret_cast<const float4*>(win_in + at + (size_t)k * De + 4 * n) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          cr.win[k][2 * n] = make_float2(p.x, p.y); cr.win[k][2 * n + 1] = make_float2(p.z, p.w);
        }
    }
    if (from != r0 && from < stop)                         // (the rows at r0 are on their way)
#pragma unroll
      for (int k = 0; k < CR_ROWS; ++k) q[k] = cr.load(min(from + k, stop - 1));
    cr.walk(from, stop, q);
    if (i < s0 || !win_out) continue;
    const int slot = s.slot_of(i);
    if (slot < 0) continue;
    if (stop < end)                                        // it goes on past the tile, which has at least k-1 of its rows: its last ones
#pragma unroll
      for (int k = 0; k < KC - 1; ++k) unpack(cr.load(end - (KC - 1) + k), cr.win[k]);
#pragma unroll
    for (int k = 0; k < KC - 1; ++k) {
      float* o = win_out + ((size_t)slot * (KC - 1) + k) * De + c;
#pragma unroll
      for (int i = 0; i < P / 2; ++i)
        *reinterpret_cast<float4*>(o + 4 * i) = make_float4(cr.win[k][2 * i].x, cr.win[k][2 * i].y, cr.win[k][2 * i + 1].x, cr.win[k][2 * i + 1].y);
    }
  }
}

template <typename T>
cudaError_t launch_conv_ragged(const rom_config& c, const Ragged& s, const void* x, int64_t ldx, const void* w, const float* bias, const float* win_in,
                               float* win_out, void* y, cudaStream_t st) {
  auto kern = c.d_conv == 2 ? conv_ragged_kernel<T, 2> : c.d_conv == 3 ? conv_ragged_kernel<T, 3> : conv_ragged_kernel<T, 4>;
  const long long cb = (c.d_inner + 32 * V16<T>::N - 1) / (32 * V16<T>::N);
  // Rows per tile: 32 (16384 x 4096: 8 rows 64.2 us, 16 56.2, 32 53.8, 56 53.1, 111 52.6), fewer while that leaves the GPU short of warps: the sequences that start in a tile are walked one after the other.
  const long long fit = (cb * s.rows + kConvWarps - 1) / kConvWarps;
  const int tile = fit < 1 ? 1 : fit > 32 ? 32 : (int)fit;
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
