// Selective scan over packed sequences (rom_scan_ragged): h_t = exp(Delta A) h_{t-1} + B-bar u_t, y_t = (C_t h_t + D u_t) SiLU(z_t), each sequence
// from its slot's state or from zeros.
//
// One warp per sequence and 8 channels, four lanes a channel with four states each, row by row.
#include "rom_serve.cuh"

namespace rom {
namespace {

struct RaggedScan {
  Ragged s;
  const void* u; const float* delta; const float* A; const float* Bm; const float* Cm; long long ldb; const float* D;
  const void* z; long long ldz; const float* h_in; float* h_out; void* y; int De;
};

template <typename T, bool ZOH>
__global__ void __launch_bounds__(128)
scan_ragged_rows(const RaggedScan p) {
  pdl_sync();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int c = blockIdx.x * 32 + (threadIdx.x >> 5) * 8 + g, De = p.De;
  const T* u = static_cast<const T*>(p.u);
  const T* z = static_cast<const T*>(p.z);
  const float4 a4 = __ldg(reinterpret_cast<const float4*>(p.A + (size_t)c * 16) + t);
  const float av[4] = {a4.x, a4.y, a4.z, a4.w}, Dc = p.D ? __ldg(p.D + c) : 0.0f;
  for (int i = blockIdx.y; i < p.s.n_seq; i += gridDim.y) {
    const int first = p.s.start_of(i), end = p.s.end_of(i), slot = p.s.slot_of(i);
    const size_t at = ((size_t)max(slot, 0) * De + c) * 16 + 4 * t;
    float4 h4 = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (p.h_in && slot >= 0 && p.s.resumes(i)) h4 = *reinterpret_cast<const float4*>(p.h_in + at);
    float h[4] = {h4.x, h4.y, h4.z, h4.w};
    for (int r = first; r < end; ++r) {
      const size_t o = (size_t)r * De + c;
      const float dl = __ldg(p.delta + o), uu = to_f32(u[o]);
      const float4 b4 = load4_any(p.Bm + (size_t)r * p.ldb + 4 * t), c4 = load4_any(p.Cm + (size_t)r * p.ldb + 4 * t);
      const float bb[4] = {b4.x, b4.y, b4.z, b4.w}, cc[4] = {c4.x, c4.y, c4.z, c4.w};
      float y = 0.0f;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        float a, e;
        decay(dl * av[n], a, e);
        h[n] = fmaf(a, h[n], (ZOH ? __fdividef(e, av[n]) : dl) * (uu * bb[n]));
        y = fmaf(cc[n], h[n], y);
      }
      y += __shfl_xor_sync(0xffffffffu, y, 1);
      y += __shfl_xor_sync(0xffffffffu, y, 2);
      if (t == 0) {
        y = fmaf(Dc, uu, y);
        if (z) y *= silu_f(to_f32(z[(size_t)r * p.ldz + c]));
        static_cast<T*>(p.y)[o] = from_f32<T>(y);
      }
    }
    if (p.h_out && slot >= 0) *reinterpret_cast<float4*>(p.h_out + at) = make_float4(h[0], h[1], h[2], h[3]);
  }
}

template <typename T>
cudaError_t launch_scan_ragged(const rom_config& c, const RaggedScan& p, cudaStream_t st) {
  auto kern = c.disc_mode == 0 ? scan_ragged_rows<T, true> : scan_ragged_rows<T, false>;
  count_launch();
  return launch_k(kern, dim3(c.d_inner / 32, p.s.n_seq < 4096 ? p.s.n_seq : 4096), 128, 0, st, p);
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
  *bytes = 256;
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
  size_t need = 0;
  if ((rc = rom_scan_ragged_workspace_size(cfg, seqs->n_seq, seqs->rows, &need)) != ROM_OK) return rc;
  if (ws_bytes < need) return ROM_ERR_WORKSPACE;
  if ((rc = check_device()) != ROM_OK) return rc;
  LaunchCounter::count = 0;
  const RaggedScan p{device_view(*seqs), u, delta, A, Bm, Cm, ld_bc, D, z, ldz, h_in, h_out, y, c.d_inner};
  auto launch = c.dtype == ROM_BF16 ? launch_scan_ragged<__nv_bfloat16> : launch_scan_ragged<float>;
  return launch(c, p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

}  // extern "C"
