// What the serving operators share: packed sequences, state slots, argument checks, the decay of one step.
#pragma once

#include "rom_internal.cuh"

namespace rom {
namespace {

constexpr int kMaxRaggedSeqs = 1 << 20;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Rows of activations may lie `ld` elements of `esz` bytes apart: wide enough, and every row on a 16-byte boundary.
inline bool pitch_ok(int64_t ld, int width, size_t esz) { return ld >= width && (ld * (int64_t)esz) % 16 == 0; }

inline int check_ragged(const rom_ragged* r) {
  if (!r || r->n_seq < 0 || r->rows < 0 || r->n_slots < 0) return ROM_ERR_INVALID_ARG;
  if (r->n_seq > kMaxRaggedSeqs || r->rows >= 1 << 30) return ROM_ERR_UNSUPPORTED;
  if (r->n_seq == 0) return ROM_OK;
  if (!r->seq_start || !aligned4(r->seq_start) || !aligned4(r->slot) || !aligned4(r->resume)) return ROM_ERR_INVALID_ARG;
  return ROM_OK;
}

// Pools of a call: 16-byte aligned, one buffer or two that do not overlap.
inline bool pools_ok(const float* in, const float* out, size_t floats) {
  if (!aligned16(in) || !aligned16(out)) return false;
  if (!in || !out || in == out) return true;
  const uintptr_t a = reinterpret_cast<uintptr_t>(in), b = reinterpret_cast<uintptr_t>(out), n = floats * sizeof(float);
  return a + n <= b || b + n <= a;
}

inline int check_device() {
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess)
    return ROM_ERR_CUDA;
  return major == 10 ? ROM_OK : ROM_ERR_ARCH;
}

// Packed sequences as a kernel sees them.
struct Ragged {
  int n_seq, rows, n_slots;
  const int32_t* start;
  const int32_t* slot;
  const int32_t* resume;
  __device__ __forceinline__ int start_of(int s) const { return min(max(__ldg(start + s), 0), rows); }      // s in [0, n_seq]
  __device__ __forceinline__ int end_of(int s) const { return max(start_of(s + 1), start_of(s)); }
  __device__ __forceinline__ int slot_of(int s) const {      // -1: no state kept
    const int v = slot ? __ldg(slot + s) : s;
    return v >= 0 && v < n_slots ? v : -1;
  }
  __device__ __forceinline__ bool resumes(int s) const { return resume && __ldg(resume + s) != 0; }
  // First sequence whose first row is `row` or later (n_seq: none).  All lanes of a warp call it; 32 sequences are looked at per round.
  __device__ __forceinline__ int first_from(int row) const {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = n_seq;
    while (lo < hi) {
      const int step = (hi - lo + 31) / 32, i = lo + lane * step;
      const unsigned m = __ballot_sync(0xffffffffu, i >= hi || start_of(min(i, n_seq - 1)) >= row);
      if (m == 0) { lo += 31 * step + 1; continue; }
      const int k = __ffs(m) - 1;
      hi = min(hi, lo + k * step);
      if (k > 0) lo += (k - 1) * step + 1;
    }
    return lo;
  }
};
inline Ragged device_view(const rom_ragged& r) { return Ragged{r.n_seq, r.rows, r.n_slots, r.seq_start, r.slot, r.resume}; }

constexpr float kLog2eServe = 1.4426950408889634f;

// a = exp(x), e = exp(x) - 1.  Near zero e comes from its power series (x^8/8! left out: below 2^-25 of e for |x| < 0.35) and a from e,
// so that both keep fp32 accuracy however small the step: the input of a zero-order hold is e / A, and a state that decays by 1e-3 a step
// adds up the errors of a thousand decays.
__device__ __forceinline__ void decay(float2 x, float2& a, float2& e) {
  auto both = [](float v) { return make_float2(v, v); };
  float2 p = __ffma2_rn(x, both(1.0f / 5040.0f), both(1.0f / 720.0f));
  p = __ffma2_rn(p, x, both(1.0f / 120.0f));
  p = __ffma2_rn(p, x, both(1.0f / 24.0f));
  p = __ffma2_rn(p, x, both(1.0f / 6.0f));
  p = __ffma2_rn(p, x, both(0.5f));
  p = __ffma2_rn(p, x, both(1.0f));
  const float2 es = __fmul2_rn(p, x), xl = __fmul2_rn(x, both(kLog2eServe)), al = make_float2(ex2_ftz(xl.x), ex2_ftz(xl.y));
  const float2 el = __fadd2_rn(al, both(-1.0f)), as = __fadd2_rn(es, both(1.0f));
  const bool s0 = fabsf(x.x) < 0.35f, s1 = fabsf(x.y) < 0.35f;
  e = make_float2(s0 ? es.x : el.x, s1 ? es.y : el.y);
  a = make_float2(s0 ? as.x : al.x, s1 ? as.y : al.y);
}

}  // namespace
}  // namespace rom
