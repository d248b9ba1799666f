// What the kernels of linear attention with a decay per head share.  All of its directions are walks of one recurrence,
//   S <- lambda S + ks k_t v_t^T,   out_t = q_t S,
// over the rows of a sequence, forwards or backwards:
//   forward   (q, k, v) = (q, k, v)           out = o    (scaled on output)
//   dq        (q, k, v) = (dout, v, k)        out = dq   (scaled on output; its state is the forward's, transposed)
//   dv        (q, k, v) = (k, q, dout)        out = dv   backwards, ks = scale; the state starts from ds_out, which meets the last row undecayed
//   dk        (q, k, v) = (v, dout, q)        out = dk   backwards; the state of dv's walk, transposed
// The packed rows are cut into segments of equal length whatever sequences they hold.  Launch 1 (state only) walks in each segment the rows of the
// sequence that reaches over its far end, launch 2 chains those states from segment to segment, launch 3 walks every segment's rows from the states
// that reach it.
#pragma once

#include "rom_serve.cuh"

namespace rom {

constexpr int kLinMaxDim = 128;      // of q, k, v and the state, each way
constexpr int kLinMaxSegs = 512;

struct LinPass {
  const void *q, *k, *v;
  int64_t ldq, ldk, ldv;           // row pitches, elements
  int qdiv, kdiv, vdiv;            // value head h uses head h / div
  int H, dk, dv;                   // inner and outer width of this walk's state
  const float* log_decay;
  float p_scale, inter_scale, k_scale;      // of q.k inside a chunk, of q S, of the keys that enter the state
  bool reverse;                    // the walk runs from a sequence's last row to its first
  bool transposed;                 // states in memory are [dv, dk] of this walk
  const float* init;               // pool of the states that sequences start from, or null
  bool init_all;                   // every sequence starts from it (else: those that resume)
  bool early;                      // it meets the first row undecayed, and the state left at the end is decayed once more
  float* last;                     // pool of the states left at the end (a sequence that does not resume leaves zeros when init_all), or null
  float* seg_state;                // [segments, H, state]: launch 1 writes, launch 2 chains in place, launch 3 reads; [b - 1] belongs to the cut before segment b
  float* init_copy;                // [segments, H, state] or null: initial states of sequences that start in a segment and reach over its end (pools in place)
  void* out;
  int64_t ldo;
  bool out_f32;                    // out is fp32 whatever the storage type
  int32_t* status;
};

struct LinCut { int seg_rows, n_seg; };

// Whether a sequence reaches over the cut before row r (0 < r < rows), and which.  All lanes of a warp call it.
__device__ __forceinline__ int lin_spanning(const Ragged& seqs, int r) {
  const int s = seqs.first_from(r) - 1;
  return s >= 0 && seqs.end_of(s) > r ? s : -1;
}
__device__ __forceinline__ const float* lin_init_of(const LinPass& p, const Ragged& seqs, int s, int head) {
  const int slot = seqs.slot_of(s);
  if (!p.init || slot < 0 || !(p.init_all || seqs.resumes(s))) return nullptr;
  return p.init + ((size_t)slot * p.H + head) * ((size_t)p.dk * p.dv);
}


// The walk (or launch 1 alone) on the tensor cores, bf16 (rom_linattn_tc.cu).
cudaError_t launch_lin_tc(const LinPass& p, const rom_ragged& seqs, LinCut cut, bool state_only, bool test_stall, cudaStream_t st);

}  // namespace rom
