// What the kernels of linear attention with a decay per head share.  All of its directions are walks of one recurrence,
//   S <- lambda S + ks k_t v_t^T,   out_t = q_t S,
// over the rows of a sequence, forwards or backwards:
//   forward   (q, k, v) = (q, k, v)           out = o    (scaled on output)
//   dq        (q, k, v) = (dout, v, k)        out = dq   (scaled on output; its state is the forward's, transposed)
//   dv        (q, k, v) = (k, q, dout)        out = dv   backwards, ks = scale; the state starts from ds_out, which meets the last row undecayed
//   dk        (q, k, v) = (v, dout, q)        out = dk   backwards; the state of dv's walk, transposed
// The packed rows of all heads, one head behind the other, are cut into equal runs of chunks, one per block, whatever sequences they hold.  Launch 1 (state only)
// walks for each cut inside a head the rows of the sequence that reaches over it, up to the cut before; launch 2 chains those states from cut to cut; launch 3
// walks every run from the states that reach it.
#pragma once

#include "rom_serve.cuh"

namespace rom {

constexpr int kLinMaxDim = 128;        // of q, k, v and the state, each way
constexpr int kLinMaxBlocks = 296;     // runs, where there are cuts inside heads
constexpr int kLinPowers = 132;        // lambda^0 .. lambda^128 of a head as fp32, and as many of what each lost (two rows of a table in the workspace)

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
  const float* powers;             // [H][2][kLinPowers]
  float* cut_state;                // [cuts, state]: launch 1 writes, launch 2 chains in place, launch 3 reads; [i - 1] belongs to the cut before run i
  float* init_copy;                // [cuts, state] or null: initial states of sequences that start in run i - 1 and reach over the cut before run i (pools in place)
  void* out;
  int64_t ldo;
  bool out_f32;                    // out is fp32 whatever the storage type
  int32_t* status;
};

// Run i of `blocks` is the chunks [units i / blocks, units (i + 1) / blocks) of all heads' chunks.
struct LinCut {
  int chunk, per_head;             // rows of a chunk; chunks of a head
  int blocks;
  long long units;                 // heads * per_head
  bool inside;                     // there are cuts inside heads
  __host__ __device__ __forceinline__ long long bound(int i) const { return units * i / blocks; }
};
// What a run has of one head: rows [a, b).
struct LinItem {
  long long u, u1;                 // next chunk, end of the run
  int head, a, b;
  bool last;                       // b is the head's end
  __device__ __forceinline__ LinItem(const LinCut& c, int run) : u(c.bound(run)), u1(c.bound(run + 1)) {}
  __device__ __forceinline__ bool next(const LinCut& c, int rows) {
    if (u >= u1) return false;
    head = (int)(u / c.per_head);
    const int c0 = (int)(u - (long long)head * c.per_head), c1 = (int)min((long long)c.per_head, c0 + (u1 - u));
    a = c0 * c.chunk;
    last = c1 == c.per_head;
    b = last ? rows : c1 * c.chunk;
    u += c1 - c0;
    return true;
  }
};
// The cut before run i: its head and row; row 0: it lies between two heads.
__device__ __forceinline__ void lin_cut_at(const LinCut& c, int i, int& head, int& row) {
  const long long u = c.bound(i);
  head = (int)(u / c.per_head);
  row = (int)(u - (long long)head * c.per_head) * c.chunk;
}
// Whether a sequence reaches over the cut before row r (0 < r < rows), and which.  All lanes of a warp call it.
__device__ __forceinline__ int lin_spanning(const Ragged& seqs, int r) {
  const int s = seqs.first_from(r) - 1;
  return s >= 0 && seqs.end_of(s) > r ? s : -1;
}
// The rows that launch 1 walks for the cut before run i (1 <= i < blocks): those of the sequence that reaches over it, back to the cut before or, backwards, on to
// the next one.  False: nothing reaches over it.  All lanes of a warp call it.
__device__ __forceinline__ bool lin_cut_rows(const LinCut& c, int i, bool reverse, const Ragged& seqs, int& head, int& r0, int& r1) {
  int row, h2, near;
  lin_cut_at(c, i, head, row);
  const int s = row > 0 ? lin_spanning(seqs, row) : -1;
  if (s < 0) return false;
  lin_cut_at(c, reverse ? i + 1 : i - 1, h2, near);
  if (reverse) {
    r0 = row;
    r1 = min(seqs.end_of(s), h2 == head ? near : seqs.rows);
  } else {
    r0 = max(seqs.start_of(s), h2 == head ? near : 0);
    r1 = row;
  }
  return r1 > r0;
}
__device__ __forceinline__ const float* lin_init_of(const LinPass& p, const Ragged& seqs, int s, int head) {
  const int slot = seqs.slot_of(s);
  if (!p.init || slot < 0 || !(p.init_all || seqs.resumes(s))) return nullptr;
  return p.init + ((size_t)slot * p.H + head) * ((size_t)p.dk * p.dv);
}


// The walk (or launch 1 alone) on the tensor cores, bf16 (rom_linattn_tc.cu).
cudaError_t launch_lin_tc(const LinPass& p, const rom_ragged& seqs, LinCut cut, bool state_only, bool test_stall, cudaStream_t st);

}  // namespace rom
