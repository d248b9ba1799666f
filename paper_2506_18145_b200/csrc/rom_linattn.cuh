// What the kernels of linear attention with a decay per head share.  All of its directions are walks of one recurrence,
//   S <- lambda S + ks k_t v_t^T,   out_t = q_t S,
// over the rows of a sequence, forwards or backwards:
//   forward   (q, k, v) = (q, k, v)           out = o    (scaled on output)
//   dq        (q, k, v) = (dout, v, k)        out = dq   (scaled on output; its state is the forward's, transposed)
//   dv        (q, k, v) = (k, q, dout)        out = dv   backwards, ks = scale; the state starts from ds_out, which meets the last row undecayed
//   dk        (q, k, v) = (v, dout, q)        out = dk   backwards; the state of dv's walk, transposed
// The packed rows of all heads, one head behind the other, are cut into equal runs, one per block.  A sequence counts as many rows more as its start costs (the loads and
// stores of its states and a chunk that is not full), so that a run of many short ones is no longer than one of a part of a long one; cuts inside a sequence come at whole
// chunks of it.  Launch 1 (state only) walks for each cut inside a head the rows of the sequence that reaches over it, up to the cut before; launch 2 chains those states from cut to cut; launch 3
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
  float* last;                     // pool of the states left at the end (when init_all, a sequence that started from zeros leaves zeros), or null
  bool none_resumes;               // every sequence started from zeros, whatever its flag says
  const float* powers;             // [H][2][kLinPowers]
  float* cut_state;                // [cuts, state]: launch 1 writes, launch 2 chains in place, launch 3 reads; [i - 1] belongs to the cut before run i
  float* init_copy;                // [cuts, state] or null: initial states of sequences that start in run i - 1 and reach over the cut before run i (pools in place)
  bool skip_single;                // sequences of one row are another launch's
  void* out;
  int64_t ldo;
  bool out_f32;                    // out is fp32 whatever the storage type
  int32_t* status;
};

// Run i of `blocks` is the units [units i / blocks, units (i + 1) / blocks) of all heads', `per_head` each: a unit is `chunk` rows, a sequence's start `start` rows.
struct LinCut {
  int chunk, start, per_head;
  int blocks;
  long long units;                 // heads * per_head
  bool inside;                     // there are cuts inside heads
  __host__ __device__ __forceinline__ long long bound(int i) const { return units * i / blocks; }
  // The row at place v of a head; monotone.  All lanes of a warp (WARP), or one thread.
  template <bool WARP>
  __device__ __forceinline__ int row_at(const Ragged& q, int v) const {
    int lo = 0, hi = q.n_seq;          // first sequence that starts behind place v
    if (WARP) {
      const int lane = threadIdx.x & 31;
      while (lo < hi) {
        const int step = (hi - lo + 31) / 32, i = lo + lane * step;
        const unsigned m = __ballot_sync(0xffffffffu, i >= hi || q.start_of(min(i, q.n_seq - 1)) + start * i > v);
        if (m == 0) { lo += 31 * step + 1; continue; }
        const int k = __ffs(m) - 1;
        hi = min(hi, lo + k * step);
        if (k > 0) lo += (k - 1) * step + 1;
      }
    } else {
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (q.start_of(mid) + start * mid > v) hi = mid; else lo = mid + 1;
      }
    }
    if (lo == 0) return min(v, q.start_of(0));
    const int first = q.start_of(lo - 1), in = max(v - (first + start * (lo - 1)) - start, 0) / chunk * chunk;
    return min(first + in, q.end_of(lo - 1));
  }
};
// What a run has of one head: rows [a, b).
struct LinItem {
  long long u, u1;                 // next unit, end of the run
  int head, a, b;
  bool last;                       // b is the head's end
  __device__ __forceinline__ LinItem(const LinCut& c, int run) : u(c.bound(run)), u1(c.bound(run + 1)) {}
  __device__ __forceinline__ bool next(const LinCut& c, const Ragged& q) {      // all lanes of a warp
    if (u >= u1) return false;
    head = (int)(u / c.per_head);
    const int c0 = (int)(u - (long long)head * c.per_head), c1 = (int)min((long long)c.per_head, c0 + (u1 - u));
    a = c0 == 0 ? 0 : c.row_at<true>(q, c0 * c.chunk);
    last = c1 == c.per_head;
    b = last ? q.rows : c.row_at<true>(q, c1 * c.chunk);
    u += c1 - c0;
    return true;
  }
};
// The cut before run i: its head and row; row 0: nothing is ahead of it.  All lanes of a warp.
__device__ __forceinline__ void lin_cut_at(const LinCut& c, const Ragged& q, int i, int& head, int& row) {
  const long long u = c.bound(i);
  head = (int)(u / c.per_head);
  const int at = (int)(u - (long long)head * c.per_head);
  row = at == 0 ? 0 : c.row_at<true>(q, at * c.chunk);
}
// Whether a sequence reaches over the cut before row r (0 < r < rows), and which.  All lanes of a warp call it.
__device__ __forceinline__ int lin_spanning(const Ragged& seqs, int r) {
  const int s = seqs.first_from(r) - 1;
  return s >= 0 && seqs.end_of(s) > r ? s : -1;
}
// The same for one thread.
__device__ __forceinline__ int lin_spanning_1(const Ragged& seqs, int r) {
  int lo = 0, hi = seqs.n_seq;         // first sequence whose first row is r or later
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (seqs.start_of(mid) >= r) hi = mid; else lo = mid + 1;
  }
  return lo > 0 && seqs.end_of(lo - 1) > r ? lo - 1 : -1;
}
// The rows that launch 1 walks for the cut before run i (1 <= i < blocks): those of the sequence that reaches over it, back to the cut before or, backwards, on to
// the next one.  False: nothing reaches over it.  All lanes of a warp call it.
__device__ __forceinline__ bool lin_cut_rows(const LinCut& c, int i, bool reverse, const Ragged& seqs, int& head, int& r0, int& r1) {
  int row, h2, near;
  lin_cut_at(c, seqs, i, head, row);
  const int s = row > 0 ? lin_spanning(seqs, row) : -1;
  if (s < 0) return false;
  lin_cut_at(c, seqs, reverse ? i + 1 : i - 1, h2, near);
  if (reverse) {
    r0 = row;
    r1 = min(seqs.end_of(s), h2 == head ? near : seqs.rows);
  } else {
    r0 = max(seqs.start_of(s), h2 == head ? near : 0);
    r1 = row;
  }
  return r1 > r0;
}
// Whether sequence s leaves zeros at its end instead of the state.
__device__ __forceinline__ bool lin_leaves_zeros(const LinPass& p, const Ragged& seqs, int s) { return p.init_all && (p.none_resumes || !seqs.resumes(s)); }
__device__ __forceinline__ const float* lin_init_of(const LinPass& p, const Ragged& seqs, int s, int head) {
  const int slot = seqs.slot_of(s);
  if (!p.init || slot < 0 || !(p.init_all || seqs.resumes(s))) return nullptr;
  return p.init + ((size_t)slot * p.H + head) * ((size_t)p.dk * p.dv);
}


// Launches 1 and 3 on the tensor cores, bf16 (rom_linattn_tc.cu): of the forward (n = 1), or of the backward (states: forward, backward; walks: dq, dv, dk).
cudaError_t launch_lin_states_tc(const LinPass* p, int n, int dk, int dv, const rom_ragged& seqs, const LinCut& cut, bool test_stall, cudaStream_t st);
cudaError_t launch_lin_walks_tc(const LinPass* p, int n, int dk, int dv, const rom_ragged& seqs, const LinCut& cut, bool test_stall, cudaStream_t st);

}  // namespace rom
