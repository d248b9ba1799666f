// Linear attention with a decay per head: the calls, the plain fp32-FMA walk (fp32 storage; bf16 as a bisecting aid), the chain of segment states, the
// sums over heads that share q and k, the single-token step.  (The bf16 walk on the tensor cores: rom_linattn_tc.cu.)
//
// Walk in chunks of C rows, i and j places in the chunk:
//   out_i = inter lambda^{i+1} q_i S + sum_{j <= i} p lambda^{i-j} (q_i . k_j) v_j,    S <- lambda^C S + sum_j lambda^{C-1-j} ks k_j v_j^T.
// Powers of lambda come from exp in 64 bits, lambda^C as two floats: a state that decays by 2^-11 a row meets the same factor every chunk, and its
// rounding would add up.
#include <math.h>

#include "rom_linattn.cuh"

namespace rom {
namespace {

struct LinJobs { LinPass p[3]; };

constexpr int SIMT_THREADS = 256;
constexpr int SIMT_C = 32;           // rows of a chunk
constexpr int SIMT_DV = 64;          // columns of the state a block owns
constexpr int SIMT_SPITCH = SIMT_DV + 4;

__device__ __forceinline__ float2 ffma2(float a, float2 b, float2 c) { return __ffma2_rn(make_float2(a, a), b, c); }

// One chunk's rows of one head into shared memory as fp32 (rows from `row0` on, or down from it), zeros beyond `len` and `width`.
template <typename T>
__device__ __forceinline__ void load_tile(float* dst, int pitch, const T* src, int64_t ld, int row0, int step, int len, int width, int fill_to) {
  const int pieces = fill_to / 8;
  for (int i = threadIdx.x; i < SIMT_C * pieces; i += SIMT_THREADS) {
    const int r = i / pieces, c = (i - r * pieces) * 8;
    float v[8];
    if (r < len && c < width) {
      Raw8<T> raw;
      raw.load(src + (int64_t)(row0 + step * r) * ld + c);
      raw.get(v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    }
    *reinterpret_cast<float4*>(dst + r * pitch + c) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(dst + r * pitch + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// A block owns up to 64 columns of a state and walks one run of one of the call's walks (blockIdx.z).  256 threads: 16 x 16, each 2 rows x 4 columns of the outputs and
// 8 x 4 of the state.  What bounds it: shared-memory reads of the operands (10 wavefronts for 16 packed FMAs in q S), and for few rows the latency of its launches (37 sequences of
// 531 rows, 8 heads of 64: 50 us a pass).
template <typename T, bool STATE>
__global__ void __launch_bounds__(SIMT_THREADS) lin_walk_simt(const __grid_constant__ LinJobs jobs, Ragged seqs, LinCut cut) {
  extern __shared__ float sm[];
  const LinPass& p = jobs.p[blockIdx.z];
  const int qp = p.dk + 4;
  float* S = sm;                              // [dk][SIMT_SPITCH]
  float* K = S + p.dk * SIMT_SPITCH;          // [C][qp]
  float* V = K + SIMT_C * qp;                 // [C][SIMT_SPITCH]
  float* Q = V + SIMT_C * SIMT_SPITCH;        // [C][qp]
  float* P = Q + (STATE ? 0 : SIMT_C * qp);   // [C][C + 1]
  __shared__ float lam[SIMT_C + 1], lam_lo[SIMT_C + 1];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int run = blockIdx.x, c0 = blockIdx.y * SIMT_DV, wv = min(SIMT_DV, p.dv - c0);
  pdl_sync();
  if (wv <= 0) return;                        // (another walk of this launch is wider)
  const size_t state = (size_t)p.dk * p.dv;
  int head = 0;
  const T *q = nullptr, *k = nullptr, *v = nullptr;
  auto enter = [&](int h) {
    head = h;
    q = static_cast<const T*>(p.q) + (size_t)(head / p.qdiv) * p.dk;
    k = static_cast<const T*>(p.k) + (size_t)(head / p.kdiv) * p.dk;
    v = static_cast<const T*>(p.v) + (size_t)(head / p.vdiv) * p.dv + c0;
    __syncthreads();
    if (tid <= SIMT_C) {
      lam[tid] = __ldcg(p.powers + (size_t)head * 2 * kLinPowers + tid);
      lam_lo[tid] = __ldcg(p.powers + (size_t)head * 2 * kLinPowers + kLinPowers + tid);
    }
    __syncthreads();
  };
  // The block's columns of a state between memory and shared memory, four adjacent numbers of the memory's rows at a time (a transposed state's are a column's).
  auto each4 = [&](auto&& f) {
    const int wide = p.transposed ? p.dk : wv, high = p.transposed ? wv : p.dk, q4 = (wide + 3) / 4, lanes = q4 <= 16 ? 16 : 32;
    for (int r = tid / lanes; r < high; r += SIMT_THREADS / lanes)
      if (tid % lanes < q4) f(r, 4 * (tid % lanes), p.transposed ? (size_t)(c0 + r) * p.dk + 4 * (tid % lanes) : (size_t)r * p.dv + c0 + 4 * (tid % lanes));
  };
  auto load_state = [&](const float* from) {
    __syncthreads();
    if (!from || wv < SIMT_DV)
      for (int i = tid; i < p.dk * SIMT_SPITCH / 4; i += SIMT_THREADS) reinterpret_cast<float4*>(S)[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (!from) return;
    if (wv < SIMT_DV) __syncthreads();
    each4([&](int r, int c, size_t at) {
      const float4 v = *reinterpret_cast<const float4*>(from + at);
      if (p.transposed) { S[c * SIMT_SPITCH + r] = v.x; S[(c + 1) * SIMT_SPITCH + r] = v.y; S[(c + 2) * SIMT_SPITCH + r] = v.z; S[(c + 3) * SIMT_SPITCH + r] = v.w; }
      else *reinterpret_cast<float4*>(S + r * SIMT_SPITCH + c) = v;
    });
  };
  auto store_state = [&](float* to, float f) {      // (never a transposed one)
    __syncthreads();
    each4([&](int r, int c, size_t at) {
      const float4 v = *reinterpret_cast<const float4*>(S + r * SIMT_SPITCH + c);
      *reinterpret_cast<float4*>(to + at) = f == 0.0f ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : make_float4(f * v.x, f * v.y, f * v.z, f * v.w);
    });
  };
  // rows [r0, r1) of one sequence; pool_init: the state they meet is a sequence's initial one
  auto walk = [&](int r0, int r1, bool pool_init) {
    int early = pool_init && p.early ? 1 : 0;
    for (int done = 0, n = r1 - r0; done < n; done += SIMT_C) {
      const int len = min(SIMT_C, n - done), row0 = p.reverse ? r1 - 1 - done : r0 + done, step = p.reverse ? -1 : 1;
      __syncthreads();
      load_tile(K, qp, k, p.ldk, row0, step, len, p.dk, p.dk);
      load_tile(V, SIMT_SPITCH, v, p.ldv, row0, step, len, wv, SIMT_DV);
      if (!STATE) load_tile(Q, qp, q, p.ldq, row0, step, len, p.dk, p.dk);
      __syncthreads();
      if constexpr (!STATE) {
        const bool mine = 2 * ty < len;        // (rows behind the last one cost nothing)
        float s[2][2] = {};
        for (int d = 0; mine && d < p.dk; d += 4) {
          float4 qv[2], kv[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) { qv[i] = *reinterpret_cast<const float4*>(Q + (2 * ty + i) * qp + d); kv[i] = *reinterpret_cast<const float4*>(K + (tx + 16 * i) * qp + d); }
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) s[i][j] = fmaf(qv[i].x, kv[j].x, fmaf(qv[i].y, kv[j].y, fmaf(qv[i].z, kv[j].z, fmaf(qv[i].w, kv[j].w, s[i][j]))));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int gap = 2 * ty + i - (tx + 16 * j);
            P[(2 * ty + i) * (SIMT_C + 1) + tx + 16 * j] = gap >= 0 ? s[i][j] * (p.p_scale * lam[gap]) : 0.0f;
          }
        __syncthreads();
        float2 o[2][2] = {};
        for (int d = 0; mine && d < p.dk; d += 4) {
          float4 qv[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) qv[i] = *reinterpret_cast<const float4*>(Q + (2 * ty + i) * qp + d);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float4 sv = *reinterpret_cast<const float4*>(S + (d + e) * SIMT_SPITCH + 4 * tx);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const float w = e == 0 ? qv[i].x : e == 1 ? qv[i].y : e == 2 ? qv[i].z : qv[i].w;
              o[i][0] = ffma2(w, make_float2(sv.x, sv.y), o[i][0]);
              o[i][1] = ffma2(w, make_float2(sv.z, sv.w), o[i][1]);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float f = p.inter_scale * lam[2 * ty + i + 1 - early];
          o[i][0] = __fmul2_rn(o[i][0], make_float2(f, f));
          o[i][1] = __fmul2_rn(o[i][1], make_float2(f, f));
        }
        for (int j = 0; mine && j <= 2 * ty + 1; ++j) {      // (a row's own and earlier ones alone: a later value may be anything)
          const float4 vv = *reinterpret_cast<const float4*>(V + j * SIMT_SPITCH + 4 * tx);
#pragma unroll
          for (int i = 0; i < 2; ++i)
            if (j <= 2 * ty + i) {
              const float w = P[(2 * ty + i) * (SIMT_C + 1) + j];
              o[i][0] = ffma2(w, make_float2(vv.x, vv.y), o[i][0]);
              o[i][1] = ffma2(w, make_float2(vv.z, vv.w), o[i][1]);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (2 * ty + i < len && 4 * tx < wv) {
            const size_t to = (size_t)(row0 + step * (2 * ty + i)) * p.ldo + (size_t)head * p.dv + c0 + 4 * tx;
            const float r[4] = {o[i][0].x, o[i][0].y, o[i][1].x, o[i][1].y};
            if (sizeof(T) == 4 || p.out_f32) *reinterpret_cast<float4*>(static_cast<float*>(p.out) + to) = make_float4(r[0], r[1], r[2], r[3]);
            else {
              const __nv_bfloat162 lo = __floats2bfloat162_rn(r[0], r[1]), hi = __floats2bfloat162_rn(r[2], r[3]);
              *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + to) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
            }
          }
        __syncthreads();
      }
      // state
      if (8 * ty < p.dk) {
        float2 s[8][2];
        const float f = lam[len - early], fl = lam_lo[len - early];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float4 sv = *reinterpret_cast<const float4*>(S + (8 * ty + e) * SIMT_SPITCH + 4 * tx);
          const float2 x = make_float2(sv.x, sv.y), y = make_float2(sv.z, sv.w);
          s[e][0] = __ffma2_rn(x, make_float2(f, f), __fmul2_rn(x, make_float2(fl, fl)));
          s[e][1] = __ffma2_rn(y, make_float2(f, f), __fmul2_rn(y, make_float2(fl, fl)));
        }
        for (int j = 0; j < len; ++j) {
          const float w = p.k_scale * lam[len - 1 - j];
          const float4 ka = *reinterpret_cast<const float4*>(K + j * qp + 8 * ty), kb = *reinterpret_cast<const float4*>(K + j * qp + 8 * ty + 4);
          const float4 vv = *reinterpret_cast<const float4*>(V + j * SIMT_SPITCH + 4 * tx);
          const float2 v0 = make_float2(w * vv.x, w * vv.y), v1 = make_float2(w * vv.z, w * vv.w);
          const float kk[8] = {ka.x, ka.y, ka.z, ka.w, kb.x, kb.y, kb.z, kb.w};
#pragma unroll
          for (int e = 0; e < 8; ++e) { s[e][0] = ffma2(kk[e], v0, s[e][0]); s[e][1] = ffma2(kk[e], v1, s[e][1]); }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) *reinterpret_cast<float4*>(S + (8 * ty + e) * SIMT_SPITCH + 4 * tx) = make_float4(s[e][0].x, s[e][0].y, s[e][1].x, s[e][1].y);
      }
      early = 0;
    }
  };

  if constexpr (STATE) {
    int h, r0, r1;
    if (!lin_cut_rows(cut, run + 1, p.reverse, seqs, h, r0, r1)) return;
    enter(h);
    load_state(nullptr);
    walk(r0, r1, false);
    store_state(p.cut_state + (size_t)run * state, 1.0f);
  } else {
    for (LinItem it(cut, run); it.next(cut, seqs);) {
      enter(it.head);
      const int a = it.a, b = it.b;
      int s = seqs.first_from(a);
      if (s > 0 && seqs.end_of(s - 1) > a) --s;
      for (; s < seqs.n_seq; ++s) {
        const int st = seqs.start_of(s), en = seqs.end_of(s), r0 = max(st, a), r1 = min(en, b);
        if (st >= b && !it.last) break;
        const int slot = seqs.slot_of(s);
        const bool empty = en <= st, over = !empty && (p.reverse ? en > b : st < a);      // its state comes over a cut
        if ((!empty && r0 >= r1) || (p.skip_single && en - st == 1)) continue;
        if (over) load_state(p.cut_state + (size_t)(p.reverse ? run : run - 1) * state);
        else if (!empty && !p.reverse && p.init_copy && en > b && lin_init_of(p, seqs, s, head)) load_state(p.init_copy + (size_t)run * state);
        else load_state(lin_init_of(p, seqs, s, head));
        if (!empty) walk(r0, r1, !over);
        if (p.last && slot >= 0 && (empty || (p.reverse ? st >= a : en <= b)))
          store_state(p.last + ((size_t)slot * p.H + head) * state, lin_leaves_zeros(p, seqs, s) ? 0.0f : !empty && p.early ? lam[1] : 1.0f);
      }
    }
  }
}

size_t simt_smem(int dk, bool state) { return sizeof(float) * (size_t)(dk * SIMT_SPITCH + SIMT_C * ((state ? 1 : 2) * (dk + 4) + SIMT_SPITCH) + (state ? 0 : SIMT_C * (SIMT_C + 1))); }

template <typename T, bool STATE>
cudaError_t launch_simt(const LinPass* p, int n, const rom_ragged& seqs, const LinCut& cut, cudaStream_t st) {
  LinJobs jobs{};
  int dk = 0, dv = 0;
  for (int i = 0; i < n; ++i) {
    jobs.p[i] = p[i];
    dk = p[i].dk > dk ? p[i].dk : dk;
    dv = p[i].dv > dv ? p[i].dv : dv;
  }
  auto kern = lin_walk_simt<T, STATE>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)simt_smem(kLinMaxDim, STATE));
  if (e != cudaSuccess) return e;
  count_launch();
  return launch_k(kern, dim3(STATE ? cut.blocks - 1 : cut.blocks, (dv + SIMT_DV - 1) / SIMT_DV, n), SIMT_THREADS, simt_smem(dk, STATE), st, jobs, device_view(seqs), cut);
}

// Before launch 1: the status block cleared, and the powers of every head's decay.
__global__ void __launch_bounds__(256) lin_powers(const float* log_decay, int H, float* powers, int32_t* status) {
  pdl_sync();
  if (blockIdx.x == 0 && threadIdx.x < kStatusInts) status[threadIdx.x] = 0;
  const int i = blockIdx.x * 256 + threadIdx.x, head = i / kLinPowers, n = i - head * kLinPowers;
  if (head >= H) return;
  const double l = exp((double)__ldg(log_decay + head) * n);
  const float hi = (float)l;
  powers[(size_t)head * 2 * kLinPowers + n] = hi;
  powers[(size_t)head * 2 * kLinPowers + kLinPowers + n] = (float)(l - (double)hi);
}

// Launch 2: the states that reach every cut, element by element.  A thread owns four adjacent elements of one head.
constexpr int CHAIN_THREADS = 128;
__global__ void __launch_bounds__(CHAIN_THREADS) lin_chain(const __grid_constant__ LinJobs jobs, Ragged seqs, LinCut cut) {
  const LinPass& p = jobs.p[blockIdx.z];
  __shared__ int how[kLinMaxBlocks];            // at the head's cuts: -3 nobody reaches over it; -2 the state comes over a cut; else a sequence starts here: its state's slot, or -1
  // of the state at the cut before, or of the sequence's initial state, in two floats: cuts are as many rows apart, and the rounding of one float would be the same at each of them
  __shared__ float weight[kLinMaxBlocks], weight_lo[kLinMaxBlocks];
  const int head = blockIdx.y;
  const double g = (double)__ldg(p.log_decay + head);
  const long long u0 = (long long)head * cut.per_head, u1 = u0 + cut.per_head;
  int first = (int)(u0 * cut.blocks / cut.units), n = 0;      // the head's cuts: first .. first + n - 1
  while (cut.bound(first) <= u0) ++first;
  while (cut.bound(first + n) < u1) ++n;
  __shared__ int rows[kLinMaxBlocks];
  for (int j = threadIdx.x; j < n; j += CHAIN_THREADS) rows[j] = cut.row_at<false>(seqs, (int)(cut.bound(first + j) - u0) * cut.chunk);
  __syncthreads();
  auto row_of = [&](int j) { return j < 0 ? 0 : j >= n ? seqs.rows : rows[j]; };
  // a thread a cut (a warp a cut, its lanes searching together, took 0.7 us for each of a head's 37)
  for (int j = threadIdx.x; j < n; j += CHAIN_THREADS) {
    const int r = row_of(j), s = lin_spanning_1(seqs, r), far = row_of(p.reverse ? j + 1 : j - 1);
    int h = -3;
    double w = 0.0;
    if (s >= 0) {
      const int away = p.reverse ? seqs.end_of(s) - r : r - seqs.start_of(s), seg = p.reverse ? far - r : r - far, slot = seqs.slot_of(s);
      h = away > seg ? -2 : p.init && (p.init_all || seqs.resumes(s)) ? slot : -1;
      w = exp(g * (h == -2 ? seg : away - (p.early ? 1 : 0)));
    }
    how[j] = h;
    weight[j] = (float)w;
    weight_lo[j] = (float)(w - (double)(float)w);
  }
  pdl_sync();                           // (the tables above come from inputs, which are older than launch 1)
  __syncthreads();
  const size_t state = (size_t)p.dk * p.dv, e = ((size_t)blockIdx.x * CHAIN_THREADS + threadIdx.x) * 4;
  if (e >= state) return;
  float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int i0 = 0; i0 < n; i0 += 4) {
    float4 add[4], init[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {      // (loads of four cuts at a time: nothing of theirs depends on the chain)
      const int j = p.reverse ? n - 1 - (i0 + u) : i0 + u;
      if (i0 + u >= n || how[j] == -3) continue;
      add[u] = *reinterpret_cast<const float4*>(p.cut_state + (size_t)(first + j - 1) * state + e);
      if (how[j] >= 0) init[u] = *reinterpret_cast<const float4*>(p.init + ((size_t)how[j] * p.H + head) * state + e);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i0 + u >= n) break;
      const int j = p.reverse ? n - 1 - (i0 + u) : i0 + u, h = how[j];
      if (h == -3) continue;
      const float w = weight[j], wl = weight_lo[j];
      if (h >= 0) {
        x = init[u];
        if (p.init_copy) *reinterpret_cast<float4*>(p.init_copy + (size_t)(first + j - 1) * state + e) = x;
      }
      x = h != -1 ? make_float4(fmaf(w, x.x, fmaf(wl, x.x, add[u].x)), fmaf(w, x.y, fmaf(wl, x.y, add[u].y)), fmaf(w, x.z, fmaf(wl, x.z, add[u].z)), fmaf(w, x.w, fmaf(wl, x.w, add[u].w)))
                  : add[u];
      *reinterpret_cast<float4*>(p.cut_state + (size_t)(first + j - 1) * state + e) = x;
    }
  }
}

// dst[row, g, :] = sum over the value heads of group g of part[row, h, :], rows that belong to a sequence.
template <typename T>
__global__ void __launch_bounds__(256) lin_sum_heads(const float* part_q, T* dq, const float* part_k, T* dk, Ragged seqs, int H, int G, int d) {
  const float* part = blockIdx.y == 0 ? part_q : part_k;
  T* dst = blockIdx.y == 0 ? dq : dk;
  pdl_sync();
  const int first = seqs.start_of(0), end = seqs.end_of(seqs.n_seq - 1), share = H / G;
  const size_t per_row = (size_t)G * d / 4, n = (size_t)seqs.rows * per_row;
  for (size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (size_t)gridDim.x * blockDim.x) {
    const int row = (int)(i / per_row);
    if (row < first || row >= end) continue;
    const int c = (int)(i - (size_t)row * per_row) * 4, g = c / d;
    const float* from = part + ((size_t)row * H + (size_t)g * share) * d + (c - g * d);
    float4 s = *reinterpret_cast<const float4*>(from);
    for (int h = 1; h < share; ++h) {
      const float4 a = *reinterpret_cast<const float4*>(from + (size_t)h * d);
      s = make_float4(s.x + a.x, s.y + a.y, s.z + a.z, s.w + a.w);
    }
    T* to = dst + (size_t)row * G * d + c;
    to[0] = from_f32<T>(s.x); to[1] = from_f32<T>(s.y); to[2] = from_f32<T>(s.z); to[3] = from_f32<T>(s.w);
  }
}

// ---------------------------------------------------------------- one token
// A block updates 32 columns of one token's and head's state: 4 warps x 4 rows x 8 column quads, every load of the state in flight at once.
// S e^g is S + S (e^g - 1) for slow decays: a factor rounded to fp32 would be off by the same 2^-25 in every one of thousands of steps.
constexpr int STEP_THREADS = 128, STEP_COLS = 32;
// PACKED: the tokens are the sequences of one row among packed ones, which a walk would load and keep a state for one by one.
template <typename T, bool PACKED>
__global__ void __launch_bounds__(STEP_THREADS) lin_step(const T* q, const T* k, const T* v, long long ldq, long long ldk, long long ldv, const float* log_decay,
                                                         const int32_t* slot, int n_slots, const float* s_in, float* s_out, T* o, int H, int share, int dk, int dv,
                                                         int slices, float scale, Ragged seqs) {
  __shared__ float part[STEP_THREADS / 32][STEP_COLS];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int slice = blockIdx.x % slices, bh = blockIdx.x / slices, head = bh % H, b = bh / H;
  const int c = slice * STEP_COLS + (lane & 7) * 4, r0 = warp * 4 + (lane >> 3);
  pdl_sync();
  int sl, row = b;
  bool from, kept = true;              // the state is loaded (else it is zero), is stored
  if (PACKED) {
    row = seqs.start_of(b);
    if (seqs.end_of(b) - row != 1) return;
    sl = seqs.slot_of(b);
    from = s_in && sl >= 0 && seqs.resumes(b);
    kept = s_out && sl >= 0;
  } else {
    sl = slot ? __ldg(slot + b) : b;
    if (sl < 0 || sl >= n_slots) return;
    from = true;
  }
  const size_t base = ((size_t)max(sl, 0) * H + head) * ((size_t)dk * dv);
  const bool mine = c < dv;
  float4 S[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    S[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (from && mine && r < dk) S[i] = *reinterpret_cast<const float4*>(s_in + base + (size_t)r * dv + c);
  }
  const T* qr = q + (size_t)row * ldq + (size_t)(head / share) * dk;
  const T* kr = k + (size_t)row * ldk + (size_t)(head / share) * dk;
  const T* vr = v + (size_t)row * ldv + (size_t)head * dv;
  float vv[4] = {};
  if (mine) { vv[0] = to_f32(vr[c]); vv[1] = to_f32(vr[c + 1]); vv[2] = to_f32(vr[c + 2]); vv[3] = to_f32(vr[c + 3]); }
  const float g = __ldg(log_decay + head), lam = expf(g), em1 = expm1f(g);
  const bool slow = g > -0.5f;
  const float f = slow ? em1 : lam;
  float acc[4] = {};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = r0 + 16 * i;
    if (mine && r < dk) {
      const float kk = to_f32(kr[r]), qq = to_f32(qr[r]);
      float s[4] = {S[i].x, S[i].y, S[i].z, S[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[e] = fmaf(kk, vv[e], slow ? fmaf(s[e], f, s[e]) : s[e] * f);
        acc[e] = fmaf(qq, s[e], acc[e]);
      }
      if (kept) __stcs(reinterpret_cast<float4*>(s_out + base + (size_t)r * dv + c), make_float4(s[0], s[1], s[2], s[3]));
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], 8);
    acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], 16);
  }
  if (lane < 8)
#pragma unroll
    for (int e = 0; e < 4; ++e) part[warp][lane * 4 + e] = acc[e];
  __syncthreads();
  const int col = slice * STEP_COLS + tid;
  if (tid < STEP_COLS && col < dv) o[((size_t)row * H + head) * dv + col] = from_f32<T>(scale * (part[0][tid] + part[1][tid] + part[2][tid] + part[3][tid]));
}

// ---------------------------------------------------------------- host
int check_lin(const rom_linattn_config* c) {
  if (!c || c->n_heads < 1 || c->n_qk_heads < 1 || c->d_k < 1 || c->d_v < 1 || c->n_heads % c->n_qk_heads != 0) return ROM_ERR_INVALID_ARG;
  if (c->dtype != ROM_F32 && c->dtype != ROM_BF16) return ROM_ERR_INVALID_ARG;
  if ((c->flags & ~(ROM_FLAG_SIMT_GEMM | ROM_FLAG_TEST_STALL)) != 0 || !isfinite(c->scale)) return ROM_ERR_INVALID_ARG;
  if (c->d_k % 8 != 0 || c->d_v % 8 != 0 || c->d_k > kLinMaxDim || c->d_v > kLinMaxDim || c->n_heads > 1024) return ROM_ERR_UNSUPPORTED;
  return ROM_OK;
}
bool on_tensor_cores(const rom_linattn_config& c) { return c.dtype == ROM_BF16 && !(c.flags & ROM_FLAG_SIMT_GEMM); }

// Runs: one head each, or, where that leaves SMs idle for longer than launches 1 and 2 take, equal runs of all heads' chunks on as many blocks as the GPU holds
// (on the tensor cores one to an SM).  Launch 1 takes about 0.6 of a chunk's time, launches 1 and 2 about six chunks of one block besides.  A function of the sizes only
// (148 SMs assumed).
struct LinSlots { int blocks, chunk, least, start; };
LinSlots slots_of(const rom_linattn_config& c) {
  if (on_tensor_cores(c)) return LinSlots{148, 128, 2, 128};
  return LinSlots{kLinMaxBlocks / ((c.d_v + SIMT_DV - 1) / SIMT_DV), SIMT_C, 1, 32};
}
int units_per_head(const LinSlots& s, int n_seq, int rows) { return (int)(((long long)rows + (long long)s.start * n_seq + s.chunk - 1) / s.chunk); }
int most_runs(const rom_linattn_config& c, int n_seq, int rows) {      // with cuts inside heads
  const LinSlots s = slots_of(c);
  const long long n = (long long)c.n_heads * units_per_head(s, n_seq, rows) / s.least;
  return (int)(n < 1 ? 1 : n < s.blocks ? n : s.blocks);
}
LinCut cut_rows(const rom_linattn_config& c, int n_seq, int rows, bool backward) {
  const LinSlots s = slots_of(c);
  LinCut cut{s.chunk, s.start, units_per_head(s, n_seq, rows), c.n_heads, 0, false};
  cut.units = (long long)c.n_heads * cut.per_head;
  // A run inside one head starts once, and heads that are cut at the same rows read memory side by side: a whole number of runs a head, where that leaves no more than a
  // fifth of the blocks out, for the backward (8 sequences, 16384 rows, 32 heads of 128: 565 us with 128 runs, 586 with 148) and for heads of 64, whose starts cost as much as
  // several chunks (23 prompts of 8186 rows, 32 heads: 100 and 109).  Elsewhere every block has a run (32 heads of 128, one prompt of 16384 rows: 221 with 128, 213 with 148; 12 of 8192: 130 and 123).
  int n = most_runs(c, n_seq, rows);
  const int aligned = n / c.n_heads * c.n_heads;
  if ((backward || (c.d_k <= 64 && c.d_v <= 64)) && aligned * 5 >= n * 4) n = aligned;
  const double whole = (double)((c.n_heads + s.blocks - 1) / s.blocks) * cut.per_head, even = 1.6 * (double)cut.units / n + 6.0;
  if (even < whole) { cut.blocks = n; cut.inside = true; }
  return cut;
}
struct LinWs { size_t status, powers, cut_a, cut_b, part_q, part_k, total; };
LinWs lin_ws(const rom_linattn_config& c, int n_seq, int rows, bool backward) {
  LinWs l{};
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes, 256); return at; };
  const size_t state = (size_t)most_runs(c, n_seq, rows) * c.d_k * c.d_v * sizeof(float);
  l.status = take(sizeof(int32_t) * kStatusInts);
  l.powers = take((size_t)c.n_heads * 2 * kLinPowers * sizeof(float));
  l.cut_a = take(state);
  l.cut_b = take(state);
  const size_t part = backward && c.n_qk_heads < c.n_heads ? (size_t)rows * c.n_heads * c.d_k * sizeof(float) : 0;
  l.part_q = take(part);
  l.part_k = take(part);
  l.total = off;
  return l;
}
int lin_ws_size(const rom_linattn_config* c, int32_t n_seq, int32_t rows, size_t* bytes, bool backward) {
  const int rc = check_lin(c);
  if (rc != ROM_OK) return rc;
  if (!bytes || n_seq < 0 || rows < 0) return ROM_ERR_INVALID_ARG;
  if (n_seq > kMaxRaggedSeqs || rows >= 1 << 30) return ROM_ERR_UNSUPPORTED;
  *bytes = lin_ws(*c, n_seq, rows, backward).total;
  return ROM_OK;
}

// Sequences of one row (continuous batching) in a launch of their own, where they may be many: fewer than 256 rows a sequence on average.  A walk takes 3 to 5 us for each of a
// run's in turn (256 sequences of 1200 rows, 32 heads of 128 bf16: 485 us a call, with this launch 320; 64 of 300, 8 heads of 64: 37.3 and 35); with few of them the launch costs its
// 2 us (37 of 531 rows, 8 heads of 64 fp32: 46 and 47.3).
bool singles_apart(const rom_linattn_config& c, const rom_ragged& seqs) {
  return seqs.n_seq > 1 && (long long)seqs.rows < 256LL * seqs.n_seq && (long long)seqs.n_seq * c.n_heads * ((c.d_v + STEP_COLS - 1) / STEP_COLS) <= INT32_MAX;
}
cudaError_t launch_singles(const rom_linattn_config& c, const LinPass& p, const rom_ragged& seqs, cudaStream_t st) {
  const int slices = (c.d_v + STEP_COLS - 1) / STEP_COLS;
  const long long blocks = (long long)seqs.n_seq * c.n_heads * slices;
  auto go = [&](auto zero) {
    using T = decltype(zero);
    count_launch();
    return launch_k(lin_step<T, true>, dim3((unsigned)blocks), STEP_THREADS, 0, st, (const T*)p.q, (const T*)p.k, (const T*)p.v, (long long)p.ldq, (long long)p.ldk, (long long)p.ldv,
                    p.log_decay, nullptr, 0, p.init, p.last, (T*)p.out, c.n_heads, c.n_heads / c.n_qk_heads, c.d_k, c.d_v, slices, c.scale, device_view(seqs));
  };
  return c.dtype == ROM_BF16 ? go(__nv_bfloat16()) : go(0.0f);
}

template <bool STATE>
cudaError_t launch_simt_by_type(const rom_linattn_config& c, const LinPass* p, int n, const rom_ragged& seqs, const LinCut& cut, cudaStream_t st) {
  return c.dtype == ROM_F32 ? launch_simt<float, STATE>(p, n, seqs, cut, st) : launch_simt<__nv_bfloat16, STATE>(p, n, seqs, cut, st);
}
cudaError_t launch_walks(const rom_linattn_config& c, const LinPass* p, int n, const rom_ragged& seqs, const LinCut& cut, cudaStream_t st) {
  if (on_tensor_cores(c) && seqs.rows > 0) return launch_lin_walks_tc(p, n, c.d_k, c.d_v, seqs, cut, (c.flags & ROM_FLAG_TEST_STALL) != 0, st);
  return launch_simt_by_type<false>(c, p, n, seqs, cut, st);
}
cudaError_t launch_powers(const LinPass& p, float* powers, cudaStream_t st) {
  count_launch();
  return launch_k(lin_powers, dim3((p.H * kLinPowers + 255) / 256), 256, 0, st, p.log_decay, p.H, powers, p.status);
}
// Launches 1 and 2: the states at the cuts.
cudaError_t launch_states(const rom_linattn_config& c, const LinPass* p, int n, const rom_ragged& seqs, const LinCut& cut, cudaStream_t st) {
  if (!cut.inside || seqs.rows == 0) return cudaSuccess;
  const cudaError_t e = on_tensor_cores(c) ? launch_lin_states_tc(p, n, c.d_k, c.d_v, seqs, cut, (c.flags & ROM_FLAG_TEST_STALL) != 0, st) : launch_simt_by_type<true>(c, p, n, seqs, cut, st);
  if (e != cudaSuccess) return e;
  LinJobs jobs{};
  for (int i = 0; i < n; ++i) jobs.p[i] = p[i];
  count_launch();
  return launch_k(lin_chain, dim3((c.d_k * c.d_v / 4 + CHAIN_THREADS - 1) / CHAIN_THREADS, c.n_heads, n), CHAIN_THREADS, 0, st, jobs, device_view(seqs), cut);
}
cudaError_t launch_sums(const rom_linattn_config& c, const float* part_q, void* dq, const float* part_k, void* dk, const rom_ragged& seqs, cudaStream_t st) {
  int sms = 0;
  const cudaError_t e = current_device_sm_count(&sms);
  if (e != cudaSuccess) return e;
  const size_t n = (size_t)seqs.rows * c.n_qk_heads * c.d_k / 4, blocks = (n + 255) / 256, most = (size_t)sms * 4;
  if (blocks == 0) return cudaSuccess;
  const dim3 grid((unsigned)(blocks < most ? blocks : most), 2);
  count_launch();
  if (c.dtype == ROM_F32) return launch_k(lin_sum_heads<float>, grid, 256, 0, st, part_q, (float*)dq, part_k, (float*)dk, device_view(seqs), c.n_heads, c.n_qk_heads, c.d_k);
  return launch_k(lin_sum_heads<__nv_bfloat16>, grid, 256, 0, st, part_q, (__nv_bfloat16*)dq, part_k, (__nv_bfloat16*)dk, device_view(seqs), c.n_heads, c.n_qk_heads, c.d_k);
}

bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + nb && y < x + na;
}

}  // namespace
}  // namespace rom

using namespace rom;

extern "C" {

int rom_linattn_ragged_workspace_size(const rom_linattn_config* cfg, int32_t n_seq, int32_t rows, size_t* bytes) { return lin_ws_size(cfg, n_seq, rows, bytes, false); }
int rom_linattn_backward_workspace_size(const rom_linattn_config* cfg, int32_t n_seq, int32_t rows, size_t* bytes) { return lin_ws_size(cfg, n_seq, rows, bytes, true); }

int rom_linattn_ragged(const rom_linattn_config* cfg, const rom_ragged* seqs, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                       const float* log_decay, const float* s_in, float* s_out, void* o, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_lin(cfg);
  if (rc != ROM_OK || (rc = check_ragged(seqs)) != ROM_OK) return rc;
  if (seqs->n_seq == 0) return ROM_OK;
  const rom_linattn_config& c = *cfg;
  const size_t esz = c.dtype == ROM_BF16 ? 2 : 4, pool = (size_t)seqs->n_slots * c.n_heads * c.d_k * c.d_v;
  if (!log_decay || !ws || (seqs->rows > 0 && (!q || !k || !v || !o)) || !aligned4(log_decay)) return ROM_ERR_INVALID_ARG;
  const void* ptrs[] = {q, k, v, o, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return ROM_ERR_INVALID_ARG;
  if (!pitch_ok(ldq, c.n_qk_heads * c.d_k, esz) || !pitch_ok(ldk, c.n_qk_heads * c.d_k, esz) || !pitch_ok(ldv, c.n_heads * c.d_v, esz)) return ROM_ERR_INVALID_ARG;
  if ((o && (o == q || o == k || o == v)) || !pools_ok(s_in, s_out, pool)) return ROM_ERR_INVALID_ARG;
  const LinWs lay = lin_ws(c, seqs->n_seq, seqs->rows, false);
  if (ws_bytes < lay.total) return ROM_ERR_WORKSPACE;
  if ((rc = check_device()) != ROM_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  LaunchCounter::count = 0;
  char* W = static_cast<char*>(ws);
  const LinCut cut = cut_rows(c, seqs->n_seq, seqs->rows, false);
  LinPass p{};
  p.q = q; p.k = k; p.v = v; p.ldq = ldq; p.ldk = ldk; p.ldv = ldv;
  p.qdiv = p.kdiv = c.n_heads / c.n_qk_heads; p.vdiv = 1;
  p.H = c.n_heads; p.dk = c.d_k; p.dv = c.d_v; p.log_decay = log_decay;
  p.p_scale = p.inter_scale = c.scale; p.k_scale = 1.0f;
  p.init = s_in; p.last = s_out;
  float* powers = reinterpret_cast<float*>(W + lay.powers);
  p.powers = powers;
  p.cut_state = reinterpret_cast<float*>(W + lay.cut_a);
  p.init_copy = cut.inside && s_in && s_in == s_out ? reinterpret_cast<float*>(W + lay.cut_b) : nullptr;
  p.out = o; p.ldo = (int64_t)c.n_heads * c.d_v;
  p.status = reinterpret_cast<int32_t*>(W + lay.status);
  if (launch_powers(p, powers, st) != cudaSuccess) return ROM_ERR_CUDA;
  p.skip_single = singles_apart(c, *seqs);
  if (launch_states(c, &p, 1, *seqs, cut, st) != cudaSuccess || launch_walks(c, &p, 1, *seqs, cut, st) != cudaSuccess) return ROM_ERR_CUDA;
  return !p.skip_single || launch_singles(c, p, *seqs, st) == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

int rom_linattn_step(const rom_linattn_config* cfg, int32_t B, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const float* log_decay,
                     const int32_t* slot, int32_t n_slots, const float* s_in, float* s_out, void* o, void* stream) {
  int rc = check_lin(cfg);
  if (rc != ROM_OK) return rc;
  const rom_linattn_config& c = *cfg;
  const size_t esz = c.dtype == ROM_BF16 ? 2 : 4;
  if (B < 0 || n_slots < 0 || (c.flags & ROM_FLAG_TEST_STALL)) return ROM_ERR_INVALID_ARG;
  if (B == 0) return ROM_OK;
  if (!q || !k || !v || !log_decay || !s_in || !s_out || !o) return ROM_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned4(log_decay) || !aligned4(slot)) return ROM_ERR_INVALID_ARG;
  if (!pitch_ok(ldq, c.n_qk_heads * c.d_k, esz) || !pitch_ok(ldk, c.n_qk_heads * c.d_k, esz) || !pitch_ok(ldv, c.n_heads * c.d_v, esz)) return ROM_ERR_INVALID_ARG;
  if (o == q || o == k || o == v || !pools_ok(s_in, s_out, (size_t)n_slots * c.n_heads * c.d_k * c.d_v)) return ROM_ERR_INVALID_ARG;
  const int slices = (c.d_v + STEP_COLS - 1) / STEP_COLS;
  const long long blocks = (long long)B * c.n_heads * slices;
  if (blocks > INT32_MAX) return ROM_ERR_UNSUPPORTED;
  if ((rc = check_device()) != ROM_OK) return rc;
  LaunchCounter::count = 0;
  count_launch();
  const dim3 grid((unsigned)blocks);
  const int share = c.n_heads / c.n_qk_heads;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto go = [&](auto zero) {
    using T = decltype(zero);
    return launch_k(lin_step<T, false>, grid, STEP_THREADS, 0, st, (const T*)q, (const T*)k, (const T*)v, (long long)ldq, (long long)ldk, (long long)ldv, log_decay, slot, n_slots,
                    s_in, s_out, (T*)o, c.n_heads, share, c.d_k, c.d_v, slices, c.scale, Ragged{});
  };
  return (c.dtype == ROM_BF16 ? go(__nv_bfloat16()) : go(0.0f)) == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

int rom_linattn_backward(const rom_linattn_config* cfg, const rom_ragged* seqs, const void* dout, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                         int64_t ldv, const float* log_decay, const float* s_in, const float* ds_out, void* dq, void* dk, void* dv, int64_t lddv, float* ds_in, void* ws,
                         size_t ws_bytes, void* stream) {
  int rc = check_lin(cfg);
  if (rc != ROM_OK || (rc = check_ragged(seqs)) != ROM_OK) return rc;
  if (seqs->n_seq == 0) return ROM_OK;
  const rom_linattn_config& c = *cfg;
  const size_t esz = c.dtype == ROM_BF16 ? 2 : 4, pool = (size_t)seqs->n_slots * c.n_heads * c.d_k * c.d_v * sizeof(float);
  if (!log_decay || !ws || (seqs->rows > 0 && (!dout || !q || !k || !v || !dq || !dk || !dv)) || !aligned4(log_decay)) return ROM_ERR_INVALID_ARG;
  const void* ptrs[] = {dout, q, k, v, s_in, ds_out, dq, dk, dv, ds_in, ws};
  for (const void* p : ptrs)
    if (!aligned16(p)) return ROM_ERR_INVALID_ARG;
  if (!pitch_ok(ldq, c.n_qk_heads * c.d_k, esz) || !pitch_ok(ldk, c.n_qk_heads * c.d_k, esz) || !pitch_ok(ldv, c.n_heads * c.d_v, esz) || !pitch_ok(lddv, c.n_heads * c.d_v, esz))
    return ROM_ERR_INVALID_ARG;
  const void *ins[] = {dout, q, k, v}, *outs[] = {dq, dk, dv};
  for (int i = 0; i < 3; ++i) {
    for (const void* a : ins)
      if (a && a == outs[i]) return ROM_ERR_INVALID_ARG;
    if (outs[i] && outs[i] == outs[(i + 1) % 3]) return ROM_ERR_INVALID_ARG;
  }
  if (overlaps(ds_in, pool, ds_out, pool) || overlaps(ds_in, pool, s_in, pool)) return ROM_ERR_INVALID_ARG;
  const LinWs lay = lin_ws(c, seqs->n_seq, seqs->rows, true);
  if (ws_bytes < lay.total) return ROM_ERR_WORKSPACE;
  if ((rc = check_device()) != ROM_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  LaunchCounter::count = 0;
  char* W = static_cast<char*>(ws);
  const LinCut cut = cut_rows(c, seqs->n_seq, seqs->rows, true);
  const int share = c.n_heads / c.n_qk_heads;
  float *part_q = share > 1 ? reinterpret_cast<float*>(W + lay.part_q) : nullptr, *part_k = share > 1 ? reinterpret_cast<float*>(W + lay.part_k) : nullptr;
  float* powers = reinterpret_cast<float*>(W + lay.powers);
  const int64_t ld_do = (int64_t)c.n_heads * c.d_v;
  LinPass base{};
  base.H = c.n_heads; base.log_decay = log_decay; base.p_scale = c.scale; base.powers = powers;
  base.status = reinterpret_cast<int32_t*>(W + lay.status);
  // the states S of the forward at the cuts, and R behind them (with which dv is walked)
  LinPass s = base, dv_walk = base;
  s.k = k; s.v = v; s.ldk = ldk; s.ldv = ldv;
  s.qdiv = s.kdiv = share; s.vdiv = 1; s.dk = c.d_k; s.dv = c.d_v;
  s.k_scale = 1.0f; s.init = s_in; s.cut_state = reinterpret_cast<float*>(W + lay.cut_a);
  dv_walk.q = k; dv_walk.k = q; dv_walk.v = dout; dv_walk.ldq = ldk; dv_walk.ldk = ldq; dv_walk.ldv = ld_do;
  dv_walk.qdiv = dv_walk.kdiv = share; dv_walk.vdiv = 1; dv_walk.dk = c.d_k; dv_walk.dv = c.d_v;
  dv_walk.inter_scale = 1.0f; dv_walk.k_scale = c.scale; dv_walk.reverse = true; dv_walk.init = ds_out; dv_walk.init_all = true; dv_walk.early = true; dv_walk.last = ds_in;
  dv_walk.none_resumes = !s_in;
  dv_walk.cut_state = reinterpret_cast<float*>(W + lay.cut_b);
  dv_walk.out = dv; dv_walk.ldo = lddv;
  // dq on S, dk on R, both transposed
  LinPass dq_walk = base, dk_walk = dv_walk;
  dq_walk.q = dout; dq_walk.k = v; dq_walk.v = k; dq_walk.ldq = ld_do; dq_walk.ldk = ldv; dq_walk.ldv = ldk;
  dk_walk.q = v; dk_walk.k = dout; dk_walk.v = q; dk_walk.ldq = ldv; dk_walk.ldk = ld_do; dk_walk.ldv = ldq;
  dq_walk.inter_scale = c.scale; dq_walk.k_scale = 1.0f; dq_walk.init = s_in; dq_walk.cut_state = s.cut_state;
  dk_walk.last = nullptr;
  for (LinPass* w : {&dq_walk, &dk_walk}) {
    w->qdiv = w->kdiv = 1; w->vdiv = share; w->dk = c.d_v; w->dv = c.d_k; w->transposed = true;
    w->ldo = (int64_t)c.n_heads * c.d_k; w->out_f32 = share > 1;
  }
  dq_walk.out = part_q ? part_q : dq;
  dk_walk.out = part_k ? part_k : dk;
  const LinPass states[2] = {s, dv_walk}, walks[3] = {dq_walk, dv_walk, dk_walk};
  if (launch_powers(base, powers, st) != cudaSuccess || launch_states(c, states, 2, *seqs, cut, st) != cudaSuccess || launch_walks(c, walks, 3, *seqs, cut, st) != cudaSuccess)
    return ROM_ERR_CUDA;
  return !part_q || launch_sums(c, part_q, dq, part_k, dk, *seqs, st) == cudaSuccess ? ROM_OK : ROM_ERR_CUDA;
}

}  // extern "C"
