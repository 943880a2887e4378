// Backward packed attention for gfx950 (see packed_fwd.hip for the layout of the sequences).
//
// dQ (query-stationary, first): one workgroup of four waves owns 128 query rows of one
//   (sequence, head), each wave 32, with Q^T and dO^T of its queries in registers. It forms
//   D_i = <dO_i, O_i> from its own rows and walks over the key tiles like the forward, computing
//   S^T, dP^T and dS^T = P^T o (dP^T - D), and dQ^T += K^T dS^T. It leaves -LSE / c and -D for the
//   other pass. Few queries before many keys: several workgroups share a block's key tiles.
// dK/dV (key-stationary): one workgroup owns 128 keys of one (sequence, key head), each wave 32,
//   K and V of its keys in registers, and walks over the query tiles of 32 of every query head
//   of the group, so that dK and dV of the shared head are summed in registers; where that leaves
//   too few workgroups, each takes a run of those tiles and fp32 partials are summed afterwards.
//   With a bias it also sums dS over every distance, in LDS.
// Both are bound by the matrix rate for long rows: 12,000 tokens causal, 16 heads, 2 key heads, D = 128: dQ 773 us,
// 1,145 TFLOP/s of its 6 D a pair, dK/dV 1,115 us, 1,058 of 8 D (the first, plain walks, operands read where they
// are used and the statistics from memory: 6.5 ms for forward and backward, now 2.3 to 2.5 by the clock). Short ones wait for a few
// tiles one after the other: captions of 8 to 256 tokens, 16 heads, D = 64, bias, 23 and 30 us.
// No atomics anywhere: results are bitwise reproducible.
#include "packed.hpp"

namespace vcja {
namespace {

constexpr int kBN = kTileTok;      // keys per dQ tile
constexpr int kBQ = 32;            // queries per dK/dV tile

__device__ __forceinline__ bf16x8 operand(const f32x16& x, int half) {
  bf16x8 y;
#pragma unroll
  for (int t = 0; t < 8; ++t) y[t] = (__bf16)x[8 * half + t];
  return y;
}

// Sums of one 32 queries x 32 keys block of dS over its diagonals (distance = key - query). Register r of
// a lane of half hi holds query row n = 8 (r / 4) + 4 hi + r % 4 of its key: rotating it by n brings
// distance t (where n + t < 32) or t - 32 to lane t, the same for every register, so that a lane adds
// its own values up; the two halves of the wave are joined at the end, the lower one keeping
// distances 0 .. 31, the upper one -32 .. -1 (as the sum of all less those: exact to the fp32 sums'
// own rounding). Additions in LDS (ds_add_f32) took three times as long as the whole walk: 32 -> 104 us
// at captions of 8 to 256 tokens.
__device__ __forceinline__ float distance_sums(const f32x16& ds, int lane) {
  const int t = lane & 31, hi = lane >> 5, y = t + 4 * hi;
  float pos = 0.0f, all = 0.0f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    if (r % 4 == 0) sched_fence();  // a few at a time: registers are the limit here
    const int n = 8 * (r >> 2) + (r & 3);
    const int from = ((4 * y + 4 * n) & 124) | (4 * (lane & 32));
    const float x = __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(from, __builtin_bit_cast(int, (float)ds[r])));
    all += x;
    pos += y < 32 - n ? x : 0.0f;
  }
  const float neg = halves_sum(all - pos);
  pos = halves_sum(pos);
  return hi ? neg : pos;
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// Rows outside every slot of a tensor's [rows, H, D]: zero (the last workgroups of a grid).
template <int D>
__device__ __forceinline__ void clear_rows(__bf16* x, __bf16* y, const int32_t* cu, int S, int total, int H, int wg, int wgs, int tid,
                                           int threads) {
  const int head = min(max(cu[0], 0), total), end = min(max(cu[S], head), total);
  const int64_t per = (int64_t)H * (D / 8);
  for (int64_t i = (int64_t)wg * threads + tid; i < (head + total - end) * per; i += (int64_t)wgs * threads) {
    const int r = (int)(i / per);
    const size_t at = (size_t)(r < head ? r : r - head + end) * H * D + i % per * 8;
    *(bf16x8*)(x + at) = zero_bf16x8();
    if (y) *(bf16x8*)(y + at) = zero_bf16x8();
  }
}

template <int D, int RMAX>
__global__ __launch_bounds__(64 * kPackedWaves, 2) void packed_dq_kernel(PackedArgs a) {
  using Rows = SwzRows<D>;
  using Reads = SwzReads<D>;
  constexpr int NW = kPackedWaves, BM = kPackedRows;
  constexpr int RT = Rows::bytes(kBN);
  constexpr int STAGE = 2 * RT;                  // K | V rows of a tile
  constexpr int CPW = kBN / Rows::RPC / NW;      // copies of each per wave
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE];
  __shared__ BiasTable<RMAX> table;
  constexpr bool BIAS = RMAX > 0;
  const float* const tb = table.tb;

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int blocks = a.blocks * a.H, items = blocks * a.dq_chunks;
  if ((int)blockIdx.x >= items) {
    clear_rows<D>(a.dq, nullptr, a.cu_q, a.S, a.Tq, a.H, blockIdx.x - items, gridDim.x - items, tid, 64 * NW);
    return;
  }
  const int chunk = (int)blockIdx.x / blocks;  // of the block's key tiles
  const PackedItem it = packed_item(a, blockIdx.x % blocks, a.cu_q, a.Tq, a.Hkv, a.G, true);
  if (it.s < 0) return;
  const SeqRows sr = seq_rows(a, it.s);
  const int b0 = it.blk * BM;
  if (b0 >= sr.sq) return;
  const int kv = it.h / a.G;
  const int qi = b0 + w * 32 + l32;
  auto limit = [&](int i) { return a.causal ? max(0, min(sr.nk, i + sr.off + 1)) : sr.nk; };
  const int qe = min(b0 + BM, sr.nq);
  const int blk_keys = qe > b0 ? limit(qe - 1) : 0;
  const int wave_keys = b0 + w * 32 < qe ? limit(min(b0 + w * 32 + 32, sr.nq) - 1) : 0;
  const int wave_all = limit(b0 + w * 32);
  const int klim = qi < sr.nq ? limit(qi) : 0;
  const int ntile = (blk_keys + kBN - 1) / kBN, kt0 = chunk * a.span, kt1 = min(ntile, kt0 + a.span);
  if (chunk > 0 && kt0 >= kt1) return;

  const SwzCopy<D, true> kc(a.k_tok, lane), vc(a.v_tok, lane);
  const __bf16* kbase = a.k + (size_t)sr.k0 * a.k_tok + kv * D;
  const __bf16* vbase = a.v + (size_t)sr.k0 * a.v_tok + kv * D;
  auto issue_j = [&](int j, bool is_k, int kt, int st) {
    const int idx = w + j * NW, first = swz_copy_row<D, true>(kt * kBN, sr.nk, idx);
    VC_LDS char* dst = (VC_LDS char*)smem + st * STAGE + (is_k ? 0 : RT) + idx * Rows::GS;
    if (is_k)
      copy16_to_lds_opaque(kbase + (size_t)first * a.k_tok, kc.offset(first, sr.nk, a.k_tok), dst);
    else
      copy16_to_lds_opaque(vbase + (size_t)first * a.v_tok, vc.offset(first, sr.nk, a.v_tok), dst);
  };
  auto issue_tile = [&](int kt, int st) {
#pragma unroll
    for (int j = 0; j < CPW; ++j) {
      issue_j(j, true, kt, st);
      issue_j(j, false, kt, st);
    }
  };

  if (kt0 < kt1) issue_tile(kt0, 0);  // in flight with the loads below
  bf16x8 qf[D / 16], dof[D / 16];
  float nls, dd;
  {
    const size_t row = query_row(a, sr, qi);
    const __bf16* qp = a.q + row * a.q_tok + it.h * D + 8 * hi;
    const size_t at = (row * a.H + it.h) * D + 8 * hi;
    float sum = 0.0f;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      qf[ks] = *(const bf16x8*)(qp + 16 * ks);
      dof[ks] = *(const bf16x8*)(a.dout + at + 16 * ks);
      const bf16x8 o = *(const bf16x8*)(a.o_in + at + 16 * ks);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf((float)o[e], (float)dof[ks][e], sum);
    }
    dd = klim == 0 ? 0.0f : -halves_sum(sum);
    const float x = a.lse[(size_t)it.h * a.Tq + row];
    nls = klim == 0 || x == -INFINITY ? -INFINITY : -x / a.scale;
  }
  table.load(a, it.h, tid, 64 * NW);

  f32x16 acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = zero_f32x16();
  const int pos0 = b0 + w * 32 + sr.off;  // position of the wave's first query
  const float nlse2 = nls * a.scale_log2;
  float rowsum = 0.0f;

  wait_all_memory();  // the loads above too: no later wait stands among copies
  // Rows of at most one tile of keys: D = sum_j P_ij dP_ij itself, by a walk over that tile beforehand. Taken
  // of the rounded O it is off by about 2^-9 |dO| |O|, which moves all dS of the row by its P; with a few keys
  // of unequal weight dS is much smaller than D, and dQ of texts of a few tokens was off by 0.5% (2^-8 by its own rounding). Over the sum of P, which is 1 but for the
  // rounding of LSE: with a bias of 10,000s that reaches 2^-8 and would move D by as much.
  // Over more keys dQ keeps the rounding of O (the other pass and the bias gradient do not: the row's sum of dS, below):
  // off by 0.24% of its 2-norm beside 0.23% without it at 300 keys and scale 1/8, by 0.7% in sharp rows (scale 2).
  // To take it out of dQ too, sum_j P_ij k_j would have to be summed beside dQ: a third more products.
  if (kt0 < kt1 && b0 < sr.nq && limit(min(b0 + 32, sr.nq) - 1) <= kBN) {  // the first wave's last query
    __syncthreads();
    if (wave_keys > 0 && wave_keys <= kBN) {
      const VC_LDS char* rp = (const VC_LDS char*)smem + Reads::row_base(perm_row(l32), hi);
      float sum = 0.0f, all = 0.0f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        f32x16 s = zero_f32x16(), dp = zero_f32x16();
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          s = mfma32(*(const VC_LDS bf16x8*)(Reads::row_at(rp, ks) + kb * Rows::bytes(32)), qf[ks], s);
          dp = mfma32(*(const VC_LDS bf16x8*)(Reads::row_at(rp, ks) + RT + kb * Rows::bytes(32)), dof[ks], dp);
        }
        const float* b = tb + kBiasPad + a.R;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = 32 * kb + acc_row(r, hi);
          float x = s[r];
          if (BIAS) x += b[min(max(key - pos0 - l32, -a.R), a.R)];
          const float p = key < klim ? fast_exp2(fmaf(x, a.scale_log2, nlse2)) : 0.0f;
          all += p;
          sum = fmaf(p, dp[r], sum);
        }
      }
      all = halves_sum(all);
      sum = halves_sum(sum);
      dd = all > 0.0f ? -sum / all : 0.0f;
    }
  }
  for (int kt = kt0; kt < kt1; ++kt) {
    const int st = (kt - kt0) & 1;
    wait_all_memory();
    __syncthreads();
    const int k0 = kt * kBN;
    const int kn = min(kt + 1, kt1 - 1);  // past the last tile: copied again, never read
    if (k0 >= wave_keys) {
      issue_tile(kn, st ^ 1);
      continue;
    }
    // The two key blocks' products in one stretch of matrix-core ops, every LDS operand read
    // PF ops ahead, the vector arithmetic of a phase placed between the ops of the next ones:
    // S0 | dP0, P0 | S1, dS0 | dP1, P1 | dQ += K0^T dS0, dS1 | dQ += K1^T dS1.
    constexpr int KSN = D / 16;
    constexpr int NB = D / 32;
    constexpr int PF = 3;
    constexpr int EP = 16 / KSN;
    const VC_LDS char* tile = (const VC_LDS char*)smem + st * STAGE;
    const VC_LDS char* rp = tile + Reads::row_base(perm_row(l32), hi);
    const VC_LDS char* tp = tile + Reads::tr_base(lane);
    bf16x8 f[4 * KSN], g[4 * NB];
    auto rd = [&](int i) {  // S0, dP0, S1, dP1, then the dQ operands
      if (i < 4 * KSN) {
        const int kb = i / (2 * KSN), v = i / KSN % 2;
        f[i] = *(const VC_LDS bf16x8*)(Reads::row_at(rp, i % KSN) + v * RT + kb * Rows::bytes(32));
      } else if (i - 4 * KSN < 4 * NB) {
        g[i - 4 * KSN] = Reads::tr_operand(tp, (i - 4 * KSN) / NB, (i - 4 * KSN) % NB);
      }
    };
    f32x16 s[2], dp[2];
    bf16x8 sb[4];
    float shift[2] = {nlse2, nlse2};
    auto form_p = [&](int kb, int r) { s[kb][r] = fast_exp2(fmaf(s[kb][r], a.scale_log2, shift[kb])); };
    auto form_ds = [&](int kb, int r) {
      dp[kb][r] *= s[kb][r];
      rowsum += dp[kb][r];
    };
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      s[kb] = zero_f32x16();
      if (BIAS) {
        const int side = bias_side(k0 + 32 * kb, k0 + 32 * kb + 31, pos0, pos0 + 31, a.R);
        if (side == 0) {
          const float* t = tb + kBiasPad + a.R + (k0 + 32 * kb + 4 * hi - pos0 - l32);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kb][r] = t[8 * (r >> 2) + (r & 3)];
        } else {
          shift[kb] = fmaf(tb[kBiasPad + (side > 0 ? 2 * a.R : 0)], a.scale_log2, nlse2);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < PF; ++i) rd(i);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int i = 0; i < KSN; ++i) {
        sched_fence();
        rd(2 * KSN * kb + i + PF);
        s[kb] = mfma32(f[2 * KSN * kb + i], qf[i], s[kb]);
        if (kb == 0) {  // the next tile's copies, spread over the ops
#pragma unroll
          for (int j = 0; j < 2 * CPW; ++j)
            if (j * KSN / (2 * CPW) == i) issue_j(j / 2, j % 2 == 0, kn, st ^ 1);
        }
        if (kb == 1 && i == 0)
#pragma unroll
          for (int e = 0; e < EP; ++e) form_p(0, (KSN - 1) * EP + e);
        if (kb == 1 && i > 0)
#pragma unroll
          for (int e = 0; e < EP; ++e) form_ds(0, (i - 1) * EP + e);
      }
      if (kb == 1) {
#pragma unroll
        for (int e = 0; e < EP; ++e) form_ds(0, (KSN - 1) * EP + e);
        sb[0] = operand(dp[0], 0);
        sb[1] = operand(dp[0], 1);
      }
      if (k0 + 32 * kb + 32 > wave_all) {
        sched_fence();
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kb][r] = k0 + 32 * kb + acc_row(r, hi) < klim ? s[kb][r] : -INFINITY;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[kb][r] = dd;  // dP - D
#pragma unroll
      for (int i = 0; i < KSN; ++i) {
        sched_fence();
        rd(2 * KSN * kb + KSN + i + PF);
        dp[kb] = mfma32(f[2 * KSN * kb + KSN + i], dof[i], dp[kb]);
        if (i > 0)
#pragma unroll
          for (int e = 0; e < EP; ++e) form_p(kb, (i - 1) * EP + e);
      }
    }
    constexpr int ED = 16 / (2 * NB);
#pragma unroll
    for (int i = 0; i < 4 * NB; ++i) {
      sched_fence();
      rd(4 * KSN + i + PF);
      acc[i % NB] = mfma32(g[i], sb[i / NB], acc[i % NB]);
      if (i == 0)
#pragma unroll
        for (int e = 0; e < EP; ++e) form_p(1, (KSN - 1) * EP + e);
      else if (i < 2 * NB)
#pragma unroll
        for (int e = 0; e < ED; ++e) form_ds(1, (i - 1) * ED + e);
      if (i == 2 * NB - 1) {
#pragma unroll
        for (int e = 0; e < ED; ++e) form_ds(1, (2 * NB - 1) * ED + e);
        sb[2] = operand(dp[1], 0);
        sb[3] = operand(dp[1], 1);
      }
    }
    sched_fence();
  }
  wait_all_memory();  // no copy outlives the workgroup

  // What dS of a row sums up to beside 0 is the error of its D, taken of the rounded O: the other
  // pass gets D without it. (Rows past the sequence's own: inert.)
  const bool split = ntile > a.span;  // several workgroups: the sum kernel finishes dQ and D
  rowsum = halves_sum(rowsum);
  if (chunk == 0 && hi == 0 && qi < ((sr.nq + 63) & ~63)) {
    const size_t p = (size_t)it.h * a.npad + packed_row(sr.q0, it.s) + qi;
    a.nls[p] = nls;
    a.dd[p] = klim == 0 ? 0.0f : split ? dd : dd - rowsum;
  }
  if (split && qi < sr.sq) {
    const size_t rows = (size_t)a.Tq * a.H, at = chunk * rows + (size_t)(sr.q0 + qi) * a.H + it.h;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *(f32x4*)(a.part + at * D + db * 32 + 8 * j + 4 * hi) =
            f32x4{acc[db][4 * j + 0], acc[db][4 * j + 1], acc[db][4 * j + 2], acc[db][4 * j + 3]};
    if (hi == 0) a.part[a.dq_chunks * rows * D + at] = rowsum;
    return;
  }
  if (qi < sr.sq) {  // rows that see no key, and rows of the slot past the sequence's own: 0
    __bf16* qp = a.dq + ((size_t)(sr.q0 + qi) * a.H + it.h) * D;
    const float c = klim > 0 ? a.scale : 0.0f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x4 t = {(__bf16)(acc[db][4 * j + 0] * c), (__bf16)(acc[db][4 * j + 1] * c), (__bf16)(acc[db][4 * j + 2] * c),
                    (__bf16)(acc[db][4 * j + 3] * c)};
        *(bf16x4*)(qp + db * 32 + 8 * j + 4 * hi) = t;
      }
  }
}

// dQ, and -D without the sums of dS, of the rows whose keys several workgroups share, in order. One wave per
// (query, head).
template <int D>
__global__ __launch_bounds__(256) void packed_dq_sum_kernel(PackedArgs a) {
  constexpr int E = D / 64;
  typedef float fe __attribute__((ext_vector_type(E)));
  const int lane = threadIdx.x & 63;
  const int x = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  int h, i, s;
  if (a.compact) {  // (row of a block, head, block)
    const int c = x / (kPackedRows * a.H);
    if (c >= a.blocks) return;
    s = find_sequence(a.cu_q, a.S, a.Tq, c);
    if (s < 0) return;
    i = __builtin_amdgcn_readfirstlane((c - min(max(a.cu_q[s], 0), a.Tq) / kPackedRows - s) * kPackedRows + x % kPackedRows);
    h = x / kPackedRows % a.H;
  } else {
    if (x >= a.S * a.max_q * a.H) return;
    h = x % a.H;
    i = x / a.H % a.max_q;
    s = x / a.H / a.max_q;
  }
  const SeqRows sr = seq_rows(a, s);
  if (i >= sr.sq) return;
  // The tiles of the row's block of rows, as the dQ kernel counts them.
  auto limit = [&](int q) { return a.causal ? max(0, min(sr.nk, q + sr.off + 1)) : sr.nk; };
  const int b0 = i / kPackedRows * kPackedRows, qe = min(b0 + kPackedRows, sr.nq);
  const int n = ((qe > b0 ? limit(qe - 1) : 0) + kBN - 1) / kBN;
  if (n <= a.span) return;  // written by its only workgroup
  const int chunks = (n + a.span - 1) / a.span;
  const size_t rows = (size_t)a.Tq * a.H, at = (size_t)(sr.q0 + i) * a.H + h;
  const bool sees = i < sr.nq && limit(i) > 0;
  fe acc;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
  float sum = 0.0f;
#pragma unroll 4
  for (int c = 0; c < chunks; ++c) {
    acc += *(const fe*)(a.part + (c * rows + at) * D + E * lane);
    sum += a.part[a.dq_chunks * rows * D + c * rows + at];
  }
#pragma unroll
  for (int e = 0; e < E; ++e) a.dq[at * D + E * lane + e] = (__bf16)(sees ? acc[e] * a.scale : 0.0f);
  if (lane == 0 && sees) a.dd[(size_t)h * a.npad + packed_row(sr.q0, s) + i] -= sum;
}

// A key block's steps: query tiles [t0, t0 + nt) of every query head of its group, heads in
// order; a call of several chunks gives each workgroup a run of them; with a bias
// the chunks are a multiple of the heads, each of one head.
struct KeySteps {
  int t0, nt, u0, u1;
};
__device__ __forceinline__ KeySteps key_steps(const PackedArgs& a, const SeqRows& sr, int b0, int chunk) {
  KeySteps k;
  auto one = [](int x) { return __builtin_amdgcn_readfirstlane(x); };  // divided: back to a scalar register
  // from the first query at or past the block's first key
  k.t0 = (a.causal ? max(0, b0 - sr.off) : 0) / kBQ;
  k.nt = b0 < sr.nk ? max(0, (sr.nq + kBQ - 1) / kBQ - k.t0) : 0;
  k.u0 = one((int)((int64_t)a.G * k.nt * chunk / a.chunks));
  k.u1 = one((int)((int64_t)a.G * k.nt * (chunk + 1) / a.chunks));
  return k;
}

template <int D, int RMAX>
__global__ __launch_bounds__(64 * kPackedWaves, 2) void packed_dkdv_kernel(PackedArgs a) {
  using Rows = SwzRows<D>;
  using Reads = SwzReads<D>;
  constexpr int NW = kPackedWaves, BM = kPackedRows;
  constexpr int RT = Rows::bytes(kBQ);
  constexpr int STAGE = 2 * RT;               // Q rows | dO rows of a tile
  constexpr int COPIES = kBQ / Rows::RPC;     // wave copies of each
  constexpr int CPW = 2 * COPIES / NW;        // copies per wave and tile, Q's first
  constexpr int STAT = 2 * STAGE;             // -LSE/c | -D of a run of SQ queries, two buffers
  constexpr int SQ = 256, SPT = SQ / kBQ;
  // Sums of dS per distance: each wave's inside (-R, R), each lane's up to -R and from R on.
  constexpr int HIST = 2 * RMAX + 1;
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE + 2 * 2 * SQ * 4];
  __shared__ BiasTable<RMAX> table;
  constexpr bool BIAS = RMAX > 0;
  const float* const tb = table.tb;
  __shared__ float hist[RMAX ? NW * HIST : 1], ends[RMAX ? NW * 128 : 1];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int items = a.blocks * a.Hkv * a.chunks;
  if ((int)blockIdx.x >= items) {
    clear_rows<D>(a.dk, a.dv, a.cu_k, a.S, a.Tk, a.Hkv, blockIdx.x - items, gridDim.x - items, tid, 64 * NW);
    return;
  }
  // Key heads (and sequences) run fastest, the chunks of a block next to each other behind them; the first key
  // blocks, the longest under the causal rule, come first.
  const int per = a.compact ? a.Hkv : a.Hkv * a.S, chunk = blockIdx.x / per % a.chunks;
  const PackedItem it = packed_item(a, blockIdx.x / per / a.chunks * per + blockIdx.x % per, a.cu_k, a.Tk, a.Hkv, 1, false);
  if (it.s < 0) return;
  const int kv = it.h, seq = it.s, blk = it.blk;
  const int b0 = blk * BM;
  const SeqRows sr = seq_rows(a, seq);
  if (BIAS && b0 + BM >= sr.sk && (b0 < sr.sk || blk == 0)) {
    // the sequence's last block (or an empty slot): no sums in the rows up to the next sequence's
    const int64_t r0 = dist_row(sr.k0, seq, b0 < sr.sk ? blk + 1 : 0, BM);
    const int64_t r1 = dist_row(min(max(__builtin_amdgcn_readfirstlane(a.cu_k[seq + 1]), 0), a.Tk), seq + 1, 0, BM);
    for (int64_t r = r0; r < r1; ++r)
      for (int i = tid; i < 2 * a.R + 1; i += 64 * NW) a.dist_part[((r * a.Hkv + kv) * a.chunks + chunk) * (2 * a.R + 1) + i] = 0.0f;
  }
  if (b0 >= sr.sk) return;
  // Registers are the limit of the walk: what follows from the lane index is formed where it is
  // used, from an index that the compiler must treat as new, and not held across the tiles.
  auto fresh_lane = [&]() {
    int x = lane;
    asm volatile("" : "+v"(x));
    return x;
  };
  auto lane_key = [&]() { return b0 + w * 32 + (fresh_lane() & 31); };  // this lane's key
  const KeySteps ks = key_steps(a, sr, b0, chunk);
  const int wave_q = a.causal ? b0 + w * 32 - sr.off : 0;  // first query that sees a key of the wave

  const unsigned o_tok = a.H * D;
  const __bf16* qbase = a.q + (size_t)sr.q0 * a.q_tok + kv * a.G * D;
  const __bf16* dbase = a.dout + (size_t)sr.q0 * o_tok + kv * a.G * D;
  const int srow = packed_row(sr.q0, seq);
  // Copy j of this wave for the tile of query row q0, head g of the group, into stage st. Rows past nq repeat the last;
  // their -LSE of -inf makes their probabilities zero.
  auto copy_is_q = [&](int j) { return COPIES % NW == 0 ? j < COPIES / NW : w < COPIES; };
  const __bf16* cbase[CPW];
  unsigned ctok[CPW];
#pragma unroll
  for (int j = 0; j < CPW; ++j) {
    cbase[j] = uniform_ptr(copy_is_q(j) ? qbase : dbase);
    ctok[j] = __builtin_amdgcn_readfirstlane(copy_is_q(j) ? a.q_tok : o_tok);
  }
  auto issue_j = [&](int j, int g, int q0, int st) {
    const int idx = (w + j * NW) % COPIES, first = swz_copy_row<D, true>(q0, sr.nq, idx);
    copy16_to_lds_opaque(cbase[j] + (size_t)first * ctok[j] + g * D, swz_copy_off<D, true>(first, ctok[j], sr.nq, fresh_lane()),
                         (VC_LDS char*)smem + st * STAGE + (copy_is_q(j) ? 0 : RT) + idx * Rows::GS);
  };
  // The row statistics of the run of SQ queries that holds tile t of head g, by the last two waves.
  const float* sbase = uniform_ptr(w == NW - 2 ? a.nls : a.dd);
  auto issue_stats = [&](int g, int t, int buf) {
    if (w < NW - 2) return;
    const bool is_l = w == NW - 2;
    const size_t p = (size_t)(kv * a.G + g) * a.npad + srow + (ks.t0 + t / SPT * SPT) * kBQ;
    copy16_to_lds_opaque(sbase + p, 16u * (unsigned)fresh_lane(),
                         (VC_LDS char*)smem + STAT + buf * 2 * SQ * 4 + (is_l ? 0 : SQ * 4));
  };

  int g = BIAS ? __builtin_amdgcn_readfirstlane(chunk / (a.chunks / a.G)) : __builtin_amdgcn_readfirstlane(ks.nt ? ks.u0 / ks.nt : 0), t = ks.u0 - g * ks.nt, buf = 0;  // scalar, as u0
  if (ks.u0 < ks.u1) {
    issue_stats(g, t, 0);
#pragma unroll
    for (int j = 0; j < CPW; ++j) issue_j(j, g, (ks.t0 + t) * kBQ, 0);
  }
  bf16x8 kf[D / 16], vf[D / 16];
  {
    const size_t row = min(sr.k0 + min(lane_key(), max(sr.nk - 1, 0)), a.Tk - 1);
    const int hi = lane >> 5;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      kf[i] = *(const bf16x8*)(a.k + row * a.k_tok + kv * D + 16 * i + 8 * hi);
      vf[i] = *(const bf16x8*)(a.v + row * a.v_tok + kv * D + 16 * i + 8 * hi);
    }
  }
  if (BIAS) {
    for (int i = tid; i < NW * HIST; i += 64 * NW) hist[i] = 0.0f;
    for (int i = tid; i < NW * 128; i += 64 * NW) ends[i] = 0.0f;
    table.load(a, kv * a.G + g, tid, 64 * NW);  // its barriers cover the sums too, also where no step follows
  }
  wait_all_memory();  // the loads above too: no later wait stands among copies

  f32x16 dk_acc[D / 32], dv_acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    dk_acc[i] = zero_f32x16();
    dv_acc[i] = zero_f32x16();
  }
  const int pos_k = b0 + w * 32;  // position of the wave's first key
  for (int u = ks.u0; u < ks.u1; ++u) {
    const int st = (u - ks.u0) & 1, q0 = (ks.t0 + t) * kBQ;
    wait_all_memory();
    if (q0 + kBQ > sr.nq) {
      // dO rows past nq that this wave copied: zero, as a probability of 0 does not silence an
      // infinite value of the last row, which they repeat.
#pragma unroll
      for (int j = 0; j < CPW; ++j) {
        const int idx = (w + j * NW) % COPIES, cl = fresh_lane();
        f32x4 z = {0.0f, 0.0f, 0.0f, 0.0f};
        asm volatile("" : "+v"(z));  // formed here: no registers hold it across the walk
        if (!copy_is_q(j) && q0 + perm_row(Rows::RPC * idx + cl / Rows::CPR) >= sr.nq)
          *(VC_LDS f32x4*)((VC_LDS char*)smem + st * STAGE + RT + idx * Rows::GS + 16 * cl) = z;
      }
    }
    __syncthreads();
    // The next step: the next tile, or the first one of the next head.
    const bool last = u + 1 == ks.u1, turn = t + 1 == ks.nt;
    const int gn = last ? g : turn ? g + 1 : g, tn = last ? t : turn ? 0 : t + 1;  // past the last: copied again, never read
    const int qn = (ks.t0 + tn) * kBQ;
    const int bufn = !last && tn % SPT == 0 ? buf ^ 1 : buf;
    if (bufn != buf) issue_stats(gn, tn, bufn);
    if (q0 + kBQ <= wave_q) {  // every query of the tile stands before the wave's keys
#pragma unroll
      for (int j = 0; j < CPW; ++j) issue_j(j, gn, qn, st ^ 1);
    } else {
      // The tile's products in one stretch of matrix-core ops, every LDS operand read PF ops
      // ahead, each phase's vector arithmetic between the ops of the next one: S = Q K^T;
      // dP = -D + dO V^T while P is formed; dV^T += dO^T P while dS is formed; dK^T += Q^T dS.
      constexpr int KSN = D / 16;
      constexpr int NB = D / 32;
      constexpr int PF = BIAS && D == 128 ? 1 : 2;  // the bias takes the registers of one operand
      constexpr int EP = 16 / KSN;
      constexpr int ED = 16 / (2 * NB);
      const VC_LDS char* tile = (const VC_LDS char*)smem + st * STAGE;
      const int ln = fresh_lane(), hi = ln >> 5;
      const VC_LDS char* rp = tile + Reads::row_base(perm_row(ln & 31), hi);
      const VC_LDS char* tp = tile + Reads::tr_base(ln);
      const VC_LDS float* stat =
          (const VC_LDS float*)((const VC_LDS char*)smem + STAT + buf * 2 * SQ * 4) + t % SPT * kBQ + 4 * hi;
      f32x16 s, dp;
      bf16x8 f[2 * KSN], gt[4 * NB];
      auto rd = [&](int i) { f[i] = *(const VC_LDS bf16x8*)(Reads::row_at(rp, i % KSN) + (i < KSN ? 0 : RT)); };
      auto rdt = [&](int i) { gt[i] = Reads::tr_operand(tp + (i < 2 * NB ? RT : 0), i / NB % 2, i % NB); };
      float shift = 0.0f;
      int side = 0;
      auto form_p = [&](int r) { s[r] = fast_exp2(BIAS ? fmaf(s[r], a.scale_log2, shift) : s[r] * a.scale_log2); };
      auto form_ds = [&](int r) { dp[r] = s[r] * dp[r]; };
#pragma unroll
      for (int i = 0; i < PF; ++i) rd(i);
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // S accumulates on top of -LSE/c, dP on top of -D of its query rows
        const f32x4 nl = *(const VC_LDS f32x4*)(stat + 8 * j), nd = *(const VC_LDS f32x4*)(stat + SQ + 8 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[4 * j + i] = nl[i];
          dp[4 * j + i] = nd[i];
        }
      }
      if (BIAS) {
        side = bias_side(pos_k, pos_k + 31, q0 + sr.off, q0 + sr.off + 31, a.R);
        if (side == 0) {
          const float* b = tb + kBiasPad + a.R + (pos_k + (ln & 31) - q0 - sr.off - 4 * hi);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] += b[-(8 * (r >> 2) + (r & 3))];
        } else {
          shift = uniform(tb[kBiasPad + (side > 0 ? 2 * a.R : 0)] * a.scale_log2);
        }
      }
#pragma unroll
      for (int i = 0; i < KSN; ++i) {
        sched_fence();
        rd(i + PF);
        s = mfma32(f[i], kf[i], s);
#pragma unroll
        for (int j = 0; j < CPW; ++j)
          if (j * KSN / CPW == i) issue_j(j, gn, qn, st ^ 1);
      }
      if (a.causal && q0 < wave_q + 31) {  // queries before this lane's key
        sched_fence();
        const int jmin = lane_key() - sr.off - q0 - 4 * (fresh_lane() >> 5);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = acc_row(r, 0) >= jmin ? s[r] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < KSN; ++i) {
        sched_fence();
        if (i + PF < KSN)
          rd(KSN + i + PF);
        else
          rdt(i + PF - KSN);
        dp = mfma32(f[KSN + i], vf[i], dp);
        if (i > 0) {
#pragma unroll
          for (int e = 0; e < EP; ++e) form_p((i - 1) * EP + e);
        }
      }
      bf16x8 pb[2], sb[2];
      sched_fence();
      pb[0] = operand(s, 0);
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i) {
        sched_fence();
        rdt(i + PF);
        dv_acc[i % NB] = mfma32(gt[i], pb[i / NB], dv_acc[i % NB]);
        if (i == 0) {
#pragma unroll
          for (int e = 0; e < EP; ++e) form_p((KSN - 1) * EP + e);
          pb[1] = operand(s, 1);
        } else {
#pragma unroll
          for (int e = 0; e < ED; ++e) form_ds((i - 1) * ED + e);
        }
      }
      sched_fence();
      if (BIAS) {  // before dK's operands need the registers
#pragma unroll
        for (int e = 0; e < ED; ++e) form_ds((2 * NB - 1) * ED + e);
        sb[1] = operand(dp, 1);
      }
      sb[0] = operand(dp, 0);
      if (BIAS) {
        const int fl = fresh_lane();
        if (lane_key() >= sr.nk) {  // a key past the sequence's own has gone along with its last one
#pragma unroll
          for (int r = 0; r < 16; ++r) dp[r] = 0.0f;
        }
        if (side == 0) {
          const float x = distance_sums(dp, fl);
          const int d = pos_k - q0 - sr.off + (fl & 31) - 32 * (fl >> 5);
          float* to = d <= -a.R ? ends + w * 128 + fl : d >= a.R ? ends + w * 128 + 64 + fl : hist + w * HIST + d + a.R;
          *to += x;
        } else {
          float x = 0.0f;
#pragma unroll
          for (int r = 0; r < 16; ++r) x += dp[r];
          ends[w * 128 + (side < 0 ? 0 : 64) + fl] += x;
        }
      }
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i) {
        sched_fence();
        if (2 * NB + i + PF < 4 * NB) rdt(2 * NB + i + PF);
        dk_acc[i % NB] = mfma32(gt[2 * NB + i], sb[i / NB], dk_acc[i % NB]);
        if (!BIAS && i == 0) {
#pragma unroll
          for (int e = 0; e < ED; ++e) form_ds((2 * NB - 1) * ED + e);
          sb[1] = operand(dp, 1);
        }
      }
      sched_fence();
    }
    g = gn;
    t = tn;
    buf = bufn;
  }
  wait_all_memory();  // no copy outlives the workgroup
  if (BIAS) {  // the head's sums per distance, waves in order
    __syncthreads();
    const int ln = fresh_lane(), nd = 2 * a.R + 1;
    float* out = a.dist_part + ((dist_row(sr.k0, seq, blk, BM) * a.Hkv + kv) * a.chunks + chunk) * nd;
    auto end_sum = [&](int side) {
      float x = 0.0f;
#pragma unroll
      for (int j = 0; j < NW; ++j) x += ends[j * 128 + side * 64 + ln];
      return wave_sum(x);
    };
    if (w == 0) {  // with R = 0 one distance stands for all
      const float x = a.R == 0 ? end_sum(0) + end_sum(1) : end_sum(0);
      if (ln == 0) out[0] = x;
    } else if (w == 1 && a.R > 0) {
      const float x = end_sum(1);
      if (ln == 0) out[nd - 1] = x;
    }
    for (int i = 1 + tid; i < nd - 1; i += 64 * NW) {
      float x = 0.0f;
#pragma unroll
      for (int j = 0; j < NW; ++j) x += hist[j * HIST + i];
      out[i] = x;
    }
  }

  const int key = lane_key(), hi = fresh_lane() >> 5;
  const bool valid = key < sr.nk;
  if (key < sr.sk) {  // rows of the slot past the sequence's own keys: exactly 0
    if (a.chunks > 1) {
      const size_t one = (size_t)a.Tk * a.Hkv * D;
      float* pk = a.key_part + (size_t)chunk * 2 * one + ((size_t)(sr.k0 + key) * a.Hkv + kv) * D;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x16 &x = dk_acc[db], &y = dv_acc[db];
          f32x4 tk, tv;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            tk[e] = valid ? x[4 * j + e] * a.scale : 0.0f;
            tv[e] = valid ? y[4 * j + e] : 0.0f;
          }
          *(f32x4*)(pk + db * 32 + 8 * j + 4 * hi) = tk;
          *(f32x4*)(pk + one + db * 32 + 8 * j + 4 * hi) = tv;
        }
      return;
    }
    const size_t at = ((size_t)(sr.k0 + key) * a.Hkv + kv) * D;
    auto kr = [&](float x) { return (__bf16)(valid ? x * a.scale : 0.0f); };
    auto vr = [&](float x) { return (__bf16)(valid ? x : 0.0f); };
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x16 &x = dk_acc[db], &y = dv_acc[db];
        *(bf16x4*)(a.dk + at + db * 32 + 8 * j + 4 * hi) = bf16x4{kr(x[4 * j]), kr(x[4 * j + 1]), kr(x[4 * j + 2]), kr(x[4 * j + 3])};
        *(bf16x4*)(a.dv + at + db * 32 + 8 * j + 4 * hi) = bf16x4{vr(y[4 * j]), vr(y[4 * j + 1]), vr(y[4 * j + 2]), vr(y[4 * j + 3])};
      }
  }
}

// dK, dV of every slot row as the sum of the chunks' partials, in order. One thread per 4 elements of each.
__global__ __launch_bounds__(256) void packed_key_sum_kernel(PackedArgs a, int per_row) {
  const int first = min(max(a.cu_k[0], 0), a.Tk), end = min(max(a.cu_k[a.S], first), a.Tk);
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, one = (size_t)a.Tk * per_row;
  const size_t at = (size_t)first * per_row + 4 * i;
  if (at >= (size_t)end * per_row) return;
  f32x4 sk = {0.0f, 0.0f, 0.0f, 0.0f}, sv = sk;
#pragma unroll 4
  for (int c = 0; c < a.chunks; ++c) {
    sk += *(const f32x4*)(a.key_part + (size_t)c * 2 * one + at);
    sv += *(const f32x4*)(a.key_part + ((size_t)c * 2 + 1) * one + at);
  }
  *(bf16x4*)(a.dk + at) = bf16x4{(__bf16)sk[0], (__bf16)sk[1], (__bf16)sk[2], (__bf16)sk[3]};
  *(bf16x4*)(a.dv + at) = bf16x4{(__bf16)sv[0], (__bf16)sv[1], (__bf16)sv[2], (__bf16)sv[3]};
}

// Bias gradient, one workgroup per head: the blocks' sums per distance added up in order, then
// the distances of each bucket. In both steps the threads share the sums of one result by runs,
// which are then joined in order (one thread per result, bounds looked up at each block: 28 us for
// captions of 8 to 256 tokens at 16 heads, so 6; 1,024 such captions 63, 4,096 251, as the workgroups stay
// one per head: a twentieth of the backward).
__global__ __launch_bounds__(1024) void packed_dbias_kernel(PackedArgs a, __bf16* dbias) {
  __shared__ float part[1024];
  __shared__ float sum[2 * kMaxBiasDistance + 1];
  __shared__ int bucket[2 * kMaxBiasDistance + 1];
  const int h = blockIdx.x, nd = 2 * a.R + 1, tid = threadIdx.x;
  for (int d = tid; d < nd; d += 1024) bucket[d] = a.buckets[d];
  const int r0 = (int)dist_row(min(max(a.cu_k[0], 0), a.Tk), 0, 0, kPackedRows);
  const int r1 = (int)dist_row(min(max(a.cu_k[a.S], 0), a.Tk), a.S, 0, kPackedRows);
  const int k = a.chunks / a.G;  // chunks of one head: k rows of sums a block
  const float* rows = a.dist_part + (size_t)h * k * nd;
  const size_t one = (size_t)a.H * k * nd;
  for (int d0 = 0; d0 < nd; d0 += 1024) {
    const int n = min(nd - d0, 1024), runs = 1024 / n, run = tid / n, d = d0 + tid % n;
    float x = 0.0f;
    if (run < runs) {
      for (int j = 0; j < k; ++j)
#pragma unroll 8
        for (int r = r0 + run; r < r1; r += runs) x += rows[r * one + (size_t)j * nd + d];
    }
    part[tid] = x;
    __syncthreads();
    if (tid < n) {
      x = 0.0f;
      for (int i = 0; i < runs; ++i) x += part[i * n + tid];
      sum[d] = x;
    }
    __syncthreads();
  }
  for (int u0 = 0; u0 < a.nb; u0 += 1024) {
    const int n = min(a.nb - u0, 1024), runs = min(1024 / n, nd), run = tid / n, u = u0 + tid % n;
    float x = 0.0f;
    if (run < runs) {
#pragma unroll 4
      for (int d = run; d < nd; d += runs) x += bucket[d] == u ? sum[d] : 0.0f;
    }
    part[tid] = x;
    __syncthreads();
    if (tid < n) {
      x = 0.0f;
      for (int i = 0; i < runs; ++i) x += part[i * n + tid];
      dbias[(size_t)h * a.nb + u] = (__bf16)x;
    }
    __syncthreads();
  }
}

}  // namespace

namespace {
template <int D, int RMAX>
void launch_bwd(PackedArgs a, __bf16* dbias, int clear, hipStream_t s) {
  const dim3 block(64 * kPackedWaves);
  set_blocks(a, a.max_q, a.Tq);
  hipLaunchKernelGGL((packed_dq_kernel<D, RMAX>), dim3(a.blocks * a.H * a.dq_chunks + clear), block, 0, s, a);
  if (a.dq_chunks > 1) {
    const int waves = a.compact ? a.blocks * a.H * kPackedRows : a.S * a.max_q * a.H;
    hipLaunchKernelGGL(packed_dq_sum_kernel<D>, dim3((waves + 3) / 4), dim3(256), 0, s, a);
  }
  set_blocks(a, a.max_k, a.Tk);
  hipLaunchKernelGGL((packed_dkdv_kernel<D, RMAX>), dim3(a.blocks * a.Hkv * a.chunks + clear), block, 0, s, a);
  if (a.chunks > 1) {
    const size_t threads = (size_t)a.Tk * a.Hkv * D / 4;
    hipLaunchKernelGGL(packed_key_sum_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a, a.Hkv * D);
  }
  if (RMAX && dbias) hipLaunchKernelGGL(packed_dbias_kernel, dim3(a.H), dim3(1024), 0, s, a, dbias);
}
}  // namespace

hipError_t launch_packed_bwd(const PackedArgs& a, int head_dim, __bf16* dbias, hipStream_t s) {
  const int clear = a.clear ? kClearGroups : 0;
  const int rmax = !a.bias ? 0 : a.R <= kSmallBiasDistance ? kSmallBiasDistance : kMaxBiasDistance;
  if (head_dim == 128 && rmax == 0)
    launch_bwd<128, 0>(a, dbias, clear, s);
  else if (head_dim == 128 && rmax == kSmallBiasDistance)
    launch_bwd<128, kSmallBiasDistance>(a, dbias, clear, s);
  else if (head_dim == 128)
    launch_bwd<128, kMaxBiasDistance>(a, dbias, clear, s);
  else if (rmax == 0)
    launch_bwd<64, 0>(a, dbias, clear, s);
  else if (rmax == kSmallBiasDistance)
    launch_bwd<64, kSmallBiasDistance>(a, dbias, clear, s);
  else
    launch_bwd<64, kMaxBiasDistance>(a, dbias, clear, s);
  return hipGetLastError();
}

}  // namespace vcja
