// Backward packed attention for gfx950 (see packed_fwd.hip for the layout of the sequences).
//
// dQ (query-stationary, first): one workgroup of eight waves owns 256 query rows of one
//   (sequence, head), each wave 32, with Q^T and dO^T of its queries in registers. It forms
//   D_i = <dO_i, O_i> from its own rows and writes -D and -LSE / c for the other pass, walks
//   over the key tiles like the forward, computing S^T, dP^T and dS^T = P^T o (dP^T - D), and
//   dQ^T += K^T dS^T.
//   With a bias it also sums dS over every distance (see distance_sums).
// dK/dV (key-stationary): one workgroup owns 256 keys of one (sequence, key head), each wave 32,
//   K and V of its keys in registers, and walks over the query tiles of 32 of every query head
//   of the group, so that dK and dV of the shared head are summed in registers.
// No atomics anywhere: results are bitwise reproducible.
#include "packed.hpp"

namespace vcja {
namespace {

constexpr int kWaves = 8;
constexpr int kBM = 32 * kWaves;   // queries (keys) per workgroup
constexpr int kBN = kTileTok;      // keys per dQ tile
constexpr int kBQ = 32;            // queries per dK/dV tile

__device__ __forceinline__ bf16x8 operand(const f32x16& x, int half) {
  bf16x8 y;
#pragma unroll
  for (int t = 0; t < 8; ++t) y[t] = (__bf16)x[8 * half + t];
  return y;
}

// Sums of one 32 keys x 32 queries block of dS^T over its diagonals (distance = key - query),
// without atomics. Register r of lane (col t, half hi) holds key row kr = 8 (r / 4) + 4 hi + r % 4:
// rotating it by kr brings distance t (where kr >= t) or t - 32 to lane t, the same for every
// register, so that a lane adds its own values up; the two halves of the wave are joined at
// the end, the lower one keeping distances 0 .. 31, the upper one -32 .. -1.
__device__ __forceinline__ float distance_sums(const f32x16& ds, int lane) {
  const int t = lane & 31, hi = lane >> 5;
  float pos = 0.0f, neg = 0.0f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int kr = acc_row(r, hi);
    const float x = __shfl(ds[r], (lane & 32) | ((kr - t) & 31), 64);
    pos += t <= kr ? x : 0.0f;
    neg += t <= kr ? 0.0f : x;
  }
  pos = halves_sum(pos);
  neg = halves_sum(neg);
  return hi ? neg : pos;
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

template <int D, bool BIAS>
__global__ __launch_bounds__(64 * kWaves, 1) void packed_dq_kernel(PackedArgs a) {
  using Rows = SwzRows<D>;
  using Reads = SwzReads<D>;
  constexpr int RT = Rows::bytes(kBN);
  constexpr int STAGE = 2 * RT;
  constexpr int CPW = kBN / Rows::RPC / kWaves;
  constexpr int HIST = 2 * kMaxBiasDistance + 1;
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE];
  __shared__ float tb[BIAS ? kBiasTable : 1];
  __shared__ float hist[BIAS ? kWaves * HIST : 1];  // each wave's sums per distance

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int items = a.nblk * a.H * a.S;
  if ((int)blockIdx.x >= items) {  // rows outside every slot
    const int wg = blockIdx.x - items, wgs = gridDim.x - items;
    const int head = min(max(a.cu_q[0], 0), a.Tq), end = min(max(a.cu_q[a.S], head), a.Tq);
    const int64_t per = (int64_t)a.H * (D / 8);
    for (int64_t i = (int64_t)wg * blockDim.x + tid; i < (head + a.Tq - end) * per; i += (int64_t)wgs * blockDim.x) {
      const int r = (int)(i / per);
      *(bf16x8*)(a.dq + (size_t)(r < head ? r : r - head + end) * a.H * D + i % per * 8) = zero_bf16x8();
    }
    return;
  }
  const PackedItem it = packed_item(blockIdx.x, a.nblk, a.Hkv, a.G, a.S);
  const SeqRows sr = seq_rows(a, it.s);
  const int b0 = it.blk * kBM;
  if (b0 >= sr.sq) return;
  const int kv = it.h / a.G;
  const int qi = b0 + w * 32 + l32;
  auto limit = [&](int i) { return a.causal ? max(0, min(sr.nk, i + sr.off + 1)) : sr.nk; };
  const int qe = min(b0 + kBM, sr.nq);
  const int blk_keys = qe > b0 ? limit(qe - 1) : 0;
  const int wave_keys = b0 + w * 32 < qe ? limit(min(b0 + w * 32 + 32, sr.nq) - 1) : 0;
  const int wave_all = limit(b0 + w * 32);
  const int klim = qi < sr.nq ? limit(qi) : 0;
  const int ntile = (blk_keys + kBN - 1) / kBN;

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
    dd = -halves_sum(sum);
    const float x = a.lse[(size_t)it.h * a.Tq + row];
    nls = klim == 0 || x == -INFINITY ? -INFINITY : -x / a.scale;
    if (klim == 0) dd = 0.0f;
    if (hi == 0 && qi < ((sr.nq + 63) & ~63)) {
      const size_t p = (size_t)it.h * a.npad + packed_row(sr.q0, it.s) + qi;
      a.nls[p] = nls;
      a.dd[p] = dd;
    }
  }
  if (BIAS) {
    load_bias_table(a, it.h, tb, tid, 64 * kWaves);
    for (int i = tid; i < kWaves * HIST; i += 64 * kWaves) hist[i] = 0.0f;
  }

  const SwzCopy<D, true> kc(a.k_tok, lane), vc(a.v_tok, lane);
  const __bf16* kbase = a.k + (size_t)sr.k0 * a.k_tok + kv * D;
  const __bf16* vbase = a.v + (size_t)sr.k0 * a.v_tok + kv * D;
  auto copy_tile = [&](int kt, int st) {
#pragma unroll
    for (int j = 0; j < CPW; ++j) {
      const int idx = w + j * kWaves, first = swz_copy_row<D, true>(kt * kBN, sr.nk, idx);
      VC_LDS char* dst = (VC_LDS char*)smem + st * STAGE + idx * Rows::GS;
      copy16_to_lds_opaque(kbase + (size_t)first * a.k_tok, kc.offset(first, sr.nk, a.k_tok), dst);
      copy16_to_lds_opaque(vbase + (size_t)first * a.v_tok, vc.offset(first, sr.nk, a.v_tok), dst + RT);
    }
  };

  f32x16 acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc[i] = zero_f32x16();
  const int pos0 = b0 + w * 32 + sr.off;
  const float nlse2 = nls * a.scale_log2;
  float far_lo = 0.0f, far_hi = 0.0f;

  if (ntile > 0) copy_tile(0, 0);
  for (int kt = 0; kt < ntile; ++kt) {
    const int st = kt & 1;
    wait_all_memory();
    __syncthreads();
    if (kt + 1 < ntile) copy_tile(kt + 1, st ^ 1);
    const int k0 = kt * kBN;
    if (k0 >= wave_keys) continue;
    const VC_LDS char* tile = (const VC_LDS char*)smem + st * STAGE;
    const VC_LDS char* rp = tile + Reads::row_base(perm_row(l32), hi);
    const VC_LDS char* tp = tile + Reads::tr_base(lane);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 s = zero_f32x16(), dp;
      int side = 0;
      if (BIAS) {
        side = bias_side(k0 + 32 * kb, k0 + 32 * kb + 31, pos0, pos0 + 31, a.R);
        const float* t = tb + kBiasPad + a.R + (k0 + 32 * kb + 4 * hi - pos0 - l32);
        const float c = tb[kBiasPad + (side > 0 ? 2 * a.R : 0)];
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = c;
        if (side == 0) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = t[8 * (r >> 2) + (r & 3)];
        }
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] = dd;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        s = mfma32(*(const VC_LDS bf16x8*)(Reads::row_at(rp, ks) + kb * Rows::bytes(32)), qf[ks], s);
        dp = mfma32(*(const VC_LDS bf16x8*)(Reads::row_at(rp, ks) + RT + kb * Rows::bytes(32)), dof[ks], dp);
      }
      if (k0 + 32 * kb + 32 > wave_all) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = k0 + 32 * kb + acc_row(r, hi) < klim ? s[r] : -INFINITY;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] *= fast_exp2(fmaf(s[r], a.scale_log2, nlse2));
      if (BIAS) {
        if (side == 0) {
          const float x = distance_sums(dp, lane);
          const int d = k0 + 32 * kb - pos0 + l32 - 32 * hi;
          if (d <= -a.R)
            far_lo += x;
          else if (d >= a.R)
            far_hi += x;
          else
            hist[w * HIST + d + a.R] += x;
        } else {
          float x = 0.0f;
#pragma unroll
          for (int r = 0; r < 16; ++r) x += dp[r];
          far_lo += side < 0 ? x : 0.0f;
          far_hi += side < 0 ? 0.0f : x;
        }
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bf16x8 sb = operand(dp, half);
#pragma unroll
        for (int db = 0; db < D / 32; ++db) acc[db] = mfma32(Reads::tr_operand(tp, 2 * kb + half, db), sb, acc[db]);
      }
    }
  }
  wait_all_memory();  // no copy outlives the workgroup

  if (BIAS) {  // the block's sums per distance, waves in order
    far_lo = wave_sum(far_lo);
    far_hi = wave_sum(far_hi);
    __syncthreads();
    if (lane == 0) {
      hist[w * HIST] += far_lo;
      hist[w * HIST + 2 * a.R] += far_hi;
    }
    __syncthreads();
    float* out = a.dist_part + (((size_t)it.s * a.nblk + it.blk) * a.H + it.h) * (2 * a.R + 1);
    for (int i = tid; i < 2 * a.R + 1; i += 64 * kWaves) {
      float x = 0.0f;
      for (int j = 0; j < kWaves; ++j) x += hist[j * HIST + i];
      out[i] = x;
    }
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

template <int D, bool BIAS>
__global__ __launch_bounds__(64 * kWaves, 1) void packed_dkdv_kernel(PackedArgs a) {
  using Rows = SwzRows<D>;
  using Reads = SwzReads<D>;
  constexpr int RT = Rows::bytes(kBQ);
  constexpr int STAGE = 2 * RT;                   // Q rows | dO rows
  constexpr int COPIES = kBQ / Rows::RPC;
  constexpr int STAT = 2 * STAGE;                 // -LSE/c[32] | -D[32] of a tile, two buffers
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE + 2 * 256];
  __shared__ float tb[BIAS ? kBiasTable : 1];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int items = a.nblk * a.Hkv * a.S;
  if ((int)blockIdx.x >= items) {  // rows outside every slot
    const int wg = blockIdx.x - items, wgs = gridDim.x - items;
    const int head = min(max(a.cu_k[0], 0), a.Tk), end = min(max(a.cu_k[a.S], head), a.Tk);
    const int64_t per = (int64_t)a.Hkv * (D / 8);
    for (int64_t i = (int64_t)wg * blockDim.x + tid; i < (head + a.Tk - end) * per; i += (int64_t)wgs * blockDim.x) {
      const int r = (int)(i / per);
      const size_t at = (size_t)(r < head ? r : r - head + end) * a.Hkv * D + i % per * 8;
      *(bf16x8*)(a.dk + at) = zero_bf16x8();
      *(bf16x8*)(a.dv + at) = zero_bf16x8();
    }
    return;
  }
  // Under the causal rule the first key blocks are the longest: dispatched first.
  const int HS = a.Hkv * a.S, kv = blockIdx.x % a.Hkv, seq = blockIdx.x / a.Hkv % a.S;
  const int b0 = (int)(blockIdx.x / HS) * kBM;
  const SeqRows sr = seq_rows(a, seq);
  if (b0 >= sr.sk) return;
  const int key = b0 + w * 32 + l32;  // this lane's key
  const bool valid = key < sr.nk;
  // Query tiles that see the block's keys: from the first query at or past its first key.
  const int first_q = a.causal ? max(0, b0 - sr.off) : 0;
  const int t0 = first_q / kBQ, nt = b0 < sr.nk ? max(0, (sr.nq + kBQ - 1) / kBQ - t0) : 0;
  const int steps = nt * a.G;
  const int wave_q = a.causal ? b0 + w * 32 - sr.off : 0;  // first query that sees a key of the wave

  const __bf16* qbase = a.q + (size_t)sr.q0 * a.q_tok;
  const unsigned o_tok = a.H * D;
  const __bf16* dbase = a.dout + (size_t)sr.q0 * o_tok;
  const int srow = packed_row(sr.q0, seq);
  auto copy_tile = [&](int u, int st) {
    const int g = u / nt, q0 = (t0 + u % nt) * kBQ, h = kv * a.G + g;
    const int idx = w % COPIES, first = swz_copy_row<D, true>(q0, sr.nq, idx);
    VC_LDS char* dst = (VC_LDS char*)smem + st * STAGE + idx * Rows::GS;
    if (D == 128 || w < COPIES)
      copy16_to_lds_opaque(qbase + (size_t)first * a.q_tok + h * D, swz_copy_off<D, true>(first, a.q_tok, sr.nq, lane), dst);
    if (D == 128 || w >= COPIES)
      copy16_to_lds_opaque(dbase + (size_t)first * o_tok + h * D, swz_copy_off<D, true>(first, o_tok, sr.nq, lane), dst + RT);
    if (w == 0) {
      const size_t p = (size_t)h * a.npad + srow + q0 + l32;
      ((VC_LDS float*)((VC_LDS char*)smem + STAT + st * 256))[lane] = hi ? a.dd[p] : a.nls[p];
    }
  };

  bf16x8 kf[D / 16], vf[D / 16];
  {
    const size_t row = min(sr.k0 + min(key, max(sr.nk - 1, 0)), a.Tk - 1);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      kf[ks] = *(const bf16x8*)(a.k + row * a.k_tok + kv * D + 16 * ks + 8 * hi);
      vf[ks] = *(const bf16x8*)(a.v + row * a.v_tok + kv * D + 16 * ks + 8 * hi);
    }
  }
  f32x16 dk_acc[D / 32], dv_acc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    dk_acc[i] = zero_f32x16();
    dv_acc[i] = zero_f32x16();
  }
  const int pos_k = b0 + w * 32;  // position of the wave's first key
  if (steps > 0) copy_tile(0, 0);
  for (int u = 0; u < steps; ++u) {
    const int st = u & 1, g = u / nt, q0 = (t0 + u % nt) * kBQ;
    wait_all_memory();
    // dO rows past nq that this wave copied: zero, as a probability of 0 does not silence an
    // infinite value of row nq - 1, which they repeat.
    if (q0 + kBQ > sr.nq && (D == 128 || w >= COPIES)) {
      const int idx = w % COPIES;
      if (q0 + perm_row(Rows::RPC * idx + lane / Rows::CPR) >= sr.nq)
        *(VC_LDS bf16x8*)((VC_LDS char*)smem + st * STAGE + RT + idx * Rows::GS + 16 * lane) = zero_bf16x8();
    }
    if (BIAS && u % nt == 0) {
      __syncthreads();  // the previous head's table is no longer read
      load_bias_table(a, kv * a.G + g, tb, tid, 64 * kWaves);
    }
    __syncthreads();
    if (u + 1 < steps) copy_tile(u + 1, st ^ 1);
    if (q0 + kBQ <= wave_q) continue;
    const VC_LDS char* tile = (const VC_LDS char*)smem + st * STAGE;
    const VC_LDS char* rp = tile + Reads::row_base(perm_row(l32), hi);
    const VC_LDS char* tp = tile + Reads::tr_base(lane);
    const VC_LDS float* stat = (const VC_LDS float*)((const VC_LDS char*)smem + STAT + st * 256) + 4 * hi;
    f32x16 s, dp;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 nl = *(const VC_LDS f32x4*)(stat + 8 * j), nd = *(const VC_LDS f32x4*)(stat + 32 + 8 * j);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[4 * j + i] = nl[i];
        dp[4 * j + i] = nd[i];
      }
    }
    float shift = 0.0f;
    if (BIAS) {
      const int side = bias_side(pos_k, pos_k + 31, q0 + sr.off, q0 + sr.off + 31, a.R);
      if (side == 0) {
        const float* t = tb + kBiasPad + a.R + (pos_k + l32 - q0 - sr.off - 4 * hi);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] += t[-(8 * (r >> 2) + (r & 3))];
      } else {
        shift = tb[kBiasPad + (side > 0 ? 2 * a.R : 0)] * a.scale_log2;
      }
    }
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      s = mfma32(*(const VC_LDS bf16x8*)Reads::row_at(rp, ks), kf[ks], s);
      dp = mfma32(*(const VC_LDS bf16x8*)(Reads::row_at(rp, ks) + RT), vf[ks], dp);
    }
    if (a.causal && q0 < wave_q + 31) {  // queries before this lane's key
      const int jmin = key - sr.off;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = q0 + acc_row(r, hi) >= jmin ? s[r] : -INFINITY;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = fast_exp2(fmaf(s[r], a.scale_log2, shift));
      dp[r] *= s[r];
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const bf16x8 pb = operand(s, half), sb = operand(dp, half);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        dv_acc[db] = mfma32(Reads::tr_operand(tp + RT, half, db), pb, dv_acc[db]);
        dk_acc[db] = mfma32(Reads::tr_operand(tp, half, db), sb, dk_acc[db]);
      }
    }
  }
  wait_all_memory();  // no copy outlives the workgroup

  if (key < sr.sk) {  // rows of the slot past the sequence's own keys: exactly 0
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

// Bias gradient: the row blocks' sums per distance added up in order (one workgroup per head),
// then the distances of each bucket.
__global__ __launch_bounds__(1024) void packed_dbias_kernel(PackedArgs a, __bf16* dbias) {
  __shared__ float part[1024];
  __shared__ float sum[2 * kMaxBiasDistance + 1];
  const int h = blockIdx.x, nd = 2 * a.R + 1, tid = threadIdx.x;
  const int groups = max(1, 1024 / nd), per = min(nd, 1024);  // threads: `groups` runs of blocks x distances
  for (int d0 = 0; d0 < nd; d0 += per) {
    const int d = d0 + tid % per, g = tid / per;
    float x = 0.0f;
    if (g < groups && d < nd) {
      for (int i = g; i < a.S * a.nblk; i += groups) {
        const SeqRows sr = seq_rows(a, i / a.nblk);
        if (i % a.nblk * kBM < sr.sq) x += a.dist_part[((size_t)i * a.H + h) * nd + d];
      }
    }
    part[tid] = x;
    __syncthreads();
    if (tid < per && d < nd) {
      float y = 0.0f;
      for (int j = 0; j < groups; ++j) y += part[j * per + tid];
      sum[d] = y;
    }
    __syncthreads();
  }
  for (int u = tid; u < a.nb; u += 1024) {
    float x = 0.0f;
    for (int d = 0; d < nd; ++d) x += a.buckets[d] == u ? sum[d] : 0.0f;
    dbias[(size_t)h * a.nb + u] = (__bf16)x;
  }
}

}  // namespace

hipError_t launch_packed_bwd(const PackedArgs& args, int head_dim, __bf16* dbias, hipStream_t s) {
  PackedArgs a = args;
  const int clear = a.clear ? 32 : 0;
  const dim3 block(64 * kWaves);
  a.nblk = (a.max_q + kBM - 1) / kBM;
  const dim3 qgrid(a.nblk * a.H * a.S + clear);
  if (head_dim == 128 && a.bias)
    hipLaunchKernelGGL((packed_dq_kernel<128, true>), qgrid, block, 0, s, a);
  else if (head_dim == 128)
    hipLaunchKernelGGL((packed_dq_kernel<128, false>), qgrid, block, 0, s, a);
  else if (a.bias)
    hipLaunchKernelGGL((packed_dq_kernel<64, true>), qgrid, block, 0, s, a);
  else
    hipLaunchKernelGGL((packed_dq_kernel<64, false>), qgrid, block, 0, s, a);
  if (dbias) hipLaunchKernelGGL(packed_dbias_kernel, dim3(a.H), dim3(1024), 0, s, a, dbias);
  a.nblk = (a.max_k + kBM - 1) / kBM;
  const dim3 kgrid(a.nblk * a.Hkv * a.S + clear);
  if (head_dim == 128 && a.bias)
    hipLaunchKernelGGL((packed_dkdv_kernel<128, true>), kgrid, block, 0, s, a);
  else if (head_dim == 128)
    hipLaunchKernelGGL((packed_dkdv_kernel<128, false>), kgrid, block, 0, s, a);
  else if (a.bias)
    hipLaunchKernelGGL((packed_dkdv_kernel<64, true>), kgrid, block, 0, s, a);
  else
    hipLaunchKernelGGL((packed_dkdv_kernel<64, false>), kgrid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace vcja
