// Forward packed attention for gfx950: sequences of different lengths laid one behind the
// other, grouped heads, causal or not, with an optional bias per bucket of the distance.
//
// One workgroup of eight waves owns 256 query rows of one (sequence, head), each wave 32 held in
// registers; keys and values stream through LDS in tiles of 64 as in the joint forward. The
// wave computes S^T = K Q^T, so that a lane's accumulator column is one query, and
// O^T += V^T P^T with P^T straight from the accumulator layout.
#include "packed.hpp"

namespace vcja {
namespace {

constexpr int kWaves = 8;
constexpr int kBM = 32 * kWaves;
constexpr int kBN = kTileTok;

template <int D, bool BIAS>
__global__ __launch_bounds__(64 * kWaves, 1) void packed_fwd_kernel(PackedArgs a) {
  using Rows = SwzRows<D>;
  using Reads = SwzReads<D>;
  constexpr int KT = Rows::bytes(kBN);
  constexpr int CPW = kBN / Rows::RPC / kWaves;  // copies of a K (V) tile per wave
  __shared__ __attribute__((aligned(1024))) char smem[4 * KT];
  __shared__ float tb[BIAS ? kBiasTable : 1];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int items = a.nblk * a.H * a.S;
  if ((int)blockIdx.x >= items) {  // rows outside every slot
    const int wg = blockIdx.x - items, wgs = gridDim.x - items;
    const int head = min(max(a.cu_q[0], 0), a.Tq), end = min(max(a.cu_q[a.S], head), a.Tq);
    const int rows = head + a.Tq - end;
    for (int64_t i = (int64_t)wg * blockDim.x + tid; i < (int64_t)rows * a.H * (D / 8); i += (int64_t)wgs * blockDim.x) {
      const int64_t rh = i / (D / 8);
      const int r0 = (int)(rh / a.H), h = (int)(rh % a.H), r = r0 < head ? r0 : r0 - head + end;
      *(bf16x8*)(a.o + ((size_t)r * a.H + h) * D + i % (D / 8) * 8) = zero_bf16x8();
      if (i % (D / 8) == 0) a.lse[(size_t)h * a.Tq + r] = -INFINITY;
    }
    return;
  }
  const PackedItem it = packed_item(blockIdx.x, a.nblk, a.Hkv, a.G, a.S);
  const SeqRows sr = seq_rows(a, it.s);
  const int b0 = it.blk * kBM;
  if (b0 >= sr.sq) return;
  const int kv = it.h / a.G;
  const int qi = b0 + w * 32 + l32;  // this lane's query
  // Keys that the block's last query, the wave's last query and this lane's query see.
  auto limit = [&](int i) { return a.causal ? max(0, min(sr.nk, i + sr.off + 1)) : sr.nk; };
  const int qe = min(b0 + kBM, sr.nq);
  const int blk_keys = qe > b0 ? limit(qe - 1) : 0;
  const int wave_keys = b0 + w * 32 < qe ? limit(min(b0 + w * 32 + 32, sr.nq) - 1) : 0;
  const int wave_all = limit(b0 + w * 32);  // keys that every query of the wave sees
  const int klim = qi < sr.nq ? limit(qi) : 0;
  const int ntile = (blk_keys + kBN - 1) / kBN;

  bf16x8 qf[D / 16];
  {
    const __bf16* qp = a.q + (size_t)query_row(a, sr, qi) * a.q_tok + it.h * D + 8 * hi;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const bf16x8*)(qp + 16 * ks);
  }
  if (BIAS) load_bias_table(a, it.h, tb, tid, 64 * kWaves);

  // Rows past nk repeat row nk - 1: such keys are masked, such values zeroed before use.
  const SwzCopy<D, false> kc(a.k_tok, lane);
  const SwzCopy<D, true> vc(a.v_tok, lane);
  const __bf16* kbase = a.k + (size_t)sr.k0 * a.k_tok + kv * D;
  const __bf16* vbase = a.v + (size_t)sr.k0 * a.v_tok + kv * D;
  auto copy_tile = [&](int kt, int slot) {
#pragma unroll
    for (int j = 0; j < CPW; ++j) {
      const int idx = w + j * kWaves;
      const int fk = swz_copy_row<D, false>(kt * kBN, sr.nk, idx), fv = swz_copy_row<D, true>(kt * kBN, sr.nk, idx);
      copy16_to_lds_opaque(kbase + (size_t)fk * a.k_tok, kc.offset(fk, sr.nk, a.k_tok), (VC_LDS char*)smem + slot * KT + idx * Rows::GS);
      copy16_to_lds_opaque(vbase + (size_t)fv * a.v_tok, vc.offset(fv, sr.nk, a.v_tok),
                           (VC_LDS char*)smem + (2 + slot) * KT + idx * Rows::GS);
    }
  };

  f32x16 oacc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) oacc[i] = zero_f32x16();
  float m = -INFINITY, l = 0.0f;
  const int pos0 = b0 + w * 32 + sr.off;  // position of the wave's first query

  if (ntile > 0) copy_tile(0, 0);
  for (int kt = 0; kt < ntile; ++kt) {
    const int slot = kt & 1;
    wait_all_memory();
    if (kt * kBN + kBN > sr.nk) {  // the value rows past nk that this wave copied
#pragma unroll
      for (int j = 0; j < CPW; ++j) {
        const int idx = w + j * kWaves;
        if (kt * kBN + perm_row(Rows::RPC * idx + lane / Rows::CPR) >= sr.nk)
          *(VC_LDS bf16x8*)((VC_LDS char*)smem + (2 + slot) * KT + idx * Rows::GS + 16 * lane) = zero_bf16x8();
      }
    }
    __syncthreads();
    if (kt + 1 < ntile) copy_tile(kt + 1, slot ^ 1);
    const int k0 = kt * kBN;
    if (k0 >= wave_keys) continue;
    const VC_LDS char* kp = (const VC_LDS char*)smem + slot * KT + Reads::row_base(l32, hi);
    const VC_LDS char* vp = (const VC_LDS char*)smem + (2 + slot) * KT + Reads::tr_base(lane);
    f32x16 s[2];
    float shift = 0.0f;
    if (BIAS) {
      const int side = bias_side(k0, k0 + kBN - 1, pos0, pos0 + 31, a.R);
      if (side == 0) {
        const float* t = tb + kBiasPad + a.R + (k0 + 4 * hi - pos0 - l32);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kb][r] = t[kb * 32 + 8 * (r >> 2) + (r & 3)];
      } else {
        const float c = tb[kBiasPad + (side > 0 ? 2 * a.R : 0)];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kb][r] = c;
      }
    } else {
      s[0] = zero_f32x16();
      s[1] = zero_f32x16();
    }
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        s[kb] = mfma32(*(const VC_LDS bf16x8*)(Reads::row_at(kp, ks) + kb * Rows::bytes(32)), qf[ks], s[kb]);
    if (k0 + kBN > wave_all) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kb][r] = k0 + kb * 32 + acc_row(r, hi) < klim ? s[kb][r] : -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
    const float m_new = fmaxf(m, halves_max(mx) * a.scale_log2);
    const float m_use = m_new == -INFINITY ? 0.0f : m_new;
    const float alpha = fast_exp2(m - m_use);
    m = m_new;
    float p[32], sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      p[i] = fast_exp2(fmaf(s[i >> 4][i & 15], a.scale_log2, shift - m_use));
      sum += p[i];  // the sum of the unrounded probabilities: LSE is exact to fp32
    }
    l = fmaf(l, alpha, sum);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) oacc[i] *= alpha;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const bf16x8 pb = to_bf16x8(p + 8 * c);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) oacc[db] = mfma32(Reads::tr_operand(vp, c, db), pb, oacc[db]);
    }
  }
  wait_all_memory();  // no copy outlives the workgroup

  // A row past the sequence's own has gone along with its wave's last one: it sees nothing.
  const float lt = klim > 0 ? halves_sum(l) : 0.0f;
  const float inv = lt > 0.0f ? 1.0f / lt : lt == 0.0f ? 0.0f : lt;
  if (qi < sr.sq) {  // rows of the slot past the sequence's own: 0, -inf
    __bf16* op = a.o + ((size_t)(sr.q0 + qi) * a.H + it.h) * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x4 t = {(__bf16)(oacc[db][4 * j + 0] * inv), (__bf16)(oacc[db][4 * j + 1] * inv),
                    (__bf16)(oacc[db][4 * j + 2] * inv), (__bf16)(oacc[db][4 * j + 3] * inv)};
        *(bf16x4*)(op + db * 32 + 8 * j + 4 * hi) = t;
      }
    if (hi == 0)
      a.lse[(size_t)it.h * a.Tq + sr.q0 + qi] = lt == 0.0f ? -INFINITY : (m + __log2f(lt)) * kLn2;
  }
}

}  // namespace

hipError_t launch_packed_fwd(const PackedArgs& args, int head_dim, hipStream_t s) {
  PackedArgs a = args;
  a.nblk = (a.max_q + kBM - 1) / kBM;
  const dim3 grid(a.nblk * a.H * a.S + (a.clear ? 32 : 0)), block(64 * kWaves);
  if (head_dim == 128 && a.bias)
    hipLaunchKernelGGL((packed_fwd_kernel<128, true>), grid, block, 0, s, a);
  else if (head_dim == 128)
    hipLaunchKernelGGL((packed_fwd_kernel<128, false>), grid, block, 0, s, a);
  else if (a.bias)
    hipLaunchKernelGGL((packed_fwd_kernel<64, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((packed_fwd_kernel<64, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace vcja
