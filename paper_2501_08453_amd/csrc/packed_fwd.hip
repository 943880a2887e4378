// Forward packed attention for gfx950: sequences of different lengths laid one behind the
// other, grouped heads, causal or not, with an optional bias per bucket of the distance.
//
// One workgroup of four or eight waves owns 128 or 256 query rows of one (sequence, head), each
// wave 32 held in registers; keys and values stream through LDS in tiles of 64 as in the joint
// forward. The wave computes S^T = K Q^T, so that a lane's accumulator column is one query, and
// O^T += V^T P^T with P^T straight from the accumulator layout. Software pipeline: at step j the
// matrix cores get the scores of tile j+1 and then O += P_j V_j, and the softmax of tile j+1
// runs on the vector ALUs among the latter. The exponent base is raised only when a lane's sum
// of 32 probabilities against it exceeds 2^13 (see the joint forward). Probabilities are summed
// unrounded, so that LSE holds to fp32; they are rounded to bf16 for the product with V, the
// matrix cores' operand type. Under the causal rule each wave stops at its own last tile.
#include <algorithm>
#include <type_traits>

#include "packed.hpp"

namespace vcja {
namespace {

constexpr int kBN = kTileTok;
constexpr float kSumLimit = 8192.0f;  // largest accepted sum of a lane's 32 probabilities

// Probabilities 2^(s c log2(e) + sub) of 8 scores (one PV operand), rounded to bf16, with their
// sum before rounding added to sum.
__device__ __forceinline__ bf16x8 probs8(const f32x16& s, int half, float scale_log2, float sub, float& sum) {
  float p[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    p[t] = fast_exp2(fmaf(s[8 * half + t], scale_log2, sub));
    sum += p[t];
  }
  return to_bf16x8(p);
}

// Raises the exponent base of the queries (lanes) that need it to the tile's maximum (both wave
// halves agree), recomputes the tile's probabilities and their sum, and returns the factor that
// rescales what was accumulated against the old base. shift: what the tile's scores lack (log2).
template <int KB>
__device__ __forceinline__ float raise_base(const f32x16* s, float scale_log2, float shift, bool need, float& m, bf16x8* pb,
                                            float& psum) {
  float mx = s[0][0];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
  const float tmax = fmaf(halves_max(mx), scale_log2, shift);
  need = need | (swap_halves(need ? 1.0f : 0.0f) != 0.0f);
  const float m_new = need ? fmaxf(m, tmax) : m;
  const float alpha = m_new == m ? 1.0f : fast_exp2(m - m_new);
  m = m_new;
  const float m_use = m == -INFINITY ? 0.0f : m;  // no valid key yet: all probabilities 0
  psum = 0.0f;
#pragma unroll
  for (int c = 0; c < 2 * KB; ++c) pb[c] = probs8(s[c >> 1], c & 1, scale_log2, shift - m_use, psum);
  return alpha;
}

// O = 0 and LSE = -inf for the rows outside every slot (the last workgroups of a grid).
template <int D>
__device__ __forceinline__ void clear_o(const PackedArgs& a, int wg, int wgs, int tid, int threads) {
  const int head = min(max(a.cu_q[0], 0), a.Tq), end = min(max(a.cu_q[a.S], head), a.Tq);
  const int64_t n = (int64_t)(head + a.Tq - end) * a.H * (D / 8);
  for (int64_t i = (int64_t)wg * threads + tid; i < n; i += (int64_t)wgs * threads) {
    const int64_t rh = i / (D / 8);
    const int r0 = (int)(rh / a.H), h = (int)(rh % a.H), r = r0 < head ? r0 : r0 - head + end;
    *(bf16x8*)(a.o + ((size_t)r * a.H + h) * D + i % (D / 8) * 8) = zero_bf16x8();
    if (i % (D / 8) == 0) a.lse[(size_t)h * a.Tq + r] = -INFINITY;
  }
}

// A chunk's unnormalised O, base and sum of one row: part is [chunks][Tq, H][D], then
// [chunks][Tq, H][2].
template <int D>
__device__ __forceinline__ void write_partial(const PackedArgs& a, int chunk, int row, int h, int hi, const f32x16* oacc, float m,
                                              float l) {
  const size_t rows = (size_t)a.Tq * a.H, at = chunk * rows + (size_t)row * a.H + h;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(f32x4*)(a.part + at * D + db * 32 + 8 * j + 4 * hi) =
          f32x4{oacc[db][4 * j + 0], oacc[db][4 * j + 1], oacc[db][4 * j + 2], oacc[db][4 * j + 3]};
  if (hi == 0) {
    float* ml = a.part + (size_t)a.chunks * rows * D + at * 2;
    ml[0] = m;
    ml[1] = l;
  }
}

// The query rows of a workgroup: row r is query r / pack, head r % pack of its block of heads
// (pack = 1: one head; pack = the group: its heads share every tile of keys).
template <int D, int NW, bool BIAS>
__global__ __launch_bounds__(64 * NW, 8 / NW) void packed_fwd_kernel(PackedArgs a) {
  using Rows = SwzRows<D>;
  using Reads = SwzReads<D>;
  constexpr int BM = 32 * NW;
  constexpr int KT = Rows::bytes(kBN);
  constexpr int CPW = kBN / Rows::RPC / NW;  // copies of a K (V) tile per wave
  __shared__ __attribute__((aligned(1024))) char smem[4 * KT];  // K ring | V ring
  __shared__ float tb[BIAS ? kBiasTable : 1];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int gh = a.G / a.pack;  // head blocks of a group
  const int items = a.nblk * a.Hkv * gh * a.S * a.chunks;
  if ((int)blockIdx.x >= items) {
    clear_o<D>(a, blockIdx.x - items, gridDim.x - items, tid, 64 * NW);
    return;
  }
  const int chunk = (int)blockIdx.x / (items / a.chunks);
  const PackedItem it = packed_item(blockIdx.x % (items / a.chunks), a.nblk, a.Hkv, gh, a.S);
  const SeqRows sr = seq_rows(a, it.s);
  const int b0 = it.blk * BM;
  if (b0 >= sr.sq * a.pack) return;
  const int kv = it.h / gh, h0 = it.h * a.pack;  // first head
  const int row = b0 + w * 32 + l32;
  const int qi = a.pack == 1 ? row : row / a.pack, h = a.pack == 1 ? h0 : h0 + row - qi * a.pack;
  // Keys that the block's last query, the wave's last and first and this lane's query see.
  auto limit = [&](int i) { return a.causal ? max(0, min(sr.nk, i + sr.off + 1)) : sr.nk; };
  const int nrow = sr.nq * a.pack, re = min(b0 + BM, nrow), w0 = b0 + w * 32, we = min(w0 + 32, nrow);
  auto query = [&](int r) { return a.pack == 1 ? r : __builtin_amdgcn_readfirstlane(r / a.pack); };
  const int blk_keys = re > b0 ? limit(query(re - 1)) : 0;
  const int wave_keys = we > w0 ? limit(query(we - 1)) : 0;
  const int wave_all = limit(query(w0));
  const int klim = qi < sr.nq ? limit(qi) : 0;
  const int kt0 = chunk * a.span, kt1 = min((blk_keys + kBN - 1) / kBN, kt0 + a.span);
  if (chunk > 0 && kt0 >= kt1) return;  // the merge does not look at it
  const int wt = (wave_keys + kBN - 1) / kBN;  // the wave's tiles: below this

  // This wave's j-th copies of tile kt's K and V rows into ring slot `slot` (rows past nk repeat row
  // nk - 1: such keys are masked, such values zeroed before use).
  const SwzCopy<D, false> kc(a.k_tok, lane);
  const SwzCopy<D, true> vc(a.v_tok, lane);
  const __bf16* kbase = a.k + (size_t)sr.k0 * a.k_tok + kv * D;
  const __bf16* vbase = a.v + (size_t)sr.k0 * a.v_tok + kv * D;
  auto k_copy = [&](int j, int kt, int slot) {
    const int idx = w + j * NW, first = swz_copy_row<D, false>(kt * kBN, sr.nk, idx);
    copy16_to_lds_opaque(kbase + (size_t)first * a.k_tok, kc.offset(first, sr.nk, a.k_tok),
                         (VC_LDS char*)smem + slot * KT + idx * Rows::GS);
  };
  auto v_copy = [&](int j, int kt, int slot) {
    const int idx = w + j * NW, first = swz_copy_row<D, true>(kt * kBN, sr.nk, idx);
    copy16_to_lds_opaque(vbase + (size_t)first * a.v_tok, vc.offset(first, sr.nk, a.v_tok),
                         (VC_LDS char*)smem + (2 + slot) * KT + idx * Rows::GS);
  };
  if (kt0 < kt1) {  // the first copies, in flight with the loads below
#pragma unroll
    for (int j = 0; j < CPW; ++j) {
      k_copy(j, kt0, 0);
      v_copy(j, kt0, 0);
      k_copy(j, min(kt0 + 1, kt1 - 1), 1);
    }
  }
  bf16x8 qf[D / 16];
  {
    const __bf16* qp = a.q + (size_t)query_row(a, sr, qi) * a.q_tok + h * D + 8 * hi;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const bf16x8*)(qp + 16 * ks);
  }
  if (BIAS) load_bias_table(a, h0, tb, tid, 64 * NW);

  const int krow = Reads::row_base(l32, hi), vtr = Reads::tr_base(lane);
  const int pos0 = w0 + sr.off;  // position of the wave's first query (with a bias: pack = 1)

  // What the scores of tile kt start from (the bias of tiles near the diagonal), and the bias of
  // tiles of one distant bucket (log2).
  auto start = [&](int kt, f32x16* s) {
    s[0] = zero_f32x16();
    s[1] = zero_f32x16();
    if (!BIAS) return 0.0f;
    const int k0 = kt * kBN, side = bias_side(k0, k0 + kBN - 1, pos0, pos0 + 31, a.R);
    if (side != 0) return tb[kBiasPad + (side > 0 ? 2 * a.R : 0)] * a.scale_log2;
    const float* t = tb + kBiasPad + a.R + (k0 + 4 * hi - pos0 - l32);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = t[kb * 32 + 8 * (r >> 2) + (r & 3)];
    return 0.0f;
  };
  // S^T of tile kt in `slot`, K fragments read two k-steps ahead; hook(j) after k-step 2j+1.
  auto scores = [&](int slot, f32x16* s, auto hook) {
    const VC_LDS char* kp = (const VC_LDS char*)smem + slot * KT + krow;
    constexpr int KSN = D / 16;
    bf16x8 f[KSN][2];
    auto rd = [&](int ks) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) f[ks][kb] = *(const VC_LDS bf16x8*)(Reads::row_at(kp, ks) + kb * Rows::bytes(32));
    };
    rd(0);
    rd(1);
#pragma unroll
    for (int ks = 0; ks < KSN; ++ks) {
      sched_fence();
      if (ks + 2 < KSN) rd(ks + 2);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s[kb] = mfma32(f[ks][kb], qf[ks], s[kb]);
      hook(ks);
    }
    sched_fence();
  };
  auto mask = [&](int kt, f32x16* s) {
    const int k0 = kt * kBN;
    if (k0 + kBN <= wave_all) return;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = k0 + kb * 32 + acc_row(r, hi) < klim ? s[kb][r] : -INFINITY;
  };

  f32x16 oacc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) oacc[i] = zero_f32x16();
  float m = -INFINITY, l = 0.0f;  // exponent base (log2 units), this half's sum
  float alpha = 1.0f;             // pending rescale of O
  bool raise = false;
  bf16x8 pb[4];                   // probabilities of the current tile as PV operands
  auto rescale = [&]() {
    if (__any(raise)) {
#pragma unroll
      for (int i = 0; i < D / 32; ++i) oacc[i] *= alpha;
    }
    raise = false;
  };
  auto load_vt = [&](int slot, int c, bf16x8* f) {
    const VC_LDS char* vp = (const VC_LDS char*)smem + (2 + slot) * KT + vtr;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) f[db] = Reads::tr_operand(vp, c, db);
  };
  auto accumulate = [&](int slot) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      bf16x8 f[D / 32];
      load_vt(slot, c, f);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) oacc[db] = mfma32(f[db], pb[c], oacc[db]);
    }
  };

  if (kt0 < kt1) {
    int par = 0;  // ring slot of the tile before `nxt`
    wait_all_memory();
    __syncthreads();
    if (kt0 < wt) {
      f32x16 s[2];
      const float shift = start(kt0, s);
      scores(0, s, [](int) {});
      mask(kt0, s);
      raise_base<2>(s, a.scale_log2, shift, true, m, pb, l);
    }
    for (int nxt = kt0 + 1; nxt < kt1; ++nxt) {
      wait_all_memory();
      __syncthreads();  // K of `nxt` and V of the tile before have landed; the other slots are free
      const int kn = min(nxt + 1, kt1 - 1);  // past the last tile: copied again, never read
      if (nxt >= wt) {                       // past the wave's own tiles
#pragma unroll
        for (int j = 0; j < CPW; ++j) {
          k_copy(j, kn, par);
          v_copy(j, nxt, par ^ 1);
        }
        if (nxt == wt) {
          rescale();
          accumulate(par);
        }
        par ^= 1;
        continue;
      }
      rescale();
      f32x16 s[2];
      const float shift = start(nxt, s);
      scores(par ^ 1, s, [&](int ks) {  // the step's copies, spread over the products
#pragma unroll
        for (int j = 0; j < 2 * CPW; ++j)
          if ((2 * j + 1) * (D / 16) / (4 * CPW) == ks) {
            if (j % 2 == 0)
              k_copy(j / 2, kn, par);
            else
              v_copy(j / 2, nxt, par ^ 1);
          }
      });
      mask(nxt, s);
      // P V of the tile before in four chunks; between them the softmax of `nxt`.
      bf16x8 fa[D / 32], fb[D / 32];
      load_vt(par, 0, fa);
      float psum = 0.0f;
      bf16x8 pn[4];
      const float sub = shift - m;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        sched_fence();
        if (c < 3) load_vt(par, c + 1, fb);
#pragma unroll
        for (int db = 0; db < D / 32; ++db) oacc[db] = mfma32(fa[db], pb[c], oacc[db]);
        pn[c] = probs8(s[c >> 1], c & 1, a.scale_log2, sub, psum);
        if (c < 3) {  // the next chunk's reads first, then products and softmax interleaved
          __builtin_amdgcn_sched_group_barrier(0x100, D / 16, 0);
#pragma unroll
          for (int db = 0; db < D / 32; ++db) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 8, 0);
          }
        }
#pragma unroll
        for (int db = 0; db < D / 32; ++db) fa[db] = fb[db];
      }
      sched_fence();
      const bool need = !(psum <= kSumLimit);
      alpha = 1.0f;
      raise = __any(need);
      if (raise) alpha = raise_base<2>(s, a.scale_log2, shift, need, m, pn, psum);
#pragma unroll
      for (int c = 0; c < 4; ++c) pb[c] = pn[c];
      l = fmaf(l, alpha, psum);
      par ^= 1;
    }
    wait_all_memory();
    if (kt1 * kBN > sr.nk) {  // the value rows past nk that this wave copied: zero (0 * inf is not)
#pragma unroll
      for (int j = 0; j < CPW; ++j) {
        const int idx = w + j * NW;
        if ((kt1 - 1) * kBN + perm_row(Rows::RPC * idx + lane / Rows::CPR) >= sr.nk)
          *(VC_LDS bf16x8*)((VC_LDS char*)smem + (2 + par) * KT + idx * Rows::GS + 16 * lane) = zero_bf16x8();
      }
    }
    __syncthreads();  // V of the last tile landed
    if (kt1 <= wt) {
      rescale();
      accumulate(par);
    }
  }

  // A row past the sequence's own has gone along with its wave's last one: it sees nothing.
  const float lt = klim > 0 ? halves_sum(l) : 0.0f;
  if (qi >= sr.sq) return;  // rows of the slot past the sequence's own: 0, -inf
  if (a.chunks > 1 && (blk_keys + kBN - 1) / kBN > a.span) {  // unnormalised, with base and sum, for the merge
    write_partial<D>(a, chunk, sr.q0 + qi, h, hi, oacc, m, lt);
    return;
  }
  const float inv = lt > 0.0f ? 1.0f / lt : lt == 0.0f ? 0.0f : lt;
  __bf16* op = a.o + ((size_t)(sr.q0 + qi) * a.H + h) * D;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bf16x4 t = {(__bf16)(oacc[db][4 * j + 0] * inv), (__bf16)(oacc[db][4 * j + 1] * inv),
                  (__bf16)(oacc[db][4 * j + 2] * inv), (__bf16)(oacc[db][4 * j + 3] * inv)};
      *(bf16x4*)(op + db * 32 + 8 * j + 4 * hi) = t;
    }
  if (hi == 0)
    a.lse[(size_t)h * a.Tq + sr.q0 + qi] = lt == 0.0f ? -INFINITY : (m + __log2f(lt)) * kLn2;
}

// O and LSE of the rows whose keys several workgroups share, from their partials in order:
// O = sum_c 2^(m_c - M) O_c / sum_c 2^(m_c - M) l_c over the chunks that hold keys (M the largest of
// their bases). One thread per 4 dims of one (query, head).
template <int D>
__global__ __launch_bounds__(256) void packed_merge_kernel(PackedArgs a, int rows_per_block) {
  const int64_t x = ((int64_t)blockIdx.x * 256 + threadIdx.x) / (D / 4);
  const int d = (int)(threadIdx.x % (D / 4)) * 4;
  if (x >= (int64_t)a.S * a.max_q * a.H) return;
  const int h = (int)(x % a.H), i = (int)(x / a.H % a.max_q), s = (int)(x / a.H / a.max_q);
  const int q0 = min(max(a.cu_q[s], 0), a.Tq), sq = min(min(max(a.cu_q[s + 1], q0), a.Tq) - q0, a.max_q);
  if (i >= sq) return;
  const int nq = a.len_q ? min(max(a.len_q[s], 0), sq) : sq;
  const int k0 = min(max(a.cu_k[s], 0), a.Tk), sk = min(min(max(a.cu_k[s + 1], k0), a.Tk) - k0, a.max_k);
  const int nk = a.len_k ? min(max(a.len_k[s], 0), sk) : sk;
  // The tiles of the row's block of rows, as the forward counts them.
  const int row = i * a.pack + h % a.pack, b0 = row / rows_per_block * rows_per_block;
  const int last = (min(b0 + rows_per_block, nq * a.pack) - 1) / a.pack;
  const int keys = b0 >= nq * a.pack ? 0 : a.causal ? max(0, min(nk, last + nk - nq + 1)) : nk;
  const int n = ((keys + kBN - 1) / kBN + a.span - 1) / a.span;
  if (n <= 1) return;  // written by its only workgroup
  const size_t rows = (size_t)a.Tq * a.H, at = (size_t)(q0 + i) * a.H + h;
  const float* ml = a.part + (size_t)a.chunks * rows * D;
  float mx = -INFINITY;
#pragma unroll 4
  for (int c = 0; c < n; ++c) {
    const float* p = ml + (c * rows + at) * 2;
    mx = fmaxf(mx, p[1] > 0.0f ? p[0] : -INFINITY);
  }
  float sum = 0.0f;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int c = 0; c < n; ++c) {
    const float* p = ml + (c * rows + at) * 2;
    const f32x4 o = *(const f32x4*)(a.part + (c * rows + at) * D + d);
    const float l = p[1], wgt = l == 0.0f ? 0.0f : exp2f(p[0] - mx);
    sum += wgt * l;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += l == 0.0f ? 0.0f : wgt * o[e];
  }
  const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
  *(bf16x4*)(a.o + at * D + d) = bf16x4{(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv),
                                        (__bf16)(acc[3] * inv)};
  if (d == 0) a.lse[(size_t)h * a.Tq + q0 + i] = sum == 0.0f ? -INFINITY : (mx + log2f(sum)) * kLn2;
}

template <int D, int NW, bool BIAS>
void launch_blocks(PackedArgs a, int clear, hipStream_t s) {
  constexpr int BM = 32 * NW;
  a.nblk = (a.max_q * a.pack + BM - 1) / BM;
  hipLaunchKernelGGL((packed_fwd_kernel<D, NW, BIAS>), dim3(a.nblk * (a.H / a.pack) * a.S * a.chunks + clear), dim3(64 * NW), 0, s, a);
  if (a.chunks > 1) {
    const int64_t threads = (int64_t)a.S * a.max_q * a.H * (D / 4);
    hipLaunchKernelGGL(packed_merge_kernel<D>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a, BM);
  }
}

}  // namespace

hipError_t launch_packed_fwd(const PackedArgs& a, int head_dim, hipStream_t s) {
  const int clear = a.clear ? 32 : 0;
  auto go = [&](auto d, auto bias) {
    if (a.small)
      launch_blocks<decltype(d)::value, 4, decltype(bias)::value>(a, clear, s);
    else
      launch_blocks<decltype(d)::value, 8, decltype(bias)::value>(a, clear, s);
  };
  using std::integral_constant;
  if (head_dim == 128 && a.bias)
    go(integral_constant<int, 128>{}, std::true_type{});
  else if (head_dim == 128)
    go(integral_constant<int, 128>{}, std::false_type{});
  else if (a.bias)
    go(integral_constant<int, 64>{}, std::true_type{});
  else
    go(integral_constant<int, 64>{}, std::false_type{});
  return hipGetLastError();
}

}  // namespace vcja
