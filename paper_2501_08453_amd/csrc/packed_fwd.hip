// Forward packed attention for gfx950: sequences of different lengths laid one behind the
// other, grouped heads, causal or not, with an optional bias per bucket of the distance.
//
// One workgroup of four waves owns 128 query rows of one (sequence, head), each wave 32 held in
// registers; two workgroups share a compute unit at D = 128 (213 to 219 registers), three at D = 64 (147 to 149,
// 37 to 43 KB of LDS). (Eight waves and 256 rows, as in the joint forward,
// are 1% faster at 8,192 tokens and up and up to twice as slow below: 509 -> 504 us there, 48 -> 90 us
// at 2,048, both at 32 heads, D = 128.) Keys and values stream through LDS in tiles of 64. The wave computes S^T = K Q^T, so that a lane's accumulator column is one query, and
// O^T += V^T P^T with P^T straight from the accumulator layout. Software pipeline: at step j the
// matrix cores get the scores of tile j+1 and then O += P_j V_j, and the softmax of tile j+1
// runs on the vector ALUs among the latter. The exponent base is raised only when a lane's sum
// of 32 probabilities against it exceeds 2^13 (see the joint forward). Probabilities are summed
// unrounded, so that LSE holds to fp32; they are rounded to bf16 for the product with V, the
// matrix cores' operand type. Under the causal rule each wave stops at its own last tile.
// What bounds it: the matrix rate for long rows (12,000 tokens causal, 16 heads, 2 key heads, D = 128: 561 us,
// 1,051 TFLOP/s; a call of 8,192 x 8,192 uncausal, 16 heads: 554 us, 992 TFLOP/s, and at D = 64, which has as many
// exponentials for half the products, 300 us, 916), and the waits of a few tiles one after the other for short
// ones (captions of 8 to 256 tokens with the bias, 16 heads, D = 64: 17 us).
#include "packed.hpp"

namespace vcja {
namespace {

constexpr int kBN = kTileTok;
constexpr int kFewWaves = 4;          // of a workgroup of the few-row kernel
constexpr int few_tile(int d) { return d == 128 ? 32 : 64; }  // keys of one of its tiles
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

// Waits until at most N vector-memory operations of this wave are in flight (they end in order).
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Waits for this wave's LDS operations.
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// O = 0 and LSE = -inf, or one of them, for the rows outside every slot (the last workgroups of a grid).
template <int D>
__device__ __forceinline__ void clear_o(const PackedArgs& a, int wg, int wgs, int tid, int threads) {
  const int head = min(max(a.cu_q[0], 0), a.Tq), end = min(max(a.cu_q[a.S], head), a.Tq);
  const int64_t n = (int64_t)(head + a.Tq - end) * a.H * (D / 8);
  for (int64_t i = (int64_t)wg * threads + tid; i < n; i += (int64_t)wgs * threads) {
    const int64_t rh = i / (D / 8);
    const int r0 = (int)(rh / a.H), h = (int)(rh % a.H), r = r0 < head ? r0 : r0 - head + end;
    if (a.clear != 3) *(bf16x8*)(a.o + ((size_t)r * a.H + h) * D + i % (D / 8) * 8) = zero_bf16x8();
    if (a.clear != 2 && i % (D / 8) == 0) a.lse[(size_t)h * a.Tq + r] = -INFINITY;
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
template <int D, int RMAX>
__global__ __launch_bounds__(64 * kPackedWaves, 2) void packed_fwd_kernel(PackedArgs a) {
  using Rows = SwzRows<D>;
  using Reads = SwzReads<D>;
  constexpr int NW = kPackedWaves, BM = kPackedRows;
  constexpr int KT = Rows::bytes(kBN);
  constexpr int CPW = kBN / Rows::RPC / NW;  // copies of a K (V) tile per wave
  __shared__ __attribute__((aligned(1024))) char smem[4 * KT];  // K ring | V ring
  __shared__ BiasTable<RMAX> table;
  constexpr bool BIAS = RMAX > 0;
  const float* const tb = table.tb;

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int gh = a.G / a.pack;  // head blocks of a group
  const int blocks = a.blocks * a.Hkv * gh, items = blocks * a.chunks;
  if ((int)blockIdx.x >= items) {
    clear_o<D>(a, blockIdx.x - items, gridDim.x - items, tid, 64 * NW);
    return;
  }
  const int chunk = (int)blockIdx.x / blocks;
  const PackedItem it = packed_item(a, blockIdx.x % blocks, a.cu_q, a.Tq, a.Hkv, gh, true);
  if (it.s < 0) return;
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
  table.load(a, h0, tid, 64 * NW);

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

// Few rows (single tokens or a few drafted ones at the end of a cache; rows of all heads of a group
// together, 32 at most): memory-bound, so the waves of a workgroup share the keys, not the
// rows. Each wave streams every NW-th tile of its chunk (8 KiB of keys and 8 KiB of values) through
// LDS of its own without a barrier, the next tile's keys in flight once the scores are formed, its
// values once they are used, eight waves a compute unit; their results are joined in LDS at the
// end. 16 sequences' single tokens, 51,188 keys together, 8 key heads, D = 128: 42 us, 5.0 TB/s (two buffers a wave and
// half the waves: 56 us).
template <int D, int RMAX>
__global__ __launch_bounds__(64 * kFewWaves, 8 / kFewWaves) void packed_few_kernel(PackedArgs a) {
  using Rows = SwzRows<D>;
  using Reads = SwzReads<D>;
  constexpr int NW = kFewWaves, KBT = few_tile(D), KB = KBT / 32;
  constexpr int KT = Rows::bytes(KBT);
  constexpr int COPIES = KBT / Rows::RPC;
  constexpr int RING = 2 * KT;       // of a wave: K | V
  constexpr int OS = D + 4;          // floats between the rows of a wave's O
  static_assert(RING >= 32 * OS * 4, "O of a wave fits its ring");
  __shared__ __attribute__((aligned(1024))) char smem[NW * RING];
  __shared__ float ml[NW][32][2];
  __shared__ BiasTable<RMAX> table;
  constexpr bool BIAS = RMAX > 0;
  const float* const tb = table.tb;

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int heads = a.H / a.pack, items = heads * a.S * a.chunks;
  if ((int)blockIdx.x >= items) {
    clear_o<D>(a, blockIdx.x - items, gridDim.x - items, tid, 64 * NW);
    return;
  }
  // Chunks run fastest: 57.5 -> 55.8 us, 53.5 -> 48.7 and 24.3 -> 20.1 against heads first.
  const int chunk = blockIdx.x % a.chunks, hb = blockIdx.x / a.chunks % heads, s = blockIdx.x / a.chunks / heads;
  const SeqRows sr = seq_rows(a, s);
  if (sr.sq == 0) return;
  const int h0 = hb * a.pack, kv = h0 / a.G;
  const int qi = a.pack == 1 ? l32 : l32 / a.pack, h = h0 + l32 - qi * a.pack;
  auto limit = [&](int i) { return a.causal ? max(0, min(sr.nk, i + sr.off + 1)) : sr.nk; };
  const int keys = sr.nq > 0 ? limit(sr.nq - 1) : 0, all = limit(0);
  const int klim = qi < sr.nq ? limit(qi) : 0;
  // This workgroup's tiles, of `few_tile` keys; the span counts tiles of 64.
  const int k_begin = chunk * a.span * kBN, k_end = min(keys, k_begin + a.span * kBN);
  if (chunk > 0 && k_begin >= k_end) return;  // the merge does not look at it
  const int t_end = (k_end + KBT - 1) / KBT;

  const SwzCopy<D, false> kc(a.k_tok, lane);
  const SwzCopy<D, true> vc(a.v_tok, lane);
  const __bf16* kbase = a.k + (size_t)sr.k0 * a.k_tok + kv * D;
  const __bf16* vbase = a.v + (size_t)sr.k0 * a.v_tok + kv * D;
  VC_LDS char* ring = (VC_LDS char*)smem + w * RING;
  auto copy_k = [&](int t) {
#pragma unroll
    for (int j = 0; j < COPIES; ++j) {
      const int first = swz_copy_row<D, false>(t * KBT, sr.nk, j);
      copy16_to_lds_opaque(kbase + (size_t)first * a.k_tok, kc.offset(first, sr.nk, a.k_tok), ring + j * Rows::GS);
    }
  };
  auto copy_v = [&](int t) {
#pragma unroll
    for (int j = 0; j < COPIES; ++j) {
      const int first = swz_copy_row<D, true>(t * KBT, sr.nk, j);
      copy16_to_lds_opaque(vbase + (size_t)first * a.v_tok, vc.offset(first, sr.nk, a.v_tok), ring + KT + j * Rows::GS);
    }
  };
  int t = k_begin / KBT + w;
  if (t < t_end) {
    copy_k(t);
    copy_v(t);
  }
  bf16x8 qf[D / 16];
  {
    const __bf16* qp = a.q + (size_t)query_row(a, sr, qi) * a.q_tok + h * D + 8 * hi;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const bf16x8*)(qp + 16 * ks);
  }
  table.load(a, h0, tid, 64 * NW);
  wait_all_memory();

  f32x16 oacc[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) oacc[i] = zero_f32x16();
  float m = -INFINITY, l = 0.0f;
  const int krow = Reads::row_base(l32, hi), vtr = Reads::tr_base(lane);
  for (; t < t_end; t += NW) {
    const bool more = t + NW < t_end;
    wait_loads<COPIES>();  // the tile's keys have landed; its values may be in flight
    const int k0 = t * KBT;
    const VC_LDS char* kp = ring + krow;
    const VC_LDS char* vp = ring + KT + vtr;
    f32x16 sc[KB];
    float shift = 0.0f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) sc[kb] = zero_f32x16();
    if (BIAS) {
      const int side = bias_side(k0, k0 + KBT - 1, sr.off, sr.off + 31, a.R);
      if (side == 0) {
        const float* b = tb + kBiasPad + a.R + (k0 + 4 * hi - sr.off - l32);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[kb][r] = b[kb * 32 + 8 * (r >> 2) + (r & 3)];
      } else {
        shift = tb[kBiasPad + (side > 0 ? 2 * a.R : 0)] * a.scale_log2;
      }
    }
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
        sc[kb] = mfma32(*(const VC_LDS bf16x8*)(Reads::row_at(kp, ks) + kb * Rows::bytes(32)), qf[ks], sc[kb]);
    if (more) {
      wait_reads();
      copy_k(t + NW);
    }
    if (k0 + KBT > all || l32 >= sr.nq * a.pack) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[kb][r] = k0 + kb * 32 + acc_row(r, hi) < klim ? sc[kb][r] : -INFINITY;
    }
    bf16x8 pb[2 * KB];
    float psum = 0.0f, alpha = 1.0f;
    const float sub = shift - m;
#pragma unroll
    for (int c = 0; c < 2 * KB; ++c) pb[c] = probs8(sc[c >> 1], c & 1, a.scale_log2, sub, psum);
    const bool need = !(psum <= kSumLimit);
    if (__any(need)) {
      alpha = raise_base<KB>(sc, a.scale_log2, shift, need, m, pb, psum);
#pragma unroll
      for (int i = 0; i < D / 32; ++i) oacc[i] *= alpha;
    }
    l = fmaf(l, alpha, psum);
    if (more)
      wait_loads<COPIES>();
    else
      wait_loads<0>();
    if (k0 + KBT > sr.nk) {  // value rows past nk: zero (0 * inf is not)
#pragma unroll
      for (int j = 0; j < COPIES; ++j)
        if (k0 + perm_row(Rows::RPC * j + lane / Rows::CPR) >= sr.nk)
          *(VC_LDS bf16x8*)(ring + KT + j * Rows::GS + 16 * lane) = zero_bf16x8();
    }
#pragma unroll
    for (int c = 0; c < 2 * KB; ++c)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) oacc[db] = mfma32(Reads::tr_operand(vp, c, db), pb[c], oacc[db]);
    if (more) {
      wait_reads();
      copy_v(t + NW);
    }
  }
  // The waves' results, joined in order: O = sum_w 2^(m_w - M) O_w, l likewise.
  l = halves_sum(l);
  wait_all_memory();
  VC_LDS float* ow = (VC_LDS float*)ring + l32 * OS;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(VC_LDS f32x4*)(ow + db * 32 + 8 * j + 4 * hi) =
          f32x4{oacc[db][4 * j + 0], oacc[db][4 * j + 1], oacc[db][4 * j + 2], oacc[db][4 * j + 3]};
  if (hi == 0) {
    ml[w][l32][0] = m;
    ml[w][l32][1] = l;
  }
  __syncthreads();
  const bool split = (keys + kBN - 1) / kBN > a.span;
  for (int i = tid; i < sr.sq * a.pack * (D / 4); i += 64 * NW) {
    const int r = i / (D / 4), d = i % (D / 4) * 4;
    const int q = r / a.pack, head = h0 + r % a.pack;
    float mx = -INFINITY, sum = 0.0f;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < NW; ++j) mx = fmaxf(mx, ml[j][r][1] == 0.0f ? -INFINITY : ml[j][r][0]);
#pragma unroll
    for (int j = 0; j < NW; ++j) {
      const float lj = ml[j][r][1], wgt = lj == 0.0f ? 0.0f : fast_exp2(ml[j][r][0] - mx);
      const f32x4 x = *(const VC_LDS f32x4*)((const VC_LDS float*)((VC_LDS char*)smem + j * RING) + r * OS + d);
      sum += wgt * lj;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += lj == 0.0f ? 0.0f : wgt * x[e];
    }
    const size_t rows = (size_t)a.Tq * a.H, at = (size_t)(sr.q0 + q) * a.H + head;
    if (split) {
      *(f32x4*)(a.part + (chunk * rows + at) * D + d) = o;
      if (d == 0) {
        float* p = a.part + (size_t)a.chunks * rows * D + (chunk * rows + at) * 2;
        p[0] = mx;
        p[1] = sum;
      }
    } else {
      const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
      *(bf16x4*)(a.o + at * D + d) = bf16x4{(__bf16)(o[0] * inv), (__bf16)(o[1] * inv), (__bf16)(o[2] * inv), (__bf16)(o[3] * inv)};
      if (d == 0) a.lse[(size_t)head * a.Tq + sr.q0 + q] = sum == 0.0f ? -INFINITY : (mx + __log2f(sum)) * kLn2;
    }
  }
}

__device__ __forceinline__ float lane_value(float x, int lane) {  // lane < 64, the same for the wave
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

// O and LSE of the rows whose keys several workgroups share, from their partials in order:
// O = sum_c 2^(m_c - M) O_c / sum_c 2^(m_c - M) l_c over the chunks that hold keys (M the largest of
// their bases). One wave per (query, head): lane c weighs chunk c, then each lane sums D / 64 dims, eight
// loads in flight. Bound by the latency of its loads: 4.8 us for 16 tokens of 32 heads, D = 128.
template <int D>
__global__ __launch_bounds__(256) void packed_merge_kernel(PackedArgs a) {
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
  // The keys of the row's block of rows, as the forward counts them.
  const int row = i * a.pack + h % a.pack, b0 = row / kPackedRows * kPackedRows;
  const int last = (min(b0 + kPackedRows, sr.nq * a.pack) - 1) / a.pack;
  const int keys = b0 >= sr.nq * a.pack ? 0 : a.causal ? max(0, min(sr.nk, last + sr.off + 1)) : sr.nk;
  const int n = ((keys + kBN - 1) / kBN + a.span - 1) / a.span;
  if (n <= 1) return;  // written by its only workgroup
  const size_t rows = (size_t)a.Tq * a.H, at = (size_t)(sr.q0 + i) * a.H + h;
  const float* p = a.part + (size_t)a.chunks * rows * D + (min(lane, n - 1) * rows + at) * 2;
  const float l = lane < n ? p[1] : 0.0f, mc = l == 0.0f ? -INFINITY : p[0];
  float mx = mc;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
  const float wgt = l == 0.0f ? 0.0f : exp2f(mc - mx);
  float sum = wgt * l;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
  fe acc;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
  for (int c0 = 0; c0 < n; c0 += 8) {  // eight loads in flight
    fe o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = *(const fe*)(a.part + (min(c0 + j, n - 1) * rows + at) * D + E * lane);
#pragma unroll
    for (int j = 0; j < 8; ++j) {  // lanes from n on weigh nothing
      const float wc = lane_value(wgt, c0 + j);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += wc == 0.0f ? 0.0f : wc * o[j][e];
    }
  }
  const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
  __bf16* to = a.o + at * D + E * lane;
#pragma unroll
  for (int e = 0; e < E; ++e) to[e] = (__bf16)(acc[e] * inv);
  if (lane == 0) a.lse[(size_t)h * a.Tq + sr.q0 + i] = sum == 0.0f ? -INFINITY : (mx + log2f(sum)) * kLn2;
}

template <int D, int RMAX>
void launch(PackedArgs a, hipStream_t s) {
  const int clear = a.clear ? kClearGroups : 0, heads = a.H / a.pack;
  set_blocks(a, a.pack > 1 ? 1 : a.max_q, a.Tq);  // heads packed into a block: one block a slot
  if (a.few) {
    hipLaunchKernelGGL((packed_few_kernel<D, RMAX>), dim3(heads * a.S * a.chunks + clear), dim3(64 * kFewWaves), 0, s, a);
  } else {
    hipLaunchKernelGGL((packed_fwd_kernel<D, RMAX>), dim3(a.blocks * heads * a.chunks + clear), dim3(64 * kPackedWaves), 0, s, a);
  }
  if (a.chunks > 1) {
    const int waves = a.compact ? a.blocks * a.H * kPackedRows : a.S * a.max_q * a.H;
    hipLaunchKernelGGL(packed_merge_kernel<D>, dim3((waves + 3) / 4), dim3(256), 0, s, a);
  }
}

}  // namespace

hipError_t launch_packed_fwd(const PackedArgs& a, int head_dim, hipStream_t s) {
  const int rmax = !a.bias ? 0 : a.R <= kSmallBiasDistance ? kSmallBiasDistance : kMaxBiasDistance;
  if (head_dim == 128 && rmax == 0)
    launch<128, 0>(a, s);
  else if (head_dim == 128 && rmax == kSmallBiasDistance)
    launch<128, kSmallBiasDistance>(a, s);
  else if (head_dim == 128)
    launch<128, kMaxBiasDistance>(a, s);
  else if (rmax == 0)
    launch<64, 0>(a, s);
  else if (rmax == kSmallBiasDistance)
    launch<64, kSmallBiasDistance>(a, s);
  else
    launch<64, kMaxBiasDistance>(a, s);
  return hipGetLastError();
}

}  // namespace vcja
