// dg_attn_paged.hip -- attention of a ragged batch of new tokens over a paged
// key/value cache, in the attention descriptor's order.
//
// Of every sequence the keys are walked in blocks of 64 from key 0, in spans
// of split_keys keys.  A span starts from m = -inf, l = +0, O = +0 and is
// walked as dg_attn.hip walks a head (a key that a query does not see drops
// out); then its state joins the row's: for span 0 (M, L, T) = (m, l, O), for
// a later one that the row sees
//   mn = max(M, m);  a = exp2(M - mn);  b = exp2(m - mn);
//   L = fma(b, l, RN(a L));  T = fma(b, O, RN(a T));  M = mn
// and the answer is T / L (or T * (1 / L)) times v_scale.  So the bits of a
// row depend on its query, the keys that it sees and the descriptor; how the
// rows are tiled, and whether one workgroup walks all the spans of a row or
// each span has its own, is free.
//
// The rows of one key head are its (token, query head) pairs, tokens first: a
// tile of RW rows shares the K and V tiles, so a decoding step reads the cache
// once for all the query heads of a key head.
//
// exp2 "inst" (INST) takes the part's own exponential and joins the scale to
// the subtraction: p_t = v_exp(fma(score_t, qk_scale, -mn)), mn the rounded
// product of the largest score; 7 VALU slots a score instead of 16.
#include "dg_attn_tile.h"

namespace dg {
namespace {

// What a key row that is not there reads as: past the walk's end zeros, on a
// page outside the cache NaN (in every one of the element types).
__device__ __attribute__((aligned(16))) const uint32_t kFill[8] = {0u, 0u, 0u, 0u, ~0u, ~0u, ~0u, ~0u};

typedef const __attribute__((address_space(1))) void* glb_void;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <bool F16>
__device__ __forceinline__ void mma(floatx16& c, const shortx8& a, const shortx8& b) {
  if constexpr (F16)
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else mfma_to(c, a, b);
}
template <bool F16>
__device__ __forceinline__ void mma(floatx4& c, const shortx8& a, const shortx8& b) {
  if constexpr (F16)
    c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else mfma_to(c, a, b);
}

// Two binary32 values rounded to the probabilities' type.
template <bool F16>
__device__ __forceinline__ uint32_t narrow2(float lo, float hi) {
  if constexpr (F16) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, h2{(_Float16)lo, (_Float16)hi});
  } else return f32x2_bf16x2(lo, hi);
}

// 2^x for x <= 0 (INST: up to a rounding above), -inf or NaN.
template <bool INST>
__device__ __forceinline__ float pow2(float x) {
  if constexpr (INST) return __builtin_amdgcn_exp2f(x);
  else return exp2_nonpos(x);
}

// The maximum to subtract: a row that has seen nothing but -inf stays at zero
// probability instead of -inf - -inf.
__device__ __forceinline__ float finite_max(float m) { return m == -__builtin_inff() ? 0.f : m; }

// The factors that join a later span's state (m) to the row's (M).
template <bool INST>
__device__ __forceinline__ void join(float& M, float m, float& ea, float& eb) {
  const float mn = __builtin_fmaxf(M, m), ms = finite_max(mn);
  ea = pow2<INST>(M - ms);
  eb = pow2<INST>(m - ms);
  M = mn;
}

// A sequence of the batch, every length brought into the bounds of the buffers.
struct Seq {
  int q0, qlen, kv;
};
__device__ __forceinline__ Seq sequence(const PagedArgs& a, int b) {
  int q0 = a.cu_q[b], q1 = a.cu_q[b + 1], kv = a.kv_len[b];
  q0 = q0 < 0 ? 0 : q0 > a.rows ? a.rows : q0;
  q1 = q1 < q0 ? q0 : q1 > a.rows ? a.rows : q1;
  kv = kv < 0 ? 0 : kv > a.kv_cap ? a.kv_cap : kv;
  return Seq{q0, q1 - q0, kv};
}
// Its rows of one key head; new tokens past max_q are left out.
__device__ __forceinline__ int rows_of(const PagedArgs& a, const Seq& s) {
  return (s.qlen < a.max_q ? s.qlen : a.max_q) * a.g;
}
// The keys that new token j of the sequence sees: 0 .. the result - 1.
__device__ __forceinline__ int visible(const PagedArgs& a, const Seq& s, int j) {
  if (!a.causal) return s.kv;
  const int n = s.kv - s.qlen + j + 1;
  return n < 0 ? 0 : n;
}

__device__ __forceinline__ void store4(const PagedArgs& a, int64_t at, const float* y) {
  if (a.out_dtype == DG_F32) *(float4*)&((float*)a.O)[at] = float4{y[0], y[1], y[2], y[3]};
  else if (a.out_dtype == DG_BF16) *(uint2*)&((uint16_t*)a.O)[at] = uint2{narrow2<false>(y[0], y[1]), narrow2<false>(y[2], y[3])};
  else *(uint2*)&((uint16_t*)a.O)[at] = uint2{narrow2<true>(y[0], y[1]), narrow2<true>(y[2], y[3])};
}

}  // namespace

// One workgroup: NW waves of RW rows of one key head of one sequence, over all
// of the keys that they see (a.rec null) or over one span of them.  Transposed
// score tiles as in attn_fwd_t (dg_attn.hip): a lane owns one row, P~ stays in
// registers, K a block ahead of V.  KT: the cache's elements, 0 bf16, 1
// binary16, 2 e4m3 (widened exactly to bf16 on the way into LDS).
template <int D, int KT, int NW, int RW, bool INST>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW == 1 ? 1 : 2))) void
attn_paged(PagedArgs a) {
  constexpr bool F16 = KT == 1, E8 = KT == 2;
  constexpr int W = 64;
  constexpr int DC = D / 8, KS = RW == 32 ? 16 : 32;       // chunks of a row; keys per P V step
  constexpr int NK = W / KS, NP = W * RW / 64;             // steps; scores per lane
  constexpr int QKS = D / KS, ND = D / RW, NT = W / RW;    // head-dimension steps, O and S tiles
  constexpr int TR = RW == 32 ? 16 : 4;                    // registers per tile
  constexpr int NQ = NT * QKS;                             // score instructions per block
  constexpr int MC = E8 ? D / 16 : DC;                     // 16-byte pieces of a row in the cache
  constexpr int NLD = W * MC / (64 * NW);                  // K (and V) loads per wave and block, 1 KB each
  static_assert(NLD >= 1 && W * MC % (64 * NW) == 0, "whole loads per wave");
  typedef std::conditional_t<RW == 32, floatx16, floatx4> tile_t;
  __shared__ __attribute__((aligned(1024))) uint16_t K0[W * D];
  __shared__ __attribute__((aligned(1024))) uint16_t V0[W * D];
  __shared__ __attribute__((aligned(1024))) uint16_t K1[W * D];
  __shared__ __attribute__((aligned(1024))) uint16_t V1[W * D];
  constexpr int RPW = W / NW;                              // rows of a block that a wave loads
  __shared__ int64_t where[4][W];
  __shared__ int spoilt[2];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & (RW - 1), G = lane / RW;
  const int kvh = blockIdx.x % a.Hkv, span = blockIdx.y, bat = blockIdx.z;
  const Seq sq = sequence(a, bat);
  const int nrow = rows_of(a, sq);
  int tile = blockIdx.x / a.Hkv;
  const int ntile = (nrow + RW * NW - 1) / (RW * NW);
  if (nrow <= a.row_lo || nrow > a.row_hi || tile >= ntile) return;
  tile = ntile - 1 - tile;                       // the longest walks first

  const int r0 = tile * (RW * NW), tile_end = r0 + RW * NW < nrow ? r0 + RW * NW : nrow;
  const int r = r0 + RW * wave + li;

  // The walk for the tile's rows from .. to - 1.  False, with nothing written: a
  // value that is not finite lies where only some of them see it.
  auto walk = [&](int from, int to) {
  const int end = visible(a, sq, (to - 1) / a.g);    // keys that some of the rows see
  const int vis_first = visible(a, sq, from / a.g);  // and that all see
  const int nb = (end + W - 1) / W;
  const int b0 = a.rec ? span * a.span_blocks : 0;
  const int b1 = a.rec && b0 + a.span_blocks < nb ? b0 + a.span_blocks : nb;
  if (span > 0 && b0 >= nb) return true;

  const bool valid = r >= from && r < to;
  const int tok = valid ? r / a.g : 0, head = kvh * a.g + (valid ? r % a.g : 0);
  const int vis = valid ? visible(a, sq, tok) : end;
  const int vis_least = __builtin_amdgcn_readfirstlane(vis);   // no row of the wave sees fewer (or none is valid)

  // the lane's fragment addresses (elements; tiles and key steps add constants,
  // which leave the swizzles as they are)
  const int kmap = key_of_row<RW>(li);
  const int vi = lane & 15, vrow = (RW == 32 ? 8 * G : 8 * (lane >> 4)) + (vi >> 2);
  const int vcol = (RW == 32 ? 16 * ((lane >> 4) & 1) : 0) + 4 * (vi & 3);
  constexpr int CPS = KS / 8;                    // chunks per head-dimension step
  int kad[QKS], vad[ND];
#pragma unroll
  for (int k = 0; k < QKS; ++k) kad[k] = 8 * (kmap * DC + ((CPS * k + G) ^ k_swz<RW, DC>(kmap)));
#pragma unroll
  for (int dt = 0; dt < ND; ++dt) vad[dt] = 8 * (vrow * DC + (((RW * dt + vcol) >> 3) ^ v_swz<RW, DC>(vrow))) + (vcol & 7);
  // first key of tile T relative to the lane's kmap
  auto tile_key = [](int T) { return RW == 32 ? 32 * T : 32 * (T >> 1) + 4 * (T & 1); };
  // score register i of the lane: the key (relative to 8 G)
  auto key_of = [](int i) { return KS * (i >> 3) + (i & 7); };

  shortx8 qf[QKS];
  const uint16_t* Qr = a.Q + (int64_t)(sq.q0 + tok) * a.q_token + head * a.q_head;
#pragma unroll
  for (int k = 0; k < QKS; ++k)
    qf[k] = valid ? *(const shortx8*)&Qr[KS * k + 8 * G] : shortx8{0, 0, 0, 0, 0, 0, 0, 0};

  float m = -__builtin_inff(), l = 0.f, M = m, L = 0.f;
  tile_t O[ND], T[ND], Sn[NT];
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int i = 0; i < TR; ++i) O[dt][i] = T[dt][i] = 0.f;

  // Where a block's rows lie.  A wave loads RPW rows of a block; lane j % RPW
  // finds row j's page (asked for a block before its use) and leaves the row's
  // byte offset in K and V, or which constant row stands for it (-1, -2), in
  // the wave's ring of four blocks in LDS.
  const char* Kb = (const char*)a.K + (int64_t)kvh * a.head_stride;
  const char* Vb = (const char*)a.V + (int64_t)kvh * a.head_stride;
  const int32_t* pages = a.page_table + (int64_t)bat * a.table_stride;
  auto page_of = [&](int key) { return (int)(((uint64_t)(uint32_t)key * a.page_mul) >> a.page_shift); };
  const int own_row = RPW * wave + (lane & (RPW - 1));
  int page = -1;
  auto ask = [&](int b) {
    const int key = W * b + own_row;
    page = b < b1 && key < end ? pages[page_of(key)] : -1;
  };
  auto locate = [&](int b) {
    const int key = W * b + own_row;
    int64_t w = -1;
    if (b < b1 && key < end)
      w = (uint32_t)page < (uint32_t)a.pages
              ? (int64_t)page * a.page_stride + (int64_t)(key - page_of(key) * a.page_size) * a.token_stride
              : -2;
    if (lane < RPW) where[b & 3][own_row] = w;
    asm volatile("" ::: "memory");               // other lanes of the wave read it
  };
  auto address = [&](const char* base, int64_t w, int c) {
    return w >= 0 ? base + w + 16 * c : (const char*)kFill + (w == -2 ? 16 : 0);
  };
  // straight into LDS (the lane fetches the piece that belongs at its place), or
  // e4m3 into registers and from there, widened, into LDS
  u32x4 kr[E8 ? NLD : 1], vr[E8 ? NLD : 1];
  auto fetch = [&](bool v, uint16_t* dst, int b) {
    if (b >= b1) return;
#pragma unroll
    for (int i = 0; i < NLD; ++i) {
      const int q = 64 * (NLD * wave + i) + lane, t = q / MC;
      if constexpr (E8) {
        (v ? vr : kr)[i] = *(const u32x4*)address(v ? Vb : Kb, where[b & 3][t], q % MC);
      } else {
        const int c = (q % MC) ^ (v ? v_swz<RW, DC>(t) : k_swz<RW, DC>(t));
        __builtin_amdgcn_global_load_lds((glb_void)address(v ? Vb : Kb, where[b & 3][t], c),
                                         (lds_void)(dst + 512 * (NLD * wave + i)), 16, 0, 0);
      }
    }
  };
  auto stash = [&](bool v, uint16_t* dst, int b) {
    if constexpr (E8) {
      if (b >= b1) return;
#pragma unroll
      for (int i = 0; i < NLD; ++i) {
        const int q = 64 * (NLD * wave + i) + lane, t = q / MC, c = 2 * (q % MC);
        const int z = v ? v_swz<RW, DC>(t) : k_swz<RW, DC>(t);
        const u32x4 x = (v ? vr : kr)[i];
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *(u32x4*)&dst[8 * (t * DC + ((c + h) ^ z))] =
              u32x4{e4m3x2_bf16x2<false>(x[2 * h]), e4m3x2_bf16x2<true>(x[2 * h]), e4m3x2_bf16x2<false>(x[2 * h + 1]),
                    e4m3x2_bf16x2<true>(x[2 * h + 1])};
      }
    }
  };
  // score instruction u of a block: head-dimension step u % QKS of tile u / QKS
  auto score = [&](const uint16_t* K_, int u) {
    const int t = u / QKS, k = u % QKS;
    if (k == 0)
#pragma unroll
      for (int i = 0; i < TR; ++i) Sn[t][i] = 0.f;
    mma<F16>(Sn[t], *(const shortx8*)&K_[kad[k] + tile_key(t) * D], qf[k]);
  };

  // One key block: its scores in Sn, its V rows in V_; the next block's K rows
  // in Kn (whose scores are left in Sn; past the last block they are not used).
  auto block = [&](int b, const uint16_t* V_, const uint16_t* Kn) {
    const int kb = W * b;
    float S[NP];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < TR; ++i) S[TR * t + i] = INST ? Sn[t][i] : Sn[t][i] * a.qk_scale;
    // keys that the row does not see drop out
    if (kb + W > vis_least) {
      const int left = vis - kb - 8 * G;
#pragma unroll
      for (int i = 0; i < NP; ++i) S[i] = key_of(i) >= left ? -__builtin_inff() : S[i];
    }
    float bm = S[0];
#pragma unroll
    for (int i = 1; i < NP; ++i) bm = __builtin_fmaxf(bm, S[i]);
    float bo = bm;
    if constexpr (RW == 16) {
      rows_swap(bm, bo);
      bm = __builtin_fmaxf(bm, bo);
      bo = bm;
    }
    halves_swap(bm, bo);
    bm = __builtin_fmaxf(bm, bo);
    if constexpr (INST) bm = bm * a.qk_scale;
    const float mn = __builtin_fmaxf(m, bm), ms = finite_max(mn);
    const float alpha = pow2<INST>(m - ms);
    m = mn;
    // rescale the output rows (skipped when every row of the wave keeps its
    // maximum: alpha = 1 and 1 x O = O exactly)
    if (__builtin_amdgcn_ballot_w64(!(alpha == 1.0f)) != 0) {
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int i = 0; i < TR; ++i) O[dt][i] = alpha * O[dt][i];
    }
    float n8[NK];
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) {
      __builtin_amdgcn_sched_barrier(0);
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        v[e] = pow2<INST>(INST ? __builtin_fmaf(S[8 * kk + e], a.qk_scale, -ms) : S[8 * kk + e] - ms);
      // P~ = p narrowed, already in operand layout
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = narrow2<F16>(v[2 * e], v[2 * e + 1]);
      const shortx8 pf = __builtin_bit_cast(shortx8, w);
      // the perfect tree over the block's keys in order
#pragma unroll
      for (int x = 1; x < 8; x <<= 1)
#pragma unroll
        for (int e = 0; e < 8; e += 2 * x) v[e] = v[e] + v[e + x];
      n8[kk] = v[0];
      // the next block's scores, then O^T = alpha O^T (+) V^T P~^T: for each
      // output the steps of KS keys in increasing order
#pragma unroll
      for (int u = kk * NQ / NK; u < (kk + 1) * NQ / NK; ++u) score(Kn, u);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(&V_[vad[dt] + KS * kk * D]));
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(&V_[vad[dt] + (KS * kk + 4) * D]));
        mma<F16>(O[dt], shortx8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}, pf);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (RW == 32) {
      // one swap turns two values spread over the halves into their two sums:
      // 2^j values -> 2^(j-1) registers (one per half), down to the root
#pragma unroll
      for (int c = NK; c > 1; c >>= 1)
#pragma unroll
        for (int e = 0; e < c / 2; ++e) {
          float x = n8[2 * e], y = n8[2 * e + 1];
          halves_swap(x, y);
          n8[e] = x + y;
        }
      float y = n8[0];
      halves_swap(n8[0], y);
      n8[0] = n8[0] + y;
    } else {
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        float y = n8[kk];
        rows_swap(n8[kk], y);
        n8[kk] = n8[kk] + y;
        y = n8[kk];
        halves_swap(n8[kk], y);
        n8[kk] = n8[kk] + y;
      }
#pragma unroll
      for (int x = 1; x < NK; x <<= 1)
#pragma unroll
        for (int kk = 0; kk < NK; kk += 2 * x) n8[kk] = n8[kk] + n8[kk + x];
    }
    l = a.l_fma ? __builtin_fmaf(alpha, l, n8[0]) : alpha * l + n8[0];
  };

  // P~ is 0 where a row does not see a key, and so is 0 x V, but for an infinity
  // or a NaN: looked for in the blocks with keys that only some of the rows see
  // (a decoding step has none), and told to all waves after the next barrier.
  // (of the blocks by parity: a wave past the barrier may look at the next one).
  bool looked = false;
  auto look = [&](int b, const uint16_t* V_) {
    looked = vis_first < (W * b + W < end ? W * b + W : end);
    if (!looked) return;
    uint32_t bad = 0;
#pragma unroll 4
    for (int i = threadIdx.x; i < W * DC; i += 64 * NW) {
      const u32x4 x = *(const u32x4*)&V_[8 * i];
#pragma unroll
      for (int e = 0; e < 4; ++e) bad |= (x[e] & 0x7fff7fffu) + (F16 ? 0x04000400u : 0x00800080u);
    }
    if (bad & 0x80008000u) spoilt[b & 1] = 1;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  auto found = [&](int b) { return looked && __builtin_amdgcn_readfirstlane(*(volatile int*)&spoilt[b & 1]) != 0; };

  // The end of a span that is not the row's last: its state joins the row's.
  auto fold = [&](int first) {
    if (first == 0) {
      M = m;
      L = l;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) T[dt] = O[dt];
    } else if (vis > W * first) {
      float ea, eb;
      join<INST>(M, m, ea, eb);
      L = __builtin_fmaf(eb, l, ea * L);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int i = 0; i < TR; ++i) T[dt][i] = __builtin_fmaf(eb, O[dt][i], ea * T[dt][i]);
    }
    m = -__builtin_inff();
    l = 0.f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int i = 0; i < TR; ++i) O[dt][i] = 0.f;
  };

  // A wave's own loads have landed once its count is zero (its LDS writes once
  // theirs is); after the barrier that follows, everybody's have, and the K
  // pair of block b and the V pair of block b - 1 are free for the loads of
  // blocks b + 2 and b + 1.
  auto turn = [&]() {
    if constexpr (E8) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    else __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
    barrier_nofence();
  };
  int folded = 0;                                // first block of the span being walked (a.rec null)
  auto step = [&](int b, uint16_t* Vc, uint16_t* Vn, uint16_t* Kc, uint16_t* Kn) {
    turn();
    if (found(b - 1)) return false;
    look(b, Vc);
    if constexpr (E8) {
      stash(false, Kc, b + 2);
      stash(true, Vn, b + 1);
      locate(b + 3);
      fetch(false, Kc, b + 3);
      fetch(true, Vn, b + 2);
      ask(b + 4);
    } else {
      locate(b + 2);
      fetch(false, Kc, b + 2);
      fetch(true, Vn, b + 1);
      ask(b + 3);
    }
    block(b, Vc, Kn);
    if (!a.rec && (b + 1 - folded == a.span_blocks || b + 1 == b1)) {
      fold(folded);
      folded = b + 1;
    }
    return true;
  };
  if (threadIdx.x < 2) spoilt[threadIdx.x] = 0;
  bool whole = true;
  if (b0 < b1) {
    ask(b0);
    locate(b0);
    fetch(false, K0, b0);
    fetch(true, V0, b0);
    stash(false, K0, b0);
    stash(true, V0, b0);
    ask(b0 + 1);
    locate(b0 + 1);
    if constexpr (E8) {
      fetch(false, K1, b0 + 1);
      stash(false, K1, b0 + 1);
      fetch(true, V1, b0 + 1);
      ask(b0 + 2);
      locate(b0 + 2);
      fetch(false, K0, b0 + 2);
      ask(b0 + 3);
      turn();
    } else {
      turn();
      fetch(false, K1, b0 + 1);
      ask(b0 + 2);
    }
#pragma unroll
    for (int u = 0; u < NQ; ++u) score(K0, u);
    for (int b = b0; whole && b < b1; b += 2) {
      whole = step(b, V0, V1, K0, K1);
      if (whole && b + 1 < b1) whole = step(b + 1, V1, V0, K1, K0);
    }
    if (looked) {
      // the last block's finding; and nobody clears it, or loads for the next
      // walk, before all waves are here
      turn();
      whole = whole && !found(b1 - 1);
      turn();
      if (!whole) return false;
    }
  }

  // the span's state as a record, or the answer; register i of tile dt holds
  // column RW dt + 8 (i / 4) + 4 G + i % 4 (RW 32) or 16 dt + 4 G + i (RW 16)
  if (!valid) return true;
  if (a.rec && vis > W * a.span_blocks) {
    if (vis <= W * b0) return true;
    const int64_t at = (a.rec_rows ? ((int64_t)bat * a.Hkv + kvh) * a.rec_rows + r
                                   : (int64_t)(sq.q0 + tok) * (a.Hkv * a.g) + head) * a.nspan + span;
    if (G == 0) a.rec_ml[at] = float2{m, l};
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int c = 0; c < TR / 4; ++c)
        *(float4*)&a.rec[at * D + RW * dt + 8 * c + 4 * G] =
            float4{O[dt][4 * c], O[dt][4 * c + 1], O[dt][4 * c + 2], O[dt][4 * c + 3]};
    return true;
  }
  if (span > 0) return true;
  if (a.rec) fold(0);
  const float rcp = 1.0f / L;
  const int64_t o = (int64_t)(sq.q0 + tok) * a.o_token + head * a.o_head;
#pragma unroll
  for (int dt = 0; dt < ND; ++dt)
#pragma unroll
    for (int c = 0; c < TR / 4; ++c) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = a.final_recip ? T[dt][4 * c + e] * rcp : T[dt][4 * c + e] / L;
        y[e] = vis > 0 ? x * a.v_scale : 0.f;    // a row that sees nothing is zero
      }
      store4(a, o + RW * dt + 8 * c + 4 * G, y);
    }
  return true;
  };

  // rows whose tile holds such values are walked a token at a time: the rows of
  // one token see the same keys
  for (int from = r0, to = tile_end;;) {
    if (!walk(from, to)) {
      to = (from / a.g + 1) * a.g < tile_end ? (from / a.g + 1) * a.g : tile_end;
      continue;
    }
    if (to == tile_end) break;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier_nofence();                           // the buffers are everybody's
    from = to;
    to = to + a.g < tile_end ? to + a.g : tile_end;
  }
}

// Joins the spans' records of the rows that have more than one, in order: one
// wave per row, D / 64 columns per lane.
template <int D, bool INST>
__global__ __launch_bounds__(256) void attn_paged_join(PagedArgs a) {
  constexpr int C = D / 64;
  typedef float cols_t __attribute__((ext_vector_type(C)));
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int Hq = a.Hkv * a.g;
  int bat, tok, head;
  if (a.rec_rows) {
    if (id >= (int64_t)a.B * a.Hkv * a.rec_rows) return;
    const int r = (int)(id % a.rec_rows), bk = (int)(id / a.rec_rows);
    bat = bk / a.Hkv;
    tok = r / a.g;
    head = bk % a.Hkv * a.g + r % a.g;
  } else {
    if (id >= (int64_t)a.rows * Hq) return;
    head = (int)(id % Hq);
    const int row = (int)(id / Hq);
    // the last sequence that starts at or before the row
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.cu_q[mid] <= row) lo = mid; else hi = mid;
    }
    bat = lo;
    tok = row - a.cu_q[bat];
  }
  const Seq sq = sequence(a, bat);
  const int nrow = rows_of(a, sq);
  if (nrow <= a.row_lo || nrow > a.row_hi || tok < 0 || tok * a.g >= nrow) return;
  const int vis = visible(a, sq, tok), keys = 64 * a.span_blocks;
  if (vis <= keys) return;                       // answered by the span's own workgroup
  const int n = (vis + keys - 1) / keys;
  const float2* ml = a.rec_ml + id * a.nspan;
  const float* rec = a.rec + id * a.nspan * D + C * lane;
  float M = ml[0].x, L = ml[0].y;
  cols_t T = *(const cols_t*)rec;
  for (int s = 1; s < n; ++s) {
    const cols_t o = *(const cols_t*)&rec[(int64_t)s * D];
    float ea, eb;
    join<INST>(M, ml[s].x, ea, eb);
    L = __builtin_fmaf(eb, ml[s].y, ea * L);
#pragma unroll
    for (int c = 0; c < C; ++c) T[c] = __builtin_fmaf(eb, o[c], ea * T[c]);
  }
  const float rcp = 1.0f / L;
  const int64_t at = (int64_t)(sq.q0 + tok) * a.o_token + head * a.o_head + C * lane;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const float y = (a.final_recip ? T[c] * rcp : T[c] / L) * a.v_scale;
    if (a.out_dtype == DG_F32) ((float*)a.O)[at + c] = y;
    else ((uint16_t*)a.O)[at + c] = (uint16_t)(a.out_dtype == DG_BF16 ? narrow2<false>(y, y) : narrow2<true>(y, y));
  }
}

namespace {

template <int D, int KT, int NW, int RW, bool INST>
hipError_t launch_one(const PagedArgs& a, hipStream_t st) {
  constexpr int R = NW * RW;
  const int64_t most = (int64_t)a.max_q * a.g;
  const int64_t rows = a.row_hi < most ? a.row_hi : most;
  const dim3 grid((unsigned)((rows + R - 1) / R * a.Hkv), (unsigned)(a.rec ? a.nspan : 1), (unsigned)a.B);
  hipLaunchKernelGGL((attn_paged<D, KT, NW, RW, INST>), grid, dim3(64 * NW), 0, st, a);
  return hipGetLastError();
}

template <int D, int KT, bool INST>
hipError_t launch_tile(const PagedArgs& a, int nw, int rw, hipStream_t st) {
  if (nw == 1) return launch_one<D, KT, 1, 16, INST>(a, st);
  return launch_one<D, KT, 4, 16, INST>(a, st);
}

template <int D, bool INST>
hipError_t launch_type(const PagedArgs& a, int nw, int rw, hipStream_t st) {
  if (a.kv_dtype == DG_E4M3) return launch_tile<D, 2, INST>(a, nw, rw, st);
  if (a.kv_dtype == DG_F16) return launch_tile<D, 1, INST>(a, nw, rw, st);
  return launch_tile<D, 0, INST>(a, nw, rw, st);
}

}  // namespace

hipError_t launch_attention_paged(const PagedArgs& a, int nw, int rw, hipStream_t st) {
  if (a.dim == 64) return a.inst ? launch_type<64, true>(a, nw, rw, st) : launch_type<64, false>(a, nw, rw, st);
  return a.inst ? launch_type<128, true>(a, nw, rw, st) : launch_type<128, false>(a, nw, rw, st);
}

hipError_t launch_attention_paged_join(const PagedArgs& a, hipStream_t st) {
  const int64_t ids = a.rec_rows ? (int64_t)a.B * a.Hkv * a.rec_rows : (int64_t)a.rows * a.Hkv * a.g;
  const dim3 grid((unsigned)((ids + 3) / 4));
  if (a.dim == 64) {
    if (a.inst) hipLaunchKernelGGL((attn_paged_join<64, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((attn_paged_join<64, false>), grid, dim3(256), 0, st, a);
  } else {
    if (a.inst) hipLaunchKernelGGL((attn_paged_join<128, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((attn_paged_join<128, false>), grid, dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace dg
