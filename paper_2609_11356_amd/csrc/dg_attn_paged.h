// dg_attn_paged.h -- device pieces shared by the paged attention kernels: the
// batch's lengths, the exponential and its joins, and the state of a wave's
// rows with the steps that fix its bits.
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
// the subtraction: p_t = v_exp(fma(score_t, qk_scale, -mn)), with mn the rounded
// product of the block's largest score where that exceeds m by more than 8, else
// m; 7 VALU slots a score instead of 16.
#pragma once

#include "dg_attn_tile.h"

namespace dg {
namespace {

// What a key row that is not there reads as: past the walk's end zeros, on a
// page outside the cache NaN (in every one of the element types).
struct Fill {
  uint32_t w[2][64];
  constexpr Fill() : w() {
    for (int i = 0; i < 64; ++i) w[1][i] = ~0u;
  }
};
__device__ __attribute__((aligned(256))) const Fill kFill;

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

typedef const __attribute__((address_space(1))) char* glb_bytes;
typedef __attribute__((address_space(3))) uint16_t* lds_u16;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) shortx8 lds_s8;
typedef __attribute__((address_space(3))) u32x4 lds_x4;
typedef __attribute__((address_space(3))) floatx4 lds_f4;

// A lane's row of the walk's blocks in the cache.  Its place moves on by 64 keys
// with every block; the row's addresses in K and V, or of the constant row that
// stands for it, go into a ring in LDS, from where the lanes that load the row
// take them.  All by selects: registers that the compiler moves about at the join
// of a divergent branch would lose the lanes that were not in it.
struct RowAddress {
  int64_t k, v;
};
typedef __attribute__((address_space(3))) RowAddress* lds_rows;
struct Row {
  int key, index, rest;          // the key of the next block to ask for; its page in the table, its place there
  int page, asked;               // the answer, and the place there of the key it is for (-1: past the end)

  __device__ __forceinline__ void start(const PagedArgs& a, int first) {
    key = first;
    index = (int)(__umulhi(2u * (uint32_t)first, a.page_mul) >> a.page_shift);
    rest = first - index * a.page_size;
  }
  // asks for the next block's page number (keys from `end` on: any page's)
  __device__ __forceinline__ void ask(const PagedArgs& a, const int32_t* table, int end) {
    const bool in = key < end;
    page = table[in ? index : 0];
    asked = in ? rest : -1;
    key += 64;
    index += a.page_step;
    rest += a.page_rest;
    const bool over = rest >= a.page_size;
    rest -= over ? a.page_size : 0;
    index += over ? 1 : 0;
  }
  // the answer as addresses; offsets within a page fit 31 bits
  __device__ __forceinline__ RowAddress locate(const PagedArgs& a, int64_t kb, int64_t vb) const {
    const bool there = (uint32_t)page < (uint32_t)a.pages;
    const uint64_t w = (uint64_t)(uint32_t)page * (uint32_t)a.page_stride + (uint32_t)asked * (uint32_t)a.token_stride;
    const int64_t fill = (int64_t)(const char*)kFill.w[0], none = fill + 256;
    const bool in = asked >= 0;
    return RowAddress{in ? (there ? kb + (int64_t)w : none) : fill, in ? (there ? vb + (int64_t)w : none) : fill};
  }
};

// INST: how far above the value that is subtracted a score may lie before that
// moves.  2^8 times the largest of the types' probabilities leaves their precision
// and range as they are, and the output is rescaled about once a span, not with
// every block in which one of a wave's rows meets a new maximum.
constexpr float SLACK = 8.0f;

// The state of a wave's RW rows over transposed score tiles, as in attn_fwd_t
// (dg_attn.hip): a lane owns one row (lane % RW), G = lane / RW names its share of
// the keys, P~ stays in registers.  KT: the cache's elements, 0 bf16, 1 binary16,
// 2 e4m3 (widened exactly to bf16).  JOINS: the wave walks more than one span; then
// TL of the registers of a lane's joined output, which is touched once a span, are in LDS.
template <int D, int KT, int RW, bool INST, bool JOINS, int TL = 0>
struct PagedTile {
  static constexpr bool F16 = KT == 1;
  static constexpr int W = 64, DC = D / 8, KS = RW == 32 ? 16 : 32;   // keys per block; chunks of a row; keys per P V step
  static constexpr int NK = W / KS, NP = W * RW / 64;             // steps; scores per lane
  static constexpr int QKS = D / KS, ND = D / RW, NT = W / RW;    // head-dimension steps, O and S tiles
  static constexpr int TR = RW == 32 ? 16 : 4;                    // registers per tile
  static constexpr int NQ = NT * QKS;                             // score instructions per block
  typedef std::conditional_t<RW == 32, floatx16, floatx4> tile_t;

  float m, l, M, L;              // the span's and the row's maximum and denominator
  tile_t O[ND], Sn[NT];          // the span's output rows (transposed); the next block's scores
  static constexpr int TV = JOINS ? (ND * TR - TL) / 4 : 0;
  floatx4 T[TV ? TV : 1];        // the row's, four columns each: the last TV, and before them
  lds_f4* tl;                    // TL / 4 in LDS, 64 places apart

  // first key of score tile t relative to the lane's kmap (key_of_row)
  static constexpr __device__ int tile_key(int t) { return RW == 32 ? 32 * t : 32 * (t >> 1) + 4 * (t & 1); }
  // score register i of the lane: the key (relative to 8 G)
  static constexpr __device__ int key_of(int i) { return KS * (i >> 3) + (i & 7); }
  // the lane's place in V rows in LDS for output tile 0 (elements; tile dt: ^ RW dt;
  // key steps add constants, which leave the swizzle as it is)
  static __device__ __forceinline__ int v_place(int lane) {
    const int vi = lane & 15, vrow = (RW == 32 ? 8 * (lane >> 5) : 8 * (lane >> 4)) + (vi >> 2);
    const int vcol = (RW == 32 ? 16 * ((lane >> 4) & 1) : 0) + 4 * (vi & 3);
    return 8 * (vrow * DC + ((vcol >> 3) ^ v_swz<RW, DC>(vrow))) + (vcol & 7);
  }
  // the same in K rows for head-dimension step 0 (step k: ^ 8 (KS / 8) k; tiles add
  // tile_key D)
  static __device__ __forceinline__ int k_place(int lane) {
    const int kmap = key_of_row<RW>(lane & (RW - 1));
    return 8 * (kmap * DC + ((lane / RW) ^ k_swz<RW, DC>(kmap)));
  }

  __device__ __forceinline__ void start_span() {
    m = -__builtin_inff();
    l = 0.f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int i = 0; i < TR; ++i) O[dt][i] = 0.f;
  }
  __device__ __forceinline__ void start() {
    start_span();
    M = m;
    L = 0.f;
  }

  // the row's output, columns column(dt, c) + 4 G + 0..3
  __device__ __forceinline__ floatx4 joined(int dt, int c) const {
    const int i = dt * (TR / 4) + c;
    return i < TL / 4 ? tl[64 * i] : T[i < TL / 4 ? 0 : i - TL / 4];
  }
  __device__ __forceinline__ void set_joined(int dt, int c, floatx4 y) {
    const int i = dt * (TR / 4) + c;
    if (i < TL / 4) tl[64 * i] = y;
    else T[i < TL / 4 ? 0 : i - TL / 4] = y;
  }
  __device__ __forceinline__ floatx4 span_part(int dt, int c) const {
    return floatx4{O[dt][4 * c], O[dt][4 * c + 1], O[dt][4 * c + 2], O[dt][4 * c + 3]};
  }

  // score instruction u of a block: head-dimension step u % QKS of tile u / QKS
  __device__ __forceinline__ void score(int u, shortx8 k, shortx8 q) {
    const int t = u / QKS;
    if (u % QKS == 0)
#pragma unroll
      for (int i = 0; i < TR; ++i) Sn[t][i] = 0.f;
    mma<F16>(Sn[t], k, q);
  }

  // One key block from key kb, its scores in Sn and its V rows at V_ (the lane's
  // place v0); load_k(u) fetches the K operand of score instruction u of the block
  // after it, whose scores are left in Sn.
  //
  // The matrix instructions of a block come in one order, with the VALU's work
  // dealt out between them: in step kk the exponentials of its KS keys, and under
  // them the step's share of the next block's scores and P~ V of step kk - 1, in
  // turn.  Operands are fetched AHEAD instructions before their use.  (Left to
  // itself the compiler waits for every operand right before its instruction: 1110
  // instead of 1037 us for a chunk of 4096 tokens over 16000 keys, of 1023 over 8192
  // in tiles of 128 rows 189 instead of 151.)
  static constexpr int AHEAD = KT == 2 && RW == 32 ? 1 : 2;   // (e4m3 rows on their way leave fewer registers)
  struct Op {
    int step;                    // the step whose exponentials it runs under (NK: after the last)
    int place, of;               // its place among the step's instructions
    bool v;                      // P~ V of step - 1 (index: output tile), else a score (index: u)
    int index;
  };
  static constexpr int OPS = NQ + NK * ND;
  static constexpr __device__ Op op_at(int o) {
    constexpr int SQ = NQ / NK;
    static_assert(SQ == ND, "scores and P~ V in turn");
    if (o < SQ) return Op{0, o, SQ, false, o};
    o -= SQ;
    if (o < (NK - 1) * 2 * ND) {
      const int step = 1 + o / (2 * ND), i = o % (2 * ND);
      return Op{step, i, 2 * ND, i % 2 == 1, i % 2 == 1 ? i / 2 : step * SQ + i / 2};
    }
    o -= (NK - 1) * 2 * ND;
    return Op{NK, o, ND, true, o};
  }
  template <typename LoadK>
  __device__ __forceinline__ void block(const PagedArgs& a, int kb, int vis, int vis_least, int G, lds_u16 V_, int v0,
                                        const shortx8* qf, LoadK&& load_k) {
    shortx8 frag[AHEAD + 1];
    auto fetch_op = [&](auto o) {
      constexpr Op op = op_at(o);
      if constexpr (op.v) {
        const int at = (v0 ^ (RW * op.index)) + KS * (op.step - 1) * D;
        const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(&V_[at]));
        const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(&V_[at + 4 * D]));
        frag[o % (AHEAD + 1)] = shortx8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      } else frag[o % (AHEAD + 1)] = load_k(op.index);
    };
    static_for<0, AHEAD + 1>([&](auto o) { fetch_op(o); });
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
    const float mn = INST ? (bm > m + SLACK ? bm : m) : __builtin_fmaxf(m, bm), ms = finite_max(mn);
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
    float n8[NK], v[8];
    shortx8 pf;
    static_for<0, OPS>([&](auto o) {
      constexpr Op op = op_at(o);
      if constexpr (op.v) mma<F16>(O[op.index], frag[o % (AHEAD + 1)], pf);
      else score(op.index, frag[o % (AHEAD + 1)], qf[op.index % QKS]);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (o + AHEAD + 1 < OPS) fetch_op(std::integral_constant<int, o + AHEAD + 1>{});
      if constexpr (op.step < NK) {
        constexpr int e0 = 8 * op.place / op.of, e1 = 8 * (op.place + 1) / op.of;
#pragma unroll
        for (int e = e0; e < e1; ++e)
          v[e] = pow2<INST>(INST ? __builtin_fmaf(S[8 * op.step + e], a.qk_scale, -ms) : S[8 * op.step + e] - ms);
      }
      if constexpr (op.step < NK && op.place == op.of - 1) {
        // P~ = p narrowed, already in operand layout
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = narrow2<F16>(v[2 * e], v[2 * e + 1]);
        pf = __builtin_bit_cast(shortx8, w);
        // the perfect tree over the block's keys in order
#pragma unroll
        for (int x = 1; x < 8; x <<= 1)
#pragma unroll
          for (int e = 0; e < 8; e += 2 * x) v[e] = v[e] + v[e + x];
        n8[op.step] = v[0];
      }
      __builtin_amdgcn_sched_barrier(0);
    });
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
  }

  // The end of a span (from key `first` on): its state joins the row's.
  __device__ __forceinline__ void fold(int first, int vis) {
    static_assert(JOINS, "a wave of one span has nothing to join");
    if (first == 0) {
      M = m;
      L = l;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int c = 0; c < TR / 4; ++c) set_joined(dt, c, span_part(dt, c));
    } else {
      // (selects, no branch: a row that does not see the span keeps its state)
      const bool sees = vis > first;
      float Mn = M, ea, eb;
      join<INST>(Mn, m, ea, eb);
      M = sees ? Mn : M;
      L = sees ? __builtin_fmaf(eb, l, ea * L) : L;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int c = 0; c < TR / 4; ++c) {
          floatx4 y = joined(dt, c);
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = sees ? __builtin_fmaf(eb, O[dt][4 * c + e], ea * y[e]) : y[e];
          set_joined(dt, c, y);
        }
    }
    start_span();
  }

  // Register i of tile dt holds column RW dt + 8 (i / 4) + 4 G + i % 4 (RW 32) or
  // 16 dt + 4 G + i (RW 16).
  static constexpr __device__ int column(int dt, int c) { return RW * dt + 8 * c; }

  // The span's state as record `at`.
  __device__ __forceinline__ void record(const PagedArgs& a, int64_t at, int G) const {
    if (G == 0) a.rec_ml[at] = float2{m, l};
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int c = 0; c < TR / 4; ++c)
        *(float4*)&a.rec[at * D + column(dt, c) + 4 * G] =
            float4{O[dt][4 * c], O[dt][4 * c + 1], O[dt][4 * c + 2], O[dt][4 * c + 3]};
  }
  // The answer at element `at` of O; a row that sees nothing is zero.
  __device__ __forceinline__ void answer(const PagedArgs& a, int64_t at, int vis, int G) const {
    const float sum = JOINS ? L : l;
    const float rcp = 1.0f / sum;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int c = 0; c < TR / 4; ++c) {
        const floatx4 o = JOINS ? joined(dt, c) : span_part(dt, c);
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = a.final_recip ? o[e] * rcp : o[e] / sum;
          y[e] = vis > 0 ? x * a.v_scale : 0.f;
        }
        store4(a, at + column(dt, c) + 4 * G, y);
      }
  }
};

// A row of a tile: where its record of a span lies.
__device__ __forceinline__ int64_t record_of(const PagedArgs& a, const Seq& sq, int bat, int kvh, int r, int tok,
                                             int head, int span) {
  const int64_t row = a.rec_rows ? ((int64_t)bat * a.Hkv + kvh) * a.rec_rows + r
                                 : (int64_t)(sq.q0 + tok) * (a.Hkv * a.g) + head;
  return row * a.nspan + span;
}

// The end of a walk over span `span` from key `first` on (a.rec null: over all):
// the row's record or its answer.
template <typename Tile>
__device__ __forceinline__ void leave(const PagedArgs& a, Tile& t, const Seq& sq, int bat, int kvh, int r, int tok,
                                      int head, int vis, int span, int first, int G) {
  if (a.rec && vis > 64 * a.span_blocks) {
    if (vis > first) t.record(a, record_of(a, sq, bat, kvh, r, tok, head, span), G);
    return;
  }
  if (span > 0) return;
  t.answer(a, (int64_t)(sq.q0 + tok) * a.o_token + head * a.o_head, vis, G);
}

// 16 bytes with an infinity or a NaN among their 8 elements: bit 15 or 31 set in
// the result.
template <bool F16>
__device__ __forceinline__ uint32_t not_finite(u32x4 x) {
  uint32_t bad = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) bad |= (x[e] & 0x7fff7fffu) + (F16 ? 0x04000400u : 0x00800080u);
  return bad & 0x80008000u;
}

}  // namespace
}  // namespace dg
