// dg_attn_paged.hip -- attention of a ragged batch of new tokens over a paged
// key/value cache, in the attention descriptor's order (dg_attn_paged.h):
// tiles of many rows, the join of spans' records, and the choice of kernel.
#include "dg_attn_paged.h"

namespace dg {

// One workgroup: NW waves of RW rows of one key head of one sequence, over all
// of the keys that they see (a.rec null) or over one span of them, K a block
// ahead of V in LDS.
template <int D, int KT, int NW, int RW, bool INST, bool JOINS, int TL>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(NW == 4 && TL ? 1 : 2))) void
attn_paged(PagedArgs a) {
  typedef PagedTile<D, KT, RW, INST, JOINS, TL> Tile;
  constexpr bool F16 = KT == 1, E8 = KT == 2;
  constexpr int W = Tile::W, DC = Tile::DC, QKS = Tile::QKS, NQ = Tile::NQ;
  constexpr int MC = E8 ? D / 16 : DC;                     // 16-byte pieces of a row in the cache
  constexpr int NLD = W * MC / (64 * NW);                  // K (and V) loads per wave and block, 1 KB each
  static_assert(NLD >= 1 && W * MC % (64 * NW) == 0, "whole loads per wave");
  __shared__ __attribute__((aligned(1024))) uint16_t K0[W * D];
  __shared__ __attribute__((aligned(1024))) uint16_t V0[W * D];
  __shared__ __attribute__((aligned(1024))) uint16_t K1[W * D];
  __shared__ __attribute__((aligned(1024))) uint16_t V1[W * D];
  constexpr int RPW = W / NW;                              // rows of a block that a wave loads
  __shared__ RowAddress where[4][W];
  __shared__ int spoilt[2];
  __shared__ __attribute__((aligned(16))) float joined[JOINS && TL ? NW * 64 * TL : 4];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.x % a.Hkv, span = blockIdx.y, bat = blockIdx.z;
  const Seq sq = sequence(a, bat);
  const int nrow = rows_of(a, sq);
  int tile = blockIdx.x / a.Hkv;
  const int ntile = (nrow + RW * NW - 1) / (RW * NW);
  if (nrow <= a.row_lo || nrow > a.row_hi || tile >= ntile) return;
  tile = ntile - 1 - tile;                       // the longest walks first

  const int r0 = tile * (RW * NW), tile_end = r0 + RW * NW < nrow ? r0 + RW * NW : nrow;
  // The walk for the tile's rows from .. to - 1.  False, with nothing written: a
  // value that is not finite lies where only some of them see it.
  auto walk = [&](int from, int to) {
    from = __builtin_amdgcn_readfirstlane(from);       // uniform, which the loop around hides
    to = __builtin_amdgcn_readfirstlane(to);
    const int end = visible(a, sq, (to - 1) / a.g);    // keys that some of the rows see
    const int vis_first = visible(a, sq, from / a.g);  // and that all see
    const int nb = (end + W - 1) / W;
    const int b0 = a.rec ? span * a.span_blocks : 0;
    const int b1 = a.rec && b0 + a.span_blocks < nb ? b0 + a.span_blocks : nb;
    if (span > 0 && b0 >= nb) return true;

    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));                        // (its addresses are worked out per walk: registers)
    lane &= 63;
    const int li = lane & (RW - 1), G = lane / RW, r = r0 + RW * wave + li;
    const bool valid = r >= from && r < to;
    // (rows that are not there: the first one again)
    const int rr = valid ? r : from, tok = rr / a.g, head = kvh * a.g + rr % a.g;
    const int vis = valid ? visible(a, sq, tok) : end;
    const int vis_least = __builtin_amdgcn_readfirstlane(vis);   // no row of the wave sees fewer (or none is valid)

    const int k0 = Tile::k_place(lane), v0 = Tile::v_place(lane);

    shortx8 qf[QKS];
    const uint16_t* Qr = a.Q + (int64_t)(sq.q0 + tok) * a.q_token + head * a.q_head;
#pragma unroll
    for (int k = 0; k < QKS; ++k)
      qf[k] = *(const shortx8*)&Qr[Tile::KS * k + 8 * G];

    Tile t;
    t.tl = (lds_f4*)joined + (JOINS && TL ? 64 * (TL / 4) * wave + lane : 0);
    t.start();

    // a wave loads RPW rows of a block; lane j finds row j % RPW (asked for a block
    // before its use; lanes of one row write the same)
    const int64_t Kb = (int64_t)a.K + (int64_t)kvh * a.head_stride, Vb = (int64_t)a.V + (int64_t)kvh * a.head_stride;
    const int32_t* table = a.page_table + (int64_t)bat * a.table_stride;
    const int last = end < W * b1 ? end : W * b1;        // the walk's last key, and one
    const int own_row = RPW * wave + (lane & (RPW - 1));
    Row row;
    row.start(a, W * b0 + own_row);
    auto ask = [&]() { row.ask(a, table, last); };
    auto locate = [&](int b) {
      where[b & 3][own_row] = row.locate(a, Kb, Vb);
      asm volatile("" ::: "memory");               // other lanes of the wave read it
    };
    // straight into LDS (the lane fetches the piece that belongs at its place), or
    // e4m3 into registers and from there, widened, into LDS
    u32x4 kr[E8 ? NLD : 1], vr[E8 ? NLD : 1];
    auto fetch = [&](bool v, lds_u16 dst, int b) {
      if (b >= b1) return;
#pragma unroll
      for (int i = 0; i < NLD; ++i) {
        const unsigned q = 64 * (NLD * wave + i) + lane, t = q / MC;
        if constexpr (E8) {
          (v ? vr : kr)[i] = *(const __attribute__((address_space(1))) u32x4*)((glb_bytes)(v ? where[b & 3][t].v : where[b & 3][t].k) + 16 * (q % MC));
        } else {
          const int c = (q % MC) ^ (v ? v_swz<RW, DC>(t) : k_swz<RW, DC>(t));
          __builtin_amdgcn_global_load_lds((glb_void)((glb_bytes)(v ? where[b & 3][t].v : where[b & 3][t].k) + 16 * c),
                                           (lds_void)(dst + 512 * (NLD * wave + i)), 16, 0, 0);
        }
      }
    };
    auto stash = [&](bool v, lds_u16 dst, int b) {
      if constexpr (E8) {
        if (b >= b1) return;
#pragma unroll
        for (int i = 0; i < NLD; ++i) {
          const unsigned q = 64 * (NLD * wave + i) + lane, t = q / MC, c = 2 * (q % MC);
          const int z = v ? v_swz<RW, DC>(t) : k_swz<RW, DC>(t);
          const u32x4 x = (v ? vr : kr)[i];
#pragma unroll
          for (int h = 0; h < 2; ++h)
            *(lds_x4*)&dst[8 * (t * DC + ((c + h) ^ z))] =
                u32x4{e4m3x2_bf16x2<false>(x[2 * h]), e4m3x2_bf16x2<true>(x[2 * h]), e4m3x2_bf16x2<false>(x[2 * h + 1]),
                      e4m3x2_bf16x2<true>(x[2 * h + 1])};
        }
      }
    };
    auto load_k = [&](lds_u16 K_, int base, int u) {
      return *(const lds_s8*)&K_[(base ^ (Tile::KS * (u % QKS))) + Tile::tile_key(u / QKS) * D];
    };

    // P~ is 0 where a row does not see a key, and so is 0 x V, but for an infinity
    // or a NaN: looked for in the blocks with keys that only some of the rows see
    // (a decoding step has none), and told to all waves after the next barrier.
    // (of the blocks by parity: a wave past the barrier may look at the next one).
    bool looked = false;
    auto look = [&](int b, lds_u16 V_) {
      looked = vis_first < (W * b + W < end ? W * b + W : end);
      if (!looked) return;
      uint32_t bad = 0;
#pragma unroll 4
      for (int i = 0; i < W * DC / (64 * NW); ++i)
        bad |= not_finite<F16>(*(const lds_x4*)&V_[8 * (64 * (NW * i + wave) + lane)]);
      if (__builtin_amdgcn_ballot_w64(bad != 0)) spoilt[b & 1] = 1;   // (by all lanes)
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    auto found = [&](int b) { return looked && __builtin_amdgcn_readfirstlane(*(volatile int*)&spoilt[b & 1]) != 0; };

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
    auto step = [&](int b, lds_u16 Vc, lds_u16 Vn, lds_u16 Kc, lds_u16 Kn) {
      turn();
      if (found(b - 1)) return false;
      look(b, Vc);
      if constexpr (E8) {
        stash(false, Kc, b + 2);
        stash(true, Vn, b + 1);
        locate(b + 3);
        fetch(false, Kc, b + 3);
        fetch(true, Vn, b + 2);
        ask();
      } else {
        locate(b + 2);
        fetch(false, Kc, b + 2);
        fetch(true, Vn, b + 1);
        ask();
      }
      int k1 = k0, v1 = v0;
      asm volatile("" : "+v"(k1), "+v"(v1));       // (their steps worked out per block: registers)
      t.block(a, W * b, vis, vis_least, G, Vc, v1, qf, [&](int u) { return load_k(Kn, k1, u); });
      if constexpr (JOINS) if (b + 1 - folded == a.span_blocks || b + 1 == b1) {
        t.fold(W * folded, vis);
        folded = b + 1;
      }
      return true;
    };
    spoilt[threadIdx.x & 1] = 0;
    bool whole = true;
    if (b0 < b1) {
      ask();
      locate(b0);
      fetch(false, (lds_u16)K0, b0);
      fetch(true, (lds_u16)V0, b0);
      stash(false, (lds_u16)K0, b0);
      stash(true, (lds_u16)V0, b0);
      ask();
      locate(b0 + 1);
      if constexpr (E8) {
        fetch(false, (lds_u16)K1, b0 + 1);
        stash(false, (lds_u16)K1, b0 + 1);
        fetch(true, (lds_u16)V1, b0 + 1);
        ask();
        locate(b0 + 2);
        fetch(false, (lds_u16)K0, b0 + 2);
        ask();
        turn();
      } else {
        turn();
        fetch(false, (lds_u16)K1, b0 + 1);
        ask();
      }
#pragma unroll
      for (int u = 0; u < NQ; ++u) t.score(u, load_k((lds_u16)K0, k0, u), qf[u % QKS]);
      for (int b = b0; whole && b < b1; b += 2) {
        whole = step(b, (lds_u16)V0, (lds_u16)V1, (lds_u16)K0, (lds_u16)K1);
        if (whole && b + 1 < b1) whole = step(b + 1, (lds_u16)V1, (lds_u16)V0, (lds_u16)K1, (lds_u16)K0);
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

    if (valid) leave(a, t, sq, bat, kvh, r, tok, head, vis, span, W * b0, G);
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
// wave per row and 64 columns.  The order is a chain, but not the loads: JN spans
// are on their way at once.
template <int D, bool INST>
__global__ __launch_bounds__(64) void attn_paged_join(PagedArgs a) {
  constexpr int JN = 16;
  const int lane = threadIdx.x, col = 64 * (blockIdx.x % (D / 64)) + lane;
  const int64_t id = blockIdx.x / (D / 64);
  const int Hq = a.Hkv * a.g;
  int bat, head, row = 0, r = 0;
  if (a.rec_rows) {
    if (id >= (int64_t)a.B * a.Hkv * a.rec_rows) return;
    r = (int)(id % a.rec_rows);
    const int bk = (int)(id / a.rec_rows);
    bat = bk / a.Hkv;
    head = bk % a.Hkv * a.g + r % a.g;
  } else {
    if (id >= (int64_t)a.rows * Hq) return;
    head = (int)(id % Hq);
    row = (int)(id / Hq);
    // the last sequence that starts at or before the row
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.cu_q[mid] <= row) lo = mid; else hi = mid;
    }
    bat = lo;
  }
  // the walk's own first row, brought into the batch, not the offset as it was given; so tok is below
  // rows, and tok * g in 31 bits
  const Seq sq = sequence(a, bat);
  const int tok = a.rec_rows ? r / a.g : row - sq.q0;
  const int nrow = rows_of(a, sq);
  if (nrow <= a.row_lo || nrow > a.row_hi || tok < 0 || tok * a.g >= nrow) return;
  const int vis = visible(a, sq, tok), keys = 64 * a.span_blocks;
  if (vis <= keys) return;                       // answered by the span's own workgroup
  const int n = (vis - 1) / keys + 1;            // (vis + keys may pass 31 bits)
  const float2* ml = a.rec_ml + id * a.nspan;
  const float* rec = a.rec + id * a.nspan * D + col;
  float M = 0.f, L = 0.f, T = 0.f;
  for (int s0 = 0; s0 < n; s0 += JN) {
    float o[JN];
    float2 st[JN];
#pragma unroll
    for (int j = 0; j < JN; ++j) {
      const int s = s0 + j < n ? s0 + j : n - 1;
      o[j] = rec[(int64_t)s * D];
      st[j] = ml[s];
    }
#pragma unroll
    for (int j = 0; j < JN; ++j) asm volatile("" : "+v"(o[j]), "+v"(st[j].x), "+v"(st[j].y));   // all asked for by now
#pragma unroll
    for (int j = 0; j < JN; ++j) {
      if (s0 + j >= n) continue;
      if (s0 + j == 0) {
        M = st[0].x;
        L = st[0].y;
        T = o[0];
        continue;
      }
      float ea, eb;
      join<INST>(M, st[j].x, ea, eb);
      L = __builtin_fmaf(eb, st[j].y, ea * L);
      T = __builtin_fmaf(eb, o[j], ea * T);
    }
  }
  const float y = (a.final_recip ? T * (1.0f / L) : T / L) * a.v_scale;
  const int64_t at = (int64_t)(sq.q0 + tok) * a.o_token + head * a.o_head + col;
  if (a.out_dtype == DG_F32) ((float*)a.O)[at] = y;
  else ((uint16_t*)a.O)[at] = (uint16_t)(a.out_dtype == DG_BF16 ? narrow2<false>(y, y) : narrow2<true>(y, y));
}

namespace {

template <int D, int KT, int NW, int RW, bool INST, bool JOINS, int TL>
hipError_t launch_one(const PagedArgs& a, hipStream_t st) {
  constexpr int R = NW * RW;
  const int64_t most = (int64_t)a.max_q * a.g;
  const int64_t rows = a.row_hi < most ? a.row_hi : most;
  const dim3 grid((unsigned)((rows + R - 1) / R * a.Hkv), (unsigned)(a.rec ? a.nspan : 1), (unsigned)a.B);
  hipLaunchKernelGGL((attn_paged<D, KT, NW, RW, INST, JOINS, TL>), grid, dim3(64 * NW), 0, st, a);
  return hipGetLastError();
}

// d = 128 with spans to join has no registers for 64 more of output: with eight
// waves a CU (one workgroup) 44 of them go to LDS, with four all of them.
template <int D, int KT, bool INST>
hipError_t launch_tile(const PagedArgs& a, int nw, int rw, hipStream_t st) {
  const bool joins = !a.rec && a.nspan > 1;
  if (rw == 16) {
    if (joins) return launch_one<D, KT, 4, 16, INST, true, 0>(a, st);
    return launch_one<D, KT, 4, 16, INST, false, 0>(a, st);
  }
  if (!joins) return launch_one<D, KT, 4, 32, INST, false, 0>(a, st);
  if constexpr (D == 64) return launch_one<D, KT, 4, 32, INST, true, 0>(a, st);
  else {
    // (nor for e4m3 rows on their way besides)
    if constexpr (KT != 2) {
      if (nw == 8) return launch_one<D, KT, 8, 32, INST, true, 44>(a, st);
    }
    return launch_one<D, KT, 4, 32, INST, true, 64>(a, st);
  }
}

template <int D, bool INST>
hipError_t launch_type(const PagedArgs& a, int nw, int rw, hipStream_t st) {
  if (a.kv_dtype == DG_E4M3) return launch_tile<D, 2, INST>(a, nw, rw, st);
  if (a.kv_dtype == DG_F16) return launch_tile<D, 1, INST>(a, nw, rw, st);
  return launch_tile<D, 0, INST>(a, nw, rw, st);
}

}  // namespace

hipError_t launch_attention_paged(const PagedArgs& a, int nw, int rw, hipStream_t st) {
  // (the few-row kernel walks one span)
  if (nw == 1 && (a.rec || a.nspan == 1)) return launch_attention_paged_few(a, st);
  if (a.dim == 64) return a.inst ? launch_type<64, true>(a, nw, rw, st) : launch_type<64, false>(a, nw, rw, st);
  return a.inst ? launch_type<128, true>(a, nw, rw, st) : launch_type<128, false>(a, nw, rw, st);
}

hipError_t launch_attention_paged_join(const PagedArgs& a, hipStream_t st) {
  const int64_t ids = a.rec_rows ? (int64_t)a.B * a.Hkv * a.rec_rows : (int64_t)a.rows * a.Hkv * a.g;
  const dim3 grid((unsigned)(ids * (a.dim / 64)));
  if (a.dim == 64) {
    if (a.inst) hipLaunchKernelGGL((attn_paged_join<64, true>), grid, dim3(64), 0, st, a);
    else hipLaunchKernelGGL((attn_paged_join<64, false>), grid, dim3(64), 0, st, a);
  } else {
    if (a.inst) hipLaunchKernelGGL((attn_paged_join<128, true>), grid, dim3(64), 0, st, a);
    else hipLaunchKernelGGL((attn_paged_join<128, false>), grid, dim3(64), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace dg
