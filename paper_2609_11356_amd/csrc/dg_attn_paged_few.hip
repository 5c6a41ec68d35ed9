// dg_attn_paged_few.hip -- paged attention (dg_attn_paged.h) for sequences of at
// most 16 rows per key head: a decoding step, a few drafted tokens.
//
// Bound: HBM, each key and value read once, so what counts is the bytes in
// flight.  One wave per workgroup takes one span of one key head and needs no
// barrier; its K rows go straight from memory into registers in the score
// instruction's operand layout, one block ahead and one more on the way; its V
// rows, which have to be transposed, into LDS (16-bit elements directly, e4m3
// through registers, widened), a block ahead.  So four (e4m3: eight) waves
// fit a CU, each with a block of K and V in flight.
#include "dg_attn_paged.h"

namespace dg {

template <int D, int KT, bool INST>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(KT == 2 && (INST || D == 64) ? 2 : 1))) void
attn_paged_few(PagedArgs a) {
  typedef PagedTile<D, KT, 16, INST, false> Tile;
  constexpr bool F16 = KT == 1, E8 = KT == 2;
  constexpr int W = Tile::W, DC = Tile::DC, QKS = Tile::QKS, NQ = Tile::NQ, NT = Tile::NT;
  constexpr int MC = E8 ? D / 16 : DC;                     // 16-byte pieces of a row in the cache
  constexpr int NLD = W * MC / 64;                         // loads of a V block, 1 KB each
  typedef std::conditional_t<E8, u32x2, shortx8> k_t;      // 8 elements of a K row
  __shared__ __attribute__((aligned(1024))) uint16_t V0[W * D];
  __shared__ __attribute__((aligned(1024))) uint16_t V1[E8 ? 8 : W * D];
  __shared__ RowAddress where[4][W];

  // `near` key heads of a span go to one XCD (workgroup i runs on XCD i % 8), one after
  // the other.  The spans' order turns from sequence to sequence, so that short ones
  // load all XCDs.
  const uint32_t near = a.near, sets = (uint32_t)a.Hkv / near, turn = blockIdx.x / 8;
  const uint32_t set = blockIdx.x % 8 + 8 * (turn / near), group = set / sets, spans = a.rec ? a.nspan : 1;
  const int kvh = (int)(near * (set % sets) + turn % near), bat = (int)(group / spans);
  const int span = (int)((near > 1 ? group + 3u * bat : group) % spans);
  if (bat >= a.B) return;
  const Seq sq = sequence(a, bat);
  const int nrow = rows_of(a, sq);
  if (nrow <= a.row_lo || nrow > a.row_hi || nrow > 16) return;

  // The walk for the rows from .. to - 1 (see attn_paged).
  auto walk = [&](int from, int to) {
    from = __builtin_amdgcn_readfirstlane(from);       // uniform, which the loop around hides
    to = __builtin_amdgcn_readfirstlane(to);
    const int end = visible(a, sq, (to - 1) / a.g);    // keys that some of the rows see
    const int vis_first = visible(a, sq, from / a.g);  // and that all see
    const int nb = (end + W - 1) / W;
    const int b0 = a.rec ? span * a.span_blocks : 0;
    const int b1 = a.rec && b0 + a.span_blocks < nb ? b0 + a.span_blocks : nb;
    if (span > 0 && b0 >= nb) return true;

    int lane = threadIdx.x;
    asm volatile("" : "+v"(lane));                      // (its addresses are worked out per walk: registers)
    lane &= 63;
    const int li = lane & 15, G = lane >> 4;
    // lane j finds where row j of a block lies
    const int64_t Kb = (int64_t)a.K + (int64_t)kvh * a.head_stride, Vb = (int64_t)a.V + (int64_t)kvh * a.head_stride;
    const int32_t* table = a.page_table + (int64_t)bat * a.table_stride;
    const int last = end < W * b1 ? end : W * b1;      // the walk's last key, and one
    Row row;
    row.start(a, W * b0 + lane);
    auto ask = [&]() { row.ask(a, table, last); };
    auto locate = [&](int b, const Row& rw) {
      where[b & 3][lane] = rw.locate(a, Kb, Vb);
      asm volatile("" ::: "memory");             // other lanes read it
    };
    Row row0, row1;                              // the first two blocks' answers
    if (b0 < b1) {
      ask();
      row0 = row;
      ask();
      row1 = row;
      ask();
    }

    const int r = li;
    const bool valid = r >= from && r < to;
    // (rows that are not there: the first one again)
    const int rr = valid ? r : from, tok = rr / a.g, head = kvh * a.g + rr % a.g;
    const int vis = valid ? visible(a, sq, tok) : end;
    shortx8 qf[QKS];
    const uint16_t* Qr = a.Q + (int64_t)(sq.q0 + tok) * a.q_token + head * a.q_head;
#pragma unroll
    for (int k = 0; k < QKS; ++k)
      qf[k] = *(const shortx8*)&Qr[32 * k + 8 * G];

    const int kmap = key_of_row<16>(li);
    const int v0 = Tile::v_place(lane);

    Tile tile;
    tile.start();
    k_t kA[NQ], kB[NQ];
    u32x4 vr[E8 ? NLD : 1];
    auto fetch_k = [&](k_t* kk, int b) {
      if (b >= b1) return;
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        glb_bytes p = (glb_bytes)where[b & 3][kmap + Tile::tile_key(x)].k + G * sizeof(k_t);
#pragma unroll
        for (int k = 0; k < QKS; ++k) kk[QKS * x + k] = *(const __attribute__((address_space(1))) k_t*)(p + 4 * k * sizeof(k_t));
      }
    };
    auto fetch_v = [&](lds_u16 dst, int b) {
      if (b >= b1) return;
#pragma unroll
      for (int i = 0; i < NLD; ++i) {
        const unsigned q = 64 * i + lane, t = q / MC;
        glb_bytes p = (glb_bytes)where[b & 3][t].v;
        if constexpr (E8) vr[i] = *(const __attribute__((address_space(1))) u32x4*)(p + 16 * (q % MC));
        else
          __builtin_amdgcn_global_load_lds((glb_void)(p + 16 * ((q % MC) ^ v_swz<16, DC>(t))),
                                           (lds_void)(dst + 512 * i), 16, 0, 0);
      }
    };
    auto stash_v = [&]() {
      if constexpr (E8) {
#pragma unroll
        for (int i = 0; i < NLD; ++i) {
          const unsigned q = 64 * i + lane, t = q / MC, c = 2 * (q % MC);
          const u32x4 x = vr[i];
#pragma unroll
          for (int h = 0; h < 2; ++h)
            *(u32x4*)&V0[8 * (t * DC + ((c + h) ^ v_swz<16, DC>(t)))] =
                u32x4{e4m3x2_bf16x2<false>(x[2 * h]), e4m3x2_bf16x2<true>(x[2 * h]),
                      e4m3x2_bf16x2<false>(x[2 * h + 1]), e4m3x2_bf16x2<true>(x[2 * h + 1])};
        }
      }
    };
    auto load_k = [&](const k_t* kk, int u) {
      if constexpr (E8) {
        const u32x4 w = {e4m3x2_bf16x2<false>(kk[u][0]), e4m3x2_bf16x2<true>(kk[u][0]), e4m3x2_bf16x2<false>(kk[u][1]),
                         e4m3x2_bf16x2<true>(kk[u][1])};
        return __builtin_bit_cast(shortx8, w);
      } else return kk[u];
    };
    // block b: its K rows were in kc, the next block's are in kn
    auto step = [&](int b, lds_u16 Vc, lds_u16 Vn, k_t* kc, const k_t* kn) {
      if constexpr (E8) stash_v();
      else __builtin_amdgcn_s_waitcnt(vmcnt_only(0));
      asm volatile("" ::: "memory");
      locate(b + 2, row);
      fetch_k(kc, b + 2);
      fetch_v(Vn, b + 1);
      ask();
      if (vis_first < (W * b + W < end ? W * b + W : end)) {
        // keys that only some of the rows see: no infinity or NaN among their values?
        uint32_t bad = 0;
#pragma unroll 4
        for (int i = 0; i < W * DC / 64; ++i) bad |= not_finite<F16>(*(const lds_x4*)&Vc[8 * (64 * i + lane)]);
        if (__builtin_amdgcn_ballot_w64(bad != 0)) return false;
      }
      int v1 = v0;
      asm volatile("" : "+v"(v1));               // (its steps worked out per block: registers)
      tile.block(a, W * b, vis, vis_first, G, Vc, v1, qf, [&](int u) { return load_k(kn, u); });
      return true;
    };
    bool whole = true;
    if (b0 < b1) {
      locate(b0, row0);
      fetch_k(kA, b0);
      fetch_v((lds_u16)V0, b0);
      locate(b0 + 1, row1);
      fetch_k(kB, b0 + 1);
#pragma unroll
      for (int u = 0; u < NQ; ++u) tile.score(u, load_k(kA, u), qf[u % QKS]);
      for (int b = b0; whole && b < b1; b += 2) {
        whole = step(b, (lds_u16)V0, E8 ? (lds_u16)V0 : (lds_u16)V1, kA, kB);
        if (whole && b + 1 < b1) whole = step(b + 1, E8 ? (lds_u16)V0 : (lds_u16)V1, (lds_u16)V0, kB, kA);
      }
      if (!whole) {
        if constexpr (!E8) __builtin_amdgcn_s_waitcnt(vmcnt_only(0));   // before the buffers' next use
        return false;
      }
    }
    if (valid) leave(a, tile, sq, bat, kvh, r, tok, head, vis, span, W * b0, G);
    return true;
  };

  // rows of several tokens, whole or, where they hold such values, a token at a time
  for (int from = 0, to = nrow;;) {
    if (!walk(from, to)) {
      to = (from / a.g + 1) * a.g < nrow ? (from / a.g + 1) * a.g : nrow;
      continue;
    }
    if (to == nrow) break;
    from = to;
    to = to + a.g < nrow ? to + a.g : nrow;
  }
}

namespace {

// Key heads of one span that go to one XCD.  A token's heads lie side by side in most
// caches, and memory is read the faster the nearer in time its neighbours are: where
// there is work for some rounds of the chip, up to 1 KB of heads of at most 128
// bytes (128 sequences of 1000 to 16000 keys, 8 heads of 128 e4m3 bytes: 1 head 522
// us, 2 497, 4 478, 8 437), or 512 bytes of larger ones (64 of 200 to 8000, 256 bytes: 1
// head 218 us, 2 or more 209; 4 of 60000 to 131072: 281, 282 and, by 4, 287).  Less
// work takes the XCDs in turn, which loads them more evenly (32 sequences of 300 to
// 4500 keys: 17 us, near by 20).  From 4096 workgroups on near is the faster one for every
// type and size (128-byte e4m3, 8 heads of 500 to 8000 keys: 32 sequences 71 us, near 64, 128
// 274 and 228; 256-byte bf16 130 and 126, 465 and 439); at 2048 it is either (bf16 of 128
// bytes 38.3 and 39.7, e4m3 48.0 and 39.2).
int near_heads(const PagedArgs& a, int64_t spans) {
  const int64_t piece = a.dim * (a.kv_dtype == DG_E4M3 ? 1 : 2), most = piece <= 128 ? 1024 : 512;
  int n = 1;
  if (spans * a.B * a.Hkv >= 4096)
    while (a.Hkv % (2 * n) == 0 && 2 * n * piece <= most) n *= 2;
  return n;
}

template <int D, int KT, bool INST>
hipError_t launch_few(PagedArgs a, hipStream_t st) {
  const int64_t spans = a.rec ? a.nspan : 1;
  a.near = near_heads(a, spans);
  const int64_t sets = spans * a.B * (a.Hkv / a.near);
  const dim3 grid((unsigned)((sets + 7) / 8 * 8 * a.near));
  hipLaunchKernelGGL((attn_paged_few<D, KT, INST>), grid, dim3(64), 0, st, a);
  return hipGetLastError();
}

template <int D, bool INST>
hipError_t launch_few_type(const PagedArgs& a, hipStream_t st) {
  if (a.kv_dtype == DG_E4M3) return launch_few<D, 2, INST>(a, st);
  if (a.kv_dtype == DG_F16) return launch_few<D, 1, INST>(a, st);
  return launch_few<D, 0, INST>(a, st);
}

}  // namespace

hipError_t launch_attention_paged_few(const PagedArgs& a, hipStream_t st) {
  if (a.dim == 64) return a.inst ? launch_few_type<64, true>(a, st) : launch_few_type<64, false>(a, st);
  return a.inst ? launch_few_type<128, true>(a, st) : launch_few_type<128, false>(a, st);
}

}  // namespace dg
