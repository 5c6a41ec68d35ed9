// dg_rope.hip -- rotary positions, and appending keys and values to a paged
// cache with the rotation on the way.
//
// Pair i of a head, (x1, x2) = (x_i, x_{i + half}) or (x_2i, x_{2i + 1}), is
// turned by the angle whose cosine and sine stand in row pos[axis_i, t] of the
// tables:  y1 = RN(RN(x1 c) - RN(x2 s)),  y2 = RN(RN(x2 c) + RN(x1 s)), then
// rounded once to the output's type; the inverse takes -s, which is the
// gradient too.  A position outside the tables turns by NaN.
//
// Bound: HBM.  A thread takes a unit of 2 PV elements of a head, PV pairs
// (16-byte loads and stores), for up to HPT heads, so that the cosines and
// sines of a unit are fetched once for all of them.  Two heads: 16384 tokens x 32 x
// 128, 268 MB, 55 us, the rate of a copy; appending 8192 tokens of 32 + 8 heads to an
// e4m3 cache, 189 MB, 51 us (40 while the inputs are in the last-level cache; a
// copy of as many bytes 37; nothing is moved twice: 84 MB are counted as written, 100 as
// read).  Four heads take 134 registers, three waves a SIMD instead of four: 54 and 63 us.
#include <algorithm>

#include "dg_device.h"
#include "dg_internal.h"

namespace dg {
namespace {

template <typename T, int N>
struct alignas(N * sizeof(T) >= 16 ? 16 : N * sizeof(T)) Pack {
  T v[N];
};

__device__ __forceinline__ float widen(uint16_t x, int32_t dtype) {
  return dtype == DG_BF16 ? bf16_f32(x) : (float)__builtin_bit_cast(_Float16, x);
}
__device__ __forceinline__ float widen(float x, int32_t) { return x; }

// PAST: stored past the caches (a template: two branches of one store are made one again)
template <bool PAST, typename P>
__device__ __forceinline__ void store(void* p, const P& o) {
  if constexpr (PAST && sizeof(P) == 16) {
    typedef uint32_t v4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(v4, o), (v4*)p);
  } else *(P*)p = o;
}
template <int N, bool PAST = false>
__device__ __forceinline__ void put(float* p, const float* y, int32_t) {
  Pack<float, N> o;
#pragma unroll
  for (int e = 0; e < N; ++e) o.v[e] = y[e];
  store<PAST>(p, o);
}
template <int N, bool PAST = false>
__device__ __forceinline__ void put(uint16_t* p, const float* y, int32_t dtype) {
  Pack<uint16_t, N> o;
#pragma unroll
  for (int e = 0; e < N; ++e)
    o.v[e] = dtype == DG_BF16 ? f32_bf16(y[e]) : __builtin_bit_cast(uint16_t, (_Float16)y[e]);
  store<PAST>(p, o);
}

// y / scale cut to +-448 (a NaN stays one).  inv: 1 / scale where that is exact and
// gives the quotient's bits (a power of two), else 0.
__device__ __forceinline__ float scaled(float y, float scale, float inv) {
  const float x = inv != 0.f ? y * inv : y / scale;
  return x > 448.0f ? 448.0f : x < -448.0f ? -448.0f : x;
}

// N elements of a row of the cache at element offset `at`, e4m3 rounded once.
template <int N>
__device__ __forceinline__ void put_cache(void* base, int64_t at, const float* y, int32_t dtype, float scale,
                                          float inv) {
  if (dtype == DG_E4M3) {
    if constexpr (N == 8) {
      uint32_t w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int x = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(y[4 * h], scale, inv), scaled(y[4 * h + 1], scale, inv), 0, false);
        w[h] = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(y[4 * h + 2], scale, inv), scaled(y[4 * h + 3], scale, inv), x, true);
      }
      *(uint2*)((uint8_t*)base + at) = uint2{w[0], w[1]};
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float x = scaled(y[e], scale, inv);
        ((uint8_t*)base)[at + e] = (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xff);
      }
    }
  } else put<N>((uint16_t*)base + at, y, dtype);
}

}  // namespace

// E: the element type's storage (uint16_t, or float without a cache); PV: pairs
// per unit; HPT: heads per thread.  A head has u_rot units that turn and u_rest
// of 2 PV elements behind them (the last one shorter).  `heads` counts the head
// groups of q, then k, then v.
template <typename E, int PV, int HPT, bool PAST>
__global__ __launch_bounds__(256) void rope(RopeArgs a, int tokens, int gq, int gk, int units) {
  const int groups = gq + 2 * gk, per = groups * units;      // threads of a token
  const int u_rot = (a.half + PV - 1) / PV;
  for (int64_t first = (int64_t)blockIdx.x * tokens; first < a.T; first += (int64_t)gridDim.x * tokens)
  for (int w = threadIdx.x; w < tokens * per; w += 256) {
    const int64_t t = first + w / per;
    if (t >= a.T) break;
    const int gr = w % per / units, u = w % units;
    const bool is_q = gr < gq, is_v = gr >= gq + gk;
    // (selects: the three places are uniform, the choice is not)
    const int head0 = (is_q ? gr : is_v ? gr - gq - gk : gr - gq) * HPT;
    const int heads = is_q ? a.q.heads : a.k.heads;
    const int64_t x_head = is_q ? a.q.x_head : is_v ? a.v.x_head : a.k.x_head;
    const E* X = (const E*)(is_q ? a.q.X : is_v ? a.v.X : a.k.X) +
                 t * (is_q ? a.q.x_token : is_v ? a.v.x_token : a.k.x_token);
    int64_t at = 0;
    if (!is_q) {
      const int64_t slot = a.slots[t];
      if (slot < 0 || slot >= a.n_slots) continue;
      const uint32_t page = __umulhi(2u * (uint32_t)slot, a.page_mul) >> a.page_shift;
      at = (int64_t)page * a.page_stride + (int64_t)((uint32_t)slot - page * (uint32_t)a.page_size) * a.token_stride;
    }
    E* Y = (E*)a.q.Y + t * a.q.y_token;
    void* cache = is_v ? a.v.Y : a.k.Y;
    const float scale = is_v ? a.v_scale : a.k_scale, inv = is_v ? a.v_inv : a.k_inv;
    // where the unit's two runs of PV elements lie (adjacent pairs, and what is
    // not turned: one run of 2 PV)
    const bool turn = u < u_rot && !is_v;
    const int e0 = u < u_rot ? (a.adjacent || is_v ? 2 * PV * u : PV * u) : 2 * a.half + 2 * PV * (u - u_rot);
    const int e1 = u < u_rot && !a.adjacent && !is_v ? e0 + a.half : e0 + PV;
    const bool second = e1 < a.dim;                          // a last short unit has one run only
    Pack<E, PV> x0[HPT], x1[HPT];
#pragma unroll
    for (int n = 0; n < HPT; ++n)
      if (head0 + n < heads) {
        x0[n] = *(const Pack<E, PV>*)&X[(head0 + n) * x_head + e0];
        if (second) x1[n] = *(const Pack<E, PV>*)&X[(head0 + n) * x_head + e1];
      }
    float c[PV], s[PV];
    if (turn) {
      const int i0 = PV * u;
      bool same = a.n_axes == 1;
      if (!same) {
        // all pairs of the unit on one axis: one position
        const uint32_t x = a.axis[i0 >> 4] >> (2 * (i0 & 15));
        same = true;
#pragma unroll
        for (int e = 1; e < PV; ++e) same = same && ((x >> (2 * e)) & 3) == (x & 3);
      }
      if (same) {
        const int64_t p = a.pos[(a.n_axes == 1 ? 0 : (int64_t)((a.axis[i0 >> 4] >> (2 * (i0 & 15))) & 3) * a.T) + t];
        const bool in = p >= 0 && p < a.table_rows;
        Pack<float, PV> cc, ss;
        if (in) {
          cc = *(const Pack<float, PV>*)&a.cos_t[p * a.half + i0];
          ss = *(const Pack<float, PV>*)&a.sin_t[p * a.half + i0];
        }
#pragma unroll
        for (int e = 0; e < PV; ++e) {
          c[e] = in ? cc.v[e] : __builtin_nanf("");
          s[e] = in ? ss.v[e] : __builtin_nanf("");
        }
      } else {
#pragma unroll
        for (int e = 0; e < PV; ++e) {
          const int i = i0 + e;
          const int64_t p = a.pos[(int64_t)((a.axis[i >> 4] >> (2 * (i & 15))) & 3) * a.T + t];
          const bool in = p >= 0 && p < a.table_rows;
          c[e] = in ? a.cos_t[p * a.half + i] : __builtin_nanf("");
          s[e] = in ? a.sin_t[p * a.half + i] : __builtin_nanf("");
        }
      }
      if (a.inverse)
#pragma unroll
        for (int e = 0; e < PV; ++e) s[e] = -s[e];
    }
#pragma unroll
    for (int n = 0; n < HPT; ++n) {
      if (head0 + n >= heads) break;
      float y0[PV], y1[PV];
#pragma unroll
      for (int e = 0; e < PV; ++e) {
        y0[e] = widen(x0[n].v[e], a.in_dtype);
        y1[e] = second ? widen(x1[n].v[e], a.in_dtype) : 0.f;
      }
      if (turn && a.adjacent) {
        float z[2 * PV];
#pragma unroll
        for (int e = 0; e < PV; ++e) {
          z[e] = y0[e];
          z[PV + e] = y1[e];
        }
#pragma unroll
        for (int e = 0; e < PV; ++e) {
          const float p = z[2 * e], q = z[2 * e + 1];
          z[2 * e] = p * c[e] - q * s[e];
          z[2 * e + 1] = q * c[e] + p * s[e];
        }
#pragma unroll
        for (int e = 0; e < PV; ++e) {
          y0[e] = z[e];
          y1[e] = z[PV + e];
        }
      } else if (turn) {
#pragma unroll
        for (int e = 0; e < PV; ++e) {
          const float p = y0[e], q = y1[e];
          y0[e] = p * c[e] - q * s[e];
          y1[e] = q * c[e] + p * s[e];
        }
      }
      if (is_q) {
        E* y = Y + (head0 + n) * a.q.y_head;
        put<PV, PAST>(y + e0, y0, a.in_dtype);
        if (second) put<PV, PAST>(y + e1, y1, a.in_dtype);
      } else {
        const int64_t row = at + (head0 + n) * a.head_stride;
        put_cache<PV>(cache, row + e0, y0, a.kv_dtype, scale, inv);
        if (second) put_cache<PV>(cache, row + e1, y1, a.kv_dtype, scale, inv);
      }
    }
  }
}

namespace {

template <typename E, int PV, int HPT, bool PAST>
hipError_t launch_heads(const RopeArgs& a, hipStream_t st) {
  const int gq = (a.q.heads + HPT - 1) / HPT, gk = (a.k.heads + HPT - 1) / HPT;
  const int units = (a.half + PV - 1) / PV + (a.dim - 2 * a.half + 2 * PV - 1) / (2 * PV);
  const int64_t per = (int64_t)(gq + 2 * gk) * units;
  const int tokens = per >= 256 ? 1 : (int)(256 / per);
  const int64_t blocks = std::min<int64_t>((a.T + tokens - 1) / tokens, 1 << 20);   // (a grid's threads fit 32 bits)
  hipLaunchKernelGGL((rope<E, PV, HPT, PAST>), dim3((unsigned)blocks), dim3(256), 0, st, a, tokens, gq, gk, units);
  return hipGetLastError();
}


// An output larger than the L2s is stored past them: they keep the inputs instead.
// Inputs from memory, 16384 tokens x 32 heads x 128 bf16: 66 -> 55 us, 5.0 TB/s (with the
// loads past them too 64); the e4m3 append of 8192 tokens 54 -> 51.  Its reader finds less
// of it in the caches, which about evens out: with a product of the whole output behind it 51 -> 49
// us at 32 MB, 71 -> 70 at 64, 95 -> 99 at 96, 124 -> 121 at 128, 225 -> 222 at 256; with a
// copy 30 -> 27, 50 -> 50, 74 -> 76, 99 -> 106 and 215 -> 210.
bool past_caches(const RopeArgs& a) {
  return a.T * a.q.heads * a.dim * (a.in_dtype == DG_F32 ? 4 : 2) >= ((int64_t)32 << 20);
}

}  // namespace

// wide: every row, run and stride a whole number of 16-byte pieces
hipError_t launch_rope(const RopeArgs& a, bool wide, hipStream_t st) {
  const bool past = past_caches(a);
  if (a.in_dtype == DG_F32) {
    if (!wide) return launch_heads<float, 1, 1, false>(a, st);
    return past ? launch_heads<float, 4, 4, true>(a, st) : launch_heads<float, 4, 4, false>(a, st);
  }
  if (!wide) return launch_heads<uint16_t, 1, 1, false>(a, st);
  return past ? launch_heads<uint16_t, 8, 2, true>(a, st) : launch_heads<uint16_t, 8, 2, false>(a, st);
}

}  // namespace dg
