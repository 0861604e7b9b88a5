// attn_f32_loop.h - the key loop of float32 attention (attn_f32.hip describes
// it): the three-plane products, the tile configuration, and one pass over a
// wave's or workgroup's key tiles, whatever rows the keys lie in.
#pragma once

#include <type_traits>

#include "attn_tile.h"
#include "wide_range.h"

namespace ditango {
namespace {

__device__ __forceinline__ f32x16 mfma32f(float a, float b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// three bf16 planes of 8 floats
struct Planes {
  bf16x8 p[3];
};
// Pairs of values: one conversion instruction packs a pair's plane, and the
// values it stands for are read back out of the packed word (the empty asm
// hides from the compiler that they are conversions, which it would repeat
// value by value).
__device__ __forceinline__ Planes split8(f32x8 x) {
  u32x4 w[3];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      uint32_t p = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
      if (j < 2) {
        asm("" : "+v"(p));
        a -= __builtin_bit_cast(float, p << 16);
        b -= __builtin_bit_cast(float, p & 0xffff0000u);
      }
      w[j][i] = p;
    }
  }
  Planes r;
#pragma unroll
  for (int j = 0; j < 3; ++j) r.p[j] = __builtin_bit_cast(bf16x8, w[j]);
  return r;
}

// 2^-110: nonzero values below it are not exact in the planes
constexpr uint32_t kPlanesMin = 0x08800000u;
__device__ __forceinline__ bool below_planes(float x) {
  return (__float_as_uint(x) & 0x7fffffffu) - 1u < kPlanesMin - 1u;
}

// the six plane products, smallest first
constexpr int kTerms = 6;
constexpr int kTermA[kTerms] = {2, 1, 0, 1, 0, 0};
constexpr int kTermB[kTerms] = {0, 1, 2, 0, 1, 0};

template <int D_, int RW_, int KW_, int WPE_, bool PIPED_>
struct CfgF {
  static constexpr int D = D_, RW = RW_, KW = KW_, WPE = WPE_;
  static constexpr bool PIPED = PIPED_;
  static constexpr int BN = 32;                   // keys per tile
  static constexpr int NT = RW * KW * 64;
  static constexpr int BM = RW * 32;              // query rows per workgroup
  static constexpr int KS = D / 16;               // bf16 MFMA k-steps over the head dim
  static constexpr int DB = D / 32;
  static constexpr int UNITS = D / 8;             // 8-element units per row
  static constexpr int ROWB = D * 2;              // bytes per plane row
  static constexpr int PLANE = BN * ROWB;
  static constexpr int TILE = 3 * PLANE;          // one operand's tile
  static constexpr int KST = D + 1;               // float rows of the float32 form
  static constexpr int VST = D + 8;
  // K and V take turns in one buffer when a wave has it to itself
  static constexpr int GROUP = RW == 1 ? TILE : 4 * TILE;
  static constexpr int UT = BN * UNITS / (RW * 64);   // units per thread and tile
  static constexpr int LDS = KW * GROUP + KW * 64 * 4 + 16;
  static_assert(RW == 1 || KW == 1, "waves share a tile or split the keys");
  static_assert(BN * VST * 4 <= TILE, "float rows fit the planes' space");
  static_assert(BN * UNITS % (RW * 64) == 0, "units divide over the threads");
  static_assert(BM * D * 4 <= TILE || KW == 1, "partial output fits the wave's space");
  static_assert(LDS <= 163840, "LDS of one compute unit");
};

// Where the keys' rows lie: at a fixed distance, or at the places a list gives
// (elements of the row and of the list are read only below the key count).
struct StridedRows {
  static constexpr bool kListed = false;
  const float* base;
  int64_t stride;             // elements
  __device__ __forceinline__ const float* row(int key) const { return base + key * stride; }
};
struct ListedRows {
  static constexpr bool kListed = true;
  const float* base;
  int64_t stride;
  const int* list;
  __device__ __forceinline__ const float* row(int key) const { return base + list[key] * stride; }
};

// One pass over this wave's (KW > 1) or workgroup's (KW = 1) key tiles
// [t0, t1): unnormalised O^T, row maximum m (base 2, scaled) and the lane's
// half of the row sum.  SPLIT: bf16 planes, otherwise the float32 MFMA, which
// takes the probabilities as 2^low exp2(scale (s - max)) against the maximum as
// it is (wide_range.h; low 0 but for rows out of range).
// `ask`: the lanes whose query values need the latter.
template <class C, bool SPLIT, class Rows>
__device__ __forceinline__ void key_loop(const float* __restrict__ qrow, bool row_ok, const Rows& kg,
                                         const Rows& vg, int kv_len, int t0, int t1,
                                         float sl2, unsigned char* buf, int gt, f32x16 (&o)[C::DB],
                                         float& m, float& l, uint64_t& ask, float low = 0.f) {
  constexpr int D = C::D;
  const int lane = threadIdx.x & 63;
  const int lr = lane & 31;
  const int g = lane >> 5;
#pragma unroll
  for (int db = 0; db < C::DB; ++db) o[db] = f32x16{};
  m = -INFINITY;
  l = 0.f;
  if (t0 >= t1) return;

  Planes qp[SPLIT ? C::KS : 1];
  float qf[SPLIT ? 1 : D / 2];
  if constexpr (SPLIT) {
#pragma unroll
    for (int s = 0; s < C::KS; ++s) {
      const f32x4 x0 = *(const f32x4*)(qrow + 16 * s + 8 * g), x1 = *(const f32x4*)(qrow + 16 * s + 8 * g + 4);
      f32x8 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = row_ok ? x0[e] : 0.f;
        x[4 + e] = row_ok ? x1[e] : 0.f;
      }
      // smallest nonzero and largest magnitude (as bits; 0 - 1 is the largest)
      uint32_t lo = ~0u, hi = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t u = __float_as_uint(x[e]) & 0x7fffffffu;
        lo = min(lo, u - 1u);
        hi = max(hi, u);
      }
      ask |= __builtin_amdgcn_ballot_w64(lo < kPlanesMin - 1u || __uint_as_float(hi) * sl2 >= 0x1p100f);
      qp[s] = split8(x);
    }
  } else {
#pragma unroll
    for (int s = 0; s < D / 2; ++s) qf[s] = row_ok ? qrow[2 * s + g] : 0.f;
  }

  // this thread's units of a tile: unit u = gt + i * RW * 64, key u / UNITS.
  // Rows past the end read the last key: their scores are masked, and in the
  // float32 form (whose operands may be infinite) they are staged as zeros.
  // A lane's byte offset from the tile's first row is the same for every
  // tile but for that clamp; the tile's base is wave-uniform.
  struct Stage {
    f32x4 x[C::UT][2];
  };
  const int last_tile = (kv_len - 1) / C::BN;
  auto load = [&](Stage& st, const Rows& src, int tile) {
    const int tb = min(tile, last_tile);
    const int lim = min(kv_len - 1 - tb * C::BN, C::BN - 1);
    const uint32_t row_bytes = (uint32_t)src.stride * 4;
    const char* base = (const char*)(src.base + (int64_t)tb * C::BN * src.stride);
#pragma unroll
    for (int i = 0; i < C::UT; ++i) {
      const int key = (gt + i * C::RW * 64) / C::UNITS;
      const uint32_t at = (uint32_t)((gt + i * C::RW * 64) % C::UNITS) * 32;
      const char* p;
      if constexpr (Rows::kListed)
        p = (const char*)src.row(tb * C::BN + min(key, lim)) + at;
      else
        p = base + (min((uint32_t)key * row_bytes, (uint32_t)lim * row_bytes) + at);
      st.x[i][0] = *(const f32x4*)p;
      st.x[i][1] = *(const f32x4*)(p + 16);
    }
  };
  auto store = [&](const Stage& st, unsigned char* buf, int tile, bool is_k) {
#pragma unroll
    for (int i = 0; i < C::UT; ++i) {
      const int u = gt + i * C::RW * 64;
      const int key = u / C::UNITS, c = u % C::UNITS;
      f32x8 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = st.x[i][0][e];
        x[4 + e] = st.x[i][1][e];
      }
      if constexpr (SPLIT) {
        const Planes pl = split8(x);
        unsigned char* p = buf + key * C::ROWB + (c ^ (is_k ? swz_k<D>(key) : swz_v<D>(key))) * 16;
#pragma unroll
        for (int j = 0; j < 3; ++j) *(bf16x8*)(p + j * C::PLANE) = pl.p[j];
      } else {
        float* p = (float*)buf + key * (is_k ? C::KST : C::VST) + c * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = tile * C::BN + key < kv_len ? x[e] : 0.f;
      }
    }
  };

  // V^T fragments by transpose reads, as in the bf16 kernel: source lane r of
  // a 16-lane group points at row 4g + r/4 (+ 16s + 8) and dims
  // 32db + 16*(group%2) + 4*(r%4)
  const int vrow = 4 * g + ((lane & 15) >> 2);
  const int vdim = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  uint32_t voff[C::DB];
#pragma unroll
  for (int db = 0; db < C::DB; ++db) {
    const int dim = 32 * db + vdim;
    voff[db] = vrow * C::ROWB + ((dim >> 3) ^ swz_v<D>(vrow)) * 16 + (dim & 7) * 2;
  }
  auto v_frag = [&](const unsigned char* vb, int plane, int s, int db) {
    const unsigned char* p = vb + plane * C::PLANE + 16 * s * C::ROWB + voff[db];
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, p)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, p + 8 * C::ROWB)));
    return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
  };

  // S^T = K Q^T of the tile in kb
  auto qk = [&](const unsigned char* kb, f32x16& sc) {
    sc = f32x16{};
    if constexpr (SPLIT) {
      f32x16 sm = f32x16{};
#pragma unroll
      for (int s = 0; s < C::KS; ++s) {
        bf16x8 ka[3];
#pragma unroll
        for (int j = 0; j < 3; ++j)
          ka[j] = *(const bf16x8*)(kb + j * C::PLANE + lr * C::ROWB + ((2 * s + g) ^ swz_k<D>(lr)) * 16);
#pragma unroll
        for (int i = 0; i < kTerms - 1; ++i) sm = mfma32(ka[kTermA[i]], qp[s].p[kTermB[i]], sm);
        sc = mfma32(ka[0], qp[s].p[0], sc);
      }
      sc += sm;
    } else {
#pragma unroll
      for (int s = 0; s < D / 2; ++s) sc = mfma32f(((const float*)kb)[lr * C::KST + 2 * s + g], qf[s], sc);
    }
  };
  // the running maximum raised to the scores' (masked past the last key)
  auto raise = [&](f32x16& sc, int t) {
    if ((t + 1) * C::BN > kv_len) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (t * C::BN + 8 * (r >> 2) + 4 * g + (r & 3) >= kv_len) sc[r] = -INFINITY;
    }
    float mx = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[r]);
    // (SPLIT: scaled)
    const float mnew = fmaxf(m, SPLIT ? pair_max(mx) * sl2 : pair_max(mx));
    // the outputs are rescaled only when some row's maximum rose
    if (__builtin_amdgcn_ballot_w64(!(mnew == m)) != 0) {
      const float alpha = mnew == m ? 1.f : fast_exp2(SPLIT ? m - mnew : (m - mnew) * sl2);
      m = mnew;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < C::DB; ++db) o[db] *= alpha;
    }
  };
  // scores -> probabilities against the running maximum (left in sc, and as
  // planes), row sums
  auto probs = [&](f32x16& sc, Planes (&pp)[2]) {
    // a row without a finite score so far (infinite operands) adds nothing
    const float mm = !SPLIT && m == -INFINITY ? 0.f : m;
    float ls = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = fast_exp2(SPLIT ? __builtin_fmaf(sc[r], sl2, -mm) : __builtin_fmaf(sc[r] - mm, sl2, low));
      ls += sc[r];
    }
    l += ls;
    if constexpr (SPLIT) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        f32x8 x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = sc[8 * s + e];
        pp[s] = split8(x);
      }
    }
  };
  // O^T += V^T P^T of the tile in vb
  auto pv = [&](const unsigned char* vb, const Planes (&pp)[2], const f32x16& sc) {
    if constexpr (SPLIT) {
      constexpr int DP = 2;                          // dim blocks in flight together
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int d0 = 0; d0 < C::DB; d0 += DP) {
          bf16x8 va[DP][3];
#pragma unroll
          for (int d = 0; d < DP; ++d)
#pragma unroll
            for (int j = 0; j < 3; ++j) va[d][j] = v_frag(vb, j, s, d0 + d);
#pragma unroll
          for (int i = 0; i < kTerms; ++i)
#pragma unroll
            for (int d = 0; d < DP; ++d) o[d0 + d] = mfma32(va[d][kTermA[i]], pp[s].p[kTermB[i]], o[d0 + d]);
        }
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r)
#pragma unroll
        for (int db = 0; db < C::DB; ++db)
          o[db] = mfma32f(((const float*)vb)[(8 * (r >> 2) + 4 * g + (r & 3)) * C::VST + db * 32 + lr], sc[r], o[db]);
    }
  };

  if constexpr (C::RW > 1) {
    // Two K and two V buffers: later tiles are split and written beside the
    // MFMAs of this one, those after them are on their way to registers; one
    // barrier per tile.
    unsigned char* vbuf = buf + 2 * C::TILE;
    Stage sk, sv;
    load(sk, kg, t0);
    load(sv, vg, t0);
    store(sk, buf, t0, true);
    store(sv, vbuf, t0, false);
    load(sk, kg, t0 + 1);
    load(sv, vg, t0 + 1);
    __syncthreads();
    if constexpr (C::PIPED) {
      // The scores of tile t+1 are computed beside the probabilities of tile
      // t, so that a wave's own vector work runs under its MFMAs.  K_{t+2}
      // replaces K_t, last read before the previous barrier.
      f32x16 s0, s1;
      qk(buf, s0);
      store(sk, buf + C::TILE, t0 + 1, true);
      load(sk, kg, t0 + 2);
      __syncthreads();
      auto iteration = [&](int t, f32x16& scur, f32x16& snxt, auto ph) {
        constexpr int cur = decltype(ph)::value * C::TILE, nxt = C::TILE - cur;
        raise(scur, t);
        Planes pp[2];
        qk(buf + nxt, snxt);
        probs(scur, pp);
        if constexpr (SPLIT) {
          // one MFMA, six vector instructions, an LDS read every other time
          __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
          for (int i = 0; i < kTerms * C::KS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
            if (i % 2) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          }
        }
        store(sv, vbuf + nxt, t + 1, false);
        load(sv, vg, t + 2);
        pv(vbuf + cur, pp, scur);
        store(sk, buf + cur, t + 2, true);
        load(sk, kg, t + 3);
        __syncthreads();
      };
      for (int t = t0; t < t1; t += 2) {
        iteration(t, s0, s1, std::integral_constant<int, 0>{});
        if (t + 1 < t1) iteration(t + 1, s1, s0, std::integral_constant<int, 1>{});
      }
    } else {
      for (int t = t0; t < t1; ++t) {
        const int cur = ((t - t0) & 1) * C::TILE, nxt = C::TILE - cur;
        store(sk, buf + nxt, t + 1, true);
        load(sk, kg, t + 2);
        f32x16 sc;
        Planes pp[2];
        qk(buf + cur, sc);
        raise(sc, t);
        probs(sc, pp);
        store(sv, vbuf + nxt, t + 1, false);
        load(sv, vg, t + 2);
        pv(vbuf + cur, pp, sc);
        __syncthreads();
      }
    }
  } else {
    // The wave's own buffer holds K_t, then V_t: LDS operations of a wave run
    // in order, so no barrier is needed.
    Stage sk, sv;
    load(sk, kg, t0);
    for (int t = t0; t < t1; ++t) {
      store(sk, buf, t, true);
      load(sv, vg, t);
      f32x16 sc;
      Planes pp[2];
      qk(buf, sc);
      raise(sc, t);
      probs(sc, pp);
      store(sv, buf, t, false);
      load(sk, kg, t + 1);
      pv(buf, pp, sc);
    }
  }
  if constexpr (!SPLIT) m = wide_max(m, sl2, low);
}

// Whether a first pass's state is out of range (a partial sum over eight waves
// still fits below 2^120): not finite, or against a maximum whose rounding after
// the scaling the exponents' fused products do not share.
template <int DB>
__device__ __forceinline__ bool state_out_of_range(const f32x16 (&o)[DB], float m, float l) {
  float hi = __builtin_elementwise_maximum(fabsf(m) * 0x1p96f, l);
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) hi = __builtin_elementwise_maximum(hi, fabsf(o[db][r]));
  return !(hi < 0x1p120f);
}

}  // namespace
}  // namespace ditango
