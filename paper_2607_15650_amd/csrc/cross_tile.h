// cross_tile.h - tile loads and the steps over one key tile that the bf16
// kernels of the cross attention share.
#pragma once

#include "attn_tile.h"
#include "layer.h"
#include "wide_range.h"

namespace ditango {
namespace {

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// The kernel's arguments, as if read for the first time: what a long loop does
// not use stays out of its scalar registers.
typedef const __attribute__((address_space(4))) CrossArgs* Args;
__device__ __forceinline__ Args args() {
  Args p = (Args)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}
// Live keys of sequence b.
__device__ __forceinline__ int live_keys(Args a, int b) {
  if (a->mask != nullptr) return a->count[b];
  return a->lens == nullptr ? a->kv_len : min(max(a->lens[b], 0), a->kv_len);
}

// This lane of the wave, counted anew: what a rare path derives from it is not
// computed, and kept, in front of the loops around that path.
__device__ __forceinline__ int lane_id() {
  int x;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
  return x;
}

// Token and head (of the G that share a key/value head) of row row0 + r; rows
// past the end give the last one's.  row0 is wave-uniform.
__device__ __forceinline__ void token_of(Args a, int row0, int r, int* tok, int* gi) {
  const int row = min(row0 + r, a->rows - 1);
  if (a->G == 1) {
    *tok = row;
    *gi = 0;
  } else {
    const int tok0 = row0 / a->G;
    const uint32_t x = (uint32_t)(row - tok0 * a->G);     // below 256 + G: the product is exact
    const uint32_t y = __umulhi(x, a->g_inverse);
    *tok = tok0 + (int)y;
    *gi = (int)(x - y * (uint32_t)a->G);
  }
}

// this wave's loads, into registers and into LDS, have landed
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Buffer descriptor of raw bytes [base, base + nbytes): loads past the end
// give zeros and do not access memory.
__device__ __forceinline__ u32x4 buffer_desc(const void* base, uint32_t nbytes) {
  const uint64_t p = (uint64_t)(uintptr_t)base;
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)p),
               (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(p >> 32)) & 0xffffu,
               (uint32_t)__builtin_amdgcn_readfirstlane(nbytes), 0x00020000u};
}

// 16-byte direct loads global -> LDS for the wave: lane l's 16 bytes land at
// LDS byte lds + 16 * l (wave-uniform).  From a descriptor and a byte offset,
// or from an address.  The waits for them are written out.
__device__ __forceinline__ void dma_desc(const u32x4& desc, uint32_t off, uint32_t lds) {
  const uint32_t m0v = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :
               : "v"(off), "s"(desc), "s"(m0v)
               : "memory", "m0");
}
__device__ __forceinline__ void dma_addr(const void* p, uint32_t lds) {
  const uint32_t m0v = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(p), "s"(m0v)
               : "memory", "m0");
}

// Fragments of a 64-key tile in LDS (rows of D elements, 16-byte units
// swizzled as attn_tile.h says) and the products with them.
template <int D>
struct FragReader {
  static constexpr int KS = D / 16, DB = D / 32, ROWB = D * 2;
  int lane, kswz, voff[DB];
  __device__ __forceinline__ explicit FragReader(int lane_) : lane(lane_) {
    const int g = lane >> 5;
    kswz = swz_k<D>(lane & 31);
    // V^T by transpose reads: source lane r of a 16-lane group points at row
    // 4g + r/4 (+ 16s + 8) and dims 32db + 16*(group%2) + 4*(r%4)
    const int vrow = 4 * g + ((lane & 15) >> 2);
    const int vdim = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const int dim = 32 * db + vdim;
      voff[db] = vrow * ROWB + ((dim >> 3) ^ swz_v<D>(vrow)) * 16 + (dim & 7) * 2;
    }
  }
  __device__ __forceinline__ bf16x8 key_frag(const unsigned char* kt, int kb, int s) const {
    return *(const bf16x8*)(kt + (kb * 32 + (lane & 31)) * ROWB + ((2 * s + (lane >> 5)) ^ kswz) * 16);
  }
  __device__ __forceinline__ bf16x8 value_frag(const unsigned char* vt, int s, int db) const {
    const unsigned char* p = vt + 16 * s * ROWB + voff[db];
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, p)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, p + 8 * ROWB)));
    return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
  }
  // The same fragment where the tile's V lies as fragments, one after another:
  // one read instead of two.
  __device__ __forceinline__ bf16x8 ordered_frag(const unsigned char* vt, int s, int db) const {
    return *(const bf16x8*)(vt + 16 * s * ROWB + db * 1024 + lane * 16);
  }
  // Rows 16s ... 16s + 15 of V -> the fragments of its DB blocks of dims, in place.
  __device__ __forceinline__ void order_values(unsigned char* vt, int s) const {
    bf16x8 x[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) x[db] = value_frag(vt, s, db);
#pragma unroll
    for (int db = 0; db < DB; ++db) *(bf16x8*)(vt + 16 * s * ROWB + db * 1024 + lane * 16) = x[db];
  }
  // S^T = K Q^T of 32 keys
  __device__ __forceinline__ f32x16 scores(const unsigned char* kt, const bf16x8 (&qf)[KS]) const {
    f32x16 sc = f32x16{};
#pragma unroll
    for (int s = 0; s < KS; ++s) sc = mfma32(key_frag(kt, 0, s), qf[s], sc);
    return sc;
  }
  // O^T += V^T P^T of 32 keys
  template <bool ORDERED, int PLANES>
  __device__ __forceinline__ void values(const unsigned char* vt, const bf16x8 (&pf)[PLANES][2], f32x16 (&o)[DB]) const {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 v = ORDERED ? ordered_frag(vt, s, db) : value_frag(vt, s, db);
#pragma unroll
        for (int j = PLANES - 1; j >= 0; --j) o[db] = mfma32(v, pf[j][s], o[db]);
      }
  }
};

// keys at or past `left` of the step -> -inf
__device__ __forceinline__ void mask_keys(f32x16& sc, int left, int g) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (8 * (r >> 2) + 4 * g + (r & 3) >= left) sc[r] = -INFINITY;
}

// Probabilities of half a step's keys (8 of a lane) as PLANES bf16 planes: the
// rounding of each, by at most 2^-8, and (PLANES = 2) that of what it leaves.
template <int PLANES>
__device__ __forceinline__ void round_probs(const f32x8& x, bf16x8 (&pf)[PLANES][2], int h) {
  pf[0][h] = __builtin_convertvector(x, bf16x8);
  if constexpr (PLANES == 2) pf[1][h] = __builtin_convertvector(x - __builtin_convertvector(pf[0][h], f32x8), bf16x8);
}

// Scores of 32 keys -> probabilities against the running maximum m, row sum l
// (this lane's keys).  m is the first step's maximum, and raised only where a
// lane's sum over a step then passes 2^40 or is not a number: below that
// float32 holds the row sums, and the result does not depend on which m was
// used.  It holds the outputs too while the values are below 2^80 or so;
// out_of_range finds the rows where it does not.
template <int DB, int PLANES>
__device__ __forceinline__ void softmax_step(const f32x16& sc, bf16x8 (&pf)[PLANES][2], f32x16 (&o)[DB], float& m, float& l,
                                             float sl2, bool first) {
  float sum;
  auto raise = [&] {
    float mx = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[r]);
    // (-FLT_MAX where every score so far is -inf: their exponentials are zeros,
    // those of any other score infinite, which raises m)
    const float mnew = fmaxf(fmaxf(m, pair_max(mx) * sl2), -0x1.fffffep127f);
    if (!first) {
      const float alpha = fast_exp2(m - mnew);
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= alpha;
    }
    m = mnew;
  };
  auto probs = [&] {
    sum = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x8 x;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[e] = fast_exp2(__builtin_fmaf(sc[8 * h + e], sl2, -m));
        sum += x[e];
      }
      round_probs(x, pf, h);
    }
  };
  if (first) raise();
  probs();
  if (!first && __builtin_amdgcn_ballot_w64(!(sum <= 0x1p40f)) != 0) {
    raise();
    probs();
  }
  l += sum;
}

// What the steps above cannot hold: a row whose probabilities, up to 2^40 of
// them against a lagging maximum, or whose number took an output to 2^120 or
// more (four partial ones below that add up inside float32), or whose maximum is
// 2^24 or more.  There the rounding of m, which the exponents' fused products do
// not share, moves every probability by a factor that passes 2^(1/2), and from
// 2^31 on can leave float32's range: 0 for all, or infinity.  NaN and infinities
// are among them, and a row whose every score was -inf.  Such rows are formed
// again, by wide_pass.  (Beside the exponentials: cross_video 119.4 -> 120.1 us,
// 9,450 rows x 40 heads against 256 keys 74.0 -> 75.2.)
template <int DB>
__device__ __forceinline__ bool out_of_range(const f32x16 (&o)[DB], float m) {
  float hi = fabsf(m) * 0x1p96f;
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) hi = __builtin_elementwise_maximum(hi, fabsf(o[db][r]));
  return !(hi < 0x1p120f);
}

// Scores of 32 keys -> probabilities 2^low exp2(scale (s - mx)) against the
// maximum mx of the scores so far as they are: the largest is 2^low exactly
// (wide_range.h has low, by which sums over all keys stay below the values they
// weigh).  In one plane: the second, 0 or negative, would make NaN of an infinite
// value.
template <int DB>
__device__ __forceinline__ void wide_step(const f32x16& sc, bf16x8 (&pf)[1][2], f32x16 (&o)[DB], float& mx, float& l,
                                          float sl2, float low) {
  float top = sc[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) top = fmaxf(top, sc[r]);
  const float mnew = fmaxf(mx, pair_max(top));
  const float at = mnew == -INFINITY ? 0.f : mnew;
  const float alpha = mx == -INFINITY ? 0.f : fast_exp2((mx - mnew) * sl2);
  mx = mnew;
  l *= alpha;
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] *= alpha;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    f32x8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = fast_exp2(__builtin_fmaf(sc[8 * h + e] - at, sl2, low));
      l += x[e];
    }
    round_probs(x, pf, h);
  }
}
// The state of 32 rows over keys [key_begin, key_end) in steps of 32 that lie
// `stride` apart, by one wave: tiles of 32 keys of K and of V in LDS of its own,
// loaded as they are needed (rows out of range are rare: simple, not fast).
template <int D, bool LIST>
__device__ __forceinline__ void wide_pass(Args a, int b, int hk, int key_begin, int key_end, int stride,
                                          unsigned char* own, const bf16x8 (&qf)[D / 16], f32x16 (&o)[D / 32], float& m,
                                          float& l) {
  constexpr int ROWB = D * 2, UNITS = D / 8, RPL = 1024 / ROWB;
  const __bf16* kg = (const __bf16*)a->k + b * a->k_batch + hk * a->k_head;
  const __bf16* vg = (const __bf16*)a->v + b * a->v_batch + hk * a->v_head;
  const int32_t* list = LIST ? a->list + (int64_t)b * a->kv_len : nullptr;
  const float sl2 = a->scale_log2, low = wide_low(key_end - key_begin);
  const int lane = lane_id();
  const FragReader<D> fr(lane);
  float mx = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) o[db] = f32x16{};
#pragma unroll 1
  for (int64_t key = key_begin; key < key_end; key += stride) {
    const int left = (int)min(key_end - key, (int64_t)32);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // the last step's reads are back
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
      for (int j = 0; j < 32 / RPL; ++j) {
        const int r = j * RPL + lane / UNITS;
        const int unit = lane % UNITS ^ (which ? swz_v<D>(r) : swz_k<D>(r));
        // (rows past the end read the last one: its scores are masked, and its
        // values replaced by zeros)
        const int64_t at = key + min(r, left - 1);
        const __bf16* p = (which ? vg : kg) + (LIST ? (int64_t)list[at] : at) * (which ? a->v_token : a->k_token);
        dma_addr(p + unit * 8, lds_addr(own) + (uint32_t)(which * 32 * ROWB + j * 1024));
      }
    wait_loads();
    if (left < 32) {
      uint32_t zero = 0;
      asm volatile("" : "+v"(zero));                       // (not kept in registers around the loops outside)
      for (int i = lane; i < (32 - left) * UNITS; i += 64)
        *(u32x4*)(own + (32 + left) * ROWB + i * 16) = u32x4{zero, zero, zero, zero};
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    f32x16 sc = fr.scores(own, qf);
    if (left < 32) mask_keys(sc, left, lane >> 5);
    bf16x8 pf[1][2];
    wide_step<D / 32>(sc, pf, o, mx, l, sl2, low);
    fr.template values<false>(own + 32 * ROWB, pf, o);
  }
  m = wide_max(mx, sl2, low);
}

// Unit `half` of a lane's row in a 32-dim block of the accumulators, times
// `x`: lanes l and l ^ 32 hold dims 8r + 4g ... + 3 (r = 0 ... 3) of row
// l % 32; here lane l gets dims 16 * half + 8g ... + 7.
__device__ __forceinline__ bf16x8 row_units(const f32x16& o, int half, float x) {
  f32x4 a, b;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    a[e] = o[8 * half + e] * x;
    b[e] = o[8 * half + 4 + e] * x;
  }
  const u32x2 pa = __builtin_bit_cast(u32x2, __builtin_convertvector(a, bf16x4));
  const u32x2 pb = __builtin_bit_cast(u32x2, __builtin_convertvector(b, bf16x4));
  const auto r0 = __builtin_amdgcn_permlane32_swap(pa[0], pb[0], false, false);
  const auto r1 = __builtin_amdgcn_permlane32_swap(pa[1], pb[1], false, false);
  return __builtin_bit_cast(bf16x8, u32x4{r0[0], r1[0], r0[1], r1[1]});
}

}  // namespace
}  // namespace ditango
