// cross_few.hip - the cross attention of few query rows (a token, or a handful,
// of each sequence), bf16 (gfx950): the keys of a head over many workgroups.
//
// Bound by HBM: K and V of every head are read once, and a single row leaves
// the matrix core nearly idle.  What it takes is bytes in flight: a workgroup
// has one chunk of a head's keys, each of its four waves every fourth tile of
// 32 of them, and a wave loads its next K tile as soon as the scores are out of
// the last one and its next V tile as soon as the product is, into LDS of its
// own, with no barrier until the four partial states are composed through LDS.
// Two such workgroups share a compute unit: up to 128 KB on their way.
// Chunks have a fixed length, so that sequences of different lengths are shared
// out evenly; what lies behind a sequence's end returns at once.
#include <type_traits>

#include "attn_tile.h"
#include "cross_tile.h"
#include "layer.h"

namespace ditango {
namespace {

template <int D_>
struct FewCfg {
  static constexpr int D = D_, NW = 4, BN = 32;
  static constexpr int NT = NW * 64, BM = 32;
  static constexpr int KS = D / 16, DB = D / 32;
  static constexpr int UNITS = D / 8, ROWB = D * 2, TILEB = BN * ROWB;
  static constexpr int RPL = 1024 / ROWB;
  static constexpr int LW = TILEB / 1024;            // loads of a tile
  static constexpr int LDS = NW * 2 * TILEB + NW * 64 * 4;
};

// Planes of the probabilities (cross_tile.h).  The matrix core waits for memory
// here, and the second one, which leaves the output little but its own rounding,
// costs 1-3 %: 8 x 24 heads of one token, 8 of them with keys, ragged lengths to
// 16,384 73.8 -> 74.7 us, 8 x 24 at D=64 against 16,384 153 -> 157.
constexpr int kPlanes = 2;

template <class C, bool LIST>
__global__ __launch_bounds__(C::NT, 2) void cross_few_kernel(const CrossArgs) {
  constexpr int D = C::D, BN = C::BN;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  Args a = args();
  int t = xcd_remap(blockIdx.x, gridDim.x);
  const int rt = t % a->row_tiles;
  t /= a->row_tiles;
  const int sp = t % a->split;
  t /= a->split;
  const int hk = t % a->Hk;
  const int b = t / a->Hk;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, g = lane >> 5;
  const int n = __builtin_amdgcn_readfirstlane(live_keys(a, b));
  const int key_begin = sp * a->chunk, key_end = min(n, key_begin + a->chunk);
  if (a->split > 1 && key_begin >= n) return;
  const int tiles = (key_end - key_begin + BN - 1) / BN;

  int tok, gi;
  token_of(a, rt * C::BM, lr, &tok, &gi);
  const __bf16* qrow = (const __bf16*)a->q + b * a->q_batch + tok * a->q_token + (int64_t)(hk * a->G + gi) * a->q_head + 8 * g;
  bf16x8 qf[C::KS];
#pragma unroll
  for (int s = 0; s < C::KS; ++s) qf[s] = *(const bf16x8*)(qrow + 16 * s);

  const __bf16* kg = (const __bf16*)a->k + b * a->k_batch + hk * a->k_head;
  const __bf16* vg = (const __bf16*)a->v + b * a->v_batch + hk * a->v_head;
  const int64_t k_token = a->k_token, v_token = a->v_token;
  const int32_t* list = LIST ? a->list + (int64_t)b * a->kv_len : nullptr;
  const __bf16* zeros = (const __bf16*)a->zeros;
  const float sl2 = a->scale_log2;
  unsigned char* mine = smem + wave * 2 * C::TILEB;  // K tile, V tile
  const uint32_t lds0 = lds_addr(mine);
  const int ld_row = lane / C::UNITS, ld_unit = lane % C::UNITS;
  int32_t at[C::LW];                                 // listed places of the tile to come
  auto places = [&](int tile) {
    if constexpr (LIST) {
#pragma unroll
      for (int j = 0; j < C::LW; ++j) {
        const int key = key_begin + tile * BN + j * C::RPL + ld_row;
        at[j] = key < key_end ? list[key] : -1;
      }
    }
  };
  auto load = [&](int tile, int which) {
    const __bf16* base = which ? vg : kg;
    const int64_t stride = which ? v_token : k_token;
    const int key0 = key_begin + tile * BN;
    u32x4 desc;
    if constexpr (!LIST)
      desc = buffer_desc(base + (int64_t)key0 * stride,
                         (uint32_t)min((int64_t)(key_end - 1 - key0) * stride * 2 + C::ROWB, (int64_t)0x7fffffff));
#pragma unroll
    for (int j = 0; j < C::LW; ++j) {
      const int r = j * C::RPL + ld_row;
      const int unit = ld_unit ^ (which ? swz_v<D>(r) : swz_k<D>(r));
      const uint32_t dst = lds0 + (uint32_t)(which * C::TILEB + j * 1024);
      if constexpr (LIST)
        dma_addr((at[j] < 0 ? zeros : base + at[j] * stride) + unit * 8, dst);
      else
        dma_desc(desc, (uint32_t)r * (uint32_t)(stride * 2) + (uint32_t)unit * 16, dst);
    }
  };

  const FragReader<D> fr(lane);
  f32x16 o[C::DB];
#pragma unroll
  for (int db = 0; db < C::DB; ++db) o[db] = f32x16{};
  float m = -INFINITY, l = 0.f;
  if (wave < tiles) {
    places(wave);
    load(wave, 0);
    load(wave, 1);
  }
#pragma unroll 1
  for (int i = wave; i < tiles; i += C::NW) {
    const bool more = i + C::NW < tiles;
    // K has landed, V may be on its way (the next K behind it)
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"(C::LW) : "memory");
    f32x16 sc = fr.scores(mine, qf);
    // every read of the tile is back before it is written again
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) {
      places(i + C::NW);
      load(i + C::NW, 0);
    }
    if (key_begin + (i + 1) * BN > key_end) mask_keys(sc, key_end - key_begin - i * BN, g);
    bf16x8 pf[kPlanes][2];
    softmax_step<C::DB>(sc, pf, o, m, l, sl2, i == wave);
    if (more)
      asm volatile("s_waitcnt vmcnt(%0)" ::"i"(C::LW) : "memory");
    else
      wait_loads();
    fr.template values<false>(mine + C::TILEB, pf, o);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (more) load(i + C::NW, 1);
  }

  a = args();
  if (wave < tiles && __builtin_amdgcn_ballot_w64(out_of_range<C::DB>(o, m)) != 0)
    wide_pass<D, LIST>(a, b, hk, key_begin + wave * BN, key_end, C::NW * BN, mine, qf, o, m, l);

  // ---- the four partial states: O rows of 16-byte units, swizzled by row
  float* part_m = (float*)(smem + C::NW * 2 * C::TILEB);
  float* part_l = part_m + C::NW * 32;
  const float lt = pair_sum(l);
  const int rows = min(a->rows - rt * C::BM, C::BM);
  if (lr < rows) {
    float* po = (float*)mine;
#pragma unroll
    for (int db = 0; db < C::DB; ++db)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = o[db][4 * r4 + e];
        *(f32x4*)(po + lr * D + ((8 * db + 2 * r4 + g) ^ (lr & 15)) * 4) = x;
      }
  }
  if (g == 0) {
    part_m[wave * 32 + lr] = m;
    part_l[wave * 32 + lr] = lt;
  }
  __syncthreads();
  for (int c = tid; c < rows * (D / 4); c += C::NT) {
    const int r = c / (D / 4), u = c % (D / 4);
    float mw[C::NW], M = -INFINITY;
#pragma unroll
    for (int w = 0; w < C::NW; ++w) {
      mw[w] = part_m[w * 32 + r];
      M = fmaxf(M, mw[w]);
    }
    float tot = 0.f;
    f32x4 acc = f32x4{};
#pragma unroll
    for (int w = 0; w < C::NW; ++w) {
      const float lw = part_l[w * 32 + r];
      const float x = mw[w] == -INFINITY && lw == 0.f ? 0.f : fast_exp2(mw[w] - M);   // (a wave without keys)
      tot = __builtin_fmaf(x, lw, tot);
      acc += x * *(const f32x4*)((const float*)(smem + w * 2 * C::TILEB) + r * D + (u ^ (r & 15)) * 4);
    }
    const float inv = tot > 0.f ? 1.0f / tot : 0.f;
    const float lse = tot > 0.f ? (M + __builtin_amdgcn_logf(tot)) * kLn2 : tot == 0.f ? -INFINITY : tot;
    int rtok, rgi;
    token_of(a, rt * C::BM, r, &rtok, &rgi);
    const int64_t row = ((int64_t)b * a->H + hk * a->G + rgi) * a->q_len + rtok;
    if (a->split > 1) {
      const int64_t ap = (int64_t)sp * a->B * a->H * a->q_len + row;
      *(f32x4*)(a->part_out + ap * D + u * 4) = acc * inv;
      if (u == 0) a->part_lse[ap] = lse;
    } else {
      acc *= inv;
      *(bf16x4*)((__bf16*)a->out + (((int64_t)b * a->q_len + rtok) * a->H + hk * a->G + rgi) * D + u * 4) =
          __builtin_convertvector(acc, bf16x4);
      if (u == 0 && a->lse != nullptr) a->lse[row] = lse;
    }
  }
}

template <class C, bool LIST>
hipError_t launch_few(const CrossArgs& a0, int dev, hipStream_t s) {
  const hipError_t e = set_kernel_lds<&cross_few_kernel<C, LIST>, C::LDS>(dev);
  if (e != hipSuccess) return e;
  CrossArgs a = a0;
  a.row_tiles = (a.rows + C::BM - 1) / C::BM;
  const int64_t grid = (int64_t)a.row_tiles * a.split * a.Hk * a.B;
  if (!launch_fits(grid, C::NT)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((cross_few_kernel<C, LIST>), dim3((unsigned)grid), dim3(C::NT), C::LDS, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cross_few(const CrossArgs& a, int D, hipStream_t s) {
  int dev = 0;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (D == 128) return a.mask ? launch_few<FewCfg<128>, true>(a, dev, s) : launch_few<FewCfg<128>, false>(a, dev, s);
  return a.mask ? launch_few<FewCfg<64>, true>(a, dev, s) : launch_few<FewCfg<64>, false>(a, dev, s);
}

}  // namespace ditango
