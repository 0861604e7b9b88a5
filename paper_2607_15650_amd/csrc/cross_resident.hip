// cross_resident.hip - the cross attention of many query rows to few keys,
// bf16 (gfx950): the keys and values of a head stay in LDS.
//
// A prompt's states of one head are small: 256 keys at D=64 take 64 KB.  A
// workgroup per compute unit, of 12 waves (D=64: 16, as many as their registers
// allow), loads them once and its waves walk over blocks of query rows by
// themselves, without a barrier: while one wave of a SIMD takes exponentials the
// others' products run.  The next block's queries are on their way from the last
// use of this one's on.
//
// 14,850 rows x 48 heads at D=64 against 256 of 333 keys: 79 us, the matrix core
// busy 28 % of it and the vector unit about half (exponentials, conversions,
// sums); a workgroup's 87 blocks of a share are 5.4 rounds of its waves, run as
// six, and at a change of head all of them wait for the mask's list and the new
// keys.  9,450 x 40 at D=128 against 256: 74-77 us, the same way.
#include <type_traits>

#include "attn_tile.h"
#include "cross_tile.h"
#include "layer.h"

namespace ditango {
namespace {

constexpr int kLds = 163840;                        // of a compute unit

template <int D_, int NW_>
struct ResidentCfg {
  static constexpr int D = D_, NW = NW_, BN = 64;
  static constexpr int NT = NW * 64, BM = 32;
  static constexpr int KS = D / 16, DB = D / 32;
  static constexpr int UNITS = D / 8, ROWB = D * 2, TILEB = BN * ROWB;
  static constexpr int RPL = 1024 / ROWB;
  static constexpr int LOADS = TILEB / 1024;       // 1 KiB loads of a tile
  static constexpr int MAX_TILES = kLds / (2 * TILEB);
};

// How the keys' rows are found: a prefix; the list of the workspace; or the
// mask, whose live keys the workgroup lists behind its tiles in LDS (the
// launch of a kernel for that alone took 6 us of 81: 14,850 rows x 48 heads at
// D=64, 256 of 333 keys live).
enum Keys { kPrefix, kList, kMask };

template <class C, Keys KEYS>
__global__ __launch_bounds__(C::NT, C::NW / 4) void cross_resident_kernel(const CrossArgs) {
  constexpr int D = C::D, BN = C::BN;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, g = lane >> 5;
  const uint32_t lds0 = lds_addr(smem);

  // this workgroup's blocks of rows: a contiguous share, of one head or a few
  Args a = args();
  const int groups = a->Hk * a->B;
  const int64_t all = (int64_t)a->row_tiles * groups;
  const int w = xcd_remap(blockIdx.x, gridDim.x);
  int64_t at = all * w / gridDim.x;
  const int64_t end = all * (w + 1) / gridDim.x;

  const int ld_row = lane / C::UNITS, ld_unit = lane % C::UNITS;
  const FragReader<D> fr(lane);
  bf16x8 qf[C::KS];
  while (at < end) {
    a = args();
    const int grp = (int)(at / a->row_tiles);
    const int hk = grp / a->B, b = grp % a->B;
    const int first = (int)(at - (int64_t)grp * a->row_tiles);
    const int last = (int)min((int64_t)a->row_tiles, first + (end - at));   // row blocks [first, last)
    at += last - first;
    __syncthreads();                                    // the head before is done with
    int n;
    int* own_list = (int*)(smem + (a->kv_len + BN - 1) / BN * 2 * C::TILEB);
    if constexpr (KEYS == kMask) {
      // places of the live keys, in order: counts by ballot, waves in order
      int* sums = own_list + a->kv_len;
      const int keys = a->lens == nullptr ? a->kv_len : min(max(a->lens[b], 0), a->kv_len);
      const uint8_t* mask = a->mask + (int64_t)b * a->kv_len;
      n = 0;
      for (int k0 = 0; k0 < keys; k0 += C::NT) {
        const int key = k0 + tid;
        const bool live = key < keys && mask[key] != 0;
        const uint64_t votes = __builtin_amdgcn_ballot_w64(live);
        if (lane == 0) sums[wave] = __builtin_popcountll(votes);
        __syncthreads();
        int before = n;
#pragma unroll
        for (int v = 0; v < C::NW; ++v) {
          if (v < wave) before += sums[v];
          n += sums[v];
        }
        if (live) own_list[before + __builtin_popcountll(votes & ((1ull << lane) - 1))] = key;
        __syncthreads();
      }
      n = __builtin_amdgcn_readfirstlane(n);
    } else {
      n = __builtin_amdgcn_readfirstlane(live_keys(a, b));
    }
    const int tiles = (n + BN - 1) / BN, steps = (n + 31) / 32;
    const float sl2 = a->scale_log2;

    // ---- K and V of the head: tile i of K, then of V
    const __bf16* kg = (const __bf16*)a->k + b * a->k_batch + hk * a->k_head;
    const __bf16* vg = (const __bf16*)a->v + b * a->v_batch + hk * a->v_head;
    for (int u = wave; u < tiles * 2 * C::LOADS; u += C::NW) {
      const int i = u / (2 * C::LOADS), which = u / C::LOADS % 2, j = u % C::LOADS;
      const __bf16* base = which ? vg : kg;
      const int64_t stride = which ? a->v_token : a->k_token;
      const uint32_t dst = lds0 + (uint32_t)((2 * i + which) * C::TILEB + j * 1024);
      const int r = j * C::RPL + ld_row;
      const int unit = ld_unit ^ (which ? swz_v<D>(r) : swz_k<D>(r));
      if constexpr (KEYS == kList) {
        const __bf16* p = (const __bf16*)a->zeros;
        if (i * BN + r < n) p = base + a->list[(int64_t)b * a->kv_len + i * BN + r] * stride;
        dma_addr(p + unit * 8, dst);
      } else if constexpr (KEYS == kMask) {
        // (places past the last live key lie past the descriptor's end)
        const u32x4 desc = buffer_desc(base, (uint32_t)((a->kv_len - 1) * stride * 2 + C::ROWB));
        const uint32_t row = i * BN + r < n ? (uint32_t)own_list[i * BN + r] * (uint32_t)(stride * 2) : 0x80000000u;
        dma_desc(desc, row + (uint32_t)unit * 16, dst);
      } else {
        const u32x4 desc = buffer_desc(base + (int64_t)i * BN * stride,
                                       (uint32_t)min((int64_t)(n - 1 - i * BN) * stride * 2 + C::ROWB, (int64_t)0x7fffffff));
        // (places past the end: also where the keys' rows overlap)
        dma_desc(desc, i * BN + r < n ? (uint32_t)r * (uint32_t)(stride * 2) + (uint32_t)unit * 16 : 0x80000000u, dst);
      }
    }
    auto load_queries = [&](int blk, int lane) {
      a = args();
      int tok, gi;
      token_of(a, blk * 32, lane & 31, &tok, &gi);
      const __bf16* p = (const __bf16*)a->q + b * a->q_batch + tok * a->q_token + (int64_t)(hk * a->G + gi) * a->q_head +
                        8 * (lane >> 5);
#pragma unroll
      for (int s = 0; s < C::KS; ++s) qf[s] = *(const bf16x8*)(p + 16 * s);
    };
    auto store_rows = [&](int blk, int lane, const f32x16 (&o)[C::DB], float m, float l) {
      a = args();
      const int lr = lane & 31, g = lane >> 5;
      // ---- the rows' state: two lanes' quarters of 16 dims make rows of 32 bytes
      const float lt = pair_sum(l);
      const float inv = lt > 0.f ? 1.0f / lt : 0.f;
      const int row = blk * 32 + lr;
      if (row < a->rows) {
        int tok, gi;
        token_of(a, blk * 32, lr, &tok, &gi);
        const int h = hk * a->G + gi;
        if (g == 0 && a->lse != nullptr)
          a->lse[((int64_t)b * a->H + h) * a->q_len + tok] =
              lt > 0.f ? (m + __builtin_amdgcn_logf(lt)) * kLn2 : lt == 0.f ? -INFINITY : lt;
        __bf16* dst = (__bf16*)a->out + (((int64_t)b * a->q_len + tok) * a->H + h) * D + 8 * g;
#pragma unroll
        for (int db = 0; db < C::DB; ++db)
#pragma unroll
          for (int half = 0; half < 2; ++half) *(bf16x8*)(dst + 32 * db + 16 * half) = row_units(o[db], half, inv);
      }
    };
    if (first + wave < last) load_queries(first + wave, lane);
    wait_loads();
    __syncthreads();
    for (int u = wave; u < tiles * 4; u += C::NW) fr.order_values(smem + (u / 4 * 2 + 1) * C::TILEB, u % 4);
    __syncthreads();

    uint64_t again = 0;
    for (int blk = first + wave, turn = 0; blk < last; blk += C::NW, ++turn) {
      f32x16 o[C::DB];
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int db = 0; db < C::DB; ++db) o[db] = f32x16{};
#pragma unroll 1
      for (int i = 0; i < steps; ++i) {
        const unsigned char* kt = smem + i / 2 * 2 * C::TILEB + i % 2 * 32 * C::ROWB;
        f32x16 sc = fr.scores(kt, qf);
        if (i + 1 == steps) {
          load_queries(blk + C::NW < last ? blk + C::NW : blk, lane);
          if ((i + 1) * 32 > n) mask_keys(sc, n - i * 32, g);
        }
        bf16x8 pf[1][2];
        softmax_step<C::DB>(sc, pf, o, m, l, sl2, i == 0);
        fr.template values<true>(kt + C::TILEB, pf, o);
      }
      if (steps == 0) load_queries(blk + C::NW < last ? blk + C::NW : blk, lane);
      // (a bit for every 64th of the wave's blocks)
      if (steps > 0 && __builtin_amdgcn_ballot_w64(out_of_range<C::DB>(o, m)) != 0) again |= 1ull << (turn & 63);
      store_rows(blk, lane, o, m, l);
    }
    if (again == 0) continue;
    // ---- the blocks with rows out of range once more, over the rows as stored
    wait_loads();
    for (int blk = first + wave, turn = 0; blk < last; blk += C::NW, ++turn) {
      if ((again >> (turn & 63) & 1) == 0) continue;
      const FragReader<D> wr(lane_id());
      load_queries(blk, wr.lane);
      f32x16 o[C::DB];
      const float low = wide_low(n);
      float mx = -INFINITY, l = 0.f;
#pragma unroll
      for (int db = 0; db < C::DB; ++db) o[db] = f32x16{};
#pragma unroll 1
      for (int i = 0; i < steps; ++i) {
        const unsigned char* kt = smem + i / 2 * 2 * C::TILEB + i % 2 * 32 * C::ROWB;
        f32x16 sc = wr.scores(kt, qf);
        if ((i + 1) * 32 > n) mask_keys(sc, n - i * 32, wr.lane >> 5);
        bf16x8 pf[1][2];
        wide_step<C::DB>(sc, pf, o, mx, l, sl2, low);
        wr.template values<true>(kt + C::TILEB, pf, o);
      }
      store_rows(blk, wr.lane, o, wide_max(mx, sl2, low), l);
    }
  }
}

template <class C>
size_t resident_lds(const CrossArgs& a, bool mask) {
  return (size_t)(a.kv_len + C::BN - 1) / C::BN * 2 * C::TILEB + (mask ? (size_t)a.kv_len * 4 + C::NW * 4 : 0);
}

template <class C, Keys KEYS>
hipError_t launch_resident(const CrossArgs& a0, int cus, int dev, hipStream_t s) {
  const hipError_t e = set_kernel_lds<&cross_resident_kernel<C, KEYS>, kLds>(dev);
  if (e != hipSuccess) return e;
  CrossArgs a = a0;
  a.row_tiles = (a.rows + C::BM - 1) / C::BM;
  const int64_t all = (int64_t)a.row_tiles * a.Hk * a.B;
  const int64_t want = (all + C::NW - 1) / C::NW;
  const int grid = (int)(want < cus ? want : cus);
  hipLaunchKernelGGL((cross_resident_kernel<C, KEYS>), dim3((unsigned)grid), dim3(C::NT),
                     resident_lds<C>(a, KEYS == kMask), s, a);
  return hipGetLastError();
}

using Resident128 = ResidentCfg<128, 12>;
using Resident64 = ResidentCfg<64, 16>;

}  // namespace

int cross_resident_keys(int D) { return (D == 128 ? Resident128::MAX_TILES : Resident64::MAX_TILES) * 64; }
int cross_resident_waves(int D) { return D == 128 ? Resident128::NW : Resident64::NW; }

bool cross_resident_lists(const CrossArgs& a, int D) {
  const int64_t stride = a.k_token > a.v_token ? a.k_token : a.v_token;
  const size_t lds = D == 128 ? resident_lds<Resident128>(a, true) : resident_lds<Resident64>(a, true);
  return lds <= (size_t)kLds && a.kv_len * stride * 2 < ((int64_t)1 << 31);
}

template <class C>
static hipError_t launch_form(const CrossArgs& a, int D, int cus, int dev, hipStream_t s) {
  if (a.mask == nullptr) return launch_resident<C, kPrefix>(a, cus, dev, s);
  return cross_resident_lists(a, D) ? launch_resident<C, kMask>(a, cus, dev, s) : launch_resident<C, kList>(a, cus, dev, s);
}

hipError_t launch_cross_resident(const CrossArgs& a, int D, hipStream_t s) {
  int dev = 0, cus = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return e;
  return D == 128 ? launch_form<Resident128>(a, D, cus, dev, s) : launch_form<Resident64>(a, D, cus, dev, s);
}

}  // namespace ditango
