// cross.hip - attention of a query block to an encoder's states (gfx950).
//
// For every batch b, query token t and head h, with the live keys c of
// sequence b (c < lens[b], mask[b][c] != 0) and the key/value head hk = h / G
// that G query heads share:
//   LSE = log sum_c exp(scale q.k_c),   OUT = sum_c exp(scale q.k_c - LSE) v_c
// by one pass over the keys with a running maximum, as the self attention's
// kernels do it (attn_bf16.hip describes the orientation, the accumulator
// layout and the LDS swizzles; S^T = K Q^T, O^T = V^T P^T).  A row without
// live keys has OUT = 0 and LSE = -inf.
//
// Rows
//   The query heads that share a key/value head are rows of one problem (row
//   r: token r / G, head hk * G + r % G), so that one K or V tile in LDS serves
//   all of them, and a single token of a shared head fills G rows of a tile.
//
// Masks
//   Keys a mask leaves out are never read: a kernel in front of this one
//   writes the places of the live ones in order, and the tile loads, whose
//   every lane has an address of its own, go by that list.  Rows past the last
//   live key come from a row of zeros (list) or from past the end of a buffer
//   descriptor (prefix), which reads as zeros: nothing that a masked place
//   holds, NaN and infinities included, enters a product.
//
// Rounding
//   Products of bf16 values, accumulated in float32.  The probabilities go to
//   bf16 for the second product, by at most 2^-8 of each (the row sum takes them
//   before that), the output once more at its store: half of the matrix core's
//   work is that product, and a second bf16 plane of the probabilities would add
//   as much again, here and in the kernels of many rows; the one of few rows,
//   which waits for memory, has it (cross_few.hip).
//
// Range
//   Rows whose sums or scores leave float32 are formed again (cross_tile.h).
#include <math.h>

#include <type_traits>

#include "attn_tile.h"
#include "cross_tile.h"
#include "layer.h"

namespace ditango {
namespace {

// One workgroup: NW * 32 rows of one key/value head, one key range.  The waves
// share the K and V tiles of 64 keys, which land in rings of two tiles by direct
// loads.
template <int D_, int NW_>
struct RowsCfg {
  static constexpr int D = D_, NW = NW_, BN = 64, NBUF = 2;
  static constexpr int NT = NW * 64, BM = NW * 32;
  static constexpr int KS = D / 16, DB = D / 32;
  static constexpr int UNITS = D / 8, ROWB = D * 2, TILEB = BN * ROWB;
  static constexpr int RPL = 1024 / ROWB;          // rows per 1 KiB load
  static constexpr int LOADS = TILEB / 1024;       // 1 KiB loads of a tile
  static constexpr int LDS = 2 * NBUF * TILEB;
  static_assert(NW * TILEB <= LDS, "a K and a V tile of 32 keys for every wave");
};

template <class C, int WPE, bool LIST>
__global__ __launch_bounds__(C::NT, WPE) void cross_kernel(const CrossArgs) {
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

  // this workgroup's key range: whole tiles
  const int n = __builtin_amdgcn_readfirstlane(live_keys(a, b));
  const int per = ((n + BN - 1) / BN + a->split - 1) / a->split * BN;
  const int key_begin = min(sp * per, n), key_end = min(key_begin + per, n);
  const int tiles = (key_end - key_begin + BN - 1) / BN;

  // ---- this lane's query row (rows past the end read the last one and are
  // not stored): B operand, Q[row][16s + 8g .. +8]
  const int row = rt * C::BM + wave * 32 + lr;
  bf16x8 qf[C::KS];
  {
    int tok, gi;
    token_of(a, rt * C::BM, wave * 32 + lr, &tok, &gi);
    const __bf16* p = (const __bf16*)a->q + b * a->q_batch + tok * a->q_token + (int64_t)(hk * a->G + gi) * a->q_head + 8 * g;
#pragma unroll
    for (int s = 0; s < C::KS; ++s) qf[s] = *(const bf16x8*)(p + 16 * s);
  }

  const __bf16* kg = (const __bf16*)a->k + b * a->k_batch + hk * a->k_head;
  const __bf16* vg = (const __bf16*)a->v + b * a->v_batch + hk * a->v_head;
  const int64_t k_token = a->k_token, v_token = a->v_token;
  const int32_t* list = LIST ? a->list + (int64_t)b * a->kv_len : nullptr;
  const __bf16* zeros = (const __bf16*)a->zeros;
  const float sl2 = a->scale_log2;
  const uint32_t lds0 = lds_addr(smem);
  const int ld_row = lane / C::UNITS, ld_unit = lane % C::UNITS;
  // tile `tile` of K and V into their rings
  auto load_tile = [&](int tile) {
    const int key0 = key_begin + tile * BN;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const uint32_t dst = lds0 + (uint32_t)((which * C::NBUF + tile % C::NBUF) * C::TILEB);
      const __bf16* base = which ? vg : kg;
      const int64_t stride = which ? v_token : k_token;
      u32x4 desc;
      if constexpr (!LIST)
        desc = buffer_desc(base + (int64_t)key0 * stride,
                           (uint32_t)min((int64_t)(key_end - 1 - key0) * stride * 2 + C::ROWB, (int64_t)0x7fffffff));
#pragma unroll
      for (int i = 0; i < (C::LOADS + C::NW - 1) / C::NW; ++i) {
        const int j = wave + i * C::NW;
        if (C::LOADS % C::NW != 0 && j >= C::LOADS) break;
        const int r = j * C::RPL + ld_row;
        const int unit = ld_unit ^ (which ? swz_v<D>(r) : swz_k<D>(r));
        if constexpr (LIST) {
          const __bf16* p = zeros;
          if (key0 + r < key_end) p = base + list[key0 + r] * stride;
          dma_addr(p + unit * 8, dst + j * 1024);
        } else {
          dma_desc(desc, (uint32_t)r * (uint32_t)(stride * 2) + (uint32_t)unit * 16, dst + j * 1024);
        }
      }
    }
  };

  const FragReader<D> fr(lane);
  f32x16 o[C::DB];
#pragma unroll
  for (int db = 0; db < C::DB; ++db) o[db] = f32x16{};
  float m = -INFINITY, l = 0.f;
  if (tiles > 0) load_tile(0);
#pragma unroll 1
  for (int i = 0; i < tiles; ++i) {
    wait_loads();                                    // tile i has landed
    __syncthreads();
    if (i + 1 < tiles) load_tile(i + 1);
    const unsigned char* kt = smem + i % C::NBUF * C::TILEB;
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      const int key = key_begin + i * BN + st * 32;
      if (st > 0 && key >= key_end) break;
      f32x16 sc = fr.scores(kt + st * 32 * C::ROWB, qf);
      if (key + 32 > key_end) mask_keys(sc, key_end - key, g);
      bf16x8 pf[1][2];
      softmax_step<C::DB>(sc, pf, o, m, l, sl2, i + st == 0);
      fr.template values<false>(kt + C::NBUF * C::TILEB + st * 32 * C::ROWB, pf, o);
    }
  }

  a = args();
  __syncthreads();                                   // the rings are done with
  if (tiles > 0 && __builtin_amdgcn_ballot_w64(out_of_range<C::DB>(o, m)) != 0)
    wide_pass<D, LIST>(a, b, hk, key_begin, key_end, 32, smem + wave * C::TILEB, qf, o, m, l);

  // ---- the rows' state (two lanes' quarters of 16 dims make 32 bytes)
  const float lt = pair_sum(l);
  const float inv = lt > 0.f ? 1.0f / lt : 0.f;
  const float lse = lt > 0.f ? (m + __builtin_amdgcn_logf(lt)) * kLn2 : lt == 0.f ? -INFINITY : lt;
  if (row >= a->rows) return;
  int tok, gi;
  token_of(a, rt * C::BM, wave * 32 + lr, &tok, &gi);
  const int h = hk * a->G + gi;
  const int64_t at = ((int64_t)b * a->H + h) * a->q_len + tok;
  if (a->split > 1) {
    const int64_t ap = (int64_t)sp * a->B * a->H * a->q_len + at;
    float* dst = a->part_out + ap * D + 4 * g;
#pragma unroll
    for (int db = 0; db < C::DB; ++db)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = o[db][4 * r4 + e] * inv;
        *(f32x4*)(dst + db * 32 + 8 * r4) = x;
      }
    if (g == 0) a->part_lse[ap] = lse;
  } else {
    __bf16* dst = (__bf16*)a->out + (((int64_t)b * a->q_len + tok) * a->H + h) * D + 8 * g;
#pragma unroll
    for (int db = 0; db < C::DB; ++db)
#pragma unroll
      for (int half = 0; half < 2; ++half) *(bf16x8*)(dst + 32 * db + 16 * half) = row_units(o[db], half, inv);
    if (g == 0 && a->lse != nullptr) a->lse[at] = lse;
  }
}

// The places of the live keys of every sequence, in order: one workgroup per
// sequence, 1,024 keys at a time (counts by ballot, waves in order).
__global__ __launch_bounds__(1024) void cross_list_kernel(const CrossArgs a) {
  __shared__ int sums[16];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = a.lens == nullptr ? a.kv_len : min(max(a.lens[b], 0), a.kv_len);
  const uint8_t* mask = a.mask + (int64_t)b * a.kv_len;
  int32_t* list = a.list + (int64_t)b * a.kv_len;
  int done = 0;
  for (int k0 = 0; k0 < n; k0 += 1024) {
    const int key = k0 + tid;
    const bool live = key < n && mask[key] != 0;
    const uint64_t votes = __builtin_amdgcn_ballot_w64(live);
    if (lane == 0) sums[wave] = __builtin_popcountll(votes);
    __syncthreads();
    int before = done, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      if (w < wave) before += sums[w];
      all += sums[w];
    }
    if (live) list[before + __builtin_popcountll(votes & ((1ull << lane) - 1))] = key;
    done += all;
    __syncthreads();
  }
  if (tid == 0) a.count[b] = done;
  if (b == 0 && tid < 128) a.zeros[tid] = 0.f;
}

// The rows of the live keys of every sequence, one after another, for a kernel
// whose tile loads take rows at a fixed distance.  A workgroup moves the rows
// of kPackKeys keys; where they go follows from the mask in front of them,
// which it counts by itself.
constexpr int kPackKeys = 16;
__global__ __launch_bounds__(256) void cross_pack_kernel(const CrossArgs a, int units) {
  __shared__ int sums[4];
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int k0 = blockIdx.x * kPackKeys;
  const int n = a.lens == nullptr ? a.kv_len : min(max(a.lens[b], 0), a.kv_len);
  const uint8_t* mask = a.mask + (int64_t)b * a.kv_len;
  int before = 0;
  for (int k = tid; k < min(k0, n); k += 256) before += mask[k] != 0;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) before += __shfl_xor(before, d, 64);
  if (lane == 0) sums[tid >> 6] = before;
  __syncthreads();
  int to = sums[0] + sums[1] + sums[2] + sums[3];
  for (int k = k0; k < min(k0 + kPackKeys, n); ++k) {
    if (mask[k] == 0) continue;
    const int64_t dst = ((int64_t)b * a.kv_len + to) * a.Hk * units;
    for (int i = tid; i < 2 * a.Hk * units; i += 256) {
      const bool v = i >= a.Hk * units;
      const int u = v ? i - a.Hk * units : i;
      const int64_t src = v ? b * a.v_batch + k * a.v_token + u / units * a.v_head
                            : b * a.k_batch + k * a.k_token + u / units * a.k_head;
      ((u32x4*)(v ? a.packed_v : a.packed_k))[dst + u] =
          *(const u32x4*)((const __bf16*)(v ? a.v : a.k) + src + u % units * 8);
    }
    ++to;
  }
  // the workgroup of the last keys has seen them all
  if (tid == 0 && blockIdx.x == gridDim.x - 1) a.count[b] = to;
}

// Composes the partial states of a split launch in the order of the key ranges:
// D / 4 lanes per row, of 16 bytes each.  Lane p of a row holds range p's weight
// (D / 4 ranges at a time), and the ranges' rows are loaded in batches.
template <typename T, int D>
__global__ __launch_bounds__(256) void cross_join_kernel(const CrossArgs a) {
  constexpr int TEAM = D / 4;
  const int64_t rows = (int64_t)a.B * a.H * a.q_len;
  const int64_t at = (int64_t)blockIdx.x * (256 / TEAM) + threadIdx.x / TEAM;
  const int64_t r = at < rows ? at : rows - 1;       // (a team past the end reads the last row)
  const int lane = threadIdx.x & (TEAM - 1), first = threadIdx.x & 63 & ~(TEAM - 1);
  const int b = (int)(r / a.q_len / a.H);
  // ranges of fixed length behind the sequence's end have not been written
  // (n + chunk may pass 31 bits)
  const int parts = a.chunk > 0 ? min(a.split, (int)(((uint32_t)cross_keys(a, b) + a.chunk - 1) / a.chunk)) : a.split;
  float mx = -INFINITY;
  bool bad = false;
  for (int p = lane; p < parts; p += TEAM) {
    const float x = a.part_lse[p * rows + r];
    bad |= x != x;
    mx = fmaxf(mx, x);
  }
#pragma unroll
  for (int d = 1; d < TEAM; d <<= 1) {
    mx = fmaxf(mx, __shfl_xor(mx, d, 64));
    bad |= __shfl_xor(bad ? 1 : 0, d, 64) != 0;
  }
  const float mm = mx == -INFINITY ? 0.f : mx;
  // The weights' sums, in units of 2^low: 0, or 16 where the outputs of some
  // ranges, near the type's largest, do not add up in float32 as they are (fewer
  // than 2^16 ranges).
  float tot, w, low = 0.f;
  f32x4 acc;
  const float* src = a.part_out + r * D + lane * 4;
  for (;;) {
    tot = 0.f;
    acc = f32x4{};
    for (int p0 = 0; p0 < parts; p0 += TEAM) {
      const float mine = p0 + lane < parts ? a.part_lse[(p0 + lane) * rows + r] : -INFINITY;
      w = fast_exp2((mine - mm) * 1.4426950408889634f - low);
      float sum = w;
#pragma unroll
      for (int d = 1; d < TEAM; d <<= 1) sum += __shfl_xor(sum, d, 64);
      tot += sum;
      const int np = min(parts - p0, TEAM);
      auto batch = [&](auto n, int q0) {
        constexpr int N = decltype(n)::value;
        f32x4 x[N];
#pragma unroll
        for (int q = 0; q < N; ++q) x[q] = *(const f32x4*)(src + (p0 + q0 + q) * rows * D);
#pragma unroll
        for (int q = 0; q < N; ++q) {
          const float wq = __shfl(w, first + q0 + q, 64);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(wq, x[q][e], acc[e]);
        }
      };
      int q0 = 0;
      for (; q0 + 8 <= np; q0 += 8) batch(std::integral_constant<int, 8>{}, q0);
      if (np & 4) batch(std::integral_constant<int, 4>{}, q0), q0 += 4;
      if (np & 2) batch(std::integral_constant<int, 2>{}, q0), q0 += 2;
      if (np & 1) batch(std::integral_constant<int, 1>{}, q0);
    }
    float hi = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) hi = __builtin_elementwise_maximum(hi, fabsf(acc[e]));
    if (low > 0.f || __builtin_amdgcn_ballot_w64(!(hi < INFINITY)) == 0) break;
    low = 16.f;
  }
  if (at >= rows) return;
  const float inv = tot > 0.f ? 1.0f / tot : bad ? NAN : 0.f;
  const int64_t tok = r % a.q_len, h = r / a.q_len % a.H;
  typedef T V __attribute__((ext_vector_type(4)));
  *(V*)((T*)a.out + ((b * a.q_len + tok) * a.H + h) * D + lane * 4) = __builtin_convertvector(acc * inv, V);
  if (lane == 0 && a.lse != nullptr)
    a.lse[r] = tot > 0.f ? mx + (__builtin_amdgcn_logf(tot) + low) * kLn2 : bad ? NAN : -INFINITY;
}

template <class C, int WPE, bool LIST>
hipError_t launch_rows_cfg(const CrossArgs& a0, hipStream_t s) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  e = set_kernel_lds<&cross_kernel<C, WPE, LIST>, C::LDS>(dev);
  if (e != hipSuccess) return e;
  CrossArgs a = a0;
  a.row_tiles = (a.rows + C::BM - 1) / C::BM;
  const int64_t grid = (int64_t)a.row_tiles * a.split * a.Hk * a.B;
  if (!launch_fits(grid, C::NT)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((cross_kernel<C, WPE, LIST>), dim3((unsigned)grid), dim3(C::NT), C::LDS, s, a);
  return hipGetLastError();
}
template <int D, bool LIST>
hipError_t launch_rows(const CrossArgs& a, hipStream_t s) {
  return launch_rows_cfg<RowsCfg<D, 4>, 2, LIST>(a, s);
}

// Estimated times in us of a launch of the two kernels that share a head's keys
// between many rows, with the split of the keys that is best for each (D=64 in
// brackets), fitted to launches of one card (100 ... 20,000 rows x 4 ... 40 heads,
// 77 ... 4,096 keys):
//  - kRows: w workgroups share a compute unit (one where there are fewer than
//    compute units, between one and two a compute unit n of them count as
//    (n + 2) / 2: some have a neighbour); a tile of 64 keys 0.96 w + 0.45
//    (0.54 w + 0.25), and 3.2 w + 2 (1.5 w + 2.5) beside the tiles;
//  - kTask: rounds of a task per compute unit, a tile 0.9 ... 1.4 (0.67 ...
//    0.89) by how full the card is (its clock falls), 7.25 (5) beside a round's
//    tiles and 3 once;
//  - a split's partial states and their join 4, and 0.45 per MB: 2 x 4,095 rows
//    x 12 heads against 2,048 keys 99 whole, 136 in two ranges; 300 x 40 against
//    4,096 74 whole, 51 in three.
// Lengths lie on the device: every sequence counts as kv_len keys.  A batch of
// different lengths is dealt out better than that by kTask, and where the two lie
// as near as 38.2 and 37.9 (2 x 4,095 rows x 12 heads, 512 keys) the choice is
// not by what its lengths take (512 and 77: kTask 30).
struct Estimate {
  double us;
  int split;
};
double split_us(int64_t s, double state_mb) { return s > 1 ? 4 + 0.45 * (double)s * state_mb : 0; }
Estimate estimate_rows(int64_t workgroups, int64_t tiles, int D, int cus, double state_mb) {
  Estimate best{1e30, 1};
  for (int64_t s = 1; s == 1 || (s <= tiles / 2 && s <= 64); ++s) {
    const double n = (double)(workgroups * s) / cus, w = n > 2 ? n : n > 1 ? (n + 2) / 2 : 1;
    const double tile = D == 128 ? 0.96 * w + 0.45 : 0.54 * w + 0.25, beside = D == 128 ? 3.2 * w + 2 : 1.5 * w + 2.5;
    const double us = (double)((tiles + s - 1) / s) * tile + beside + split_us(s, state_mb);
    if (us < best.us) best = {us, (int)s};
  }
  return best;
}
Estimate estimate_task(int64_t tasks, int64_t tiles, int D, int cus, double state_mb) {
  Estimate best{1e30, 1};
  for (int64_t s = 1; s == 1 || (s <= tiles / 8 && s <= 16); ++s) {
    const double rounds = (double)((tasks * s + cus - 1) / cus), full = (double)(tasks * s) / (rounds * cus);
    const double tile = D == 128 ? 0.9 + 0.5 * full : 0.67 + 0.22 * full, beside = D == 128 ? 7.25 : 5;
    const double us = rounds * ((double)((tiles + s - 1) / s) * tile + beside) + 3 + split_us(s, state_mb);
    if (us < best.us) best = {us, (int)s};
  }
  return best;
}

// The kernel a bf16 call runs, and its split.
//  - kFew for up to 32 rows of a key/value head: 8 x 24 heads, 8 of them with
//    keys, of one token against 16,384 keys 103 us (kRows 111), 12 heads against
//    77 keys 4.7 us (5.4).
//  - kResident where the keys fit LDS and its waves have work on them: one and a
//    half blocks of rows each over all heads, and two and a half of each head,
//    whose keys the waves wait for together: 9,450 rows x 40 heads against 256
//    keys 68 us (kRows 81, kTask 78), 20,000 x 8 against 256 33 (39, 41), 14,850 x
//    48 at D=64 against 512 112 (117, 137); but 9,450 x 12 against 256 33 (30,
//    29), and 64 x 8,192 at D=64 against 256 242 (kRows 136), 512 x 8,192 519
//    (422), 1,024 x 8,192 869 (856), 64 x 8,192 at D=128 against 320 441 (343).
//  - kTask or kRows as estimated: 9,450 x 40 against 512 keys 113 us (kRows 125),
//    against 1,024 183 (218); 700 x 24 against 512 19 (16).
void choose_form(const CrossArgs& a, int D, int cus, CrossPlan* p) {
  const int64_t heads = (int64_t)a.Hk * a.B, rows = a.rows, tiles = (a.kv_len + 63) / 64;
  if (rows <= 32) {
    p->form = CrossPlan::kFew;
    if (a.kv_len > 768) {
      // four workgroups for a compute unit, of 256 keys at least.  Where fewer
      // keys leave compute units idle a key of a range takes 7 ns and a range
      // 90 ns in the join: least together at sqrt(12.5 kv_len) keys (a token of
      // 8 heads on one head's 100,000 keys: 256 a range 42 us, 1,152 23 us;
      // 6 on 40,000: 25 us, 768 18 us)
      const int64_t want = (4 * (int64_t)cus + heads - 1) / heads;
      int64_t chunk = (a.kv_len + want - 1) / want;
      const int64_t least = (int64_t)sqrt(12.5 * a.kv_len);
      if (chunk < least) chunk = least;
      if (chunk < 256) chunk = 256;
      p->chunk = (int)((chunk + 127) / 128 * 128);
      p->split = (int)(((int64_t)a.kv_len + p->chunk - 1) / p->chunk);
    } else {
      p->chunk = a.kv_len;
    }
    return;
  }
  const int64_t blocks = (rows + 31) / 32, waves = cross_resident_waves(D);
  if (a.kv_len <= cross_resident_keys(D) && 2 * blocks * heads >= 3 * waves * cus && 2 * blocks >= 5 * waves) {
    p->form = CrossPlan::kResident;
    return;
  }
  const double state_mb = (double)a.B * a.H * a.q_len * D * 4e-6;
  const Estimate r = estimate_rows((rows + 127) / 128 * heads, tiles, D, cus, state_mb);
  p->split = r.split;
  CrossArgs t = a;
  if (a.mask != nullptr) t.k_token = t.v_token = (int64_t)a.Hk * D;     // as packed
  if (!cross_task_fits(t, D) || (a.mask != nullptr && a.B > 65535)) return;   // (the packing's grid)
  Estimate k = estimate_task((rows + 255) / 256 * heads, tiles, D, cus, state_mb);
  if (k.us < r.us) {
    p->form = CrossPlan::kTask;
    p->split = k.split;
  }
}

}  // namespace

hipError_t plan_cross(const CrossArgs& a, ditango_dtype dt, int D, CrossPlan* p) {
  *p = CrossPlan{CrossPlan::kRows, 1, 0, 0, 0};
  int dev = 0, cus = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return e;
  const size_t keys = (size_t)a.B * a.kv_len;
  if (dt == DITANGO_BF16) {
    choose_form(a, D, cus, p);
  } else {
    // a launch that leaves half the compute units idle splits its keys, two
    // tiles at least in each range
    const int bm = cross_f32_rows(a, D, cus);
    const int64_t groups = (int64_t)((a.rows + bm - 1) / bm) * a.Hk * a.B, tiles = (a.kv_len + 63) / 64;
    const int64_t split = 2 * groups <= cus ? 2 * (int64_t)cus / groups : 1;
    p->split = (int)(split < tiles / 2 ? split : tiles / 2 > 1 ? tiles / 2 : 1);
  }
  if (a.mask != nullptr)
    p->need = align_up256((size_t)a.B * 4) +
              (p->form == CrossPlan::kTask ? 2 * align_up256(keys * a.Hk * D * 2) : align_up256(keys * 4) + 512);
  p->bytes = p->need;
  if (p->split > 1) {
    const size_t rows = (size_t)a.B * a.H * a.q_len;
    p->bytes += align_up256(p->split * rows * D * 4) + align_up256(p->split * rows * 4);
  }
  return hipSuccess;
}

hipError_t launch_cross(const CrossArgs& a0, const CrossPlan& p, ditango_dtype dt, int D, void* ws, size_t ws_bytes,
                        hipStream_t s) {
  CrossArgs a = a0;
  hipError_t e = hipSuccess;
  char* w = (char*)ws;
  const size_t keys = (size_t)a.B * a.kv_len;
  if (a.mask != nullptr) {
    a.count = (int32_t*)w;
    char* at = w + align_up256((size_t)a.B * 4);
    if (p.form == CrossPlan::kTask) {
      a.packed_k = at;
      a.packed_v = at + align_up256(keys * a.Hk * D * 2);
      const dim3 grid((unsigned)((a.kv_len + kPackKeys - 1) / kPackKeys), (unsigned)a.B);
      hipLaunchKernelGGL(cross_pack_kernel, grid, dim3(256), 0, s, a, D / 8);
      // what follows sees the live keys as a prefix of dense rows
      a.k = a.packed_k;
      a.v = a.packed_v;
      a.k_head = a.v_head = D;
      a.k_token = a.v_token = (int64_t)a.Hk * D;
      a.k_batch = a.v_batch = a.kv_len * a.k_token;
      a.lens = a.count;
      a.mask = nullptr;
    } else if (p.form != CrossPlan::kResident || !cross_resident_lists(a, D)) {
      a.list = (int32_t*)at;
      a.zeros = (float*)(at + align_up256(keys * 4));
      hipLaunchKernelGGL(cross_list_kernel, dim3(a.B), dim3(1024), 0, s, a);
    }
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  // (one chunk, of all keys, without room for the partial states)
  a.split = 1;
  a.chunk = p.chunk > 0 ? a.kv_len : 0;
  const size_t rows = (size_t)a.B * a.H * a.q_len;
  if (p.split > 1 && ws_bytes >= p.bytes) {
    a.split = p.split;
    a.chunk = p.chunk;
    a.part_out = (float*)(w + p.need);
    a.part_lse = (float*)((char*)a.part_out + align_up256(p.split * rows * D * 4));
  }
  if (p.form == CrossPlan::kTask)
    e = launch_cross_task(a, D, s);
  else if (p.form == CrossPlan::kResident)
    e = launch_cross_resident(a, D, s);
  else if (p.form == CrossPlan::kFew)
    e = launch_cross_few(a, D, s);
  else if (dt == DITANGO_F32)
    e = launch_cross_f32(a, D, s);
  else if (D == 128)
    e = a.mask ? launch_rows<128, true>(a, s) : launch_rows<128, false>(a, s);
  else
    e = a.mask ? launch_rows<64, true>(a, s) : launch_rows<64, false>(a, s);
  if (e != hipSuccess || a.split == 1) return e;
  const int64_t per = 256 / (D / 4), join = ((int64_t)rows + per - 1) / per;
  if (!launch_fits(join, 256)) return hipErrorInvalidConfiguration;
  const dim3 grid((unsigned)join);
  if (dt == DITANGO_F32 && D == 128) hipLaunchKernelGGL((cross_join_kernel<float, 128>), grid, dim3(256), 0, s, a);
  if (dt == DITANGO_F32 && D == 64) hipLaunchKernelGGL((cross_join_kernel<float, 64>), grid, dim3(256), 0, s, a);
  if (dt == DITANGO_BF16 && D == 128) hipLaunchKernelGGL((cross_join_kernel<__bf16, 128>), grid, dim3(256), 0, s, a);
  if (dt == DITANGO_BF16 && D == 64) hipLaunchKernelGGL((cross_join_kernel<__bf16, 64>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace ditango
