// cross_task.hip - the cross attention of many query rows, bf16 (gfx950): the
// hand-scheduled key loop (cross_d128_loop.inc, cross_d64_loop.inc, written by
// gen_attn_loop.py) in workgroups that run one task after another.
//
// A task is 256 rows of one key/value head of one sequence, over all its live
// keys or a range of them: 4 waves, one per SIMD, two 32-row query blocks each,
// so that every fragment read from LDS feeds two MFMAs.  An encoder's states are
// few: at 512 keys a task is 8 key tiles, about as long as the memory latencies
// around it (queries in, rows out).  A workgroup per compute unit therefore
// stays: the next task's query rows come into registers of their own while the
// last three key tiles are worked on, its first tiles while the rows go out.
//
// Bound by the matrix core's power and, between tasks, by latency: of 32.8
// thousand cycles of a task of 512 keys 24.2 are the key loop (16.4 of them
// MFMAs), 9,450 rows x 40 heads take 117-122 us (830 TFLOP/s); 8,192 x 24 heads
// against 4,099 keys of 8 311-328 (1.26-1.33 PFLOP/s; 322-379 under a profiler,
// at lower clocks).
#include <type_traits>

#include "attn_tile.h"
#include "cross_d128_loop.inc"
#include "cross_d64_loop.inc"
#include "cross_tile.h"
#include "layer.h"

namespace ditango {
namespace {

template <int D_>
struct TaskCfg {
  static constexpr int D = D_, QB = 2, NW = 4, BN = 64;
  static constexpr int NT = NW * 64, BM = NW * QB * 32;
  static constexpr int KS = D / 16, DB = D / 32;
  static constexpr int ROWB = D * 2, UNITS = D / 8, RPL = 1024 / ROWB;
  static constexpr int TILEB = BN * ROWB;
  static constexpr int LW = TILEB / 1024 / NW;      // 1 KiB loads per wave and tile
  static constexpr int RING = 8 * TILEB;            // 4 K tiles, 4 V tiles
  static constexpr int STAGE = QB * 32 * ROWB;      // a wave's output rows
  static constexpr int EXTRA = RING + 1024;
  static constexpr int LDS = EXTRA + STAGE;
  static constexpr int NQ = QB * KS / 4;            // registers of query rows, by 16
  static_assert(STAGE == TILEB, "a wave's output rows take one ring slot, as a K and a V tile of 32 keys do");
  // Where a wave's output rows are staged: ring slots that the next task's
  // first tiles (K 0 ... 2, V 0 and 1) do not go to, then past the ring.
  static constexpr __device__ int stage(int wave) {
    return wave == 0 ? 3 * TILEB : wave == 1 ? 6 * TILEB : wave == 2 ? 7 * TILEB : EXTRA;
  }
};

// Bound on a lane's row sum below which the fast loop's result is the checked
// loop's (attn_bf16.hip), as long as the outputs are in range (cross_tile.h).
constexpr float kRowSumBound = 1099511627776.0f;   // 2^40

// x / d for wave-uniform 0 <= x < 2^31, with 2^32 / d rounded down (d = 1:
// 2^32 - 1): the product's high half is the quotient or one less.
__device__ __forceinline__ int divide(int x, int d, uint32_t inverse) {
  const int q = (int)__umulhi((uint32_t)x, inverse);
  return q + (x - q * d >= d ? 1 : 0);
}
inline uint32_t inverse_of(int d) { return d == 1 ? 0xffffffffu : (uint32_t)(((uint64_t)1 << 32) / (uint32_t)d); }

// The query blocks of `which` (a bit each) of a wave's rows, formed by wide_pass
// and stored.
template <int D>
__device__ __forceinline__ void form_again(Args a, int b, int hk, int part, int row0, int wave, uint32_t which,
                                           unsigned char* own) {
  using C = TaskCfg<D>;
  const int n = __builtin_amdgcn_readfirstlane(live_keys(a, b));
  const int per = ((n + C::BN - 1) / C::BN + a->split - 1) / a->split * C::BN;
  const int first = min(part * per, n), end = min(first + per, n);
  const int lane = lane_id();
  const int lr = lane & 31, g = lane >> 5;
  wait_loads();                                      // (the rows as stored first)
#pragma unroll 1
  for (int qb = 0; qb < C::QB; ++qb) {
    if ((which >> qb & 1) == 0) continue;
    const int r = (wave * C::QB + qb) * 32 + lr;
    int tok, gi;
    token_of(a, row0, r, &tok, &gi);
    const __bf16* p = (const __bf16*)a->q + b * a->q_batch + tok * a->q_token + (int64_t)(hk * a->G + gi) * a->q_head + 8 * g;
    bf16x8 qf[C::KS];
#pragma unroll
    for (int s = 0; s < C::KS; ++s) qf[s] = *(const bf16x8*)(p + 16 * s);
    f32x16 o[C::DB];
    float m, l;
    wide_pass<D, false>(a, b, hk, first, end, 32, own, qf, o, m, l);
    const float lt = pair_sum(l), inv = lt > 0.f ? 1.0f / lt : 0.f;
    const float lse = lt > 0.f ? (m + __builtin_amdgcn_logf(lt)) * kLn2 : lt == 0.f ? -INFINITY : lt;
    if (row0 + r >= a->rows) continue;
    const int h = hk * a->G + gi;
    const int64_t at = ((int64_t)b * a->H + h) * a->q_len + tok;
    if (a->split > 1) {
      const int64_t ap = (int64_t)part * a->B * a->H * a->q_len + at;
#pragma unroll
      for (int db = 0; db < C::DB; ++db)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = o[db][4 * r4 + e] * inv;
          *(f32x4*)(a->part_out + ap * D + 4 * g + db * 32 + 8 * r4) = x;
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
}

template <int D_>
__global__ __launch_bounds__(256, 1) void cross_task_kernel(const CrossArgs) {
  using C = TaskCfg<D_>;
  constexpr int D = C::D, QB = C::QB, KS = C::KS, DB = C::DB, LW = C::LW;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  // The block of assembly leaves no vector register and few scalar ones for
  // values that live across it: the lane is counted and the arguments are read
  // again behind it.
  Args a = args();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int lane = lane_id();
  int lr = lane & 31, g = lane >> 5;

  // This workgroup's tasks: of every class (the tasks of a sequence and key
  // range, or all where these are few) its XCD takes a contiguous eighth, whose
  // workgroups then share the K and V rows of a head, and the workgroup every
  // (gridDim / 8)-th of the eighths in turn: sequences of different lengths are
  // shared out evenly (2 x 4,095 rows x 12 heads against 512 and 77 keys 35 ->
  // 31 us).
  const int xcd = blockIdx.x & 7, step = gridDim.x >> 3;
  const int eighth = xcd_len(xcd, a->class_tasks), end = eighth * a->classes;
  int at = blockIdx.x >> 3;                          // in the XCD's list
  if (at >= end) return;
  const int eighth_first = xcd_first(xcd, a->class_tasks);
  const uint32_t eighth_inverse = eighth == 1 ? 0xffffffffu : __builtin_amdgcn_readfirstlane(0xffffffffu / (uint32_t)eighth);
  auto task_at = [&](Args a, int i) {
    const int c = divide(i, eighth, eighth_inverse);
    return c * a->class_tasks + eighth_first + (i - c * eighth);
  };

  // a task's sequence, key/value head, first row and key range
  struct Rows {
    int b, hk, row0, part;
  };
  auto rows_of = [](Args a, int t) {
    Rows r;
    const int u = divide(t, a->row_tiles, a->tiles_inverse), w = divide(u, a->Hk, a->heads_inverse);
    r.row0 = (t - u * a->row_tiles) * C::BM;
    r.hk = u - w * a->Hk;
    r.part = divide(w, a->B, a->batch_inverse);
    r.b = w - r.part * a->B;
    return r;
  };
  // its keys, and the first of them
  auto keys_of = [](Args a, const Rows& t, int* first) {
    const int n = __builtin_amdgcn_readfirstlane(live_keys(a, t.b));
    if (a->split == 1) {
      *first = 0;
      return n;
    }
    const int per = ((n + C::BN - 1) / C::BN + a->split - 1) / a->split * C::BN;
    *first = min(t.part * per, n);
    return min(per, n - *first);
  };
  const __bf16* qbase;
  uint32_t qoff[QB];
  auto query_rows = [&](Args a, const Rows& t) {
    const int tok0 = t.row0 / a->G;
    qbase = (const __bf16*)a->q + t.b * a->q_batch + tok0 * a->q_token + (int64_t)t.hk * a->G * a->q_head;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      int tok, gi;
      token_of(a, t.row0, (wave * QB + qb) * 32 + lr, &tok, &gi);
      qoff[qb] = (uint32_t)(tok - tok0) * (uint32_t)(a->q_token * 2) + (uint32_t)gi * (uint32_t)(a->q_head * 2) + 16u * g;
    }
  };
  f32x16 qn[C::NQ];
  auto load_queries = [&]() {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const f32x4 x = *(const f32x4*)((const char*)qbase + qoff[qb] + 32 * s);
#pragma unroll
        for (int e = 0; e < 4; ++e) qn[qb * (KS / 4) + s / 4][4 * (s % 4) + e] = x[e];
      }
  };

  const uint32_t smem_lds = lds_addr(smem);
  // this lane's LDS addresses and tile-load offsets, as the loop wants them
  uint32_t kaddr[KS], vaddr[DB], dmak[LW], dmav[LW];
  const uint32_t row_bytes = (uint32_t)a->k_token * 2;
#pragma unroll
  for (int s = 0; s < KS; ++s) kaddr[s] = smem_lds + lr * C::ROWB + (uint32_t)(((2 * s + g) ^ swz_k<D>(lr)) * 16);
  const int vrow = 4 * g + ((lane & 15) >> 2);
  const int vdim = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const int dim = 32 * db + vdim;
    vaddr[db] = smem_lds + C::RING / 2 + vrow * C::ROWB + (uint32_t)(((dim >> 3) ^ swz_v<D>(vrow)) * 16) + (dim & 7) * 2;
  }
  const int ld_row = lane / C::UNITS, ld_unit = lane % C::UNITS;
#pragma unroll
  for (int j = 0; j < LW; ++j) {
    // (load j adds j KiB to both of its addresses)
    const int row = (wave * LW + j) * C::RPL + ld_row;
    dmak[j] = row * row_bytes + (uint32_t)((ld_unit ^ swz_k<D>(row)) * 16) - 1024u * j;
    dmav[j] = row * row_bytes + (uint32_t)((ld_unit ^ swz_v<D>(row)) * 16) - 1024u * j;
  }
  const uint32_t wlds = __builtin_amdgcn_readfirstlane(smem_lds + (uint32_t)wave * (LW * 1024u));
  const uint32_t tileb = __builtin_amdgcn_readfirstlane(row_bytes * C::BN);

  // a task's first tiles (K 0 ... 2, V 0 and 1) on their way into the ring, and
  // the descriptors of what follows them
  auto first_tiles = [&](Args a, const Rows& t, int first, int n, u32x4* kd, u32x4* vd) {
    const uint32_t nrec = n > 0 ? (uint32_t)(n - 1) * row_bytes + C::ROWB : 0;
    *kd = buffer_desc((const __bf16*)a->k + t.b * a->k_batch + t.hk * a->k_head + first * a->k_token, nrec);
    *vd = buffer_desc((const __bf16*)a->v + t.b * a->v_batch + t.hk * a->v_head + first * a->v_token, nrec);
    if constexpr (D == 128) {
      asm volatile(DITANGO_CROSS_D128_LOAD_ASM
                   : "+{s[48:51]}"(*kd), "+{s[52:55]}"(*vd)
                   : "{v246}"(dmak[0]), "{v247}"(dmak[1]), "{v248}"(dmak[2]), "{v249}"(dmak[3]), "{v250}"(dmav[0]),
                     "{v251}"(dmav[1]), "{v252}"(dmav[2]), "{v253}"(dmav[3]), "{s44}"(wlds), "{s45}"(tileb)
                   : "m0", "scc", "memory");
    } else {
      asm volatile(DITANGO_CROSS_D64_LOAD_ASM
                   : "+{s[48:51]}"(*kd), "+{s[52:55]}"(*vd)
                   : "{v240}"(dmak[0]), "{v241}"(dmak[1]), "{v242}"(dmav[0]), "{v243}"(dmav[1]), "{s44}"(wlds),
                     "{s45}"(tileb)
                   : "m0", "scc", "memory");
    }
  };
  // this wave's loads have landed
  auto landed = [] { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };

  // a task's flag of a second pass, of three in turn: the one cleared here is
  // two tasks old, and every wave has passed a barrier since it was read
  int* redo = (int*)(smem + C::RING);
  if (threadIdx.x < 3) redo[threadIdx.x] = 0;
  int turn = 0;

  Rows t = rows_of(a, task_at(a, at));
  query_rows(a, t);
  load_queries();
  int key0, n = keys_of(a, t, &key0);
  u32x4 kd, vd;
  first_tiles(a, t, key0, n, &kd, &vd);
  landed();
  __syncthreads();
  for (;;) {
    a = args();
    const bool more = at + step < end;
    const Rows next = more ? rows_of(a, task_at(a, at + step)) : t;
    f32x16 q[C::NQ];
#pragma unroll
    for (int i = 0; i < C::NQ; ++i) q[i] = qn[i];
    query_rows(a, next);
    const int clear = turn == 2 ? 0 : turn + 1;
    if (wave == 0 && lane == 0) redo[clear] = 0;

    f32x16 o[QB][DB];
    float m[QB], l[QB];
    // the loop over the keys; `checked` tests every tile for the maximum
    auto key_loop = [&](auto checked) {
      a = args();
      // (without keys: one tile of zeros, whose sum and products are dropped below)
      const uint32_t ntiles = (uint32_t)((max(n, 1) + C::BN - 1) / C::BN), kvl = (uint32_t)n;
      const float sl2 = a->scale_log2;
      if constexpr (D == 128) {
#define DITANGO_CALL(BODY)                                                                                            \
asm volatile(BODY                                                                                                   \
             : "={a[0:15]}"(o[0][0]), "={a[16:31]}"(o[0][1]), "={a[32:47]}"(o[0][2]), "={a[48:63]}"(o[0][3]),      \
               "={a[64:79]}"(o[1][0]), "={a[80:95]}"(o[1][1]), "={a[96:111]}"(o[1][2]), "={a[112:127]}"(o[1][3]),   \
               "={v230}"(m[0]), "={v231}"(m[1]), "={v232}"(l[0]), "={v233}"(l[1]),                                  \
               "+{s[48:51]}"(kd), "+{s[52:55]}"(vd), "+{a[128:143]}"(q[0]), "+{a[144:159]}"(q[1]),                  \
               "+{a[160:175]}"(q[2]), "+{a[176:191]}"(q[3]), "={a[192:207]}"(qn[0]), "={a[208:223]}"(qn[1]),        \
               "={a[224:239]}"(qn[2]), "={a[240:255]}"(qn[3])                                                       \
             : "{v234}"(kaddr[0]), "{v235}"(kaddr[1]), "{v236}"(kaddr[2]), "{v237}"(kaddr[3]),                      \
               "{v238}"(kaddr[4]), "{v239}"(kaddr[5]), "{v240}"(kaddr[6]), "{v241}"(kaddr[7]),                      \
               "{v242}"(vaddr[0]), "{v243}"(vaddr[1]), "{v244}"(vaddr[2]), "{v245}"(vaddr[3]),                      \
               "{v246}"(dmak[0]), "{v247}"(dmak[1]), "{v248}"(dmak[2]), "{v249}"(dmak[3]),                          \
               "{v250}"(dmav[0]), "{v251}"(dmav[1]), "{v252}"(dmav[2]), "{v253}"(dmav[3]),                          \
               "{v254}"(qoff[0]), "{v255}"(qoff[1]), "{s[68:69]}"(qbase),                                           \
               "{s40}"(sl2), "{s41}"(ntiles), "{s42}"(kvl), "{s44}"(wlds), "{s45}"(tileb)                           \
             : DITANGO_CROSS_D128_LOOP_CLOBBERS)
        if constexpr (decltype(checked)::value) {
          DITANGO_CALL(DITANGO_CROSS_D128_LOOP_ASM);
        } else {
          DITANGO_CALL(DITANGO_CROSS_D128_FAST_ASM);
        }
#undef DITANGO_CALL
      } else {
#define DITANGO_CALL(BODY)                                                                                            \
asm volatile(BODY                                                                                                   \
             : "={a[0:15]}"(o[0][0]), "={a[16:31]}"(o[0][1]), "={a[32:47]}"(o[1][0]), "={a[48:63]}"(o[1][1]),      \
               "={v230}"(m[0]), "={v231}"(m[1]), "={v232}"(l[0]), "={v233}"(l[1]),                                  \
               "+{s[48:51]}"(kd), "+{s[52:55]}"(vd), "+{a[128:143]}"(q[0]), "+{a[160:175]}"(q[1]),                  \
               "={a[192:207]}"(qn[0]), "={a[224:239]}"(qn[1])                                                       \
             : "{v234}"(kaddr[0]), "{v235}"(kaddr[1]), "{v236}"(kaddr[2]), "{v237}"(kaddr[3]),                      \
               "{v238}"(vaddr[0]), "{v239}"(vaddr[1]), "{v240}"(dmak[0]), "{v241}"(dmak[1]),                        \
               "{v242}"(dmav[0]), "{v243}"(dmav[1]),                                                                \
               "{v254}"(qoff[0]), "{v255}"(qoff[1]), "{s[68:69]}"(qbase),                                           \
               "{s40}"(sl2), "{s41}"(ntiles), "{s42}"(kvl), "{s44}"(wlds), "{s45}"(tileb)                           \
             : DITANGO_CROSS_D64_LOOP_CLOBBERS)
        if constexpr (decltype(checked)::value) {
          DITANGO_CALL(DITANGO_CROSS_D64_LOOP_ASM);
        } else {
          DITANGO_CALL(DITANGO_CROSS_D64_FAST_ASM);
        }
#undef DITANGO_CALL
      }
      lane = lane_id();
      lr = lane & 31, g = lane >> 5;
    };
    key_loop(std::false_type{});
    // The fast form's sums may be too large, or not numbers: then the task
    // runs again in the checked form.  The barrier also says that every
    // wave's reads of the ring are done.
    const bool over = !(l[0] <= kRowSumBound && l[1] <= kRowSumBound);
    if (__builtin_amdgcn_ballot_w64(over) != 0 && lane == 0) redo[turn] = 1;
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(redo[turn]) != 0) {
      // (the queries are not kept beside the next task's)
      a = args();
      query_rows(a, t);
      load_queries();
#pragma unroll
      for (int i = 0; i < C::NQ; ++i) q[i] = qn[i];
      query_rows(a, next);
      first_tiles(a, t, key0, n, &kd, &vd);
      landed();
      key_loop(std::true_type{});
      __syncthreads();
    }
    turn = clear;
    a = args();
    // the next task's first tiles come in while this one's rows go out; the
    // rows' stores wait for them, because the waits of the loop go by order
    const bool keys = n > 0;
    n = keys_of(a, next, &key0);
    first_tiles(a, next, key0, n, &kd, &vd);
    lane = lane_id();
    lr = lane & 31, g = lane >> 5;
    // (without keys the tile of zeros leaves NaN where a query is no number)
    if (!keys) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int db = 0; db < DB; ++db) o[qb][db] = f32x16{};
    }
    // the query blocks whose state left the range
    uint32_t again = 0;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
      if (keys && __builtin_amdgcn_ballot_w64(out_of_range<DB>(o[qb], m[qb])) != 0) again |= 1u << qb;

    if (a->split > 1) {
      // ---- the partial state of a key range, as it lies in the registers
      landed();
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const float lt = keys ? pair_sum(l[qb]) : 0.f;
        const float inv = lt > 0.f ? 1.0f / lt : 0.f;
        const int r = (wave * QB + qb) * 32 + lr;
        if (t.row0 + r < a->rows) {
          int tok, gi;
          token_of(a, t.row0, r, &tok, &gi);
          const int64_t at = (((int64_t)t.part * a->B + t.b) * a->H + t.hk * a->G + gi) * a->q_len + tok;
          float* dst = a->part_out + at * D + 4 * g;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
              f32x4 x;
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = o[qb][db][4 * r4 + e] * inv;
              *(f32x4*)(dst + db * 32 + 8 * r4) = x;
            }
          if (g == 0)
            a->part_lse[at] = lt > 0.f ? (m[qb] + __builtin_amdgcn_logf(lt)) * kLn2 : lt == 0.f ? -INFINITY : lt;
        }
      }
    } else {
      // ---- the rows' state: through LDS (16-byte units swizzled by row, the
      // halves of a unit by row / 16), then stored whole
      unsigned char* stage = smem + C::stage(wave);
      auto swz_out = [](int row) { return row & (C::UNITS - 1); };
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const float lt = keys ? pair_sum(l[qb]) : 0.f;
        const float inv = lt > 0.f ? 1.0f / lt : 0.f;
        unsigned char* srow = stage + (qb * 32 + lr) * C::ROWB;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4) {
            f32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = o[qb][db][4 * r4 + e] * inv;
            const int unit = (4 * db + r4) ^ swz_out(qb * 32 + lr);
            *(bf16x4*)(srow + unit * 16 + 8 * (g ^ ((lr >> 4) & 1))) = __builtin_convertvector(x, bf16x4);
          }
        l[qb] = lt;
      }
      const int out_row = lane / C::UNITS, out_unit = lane % C::UNITS;
      bf16x8 x[QB * 32 / C::RPL];
#pragma unroll
      for (int i = 0; i < QB * 32 / C::RPL; ++i) {
        const int row = i * C::RPL + out_row;
        x[i] = *(const bf16x8*)(stage + row * C::ROWB + ((out_unit ^ swz_out(row)) * 16));
        if ((row >> 4) & 1) x[i] = __builtin_shufflevector(x[i], x[i], 4, 5, 6, 7, 0, 1, 2, 3);
      }
      landed();
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        const int r = (wave * QB + qb) * 32 + lr;
        if (g == 0 && a->lse != nullptr && t.row0 + r < a->rows) {
          int tok, gi;
          token_of(a, t.row0, r, &tok, &gi);
          a->lse[((int64_t)t.b * a->H + t.hk * a->G + gi) * a->q_len + tok] =
              l[qb] > 0.f ? (m[qb] + __builtin_amdgcn_logf(l[qb])) * kLn2 : l[qb] == 0.f ? -INFINITY : l[qb];
        }
      }
      const int64_t out_row_elems = (int64_t)a->H * D;
      __bf16* out = (__bf16*)a->out + ((int64_t)t.b * a->q_len * a->H + t.hk * a->G) * D + out_unit * 8;
      if (a->G == 1) {
        // rows at a fixed distance
        const int r0 = t.row0 + wave * QB * 32 + out_row;
        __bf16* p = out + r0 * out_row_elems;
#pragma unroll
        for (int i = 0; i < QB * 32 / C::RPL; ++i) {
          if (r0 + i * C::RPL < a->rows) __builtin_nontemporal_store(x[i], (bf16x8*)p);
          p += C::RPL * out_row_elems;
        }
      } else {
#pragma unroll
        for (int i = 0; i < QB * 32 / C::RPL; ++i) {
          const int r = wave * QB * 32 + i * C::RPL + out_row;
          if (t.row0 + r < a->rows) {
            int tok, gi;
            token_of(a, t.row0, r, &tok, &gi);
            __builtin_nontemporal_store(x[i], (bf16x8*)(out + tok * out_row_elems + gi * D));
          }
        }
      }
    }
    // ---- those that left the range: once more, by this wave alone, over the
    // rows as stored, in the LDS they were staged in
    if (again != 0) form_again<D>(a, t.b, t.hk, t.part, t.row0, wave, again, smem + C::stage(wave));
    if (!more) break;
    at += step;
    t = next;
  }
}

template <int D>
hipError_t launch_task(const CrossArgs& a0, int cus, int dev, hipStream_t s) {
  using C = TaskCfg<D>;
  const hipError_t e = set_kernel_lds<&cross_task_kernel<D>, C::LDS>(dev);
  if (e != hipSuccess) return e;
  CrossArgs a = a0;
  a.row_tiles = (a.rows + C::BM - 1) / C::BM;
  const int64_t tasks = (int64_t)a.row_tiles * a.Hk * a.B * a.split;
  if (tasks > 0x7fffffff - 4096) return hipErrorInvalidConfiguration;
  // classes where each gives an XCD eight tasks
  const int64_t one = (int64_t)a.row_tiles * a.Hk;
  a.class_tasks = (int)(one >= 64 ? one : tasks);
  a.classes = one >= 64 ? a.B * a.split : 1;
  a.tiles_inverse = inverse_of(a.row_tiles);
  a.heads_inverse = inverse_of(a.Hk);
  a.batch_inverse = inverse_of(a.B);
  const int64_t per_xcd = (int64_t)a.classes * ((a.class_tasks + 7) / 8), most = cus / 8 > 0 ? cus / 8 : 1;
  const int grid = (int)(8 * (per_xcd < most ? per_xcd : most));
  hipLaunchKernelGGL((cross_task_kernel<D>), dim3((unsigned)grid), dim3(C::NT), C::LDS, s, a);
  return hipGetLastError();
}

}  // namespace

bool cross_task_fits(const CrossArgs& a, int D) {
  // K and V share their tiles' distance; a head's keys lie within the tile
  // loads' 32-bit bounds, a task's query rows within 32-bit offsets
  return a.k_token == a.v_token && a.k_token >= D && (int64_t)a.kv_len * a.k_token * 2 < ((int64_t)1 << 31) &&
         a.q_token < (1 << 21) && a.q_head < (1 << 21) && a.G <= 256;
}

hipError_t launch_cross_task(const CrossArgs& a, int D, hipStream_t s) {
  int dev = 0, cus = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return e;
  return D == 128 ? launch_task<128>(a, cus, dev, s) : launch_task<64>(a, cus, dev, s);
}

}  // namespace ditango
