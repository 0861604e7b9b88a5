// attn_f32.hip - fresh attention states of selected key/value partitions,
// float32 inputs and states (gfx950).
//
// Same computation as the bf16 kernel (the blocked attention state of Sec.
// 2.2.4, Eq. attention_state, by online softmax over key tiles), in float32
// precision.  Scores are computed transposed, S^T = K Q^T, so that each lane
// holds one query's scores; the output is accumulated as O^T = V^T P^T.
//
// Products
//   The float32 MFMA runs at a sixteenth of the bf16 one.  Every float32
//   operand x is split into three bf16 planes, x = x1 + x2 + x3 (each the
//   rounding of what the planes before it leave: 3 x 8 bits, exact), and a
//   product is the sum of six bf16 MFMAs with float32 accumulation,
//     x3 y1 + x2 y2 + x1 y3 + x2 y1 + x1 y2 + x1 y1,
//   6/16 of the float32 MFMA's time.  The three products left out come to at
//   most 2^-24 |x y| (two of 2^-8 x 2^-17; the rounding of one float32
//   product) and to 2^-27 ... 2^-26.5 as a root mean square, and there are
//   fewer accumulations: against 64 bits, OUT is off by
//   2e-7 ... 7e-7 (norm ratio, 1,000 ... 2,000 keys) where the float32 MFMA's
//   was off by 5e-7 ... 9e-7; LSE is the same.  The scores' five small terms
//   have an accumulator of their own.
//   What the planes cannot hold goes through the float32 MFMA: a workgroup
//   runs its task again with it
//    - where some row's sum or output ends up not finite, or beyond 2^120, or
//      its maximum at 2^24 or more (state_out_of_range).  A value that is not
//      finite, or rounds to infinity in bf16, gives NaN in the planes and in
//      every row it enters; the float32 MFMA treats infinities as float32
//      arithmetic does;
//    - where nonzero values below 2^-110 matter.  Their third plane falls
//      under bf16's smallest subnormal (2^-133), so such a value is off by up
//      to 2^-134.  Its queries are looked at as they are split: one of these
//      values, or one so large (2^100 after scaling) that what a key of this
//      kind is off by would show in the scores (below it: 2^-27 at most).  In
//      V the error is under 2^-34 of an output of 2^-100 or more, so V is
//      looked through only where some output is smaller or zero (a column of
//      zeros in V: 7,750 keys in the 128-row form 670 -> 753 us; 2,000 keys
//      and 24 heads in the 256-row form 890 -> 938).
//   Probabilities under 2^-110 are off by 2^-134 too: OUT by 2^-134 max|v|.
//
// Work decomposition
//   A workgroup has RW x KW waves and 32 * RW query rows of one (partition,
//   batch, head).  RW waves share 32-key tiles: together they load a tile's
//   float32 rows, split them once and write the planes to LDS, double
//   buffered.  With KW > 1 the waves split the partition's keys instead
//   (RW = 1): each wave stages its own tiles in its own LDS, without
//   barriers, and the KW partial states are composed through LDS at the end.
//
// What bounds it: at D=128 the MFMAs (96 per wave and tile, busy 69 % of the
// cycles at 1.84 GHz); at D=64 MFMAs and vector work alike (48 MFMAs, busy
// 53-58 %, beside about 280 vector instructions: the planes of the staged
// tile and of the probabilities take 11 per pair of values).
#include "attn_f32_loop.h"
#include "internal.h"
#include "kernel_lds.h"

namespace ditango {
namespace {

template <class C>
__global__ __launch_bounds__(C::NT, C::WPE) void attn_f32_kernel(const AttnArgs a) {
  constexpr int D = C::D;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];

  const int task = xcd_remap(blockIdx.x, gridDim.x);
  const int qt = task % a.q_tiles;
  int t = task / a.q_tiles;
  const int h = t % a.H;
  t /= a.H;
  const int b = t % a.B;
  const int sel = t / a.B;

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31;
  const int g = lane >> 5;

  const int64_t HD = (int64_t)a.H * D;
  const int kv_len = a.kv_len[sel];
  const int64_t kv0 = a.kv_begin[sel];
  const int slot = a.slot[sel];
  const float* kg = (const float*)a.k + ((int64_t)b * a.S + kv0) * HD + (int64_t)h * D;
  const float* vg = (const float*)a.v + ((int64_t)b * a.S + kv0) * HD + (int64_t)h * D;
  const StridedRows kr{kg, HD}, vr{vg, HD};
  const int rl = (C::KW == 1 ? wave * 32 : 0) + lr;          // row within the workgroup's tile
  const int64_t row = (int64_t)qt * C::BM + rl;
  const bool row_ok = row < a.q_len;
  const float* qrow = (const float*)a.q + (int64_t)b * a.q_stride + (row_ok ? row : 0) * HD + (int64_t)h * D;

  // this wave's key tiles, and its tile space in LDS
  const int tiles = (kv_len + C::BN - 1) / C::BN;
  const int per = (tiles + C::KW - 1) / C::KW;
  const int kw = C::KW == 1 ? 0 : wave;
  const int t0 = min(kw * per, tiles), t1 = min(t0 + per, tiles);
  unsigned char* kb = smem + kw * C::GROUP;
  const int gt = C::KW == 1 ? tid : lane;
  float* part_m = (float*)(smem + C::KW * C::GROUP);         // [KW][32] maximum, then [KW][32] row sum
  float* part_l = part_m + C::KW * 32;
  // run the task again; look through V; V asks for it; run it again for a state
  // out of range (a word each: a wave may still be reading one when another
  // writes the next)
  int* redo = (int*)(part_l + C::KW * 32);

  f32x16 o[C::DB];
  float m, l;
  if (tid < 4) redo[tid] = 0;
  uint64_t ask = 0;
  key_loop<C, true>(qrow, row_ok, kr, vr, kv_len, t0, t1, a.scale_log2, kb, gt, o, m, l, ask);
  const bool range = t0 < t1 && state_out_of_range(o, m, l);
  float small_o = INFINITY;
#pragma unroll
  for (int db = 0; db < C::DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) small_o = fminf(small_o, fabsf(o[db][r]));
  const float below = pair_sum(l) * 0x1p-100f;
  const bool small = row_ok && small_o < below;
  __syncthreads();
  if (ask != 0 && lane == 0) redo[0] = 1;
  if (__builtin_amdgcn_ballot_w64(range) != 0 && lane == 0) redo[3] = 1;
  if (__builtin_amdgcn_ballot_w64(small) != 0 && lane == 0) redo[1] = 1;
  __syncthreads();
  const bool far = __builtin_amdgcn_readfirstlane(redo[3]) != 0;
  bool again = far || __builtin_amdgcn_readfirstlane(redo[0]) != 0;
  if (!again && __builtin_amdgcn_readfirstlane(redo[1]) != 0) {
    constexpr int kBatch = 8;                                // loads in flight
    const int64_t units = (int64_t)kv_len * (D / 4);
    bool found = false;
    for (int64_t i0 = tid; i0 < units; i0 += kBatch * C::NT) {
      f32x4 x[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int64_t u = min(i0 + i * C::NT, units - 1);
        x[i] = *(const f32x4*)(vg + u / (D / 4) * HD + u % (D / 4) * 4);
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) found |= below_planes(x[i][e]);
    }
    if (__builtin_amdgcn_ballot_w64(found) != 0 && lane == 0) redo[2] = 1;
    __syncthreads();
    again = __builtin_amdgcn_readfirstlane(redo[2]) != 0;
  }
  if (again) {
    key_loop<C, false>(qrow, row_ok, kr, vr, kv_len, t0, t1, a.scale_log2, kb, gt, o, m, l, ask,
                       far ? wide_low(kv_len) : 0.f);
    __syncthreads();
  }

  const float lt = pair_sum(l);
  const int64_t slot_elems = (int64_t)a.B * a.q_len * HD;
  float* outg = (float*)a.out_states + (int64_t)slot * slot_elems + (int64_t)b * a.q_len * HD + (int64_t)h * D;
  float* lseg = a.lse_states + (((int64_t)slot * a.B + b) * a.H + h) * a.q_len;
  if constexpr (C::KW == 1) {
    if (row_ok) {
      const float inv = lt > 0.f ? 1.0f / lt : 0.f;
      float* dst = outg + row * HD + 4 * g;
#pragma unroll
      for (int db = 0; db < C::DB; ++db)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = o[db][4 * r4 + e] * inv;
          *(f32x4*)(dst + db * 32 + 8 * r4) = x;
        }
      if (g == 0) lseg[row] = lt > 0.f ? (m + __builtin_amdgcn_logf(lt)) * kLn2 : -INFINITY;
    }
  } else {
    // partial states through LDS: O rows of 16-byte units, swizzled by row
    float* po = (float*)kb;
#pragma unroll
    for (int db = 0; db < C::DB; ++db)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = o[db][4 * r4 + e];
        *(f32x4*)(po + lr * D + (((8 * db + 2 * r4 + g) ^ (lr & 15)) * 4)) = x;
      }
    if (g == 0) {
      part_m[kw * 32 + lr] = m;
      part_l[kw * 32 + lr] = lt;
    }
    __syncthreads();
    constexpr int CH = 32 * D / 4;
    static_assert(CH % C::NT == 0, "chunks divide over the threads");
#pragma unroll
    for (int i = 0; i < CH / C::NT; ++i) {
      const int c = tid + i * C::NT;
      const int r = c / (D / 4), u = c % (D / 4);
      if ((int64_t)qt * C::BM + r >= a.q_len) continue;
      float mk[C::KW], M = -INFINITY;
#pragma unroll
      for (int k = 0; k < C::KW; ++k) {
        mk[k] = part_m[k * 32 + r];
        M = fmaxf(M, mk[k]);
      }
      float tot = 0.f;
      f32x4 acc = f32x4{};
#pragma unroll
      for (int k = 0; k < C::KW; ++k) {
        // a range without keys has m = -inf, sum 0 and output 0
        const float w = mk[k] == -INFINITY && part_l[k * 32 + r] == 0.f ? 0.f : fast_exp2(mk[k] - M);
        tot = __builtin_fmaf(w, part_l[k * 32 + r], tot);
        acc += w * *(const f32x4*)((const float*)(smem + k * C::GROUP) + r * D + ((u ^ (r & 15)) * 4));
      }
      const float inv = tot > 0.f ? 1.0f / tot : 0.f;
      *(f32x4*)(outg + ((int64_t)qt * C::BM + r) * HD + u * 4) = acc * inv;
      if (u == 0) lseg[(int64_t)qt * C::BM + r] = tot > 0.f ? (M + __builtin_amdgcn_logf(tot)) * kLn2 : -INFINITY;
    }
  }
}

template <class C>
hipError_t launch_cfg_f(const AttnArgs& a0, int dev, hipStream_t s) {
  const hipError_t attr = set_kernel_lds<&attn_f32_kernel<C>, C::LDS>(dev);
  if (attr != hipSuccess) return attr;
  AttnArgs a = a0;
  a.q_tiles = (int)((a.q_len + C::BM - 1) / C::BM);
  const int64_t nblk = (int64_t)a.q_tiles * a.H * a.B * a.n_sel;
  if (nblk <= 0) return hipSuccess;
  if (nblk > 0x7fffffff) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((attn_f32_kernel<C>), dim3((unsigned)nblk), dim3(C::NT), C::LDS, s, a);
  return hipGetLastError();
}

// Which form a launch runs, by how its workgroups fill the compute units
// (times on one card, float32 MFMA kernel before / the forms of this one):
//  - Split, 32 rows and all the waves on one tile of rows, up to two rounds.
//    It splits every key tile per 32 rows and is bound by that vector work,
//    but fills the chip with the fewest rows: 1,024 rows x 2 heads x 4
//    partitions of 1,024 keys at D=64 24 us (93; Shared 52), 1,024 rows x 4
//    heads x 2 partitions at D=128 45 us (161; Shared 114).  At three rounds
//    Mid and Shared are as fast.
//  - Mid, 128 rows, while every workgroup has a compute unit to itself: one
//    wave per SIMD (D=128; 7,750 rows x 4 heads x 7,750 keys 654 us, Shared
//    815, Split 1,062).  At D=64 two workgroups share a compute unit and
//    Mid is Shared.
//  - Shared otherwise: 256 rows at D=128, two waves per SIMD (2,000 rows x 24
//    heads x 4 partitions of 2,000 keys: 0.88 ms, 224 TFLOP/s, MFMAs busy
//    69 %, against 1.87 ms and 105 TFLOP/s; Mid 1.13 ms); 128 rows at D=64
//    (the same: 0.51 ms, 194 TFLOP/s, against 0.93 ms and 106 TFLOP/s; with
//    the scores not pipelined 0.55 ms).
template <class Shared, class Mid, class Split>
hipError_t launch_f32(const AttnArgs& a, hipStream_t s) {
  int dev = 0, cus = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return e;
  const int64_t tiles = (int64_t)a.H * a.B * a.n_sel;
  if ((a.q_len + Split::BM - 1) / Split::BM * tiles <= 2 * (int64_t)cus) return launch_cfg_f<Split>(a, dev, s);
  if ((a.q_len + Mid::BM - 1) / Mid::BM * tiles <= cus) return launch_cfg_f<Mid>(a, dev, s);
  return launch_cfg_f<Shared>(a, dev, s);
}

}  // namespace

hipError_t launch_attn_f32(const AttnArgs& a, int D, hipStream_t s) {
  if (D == 128)
    return launch_f32<CfgF<128, 8, 1, 2, false>, CfgF<128, 4, 1, 1, true>, CfgF<128, 1, 4, 1, false>>(a, s);
  if (D == 64) return launch_f32<CfgF<64, 4, 1, 2, true>, CfgF<64, 4, 1, 2, true>, CfgF<64, 1, 8, 2, false>>(a, s);
  return hipErrorInvalidValue;
}

}  // namespace ditango
