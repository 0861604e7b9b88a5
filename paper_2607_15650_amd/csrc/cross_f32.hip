// cross_f32.hip - the cross attention of cross.hip for float32 inputs
// (gfx950): the key loop of attn_f32_loop.h (float32 products as six bf16
// MFMAs) over rows that are strided or listed, and the same second pass with
// the float32 MFMA where the planes cannot hold a value.
//
// As there, a workgroup has RW x KW waves: RW of them share the key tiles, 32
// rows each, or (RW = 1) KW of them split the keys of its range, stage their own
// tiles without barriers, and compose their partial states through LDS.
#include "attn_f32_loop.h"
#include "layer.h"

namespace ditango {
namespace {

template <class C, class Rows>
__global__ __launch_bounds__(C::NT, C::WPE) void cross_f32_kernel(const CrossArgs a) {
  constexpr int D = C::D;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];

  int t = xcd_remap(blockIdx.x, gridDim.x);
  const int rt = t % a.row_tiles;
  t /= a.row_tiles;
  const int sp = t % a.split;
  t /= a.split;
  const int hk = t % a.Hk;
  const int b = t / a.Hk;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, g = lane >> 5;

  const int n = __builtin_amdgcn_readfirstlane(cross_keys(a, b));
  const int all = (n + C::BN - 1) / C::BN;
  const int tiles_per = (all + a.split - 1) / a.split;
  const int tb = min(sp * tiles_per, all), te = min(tb + tiles_per, all);
  const int kv_len = n;

  Rows kr, vr;
  kr.base = (const float*)a.k + b * a.k_batch + hk * a.k_head;
  vr.base = (const float*)a.v + b * a.v_batch + hk * a.v_head;
  kr.stride = a.k_token;
  vr.stride = a.v_token;
  if constexpr (Rows::kListed) kr.list = vr.list = a.list + (int64_t)b * a.kv_len;

  const int row = rt * C::BM + (C::KW == 1 ? wave * 32 : 0) + lr;
  const bool row_ok = row < a.rows;
  const int tok = min(row, a.rows - 1) / a.G, gi = min(row, a.rows - 1) % a.G;
  const float* qrow = (const float*)a.q + b * a.q_batch + tok * a.q_token + (int64_t)(hk * a.G + gi) * a.q_head;

  const int kw = C::KW == 1 ? 0 : wave;
  const int per = (te - tb + C::KW - 1) / C::KW;
  const int t0 = min(tb + kw * per, te), t1 = min(t0 + per, te);
  unsigned char* kb = smem + kw * C::GROUP;
  const int gt = C::KW == 1 ? tid : lane;
  float* part_m = (float*)(smem + C::KW * C::GROUP);
  float* part_l = part_m + C::KW * 32;
  int* redo = (int*)(part_l + C::KW * 32);

  f32x16 o[C::DB];
  float m, l;
  if (tid < 4) redo[tid] = 0;
  uint64_t ask = 0;
  key_loop<C, true>(qrow, row_ok, kr, vr, kv_len, t0, t1, a.scale_log2, kb, gt, o, m, l, ask);
  // what the planes cannot hold, as attn_f32_kernel finds it
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
    constexpr int kBatch = 8;
    const int first = tb * C::BN;
    const int64_t units = (int64_t)(min(te * C::BN, n) - first) * (D / 4);
    bool found = false;
    for (int64_t i0 = tid; i0 < units; i0 += kBatch * C::NT) {
      f32x4 x[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int64_t u = min(i0 + i * C::NT, units - 1);
        x[i] = *(const f32x4*)(vr.row(first + (int)(u / (D / 4))) + u % (D / 4) * 4);
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
                       far ? wide_low(n) : 0.f);
    __syncthreads();
  }

  const float lt = pair_sum(l);
  if constexpr (C::KW == 1) {
    if (row_ok) {
      const float inv = lt > 0.f ? 1.0f / lt : 0.f;
      const float lse = lt > 0.f ? (m + __builtin_amdgcn_logf(lt)) * kLn2 : lt == 0.f ? -INFINITY : lt;
      const int h = hk * a.G + gi;
      const int64_t at = ((int64_t)b * a.H + h) * a.q_len + tok, ap = (int64_t)sp * a.B * a.H * a.q_len + at;
      float* dst = (a.split > 1 ? a.part_out + ap * D : (float*)a.out + (((int64_t)b * a.q_len + tok) * a.H + h) * D) + 4 * g;
#pragma unroll
      for (int db = 0; db < C::DB; ++db)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = o[db][4 * r4 + e] * inv;
          *(f32x4*)(dst + db * 32 + 8 * r4) = x;
        }
      if (g == 0) {
        if (a.split > 1)
          a.part_lse[ap] = lse;
        else if (a.lse != nullptr)
          a.lse[at] = lse;
      }
    }
    return;
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
    part_m[wave * 32 + lr] = m;
    part_l[wave * 32 + lr] = lt;
  }
  __syncthreads();
  constexpr int CH = 32 * D / 4;
  static_assert(CH % C::NT == 0, "chunks divide over the threads");
#pragma unroll
  for (int i = 0; i < CH / C::NT; ++i) {
    const int c = tid + i * C::NT;
    const int r = c / (D / 4), u = c % (D / 4);
    if (rt * C::BM + r >= a.rows) continue;
    const int rtok = (rt * C::BM + r) / a.G, h = hk * a.G + (rt * C::BM + r) % a.G;
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
      const float w = mk[k] == -INFINITY && part_l[k * 32 + r] == 0.f ? 0.f : fast_exp2(mk[k] - M);
      tot = __builtin_fmaf(w, part_l[k * 32 + r], tot);
      acc += w * *(const f32x4*)((const float*)(smem + k * C::GROUP) + r * D + ((u ^ (r & 15)) * 4));
    }
    const float inv = tot > 0.f ? 1.0f / tot : 0.f;
    const float lse = tot > 0.f ? (M + __builtin_amdgcn_logf(tot)) * kLn2 : tot == 0.f ? -INFINITY : tot;
    const int64_t at = ((int64_t)b * a.H + h) * a.q_len + rtok;
    if (a.split > 1) {
      const int64_t ap = (int64_t)sp * a.B * a.H * a.q_len + at;
      *(f32x4*)(a.part_out + ap * D + u * 4) = acc * inv;
      if (u == 0) a.part_lse[ap] = lse;
    } else {
      *(f32x4*)((float*)a.out + (((int64_t)b * a.q_len + rtok) * a.H + h) * D + u * 4) = acc * inv;
      if (u == 0 && a.lse != nullptr) a.lse[at] = lse;
    }
  }
  }
}

template <class C, class Rows>
hipError_t launch_f32_rows(const CrossArgs& a0, hipStream_t s) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  e = set_kernel_lds<&cross_f32_kernel<C, Rows>, C::LDS>(dev);
  if (e != hipSuccess) return e;
  CrossArgs a = a0;
  a.row_tiles = (a.rows + C::BM - 1) / C::BM;
  const int64_t grid = (int64_t)a.row_tiles * a.split * a.Hk * a.B;
  if (!launch_fits(grid, C::NT)) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((cross_f32_kernel<C, Rows>), dim3((unsigned)grid), dim3(C::NT), C::LDS, s, a);
  return hipGetLastError();
}

}  // namespace

// The form of a launch, by how its workgroups fill the compute units, as the
// float32 attention chooses it (attn_f32.hip): 32 rows and the waves on the
// keys up to two rounds, then 128 rows while every workgroup has a compute unit
// to itself, then 256 (D=64: 128).  2,047 rows x 12 heads against 333 keys at
// D=128: 32 rows 61 us, 128 rows 45 us.
using Split128 = CfgF<128, 1, 4, 1, false>;
using Mid128 = CfgF<128, 4, 1, 1, true>;
using Shared128 = CfgF<128, 8, 1, 2, false>;
using Split64 = CfgF<64, 1, 8, 2, false>;
using Shared64 = CfgF<64, 4, 1, 2, true>;

int cross_f32_rows(const CrossArgs& a, int D, int cus) {
  const int64_t heads = (int64_t)a.Hk * a.B;
  if ((int64_t)(a.rows + 31) / 32 * heads <= 2 * (int64_t)cus) return 32;
  if (D == 64 || (int64_t)(a.rows + 127) / 128 * heads <= cus) return 128;
  return 256;
}

hipError_t launch_cross_f32(const CrossArgs& a, int D, hipStream_t s) {
  int dev = 0, cus = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return e;
  const int rows = cross_f32_rows(a, D, cus);
  if (D == 64) {
    if (rows == 32) return a.mask ? launch_f32_rows<Split64, ListedRows>(a, s) : launch_f32_rows<Split64, StridedRows>(a, s);
    return a.mask ? launch_f32_rows<Shared64, ListedRows>(a, s) : launch_f32_rows<Shared64, StridedRows>(a, s);
  }
  if (rows == 32) return a.mask ? launch_f32_rows<Split128, ListedRows>(a, s) : launch_f32_rows<Split128, StridedRows>(a, s);
  if (rows == 128) return a.mask ? launch_f32_rows<Mid128, ListedRows>(a, s) : launch_f32_rows<Mid128, StridedRows>(a, s);
  return a.mask ? launch_f32_rows<Shared128, ListedRows>(a, s) : launch_f32_rows<Shared128, StridedRows>(a, s);
}

}  // namespace ditango
