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
//   bf16 for the second product (2^-9 of each; the row sum takes them before
//   that), the output once more at its store.
#include <type_traits>

#include "attn_tile.h"
#include "internal.h"

namespace ditango {
namespace {

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// s_waitcnt immediate: at most n vector-memory operations outstanding
constexpr int vmcnt_imm(int n) { return (n & 15) | ((n >> 4) << 14) | 0x0F70; }

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
// or from an address.  The waits for them are written out (s_waitcnt vmcnt).
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

template <int D_>
struct CrossCfg {
  static constexpr int D = D_, NW = 4, BN = 64, NBUF = 2;
  static constexpr int NT = NW * 64, BM = NW * 32;
  static constexpr int KS = D / 16, KB = BN / 32, DB = D / 32, PS = BN / 16;
  static constexpr int UNITS = D / 8, ROWB = D * 2, TILEB = BN * ROWB;
  static constexpr int RPL = 1024 / ROWB;          // rows per 1 KiB load
  static constexpr int LW = TILEB / 1024 / NW;     // loads per wave and tile
  static constexpr int LDS = 2 * NBUF * TILEB;
  static_assert(NW * 32 * ROWB <= LDS, "output staging inside the ring");
};

// One workgroup: 128 rows of one key/value head, one key range.  Four waves of
// 32 rows share the K and V tiles, which land in a ring of two by direct loads.
template <int D_, bool LIST>
__global__ __launch_bounds__(256, 2) void cross_kernel(const CrossArgs a) {
  using C = CrossCfg<D_>;
  constexpr int D = C::D, BN = C::BN;
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

  // this workgroup's key range: whole tiles
  const int n = __builtin_amdgcn_readfirstlane(cross_keys(a, b));
  const int per = ((n + BN - 1) / BN + a.split - 1) / a.split * BN;
  const int key_begin = min(sp * per, n), key_end = min(key_begin + per, n);
  const int tiles = (key_end - key_begin + BN - 1) / BN;

  const __bf16* kg = (const __bf16*)a.k + b * a.k_batch + hk * a.k_head;
  const __bf16* vg = (const __bf16*)a.v + b * a.v_batch + hk * a.v_head;

  // ---- this lane's query row (rows past the end read the last one and are
  // not stored): B operand, Q[row][16s + 8g .. +8]
  const int row0 = rt * C::BM + wave * 32;
  const int row = row0 + lr;
  const int tok = min(row, a.rows - 1) / a.G, gi = min(row, a.rows - 1) % a.G;
  const __bf16* qrow = (const __bf16*)a.q + b * a.q_batch + tok * a.q_token + (int64_t)(hk * a.G + gi) * a.q_head;
  bf16x8 qf[C::KS];
#pragma unroll
  for (int s = 0; s < C::KS; ++s) qf[s] = *(const bf16x8*)(qrow + 16 * s + 8 * g);

  f32x16 o[C::DB];
#pragma unroll
  for (int db = 0; db < C::DB; ++db) o[db] = f32x16{};
  float m = -INFINITY, l = 0.f;

  const uint32_t lds0 = lds_addr(smem);
  const int ld_row = lane / C::UNITS, ld_unit = lane % C::UNITS;
  // Tile `tile` of K (which = 0) or V (1) into ring slot tile % 2.
  auto load_tile = [&](int tile, int which) {
    const int key0 = key_begin + tile * BN;
    const uint32_t dst = lds0 + (uint32_t)((which * C::NBUF + tile % C::NBUF) * C::TILEB + wave * C::LW * 1024);
    const __bf16* base = which ? vg : kg;
    const int64_t stride = which ? a.v_token : a.k_token;
    if constexpr (LIST) {
#pragma unroll
      for (int i = 0; i < C::LW; ++i) {
        const int r = (wave * C::LW + i) * C::RPL + ld_row;
        const int unit = ld_unit ^ (which ? swz_v<D>(r) : swz_k<D>(r));
        const __bf16* p = (const __bf16*)a.zeros;
        if (key0 + r < key_end) p = base + a.list[(int64_t)b * a.kv_len + key0 + r] * stride;
        dma_addr(p + unit * 8, dst + i * 1024);
      }
    } else {
      const int64_t left = key_end > key_begin + tile * BN ? (int64_t)(key_end - 1 - key0) * stride * 2 + C::ROWB : 0;
      const u32x4 desc = buffer_desc(base + (int64_t)key0 * stride, (uint32_t)min(left, (int64_t)0x7fffffff));
#pragma unroll
      for (int i = 0; i < C::LW; ++i) {
        const int r = (wave * C::LW + i) * C::RPL + ld_row;
        const int unit = ld_unit ^ (which ? swz_v<D>(r) : swz_k<D>(r));
        dma_desc(desc, (uint32_t)r * (uint32_t)(stride * 2) + (uint32_t)unit * 16, dst + i * 1024);
      }
    }
  };

  // V^T fragments by transpose reads
  const int vrow = 4 * g + ((lane & 15) >> 2);
  const int vdim = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  int voff[C::DB];
#pragma unroll
  for (int db = 0; db < C::DB; ++db) {
    const int dim = 32 * db + vdim;
    voff[db] = vrow * C::ROWB + ((dim >> 3) ^ swz_v<D>(vrow)) * 16 + (dim & 7) * 2;
  }
  auto v_frag = [&](const unsigned char* vs, int s, int db) {
    const unsigned char* p = vs + 16 * s * C::ROWB + voff[db];
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, p)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, p + 8 * C::ROWB)));
    return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
  };

  if (tiles > 0) {
    load_tile(0, 0);
    load_tile(0, 1);
    for (int i = 0; i < tiles; ++i) {
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));      // tile i has landed
      __syncthreads();
      if (i + 1 < tiles) {
        load_tile(i + 1, 0);
        load_tile(i + 1, 1);
      }
      const unsigned char* kb = smem + (i % C::NBUF) * C::TILEB;
      const unsigned char* vb = smem + (C::NBUF + i % C::NBUF) * C::TILEB;
      f32x16 sc[C::KB];
#pragma unroll
      for (int k = 0; k < C::KB; ++k) {
        sc[k] = f32x16{};
#pragma unroll
        for (int s = 0; s < C::KS; ++s)
          sc[k] = mfma32(*(const bf16x8*)(kb + (k * 32 + lr) * C::ROWB + ((2 * s + g) ^ swz_k<D>(lr)) * 16), qf[s], sc[k]);
      }
      if (key_begin + (i + 1) * BN > key_end) {
#pragma unroll
        for (int k = 0; k < C::KB; ++k)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (key_begin + i * BN + k * 32 + 8 * (r >> 2) + 4 * g + (r & 3) >= key_end) sc[k][r] = -INFINITY;
      }
      float mx = sc[0][0];
#pragma unroll
      for (int k = 0; k < C::KB; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[k][r]);
      const float mnew = fmaxf(m, pair_max(mx) * a.scale_log2);
      const float alpha = m == -INFINITY ? 0.f : fast_exp2(m - mnew);
      const float mm = mnew == -INFINITY ? 0.f : mnew;
      m = mnew;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < C::DB; ++db) o[db] *= alpha;
      bf16x8 pf[C::PS];
#pragma unroll
      for (int k = 0; k < C::KB; ++k)
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          f32x8 x;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[e] = fast_exp2(__builtin_fmaf(sc[k][8 * hh + e], a.scale_log2, -mm));
            l += x[e];
          }
          pf[2 * k + hh] = __builtin_convertvector(x, bf16x8);
        }
#pragma unroll
      for (int s = 0; s < C::PS; ++s)
#pragma unroll
        for (int db = 0; db < C::DB; ++db) o[db] = mfma32(v_frag(vb, s, db), pf[s], o[db]);
    }
  }
  __syncthreads();                                   // the ring is free

  // ---- epilogue
  const float lt = pair_sum(l);
  const float inv = lt > 0.f ? 1.0f / lt : 0.f;
  const float lse = lt > 0.f ? (m + __builtin_amdgcn_logf(lt)) * kLn2 : lt == 0.f ? -INFINITY : lt;
  const bool ok = row < a.rows;
  const int h = hk * a.G + gi;
  if (a.split > 1) {
    const int64_t at = (((int64_t)sp * a.B + b) * a.H + h) * a.q_len + tok;
    if (ok) {
      float* dst = a.part_out + at * D + 4 * g;
#pragma unroll
      for (int db = 0; db < C::DB; ++db)
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) {
          f32x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = o[db][4 * r4 + e] * inv;
          *(f32x4*)(dst + db * 32 + 8 * r4) = x;
        }
      if (g == 0) a.part_lse[at] = lse;
    }
    return;
  }
  if (ok && g == 0 && a.lse != nullptr) a.lse[((int64_t)b * a.H + h) * a.q_len + tok] = lse;
  // rows through LDS (16-byte units swizzled by row), then stored whole
  unsigned char* stage = smem + wave * 32 * C::ROWB;
#pragma unroll
  for (int db = 0; db < C::DB; ++db)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = o[db][4 * r4 + e] * inv;
      const int unit = (4 * db + r4) ^ (lr & (C::UNITS - 1));
      *(bf16x4*)(stage + lr * C::ROWB + unit * 16 + 8 * g) = __builtin_convertvector(x, bf16x4);
    }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 32 / C::RPL; ++i) {
    const int r = i * C::RPL + ld_row;
    if (row0 + r < a.rows) {
      const int rtok = (row0 + r) / a.G, rh = hk * a.G + (row0 + r) % a.G;
      *(bf16x8*)((__bf16*)a.out + (((int64_t)b * a.q_len + rtok) * a.H + rh) * D + ld_unit * 8) =
          *(const bf16x8*)(stage + r * C::ROWB + (ld_unit ^ (r & (C::UNITS - 1))) * 16);
    }
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

// Composes the partial states of a split launch: a wave per row, in the order
// of the key ranges.
template <typename T, int D>
__global__ __launch_bounds__(256) void cross_join_kernel(const CrossArgs a) {
  constexpr int E = D / 64;
  const int64_t rows = (int64_t)a.B * a.H * a.q_len;
  const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= rows) return;
  const int lane = threadIdx.x & 63;
  float mx = -INFINITY;
  bool bad = false;
  for (int p = 0; p < a.split; ++p) {
    const float x = a.part_lse[p * rows + r];
    bad |= x != x;
    mx = fmaxf(mx, x);
  }
  const float mm = mx == -INFINITY ? 0.f : mx;
  float tot = 0.f, acc[E] = {};
  for (int p = 0; p < a.split; ++p) {
    const float w = fast_exp2((a.part_lse[p * rows + r] - mm) * 1.4426950408889634f);
    tot += w;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = __builtin_fmaf(w, a.part_out[(p * rows + r) * D + lane * E + e], acc[e]);
  }
  const float inv = tot > 0.f ? 1.0f / tot : bad ? NAN : 0.f;
  const int64_t tok = r % a.q_len, h = r / a.q_len % a.H, b = r / a.q_len / a.H;
  T* dst = (T*)a.out + ((b * a.q_len + tok) * a.H + h) * D + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) dst[e] = (T)(acc[e] * inv);
  if (lane == 0 && a.lse != nullptr)
    a.lse[r] = tot > 0.f ? mx + __builtin_amdgcn_logf(tot) * kLn2 : bad ? NAN : -INFINITY;
}

template <int D, bool LIST>
hipError_t launch_rows(const CrossArgs& a0, hipStream_t s) {
  using C = CrossCfg<D>;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  e = set_kernel_lds<&cross_kernel<D, LIST>, C::LDS>(dev);
  if (e != hipSuccess) return e;
  CrossArgs a = a0;
  a.row_tiles = (a.rows + C::BM - 1) / C::BM;
  const int64_t grid = (int64_t)a.row_tiles * a.split * a.Hk * a.B;
  if (grid > 0x7fffffff) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((cross_kernel<D, LIST>), dim3((unsigned)grid), dim3(C::NT), C::LDS, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t plan_cross(const CrossArgs& a, ditango_dtype dt, int D, CrossPlan* p) {
  *p = CrossPlan{1, 0};
  int dev = 0, cus = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return e;
  const int bm = dt == DITANGO_BF16 ? 128 : cross_f32_rows(D);
  const int64_t groups = (int64_t)((a.rows + bm - 1) / bm) * a.Hk * a.B;
  // a launch that leaves compute units idle splits its keys: two tiles at
  // least in each range
  const int64_t tiles = (a.kv_len + 63) / 64;
  int64_t split = (2 * (int64_t)cus + groups - 1) / groups;
  split = split < tiles / 2 ? split : tiles / 2;
  p->split = split > 1 ? (int)split : 1;
  p->bytes = cross_list_bytes(a);
  if (p->split > 1) {
    const size_t rows = (size_t)a.B * a.H * a.q_len;
    p->bytes += align_up256(p->split * rows * D * 4) + align_up256(p->split * rows * 4);
  }
  return hipSuccess;
}

hipError_t launch_cross(const CrossArgs& a0, ditango_dtype dt, int D, void* ws, size_t ws_bytes, hipStream_t s) {
  CrossPlan p;
  hipError_t e = plan_cross(a0, dt, D, &p);
  if (e != hipSuccess) return e;
  CrossArgs a = a0;
  char* w = (char*)ws;
  if (a.mask != nullptr) {
    a.list = (int32_t*)w;
    a.count = (int32_t*)(w + align_up256((size_t)a.B * a.kv_len * 4));
    a.zeros = (float*)((char*)a.count + align_up256((size_t)a.B * 4));
    hipLaunchKernelGGL(cross_list_kernel, dim3(a.B), dim3(1024), 0, s, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  a.split = 1;
  const size_t rows = (size_t)a.B * a.H * a.q_len;
  if (p.split > 1 && ws_bytes >= p.bytes) {
    a.split = p.split;
    a.part_out = (float*)(w + cross_list_bytes(a));
    a.part_lse = (float*)((char*)a.part_out + align_up256(p.split * rows * D * 4));
  }
  if (dt == DITANGO_F32)
    e = launch_cross_f32(a, D, s);
  else if (D == 128)
    e = a.mask ? launch_rows<128, true>(a, s) : launch_rows<128, false>(a, s);
  else
    e = a.mask ? launch_rows<64, true>(a, s) : launch_rows<64, false>(a, s);
  if (e != hipSuccess || a.split == 1) return e;
  const dim3 grid((unsigned)((rows + 3) / 4));
  if (dt == DITANGO_F32 && D == 128) hipLaunchKernelGGL((cross_join_kernel<float, 128>), grid, dim3(256), 0, s, a);
  if (dt == DITANGO_F32 && D == 64) hipLaunchKernelGGL((cross_join_kernel<float, 64>), grid, dim3(256), 0, s, a);
  if (dt == DITANGO_BF16 && D == 128) hipLaunchKernelGGL((cross_join_kernel<__bf16, 128>), grid, dim3(256), 0, s, a);
  if (dt == DITANGO_BF16 && D == 64) hipLaunchKernelGGL((cross_join_kernel<__bf16, 64>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace ditango
