// rotary.hip - rotary positions of queries and keys, with the root-mean-square
// norm before them (gfx950).
//
//   x^ = x or x * rsqrt(mean(x^2) + eps) * w,   (y0, y1) = (x^0, x^1) turned by
//   the angle positions[axis] * freq, for each pair of the rotated dims.
//
// Bound by HBM: every element is read and written once, the norm's sum and the
// rotation are taken from the registers a token was loaded into.
//
// Work decomposition
//   A team of threads per token, of both tensors (queries and keys of the same
//   tokens share the angles).  The cosines and sines of a token, at most 64
//   pairs, are formed once, by as many threads, and shared through LDS; the
//   loads of the token's first elements are on their way meanwhile.  A thread
//   takes units of two vectors: the two halves of VEC pairs.  A head's units
//   lie in consecutive lanes, 4 ... 64 of them, which add up its squares
//   without LDS.
//
// Angles
//   position * freq in turns, float64, its fraction rounded to float32: the
//   error is 2^-26 of a turn from the rounding and 2^-53 |position * freq|
//   from the product, whatever the position.
#include <type_traits>

#include "attn_tile.h"
#include "internal.h"

namespace ditango {
namespace {

template <typename T, int N> struct Vec {
  typedef T type __attribute__((ext_vector_type(N)));
};
template <typename T> struct Vec<T, 1> { typedef T type; };

// VEC elements (a power of two) as floats
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T* p, float (&x)[VEC]) {
  typedef typename Vec<T, VEC>::type V;
  const V v = *(const V*)p;
  if constexpr (VEC == 1) {
    x[0] = (float)v;
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = (float)v[e];
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T* p, const float (&x)[VEC]) {
  typedef typename Vec<T, VEC>::type V;
  if constexpr (VEC == 1) {
    *p = (T)x[0];
  } else {
    V v;
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = (T)x[e];
    *(V*)p = v;
  }
}

constexpr int kHeld = 2;      // units of a token that a thread holds

template <typename T, int D, int VEC, bool HALF, int NORM>
__global__ __launch_bounds__(1024) void rotary_kernel(const RotaryArgs a) {
  constexpr int UD = D / (2 * VEC);           // units of a head
  static_assert((UD & (UD - 1)) == 0 && UD <= 64, "a head's units lie in one wave");
  extern __shared__ float2 turned[];          // [tokens of the workgroup][rot / 2]
  __shared__ float sums[2][16];

  const int tid = threadIdx.x;
  const int team = a.team;                    // threads of a token: below 64 a power of two, or all
  const int in_team = tid % team, my = tid / team;
  const int per_block = blockDim.x / team;
  const int64_t tokens = (int64_t)a.B * a.S;
  const int64_t tok0 = (int64_t)blockIdx.x * per_block;
  const int64_t tok = tok0 + my;
  const bool live = tok < tokens;
  const int64_t b = (live ? tok : 0) / a.S, s = (live ? tok : 0) % a.S;
  const int pairs = a.rot >> 1;
  const int all = a.units[0] + a.units[1];

  // unit u of the token: its tensor, head and place in the head
  struct Place {
    const T* x;
    T* y;
    const T* w;
    int which, at, p0, p1;                    // unit in the head; its vectors' first elements
  };
  auto place = [&](int u) {
    Place p;
    p.which = u >= a.units[0] ? 1 : 0;
    const ditango_rotary_tensor& t = a.t[p.which];
    const int v = u - (p.which ? a.units[0] : 0);
    const int h = v / UD;
    p.at = v % UD;
    const bool turn = p.at * VEC < pairs;
    p.p0 = HALF && turn ? p.at * VEC : p.at * 2 * VEC;
    p.p1 = HALF && turn ? p.p0 + pairs : p.p0 + VEC;
    p.x = (const T*)t.x + b * t.x_strides[0] + s * t.x_strides[1] + h * t.x_strides[2];
    p.y = (T*)t.y + b * t.y_strides[0] + s * t.y_strides[1] + h * t.y_strides[2];
    p.w = (const T*)t.weight + (NORM == 2 ? h * D : 0);
    return p;
  };
  auto squares = [&](const float (&x0)[VEC], const float (&x1)[VEC]) {
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) q = __builtin_fmaf(x0[e], x0[e], __builtin_fmaf(x1[e], x1[e], q));
    return q;
  };

  // ---- the token's first units are on their way while the angles are formed
  float x0[kHeld][VEC], x1[kHeld][VEC];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int u = in_team + i * team;
#pragma unroll
    for (int e = 0; e < VEC; ++e) x0[i][e] = x1[i][e] = 0.f;
    if (live && u < all) {
      const Place p = place(u);
      load_vec<T, VEC>(p.x + p.p0, x0[i]);
      load_vec<T, VEC>(p.x + p.p1, x1[i]);
    }
  }
  for (int i = tid; i < per_block * pairs; i += blockDim.x) {
    const int64_t tk = tok0 + i / pairs;
    if (tk >= tokens) break;
    const int pr = i % pairs;
    const double at = a.turns[pr] * (double)a.pos[(tk / a.S) * a.pos_batch + tk % a.S * a.axes + a.axis[pr]];
    float sn, cs;
    sincospif(2.f * (float)(at - __builtin_rint(at)), &sn, &cs);
    turned[i] = float2{cs * a.factor, sn * a.factor};
  }

  // ---- the norm over the token's row: both tensors' sums of squares
  float scale[2] = {1.f, 1.f};
  if constexpr (NORM == 2) {
    float sq[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const float q = squares(x0[i], x1[i]);
      if (in_team + i * team < a.units[0]) sq[0] += q; else sq[1] += q;
    }
    for (int u = in_team + kHeld * team; u < all; u += team) {
      if (!live) break;
      const Place p = place(u);
      float y0[VEC], y1[VEC];
      load_vec<T, VEC>(p.x + p.p0, y0);
      load_vec<T, VEC>(p.x + p.p1, y1);
      const float q = squares(y0, y1);
      if (p.which == 0) sq[0] += q; else sq[1] += q;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      for (int d = 1; d < (team < 64 ? team : 64); d <<= 1) sq[k] += __shfl_xor(sq[k], d, 64);
      if (team > 64 && (tid & 63) == 0) sums[k][tid >> 6] = sq[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (team > 64) {
        sq[k] = 0.f;
        for (int w = 0; w < (int)blockDim.x >> 6; ++w) sq[k] += sums[k][w];
      }
      if (k < a.n) scale[k] = rsqrtf(sq[k] / (float)(a.t[k].heads * D) + a.eps);
    }
  } else {
    __syncthreads();
  }

  auto finish = [&](const Place& p, float (&y0)[VEC], float (&y1)[VEC]) {
    if constexpr (NORM != 0) {
      float w0[VEC], w1[VEC], r = p.which ? scale[1] : scale[0];
      if constexpr (NORM == 1) {
        float q = squares(y0, y1);
#pragma unroll
        for (int d = 1; d < UD; d <<= 1) q += __shfl_xor(q, d, 64);
        r = rsqrtf(q * (1.f / D) + a.eps);
      }
      load_vec<T, VEC>(p.w + p.p0, w0);
      load_vec<T, VEC>(p.w + p.p1, w1);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        y0[e] = y0[e] * r * w0[e];
        y1[e] = y1[e] * r * w1[e];
      }
    }
    if (p.at * VEC < pairs) {
      const float2* cs = turned + my * pairs + p.at * VEC;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float2 c = cs[e];
        float& u = HALF ? y0[e] : 2 * e < VEC ? y0[2 * e % VEC] : y1[2 * e % VEC];
        float& v = HALF || VEC == 1 ? y1[e] : 2 * e < VEC ? y0[(2 * e + 1) % VEC] : y1[(2 * e + 1) % VEC];
        const float t = u * c.x - v * c.y;
        v = u * c.y + v * c.x;
        u = t;
      }
    }
    store_vec<T, VEC>(p.y + p.p0, y0);
    store_vec<T, VEC>(p.y + p.p1, y1);
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int u = in_team + i * team;
    // (a head's units are in or out together, so its lanes meet in the norm)
    if (live && u < all) finish(place(u), x0[i], x1[i]);
  }
  for (int u = in_team + kHeld * team; u < all; u += team) {
    if (!live) break;
    const Place p = place(u);
    float y0[VEC], y1[VEC];
    load_vec<T, VEC>(p.x + p.p0, y0);
    load_vec<T, VEC>(p.x + p.p1, y1);
    finish(p, y0, y1);
  }
}

template <typename T, int D, int VEC, bool HALF, int NORM>
hipError_t launch_vec(const RotaryArgs& a0, hipStream_t s) {
  RotaryArgs a = a0;
  constexpr int UD = D / (2 * VEC);
  int all = 0;
  for (int i = 0; i < a.n; ++i) all += a.units[i] = a.t[i].heads * UD;
  // a team holds kHeld units a thread; teams below a wave are powers of two
  // (their sums stay inside them), those above one are the workgroup
  int threads = 256;
  const int want = (all + kHeld - 1) / kHeld;
  if (want <= 32) {
    a.team = UD;
    while (a.team < want) a.team *= 2;
  } else {
    a.team = threads = want >= 1024 ? 1024 : (want + 63) / 64 * 64;
  }
  const int64_t per_block = threads / a.team;
  const int64_t grid = ((int64_t)a.B * a.S + per_block - 1) / per_block;
  const size_t lds = (size_t)per_block * (a.rot / 2) * sizeof(float2);
  hipLaunchKernelGGL((rotary_kernel<T, D, VEC, HALF, NORM>), dim3((unsigned)grid), dim3(threads), lds, s, a);
  return hipGetLastError();
}

template <typename T, int D, bool HALF, int NORM>
hipError_t launch_norm(const RotaryArgs& a, hipStream_t s) {
  // the widest vector that sizes, strides and addresses allow
  uint64_t bits = (uint64_t)a.rot / 2 * sizeof(T) | (uint64_t)(D - a.rot) / 2 * sizeof(T);
  for (int i = 0; i < a.n; ++i) {
    const ditango_rotary_tensor& t = a.t[i];
    bits |= (uint64_t)(uintptr_t)t.x | (uint64_t)(uintptr_t)t.y;
    if (NORM != 0) bits |= (uint64_t)(uintptr_t)t.weight;
    for (int k = 0; k < 3; ++k) bits |= (uint64_t)(t.x_strides[k] | t.y_strides[k]) * sizeof(T);
  }
  constexpr int V = 16 / sizeof(T);
  if (bits % 16 == 0) return launch_vec<T, D, V, HALF, NORM>(a, s);
  if (bits % 8 == 0) return launch_vec<T, D, V / 2, HALF, NORM>(a, s);
  return launch_vec<T, D, 1, HALF, NORM>(a, s);
}

template <typename T, int D>
hipError_t launch_layout(const RotaryArgs& a, ditango_rotary_layout layout, ditango_rotary_norm norm, hipStream_t s) {
  if (layout == DITANGO_ROTARY_HALF) {
    if (norm == DITANGO_NORM_NONE) return launch_norm<T, D, true, 0>(a, s);
    if (norm == DITANGO_NORM_HEAD) return launch_norm<T, D, true, 1>(a, s);
    return launch_norm<T, D, true, 2>(a, s);
  }
  if (norm == DITANGO_NORM_NONE) return launch_norm<T, D, false, 0>(a, s);
  if (norm == DITANGO_NORM_HEAD) return launch_norm<T, D, false, 1>(a, s);
  return launch_norm<T, D, false, 2>(a, s);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, ditango_dtype dt, int D, ditango_rotary_layout layout,
                         ditango_rotary_norm norm, hipStream_t s) {
  if (dt == DITANGO_BF16)
    return D == 128 ? launch_layout<__bf16, 128>(a, layout, norm, s) : launch_layout<__bf16, 64>(a, layout, norm, s);
  return D == 128 ? launch_layout<float, 128>(a, layout, norm, s) : launch_layout<float, 64>(a, layout, norm, s);
}

}  // namespace ditango
