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
//   loads of the token's first elements and weights are on their way meanwhile.
//   A thread takes units of two vectors: the two halves of VEC pairs.  A head's
//   units lie in consecutive lanes, 4 ... 64 of them, which add up its squares
//   without LDS.
//
// Angles
//   position * freq in turns, float64, its fraction rounded to float32: the
//   error is 2^-26 of a turn from the rounding and 2^-53 |position * freq|
//   from the product, whatever the position.
//
// Range of the norm
//   Squares leave float32 from 2^64 on, and below 2^-74 where eps is as small.
//   Where a mean ends up near those ends the sum is taken again over elements
//   scaled by a power of two, which the norm's factor undoes.
#include <type_traits>

#include "attn_tile.h"
#include "layer.h"

namespace ditango {
namespace {

template <typename T, int N> struct Vec {
  typedef T type __attribute__((ext_vector_type(N)));
};
template <typename T> struct Vec<T, 1> { typedef T type; };

// VEC elements (a power of two), as loaded, and as floats
template <typename T, int VEC>
__device__ __forceinline__ typename Vec<T, VEC>::type load_raw(const T* p) {
  return *(const typename Vec<T, VEC>::type*)p;
}
template <typename T, int VEC>
__device__ __forceinline__ void widen(const typename Vec<T, VEC>::type& v, float (&x)[VEC]) {
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
    __builtin_nontemporal_store(v, (V*)p);
  }
}

// Scale of the elements for a mean of squares (eps included) that lies near the
// ends of float32, 1 otherwise.
constexpr float kUp = 0x1p100f, kDown = 0x1p-80f;
__device__ __forceinline__ float range_scale(float mean) {
  return mean > 0x1p-100f && mean < 0x1p120f ? 1.f : mean < 1.f ? kUp : kDown;
}

// Units of a token that a thread holds: one of each tensor, or two of one.
constexpr int kHeld = 2;

template <typename T, int D, int VEC, bool HALF, int NORM>
__global__ __launch_bounds__(1024) void rotary_kernel(const RotaryArgs a) {
  constexpr int UD = D / (2 * VEC);           // units of a head
  static_assert((UD & (UD - 1)) == 0 && UD <= 64, "a head's units lie in one wave");
  extern __shared__ float2 turned[];          // [tokens of the workgroup][rot / 2]
  __shared__ float sums[2][16];

  const int tid = threadIdx.x;
  const int team = a.team;                    // threads of a token: below 64 a power of two, or all
  const int per_block = a.tokens;             // of a workgroup
  const int in_team = per_block == 1 ? tid : tid & (team - 1), my = per_block == 1 ? 0 : tid / team;
  const int64_t tokens = (int64_t)a.B * a.S;
  const int64_t tok0 = (int64_t)blockIdx.x * per_block;
  const int64_t tok = tok0 + my;
  const bool live = tok < tokens;
  // (a team without a token reads the last one's)
  const int64_t at_tok = live ? tok : tokens - 1;
  const int b = a.B == 1 ? 0 : (int)(at_tok / a.S);
  const int64_t s = at_tok - b * a.S;
  const int pairs = a.rot >> 1;

  // unit v of tensor k: its vectors, and those of its weights
  struct Place {
    const T *x0, *x1, *w0, *w1;
    T *y0, *y1;
    int at;                                   // unit of the head
  };
  auto place = [&](int k, int v) {            // (k is the same for all threads)
    const ditango_rotary_tensor& t = a.t[k];
    const int h = v / UD;
    Place p;
    p.at = v % UD;
    const bool turn = p.at * VEC < pairs;
    const int p0 = HALF && turn ? p.at * VEC : p.at * 2 * VEC;
    const int p1 = HALF && turn ? p0 + pairs : p0 + VEC;
    const T* x = (const T*)t.x + b * t.x_strides[0] + s * t.x_strides[1] + h * t.x_strides[2];
    T* y = (T*)t.y + b * t.y_strides[0] + s * t.y_strides[1] + h * t.y_strides[2];
    const T* w = (const T*)t.weight + (NORM == 2 ? h * D : 0);
    p.x0 = x + p0, p.x1 = x + p1, p.y0 = y + p0, p.y1 = y + p1, p.w0 = w + p0, p.w1 = w + p1;
    return p;
  };
  auto squares = [&](const float (&x0)[VEC], const float (&x1)[VEC]) {
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) q = __builtin_fmaf(x0[e], x0[e], __builtin_fmaf(x1[e], x1[e], q));
    return q;
  };
  auto scaled = [&](float (&x0)[VEC], float (&x1)[VEC], float by) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) x0[e] *= by, x1[e] *= by;
  };
  // tensor and unit of held slot i; the first unit of tensor k that is not held
  const bool two = a.n == 2;
  auto tensor_of = [&](int i) { return two ? i : 0; };
  auto unit_of = [&](int i) { return two ? in_team : in_team + i * team; };
  const int rest = two ? team : kHeld * team;

  // ---- the token's first units are on their way while the angles are formed
  // (without a condition: a load under one is waited for inside it; a thread
  // without a unit reads the tensor's last one)
  typedef typename Vec<T, VEC>::type V;
  V x0[kHeld], x1[kHeld], w0[kHeld], w1[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int k = tensor_of(i);
    const Place p = place(k, min(unit_of(i), a.units[k] - 1));
    x0[i] = load_raw<T, VEC>(p.x0);
    x1[i] = load_raw<T, VEC>(p.x1);
    if constexpr (NORM != 0) {
      w0[i] = load_raw<T, VEC>(p.w0);
      w1[i] = load_raw<T, VEC>(p.w1);
    }
  }
  for (int i = tid; i < per_block * pairs; i += blockDim.x) {
    const int64_t tk = tok0 + i / pairs;
    if (tk >= tokens) break;
    const int pr = i % pairs;
    const int bk = a.B == 1 ? 0 : (int)(tk / a.S);
    const double at = a.turns[pr] * (double)a.pos[bk * a.pos_batch + (tk - bk * a.S) * a.axes + a.axis[pr]];
    float sn, cs;
    sincospif(2.f * (float)(at - __builtin_rint(at)), &sn, &cs);
    turned[i] = float2{cs * a.factor, sn * a.factor};
  }

  // ---- the norm over the token's row: both tensors' sums of squares
  float scale[2] = {1.f, 1.f};
  if constexpr (NORM == 2) {
    // (in all of a workgroup where its team is larger than a wave, in the team otherwise)
    auto reduce = [&](float (&sq)[2]) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        for (int d = 1; d < (team < 64 ? team : 64); d <<= 1) sq[k] += __shfl_xor(sq[k], d, 64);
        if (team > 64 && (tid & 63) == 0) sums[k][tid >> 6] = sq[k];
      }
    };
    auto mean_of = [&](int k, float sq, float eps) {
      if (team > 64) {
        sq = 0.f;
        for (int w = 0; w < (int)blockDim.x >> 6; ++w) sq += sums[k][w];
      }
      return sq / (float)(a.t[k].heads * D) + eps;
    };
    float sq[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      float y0[VEC], y1[VEC];
      widen<T, VEC>(x0[i], y0);
      widen<T, VEC>(x1[i], y1);
      const float q = unit_of(i) < a.units[tensor_of(i)] ? squares(y0, y1) : 0.f;
      if (tensor_of(i) == 0) sq[0] += q; else sq[1] += q;
    }
    for (int k = 0; k < a.n; ++k)
      for (int u = in_team + rest; u < a.units[k]; u += team) {
        const Place p = place(k, u);
        float y0[VEC], y1[VEC];
        widen<T, VEC>(load_raw<T, VEC>(p.x0), y0);
        widen<T, VEC>(load_raw<T, VEC>(p.x1), y1);
        const float q = squares(y0, y1);
        if (k == 0) sq[0] += q; else sq[1] += q;
      }
    reduce(sq);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (k < a.n) scale[k] = mean_of(k, sq[k], a.eps);
    const float by0 = range_scale(scale[0]), by1 = range_scale(scale[1]);
    scale[0] = rsqrtf(scale[0]), scale[1] = rsqrtf(scale[1]);
    if (by0 != 1.f || by1 != 1.f) {
      // (the token read again: nothing of it has been written)
      if (team > 64) __syncthreads();                 // every wave has read the sums
      // (an element at a time: rare, and as few registers as the waves want)
      int64_t s_again = s;
      int b_again = b, u_again = in_team;
      asm volatile("" : "+v"(s_again), "+v"(b_again), "+v"(u_again));
      sq[0] = sq[1] = 0.f;
#pragma unroll 1
      for (int k = 0; k < a.n; ++k) {
        const ditango_rotary_tensor& t = a.t[k];
        const T* row = (const T*)t.x + b_again * t.x_strides[0] + s_again * t.x_strides[1];
        float q = 0.f;
#pragma unroll 1
        for (int e = u_again; e < t.heads * D; e += team) {
          const float x = (float)row[e / D * t.x_strides[2] + e % D] * (k == 0 ? by0 : by1);
          q = __builtin_fmaf(x, x, q);
        }
        if (k == 0) sq[0] = q; else sq[1] = q;
      }
      reduce(sq);
      if (team > 64) __syncthreads();
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float by = k == 0 ? by0 : by1;
        if (k < a.n && by != 1.f) {
          const float r = rsqrtf(mean_of(k, sq[k], a.eps * by * by));
          scale[k] = by < 1.f ? r * by : -r;          // (negative: of the elements times kUp)
        }
      }
    }
  } else {
    __syncthreads();
  }

  auto finish = [&](const Place& p, float r, const V& x0, const V& x1, const V& w0, const V& w1) {
    float y0[VEC], y1[VEC];
    widen<T, VEC>(x0, y0);
    widen<T, VEC>(x1, y1);
    if constexpr (NORM != 0) {
      float v0[VEC], v1[VEC];
      widen<T, VEC>(w0, v0);
      widen<T, VEC>(w1, v1);
      if constexpr (NORM == 1) {
        auto mean = [&](float eps) {
          float q = squares(y0, y1);
#pragma unroll
          for (int d = 1; d < UD; d <<= 1) q += __shfl_xor(q, d, 64);
          return q * (1.f / D) + eps;
        };
        float m = mean(a.eps);
        const float by = range_scale(m);                // (the same in all lanes of the head)
        if (by != 1.f) {
          scaled(y0, y1, by);
          m = mean(a.eps * by * by);
        }
        r = rsqrtf(m);
      } else if (r < 0.f) {
        scaled(y0, y1, kUp);
        r = -r;
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        y0[e] = y0[e] * r * v0[e];
        y1[e] = y1[e] * r * v1[e];
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
    store_vec<T, VEC>(p.y0, y0);
    store_vec<T, VEC>(p.y1, y1);
  };
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int k = tensor_of(i), u = unit_of(i);
    // (a head's units are in or out together, so its lanes meet in the norm)
    if (live && u < a.units[k]) finish(place(k, u), k == 0 ? scale[0] : scale[1], x0[i], x1[i], w0[i], w1[i]);
  }
  for (int k = 0; k < a.n; ++k)
    for (int u = in_team + rest; u < a.units[k]; u += team) {
      if (!live) break;
      const Place p = place(k, u);
      V v0 = {}, v1 = {};
      if constexpr (NORM != 0) {
        v0 = load_raw<T, VEC>(p.w0);
        v1 = load_raw<T, VEC>(p.w1);
      }
      finish(p, k == 0 ? scale[0] : scale[1], load_raw<T, VEC>(p.x0), load_raw<T, VEC>(p.x1), v0, v1);
    }
}

template <typename T, int D, int VEC, bool HALF, int NORM>
hipError_t launch_vec(const RotaryArgs& a0, hipStream_t s) {
  RotaryArgs a = a0;
  constexpr int UD = D / (2 * VEC);
  for (int i = 0; i < a.n; ++i) a.units[i] = a.t[i].heads * UD;
  // a team holds a token's units where it can; teams of a wave or less are
  // powers of two (their sums stay inside them), larger ones the workgroup
  const int want = a.n == 2 ? (a.units[0] > a.units[1] ? a.units[0] : a.units[1]) : (a.units[0] + 1) / 2;
  int threads = 256;
  if (want <= 64) {
    a.team = UD;
    while (a.team < want) a.team *= 2;
  } else {
    a.team = threads = want >= 1024 ? 1024 : (want + 63) / 64 * 64;
  }
  a.tokens = threads / a.team;
  const int64_t grid = ((int64_t)a.B * a.S + a.tokens - 1) / a.tokens;
  if (!launch_fits(grid, threads)) return hipErrorInvalidConfiguration;
  const size_t lds = (size_t)a.tokens * (a.rot / 2) * sizeof(float2);
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
