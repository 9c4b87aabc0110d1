// Products with a matrix of 4-bit levels on gfx950:
//
//   y[n][r] = bias[r] + sum_d s[r][d / G] (q[r][d] - z[r][d / G]) x[n][d].
//
// The levels enter v_mfma_f32_16x16x32_bf16 as whole numbers that bf16 holds
// exactly, moved by a constant o that their bits make cheap, and the zero level
// comes off with the group's sum of x:
//
//   y = bias + sum_g s (sum_d (q + o) x - (z + o) sum_d x),   sums and scales fp32.
//
// A = 16 rows of the matrix, B = 16 rows of x: lane l holds A[l%16][8 (l/16) .. +7],
// B[8 (l/16) .. +7][l%16] and results of rows 4 (l/16) .. +3, column l%16.
// bf16 x: o = 16, a level in the top bits of the mantissa of 16 .. 31 (two operations
// a pair).  fp32 x: three bf16 parts of 8 bits each (exact), and o = -7.5, so that the
// sums are not larger than they have to be.
//
// Store: [row tile of 16][block of 128 columns][lane][4 steps] words of eight levels:
// a lane's weights of a block are one 16-byte load, a wave's 1 KB in a row.  In a
// word, columns 0, 2, 4, 6 of the eight stand in the low half, 1, 3, 5, 7 in the high
// one, which is where the pairs of a bf16 operand want them.  Rows and columns that
// pad a tile hold level 0 and scale 0.
#include <algorithm>
#include <type_traits>

#include "device_common.hpp"
#include "gated.hpp"

#pragma clang fp contract(off)

namespace alstm {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

constexpr int kBlockCols = 128;

__device__ __forceinline__ f32x4 mfma(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// the lane's number, of no register that lives until then
__device__ __forceinline__ int lane_now() {
  unsigned all = ~0u;
  asm volatile("" : "+s"(all));
  return __builtin_amdgcn_mbcnt_hi(all, __builtin_amdgcn_mbcnt_lo(all, 0u));
}

// word of the store that holds level (r, d), and its bit
struct Place {
  size_t word;
  int bit;
};
__device__ __forceinline__ Place place_of(const Q4Matrix& m, int r, int d) {
  const int kb = d / kBlockCols, k = d % kBlockCols, step = k / 32, lane = (r & 15) + 16 * ((k & 31) / 8), e = k & 7;
  return {(((size_t)(r >> 4) * m.blocks + kb) * 64 + lane) * 4 + step, 4 * (e / 2 + 4 * (e & 1))};
}

__global__ void __launch_bounds__(256) q4_layout_kernel(Q4Matrix m, const uint8_t* q, const float* scale,
                                                        const uint8_t* zero, int* bad) {
  const size_t row_bytes = ((size_t)m.D + 1) / 2, words = (size_t)m.tiles * m.blocks * 256;
  const size_t first = (size_t)blockIdx.x * 256 + threadIdx.x, by = (size_t)gridDim.x * 256;
  for (size_t i = first; i < words; i += by) {
    const int step = (int)(i & 3), lane = (int)(i >> 2) & 63;
    const size_t tile = (i >> 8) / m.blocks;
    const int kb = (int)((i >> 8) % m.blocks);
    const size_t r = tile * 16 + (lane & 15), d0 = (size_t)kb * kBlockCols + 32 * step + 8 * (lane >> 4);
    unsigned w = 0;
    for (int e = 0; e < 8; ++e)
      if (r < (size_t)m.R && d0 + e < (size_t)m.D)
        w |= (unsigned)((q[r * row_bytes + (d0 + e) / 2] >> (4 * (e & 1))) & 15) << (4 * (e / 2 + 4 * (e & 1)));
    m.q[i] = w;
  }
  const size_t ns = (size_t)m.tiles * m.padded * 16;
  for (size_t i = first; i < ns; i += by) {
    const size_t r = i / 16 / m.padded * 16 + (i & 15);
    const int g = (int)(i / 16 % m.padded);
    float s = 0.f;
    int z = 0;
    if (r < (size_t)m.R && g < m.groups) {
      s = scale[r * m.groups + g];
      z = zero ? zero[r * m.groups + g] : 8;
      if (z > 15) *bad = 1;
    }
    m.s[i] = s;
    m.z[i] = (uint8_t)z;
  }
}

__global__ void __launch_bounds__(256) q4_unpack_kernel(Q4Matrix m, uint8_t* q, float* scale, uint8_t* zero) {
  const size_t row_bytes = ((size_t)m.D + 1) / 2, nq = (size_t)m.R * row_bytes, ns = (size_t)m.R * m.groups;
  const size_t first = (size_t)blockIdx.x * 256 + threadIdx.x, by = (size_t)gridDim.x * 256;
  for (size_t i = first; i < nq; i += by) {
    const int r = (int)(i / row_bytes), d = 2 * (int)(i % row_bytes);
    unsigned b = 0;
    for (int e = 0; e < 2; ++e)
      if (d + e < m.D) {
        const Place p = place_of(m, r, d + e);
        b |= ((m.q[p.word] >> p.bit) & 15u) << (4 * e);
      }
    q[i] = (uint8_t)b;
  }
  for (size_t i = first; i < ns; i += by) {
    const size_t r = i / m.groups, at = ((r / 16) * m.padded + i % m.groups) * 16 + r % 16;
    scale[i] = m.s[at];
    zero[i] = m.z[at];
  }
}

// Eight levels of a word as bf16 16 + q.
__device__ __forceinline__ bf16x8 levels_16(unsigned w) {
  constexpr unsigned kMask = 0x00780078u;
  unsigned kOne = 0x41804180u;   // 16.0 in both halves
  asm("" : "+v"(kOne));          // (in a vector register: one instruction masks and sets, and it takes one constant)
  const u32x4 v{((w << 3) & kMask) | kOne, ((w >> 1) & kMask) | kOne, ((w >> 5) & kMask) | kOne,
                ((w >> 9) & kMask) | kOne};
  return __builtin_bit_cast(bf16x8, v);
}

// Eight levels of a word as bf16 q - 7.5 = +-(m + 1/2), m = 0 .. 7: m picks the two
// bytes of m + 1/2 from a table, bit 3 of the level is the sign.
__device__ __forceinline__ bf16x8 levels_centred(unsigned w) {
  const unsigned neg = ~w & 0x88888888u;        // levels below 8: m = 7 - q
  w ^= neg - (neg >> 3);
  const unsigned sign = neg;
  constexpr unsigned kHi0 = 0x40403F3Fu, kHi1 = 0x40404040u, kLo0 = 0x6020C000u, kLo1 = 0xF0D0B090u;
  // nibbles 0, 2, 4, 6 and 1, 3, 5, 7 of the word: columns 0, 4, 1, 5 and 2, 6, 3, 7
  const unsigned ma = w & 0x07070707u, mb = (w >> 4) & 0x07070707u;
  const unsigned ha = __builtin_amdgcn_perm(kHi1, kHi0, ma) | ((sign << 4) & 0x80808080u);
  const unsigned hb = __builtin_amdgcn_perm(kHi1, kHi0, mb) | (sign & 0x80808080u);
  const unsigned la = __builtin_amdgcn_perm(kLo1, kLo0, ma), lb = __builtin_amdgcn_perm(kLo1, kLo0, mb);
  // byte i of ha, la: nibbles 0, 2, 4, 6 are columns 0, 4, 1, 5
  const u32x4 v{__builtin_amdgcn_perm(ha, la, 0x06020400u), __builtin_amdgcn_perm(hb, lb, 0x06020400u),
                __builtin_amdgcn_perm(ha, la, 0x07030501u), __builtin_amdgcn_perm(hb, lb, 0x07030501u)};
  return __builtin_bit_cast(bf16x8, v);
}

// Eight values of a row of x from column k, zeros past its end; `whole`: none is.
// Loads of these types need be aligned to their elements only, but a load that is not
// aligned to 4 bytes takes several times as long: where rows of bf16 begin at odd
// elements (`odd`), a lane loads the words that its values stand in, which all hold one
// of them, and shifts (row kernel, 16 rows, 2048 x 7507: 13 us, without 22; the tile
// kernel, whose threads load little at a time, is slower with it: 2000 rows, 44 and 37).
template <class T>
struct XVec;
template <>
struct XVec<__bf16> {
  typedef bf16x8 Raw;
  typedef bf16x8 Any __attribute__((aligned(2)));
};
template <>
struct XVec<float> {
  typedef f32x8 Raw;
  typedef f32x8 Any __attribute__((aligned(4)));
};
template <class T>
__device__ __forceinline__ typename XVec<T>::Raw load_eight(const T* p, bool odd) {
  if constexpr (sizeof(T) == 2) {
    if (odd) {
      typedef u32x4 Words __attribute__((aligned(4)));
      const unsigned off = (unsigned)(reinterpret_cast<uintptr_t>(p) & 2u), shift = 8 * off;
      const unsigned* w = reinterpret_cast<const unsigned*>(reinterpret_cast<const char*>(p) - off);
      const u32x4 v = *reinterpret_cast<const Words*>(w);
      const unsigned last = w[off ? 4 : 3];
      return __builtin_bit_cast(
          bf16x8, u32x4{__builtin_amdgcn_alignbit(v[1], v[0], shift), __builtin_amdgcn_alignbit(v[2], v[1], shift),
                        __builtin_amdgcn_alignbit(v[3], v[2], shift), __builtin_amdgcn_alignbit(last, v[3], shift)});
    }
  }
  return *reinterpret_cast<const typename XVec<T>::Any*>(p);
}
template <class T>
__device__ __forceinline__ bool odd_rows(const T* x, int D) {
  return sizeof(T) == 2 && ((D & 1) || (reinterpret_cast<uintptr_t>(x) & 2u));
}

template <class T>
__device__ __forceinline__ typename XVec<T>::Raw load_x(const T* row, int k, int D, bool whole, bool odd) {
  if (whole) return load_eight<T>(row + k, odd);
  typename XVec<T>::Raw v{};
  if (k + 8 <= D) {
    v = load_eight<T>(row + k, odd);
  } else if (k < D) {   // (eight loads at once, not one after another)
    T t[8];
    int last = D - 1;
    asm volatile("" : "+s"(last));   // (the row's end found here: kept from before a loop it would take registers there)
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = row[min(k + e, last)];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = k + e < D ? t[e] : (T)0.f;
  }
  return v;
}

// The bf16 parts of eight values: kParts of them, whose sum is the value.
template <class T>
struct Parts;
template <>
struct Parts<__bf16> {
  static constexpr int kParts = 1;
  static constexpr float kOffset = 16.f;
  bf16x8 p[1];
  __device__ __forceinline__ explicit Parts(const bf16x8& x) : p{x} {}
  static __device__ __forceinline__ bf16x8 levels(unsigned w) { return levels_16(w); }
};
template <>
struct Parts<float> {
  static constexpr int kParts = 3;
  static constexpr float kOffset = -7.5f;
  bf16x8 p[3];
  // cut, not rounded: the rest is exact, and the largest fp32 stays finite
  __device__ __forceinline__ explicit Parts(const f32x8& x) {
    u32x4 v[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      unsigned h[2], m[2], l[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float f = x[2 * i + j];
        h[j] = __float_as_uint(f);
        const float r = f - __uint_as_float(h[j] & 0xFFFF0000u);
        m[j] = __float_as_uint(r);
        l[j] = __float_as_uint(r - __uint_as_float(m[j] & 0xFFFF0000u));
      }
      v[0][i] = __builtin_amdgcn_perm(h[1], h[0], 0x07060302u);
      v[1][i] = __builtin_amdgcn_perm(m[1], m[0], 0x07060302u);
      v[2][i] = __builtin_amdgcn_perm(l[1], l[0], 0x07060302u);
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) p[k] = __builtin_bit_cast(bf16x8, v[k]);
  }
  static __device__ __forceinline__ bf16x8 levels(unsigned w) { return levels_centred(w); }
};

// the sum of eight values
__device__ __forceinline__ float sum8(const f32x8& v) {
  return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}
__device__ __forceinline__ float sum8(const bf16x8& v) { return sum8(__builtin_convertvector(v, f32x8)); }

__device__ __forceinline__ bool finite(const f32x4& v) {
  const float t = __builtin_fmaf(v[3], 0.f, __builtin_fmaf(v[2], 0.f, __builtin_fmaf(v[1], 0.f, v[0] * 0.f)));
  return t == 0.f;   // (NaN where one is not)
}

// scales and moved zero levels of four rows
struct Scale {
  f32x4 s, z;
};
template <class T>
__device__ __forceinline__ Scale load_scale(const Q4Matrix& m, int tile, int g, int lg) {
  const size_t at = ((size_t)tile * m.padded + g) * 16 + 4 * lg;
  const unsigned z = *reinterpret_cast<const unsigned*>(m.z + at);
  Scale v;
  v.s = *reinterpret_cast<const f32x4*>(m.s + at);
#pragma unroll
  for (int i = 0; i < 4; ++i) v.z[i] = (float)((z >> (8 * i)) & 255u) + Parts<T>::kOffset;
  return v;
}

// y rows n, four columns from r
template <class T>
__device__ __forceinline__ void store_y(T* y, const float* bias, int R, size_t n, int r, f32x4 v) {
  T* p = y + n * R + r;
  if (r + 4 <= R) {
    typedef T Four __attribute__((ext_vector_type(4)));
    typedef Four Any __attribute__((aligned(sizeof(T))));
    if (bias)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += bias[r + i];
    *reinterpret_cast<Any*>(p) = __builtin_convertvector(v, Four);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (r + i < R) p[i] = (T)(v[i] + (bias ? bias[r + i] : 0.f));
  }
}

// One result once more, column after column by the formula, in fp64, whose range no sum of
// products of three fp32 numbers leaves; it stays as it was where that is not finite either
// (a scale or the bias is not, or y is beyond its type).
template <class T, int G>
__device__ __forceinline__ void mend_one(const Q4Matrix& m, const T* row, const float* bias, T* to, int r) {
  double t = bias ? (double)bias[r] : 0.0;
#pragma unroll 1
  for (int d = 0; d < m.D && fabs(t) < __builtin_inf(); d += 8) {
    const size_t at = ((size_t)(r >> 4) * m.padded + d / G) * 16 + (r & 15);
    const double s = m.s[at];
    const int z = m.z[at];
    const unsigned w = m.q[place_of(m, r, d).word];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double v = d + e < m.D ? (double)(float)row[d + e] : 0.0;
      t = __builtin_fma(s * (double)((int)((w >> (4 * (e / 2 + 4 * (e & 1)))) & 15u) - z), v, t);
    }
  }
  if (fabs(t) < __builtin_inf()) *to = (T)(float)t;
}

// A finite x from 2^115, or a large scale, takes sums past fp32 where y itself is not:
// lanes whose sums for row n were not finite (`bad`) do those results (rows r .. r + count
// - 1 of each of `tiles` row tiles) over, unless the row of x is not finite itself: its
// results stay as they are.  All lanes of a wave come here, and look through one row of x
// together at a time (4096 rows with an infinity in each, 2048 x 2048, bf16: 151 us, without
// 52).  No call with ordinary values gets here.
template <class T, int G>
__device__ __forceinline__ void mend(const Q4Matrix& m, const T* x, int n, const float* bias, T* y, int r, int tiles, int count,
                                     bool bad) {
  unsigned long long todo = __ballot(bad);
#pragma unroll 1
  while (todo) {
    const int now = __builtin_amdgcn_readlane(n, __builtin_ctzll(todo));
    const bool mine = bad && n == now;
    todo &= ~__ballot(mine);
    const T* row = x + (size_t)now * m.D;
    bool whole = true;
#pragma unroll 1
    for (int k = 8 * lane_now(); k < m.D; k += 512) {
      const f32x8 v = __builtin_convertvector(load_x<T>(row, k, m.D, false, false), f32x8);
#pragma unroll
      for (int e = 0; e < 8; ++e) whole = whole && fabsf(v[e]) < __builtin_inff();
    }
    if (__all(whole) && mine) {
#pragma unroll 1
      for (int i = 0; i < tiles * count; ++i) {
        const int at = r + 16 * (i / count) + i % count;
        T* to = y + (size_t)now * m.R + at;
        if (at < m.R && !(fabsf((float)*to) < __builtin_inff())) mend_one<T, G>(m, row, bias, to, at);
      }
    }
  }
}

// Few rows of x: what bounds it is reading the matrix, so every workgroup reads RT
// row tiles of it once, its KW waves every KW-th block of columns, for up to 16 NT
// rows of x straight from L2; the waves' sums meet in LDS, in order.  A few blocks a wave
// leave it to latency: 48 rows of x, 8192 x 2048, bf16 8.7 us (G = 128: 8.4 MB of levels and 0.7
// of scales; G = 64 11.1); 16 rows, 32768 x 8192 39 us (145 MB, 3.7 TB/s).  fp32 is bound by splitting x
// (44 operations a step of 32 columns, 22 for the levels): 100 rows of 8256 columns, 256
// rows of the matrix, G = 32: 22 us on 112 compute units.  Loading x a block ahead too
// changes nothing.
template <class T, int G, int RT, int NT, int KW>
__global__ void __launch_bounds__(64 * KW) q4_rows_kernel(Q4Matrix m, const T* x, int N, const float* bias, T* y) {
  constexpr int kSteps = kBlockCols / 32, kGroupSteps = G / 32, kParts = Parts<T>::kParts;
  __shared__ f32x4 part[KW][RT * NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4;
  const int tile0 = blockIdx.x * RT, n0 = blockIdx.y * (16 * NT);
  const bool odd = odd_rows(x, m.D);
  const T* row[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) row[t] = x + (size_t)min(n0 + 16 * t + li, N - 1) * m.D;
  f32x4 acc[RT][NT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
  u32x4 w[RT];   // the next block's, under way while a block is multiplied
  auto load_w = [&](int kb) {
#pragma unroll
    for (int r = 0; r < RT; ++r)
      w[r] = *reinterpret_cast<const u32x4*>(
          m.q + (((size_t)min(tile0 + r, m.tiles - 1) * m.blocks + kb) * 64 + lane) * 4);
  };
  if (wave < m.blocks) load_w(wave);
  for (int kb = wave; kb < m.blocks; kb += KW) {
    const bool whole = (kb + 1) * kBlockCols <= m.D;
    typename XVec<T>::Raw xr[kSteps][NT];
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
      for (int t = 0; t < NT; ++t) xr[s][t] = load_x<T>(row[t], kb * kBlockCols + 8 * lg + 32 * s, m.D, whole, odd);
    u32x4 now[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) now[r] = w[r];
    if (kb + KW < m.blocks) load_w(kb + KW);
    f32x4 p[RT][NT], sum[NT];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      if (s % kGroupSteps == 0) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int r = 0; r < RT; ++r) p[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
      }
      bf16x8 a[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) a[r] = Parts<T>::levels(now[r][s]);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const Parts<T> b(xr[s][t]);
#pragma unroll
        for (int k = kParts - 1; k >= 0; --k) {   // the small parts first
          sum[t] = mfma(ones, b.p[k], sum[t]);
#pragma unroll
          for (int r = 0; r < RT; ++r) p[r][t] = mfma(a[r], b.p[k], p[r][t]);
        }
      }
      if (s % kGroupSteps == kGroupSteps - 1) {
        const int g = kb * (kBlockCols / G) + s / kGroupSteps;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const Scale c = load_scale<T>(m, min(tile0 + r, m.tiles - 1), g, lg);
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              acc[r][t][i] = __builtin_fmaf(c.s[i], __builtin_fmaf(-c.z[i], sum[t][i], p[r][t][i]), acc[r][t][i]);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t) part[wave][r * NT + t][lane] = acc[r][t];
  __syncthreads();
  for (int j = wave; j < RT * NT; j += KW) {
    const int r = j / NT, t = j % NT, n = n0 + 16 * t + li, at = (tile0 + r) * 16 + 4 * lg;
    f32x4 v = part[0][j][lane];
#pragma unroll
    for (int k = 1; k < KW; ++k) v += part[k][j][lane];
    const bool here = n < N && at < m.R;
    if (here) store_y<T>(y, bias, m.R, n, at, v);
    if (__any(here && !finite(v))) mend<T, G>(m, x, n, bias, y, at, 1, 4, here && !finite(v));
  }
}

// One or two rows of x in fp32: with 14 of 16 columns of an operand idle, splitting x
// and centring the levels costs more than multiplying on the vector units.  A lane
// has the row of the matrix and the columns that its words hold; its products begin
// at -z sum x, so that they end up no larger than they have to be.  32768 x 8192, fp32:
// 32.5 us for 145 MB (4.5 TB/s; cached loads of the levels 35 us, the row kernel 59).
template <class T, int G, int RT, int NX, int KW>
__global__ void __launch_bounds__(64 * KW) q4_dot_kernel(Q4Matrix m, const T* x, int N, const float* bias, T* y) {
  constexpr int kSteps = kBlockCols / 32, kGroupSteps = G / 32, kGroups = kBlockCols / G;
  __shared__ float part[KW][RT * NX][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4, tile0 = blockIdx.x * RT;
  const bool odd = odd_rows(x, m.D);
  float acc[RT][NX] = {};
  const unsigned* wp[RT];
  size_t at_scale[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const size_t tile = (size_t)min(tile0 + r, m.tiles - 1);
    wp[r] = m.q + (tile * m.blocks * 64 + lane) * 4;
    at_scale[r] = tile * m.padded * 16 + li;
  }
  u32x4 w[RT];
  float s[RT][kGroups];
  unsigned z[RT][kGroups];
  auto load = [&](int kb) {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      w[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(wp[r] + (size_t)kb * 256));
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        s[r][g] = m.s[at_scale[r] + (size_t)(kb * kGroups + g) * 16];
        z[r][g] = m.z[at_scale[r] + (size_t)(kb * kGroups + g) * 16];
      }
    }
  };
  for (int kb = wave; kb < m.blocks; kb += KW) {
    load(kb);
    const int k0 = kb * kBlockCols + 8 * lg;
    const bool whole = (kb + 1) * kBlockCols <= m.D;
    f32x8 xv[kSteps][NX];
    float sum[kSteps][NX];
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
#pragma unroll
      for (int n = 0; n < NX; ++n) {
        xv[k][n] = __builtin_convertvector(load_x<T>(x + (size_t)min(n, N - 1) * m.D, k0 + 32 * k, m.D, whole, odd), f32x8);
        sum[k][n] = sum8(xv[k][n]);
      }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        float t[NX] = {};
        const float zf = -(float)z[r][g];
#pragma unroll
        for (int j = 0; j < kGroupSteps; ++j) {
          const int k = g * kGroupSteps + j;
          const unsigned a = w[r][k] & 0x0F0F0F0Fu, b = (w[r][k] >> 4) & 0x0F0F0F0Fu;
          // bytes of a: columns 0, 4, 1, 5; of b: 2, 6, 3, 7
          const float q[8] = {(float)(a & 255u), (float)((a >> 16) & 255u), (float)(b & 255u), (float)((b >> 16) & 255u),
                              (float)((a >> 8) & 255u), (float)(a >> 24), (float)((b >> 8) & 255u), (float)(b >> 24)};
#pragma unroll
          for (int n = 0; n < NX; ++n) {
            t[n] = __builtin_fmaf(zf, sum[k][n], t[n]);
#pragma unroll
            for (int e = 0; e < 8; ++e) t[n] = __builtin_fmaf(q[e], xv[k][n][e], t[n]);
          }
        }
#pragma unroll
        for (int n = 0; n < NX; ++n) acc[r][n] = __builtin_fmaf(s[r][g], t[n], acc[r][n]);
      }
  }
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int n = 0; n < NX; ++n) part[wave][r * NX + n][lane] = acc[r][n];
  __syncthreads();
  for (int j0 = 64 * wave; j0 < 16 * RT * NX; j0 += 64 * KW) {
    const int j = j0 + lane, i = j & 15, k = min(j >> 4, RT * NX - 1), n = k % NX, at = (tile0 + k / NX) * 16 + i;
    const bool here = j < 16 * RT * NX && n < N && at < m.R;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w)
#pragma unroll
      for (int g = 0; g < 4; ++g) v += part[w][k][16 * g + i];
    if (here) y[(size_t)n * m.R + at] = (T)(v + (bias ? bias[at] : 0.f));
    const bool bad = here && !(fabsf(v) < __builtin_inff());
    if (__any(bad)) mend<T, G>(m, x, n, bias, y, at, 1, 1, bad);
  }
}

// Many rows of x: a matrix product.  A workgroup takes 256 rows of the matrix and 64
// or 32 of x; its four waves 64 rows each, whose levels go from the store to operands
// without LDS (nobody else needs them), while x, which all four need, is staged
// there a block of columns at a time, the next block's loads under way meanwhile; with
// KS = 2 there are eight, the second four on every other block of columns.  The
// group sums of x are formed by the threads that stage it, and the scales stand beside
// them.  4096 rows of x, 2048 x 2048, bf16, G = 128: 45 to 50 us (690 to 764 TFLOP/s, a large
// library product in bf16 1210 to 1280); R = 8192 181 us (760).  A wave's block is 64 matrix
// instructions (1024 cycles) and 380 others (1500): bound by those and, at two
// waves a unit, by the wait for the next block of x.  Tried: loads two blocks ahead in
// registers (spills: 57 us); scales read at the end of a group instead of staged (67).
constexpr int kTileRows = 256, kTileThreads = 256;
constexpr int kTileLd = kBlockCols + 8;   // LDS row (bf16): 16-byte reads of 16 rows in distinct banks

template <class T, int G, int X>
struct TileLds {
  alignas(16) uint16_t x[Parts<T>::kParts][X][kTileLd];
  alignas(16) float s[kBlockCols / G][kTileRows];   // scales and moved zero levels of the rows
  alignas(16) float z[kBlockCols / G][kTileRows];
  float sum[kBlockCols / G][X];                     // group sums of x
};

template <class T, int G, int NT, int KS>
__global__ void __launch_bounds__(kTileThreads * KS, NT == 4 || KS == 2 || sizeof(T) == 4 ? 2 : 3)
    q4_tile_kernel(Q4Matrix m, const T* x, int N, const float* bias, T* y,
                                                               int row_blocks, int x_blocks) {
  constexpr int RT = 4, kTileX = 16 * NT, kSteps = kBlockCols / 32, kGroupSteps = G / 32, kGroups = kBlockCols / G,
                kParts = Parts<T>::kParts, kChunks = kTileX * kBlockCols / 8 / kTileThreads;
  __shared__ TileLds<T, G, kTileX> lds[KS][2];
  const int part = __builtin_amdgcn_readfirstlane(threadIdx.x / kTileThreads), tid = threadIdx.x % kTileThreads;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, lg = lane >> 4;
  // consecutive workgroups go to the 8 XCDs in turn: an XCD takes whole blocks of x
  const int b = blockIdx.x, xb = (b % 8) + 8 * (b / (8 * row_blocks)), rb = (b / 8) % row_blocks;
  if (xb >= x_blocks) return;
  const int tile0 = rb * (kTileRows / 16) + wave * RT, n0 = xb * kTileX;
  const T* row[kChunks];
  int col[kChunks];
#pragma unroll
  for (int j = 0; j < kChunks; ++j) {
    const int i = tid + kTileThreads * j;
    row[j] = x + (size_t)min(n0 + i / 16, N - 1) * m.D;
    col[j] = (i % 16) * 8;
  }
  const unsigned* wp[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) wp[r] = m.q + ((size_t)min(tile0 + r, m.tiles - 1) * m.blocks * 64 + lane) * 4;
  const size_t at_scale = (size_t)min(rb * (kTileRows / 16) + tid / 16, m.tiles - 1) * m.padded * 16 + (tid & 15);
  typename XVec<T>::Raw xr[kChunks];
  u32x4 w[RT];
  float rs[kGroups];
  unsigned rz[kGroups];
  auto load = [&](int kb) {
    const bool whole = (kb + 1) * kBlockCols <= m.D;
#pragma unroll
    for (int j = 0; j < kChunks; ++j) xr[j] = load_x<T>(row[j], kb * kBlockCols + col[j], m.D, whole, false);
#pragma unroll
    for (int r = 0; r < RT; ++r) w[r] = *reinterpret_cast<const u32x4*>(wp[r] + (size_t)kb * 256);
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      rs[g] = m.s[at_scale + (size_t)(kb * kGroups + g) * 16];
      rz[g] = m.z[at_scale + (size_t)(kb * kGroups + g) * 16];
    }
  };
  f32x4 acc[RT][NT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  load(min(part, m.blocks - 1));
  for (int it = 0; it * KS < m.blocks; ++it) {
    const int kb = it * KS + part;
    TileLds<T, G, kTileX>& l = lds[part][it % 2];
    u32x4 now[RT];
#pragma unroll
    for (int j = 0; j < kChunks; ++j) {
      const int i = tid + kTileThreads * j;
      const Parts<T> v(xr[j]);
#pragma unroll
      for (int k = 0; k < kParts; ++k) *reinterpret_cast<bf16x8*>(&l.x[k][i / 16][(i % 16) * 8]) = v.p[k];
      const float s = group_sum<G / 8>(sum8(xr[j]));
      if (i % (G / 8) == 0) l.sum[(i % 16) / (G / 8)][i / 16] = s;
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      l.s[g][tid] = rs[g];
      l.z[g][tid] = (float)rz[g] + Parts<T>::kOffset;
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) now[r] = w[r];
    lds_barrier();
    if (kb >= m.blocks) break;   // (in the last round alone)
    if (kb + KS < m.blocks) load(kb + KS);
    f32x4 p[RT][NT];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      if (s % kGroupSteps == 0) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int t = 0; t < NT; ++t) p[r][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      bf16x8 a[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) a[r] = Parts<T>::levels(now[r][s]);
#pragma unroll
      for (int k = kParts - 1; k >= 0; --k)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const bf16x8 v = *reinterpret_cast<const bf16x8*>(&l.x[k][16 * t + li][32 * s + 8 * lg]);
#pragma unroll
          for (int r = 0; r < RT; ++r) p[r][t] = mfma(a[r], v, p[r][t]);
        }
      if (s % kGroupSteps == kGroupSteps - 1) {
        const int g = s / kGroupSteps;
        float sum[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[t] = l.sum[g][16 * t + li];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const f32x4 cs = *reinterpret_cast<const f32x4*>(&l.s[g][64 * wave + 16 * r + 4 * lg]);
          const f32x4 cz = *reinterpret_cast<const f32x4*>(&l.z[g][64 * wave + 16 * r + 4 * lg]);
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              acc[r][t][i] = __builtin_fmaf(cs[i], __builtin_fmaf(-cz[i], sum[t], p[r][t][i]), acc[r][t][i]);
        }
      }
    }
  }
  if constexpr (KS == 2) {   // the second half's sums onto the first's, through the buffers
    static_assert(sizeof(lds) >= sizeof(f32x4) * 64 * 4 * RT * NT, "room for the sums");
    f32x4(*sums)[RT * NT][64] = reinterpret_cast<f32x4(*)[RT * NT][64]>(&lds);
    lds_barrier();
    if (part == 1)
#pragma unroll
      for (int j = 0; j < RT * NT; ++j) sums[wave][j][lane] = acc[j / NT][j % NT];
    lds_barrier();
    if (part == 1) return;
#pragma unroll
    for (int j = 0; j < RT * NT; ++j) acc[j / NT][j % NT] += sums[wave][j][lane];
  }
  const int now = lane_now(), ci = now & 15, cg = now >> 4;
  unsigned bad = 0;   // bit t: sums of the t-th 16 rows of x that are not finite
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int n = n0 + 16 * t + ci, at = (tile0 + r) * 16 + 4 * cg;
      if (n < N && at < m.R) store_y<T>(y, bias, m.R, n, at, acc[r][t]);
      bad |= finite(acc[r][t]) ? 0u : 1u << t;
    }
  if (__any(bad != 0))
#pragma unroll 1
    for (int t = 0; t < NT; ++t) {
      const int n = n0 + 16 * t + ci;
      mend<T, G>(m, x, n, bias, y, tile0 * 16 + 4 * cg, RT, 4, n < N && (bad >> t & 1));
    }
}

template <class T, int G, int NT, int KS>
void launch_tile(const Q4Matrix& m, const T* x, int N, const float* bias, T* y, hipStream_t stream) {
  const int rb = (m.R + kTileRows - 1) / kTileRows, xb = (N + 16 * NT - 1) / (16 * NT);
  q4_tile_kernel<T, G, NT, KS><<<(unsigned)((xb + 7) / 8 * 8 * rb), kTileThreads * KS, 0, stream>>>(m, x, N, bias, y, rb, xb);
}

template <class T, int G, int RT, int NT, int KW>
void launch_rows(const Q4Matrix& m, const T* x, int N, const float* bias, T* y, hipStream_t stream) {
  const dim3 grid((m.tiles + RT - 1) / RT, (N + 16 * NT - 1) / (16 * NT));
  q4_rows_kernel<T, G, RT, NT, KW><<<grid, 64 * KW, 0, stream>>>(m, x, N, bias, y);
}

template <class T, int G, int RT, int NX, int KW>
void launch_dot(const Q4Matrix& m, const T* x, int N, const float* bias, T* y, hipStream_t stream) {
  q4_dot_kernel<T, G, RT, NX, KW><<<(m.tiles + RT - 1) / RT, 64 * KW, 0, stream>>>(m, x, N, bias, y);
}

template <class T, int G>
void launch_group(const Q4Matrix& m, const T* x, int N, const float* bias, T* y, int num_cu, hipStream_t stream) {
  constexpr bool kHalf = sizeof(T) == 2;
  const Q4Form f = q4_form(m, N, kHalf, num_cu);
  auto is = [&](Q4Kernel k, int tiles, int x_rows, int split) {
    return f.kernel == k && f.tiles == tiles && f.x == x_rows && f.split == split;
  };
  if constexpr (kHalf) {
    if (is(kQ4Tile, 4, 4, 1)) return launch_tile<T, G, 4, 1>(m, x, N, bias, y, stream);
  } else {
    if (is(kQ4Dot, 2, 2, 8)) return launch_dot<T, G, 2, 2, 8>(m, x, N, bias, y, stream);
    if (is(kQ4Dot, 1, 2, 16)) return launch_dot<T, G, 1, 2, 16>(m, x, N, bias, y, stream);
  }
  if (is(kQ4Tile, 4, 2, 1)) launch_tile<T, G, 2, 1>(m, x, N, bias, y, stream);
  else if (is(kQ4Tile, 4, 2, 2)) launch_tile<T, G, 2, 2>(m, x, N, bias, y, stream);
  else if (is(kQ4Dot, 4, 1, 8)) launch_dot<T, G, 4, 1, 8>(m, x, N, bias, y, stream);
  else if (is(kQ4Dot, 2, 1, 8)) launch_dot<T, G, 2, 1, 8>(m, x, N, bias, y, stream);
  else if (is(kQ4Dot, 1, 1, 16)) launch_dot<T, G, 1, 1, 16>(m, x, N, bias, y, stream);
  else if (is(kQ4Rows, 4, 1, 8)) launch_rows<T, G, 4, 1, 8>(m, x, N, bias, y, stream);
  else if (is(kQ4Rows, 2, 1, 8)) launch_rows<T, G, 2, 1, 8>(m, x, N, bias, y, stream);
  else if (is(kQ4Rows, 4, 2, 8)) launch_rows<T, G, 4, 2, 8>(m, x, N, bias, y, stream);
  else if (is(kQ4Rows, 2, 2, 8)) launch_rows<T, G, 2, 2, 8>(m, x, N, bias, y, stream);
  else launch_rows<T, G, 1, 1, 16>(m, x, N, bias, y, stream);
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

// What both sides took, in us, D = 2048 unless given:
// - many rows of x: the tile kernel once the row kernel (32 of them and 64 of the matrix a
//   workgroup) makes more than two workgroups a unit.  Row kernel / tile kernel: two a
//   unit, R = 2048, N = 512, bf16 16.8 / 18.7, fp32 28.7 / 31.6, R = 8192, N = 128 16.3 / 19.9,
//   28.9 / 33.9 (but N > R, x past the caches: R = 256, N = 4096 18.8 / 18.0, 40 / 32.5); more,
//   N = 640 23.4 / 18.7, 41 / 32; N = 1024 31 / 19, 54 / 33; R = 256, N = 8192 34 / 20, 69 /
//   37.  64 rows of x at a time where that makes two a unit (bf16, 4096 x 2048: 49, 32 at a
//   time 54; 2048 x 2048: 36 and 31), in fp32 always 32 (8192 x 2048: 211, 64 at a time
//   254 with spilled registers); the columns in two halves where there is at most a
//   workgroup a unit (R = 2048, N = 1024, bf16 19, whole 23, fp32 34 and 40; R = 3716, D =
//   2951, N = 730, 345 workgroups: 52 and 45).
// - one row, in fp32 two: the dot kernel (fp32, G = 32, R = 32768, D = 8192: 40, row
//   kernel 113; R = 2048, D = 8256: 10, 16), as many row tiles a workgroup as leave
//   two workgroups a unit, and sixteen waves where there are fewer than one (R = 2048,
//   D = 8256: 8.4, eight waves 14).
// - else the row kernel, in the widest shape that still has a workgroup a unit: fp32,
//   R = 8192, N = 12: 32 x 16 7.2, 64 x 16 10.4; N = 48 64 x 32 15, 32 x 64 19; R = 256,
//   D = 8256, N = 100: 16 x 16 23, 32 x 64 87.  Below that 16 x 16 on sixteen waves, but
//   32 x 32 once they do not all run at once (bf16, G = 32, R = 1000, D = 2000, N = 200:
//   13 and 7.8; R = 2048, D = 4096, N = 64, two a unit: 10.4 and 11.9).
Q4Form q4_form(const Q4Matrix& m, int N, int bf16, int num_cu) {
  const size_t tiles = m.tiles, cu = num_cu;
  auto cover = [](size_t n, size_t by) { return (n + by - 1) / by; };
  const size_t wide = cover(m.R, kTileRows) * cover(N, 64), narrow = cover(m.R, kTileRows) * cover(N, 32);
  if (N > 64 && bf16 && wide >= 2 * cu) return {kQ4Tile, 4, 4, 1};
  if (N > 64 && narrow > cu) return {kQ4Tile, 4, 2, 1};
  if (N > 64 && (2 * narrow > cu || (2 * narrow == cu && N > m.R))) return {kQ4Tile, 4, 2, 2};
  if (N == 1 && tiles >= 4 * cu) return {kQ4Dot, 4, 1, 8};
  if (N == 1 && tiles >= 2 * cu) return {kQ4Dot, 2, 1, 8};
  if (N == 1) return {kQ4Dot, 1, 1, 16};
  if (N == 2 && !bf16) return tiles >= 2 * cu ? Q4Form{kQ4Dot, 2, 2, 8} : Q4Form{kQ4Dot, 1, 2, 16};
  if (N <= 16 && tiles >= 4 * cu) return {kQ4Rows, 4, 1, 8};
  if (N <= 16 && tiles >= 2 * cu) return {kQ4Rows, 2, 1, 8};
  if (N > 16 && cover(tiles, 4) * cover(N, 32) >= cu) return {kQ4Rows, 4, 2, 8};
  if (N > 16 && (cover(tiles, 2) * cover(N, 32) >= cu || tiles * cover(N, 16) > 2 * cu)) return {kQ4Rows, 2, 2, 8};
  return {kQ4Rows, 1, 1, 16};
}

void q4_shape(Q4Matrix& m, int R, int D, int G) {
  m.R = R, m.D = D, m.G = G;
  m.groups = (D + G - 1) / G;
  m.tiles = (R + 15) / 16;
  m.blocks = (D + kBlockCols - 1) / kBlockCols;
  m.padded = m.blocks * (kBlockCols / G);
}

size_t q4_bytes(const Q4Matrix& m) {
  const size_t scales = (size_t)m.tiles * m.padded * 16;
  return (size_t)m.tiles * m.blocks * 1024 + up256(scales * 4) + up256(scales);
}

void q4_place(Q4Matrix& m, uint8_t* store) {
  const size_t scales = (size_t)m.tiles * m.padded * 16;
  m.q = reinterpret_cast<unsigned*>(store);
  store += (size_t)m.tiles * m.blocks * 1024;
  m.s = reinterpret_cast<float*>(store);
  m.z = store + up256(scales * 4);
}

hipError_t launch_q4_layout(const Q4Matrix& m, const uint8_t* q, const float* scale, const uint8_t* zero, int* bad,
                            hipStream_t stream) {
  q4_layout_kernel<<<2048, 256, 0, stream>>>(m, q, scale, zero, bad);
  return hipGetLastError();
}

hipError_t launch_q4_unpack(const Q4Matrix& m, uint8_t* q, float* scale, uint8_t* zero, hipStream_t stream) {
  q4_unpack_kernel<<<2048, 256, 0, stream>>>(m, q, scale, zero);
  return hipGetLastError();
}

hipError_t launch_q4(const Q4Matrix& m, const void* x, int N, int bf16, const float* bias, void* y, int num_cu,
                     hipStream_t stream) {
  auto go = [&](auto g) {
    constexpr int G = decltype(g)::value;
    for (int n = 0; n < N; n += std::min(N - n, kQ4MostRows)) {
      const int c = std::min(N - n, kQ4MostRows);
      const size_t in = (size_t)n * m.D, out = (size_t)n * m.R;
      if (bf16) launch_group<__bf16, G>(m, (const __bf16*)x + in, c, bias, (__bf16*)y + out, num_cu, stream);
      else launch_group<float, G>(m, (const float*)x + in, c, bias, (float*)y + out, num_cu, stream);
    }
  };
  if (m.G == 32) go(std::integral_constant<int, 32>{});
  else if (m.G == 64) go(std::integral_constant<int, 64>{});
  else go(std::integral_constant<int, 128>{});
  return hipGetLastError();
}

}  // namespace alstm
