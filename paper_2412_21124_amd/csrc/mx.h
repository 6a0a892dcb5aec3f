// What the kernels on microscaled matrices share: eight elements of a lane, blocks of 32 in four lanes, and the two code formats.
#ifndef NT_MX_H
#define NT_MX_H
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "normtest.h"

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
// one access per lane whatever the alignment: gfx950 serves global loads and stores of 8 and 16 bytes from any element's address
typedef uint32_t u32_any __attribute__((aligned(1)));
typedef uint32_t u32x4_half __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_word __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_byte __attribute__((ext_vector_type(4), aligned(1)));

#define NT_MX_BLOCK 32
constexpr int code_bytes(int format) { return format == NT_MX_E2M1 ? 16 : 32; }   // of a block
__host__ __device__ inline constexpr int64_t blocks_of(int64_t n) { return (n + NT_MX_BLOCK - 1) / NT_MX_BLOCK; }
__host__ __device__ inline constexpr int type_bytes(int dtype) { return dtype == NT_F32 ? 4 : 2; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int hip_code(hipError_t e) { return e == hipSuccess ? NT_OK : NT_ERR_HIP_BASE - (int)e; }
inline bool finite_in_fp32(double x) { return std::isfinite((float)x); }

// A matrix of numbers as an argument: any element-aligned address, ld >= cols.
inline int check_matrix(const void* p, int dtype, int64_t rows, int64_t cols, int64_t ld) {
  if (dtype < 0 || dtype > 2) return NT_ERR_UNSUPPORTED;
  if (rows < 0 || cols < 0) return NT_ERR_BAD_ARG;
  if (rows == 0 || cols == 0) return NT_OK;
  if (!p || ((uintptr_t)p & (type_bytes(dtype) - 1)) || (rows > 1 && ld < cols)) return NT_ERR_BAD_ARG;
  if (rows > 1 && ld > (1ll << 60) / rows) return NT_ERR_TOO_LARGE;
  return cols > 1ll << 60 ? NT_ERR_TOO_LARGE : NT_OK;
}
inline int check_mx(const nt_mx& m) {
  if (m.format != NT_MX_E2M1 && m.format != NT_MX_E4M3) return NT_ERR_UNSUPPORTED;
  if (m.rows < 0 || m.cols < 0 || m.reserved != 0) return NT_ERR_BAD_ARG;
  if (m.rows == 0 || m.cols == 0) return NT_OK;
  if (m.cols > 1ll << 56) return NT_ERR_TOO_LARGE;
  if (!m.codes || !m.scales || ((uintptr_t)m.codes & 15) || (m.ld & 15) || m.ld < blocks_of(m.cols) * code_bytes(m.format) ||
      m.scale_ld < blocks_of(m.cols))
    return NT_ERR_BAD_ARG;
  return m.ld > (1ll << 60) / m.rows || m.scale_ld > (1ll << 60) / m.rows ? NT_ERR_TOO_LARGE : NT_OK;
}

// A number for block b of `total`, so that the blocks that one of the eight dies is given (every eighth) have neighbouring ones.
__device__ inline uint32_t by_die(uint32_t b, uint32_t total) {
  const uint32_t each = total / 8, more = total % 8, die = b % 8;
  return b / 8 + die * each + (die < more ? die : more);
}
// Which of down x across tiles block b of as many takes: numbered so that the blocks that one of the eight dies is given (every eighth) are
// neighbours, 8 rows of tiles at a time.
__device__ inline void tile_at(uint32_t b, uint32_t total, uint32_t down, uint32_t across, int64_t& m, int64_t& n) {
  const uint32_t t = by_die(b, total);
  const uint32_t group = t / (8 * across), first = group * 8, high = down - first < 8 ? down - first : 8, in = t - group * 8 * across;
  m = first + in % high;
  n = in / high;
}

// ---- eight elements of a lane --------------------------------------------------------------

template <int DT>
struct Raw {   // as loaded
  u32x4 w[DT == NT_F32 ? 2 : 1];
};
template <int DT>
__device__ inline Raw<DT> load8(const void* p) {
  Raw<DT> r;
  if (DT == NT_F32) {
    r.w[0] = ((const u32x4_word*)p)[0];
    r.w[DT == NT_F32] = ((const u32x4_word*)p)[1];
  } else {
    r.w[0] = *(const u32x4_half*)p;
  }
  return r;
}
// The first n < 8, zeros behind them: four, two and one of them as n's bits say, each with an access of its own.  (Element by element the
// seven branches, eight octets to a thread, ran out of scalar registers.)
template <int DT>
__device__ inline Raw<DT> load_part(const void* p, int n) {
  typedef uint32_t word_half __attribute__((aligned(2)));
  typedef uint32_t u32x2_half __attribute__((ext_vector_type(2), aligned(2)));
  typedef uint32_t u32x2_word __attribute__((ext_vector_type(2), aligned(4)));
  Raw<DT> r;
  r.w[0] = r.w[DT == NT_F32] = u32x4{0u, 0u, 0u, 0u};
  if (n <= 0) return r;
  const char* at = (const char*)p;
  if (DT == NT_F32) {
    u32x4 four = {0u, 0u, 0u, 0u};
    u32x2 two = {0u, 0u};
    uint32_t one = 0;
    if (n & 4) four = *(const u32x4_word*)at, at += 16;
    if (n & 2) two = *(const u32x2_word*)at, at += 8;
    if (n & 1) one = *(const uint32_t*)at;
    const uint32_t a = n & 2 ? two[0] : one, b = n & 2 ? two[1] : 0u, c = n & 2 ? one : 0u;
    r.w[0] = n & 4 ? four : u32x4{a, b, c, 0u};
    r.w[DT == NT_F32] = n & 4 ? u32x4{a, b, c, 0u} : u32x4{0u, 0u, 0u, 0u};
  } else {
    u32x2 four = {0u, 0u};
    uint32_t two = 0, one = 0;
    if (n & 4) four = *(const u32x2_half*)at, at += 8;
    if (n & 2) two = *(const word_half*)at, at += 4;
    if (n & 1) one = *(const uint16_t*)at;
    const uint32_t a = n & 2 ? two : one, b = n & 2 ? one : 0u;
    r.w[0] = n & 4 ? u32x4{four[0], four[1], a, b} : u32x4{a, b, 0u, 0u};
  }
  return r;
}
template <int DT>
__device__ inline Raw<DT> load_n(const void* p, int n) {
  return n >= 8 ? load8<DT>(p) : load_part<DT>(p, n);
}
template <int DT>
__device__ inline float value(const Raw<DT>& r, int e) {
  if (DT == NT_F32) {
    const uint32_t w = r.w[DT == NT_F32 && e >= 4][e & 3];   // a bit cast of the vector's element itself takes its first one
    return __builtin_bit_cast(float, w);
  }
  const uint32_t w = r.w[0][e >> 1];
  if (DT == NT_BF16) return __builtin_bit_cast(float, (e & 1) ? (w & 0xffff0000u) : (w << 16));
  return (float)__builtin_bit_cast(_Float16, (uint16_t)((e & 1) ? w >> 16 : w));
}
__device__ inline uint32_t half_bits(int dtype, float x) {
  return dtype == NT_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)x) : __builtin_bit_cast(uint16_t, (_Float16)x);
}
template <int DT>
__device__ inline Raw<DT> rounded(const float (&x)[8]) {
  Raw<DT> r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT == NT_F32) {
      r.w[0][i] = __builtin_bit_cast(uint32_t, x[i]);
      r.w[DT == NT_F32][i] = __builtin_bit_cast(uint32_t, x[4 + i]);
    } else {
      r.w[0][i] = half_bits(DT, x[2 * i]) | half_bits(DT, x[2 * i + 1]) << 16;
    }
  }
  return r;
}
template <int DT>
__device__ inline void store_n(void* p, const Raw<DT>& r, int n) {
  if (n >= 8) {
    if (DT == NT_F32) {
      ((u32x4_word*)p)[0] = r.w[0];
      ((u32x4_word*)p)[1] = r.w[DT == NT_F32];
    } else {
      *(u32x4_half*)p = r.w[0];
    }
    return;
  }
  typedef uint32_t word_half __attribute__((aligned(2)));
  typedef uint32_t u32x2_half __attribute__((ext_vector_type(2), aligned(2)));
  typedef uint32_t u32x2_word __attribute__((ext_vector_type(2), aligned(4)));
  char* at = (char*)p;
  if (DT == NT_F32) {
    u32x4 x = r.w[0];
    if (n & 4) *(u32x4_word*)at = x, x = r.w[DT == NT_F32], at += 16;
    if (n & 2) *(u32x2_word*)at = u32x2{x[0], x[1]}, x[0] = x[2], at += 8;
    if (n & 1) *(uint32_t*)at = x[0];
  } else {
    u32x4 x = r.w[0];
    if (n & 4) *(u32x2_half*)at = u32x2{x[0], x[1]}, x[0] = x[2], x[1] = x[3], at += 8;
    if (n & 2) *(word_half*)at = x[0], x[0] = x[1], at += 4;
    if (n & 1) *(uint16_t*)at = (uint16_t)x[0];
  }
}

// ---- blocks and their scales ---------------------------------------------------------------

// largest over four lanes that hold a block, by neighbours within the quad
__device__ inline uint32_t quad_max(uint32_t x) {
  uint32_t y = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true);   // lanes 1 0 3 2
  x = x > y ? x : y;
  y = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true);            // lanes 2 3 0 1
  return x > y ? x : y;
}
__device__ inline uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }
// The scale byte for a block whose largest magnitude has these bits.  floor(log2) is the exponent field; a subnormal's 0 is held at the
// byte 0 as everything below 2^-125 or 2^-119 is.  6 is 1.5 2^2 and 448 is 1.75 2^8: a mantissa beyond asks for one more where it has to fit.
__device__ inline uint32_t scale_byte(int format, bool fit, uint32_t top) {
  const int exponent = (int)(top >> 23);
  if (exponent == 255) return 255u;
  int b = exponent - (format == NT_MX_E2M1 ? 2 : 8);
  if (fit && (top & 0x7fffffu) > (format == NT_MX_E2M1 ? 0x400000u : 0x600000u)) ++b;
  return b < 0 ? 0u : (uint32_t)b;
}
// 2^(127 - byte), by which a block's elements are multiplied; exact, as is the product where it is not far below the smallest code
__device__ inline float shrink(uint32_t byte) { return __builtin_bit_cast(float, byte == 254u ? 0x00400000u : (254u - byte) << 23); }
// 2^(byte - 127); NaN for 255
__device__ inline float grow(uint32_t byte) {
  return __builtin_bit_cast(float, byte == 0u ? 0x00400000u : byte == 255u ? 0x7fc00000u : byte << 23);
}

// x, already scaled, within the format's range, and for a random byte on its grid: up iff noise + 1/2 < 256 times the fraction of a step
template <int FMT>
__device__ inline float clamped(float x) {
  const float most = FMT == NT_MX_E2M1 ? 6.f : 448.f;
  return __builtin_amdgcn_fmed3f(x, -most, most);
}
// Rounding to a format with M bits behind the leading one cuts a binary32 below bit S = 23 - M, and goes up iff what is cut is over (2 noise + 1)
// 2^(S - 9): iff adding 2^S - 1 less that carries.  Below the least normal number 2^E codes are as far apart as in the binade behind it, so 2^E is added
// there before and taken off behind.  That sum is exact where it counts for a 16-bit source (what it rounds off is too small to go up at all),
// but not for an fp32 one, whose fraction is taken apart instead: 16 operations an element against 9.
template <int FMT, bool SHORT>
__device__ inline float chosen(float x, uint32_t noise) {
  constexpr int M = FMT == NT_MX_E2M1 ? 1 : 3, E = FMT == NT_MX_E2M1 ? 0 : -6, S = 23 - M;
  if (SHORT) {
    constexpr float least = FMT == NT_MX_E2M1 ? 1.f : 0.015625f;
    const float a = __builtin_fabsf(x), more = a < least ? least : 0.f;
    const uint32_t carry = ((511u << (S - 9)) - 1u) - (noise << (S - 8));
    const uint32_t bits = (__builtin_bit_cast(uint32_t, a + more) + carry) & ~((1u << S) - 1u);
    return __builtin_copysignf(__builtin_bit_cast(float, bits) - more, x);
  }
  const uint32_t bits = magnitude(x);
  int e = (int)(bits >> 23) - 127;
  e = (e < E ? E : e) - M;
  const float parts = __builtin_bit_cast(float, bits) * __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);   // in steps
  const float low = __builtin_floorf(parts);
  const float up = (float)noise + 0.5f < 256.f * (parts - low) ? low + 1.f : low;
  return __builtin_copysignf(up * __builtin_bit_cast(float, (uint32_t)(127 + e) << 23), x);
}
// two codes, the first one lower; rounded to nearest even.  which: the byte (E2M1) or half word (E4M3) of `into`
template <int FMT, int WHICH>
__device__ inline uint32_t encode2(uint32_t into, float a, float b) {
  if (FMT == NT_MX_E2M1) return (uint32_t)__builtin_amdgcn_cvt_scalef32_pk_fp4_f32(into, a, b, 1.f, FMT == NT_MX_E2M1 ? WHICH : 0);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)into, (WHICH & 1) != 0);
}
// Codes of eight scaled elements: one word (E2M1) or two.
template <int FMT>
__device__ inline u32x2 encode8(const float (&x)[8]) {
  u32x2 r = {0u, 0u};
  if (FMT == NT_MX_E2M1) {
    r[0] = encode2<FMT, 0>(r[0], x[0], x[1]);
    r[0] = encode2<FMT, 1>(r[0], x[2], x[3]);
    r[0] = encode2<FMT, 2>(r[0], x[4], x[5]);
    r[0] = encode2<FMT, 3>(r[0], x[6], x[7]);
  } else {
    r[0] = encode2<FMT, 0>(r[0], x[0], x[1]);
    r[0] = encode2<FMT, 1>(r[0], x[2], x[3]);
    r[1] = encode2<FMT, 0>(r[1], x[4], x[5]);
    r[1] = encode2<FMT, 1>(r[1], x[6], x[7]);
  }
  return r;
}
// Magnitudes of two 16-bit elements to a word, the larger of each half, and a half's bits as those of the same binary32 (NaN and infinity stay such).
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t larger2(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int DT>
__device__ inline uint32_t as_binary32(uint32_t half) {
  if (DT == NT_BF16) return half << 16;
  return __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)half));
}
// bits of the largest magnitude of eight elements
template <int DT>
__device__ inline uint32_t top8(const Raw<DT>& r) {
  if (DT != NT_F32) {
    uint32_t t = r.w[0][0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < 4; ++i) t = larger2(t, r.w[0][i] & 0x7fff7fffu);
    return as_binary32<DT>((t & 0xffffu) > t >> 16 ? t & 0xffffu : t >> 16);
  }
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t m = magnitude(value<DT>(r, e));
    top = m > top ? m : top;
  }
  return top;
}
// Codes of eight elements (zeros behind the row's end) of a block with this scale byte.  SHORT: of a 16-bit type.
template <int FMT, bool NOISE, bool SHORT>
__device__ inline u32x2 codes8(const float (&x)[8], uint32_t byte, const uint64_t noise) {
  const float by = shrink(byte == 255u ? 127u : byte);
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] = clamped<FMT>(x[e] * by);
    if (NOISE) y[e] = chosen<FMT, SHORT>(y[e], (uint32_t)(noise >> (8 * e)) & 255u);
  }
  const u32x2 r = encode8<FMT>(y);
  return byte == 255u ? u32x2{0u, 0u} : r;
}
// Eight elements as loaded, of a block in four lanes: its scale byte, which all four have, and the lane's codes.
template <int DT, int FMT, bool NOISE>
__device__ inline u32x2 quantize8(const Raw<DT>& raw, bool fit, const uint64_t noise, uint32_t& byte) {
  byte = scale_byte(FMT, fit, quad_max(top8<DT>(raw)));
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = value<DT>(raw, e);
  return codes8<FMT, NOISE, DT != NT_F32>(x, byte, noise);
}
// eight values from a lane's codes, before scaling
template <int FMT>
__device__ inline void decode8(const u32x2& c, float (&x)[8]) {
  f32x2 v;
#define NT_DECODE(I, WORD, WHICH)                                                                   \
  v = FMT == NT_MX_E2M1 ? (f32x2)__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[0], 1.f, I)             \
                        : (f32x2)__builtin_amdgcn_cvt_pk_f32_fp8((int)c[WORD], WHICH);              \
  x[2 * I] = v[0];                                                                                  \
  x[2 * I + 1] = v[1]
  NT_DECODE(0, 0, false);
  NT_DECODE(1, 0, true);
  NT_DECODE(2, 1, false);
  NT_DECODE(3, 1, true);
#undef NT_DECODE
}
// the lane's codes of the octet at `at` (of its row)
template <int FMT>
__device__ inline void store_codes(uint8_t* row, int64_t octet, const u32x2& c) {
  if (FMT == NT_MX_E2M1)
    *(uint32_t*)(row + 4 * octet) = c[0];
  else
    *(u32x2*)(row + 8 * octet) = c;
}

}  // namespace
#endif
