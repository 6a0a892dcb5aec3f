// Microscaled matrices: quantisation, its inverse, and the RMS norm with the residual's addition that writes one, forward and backward;
// hand-written for gfx950 (MI355X).  The product of such matrices is in mx_matmul.hip.
//
// All of it is bound by memory, but for quantisation in both directions.  A lane holds eight consecutive elements of a row (16 bytes of a 16-bit type: one access), four lanes a block
// of 32, whose largest magnitude goes round the four by quad permutes; codes and scales come from the registers that the row was read into.
#include "mx.h"

// Sizes and shapes.
#define NT_MX_THREADS 256
#define NT_MX_TILE 128             // rows and columns of a tile that is quantised in both directions
#define NT_MX_MOST_BLOCKS (1u << 20)
#define NT_BWD_BLOCKS 256          // blocks that walk the rows of the norm's backward pass, each with a sum of its own for every column
#define NT_JOIN_COLS 16            // columns and parts at a time of the kernel that adds those up
#define NT_JOIN_PARTS 16
#define NT_NORM_MOST_COLS 32768

namespace {

// ---------------------------------------------------------------------------------------------
// Rows
// ---------------------------------------------------------------------------------------------
// How rows of octets (four for a block) are given to threads: 2^lanes threads of a block to a row, as many rows as fit, `chunks` blocks to
// a longer row.
struct Spread {
  int64_t rows, parts;   // parts: groups of rows times chunks
  uint32_t octets, chunks;
  int lanes;
};
Spread spread_of(int64_t rows, int64_t cols) {
  Spread s;
  s.rows = rows;
  s.octets = (uint32_t)(4 * blocks_of(cols));
  s.lanes = 2;
  while (s.lanes < 8 && (1u << s.lanes) < s.octets) ++s.lanes;
  s.chunks = (s.octets + (1u << s.lanes) - 1) >> s.lanes;
  s.parts = ceil_div(rows, NT_MX_THREADS >> s.lanes) * s.chunks;
  return s;
}
// the row and octet of this thread in a part; false: none
__device__ inline bool place(const Spread& s, int64_t part, int64_t& row, uint32_t& octet) {
  const int64_t group = part / s.chunks;
  row = group * (NT_MX_THREADS >> s.lanes) + (threadIdx.x >> s.lanes);
  octet = (uint32_t)(part - group * s.chunks) * (1u << s.lanes) + (threadIdx.x & ((1u << s.lanes) - 1));
  return row < s.rows && octet < s.octets;
}

struct QuantizeArgs {
  const char* src;
  const uint8_t* noise;
  int64_t rows, cols, ld, noise_ld;
  uint8_t *codes, *scales;
  int64_t code_ld, scale_ld;
  uint8_t *codes_t, *scales_t;
  int64_t code_ld_t, scale_ld_t;
  int fit;
};
__device__ inline uint64_t noise8(const uint8_t* p, int n) {
  typedef uint64_t u64_any __attribute__((aligned(1)));
  if (n >= 8) return *(const u64_any*)p;
  uint64_t r = 0;
#pragma unroll
  for (int e = 0; e < 7; ++e)
    if (e < n) r |= (uint64_t)p[e] << (8 * e);
  return r;
}

// Bound by memory, and for one row (1 x 768: 1.6 us) by a trip to it and the launch.
template <int DT, int FMT, bool NOISE>
__global__ __launch_bounds__(NT_MX_THREADS) void k_mx_rows(QuantizeArgs a, Spread s) {
  for (int64_t part = blockIdx.x; part < s.parts; part += gridDim.x) {
    int64_t row;
    uint32_t octet;
    if (!place(s, part, row, octet)) continue;   // all four lanes of a block, or none
    const int64_t col = 8 * (int64_t)octet, left = a.cols - col;
    const int n = left < 8 ? (int)left : 8;      // may be none or negative: the last block's end
    const Raw<DT> raw = load_n<DT>(a.src + (row * a.ld + col) * type_bytes(DT), n);
    const uint64_t noise = NOISE ? noise8(a.noise + row * a.noise_ld + col, n) : 0;
    uint32_t byte;
    const u32x2 c = quantize8<DT, FMT, NOISE>(raw, a.fit, noise, byte);
    store_codes<FMT>(a.codes + row * a.code_ld, octet, c);
    if ((octet & 3) == 0) a.scales[row * a.scale_ld + (octet >> 2)] = (uint8_t)byte;
  }
}

// ---------------------------------------------------------------------------------------------
// The transpose, and both
// ---------------------------------------------------------------------------------------------
// A tile of 128 x 128 goes through LDS once: rows are quantised from the registers they were loaded into, columns from LDS, two neighbouring ones of 32
// elements to a thread.  Four threads take a column's four blocks, so that a row of the transpose is written 64 or 128 bytes at a time.  Rows
// in LDS are 16 bytes longer than they need, and each 32 of them begin 32 or 64 bytes further on, so that the four blocks of a column lie in
// different banks.  Nothing is loaded while a tile is converted and stored, and two (fp32) to four blocks fit a CU, so memory is not kept busy: 16384 x 8192
// in bf16 to 4 bits takes 98 us, call after call, for 64 at the yardstick's rate, and with random bytes 136 for 85 (165 between a layer's other calls);
// 4096 x 4096 in fp32 26 for 13.  Of the 38 us that random bytes add their own reading is 21, the rest their additions, twice for every element.  Tiles of
// 128: what one writes of a row of the transpose is a whole line of 64 bytes in 4 bits.  They are taken in order of memory: neighbours on one die were slower
// (16384 x 8192 and back 284 -> 309).
template <int DT>
struct Tile {
  static constexpr int E = type_bytes(DT), PITCH = NT_MX_TILE * E + 16, SHIFT = 16 * E, BYTES = NT_MX_TILE * PITCH + 4 * SHIFT;
  static constexpr int NOISE_PITCH = NT_MX_TILE + 4, NOISE_BYTES = NT_MX_TILE * NOISE_PITCH + 4 * 16;
  __device__ static inline int at(int row, int col) { return row * PITCH + (row >> 5) * SHIFT + col * E; }
  __device__ static inline int noise_at(int row, int col) { return row * NOISE_PITCH + (row >> 5) * 16 + col; }
};

template <int DT, int FMT, int FMT_T, bool ROWS, bool NOISE>
__global__ __launch_bounds__(NT_MX_THREADS) void k_mx_both(QuantizeArgs a, uint32_t across, int64_t tiles) {
  typedef Tile<DT> T;
  __shared__ __align__(16) uint8_t lds[T::BYTES];
  __shared__ __align__(16) uint8_t lds_noise[NOISE ? T::NOISE_BYTES : 16];
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const int64_t row0 = tile / across * NT_MX_TILE, col0 = tile % across * NT_MX_TILE;
    constexpr int PER = NT_MX_TILE * NT_MX_TILE / 8 / NT_MX_THREADS, STEP = NT_MX_THREADS / (NT_MX_TILE / 8);
    const int c = 8 * (threadIdx.x % (NT_MX_TILE / 8)), r0 = threadIdx.x / (NT_MX_TILE / 8);
    const int64_t left = a.cols - col0 - c;
    Raw<DT> raw[PER];
    uint64_t noise[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int64_t row = row0 + r0 + i * STEP;
      const int n = row < a.rows && left > 0 ? (left < 8 ? (int)left : 8) : 0;
      raw[i] = load_n<DT>(a.src + (row * a.ld + col0 + c) * type_bytes(DT), n);
      noise[i] = NOISE ? noise8(a.noise + row * a.noise_ld + col0 + c, n) : 0;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int r = r0 + i * STEP;
      *(u32x4*)(lds + T::at(r, c)) = raw[i].w[0];
      if (DT == NT_F32) *(u32x4*)(lds + T::at(r, c) + 16) = raw[i].w[DT == NT_F32];
      if (NOISE) {
        *(uint32_t*)(lds_noise + T::noise_at(r, c)) = (uint32_t)noise[i];
        *(uint32_t*)(lds_noise + T::noise_at(r, c) + 4) = (uint32_t)(noise[i] >> 32);
      }
    }
    if (ROWS) {
      const uint32_t octet = (uint32_t)((col0 + c) / 8);
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int64_t row = row0 + r0 + i * STEP;
        uint32_t byte;
        const u32x2 codes = quantize8<DT, FMT, NOISE>(raw[i], a.fit, noise[i], byte);
        if (row < a.rows && octet < 4 * blocks_of(a.cols)) {
          store_codes<FMT>(a.codes + row * a.code_ld, octet, codes);
          if ((octet & 3) == 0) a.scales[row * a.scale_ld + (octet >> 2)] = (uint8_t)byte;
        }
      }
    }
    __syncthreads();
    // two neighbouring columns to a thread: one access for both
    const int col = 2 * (int)(threadIdx.x >> 2), block = threadIdx.x & 3;
    constexpr int WORDS = DT == NT_F32 ? 2 : 1;
    uint32_t w[32][WORDS], top[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      const uint8_t* p = lds + T::at(32 * block + e, col);
      if (DT == NT_F32) {
        const u32x2 two = *(const u32x2*)p;
        w[e][0] = two[0];
        w[e][WORDS - 1] = two[1];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint32_t m = two[k] & 0x7fffffffu;
          top[k] = m > top[k] ? m : top[k];
        }
      } else {
        w[e][0] = *(const uint32_t*)p;
        top[0] = larger2(top[0], w[e][0] & 0x7fff7fffu);
      }
    }
    if (DT != NT_F32) {
      top[1] = as_binary32<DT>(top[0] >> 16);
      top[0] = as_binary32<DT>(top[0] & 0xffffu);
    }
    u32x2 codes[2][4];
    uint32_t byte[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) byte[k] = scale_byte(FMT_T, a.fit, top[k]);
#pragma unroll
    for (int o = 0; o < 4; ++o) {
      uint64_t noise2[2] = {0, 0};
      float x[2][8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int row = 8 * o + e;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (DT == NT_F32)
            x[k][e] = __builtin_bit_cast(float, w[row][k * (WORDS - 1)]);
          else if (DT == NT_BF16)
            x[k][e] = __builtin_bit_cast(float, k ? w[row][0] & 0xffff0000u : w[row][0] << 16);
          else
            x[k][e] = (float)__builtin_bit_cast(_Float16, (uint16_t)(k ? w[row][0] >> 16 : w[row][0]));
        }
        if (NOISE) {
          const uint32_t two = *(const uint16_t*)(lds_noise + T::noise_at(32 * block + row, col));
          noise2[0] |= (uint64_t)(two & 255u) << (8 * e);
          noise2[1] |= (uint64_t)(two >> 8) << (8 * e);
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) codes[k][o] = codes8<FMT_T, NOISE, DT != NT_F32>(x[k], byte[k], noise2[k]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int64_t row = col0 + col + k, b = row0 / 32 + block;   // of the transpose
      if (row < a.cols && b < blocks_of(a.rows)) {
        uint8_t* const to = a.codes_t + row * a.code_ld_t + b * code_bytes(FMT_T);
        const u32x2(&c)[4] = codes[k];
        if (FMT_T == NT_MX_E2M1) {
          *(u32x4*)to = u32x4{c[0][0], c[1][0], c[2][0], c[3][0]};
        } else {
          ((u32x4*)to)[0] = u32x4{c[0][0], c[0][1], c[1][0], c[1][1]};
          ((u32x4*)to)[1] = u32x4{c[2][0], c[2][1], c[3][0], c[3][1]};
        }
        a.scales_t[row * a.scale_ld_t + b] = (uint8_t)byte[k];
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------
// Back to numbers
// ---------------------------------------------------------------------------------------------
// Bound by the stores: 16384 x 8192 from 4 bits to bf16 72 us (4.7 TB/s).
template <int DT, int FMT>
__global__ __launch_bounds__(NT_MX_THREADS) void k_mx_values(const uint8_t* codes, const uint8_t* scales, int64_t code_ld, int64_t scale_ld,
                                                             int64_t cols, char* out, int64_t ld, Spread s) {
  for (int64_t part = blockIdx.x; part < s.parts; part += gridDim.x) {
    int64_t row;
    uint32_t octet;
    if (!place(s, part, row, octet)) continue;
    const int64_t left = cols - 8 * (int64_t)octet;
    if (left <= 0) continue;
    u32x2 c = {0u, 0u};
    if (FMT == NT_MX_E2M1)
      c[0] = *(const uint32_t*)(codes + row * code_ld + 4 * (int64_t)octet);
    else
      c = *(const u32x2*)(codes + row * code_ld + 8 * (int64_t)octet);
    const float by = grow(scales[row * scale_ld + (octet >> 2)]);
    float x[8];
    decode8<FMT>(c, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= by;
    store_n<DT>(out + (row * ld + 8 * (int64_t)octet) * type_bytes(DT), rounded<DT>(x), left < 8 ? (int)left : 8);
  }
}

// ---------------------------------------------------------------------------------------------
// RMS norm
// ---------------------------------------------------------------------------------------------
// T threads hold a row, V octets each, from its first reading to its codes: x and the residual are read once.  Sums are in an order that
// the shape alone fixes; the squares' in fp64, so that none overflows or vanishes.
// Bound by memory: 16384 x 4096 in bf16 with a sum, to 8 bits, 100 to 102 us (4.7 TB/s; 97 with results rounded twice); one row of 4096 4.2 us, two trips to
// memory with the row's sum between.
template <int T, class F>
__device__ inline F row_sum(F x, F* scratch) {   // over the T threads of a row, in all of them; scratch: one sum a wave
#pragma unroll
  for (int by = 32; by; by >>= 1) x += __shfl_xor(x, by, 64);
  if (T == 64) return x;
  const int wave = threadIdx.x % T / 64;
  __syncthreads();
  if (threadIdx.x % 64 == 0) scratch[wave] = x;
  __syncthreads();
  F r = 0;
#pragma unroll
  for (int w = 0; w < T / 64; ++w) r += scratch[w];
  return r;
}

// 1 / sqrt(x) for a positive x, as the nearest fp32 number and what is left of it: in fp32 of the x over a power of four that lies in 1/2 .. 2, then
// one of Newton's steps in fp64.
__device__ inline float inverse_root(double x, float& rest) {
  const int half = (int)(((uint32_t)__double2hiint(x) >> 20) & 0x7ffu) / 2 - 511;   // 512 for infinity and NaN, which stay such
  const float near = __builtin_ldexpf(1.f / __builtin_sqrtf((float)__builtin_ldexp(x, -2 * half)), -half);
  rest = 0.f;
  if (half == 512) return near;
  const double r = near * (1.5 - 0.5 * (x * near * near));
  rest = (float)(r - (float)r);
  return (float)r;
}

struct NormArgs {
  const char *x, *residual;
  const float* weight;
  char *sum, *out;
  uint8_t *codes, *scales;
  float* rstd;
  int64_t x_ld, residual_ld, sum_ld, out_ld, code_ld, scale_ld, rows;
  int32_t cols, format, fit;
  float eps;
  double each;   // 1 / cols
};

template <int DT, int T, int V>
__global__ __launch_bounds__(T < 256 ? 256 : T) void k_rms_norm(NormArgs a) {
  __shared__ double scratch[16];
  constexpr int ROWS = T < 256 ? 256 / T : 1, E = type_bytes(DT);
  const int lane = threadIdx.x % T;
  constexpr bool AHEAD = T * V <= 2048;   // all of a row's loads before the first is used, where registers allow
  for (int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / T; row < a.rows; row += (int64_t)gridDim.x * ROWS) {
    float h[V][8];
    double squares = 0.;
    Raw<DT> x[AHEAD ? V : 1], r[AHEAD ? V : 1];
    auto load = [&](int v) {
      const int col = 8 * (v * T + lane), n = a.cols - col;
      x[AHEAD ? v : 0] = load_n<DT>(a.x + (row * a.x_ld + col) * E, n);
      if (a.residual) r[AHEAD ? v : 0] = load_n<DT>(a.residual + (row * a.residual_ld + col) * E, n);
    };
    if (AHEAD) {
#pragma unroll
      for (int v = 0; v < V; ++v) load(v);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = 8 * (v * T + lane), n = a.cols - col;
      if (!AHEAD) load(v);
      Raw<DT> stored = x[AHEAD ? v : 0];
#pragma unroll
      for (int e = 0; e < 8; ++e) h[v][e] = value<DT>(stored, e);
      if (a.residual) {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[v][e] += value<DT>(r[AHEAD ? v : 0], e);
        stored = rounded<DT>(h[v]);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[v][e] = value<DT>(stored, e);   // as it is stored: the backward pass reads that
      }
      if (a.sum && n > 0) store_n<DT>(a.sum + (row * a.sum_ld + col) * E, stored, n);
#pragma unroll
      for (int e = 0; e < 8; ++e) squares = __builtin_fma((double)h[v][e], (double)h[v][e], squares);
    }
    squares = row_sum<T>(squares, scratch);
    float rest;
    const float rstd = inverse_root(__builtin_fma(squares, a.each, (double)a.eps), rest);
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
    if (!a.out && !a.codes) continue;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int octet = v * T + lane, col = 8 * octet, n = a.cols - col;
      float y[8];
      // h (rstd + rest) as a number and what is left, times the weight: rounded once to fp32, which `rounded` and quantize8 start from.  (Twice, and
      // with a rounded rstd, moves more elements across a border of their codes; the operations hide behind memory.)
      const Raw<NT_F32> w = a.weight ? load_n<NT_F32>(a.weight + col, n) : Raw<NT_F32>();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float by = a.weight ? value<NT_F32>(w, e) : 1.f, top = h[v][e] * rstd;
        const float low = __builtin_fmaf(h[v][e], rest, __builtin_fmaf(h[v][e], rstd, -top));
        const float all = __builtin_fmaf(top, by, low * by);
        y[e] = all == all ? all : top * by;   // an infinite weight's 0 inf is none of the formula
      }
      if (n < 8) {   // behind the row's end: zero codes, also where rstd is infinite or NaN
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = e < n ? y[e] : 0.f;
      }
      if (a.out && n > 0) store_n<DT>(a.out + (row * a.out_ld + col) * E, rounded<DT>(y), n);
      if (a.codes) {
        uint32_t byte;
        const Raw<NT_F32> exact = rounded<NT_F32>(y);
        const u32x2 c = a.format == NT_MX_E2M1 ? quantize8<NT_F32, NT_MX_E2M1, false>(exact, a.fit, 0, byte)
                                               : quantize8<NT_F32, NT_MX_E4M3, false>(exact, a.fit, 0, byte);
        if (col < 32 * (int)blocks_of(a.cols)) {
          if (a.format == NT_MX_E2M1)
            store_codes<NT_MX_E2M1>(a.codes + row * a.code_ld, octet, c);
          else
            store_codes<NT_MX_E4M3>(a.codes + row * a.code_ld, octet, c);
          if ((octet & 3) == 0) a.scales[row * a.scale_ld + (octet >> 2)] = (uint8_t)byte;
        }
      }
    }
  }
}

struct BackwardArgs {
  const char *dy, *h, *dsum;
  const float *weight, *rstd;
  char* dx;
  float* parts;   // one sum for every column from every block; NULL: not asked for
  int64_t dy_ld, h_ld, dsum_ld, dx_ld, rows;
  int32_t cols;
};

// Blocks walk the rows, R at a time, T threads to a row.  A row is read once where its octets fit a thread's registers beside the columns'
// sums, else twice.  The weight is in LDS: read through the caches for every row it was 2/3 as many bytes again.  With rows side by side the chip is
// full with 256 blocks, so that few sums are left to join (16384 x 4096 in bf16, both kernels, 137 -> 105 to 107 us, 5.0 TB/s; 512 blocks 108).
template <int DT, int T, int V, int R>
__global__ __launch_bounds__(T * R) void k_rms_backward(BackwardArgs a) {
  constexpr int E = type_bytes(DT), COLS = 8 * T * V;
  constexpr bool KEEP = T * V <= 2048;
  __shared__ float scratch[R][T / 64];
  __shared__ __align__(16) float shared[COLS];   // the weight, then the sums of rows beside the first
  const int lane = threadIdx.x % T, beside = threadIdx.x / T;
  for (int i = threadIdx.x; i < COLS; i += T * R) shared[i] = !a.weight ? 1.f : i < a.cols ? a.weight[i] : 0.f;
  __syncthreads();
  float dw[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[v][e] = 0.f;
  for (int64_t row0 = (int64_t)blockIdx.x * R; row0 < a.rows; row0 += (int64_t)gridDim.x * R) {
    const int64_t row = row0 + beside;
    const bool there = row < a.rows;   // all threads take part in the sums
    Raw<DT> dy[KEEP ? V : 1], h[KEEP ? V : 1], s[KEEP ? V : 1];
    auto load = [&](int v, Raw<DT>& y, Raw<DT>& x) {
      const int col = 8 * (v * T + lane), n = there ? a.cols - col : 0;
      y = load_n<DT>(a.dy + (row * a.dy_ld + col) * E, n);
      x = load_n<DT>(a.h + (row * a.h_ld + col) * E, n);
    };
    auto load_sum = [&](int v, Raw<DT>& x) {
      const int col = 8 * (v * T + lane), n = there && a.dx ? a.cols - col : 0;
      x = load_n<DT>(a.dsum + (row * a.dsum_ld + col) * E, n);
    };
    auto weight = [&](int v, int e) { return shared[8 * (v * T + lane) + e]; };
    const float rstd = there ? a.rstd[row] : 0.f;
    float inner = 0.f;
    if (KEEP) {
#pragma unroll
      for (int v = 0; v < V; ++v) load(v, dy[KEEP ? v : 0], h[KEEP ? v : 0]);
      if (a.dsum) {
#pragma unroll
        for (int v = 0; v < V; ++v) load_sum(v, s[KEEP ? v : 0]);
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!KEEP) load(v, dy[0], h[0]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = value<DT>(dy[KEEP ? v : 0], e), hat = value<DT>(h[KEEP ? v : 0], e) * rstd;
        inner = __builtin_fmaf(y * weight(v, e), hat, inner);
        dw[v][e] = __builtin_fmaf(y, hat, dw[v][e]);
      }
    }
    if (!a.dx) continue;
    inner = row_sum<T>(inner, scratch[beside]) / (float)a.cols;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = 8 * (v * T + lane), n = there ? a.cols - col : 0;
      if (!KEEP) {
        load(v, dy[0], h[0]);
        if (a.dsum) load_sum(v, s[0]);
      }
      float d[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float hat = value<DT>(h[KEEP ? v : 0], e) * rstd, back = a.dsum ? value<DT>(s[KEEP ? v : 0], e) : 0.f;
        d[e] = __builtin_fmaf(rstd, __builtin_fmaf(-hat, inner, value<DT>(dy[KEEP ? v : 0], e) * weight(v, e)), back);
      }
      if (n > 0) store_n<DT>(a.dx + (row * a.dx_ld + col) * E, rounded<DT>(d), n);
    }
  }
  if (!a.parts) return;
  // the sums of the rows side by side, one after the other, through LDS to the first
#pragma unroll
  for (int r = 1; r < R; ++r) {
    __syncthreads();
    if (beside == r) {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) shared[8 * (v * T + lane) + e] = dw[v][e];
    }
    __syncthreads();
    if (beside == 0) {
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[v][e] += shared[8 * (v * T + lane) + e];
    }
  }
  if (beside) return;
  float* const to = a.parts + (int64_t)blockIdx.x * a.cols;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int col = 8 * (v * T + lane);
    if (col < a.cols) store_n<NT_F32>(to + col, rounded<NT_F32>(dw[v]), a.cols - col);
  }
}

// dweight <- beta dweight + scale sum over the blocks' sums: 16 columns to a block, every 16th part to a thread, four at a time, joined in order
__global__ __launch_bounds__(NT_JOIN_COLS * NT_JOIN_PARTS) void k_join_columns(const float* parts, int nparts, int32_t cols, float* dweight,
                                                                               float scale, float beta) {
  __shared__ float sums[NT_JOIN_PARTS][NT_JOIN_COLS];
  const int c = threadIdx.x % NT_JOIN_COLS, p0 = threadIdx.x / NT_JOIN_COLS;
  const int64_t col = (int64_t)blockIdx.x * NT_JOIN_COLS + c;
  float x = 0.f;
  if (col < cols) {
    int p = p0;
    for (; p + 3 * NT_JOIN_PARTS < nparts; p += 4 * NT_JOIN_PARTS) {
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = parts[(int64_t)(p + i * NT_JOIN_PARTS) * cols + col];
      x += (y[0] + y[1]) + (y[2] + y[3]);
    }
    for (; p < nparts; p += NT_JOIN_PARTS) x += parts[(int64_t)p * cols + col];
  }
  sums[p0][c] = x;
  __syncthreads();
  if (p0 || col >= cols) return;
  x = 0.f;
#pragma unroll
  for (int p = 0; p < NT_JOIN_PARTS; ++p) x += sums[p][c];
  x *= scale;
  dweight[col] = beta == 0.f ? x : __builtin_fmaf(beta, dweight[col], x);
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
template <class F>
int with_type(int dtype, F f) {
  return dtype == NT_F32 ? f(std::integral_constant<int, NT_F32>()) : dtype == NT_BF16 ? f(std::integral_constant<int, NT_BF16>())
                                                                                       : f(std::integral_constant<int, NT_F16>());
}
template <class F>
int with_format(int format, F f) {
  return format == NT_MX_E2M1 ? f(std::integral_constant<int, NT_MX_E2M1>()) : f(std::integral_constant<int, NT_MX_E4M3>());
}
uint32_t grid_of(int64_t parts) { return (uint32_t)(parts < NT_MX_MOST_BLOCKS ? parts : NT_MX_MOST_BLOCKS); }

template <int T, int V>
struct Shape {
  static constexpr int threads = T, octets = V;
};
// Threads and octets of a row.
template <class F>
int with_shape(int64_t cols, F f) {
  if (cols <= 512) return f(Shape<64, 1>());
  if (cols <= 1024) return f(Shape<64, 2>());
  if (cols <= 2048) return f(Shape<256, 1>());
  if (cols <= 4096) return f(Shape<256, 2>());
  if (cols <= 8192) return f(Shape<256, 4>());
  if (cols <= 16384) return f(Shape<1024, 2>());
  return f(Shape<1024, 4>());
}
// Rows side by side in a block of the backward pass: as many as 1024 threads, or their registers, allow.
template <int T, int V>
constexpr int rows_beside() {
  return T == 64 ? 8 : T == 256 ? (V <= 2 ? 4 : 2) : 1;
}
int64_t backward_blocks(int64_t rows, int64_t cols) {
  const int64_t beside = with_shape(cols, [&](auto s) { return rows_beside<decltype(s)::threads, decltype(s)::octets>(); });
  const int64_t n = ceil_div(rows, beside), most = cols <= 1024 ? 2 * NT_BWD_BLOCKS : NT_BWD_BLOCKS;
  return n < most ? n : most;
}

}  // namespace

extern "C" {

int normtest_mx_quantize(const void* src, nt_dtype dtype, int64_t rows, int64_t cols, int64_t ld, const uint8_t* noise, int64_t noise_ld,
                         const nt_mx* out, const nt_mx* out_t, uint32_t flags, void* hip_stream) {
  int rc = check_matrix(src, dtype, rows, cols, ld);
  if (rc == NT_OK && out) rc = check_mx(*out);
  if (rc == NT_OK && out_t) rc = check_mx(*out_t);
  if (rc != NT_OK) return rc;
  if ((!out && !out_t) || (flags & ~(uint32_t)NT_MX_FIT) || (out && (out->rows != rows || out->cols != cols)) ||
      (out_t && (out_t->rows != cols || out_t->cols != rows)) || (noise && rows > 1 && noise_ld < cols))
    return NT_ERR_BAD_ARG;
  if (rows == 0 || cols == 0) return NT_OK;
  if (cols > 1ll << 33 || (noise && rows > 1 && noise_ld > (1ll << 60) / rows)) return NT_ERR_TOO_LARGE;
  QuantizeArgs a = {(const char*)src, noise, rows, cols, ld, noise_ld, nullptr, nullptr, 0, 0, nullptr, nullptr, 0, 0, (int)(flags & NT_MX_FIT)};
  if (out) {
    a.codes = (uint8_t*)out->codes;
    a.scales = (uint8_t*)out->scales;
    a.code_ld = out->ld;
    a.scale_ld = out->scale_ld;
  }
  hipStream_t st = (hipStream_t)hip_stream;
  if (!out_t) {
    const Spread s = spread_of(rows, cols);
    return with_type(dtype, [&](auto dt) {
      return with_format(out->format, [&](auto f) {
        auto kernel = noise ? k_mx_rows<dt(), f(), true> : k_mx_rows<dt(), f(), false>;
        hipLaunchKernelGGL(kernel, dim3(grid_of(s.parts)), dim3(NT_MX_THREADS), 0, st, a, s);
        return hip_code(hipGetLastError());
      });
    });
  }
  a.codes_t = (uint8_t*)out_t->codes;
  a.scales_t = (uint8_t*)out_t->scales;
  a.code_ld_t = out_t->ld;
  a.scale_ld_t = out_t->scale_ld;
  const int64_t across = ceil_div(cols, NT_MX_TILE), tiles = across * ceil_div(rows, NT_MX_TILE);
  return with_type(dtype, [&](auto dt) {
    return with_format(out ? out->format : out_t->format, [&](auto f) {
      return with_format(out_t->format, [&](auto g) {
        auto kernel = out ? (noise ? k_mx_both<dt(), f(), g(), true, true> : k_mx_both<dt(), f(), g(), true, false>)
                          : (noise ? k_mx_both<dt(), g(), g(), false, true> : k_mx_both<dt(), g(), g(), false, false>);
        hipLaunchKernelGGL(kernel, dim3(grid_of(tiles)), dim3(NT_MX_THREADS), 0, st, a, (uint32_t)across, tiles);
        return hip_code(hipGetLastError());
      });
    });
  });
}

int normtest_mx_dequantize(const nt_mx* src, void* out, nt_dtype dtype, int64_t ld, void* hip_stream) {
  if (!src) return NT_ERR_BAD_ARG;
  int rc = check_mx(*src);
  if (rc == NT_OK) rc = check_matrix(out, dtype, src->rows, src->cols, ld);
  if (rc != NT_OK) return rc;
  if (src->rows == 0 || src->cols == 0) return NT_OK;
  if (src->cols > 1ll << 33) return NT_ERR_TOO_LARGE;
  const Spread s = spread_of(src->rows, src->cols);
  return with_type(dtype, [&](auto dt) {
    return with_format(src->format, [&](auto f) {
      hipLaunchKernelGGL((k_mx_values<dt(), f()>), dim3(grid_of(s.parts)), dim3(NT_MX_THREADS), 0, (hipStream_t)hip_stream, (const uint8_t*)src->codes,
                         (const uint8_t*)src->scales, src->ld, src->scale_ld, src->cols, (char*)out, ld, s);
      return hip_code(hipGetLastError());
    });
  });
}

int normtest_rms_norm(const void* x, int64_t x_ld, const void* residual, int64_t residual_ld, const float* weight, double eps, nt_dtype dtype,
                      int64_t rows, int64_t cols, void* sum_out, int64_t sum_ld, void* out, int64_t out_ld, const nt_mx* out_mx, float* rstd,
                      uint32_t flags, void* hip_stream) {
  int rc = check_matrix(x, dtype, rows, cols, x_ld);
  if (rc == NT_OK && residual) rc = check_matrix(residual, dtype, rows, cols, residual_ld);
  if (rc == NT_OK && sum_out) rc = check_matrix(sum_out, dtype, rows, cols, sum_ld);
  if (rc == NT_OK && out) rc = check_matrix(out, dtype, rows, cols, out_ld);
  if (rc == NT_OK && out_mx) rc = check_mx(*out_mx);
  if (rc != NT_OK) return rc;
  if (((uintptr_t)weight & 3) || ((uintptr_t)rstd & 3) || !((float)eps > 0.f) || !finite_in_fp32(eps) || (flags & ~(uint32_t)NT_MX_FIT) ||
      (out_mx && (out_mx->rows != rows || out_mx->cols != cols)))
    return NT_ERR_BAD_ARG;
  if (cols > NT_NORM_MOST_COLS) return NT_ERR_TOO_LARGE;
  if (rows == 0 || cols == 0) return NT_OK;
  NormArgs a = {(const char*)x, (const char*)residual, weight, (char*)sum_out, (char*)out, nullptr, nullptr, rstd,
                x_ld, residual_ld, sum_ld, out_ld, 0, 0, rows, (int32_t)cols, 0, (int32_t)(flags & NT_MX_FIT), (float)eps, 1. / (double)cols};
  if (out_mx) {
    a.codes = (uint8_t*)out_mx->codes;
    a.scales = (uint8_t*)out_mx->scales;
    a.code_ld = out_mx->ld;
    a.scale_ld = out_mx->scale_ld;
    a.format = out_mx->format;
  }
  return with_type(dtype, [&](auto dt) {
    return with_shape(cols, [&](auto s) {
      constexpr int T = s.threads, V = s.octets, ROWS = T < 256 ? 256 / T : 1;
      hipLaunchKernelGGL((k_rms_norm<dt(), T, V>), dim3(grid_of(ceil_div(rows, ROWS))), dim3(T < 256 ? 256 : T), 0, (hipStream_t)hip_stream, a);
      return hip_code(hipGetLastError());
    });
  });
}

size_t normtest_rms_norm_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || cols > NT_NORM_MOST_COLS) return 0;
  return (size_t)(backward_blocks(rows, cols) * cols) * sizeof(float);
}

int normtest_rms_norm_backward(const void* dy, int64_t dy_ld, const void* h, int64_t h_ld, const float* weight, const float* rstd,
                               const void* dsum, int64_t dsum_ld, nt_dtype dtype, int64_t rows, int64_t cols, void* dx, int64_t dx_ld,
                               float* dweight, double scale, double beta, void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = check_matrix(dy, dtype, rows, cols, dy_ld);
  if (rc == NT_OK) rc = check_matrix(h, dtype, rows, cols, h_ld);
  if (rc == NT_OK && dsum) rc = check_matrix(dsum, dtype, rows, cols, dsum_ld);
  if (rc == NT_OK && dx) rc = check_matrix(dx, dtype, rows, cols, dx_ld);
  if (rc != NT_OK) return rc;
  if (((uintptr_t)weight & 3) || ((uintptr_t)rstd & 3) || ((uintptr_t)dweight & 3) || (!rstd && rows > 0 && cols > 0) || (!dx && !dweight) ||
      !finite_in_fp32(scale) || !finite_in_fp32(beta))
    return NT_ERR_BAD_ARG;
  if (cols > NT_NORM_MOST_COLS) return NT_ERR_TOO_LARGE;
  if (cols == 0 || (rows == 0 && !dweight)) return NT_OK;
  const int64_t blocks = backward_blocks(rows, cols);
  if (dweight && rows > 0) {
    if (workspace_bytes < normtest_rms_norm_workspace_bytes(rows, cols) || !workspace) return NT_ERR_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)workspace & 15) return NT_ERR_BAD_ARG;
  }
  hipStream_t st = (hipStream_t)hip_stream;
  if (rows > 0) {
    const BackwardArgs a = {(const char*)dy, (const char*)h, (const char*)dsum, weight, rstd, (char*)dx, dweight ? (float*)workspace : nullptr,
                            dy_ld, h_ld, dsum_ld, dx_ld, rows, (int32_t)cols};
    rc = with_type(dtype, [&](auto dt) {
      return with_shape(cols, [&](auto s) {
        constexpr int T = s.threads, V = s.octets, R = rows_beside<T, V>();
        hipLaunchKernelGGL((k_rms_backward<dt(), T, V, R>), dim3((uint32_t)blocks), dim3(T * R), 0, st, a);
        return hip_code(hipGetLastError());
      });
    });
    if (rc != NT_OK || !dweight) return rc;
  }
  hipLaunchKernelGGL(k_join_columns, dim3((uint32_t)ceil_div(cols, NT_JOIN_COLS)), dim3(NT_JOIN_COLS * NT_JOIN_PARTS), 0, st,
                     (const float*)workspace, (int)blocks, (int32_t)cols, dweight, (float)scale, (float)beta);
  return hip_code(hipGetLastError());
}

}  // extern "C"
