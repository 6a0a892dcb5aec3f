// The product of microscaled matrices, out <- beta out + scale A B^T, hand-written for gfx950 (MI355X).
//
// The matrix cores multiply 4- and 8-bit codes as they are, 16 x 16 results from 128 columns at a time, with a scale byte for every 32 of them.
// A lane gives 32 elements of one row: in 4 bits a whole block, lane l block l / 16 of row l % 16; in 8 bits the elements 16 (l / 16) .. of the
// first and of the second 64.  The scale byte of lane l is block l / 16's either way.  Which columns take part in one instruction is free, as
// long as A and B agree, so a lane's blocks are chosen to lie side by side in memory.
//
// 8-bit products are added up in groups of 8 neighbours, each cut below 2^-13 of the group's largest (measured: 256 + 2^-6 is 256, and
// 3 2^-6 beside 256 counts as 2^-5; between groups nothing is lost down to 2^-27).  Sums of normal data are 2e-5 to 3e-5 of their usual size off by
// that.  For fp32 results with an 8-bit operand both operands are widened to bf16, scale included: every code is a bf16 number, and
// products of those are added in full.  16-bit results are left to the 8-bit instructions unless the caller asks for full sums: of 8 x 4 (8 x 8)
// bits 0.7 % (1.6 %) of bf16 results and 4 % (9 %) of fp16 ones then are the number beside the one that full sums round to, and their distance from the
// fp32 result, in 2-norm, is the same to 0.1 % (0.5 %); but one that cancels to a hundredth of the usual size is 3e-3 of itself off, 0.8 half steps of bf16
// and 6 of fp16.  Full sums of 8192 x 16384 x 4096 take 920 us for 502, of 1 x 16384 x 4096 9.6 for 8.8.
#include "mx.h"

#define NT_MM_CHUNK 512            // columns that a wave takes at a time: 16 blocks, four for a lane
#define NT_MM_CHUNK_BLOCKS 16
#define NT_MM_THIN_WAVES 4
// Up to 32 rows always, and up to 64 where 128 x 128 tiles are too few (64 x 2048 x 2048 11.6 -> 7.4 us; 64 x 16384 x 4096, 128 tiles, 19.7 -> 25.3).
#define NT_MM_THIN_ROWS 32
#define NT_MM_THIN_MORE_ROWS 64
#define NT_MM_THIN_TILES 96
#define NT_MM_THIN_MANY 512        // blocks from which a wave takes 32 columns and not 16 (24 x 50257 x 768 16.4 -> 13.5 us, 1 x 16384 x 4096 8.8 -> 8.2)
#define NT_MM_TILE_LD (1ll << 22)   // bytes from row to row that 32-bit offsets into a tile allow
#define NT_MM_MOST_TILES ((1ll << 23) - 1)   // of a result: a launch holds less than 2^32 threads
#define NT_MM_MOST_DOWN 65535                // groups of rows in a launch of k_mm_thin

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct Operand {
  const uint8_t *codes, *scales;
  int64_t rows, ld, scale_ld;
};
struct MatmulArgs {
  Operand a, b;
  int64_t blocks;      // of a row
  char* out;
  int64_t ld;
  float* parts;        // sums over parts of the columns, M x N each; NULL: out is written
  float scale, beta;
  int32_t dtype;
};

// ---------------------------------------------------------------------------------------------
// Results
// ---------------------------------------------------------------------------------------------
__device__ inline float read_as(int dtype, const char* p) {
  if (dtype == NT_F32) return *(const float*)p;
  const uint16_t h = *(const uint16_t*)p;
  return dtype == NT_BF16 ? __builtin_bit_cast(float, (uint32_t)h << 16) : (float)__builtin_bit_cast(_Float16, h);
}
// n <= 4 results of row m from column `col` on
__device__ inline void put4(const MatmulArgs& a, int64_t m, int64_t col, f32x4 x, int n) {
  typedef uint32_t u32x2_half __attribute__((ext_vector_type(2), aligned(2)));
  if (a.parts) {
    float* const to = a.parts + m * a.b.rows + col;
    if (n == 4) {
      *(u32x4_word*)to = __builtin_bit_cast(u32x4, x);
    } else {
      for (int i = 0; i < 3; ++i)
        if (i < n) to[i] = x[i];
    }
    return;
  }
  char* const to = a.out + (m * a.ld + col) * type_bytes(a.dtype);
  x *= a.scale;
  if (n == 4) {
    if (a.dtype == NT_F32) {
      if (a.beta != 0.f) {
        const f32x4 old = __builtin_bit_cast(f32x4, (u32x4) * (const u32x4_word*)to);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_fmaf(a.beta, old[i], x[i]);
      }
      *(u32x4_word*)to = __builtin_bit_cast(u32x4, x);
    } else {
      if (a.beta != 0.f) {
        const u32x2 old = *(const u32x2_half*)to;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint16_t h = (uint16_t)(old[i >> 1] >> (16 * (i & 1)));
          x[i] = __builtin_fmaf(a.beta, a.dtype == NT_BF16 ? __builtin_bit_cast(float, (uint32_t)h << 16) : (float)__builtin_bit_cast(_Float16, h), x[i]);
        }
      }
      *(u32x2_half*)to = u32x2{half_bits(a.dtype, x[0]) | half_bits(a.dtype, x[1]) << 16, half_bits(a.dtype, x[2]) | half_bits(a.dtype, x[3]) << 16};
    }
    return;
  }
  for (int i = 0; i < 3; ++i)
    if (i < n) {
      char* const p = to + i * type_bytes(a.dtype);
      float y = x[i];
      if (a.beta != 0.f) y = __builtin_fmaf(a.beta, read_as(a.dtype, p), y);
      if (a.dtype == NT_F32)
        *(float*)p = y;
      else
        *(uint16_t*)p = (uint16_t)half_bits(a.dtype, y);
    }
}

// The parts' sum, in order, four columns of a row to a thread.  Bound by memory (four parts of 768 x 2304 added to a result in fp32: 42 MB in 8.2 to 8.9 us).
__global__ __launch_bounds__(256) void k_mm_join(MatmulArgs a, int splits, uint32_t quads) {
  const int64_t n = a.a.rows * a.b.rows, all = a.a.rows * quads;
  const float* const parts = a.parts;
  a.parts = nullptr;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t m = all < 1ll << 32 ? (uint32_t)i / quads : i / quads, col = 4 * (i - m * quads), left = a.b.rows - col;
    const float* p = parts + m * a.b.rows + col;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s, p += n) {
      const Raw<NT_F32> r = left >= 4 ? Raw<NT_F32>{{*(const u32x4_word*)p, {}}} : load_part<NT_F32>(p, (int)left);
      x += __builtin_bit_cast(f32x4, r.w[0]);
    }
    put4(a, m, col, x, left < 4 ? (int)left : 4);
  }
}

// ---------------------------------------------------------------------------------------------
// Fragments
// ---------------------------------------------------------------------------------------------
// A lane's 32 elements for one instruction, and their product.
template <int F>
struct Frag {
  u32x4 w[F == NT_MX_E4M3 ? 2 : 1];
};
template <int F>
__device__ inline i32x8 registers(const Frag<F>& f) {
  const u32x4 lo = f.w[0], hi = F == NT_MX_E4M3 ? f.w[F == NT_MX_E4M3] : u32x4{0u, 0u, 0u, 0u};
  return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}
// eight elements as bf16, scale included
template <int F>
__device__ inline bf16x8 widened(const Frag<F>& f, int part, float by) {
  bf16x2 p[4];
  if (F == NT_MX_E2M1) {
    const uint32_t w = f.w[0][part];
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, 3);
  } else {
    const uint32_t lo = f.w[F == NT_MX_E4M3 ? part >> 1 : 0][2 * (part & 1)], hi = f.w[F == NT_MX_E4M3 ? part >> 1 : 0][2 * (part & 1) + 1];
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, true);
  }
  return bf16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}
// columns of B down, rows of A across: a lane then holds four neighbouring columns of one row of the result
template <int FA, int FB, int BYTE>
__device__ inline f32x4 multiply(const Frag<FB>& b, uint32_t sb, const Frag<FA>& a, uint32_t sa, f32x4 c) {
  constexpr int CODE_B = FB == NT_MX_E2M1 ? 4 : 0, CODE_A = FA == NT_MX_E2M1 ? 4 : 0;
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(registers(b), registers(a), c, CODE_B, CODE_A, BYTE, (int)sb, BYTE, (int)sa);
}

// Lane (r, g) has the scales of blocks 4 g .. 4 g + 3 of a row, and gets those of the blocks g, 4 + g, 8 + g and 12 + g, the row's at each of four steps:
// 4 x 4 bytes change places across the lanes that are 32 and 16 apart.
__device__ inline uint32_t by_step(uint32_t w, int g) {
  auto p = __builtin_amdgcn_permlane32_swap(w, w, false, false);      // of lanes 0 .. 31, and of lanes 32 .. 63
  w = __builtin_amdgcn_perm(p[1], p[0], g & 2 ? 0x07060302u : 0x05040100u);
  p = __builtin_amdgcn_permlane16_swap(w, w, false, false);           // of rows 0 and 2 of 16 lanes, and of 1 and 3
  return __builtin_amdgcn_perm(p[1], p[0], g & 1 ? 0x07030501u : 0x06020400u);
}

// ---------------------------------------------------------------------------------------------
// Few rows
// ---------------------------------------------------------------------------------------------
// A wave takes NT x 16 columns of the result and MT x 16 rows, straight from memory to registers, U x 128 columns of A and B at a time.  `along` of
// a block's four waves (and blockIdx.z) share those out, and are joined through LDS; the others have columns of their own.  Lanes that hold pieces
// of one row load 64 bytes of it side by side, and one word of scales each, for 512 columns, which then change places.  (Four blocks of a lane side by
// side need no change, but every lane loads from a cache line of its own: 24 x 50257 x 768 19.7 us.)  Bound by memory where there is one row (1 x 16384 x
// 4096 8.4 us, 4.3 TB/s), by the time of a wave, load to last product, where there are more.  Hence U = 2 for fewer than 2048 columns: 24 x 50257 x 768 13.4 ->
// 12.7, of 1536 21.7 -> 19.6 (8 x 50257 x 1024 8.4 -> 8.7).  Blocks side by side are on one die, where the lines that they share are written once: 12.7 -> 12.2,
// the single row 8.4 to 8.8 -> 8.2.
template <int F, bool WIDE, int U>
struct Chunk {
  Frag<F> f[U];
  uint32_t scales;
  int shift;        // of the scales: 16 where U is 2 and this is the upper half of what one word holds
  __device__ inline void load(const Operand& o, int64_t row, int64_t block0, int64_t blocks, bool whole) {
    const int g = (threadIdx.x & 63) / 16;
    const bool there = row < o.rows;
    const uint8_t* const codes = o.codes + row * o.ld;
    auto piece = [&](int64_t block, int half) {
      u32x4 x = {0u, 0u, 0u, 0u};
      if (there && (whole || block < blocks)) x = *(const u32x4*)(codes + block * code_bytes(F) + 16 * half);
      return x;
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t first = block0 + 4 * u;
      if (F == NT_MX_E2M1) {
        f[u].w[0] = piece(first + g, 0);
      } else if (WIDE) {
        f[u].w[0] = piece(first + g, 0);
        f[u].w[F == NT_MX_E4M3] = piece(first + g, 1);
      } else {   // elements 16 g .. of the instruction's first and second 64
        f[u].w[0] = piece(first + g / 2, g & 1);
        f[u].w[F == NT_MX_E4M3] = piece(first + 2 + g / 2, g & 1);
      }
    }
    uint32_t word = 0;
    const int64_t b0 = block0 / 16 * 16 + 4 * g;   // of all 512
    if (there) {
      const uint8_t* const s = o.scales + row * o.scale_ld;
      if (b0 + 4 <= blocks) {
        word = *(const u32_any*)(s + b0);
      } else {
        for (int u = 0; u < 3; ++u)
          if (b0 + u < blocks) word |= (uint32_t)s[b0 + u] << (8 * u);
      }
    }
    scales = word;
    shift = U == 4 ? 0 : (int)(block0 & 8) * 2;
  }
  // where the scales are needed: what the lane loaded is its neighbours'
  __device__ inline void settle() { scales = by_step(scales, (threadIdx.x & 63) / 16) >> shift; }
};

template <int FA, int FB, bool WIDE, int MT, int NT, int U>
__global__ __launch_bounds__(64 * NT_MM_THIN_WAVES) void k_mm_thin(MatmulArgs a, int along) {
  __shared__ f32x4 sums[NT_MM_THIN_WAVES][MT * NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, r = lane % 16, part = wave % along;
  const int64_t n0 = ((int64_t)by_die(blockIdx.x, gridDim.x) * (NT_MM_THIN_WAVES / along) + wave / along) * (16 * NT), m0 = (int64_t)blockIdx.y * (16 * MT);
  f32x4 acc[MT][NT];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t chunks = (a.blocks + 4 * U - 1) / (4 * U), step = (int64_t)gridDim.z * along;
  for (int64_t c = (int64_t)blockIdx.z * along + part; c < chunks; c += step) {
    const int64_t block0 = c * (4 * U);
    const bool whole = block0 + 4 * U <= a.blocks;
    Chunk<FB, WIDE, U> b[NT];
    Chunk<FA, WIDE, U> x[MT];
#pragma unroll
    for (int n = 0; n < NT; ++n) b[n].load(a.b, n0 + 16 * n + r, block0, a.blocks, whole);
#pragma unroll
    for (int t = 0; t < MT; ++t) x[t].load(a.a, m0 + 16 * t + r, block0, a.blocks, whole);
#pragma unroll
    for (int n = 0; n < NT; ++n) b[n].settle();
#pragma unroll
    for (int t = 0; t < MT; ++t) x[t].settle();
    if constexpr (!WIDE) {
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          acc[t][n] = multiply<FA, FB, 0>(b[n].f[0], b[n].scales, x[t].f[0], x[t].scales, acc[t][n]);
          acc[t][n] = multiply<FA, FB, 1>(b[n].f[1], b[n].scales, x[t].f[1], x[t].scales, acc[t][n]);
          if constexpr (U == 4) {
            acc[t][n] = multiply<FA, FB, 2>(b[n].f[2], b[n].scales, x[t].f[2], x[t].scales, acc[t][n]);
            acc[t][n] = multiply<FA, FB, 3>(b[n].f[3], b[n].scales, x[t].f[3], x[t].scales, acc[t][n]);
          }
        }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          bf16x8 wb[NT];
#pragma unroll
          for (int n = 0; n < NT; ++n) wb[n] = widened<FB>(b[n].f[u], p, grow((b[n].scales >> (8 * u)) & 255u));
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            const bf16x8 wa = widened<FA>(x[t].f[u], p, grow((x[t].scales >> (8 * u)) & 255u));
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[n], wa, acc[t][n], 0, 0, 0);
          }
        }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int n = 0; n < NT; ++n) sums[wave][t * NT + n][lane] = acc[t][n];
  __syncthreads();
  if (gridDim.z > 1) a.parts += (int64_t)blockIdx.z * a.a.rows * a.b.rows;
  for (int i = part; i < MT * NT; i += along) {   // the waves that share columns write them, a 16 x 16 piece each
    f32x4 y = sums[wave - part][i][lane];
    for (int w = 1; w < along; ++w) y += sums[wave - part + w][i][lane];
    const int64_t m = m0 + 16 * (i / NT) + r, col = n0 + 16 * (i % NT) + 4 * (lane / 16), left = a.b.rows - col;
    if (m < a.a.rows && left > 0) put4(a, m, col, y, left < 4 ? (int)left : 4);
  }
}

// ---------------------------------------------------------------------------------------------
// Tiles
// ---------------------------------------------------------------------------------------------
// A block takes BM x BN of the result.  Steps of 256 (4 bits both) or 128 columns of A and B go from memory to LDS without passing
// registers, into one half while the other is multiplied; a chunk's scales, 16 bytes a row, go through registers, where their
// bytes are transposed, so that lane (r, g) reads the four scales that it needs for the chunk's four instructions as one word.
// A row of LDS has 64 or 128 bytes without a gap (what goes there directly lies as the lanes do), so 16-byte pieces of neighbouring rows change places
// by the row's number: 16 lanes that read one piece of 16 rows then meet all banks.
// Below 256 tiles the columns are in parts, as many as 512 blocks (two to a CU) allow: 768 x 2304 x 16384 widened, 108 tiles, four parts 73.8 us, three
// 85, six 88, nine 84.  There the matrix cores (0.8 PF/s, a library's product in bf16 1.6) share the time with widening (20 %).
template <int FA, int FB>
constexpr int step_columns() {
  return FA == NT_MX_E2M1 && FB == NT_MX_E2M1 ? 256 : 128;
}
template <int F>
constexpr int row_bytes(int columns) {
  return F == NT_MX_E2M1 ? columns / 2 : columns;
}
template <int BYTES>   // of a row
__device__ inline int swapped(int row, int piece) {
  return piece ^ ((row >> 1) & (BYTES / 16 - 1));
}

// 16 bytes a lane from memory to consecutive bytes of LDS.  What lies beyond the descriptor's size reads as zeros.  The compiler does not know
// of these loads: whoever reads the LDS waits for them by landed().  Nor does it see that the descriptor is read here: a vector instruction (reading
// the first lane) that has just written one of its registers needs five wait states before, or an old value is used.
__device__ inline void to_lds(u32x4 from, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(offset), "s"(from), "s"(to) : "memory", "m0");
}
// all loads of this wave have arrived, all its LDS accesses are done, and every other wave of the block is here too
__device__ inline void landed() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

// A tile's rows of one operand, a step of columns at a time.  What moves, from row to row and from step to step, moves the descriptor, on the scalar
// unit: one offset a lane serves all loads.  (With an offset for each, spilled registers were read back between the loads, and each waited for the last.)
template <int F, int TILE, int COLUMNS, int WAVES>
struct Loader {
  static constexpr int BYTES = row_bytes<F>(COLUMNS), PIECES = BYTES / 16, ROWS = 64 / PIECES, TURNS = TILE / (ROWS * WAVES);
  static_assert(TURNS * ROWS * WAVES == TILE, "whole turns");
  uint64_t at;
  int32_t size, turn;          // turn: bytes from one of a wave's loads to the next; size: none left where it is not positive
  uint32_t wave;
  uint32_t offset, piece;      // of this lane; piece: bytes into the step
  __device__ inline void init(const Operand& o, int64_t row0, int64_t block0, int64_t blocks) {
    const int lane = threadIdx.x & 63;
    wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / 64));
    const int row = (int)wave * ROWS + lane / PIECES;
    const int64_t rows = o.rows - row0 < TILE ? o.rows - row0 : TILE;
    at = (uint64_t)(uintptr_t)(o.codes + row0 * o.ld + block0 * code_bytes(F));
    size = (int32_t)((rows - 1) * o.ld + (blocks - block0) * code_bytes(F));
    piece = (uint32_t)swapped<BYTES>(row, lane % PIECES) * 16;
    offset = (uint32_t)row * (uint32_t)o.ld + piece;
    turn = ROWS * WAVES * (int32_t)o.ld;
  }
  // One of the step's loads.  left: bytes of a row from this step on; none or fewer: zeros.
  __device__ inline void load(uint32_t to, int32_t left, int i) const {
    const uint32_t off = (int32_t)piece < left ? offset : 0x80000000u;   // behind the row's last block: beyond the descriptor's size too
    const uint64_t from = at + (uint64_t)(uint32_t)(i * turn);
    const int32_t here = size - i * turn;
    to_lds(u32x4{(uint32_t)from, (uint32_t)(from >> 32), (uint32_t)(here > 0 ? here : 0), 0x00020000u}, off, to + (uint32_t)(i * WAVES * 1024) + wave * 1024u);
  }
  __device__ inline void next() {
    at += BYTES;
    size -= BYTES;
  }
  __device__ inline void step(uint32_t to, int32_t left) {
#pragma unroll
    for (int i = 0; i < TURNS; ++i) load(to, left, i);
    next();
  }
};

// rows of 16 scale bytes to words by lane group
__device__ inline u32x4 by_group(const u32x4& w) {
  const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);   // 0 0' 1 1', 2 2' 3 3'
  const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  return u32x4{__builtin_amdgcn_perm(c, a, 0x05040100u), __builtin_amdgcn_perm(c, a, 0x07060302u), __builtin_amdgcn_perm(d, b, 0x05040100u),
               __builtin_amdgcn_perm(d, b, 0x07060302u)};
}
__device__ inline u32x4 load_scales(const Operand& o, int64_t row, int64_t block0, int64_t blocks) {
  u32x4 w = {0u, 0u, 0u, 0u};
  if (row >= o.rows) return w;
  const uint8_t* const p = o.scales + row * o.scale_ld + block0;
  if (block0 + 16 <= blocks) return *(const u32x4_byte*)p;
  for (int i = 0; i < (int)(blocks - block0); ++i) w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
  return w;
}

template <int FA, int FB, bool WIDE, int BM, int BN, int WM, int WN>
struct TileShape {
  static constexpr int THREADS = 64 * WM * WN, STEP = step_columns<FA, FB>(), STEPS = NT_MM_CHUNK / STEP;
  static constexpr int A_BYTES = BM * row_bytes<FA>(STEP), B_BYTES = BN * row_bytes<FB>(STEP), STAGE = A_BYTES + B_BYTES;
  static constexpr int SCALES = 2 * STAGE, LDS = SCALES + 2 * 16 * (BM + BN);
};

template <int FA, int FB, bool WIDE, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_mm_tile(MatmulArgs a, uint32_t down, uint32_t across, int32_t chunks_each) {
  typedef TileShape<FA, FB, WIDE, BM, BN, WM, WN> S;
  extern __shared__ __align__(1024) uint8_t lds[];
  constexpr int MT = BM / WM / 16, NT = BN / WN / 16, RA = row_bytes<FA>(S::STEP), RB = row_bytes<FB>(S::STEP), WAVES = WM * WN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, r = lane % 16, g = lane / 16;
  const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);

  int64_t m0, n0;
  tile_at(blockIdx.x, gridDim.x, down, across, m0, n0);
  m0 *= BM;
  n0 *= BN;
  const int64_t chunk0 = (int64_t)blockIdx.y * chunks_each, block0 = chunk0 * NT_MM_CHUNK_BLOCKS;
  const int64_t end = (chunk0 + chunks_each) * NT_MM_CHUNK_BLOCKS, blocks = end < a.blocks ? end : a.blocks;   // of this part of the columns
  const int steps = (int)((blocks - block0 + S::STEP / 32 - 1) / (S::STEP / 32));

  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
  Loader<FA, BM, S::STEP, WAVES> la;
  Loader<FB, BN, S::STEP, WAVES> lb;
  la.init(a.a, m0, block0, blocks);
  lb.init(a.b, n0, block0, blocks);
  auto load = [&](int step) {
    const int32_t left = (int32_t)(blocks - block0) - step * (S::STEP / 32);
    const uint32_t to = base + (uint32_t)(step & 1) * S::STAGE;
    la.step(to, left * code_bytes(FA));
    lb.step(to + S::A_BYTES, left * code_bytes(FB));
  };
  constexpr int SCALE_TURNS = (BM + BN + S::THREADS - 1) / S::THREADS;
  u32x4 scales[SCALE_TURNS];
  auto fetch = [&](int64_t block) {
#pragma unroll
    for (int i = 0; i < SCALE_TURNS; ++i) {
      const int row = i * S::THREADS + (int)threadIdx.x;
      if (row < BM + BN) scales[i] = row < BM ? load_scales(a.a, m0 + row, block, blocks) : load_scales(a.b, n0 + row - BM, block, blocks);
    }
  };
  auto keep = [&](int chunk) {
#pragma unroll
    for (int i = 0; i < SCALE_TURNS; ++i) {
      const int row = i * S::THREADS + (int)threadIdx.x;
      if (row < BM + BN) *(u32x4*)(lds + S::SCALES + (chunk & 1) * 16 * (BM + BN) + 16 * row) = by_group(scales[i]);
    }
  };

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  // where this lane's pieces are in a stage: rows 16 apart have their pieces in the same order
  constexpr int PARTS = S::STEP / 128;
  int at_a[PARTS][2], at_b[PARTS][2];
#pragma unroll
  for (int u = 0; u < PARTS; ++u)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int ia = FA == NT_MX_E2M1 ? 4 * u + g : WIDE ? 2 * g + h : 4 * h + g, ib = FB == NT_MX_E2M1 ? 4 * u + g : WIDE ? 2 * g + h : 4 * h + g;
      at_a[u][h] = (wm + r) * RA + swapped<RA>(r, ia) * 16;
      at_b[u][h] = S::A_BYTES + (wn + r) * RB + swapped<RB>(r, ib) * 16;
    }

  fetch(block0);
  load(0);
  keep(0);
  landed();

  uint32_t sa[MT], sb[NT];
  for (int at = 0; at < steps; ++at) {
    const int chunk = at / S::STEPS;
    const int64_t next = block0 + (int64_t)(chunk + 1) * NT_MM_CHUNK_BLOCKS;
    if (at % S::STEPS == 0) {
      const uint8_t* const ps = lds + S::SCALES + (chunk & 1) * 16 * (BM + BN) + 4 * g;
#pragma unroll
      for (int i = 0; i < MT; ++i) sa[i] = *(const uint32_t*)(ps + 16 * (wm + 16 * i + r));
#pragma unroll
      for (int j = 0; j < NT; ++j) sb[j] = *(const uint32_t*)(ps + 16 * (BM + wn + 16 * j + r));
      if (next < blocks) fetch(next);
    }
    load(at + 1);   // zeros behind the last one
    const uint8_t* const stage = lds + (at & 1) * S::STAGE;
#pragma unroll
    for (int u = 0; u < PARTS; ++u) {
      if (u) __builtin_amdgcn_sched_barrier(0);   // its fragments in the registers of the part before
      Frag<FA> fa[MT];
      Frag<FB> fb[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        fb[j].w[0] = *(const u32x4*)(stage + at_b[u][0] + 16 * j * RB);
        if (FB == NT_MX_E4M3) fb[j].w[FB == NT_MX_E4M3] = *(const u32x4*)(stage + at_b[u][1] + 16 * j * RB);
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        fa[i].w[0] = *(const u32x4*)(stage + at_a[u][0] + 16 * i * RA);
        if (FA == NT_MX_E4M3) fa[i].w[FA == NT_MX_E4M3] = *(const u32x4*)(stage + at_a[u][1] + 16 * i * RA);
      }
      if constexpr (!WIDE) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j)
            acc[i][j] = u == 0 ? multiply<FA, FB, 0>(fb[j], sb[j], fa[i], sa[i], acc[i][j]) : multiply<FA, FB, 1>(fb[j], sb[j], fa[i], sa[i], acc[i][j]);
      } else {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          bf16x8 x[MT];
#pragma unroll
          for (int i = 0; i < MT; ++i) x[i] = widened<FA>(fa[i], p, grow(sa[i] & 255u));
#pragma unroll
          for (int j = 0; j < NT; ++j) {
            const bf16x8 y = widened<FB>(fb[j], p, grow(sb[j] & 255u));
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, x[i], acc[i][j], 0, 0, 0);
          }
        }
      }
    }
    // the next step's scales come down to the lowest bytes
#pragma unroll
    for (int i = 0; i < MT; ++i) sa[i] >>= 8 * PARTS;
#pragma unroll
    for (int j = 0; j < NT; ++j) sb[j] >>= 8 * PARTS;
    if (at % S::STEPS == S::STEPS - 1 && next < blocks) keep(chunk + 1);
    landed();
  }

  if (gridDim.y > 1) a.parts += (int64_t)blockIdx.y * a.a.rows * a.b.rows;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = m0 + wm + 16 * i + r;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int64_t col = n0 + wn + 16 * j + 4 * g, left = a.b.rows - col;
      if (m < a.a.rows && left > 0) put4(a, m, col, acc[i][j], left < 4 ? (int)left : 4);
    }
  }
}

// The same for many tiles: 256 x 256 by eight waves, one block to a CU, steps of 128 columns in a ring of two to four stages, all but one of which are
// on their way.  Scales, 16 bytes a row for four steps, go to LDS directly too, which asks for rows of scales at multiples of 16 bytes.
// From 192 tiles on, three quarters of the CUs: 8192^3 in 4 bits 311 us (3.5 PF/s), by tiles of 128 401; 8192 x 16384 x 4096 in 8 x 4 bits 499 and 643; 8192^3 in
// 8 bits 492 and 670 (cards differ by 5 %).  Bound by the way from cache to LDS and by its place behind the products: in a run of 296 us in 4 bits the loads alone
// took 184, the products alone 187, and they overlapped by a third.
template <int FA, int FB>
struct LargeShape {
  static constexpr int TILE = 256, WM = 2, WN = 4, WAVES = WM * WN, THREADS = 64 * WAVES, STEP = 128, STEPS = NT_MM_CHUNK / STEP;
  static constexpr int RA = row_bytes<FA>(STEP), RB = row_bytes<FB>(STEP), A_BYTES = TILE * RA, STAGE = TILE * (RA + RB);
  static constexpr int SCALES = 2 * TILE * 16;   // of a chunk; two of them
  static constexpr int FIT = (163840 - 2 * SCALES) / STAGE, STAGES = FIT > 4 ? 4 : FIT, LDS = STAGES * STAGE + 2 * SCALES;
};
__device__ inline uint64_t scalar(uint64_t x) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
}
// waits until at most N of this wave's loads are on their way, and for the block
template <int N>
__device__ inline void landed_but() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
}

template <int FA, int FB>
__global__ __launch_bounds__(512) void k_mm_large(MatmulArgs a, uint32_t down, uint32_t across) {
  typedef LargeShape<FA, FB> S;
  extern __shared__ __align__(1024) uint8_t lds[];
  constexpr int MT = S::TILE / S::WM / 16, NT = S::TILE / S::WN / 16, RA = S::RA, RB = S::RB, AHEAD = S::STAGES - 1;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, r = lane % 16, g = lane / 16;
  const int wm = wave / S::WN * (S::TILE / S::WM), wn = wave % S::WN * (S::TILE / S::WN);
  int64_t m0, n0;
  tile_at(blockIdx.x, gridDim.x, down, across, m0, n0);
  m0 *= S::TILE;
  n0 *= S::TILE;
  const int32_t blocks = (int32_t)a.blocks, steps = (blocks + 3) / 4;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;

  typedef Loader<FA, S::TILE, S::STEP, S::WAVES> LoadA;
  typedef Loader<FB, S::TILE, S::STEP, S::WAVES> LoadB;
  constexpr int LOADS = LoadA::TURNS + LoadB::TURNS;
  LoadA la;
  LoadB lb;
  la.init(a.a, m0, 0, blocks);
  lb.init(a.b, n0, 0, blocks);
  uint32_t slot = 0;   // where the next step goes
  int32_t left = blocks;
  auto done = [&] {
    la.next();
    lb.next();
    left -= 4;
    slot = slot + S::STAGE == S::STAGES * S::STAGE ? 0 : slot + S::STAGE;
  };
  auto load = [&] {
#pragma unroll
    for (int i = 0; i < LoadA::TURNS; ++i) la.load(base + slot, left * code_bytes(FA), i);
#pragma unroll
    for (int i = 0; i < LoadB::TURNS; ++i) lb.load(base + slot + S::A_BYTES, left * code_bytes(FB), i);
    done();
  };
  // Scales of a chunk: waves 0 to 3 those of A, 64 rows each, the others B's.  Bytes behind the row's last block may be there too and are not looked at.
  const uint32_t uwave = (uint32_t)__builtin_amdgcn_readfirstlane(wave);
  const bool of_a = uwave < 4;
  const Operand& so = of_a ? a.a : a.b;
  const int64_t srow0 = of_a ? m0 : n0, srows = so.rows - srow0 < S::TILE ? so.rows - srow0 : S::TILE;
  uint64_t scales_at = (uint64_t)(uintptr_t)(so.scales + srow0 * so.scale_ld);
  int32_t scales_left = (int32_t)((srows - 1) * so.scale_ld + (blocks + 15) / 16 * 16), chunk_slot = 0;
  const uint32_t scale_offset = ((uwave & 3) * 64 + lane) * (uint32_t)so.scale_ld;
  auto load_scales = [&] {
    const uint64_t from = scalar(scales_at);
    const uint32_t size = (uint32_t)__builtin_amdgcn_readfirstlane(scales_left > 0 ? scales_left : 0);
    to_lds(u32x4{(uint32_t)from, (uint32_t)(from >> 32), size, 0x00020000u}, scale_offset, base + S::STAGES * S::STAGE + chunk_slot + uwave * 1024u);
    scales_at += 16;
    scales_left -= 16;
    chunk_slot ^= S::SCALES;
  };

  // where this lane's pieces are in a stage, and its words of scales: rows 16 apart are alike
  int at_a[2], at_b[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    at_a[h] = (wm + r) * RA + swapped<RA>(r, FA == NT_MX_E2M1 ? g : 4 * h + g) * 16;
    at_b[h] = S::A_BYTES + (wn + r) * RB + swapped<RB>(r, FB == NT_MX_E2M1 ? g : 4 * h + g) * 16;
  }
  const uint8_t* const scales_a = lds + S::STAGES * S::STAGE + 16 * (wm + r) + 4 * g;
  const uint8_t* const scales_b = lds + S::STAGES * S::STAGE + 16 * (S::TILE + wn + r) + 4 * g;

  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  load_scales();
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) load();
  landed_but<(AHEAD - 1) * LOADS>();

  uint32_t here = 0, sa[MT], sb[NT];
  for (int at = 0; at < steps; ++at) {
    const uint8_t* const stage = lds + here;
    if (at % S::STEPS == 0) {
      // bytes behind the last block may be any, and NaN
      const int32_t there = blocks - 4 * at - 4 * g;
      const uint32_t mask = there >= 4 ? 0xffffffffu : there > 0 ? (1u << (8 * there)) - 1 : 0u;
      const int chunk = (at / S::STEPS & 1) * S::SCALES;
#pragma unroll
      for (int j = 0; j < NT; ++j) sb[j] = by_step(*(const uint32_t*)(scales_b + chunk + 256 * j) & mask, g);
#pragma unroll
      for (int i = 0; i < MT; ++i) sa[i] = by_step(*(const uint32_t*)(scales_a + chunk + 256 * i) & mask, g);
      load_scales();   // of the next chunk: beyond the descriptor behind the last one
    }
    // The step's loads go one by one between the products: all at once they keep the wave from reading and multiplying until they are
    // accepted.  Not where the very next step needs them (8 bits both).
    if (AHEAD == 1) load();
    Frag<FA> fa[MT];
    Frag<FB> fb[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      fb[j].w[0] = *(const u32x4*)(stage + at_b[0] + 16 * j * RB);
      if (FB == NT_MX_E4M3) fb[j].w[FB == NT_MX_E4M3] = *(const u32x4*)(stage + at_b[1] + 16 * j * RB);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      fa[i].w[0] = *(const u32x4*)(stage + at_a[0] + 16 * i * RA);
      if (FA == NT_MX_E4M3) fa[i].w[FA == NT_MX_E4M3] = *(const u32x4*)(stage + at_a[1] + 16 * i * RA);
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = multiply<FA, FB, 0>(fb[j], sb[j], fa[i], sa[i], acc[i][j]);
      if (AHEAD > 1) {
        __builtin_amdgcn_sched_barrier(0);
        if (i < LoadA::TURNS)
          la.load(base + slot, left * code_bytes(FA), i);
        else if (i < LOADS)
          lb.load(base + slot + S::A_BYTES, left * code_bytes(FB), i - LoadA::TURNS);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (AHEAD > 1) done();
#pragma unroll
    for (int i = 0; i < MT; ++i) sa[i] >>= 8;
#pragma unroll
    for (int j = 0; j < NT; ++j) sb[j] >>= 8;
    here = here + S::STAGE == S::STAGES * S::STAGE ? 0 : here + S::STAGE;
    landed_but<(AHEAD - 1) * LOADS>();
  }
  landed_but<0>();   // what was asked for behind the last step has gone to LDS too

#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t m = m0 + wm + 16 * i + r;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int64_t col = n0 + wn + 16 * j + 4 * g, over = a.b.rows - col;
      if (m < a.a.rows && over > 0) put4(a, m, col, acc[i][j], over < 4 ? (int)over : 4);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
enum { THIN, MIDDLE, LARGE };
struct MatmulPlan {
  bool wide;
  int kind, rows, cols, along, steps;   // of THIN: 16-row and 16-column groups of a wave, the block's waves that share columns, and 128s at a time
  uint32_t down, across; // tiles
  int splits, chunks;    // parts of the columns, and chunks of 512 in each
};
// rows of scales at multiples of 16 bytes, within the reach of 32-bit offsets
bool aligned16(const nt_mx& m) { return (((uintptr_t)m.scales | (uintptr_t)m.scale_ld) & 15) == 0 && m.scale_ld <= NT_MM_TILE_LD; }
// full: sums in full for 16-bit results too.  The workspace's size does not know of it: what it changes, large tiles, is never in parts either way.
MatmulPlan plan_of(int64_t M, int64_t N, int64_t K, int fa, int fb, int dtype, int64_t ld, bool aligned, bool full) {
  MatmulPlan p;
  p.wide = (dtype == NT_F32 || full) && (fa == NT_MX_E4M3 || fb == NT_MX_E4M3);
  const int64_t chunks = ceil_div(K, NT_MM_CHUNK);
  p.rows = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  p.steps = chunks < 4 ? 2 : 4;
  const int64_t pieces = ceil_div(K, 128 * p.steps);
  p.along = pieces > 2 ? 4 : pieces == 2 ? 2 : 1;
  p.cols = 1;
  int64_t z = 1;
  if (M <= NT_MM_THIN_ROWS || (M <= NT_MM_THIN_MORE_ROWS && ceil_div(N, 128) < NT_MM_THIN_TILES) || ld > NT_MM_TILE_LD) {
    p.kind = THIN;
    const int beside = NT_MM_THIN_WAVES / p.along;
    p.down = (uint32_t)ceil_div(M, 16 * p.rows);
    if (ceil_div(N, 32 * beside) * p.down >= NT_MM_THIN_MANY) p.cols = 2;
    p.across = (uint32_t)ceil_div(N, 16 * p.cols * beside);
    const int64_t tiles = (int64_t)p.across * p.down, turns = ceil_div(pieces, p.along);
    if (tiles < 256 && ld <= NT_MM_TILE_LD) z = ceil_div(512, tiles);   // the workspace's size does not know ld, and need not
    if (z > turns) z = turns;
    p.chunks = 0;
  } else {
    p.kind = aligned && !p.wide && ceil_div(M, 256) * ceil_div(N, 256) >= 192 ? LARGE : MIDDLE;
    const int tile = p.kind == LARGE ? 256 : 128;
    p.down = (uint32_t)ceil_div(M, tile);
    p.across = (uint32_t)ceil_div(N, tile);
    const int64_t tiles = (int64_t)p.across * p.down;
    if (p.kind == MIDDLE && tiles < 256) z = 512 / tiles;
    if (z > chunks / 2) z = chunks / 2;
    if (z < 1) z = 1;
    p.chunks = (int)ceil_div(chunks, z);
    z = ceil_div(chunks, p.chunks);
  }
  p.splits = (int)z;
  return p;
}
template <class F>
int with_format(int format, F f) {
  return format == NT_MX_E2M1 ? f(std::integral_constant<int, NT_MX_E2M1>()) : f(std::integral_constant<int, NT_MX_E4M3>());
}
// beta out where there is nothing to multiply
__global__ __launch_bounds__(256) void k_mm_empty(MatmulArgs a) {
  const int64_t n = a.a.rows * a.b.rows;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / a.b.rows;
    put4(a, m, i - m * a.b.rows, f32x4{0.f, 0.f, 0.f, 0.f}, 1);
  }
}
uint32_t grid_of(int64_t n) {
  const int64_t blocks = ceil_div(n, 256);
  return (uint32_t)(blocks < 1 << 16 ? blocks : 1 << 16);
}

int matmul(const nt_mx* a, const nt_mx* b, double scale, double beta, void* out, nt_dtype dtype, int64_t ld, void* workspace, size_t workspace_bytes,
           bool full, void* hip_stream) {
  if (!a || !b) return NT_ERR_BAD_ARG;
  int rc = check_mx(*a);
  if (rc == NT_OK) rc = check_mx(*b);
  if (rc == NT_OK) rc = check_matrix(out, dtype, a->rows, b->rows, ld);
  if (rc != NT_OK) return rc;
  if (a->cols != b->cols || !finite_in_fp32(scale) || !finite_in_fp32(beta)) return NT_ERR_BAD_ARG;
  const int64_t M = a->rows, N = b->rows, K = a->cols;
  if (M == 0 || N == 0) return NT_OK;
  if (K > 1 << 22 || M > (1ll << 31) - 1 || N > 1 << 28) return NT_ERR_TOO_LARGE;
  hipStream_t st = (hipStream_t)hip_stream;
  MatmulArgs args = {{(const uint8_t*)a->codes, (const uint8_t*)a->scales, M, a->ld, a->scale_ld},
                     {(const uint8_t*)b->codes, (const uint8_t*)b->scales, N, b->ld, b->scale_ld},
                     blocks_of(K), (char*)out, ld, nullptr, (float)scale, (float)beta, dtype};
  if (K == 0) {
    hipLaunchKernelGGL(k_mm_empty, dim3(grid_of(M * N)), dim3(256), 0, st, args);
    return hip_code(hipGetLastError());
  }
  // a single row's ld means nothing, and may be anything
  if (M == 1) args.a.ld = 0;
  if (N == 1) args.b.ld = 0;
  const MatmulPlan p = plan_of(M, N, K, a->format, b->format, dtype, args.a.ld > args.b.ld ? args.a.ld : args.b.ld, aligned16(*a) && aligned16(*b), full);
  if (p.kind == THIN ? p.down > NT_MM_MOST_DOWN : (int64_t)p.down * p.across > NT_MM_MOST_TILES) return NT_ERR_TOO_LARGE;
  if (p.splits > 1) {
    if (!workspace || workspace_bytes < (size_t)p.splits * (size_t)M * (size_t)N * sizeof(float)) return NT_ERR_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)workspace & 15) return NT_ERR_BAD_ARG;
    args.parts = (float*)workspace;
  }
  rc = with_format(a->format, [&](auto fa) {
    return with_format(b->format, [&](auto fb) {
      constexpr int A = decltype(fa)::value, B = decltype(fb)::value;
      constexpr bool W = A == NT_MX_E4M3 || B == NT_MX_E4M3;
      auto thin = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(p.across, p.down, (uint32_t)p.splits), dim3(64 * NT_MM_THIN_WAVES), 0, st, args, p.along);
        return hip_code(hipGetLastError());
      };
      auto tile = [&](auto kernel, int threads, int lds) {
        hipLaunchKernelGGL(kernel, dim3(p.down * p.across, (uint32_t)p.splits), dim3(threads), lds, st, args, p.down, p.across, p.chunks);
        return hip_code(hipGetLastError());
      };
      if (p.kind == THIN) {
        auto columns = [&](auto wide, auto rows) {
          constexpr int MT = decltype(rows)::value;
          constexpr bool V = decltype(wide)::value;
          return p.cols == 1 ? (p.steps == 2 ? thin(k_mm_thin<A, B, V, MT, 1, 2>) : thin(k_mm_thin<A, B, V, MT, 1, 4>))
                             : (p.steps == 2 ? thin(k_mm_thin<A, B, V, MT, 2, 2>) : thin(k_mm_thin<A, B, V, MT, 2, 4>));
        };
        auto rows = [&](auto wide) {
          return p.rows == 1 ? columns(wide, std::integral_constant<int, 1>()) : p.rows == 2 ? columns(wide, std::integral_constant<int, 2>())
                                                                                           : columns(wide, std::integral_constant<int, 4>());
        };
        return p.wide ? rows(std::integral_constant<bool, W>()) : rows(std::false_type());
      }
      if (p.kind == LARGE) {
        hipLaunchKernelGGL((k_mm_large<A, B>), dim3(p.down * p.across), dim3(512), (LargeShape<A, B>::LDS), st, args, p.down, p.across);
        return hip_code(hipGetLastError());
      }
      if (p.wide) return tile(k_mm_tile<A, B, W, 128, 128, 2, 2>, 256, TileShape<A, B, W, 128, 128, 2, 2>::LDS);
      return tile(k_mm_tile<A, B, false, 128, 128, 2, 2>, 256, TileShape<A, B, false, 128, 128, 2, 2>::LDS);
    });
  });
  if (rc != NT_OK || p.splits == 1) return rc;
  const int64_t quads = ceil_div(N, 4);
  hipLaunchKernelGGL(k_mm_join, dim3(grid_of(M * quads)), dim3(256), 0, st, args, p.splits, (uint32_t)quads);
  return hip_code(hipGetLastError());
}

}  // namespace

extern "C" {

size_t normtest_mx_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, nt_mx_format a, nt_mx_format b, nt_dtype dtype) {
  if (M <= 0 || N <= 0 || K <= 0) return 0;
  const MatmulPlan p = plan_of(M, N, K, a, b, dtype, 0, true, false);
  return p.splits > 1 ? (size_t)p.splits * (size_t)M * (size_t)N * sizeof(float) : 0;
}

int normtest_mx_matmul(const nt_mx* a, const nt_mx* b, double scale, double beta, void* out, nt_dtype dtype, int64_t ld, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
  return matmul(a, b, scale, beta, out, dtype, ld, workspace, workspace_bytes, false, hip_stream);
}
int normtest_mx_matmul_full(const nt_mx* a, const nt_mx* b, double scale, double beta, void* out, nt_dtype dtype, int64_t ld, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
  return matmul(a, b, scale, beta, out, dtype, ld, workspace, workspace_bytes, true, hip_stream);
}

}  // extern "C"
