// The product of microscaled matrices, out <- beta out + scale A B^T, hand-written for gfx950 (MI355X).
//
// The matrix cores multiply 4- and 8-bit codes as they are, 16 x 16 results from 128 columns at a time, with a scale byte for every 32 of them.
// A lane gives 32 elements of one row: in 4 bits a whole block, lane l block l / 16 of row l % 16; in 8 bits the elements 16 (l / 16) .. of the
// first and of the second 64.  The scale byte of lane l is block l / 16's either way.  Which columns take part in one instruction is free, as
// long as A and B agree, so a lane's blocks are chosen to lie side by side in memory.
//
// 8-bit products are added up in groups of 8 neighbours, each cut below 2^-13 of the group's largest (measured: 256 + 2^-6 is 256, and
// 3 2^-6 beside 256 counts as 2^-5; between groups nothing is lost down to 2^-27).  Results of normal data are 2e-5 to 3e-5 off by that, which no 16-bit
// result shows, but an fp32 one does.  For fp32 results with an 8-bit operand both operands are widened to bf16, scale included: every code
// is a bf16 number, and products of those are added in full.
#include "mx.h"

#define NT_MM_CHUNK 512            // columns that a wave takes at a time: 16 blocks, four for a lane
#define NT_MM_CHUNK_BLOCKS 16
#define NT_MM_THIN_WAVES 4

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
  if (a.parts) {
    float* const to = a.parts + m * a.b.rows + col;
    for (int i = 0; i < 4; ++i)
      if (i < n) to[i] = x[i];
    return;
  }
  char* const to = a.out + (m * a.ld + col) * type_bytes(a.dtype);
  for (int i = 0; i < 4; ++i)
    if (i < n) {
      char* const p = to + i * type_bytes(a.dtype);
      float y = x[i] * a.scale;
      if (a.beta != 0.f) y = __builtin_fmaf(a.beta, read_as(a.dtype, p), y);
      if (a.dtype == NT_F32)
        *(float*)p = y;
      else
        *(uint16_t*)p = (uint16_t)half_bits(a.dtype, y);
    }
}

__global__ __launch_bounds__(256) void k_mm_join(MatmulArgs a, int splits) {
  const int64_t n = a.a.rows * a.b.rows;
  const float* const parts = a.parts;
  a.parts = nullptr;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s) x[0] += parts[s * n + i];
    const int64_t m = i / a.b.rows;
    put4(a, m, i - m * a.b.rows, x, 1);
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

// ---------------------------------------------------------------------------------------------
// Few rows
// ---------------------------------------------------------------------------------------------
// A wave takes 16 columns of the result and MT x 16 rows, straight from memory to registers; the waves of a block (and blockIdx.z) take every
// 4th (4 gridDim.z-th) chunk of 512 columns of A and B, and are joined through LDS.  Lane (r, g) has of a chunk the blocks 4 g .. 4 g + 3 of row r, 64
// consecutive bytes in 4 bits, and one word of scales.
template <int F, bool WIDE>
struct Chunk {
  Frag<F> f[4];
  uint32_t scales;
  __device__ inline void load(const Operand& o, int64_t row, int64_t block0, int64_t blocks, bool whole) {
    const int g = (threadIdx.x & 63) / 16;
    const bool there = row < o.rows;
    const uint8_t* const codes = o.codes + row * o.ld;
    const int64_t b0 = block0 + 4 * g;
    auto piece = [&](int64_t block, int half) {
      u32x4 x = {0u, 0u, 0u, 0u};
      if (there && (whole || block < blocks)) x = *(const u32x4*)(codes + block * code_bytes(F) + 16 * half);
      return x;
    };
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (F == NT_MX_E2M1) {
        f[u].w[0] = piece(b0 + u, 0);
      } else if (WIDE) {
        f[u].w[0] = piece(b0 + u, 0);
        f[u].w[F == NT_MX_E4M3] = piece(b0 + u, 1);
      } else {   // elements 16 g .. of the instruction's first and second 64
        f[u].w[0] = piece(block0 + 4 * (g / 2) + u, g & 1);
        f[u].w[F == NT_MX_E4M3] = piece(block0 + 4 * (2 + g / 2) + u, g & 1);
      }
    }
    scales = 0;
    if (there) {
      const uint8_t* const s = o.scales + row * o.scale_ld;
      if (whole || b0 + 4 <= blocks) {
        scales = *(const u32_any*)(s + b0);
      } else {
        for (int u = 0; u < 3; ++u)
          if (b0 + u < blocks) scales |= (uint32_t)s[b0 + u] << (8 * u);
      }
    }
  }
};

template <int FA, int FB, bool WIDE, int MT>
__global__ __launch_bounds__(64 * NT_MM_THIN_WAVES) void k_mm_thin(MatmulArgs a) {
  __shared__ f32x4 sums[NT_MM_THIN_WAVES][MT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, r = lane % 16;
  const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (16 * MT);
  f32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t chunks = (a.blocks + NT_MM_CHUNK_BLOCKS - 1) / NT_MM_CHUNK_BLOCKS;
  for (int64_t c = (int64_t)blockIdx.z * NT_MM_THIN_WAVES + wave; c < chunks; c += (int64_t)gridDim.z * NT_MM_THIN_WAVES) {
    const int64_t block0 = c * NT_MM_CHUNK_BLOCKS;
    const bool whole = block0 + NT_MM_CHUNK_BLOCKS <= a.blocks;
    Chunk<FB, WIDE> b;
    Chunk<FA, WIDE> x[MT];
    b.load(a.b, n0 + r, block0, a.blocks, whole);
#pragma unroll
    for (int t = 0; t < MT; ++t) x[t].load(a.a, m0 + 16 * t + r, block0, a.blocks, whole);
    if (!WIDE) {
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        acc[t] = multiply<FA, FB, 0>(b.f[0], b.scales, x[t].f[0], x[t].scales, acc[t]);
        acc[t] = multiply<FA, FB, 1>(b.f[1], b.scales, x[t].f[1], x[t].scales, acc[t]);
        acc[t] = multiply<FA, FB, 2>(b.f[2], b.scales, x[t].f[2], x[t].scales, acc[t]);
        acc[t] = multiply<FA, FB, 3>(b.f[3], b.scales, x[t].f[3], x[t].scales, acc[t]);
      }
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float sb = grow((b.scales >> (8 * u)) & 255u);
        float sa[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) sa[t] = grow((x[t].scales >> (8 * u)) & 255u);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const bf16x8 wb = widened<FB>(b.f[u], p, sb);
#pragma unroll
          for (int t = 0; t < MT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb, widened<FA>(x[t].f[u], p, sa[t]), acc[t], 0, 0, 0);
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) sums[wave][t][lane] = acc[t];
  __syncthreads();
  if (gridDim.z > 1) a.parts += (int64_t)blockIdx.z * a.a.rows * a.b.rows;
  for (int t = wave; t < MT; t += NT_MM_THIN_WAVES) {
    f32x4 x = sums[0][t][lane];
#pragma unroll
    for (int w = 1; w < NT_MM_THIN_WAVES; ++w) x += sums[w][t][lane];
    const int64_t m = m0 + 16 * t + r, col = n0 + 4 * (lane / 16), left = a.b.rows - col;
    if (m < a.a.rows && left > 0) put4(a, m, col, x, left < 4 ? (int)left : 4);
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
struct MatmulPlan {
  bool wide;
  int rows;      // 16-row groups of a wave
  int splits;
  dim3 grid;
};
MatmulPlan plan_of(int64_t M, int64_t N, int64_t K, int fa, int fb, int dtype) {
  MatmulPlan p;
  p.wide = dtype == NT_F32 && (fa == NT_MX_E4M3 || fb == NT_MX_E4M3);
  p.rows = M <= 16 ? 1 : 2;
  const int64_t across = ceil_div(N, 16), down = ceil_div(M, 16 * p.rows), turns = ceil_div(ceil_div(K, NT_MM_CHUNK), NT_MM_THIN_WAVES);
  int64_t z = 1;
  if (across * down < 256) z = ceil_div(512, across * down);
  if (z > turns) z = turns;
  p.splits = z < 1 ? 1 : (int)z;
  p.grid = dim3((uint32_t)across, (uint32_t)down, (uint32_t)p.splits);
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

}  // namespace

extern "C" {

size_t normtest_mx_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K, nt_mx_format a, nt_mx_format b, nt_dtype dtype) {
  if (M <= 0 || N <= 0 || K <= 0) return 0;
  const MatmulPlan p = plan_of(M, N, K, a, b, dtype);
  return p.splits > 1 ? (size_t)p.splits * (size_t)M * (size_t)N * sizeof(float) : 0;
}

int normtest_mx_matmul(const nt_mx* a, const nt_mx* b, double scale, double beta, void* out, nt_dtype dtype, int64_t ld, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
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
  const MatmulPlan p = plan_of(M, N, K, a->format, b->format, dtype);
  if (p.splits > 1) {
    if (!workspace || workspace_bytes < normtest_mx_matmul_workspace_bytes(M, N, K, (nt_mx_format)a->format, (nt_mx_format)b->format, dtype))
      return NT_ERR_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)workspace & 15) return NT_ERR_BAD_ARG;
    args.parts = (float*)workspace;
  }
  rc = with_format(a->format, [&](auto fa) {
    return with_format(b->format, [&](auto fb) {
      auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, p.grid, dim3(64 * NT_MM_THIN_WAVES), 0, st, args);
        return hip_code(hipGetLastError());
      };
      constexpr int A = decltype(fa)::value, B = decltype(fb)::value;
      constexpr bool W = A == NT_MX_E4M3 || B == NT_MX_E4M3;
      if (p.wide) return p.rows == 1 ? launch(k_mm_thin<A, B, W, 1>) : launch(k_mm_thin<A, B, W, 2>);
      return p.rows == 1 ? launch(k_mm_thin<A, B, false, 1>) : launch(k_mm_thin<A, B, false, 2>);
    });
  });
  if (rc != NT_OK || p.splits == 1) return rc;
  hipLaunchKernelGGL(k_mm_join, dim3(grid_of(M * N)), dim3(256), 0, st, args, p.splits);
  return hip_code(hipGetLastError());
}

}  // extern "C"
