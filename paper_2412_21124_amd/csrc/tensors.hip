// Norms, clipping, accumulation and AdamW over lists of tensors, hand-written for gfx950 (MI355X).
//
// A list is cut into items, pieces of one tensor each, by a plan that the host makes once (normtest_plan_make): for the calls that
// write, items of NT_ITEM elements, four for each thread of a block; for the norm alone, which only reads, longer ones.  A block
// takes one item: which tensor it belongs to and where it begins is one 16-byte record, the tensor's address a second one.
// All of it is bound by memory (2 operations a byte), so nothing here is a matrix product.
//
// Norms.  x^2 is formed and summed in fp64, so no finite value overflows and no rounding of the sum is seen; the largest
// magnitude is the largest |x| by its bits as an integer, where a NaN is larger than infinity and so survives.  A block leaves
// one partial; the blocks of a slab of items count themselves, the last one adds the slab's partials up, and the last slab of a group
// the group's slabs, and writes its record: one launch, no floating-point atomics, sums in an order that the plan alone fixes.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstring>
#include <initializer_list>
#include <new>

#include "normtest.h"

#define NT_ITEM 4096            // elements of an item: four per thread of a block of the kernels that write
#define NT_THREADS 1024         // threads of those
#define NT_NORM_THREADS 256     // threads of a block of the norm's kernel
#define NT_LONG_ITEM 32768      // elements of its items in a long list
#define NT_LONG_LIST (1ll << 23)   // elements from which a list is long
#define NT_MOST_BLOCKS (1u << 20)  // blocks of one launch
#define NT_PLAN_MAGIC 0x4e54504cu
#define NT_COUNTER_WORDS 16     // a counter has 64 bytes of its own, so that counting blocks of different slabs do not meet

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
// one access per lane whatever the alignment: gfx950 serves global loads and stores of 8 and 16 bytes from any element's address
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(4)));

#define NT_GLOBAL __attribute__((address_space(1)))
#define NT_CONST __attribute__((address_space(4)))   // written before the launch and not during it: scalar loads serve
template <class T>
__device__ inline const T NT_CONST* constant(const T* p) {
  return (const T NT_CONST*)(uintptr_t)p;
}

// ---------------------------------------------------------------------------------------------
// The plan's image
// ---------------------------------------------------------------------------------------------
// An item: elements idx * size .. of a tensor with one row, `count` of them; of a tensor with rows (NT_ROWS set in count) the count
// rows from row idx * rows_per_item on, or, where a row is longer than an item, part idx % per_row of row idx / per_row.
// count 0: a group without elements, whose record somebody has to write.
#define NT_ROWS 0x80000000u
struct Item {
  uint32_t tensor, idx, slab, count;
};
__device__ inline Item item_at(const Item* items, uint32_t i) {
  return __builtin_bit_cast(Item, ((const u32x4 NT_CONST*)(uintptr_t)items)[i]);
}
struct Slab {
  uint32_t first, n, group, pad;   // items first .. first + n - 1
};
struct Group {
  uint32_t first, n;               // slabs
  int64_t elements;
};
struct Shape {
  int64_t rows, cols;
  uint32_t per_row[2], rows_per_item[2];   // at both item sizes; per_row 0: whole rows
};

// One way of cutting a list: items of one size, and what adds up their partials.
struct Cut {
  const Item* items;
  const Slab* slabs;
  const Group* groups;
  uint32_t* counters;   // of the slabs, then of the groups; zero before and after every launch
  double* partials;     // one per item
  double* sums;         // one per slab
  uint32_t nslabs;
};
struct Layout {
  size_t shapes, items[2], slabs[2], groups[2], counters[2], upload, partials[2], sums[2], bytes;
};
Layout layout_of(const nt_plan& p) {
  Layout l;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 63) / 64 * 64;
    return here;
  };
  l.shapes = take(sizeof(Shape) * (size_t)p.tensors);
  for (int k = 0; k < 2; ++k) {
    l.items[k] = take(sizeof(Item) * (size_t)p.items[k]);
    l.slabs[k] = take(sizeof(Slab) * (size_t)p.slabs[k]);
    l.groups[k] = take(p.items[k] ? sizeof(Group) * (size_t)p.groups : 0);
    l.counters[k] = take(p.items[k] ? 4 * NT_COUNTER_WORDS * ((size_t)p.slabs[k] + p.groups) : 0);
  }
  l.upload = at;
  for (int k = 0; k < 2; ++k) {
    l.partials[k] = take(sizeof(double) * (size_t)p.items[k]);
    l.sums[k] = take(sizeof(double) * (size_t)p.slabs[k]);
  }
  l.bytes = at;
  return l;
}

// ---------------------------------------------------------------------------------------------
// Four elements of a lane
// ---------------------------------------------------------------------------------------------
__device__ __host__ inline int size_shift(int dtype) { return dtype == NT_F32 ? 2 : 1; }

// as loaded: 16-bit types in the first two words
__device__ inline u32x4 load4(int dtype, const char NT_GLOBAL* p) {
  if (dtype == NT_F32) return *(const u32x4_any NT_GLOBAL*)p;
  const u32x2 x = *(const u32x2_any NT_GLOBAL*)p;
  return u32x4{x[0], x[1], 0u, 0u};
}
// the first n < 4, zeros behind them
__device__ inline u32x4 load_part(int dtype, const char NT_GLOBAL* p, int n) {
  u32x4 r = {0u, 0u, 0u, 0u};
  if (dtype == NT_F32) {
    const uint32_t NT_GLOBAL* q = (const uint32_t NT_GLOBAL*)p;
    if (n > 0) r[0] = q[0];
    if (n > 1) r[1] = q[1];
    if (n > 2) r[2] = q[2];
  } else {
    const uint16_t NT_GLOBAL* q = (const uint16_t NT_GLOBAL*)p;
    if (n > 0) r[0] = q[0];
    if (n > 1) r[0] |= (uint32_t)q[1] << 16;
    if (n > 2) r[1] = q[2];
  }
  return r;
}
__device__ inline f32x4 values(int dtype, const u32x4& r) {
  if (dtype == NT_F32) return __builtin_bit_cast(f32x4, r);
  f32x4 x;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t w = r[e >> 1];
    if (dtype == NT_BF16)   // the high half of a binary32
      x[e] = __builtin_bit_cast(float, (e & 1) ? (w & 0xffff0000u) : (w << 16));
    else
      x[e] = (float)__builtin_bit_cast(_Float16, (uint16_t)((e & 1) ? w >> 16 : w));
  }
  return x;
}
// rounded to nearest even; as they are stored
__device__ inline u32x4 rounded(int dtype, const f32x4& x) {
  if (dtype == NT_F32) return __builtin_bit_cast(u32x4, x);
  u32x4 r = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t h = dtype == NT_BF16 ? __builtin_bit_cast(uint16_t, (__bf16)x[e]) : __builtin_bit_cast(uint16_t, (_Float16)x[e]);
    r[e >> 1] |= h << (16 * (e & 1));
  }
  return r;
}
__device__ inline void store4(int dtype, char NT_GLOBAL* p, const u32x4& r) {
  if (dtype == NT_F32)
    *(u32x4_any NT_GLOBAL*)p = r;
  else
    *(u32x2_any NT_GLOBAL*)p = u32x2{r[0], r[1]};
}
__device__ inline void store_part(int dtype, char NT_GLOBAL* p, const u32x4& r, int n) {
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) {
      if (dtype == NT_F32)
        ((uint32_t NT_GLOBAL*)p)[e] = r[e];
      else
        ((uint16_t NT_GLOBAL*)p)[e] = (uint16_t)(r[e >> 1] >> (16 * (e & 1)));
    }
}

// Where group q of four elements of an item lies: row and first column, and how many of the four there are (at most 0: none).
struct Spot {
  int64_t row, col;
  int n;
};
__device__ inline Spot spot(const Item& it, const Shape* shapes, int level, int64_t size, uint32_t q) {
  if (!(it.count & NT_ROWS)) {
    const int64_t left = (int64_t)it.count - 4 * (int64_t)q;
    return {0, it.idx * size + 4 * (int64_t)q, (int)(left < 4 ? left : 4)};
  }
  const Shape NT_CONST* s = constant(shapes) + it.tensor;
  const int64_t cols = s->cols;
  const uint32_t per_row = s->per_row[level], count = it.count & ~NT_ROWS;
  if (per_row) {
    const int64_t row = it.idx / per_row, col = (it.idx % per_row) * size + 4 * (int64_t)q;
    const int64_t end = (it.idx % per_row + 1) * size, left = (end < cols ? end : cols) - col;
    return {row, col, (int)(left < 4 ? (left < 0 ? 0 : left) : 4)};
  }
  const uint32_t quads = (uint32_t)((cols + 3) / 4);
  const uint32_t r = q / quads, c = 4 * (q % quads);
  const int64_t left = r < count ? cols - c : 0;
  return {(int64_t)it.idx * s->rows_per_item[level] + r, c, (int)(left < 4 ? left : 4)};
}
__device__ inline char NT_GLOBAL* address(const nt_tensor NT_CONST* t, int dtype, const Spot& s) {
  return (char NT_GLOBAL*)t->data + ((s.row * t->ld + s.col) << size_shift(dtype));
}

// ---------------------------------------------------------------------------------------------
// Partials of a norm
// ---------------------------------------------------------------------------------------------
struct Square {
  typedef double T;
  __device__ static inline void add(T& acc, float x) {
    const double y = (double)x;
    acc = __builtin_fma(y, y, acc);
  }
  __device__ static inline T join(T a, T b) { return a + b; }
  __device__ static inline double norm(T a) { return __builtin_sqrt(a); }
};
struct Largest {
  typedef uint64_t T;
  __device__ static inline void add(T& acc, float x) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
    if (b > (uint32_t)acc) acc = b;
  }
  __device__ static inline T join(T a, T b) { return a > b ? a : b; }
  __device__ static inline double norm(T a) { return (double)__builtin_bit_cast(float, (uint32_t)a); }
};
// the value of lane ^ MASK
template <class T>
__device__ inline T across(T x, int mask) {
  uint64_t w = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __shfl_xor((int)(uint32_t)w, mask), hi = __shfl_xor((int)(w >> 32), mask);
  return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
}
template <class K>
__device__ inline typename K::T wave_total(typename K::T x) {
#pragma unroll
  for (int mask = 32; mask > 0; mask >>= 1) x = K::join(x, across(x, mask));
  return x;
}

struct NormOut {
  Cut cut;
  double max_norm, grad_scale;
  nt_norm* norms;
};
template <class K>
__device__ inline void write_norm(const NormOut& o, uint32_t group, int64_t elements, typename K::T total) {
  const double raw = K::norm(total), norm = raw * __builtin_fabs(o.grad_scale);
  const bool finite = __builtin_isfinite(norm);
  nt_norm r;
  r.norm = norm;
  r.coef = 1.0;
  if (o.max_norm > 0.0 && finite) {
    const double c = o.max_norm / (norm + 1e-6);
    if (c < 1.0) r.coef = c;
  }
  r.norm32 = (float)norm;
  r.factor = (float)(o.grad_scale * r.coef);
  r.status = finite ? (norm == 0.0 ? NT_STATUS_ZERO_GRAD_NORM : 0u) : NT_STATUS_NONFINITE;
  r.clipped = r.coef < 1.0;
  r.elements = elements;
  o.norms[group] = r;
}

// The value goes through this XCD's L2 to memory and the count follows it.  Both are relaxed on purpose, since a release would write
// back all of the L2 in every block: on gfx950 a store of agent scope is written through, s_waitcnt vmcnt(0) returns once it has reached
// the memory that all XCDs share, and the same wave counts behind it.  The last one's acquire drops what its caches hold.  Nobody waits
// for another block.  True in the whole wave for the last of n.
template <class T>
__device__ inline bool last_of(T value, double* to, uint32_t* counter, uint32_t n) {
  uint32_t before = 0;
  if ((threadIdx.x & 63) == 0) {
    __hip_atomic_store((uint64_t*)to, __builtin_bit_cast(uint64_t, value), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if ((uint32_t)__builtin_amdgcn_readfirstlane((int)before) != n - 1) return false;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  if ((threadIdx.x & 63) == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}
// total of n stored values, in the whole wave
template <class K>
__device__ inline typename K::T total_of(const double* from, uint32_t n) {
  typename K::T t = 0;
  for (uint32_t i = threadIdx.x & 63; i < n; i += 64) t = K::join(t, __builtin_bit_cast(typename K::T, from[i]));
  return wave_total<K>(t);
}
// End of an item whose partial the block's lanes hold.
template <class K, int THREADS>
__device__ inline void end_item(const NormOut& o, uint32_t item, uint32_t slab_no, typename K::T acc) {
  __shared__ typename K::T red[THREADS / 64];
  acc = wave_total<K>(acc);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = acc;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  typename K::T total = red[0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) total = K::join(total, red[w]);
  const Slab NT_CONST* slab = constant(o.cut.slabs) + slab_no;
  const uint32_t first = slab->first, n = slab->n, g = slab->group;
  const Group NT_CONST* group = constant(o.cut.groups) + g;
  const uint32_t slab0 = group->first, slabs = group->n;
  if (n > 1) {
    if (!last_of(total, o.cut.partials + item, o.cut.counters + (size_t)NT_COUNTER_WORDS * slab_no, n)) return;
    total = total_of<K>(o.cut.partials + first, n);
  }
  if (slabs > 1) {
    if (!last_of(total, o.cut.sums + slab_no, o.cut.counters + (size_t)NT_COUNTER_WORDS * (o.cut.nslabs + g), slabs)) return;
    total = total_of<K>(o.cut.sums + slab0, slabs);
  }
  if (threadIdx.x == 0) write_norm<K>(o, g, group->elements, total);
}

// ---------------------------------------------------------------------------------------------
// Kernels
// ---------------------------------------------------------------------------------------------
struct ListArgs {
  const Shape* shapes;
  const Item* items;
  const Slab* slabs;
  uint32_t item0;       // of this launch
};

template <class K>
__global__ __launch_bounds__(NT_NORM_THREADS) void k_norm(ListArgs a, const nt_tensor* list, int level, uint32_t size, NormOut o) {
  const uint32_t item = a.item0 + blockIdx.x;
  const Item it = item_at(a.items, item);
  typename K::T acc = 0;
  if (it.count) {
    const nt_tensor NT_CONST* t = constant(list) + it.tensor;
    const int dtype = t->dtype;
    for (uint32_t q = threadIdx.x; q < size / 4; q += NT_NORM_THREADS) {
      const Spot s = spot(it, a.shapes, level, size, q);
      if (s.n <= 0) continue;
      const char NT_GLOBAL* p = address(t, dtype, s);
      const f32x4 x = values(dtype, s.n == 4 ? load4(dtype, p) : load_part(dtype, p, s.n));
#pragma unroll
      for (int e = 0; e < 4; ++e) K::add(acc, x[e]);   // the zeros of a part add nothing
    }
  }
  end_item<K, NT_NORM_THREADS>(o, item, it.slab, acc);
}

struct UpdateArgs {
  const nt_tensor* dst;
  const nt_tensor* src;
  const nt_norm* norms;   // of src, may be null
  double scale;
  float beta;
  int in_place;           // dst is src, and nothing is to be done where the factor is 1
};
// dst <- beta dst + scale factor src
template <bool READ, class K>
__global__ __launch_bounds__(NT_THREADS) void k_update(ListArgs a, UpdateArgs u, NormOut o) {
  constexpr bool NORM = !__is_same(K, void);
  const uint32_t item = a.item0 + blockIdx.x;
  const Item it = item_at(a.items, item);
  f32x4 stored = {0.f, 0.f, 0.f, 0.f};
  if (it.count) {
    const nt_tensor NT_CONST* x = constant(u.src) + it.tensor;
    const nt_tensor NT_CONST* y = constant(u.dst) + it.tensor;
    float scale = (float)u.scale;
    if (u.norms) {
      const float factor = (constant(u.norms) + (constant(a.slabs) + it.slab)->group)->factor;
      if (u.in_place && factor == 1.f) return;
      scale = (float)(u.scale * (double)factor);
    }
    const Spot s = spot(it, a.shapes, 0, NT_ITEM, threadIdx.x);
    if (s.n > 0) {
      const int xt = x->dtype, yt = y->dtype;
      const char NT_GLOBAL* from = address(x, xt, s);
      char NT_GLOBAL* to = address(y, yt, s);
      const u32x4 xr = s.n == 4 ? load4(xt, from) : load_part(xt, from, s.n);
      u32x4 yr = {0u, 0u, 0u, 0u};
      if constexpr (READ) yr = s.n == 4 ? load4(yt, to) : load_part(yt, to, s.n);
      const f32x4 xv = values(xt, xr), yv = values(yt, yr);
      f32x4 z;
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = READ ? __builtin_fmaf(scale, xv[e], u.beta * yv[e]) : scale * xv[e];
      const u32x4 zr = rounded(yt, z);
      if (s.n == 4)
        store4(yt, to, zr);
      else
        store_part(yt, to, zr, s.n);
      if constexpr (NORM) {
        stored = values(yt, zr);
#pragma unroll
        for (int e = 0; e < 4; ++e) stored[e] = e < s.n ? stored[e] : 0.f;   // inf * 0 of a part's end
      }
    }
  }
  if constexpr (NORM) {
    typename K::T acc = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) K::add(acc, stored[e]);
    end_item<K, NT_THREADS>(o, item, it.slab, acc);
  }
}

struct AdamwArgs {
  const nt_tensor *grads, *w, *m, *v, *copy;
  const nt_norm* norms;   // may be null
  double grad_scale;
  uint32_t flags;
  float beta1, omb1, beta2, omb2;   // omb = 1 - beta
  float decay;                      // 1 - lr * weight_decay
  float step_size;                  // lr / (1 - beta1^k)
  float inv_sqrt_bc2;               // 1 / sqrt(1 - beta2^k)
  float eps;
};
// AdamW on one element, with the operations and so the bits of the flat vector's kernels: sqrt and reciprocal are the 1-ulp hardware
// forms, and since that square root takes a subnormal for zero, a second moment below 2^-96 is scaled by 2^64 first.
__device__ inline void adamw_element(const AdamwArgs& p, float g, float& w, float& m, float& v) {
  m = __builtin_fmaf(p.beta1, m, p.omb1 * g);
  v = __builtin_fmaf(p.beta2, v, (p.omb2 * g) * g);
  const bool tiny = v < 0x1p-96f;
  float root = __builtin_amdgcn_sqrtf(tiny ? v * 0x1p+64f : v);
  root = tiny ? root * 0x1p-32f : root;
  const float denom = __builtin_fmaf(root, p.inv_sqrt_bc2, p.eps);
  const float upd = (p.step_size * m) * __builtin_amdgcn_rcpf(denom);
  w = __builtin_fmaf(p.decay, w, -upd);
}
__global__ __launch_bounds__(NT_THREADS) void k_adamw(ListArgs a, AdamwArgs u) {
  const Item it = item_at(a.items, a.item0 + blockIdx.x);
  if (!it.count) return;
  const nt_tensor NT_CONST* gt = constant(u.grads) + it.tensor;
  const nt_tensor NT_CONST* wt = constant(u.w) + it.tensor;
  const nt_tensor NT_CONST* mt = constant(u.m) + it.tensor;
  const nt_tensor NT_CONST* vt = constant(u.v) + it.tensor;
  float scale = (float)u.grad_scale;
  if (u.norms) {
    const nt_norm NT_CONST* n = constant(u.norms) + (constant(a.slabs) + it.slab)->group;
    if ((u.flags & NT_SKIP_NONFINITE) && (n->status & NT_STATUS_NONFINITE)) return;
    scale = (float)u.grad_scale * n->factor;
  }
  const Spot s = spot(it, a.shapes, 0, NT_ITEM, threadIdx.x);
  if (s.n <= 0) return;
  const int dtype = gt->dtype;
  const char NT_GLOBAL* gp = address(gt, dtype, s);
  char NT_GLOBAL *wp = address(wt, NT_F32, s), *mp = address(mt, NT_F32, s), *vp = address(vt, NT_F32, s);
  u32x4 gr, wr, mr, vr;
  if (s.n == 4) {
    gr = load4(dtype, gp);
    wr = load4(NT_F32, wp);
    mr = load4(NT_F32, mp);
    vr = load4(NT_F32, vp);
  } else {
    gr = load_part(dtype, gp, s.n);
    wr = load_part(NT_F32, wp, s.n);
    mr = load_part(NT_F32, mp, s.n);
    vr = load_part(NT_F32, vp, s.n);
  }
  const f32x4 g = values(dtype, gr);
  f32x4 w = __builtin_bit_cast(f32x4, wr), m = __builtin_bit_cast(f32x4, mr), v = __builtin_bit_cast(f32x4, vr);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float we = w[e], me = m[e], ve = v[e];
    adamw_element(u, scale * g[e], we, me, ve);
    w[e] = we;
    m[e] = me;
    v[e] = ve;
  }
  wr = __builtin_bit_cast(u32x4, w);
  mr = __builtin_bit_cast(u32x4, m);
  vr = __builtin_bit_cast(u32x4, v);
  if (s.n == 4) {
    store4(NT_F32, wp, wr);
    store4(NT_F32, mp, mr);
    store4(NT_F32, vp, vr);
  } else {
    store_part(NT_F32, wp, wr, s.n);
    store_part(NT_F32, mp, mr, s.n);
    store_part(NT_F32, vp, vr, s.n);
  }
  if (u.copy) {
    const nt_tensor NT_CONST* ct = constant(u.copy) + it.tensor;
    const int to = ct->dtype;
    const u32x4 c = rounded(to, w);
    if (s.n == 4)
      store4(to, address(ct, to, s), c);
    else
      store_part(to, address(ct, to, s), c, s.n);
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
inline int hip_code(hipError_t e) { return e == hipSuccess ? NT_OK : NT_ERR_HIP_BASE - (int)e; }
inline bool misaligned8(const void* p) { return ((uintptr_t)p & 7u) != 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The pieces of one tensor at one item size: NT_OK and how many, or an error.
struct Pieces {
  int64_t n;
  uint32_t per_row, rows_per_item;
};
Pieces pieces_of(int64_t rows, int64_t cols, int64_t size) {
  if (rows == 0 || cols == 0) return {0, 0, 0};
  if (rows == 1) return {ceil_div(cols, size), 0, 0};
  if (cols > size) return {rows * ceil_div(cols, size), (uint32_t)ceil_div(cols, size), 0};
  const int64_t per_item = (size / 4) / ceil_div(cols, 4);
  return {ceil_div(rows, per_item), 0, (uint32_t)per_item};
}
// Items of a slab: about as many as there are slabs, so that neither count is long.
uint32_t slab_items(int64_t items) {
  uint32_t n = 16;
  while (n < 256 && (int64_t)n * n < items) n *= 2;
  return n;
}

Cut cut_of(const nt_plan& p, const Layout& l, int k) {
  char* const b = (char*)p.image;
  return {(const Item*)(b + l.items[k]), (const Slab*)(b + l.slabs[k]), (const Group*)(b + l.groups[k]), (uint32_t*)(b + l.counters[k]),
          (double*)(b + l.partials[k]), (double*)(b + l.sums[k]), p.slabs[k]};
}

int check_plan(const nt_plan* p) {
  if (!p || p->magic != NT_PLAN_MAGIC || !p->image || ((uintptr_t)p->image & 15u) || p->groups < 1 || p->tensors < 0) return NT_ERR_BAD_ARG;
  return NT_OK;
}
int check_list(const nt_plan& p, const nt_tensor* list) {
  return (p.tensors > 0 && !list) || misaligned8(list) ? NT_ERR_BAD_ARG : NT_OK;
}
int check_norm(int32_t kind, double max_norm, double grad_scale, const nt_norm* norms) {
  if ((kind != NT_NORM_L2 && kind != NT_NORM_MAX) || std::isnan(max_norm) || !std::isfinite(grad_scale)) return NT_ERR_BAD_ARG;
  return !norms || misaligned8(norms) ? NT_ERR_BAD_ARG : NT_OK;
}

// LAUNCH(first item, blocks) over all items of a cut
template <class LAUNCH>
int in_launches(uint32_t items, uint32_t most, LAUNCH launch) {
  for (uint32_t at = 0; at < items;) {
    const uint32_t n = items - at < most ? items - at : most;
    launch(at, n);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_code(e);
    at += n;
  }
  return NT_OK;
}

template <bool READ>
int enqueue_update(const nt_plan& p, const Layout& l, const UpdateArgs& u, int kind, const NormOut& o, hipStream_t st) {
  const Cut cut = cut_of(p, l, 0);
  ListArgs a = {(const Shape*)((char*)p.image + l.shapes), cut.items, cut.slabs, 0};
  return in_launches(p.items[0], NT_MOST_BLOCKS, [&](uint32_t at, uint32_t n) {
    a.item0 = at;
    if (!o.norms)
      hipLaunchKernelGGL((k_update<READ, void>), dim3(n), dim3(NT_THREADS), 0, st, a, u, o);
    else if (kind == NT_NORM_L2)
      hipLaunchKernelGGL((k_update<READ, Square>), dim3(n), dim3(NT_THREADS), 0, st, a, u, o);
    else
      hipLaunchKernelGGL((k_update<READ, Largest>), dim3(n), dim3(NT_THREADS), 0, st, a, u, o);
  });
}

}  // namespace

extern "C" {

int normtest_plan_make(const nt_tensor* tensors, int32_t N, int32_t G, nt_plan* plan, void* image, size_t image_bytes) {
  if (!plan || N < 0 || G < 1 || (N > 0 && !tensors) || misaligned8(image)) return NT_ERR_BAD_ARG;
  nt_plan p;
  std::memset(&p, 0, sizeof(p));
  int64_t elements = 0;
  for (int32_t i = 0; i < N; ++i) {
    const nt_tensor& t = tensors[i];
    if (t.rows < 0 || t.cols < 0 || t.group < 0 || t.group >= G) return NT_ERR_BAD_ARG;
    if (t.rows > 1 && t.ld < t.cols) return NT_ERR_BAD_ARG;
    int64_t n;
    if (__builtin_mul_overflow(t.rows, t.cols, &n) || __builtin_add_overflow(elements, n, &elements) || elements > (1ll << 43))
      return NT_ERR_TOO_LARGE;
  }
  p.elements = elements;
  p.tensors = N;
  p.groups = G;
  p.magic = NT_PLAN_MAGIC;
  const int cuts = elements >= NT_LONG_LIST ? 2 : 1;
  const int64_t sizes[2] = {NT_ITEM, NT_LONG_ITEM};

  // the tensors in the order of their groups; a group without items gets an empty one
  int64_t* const first = new (std::nothrow) int64_t[(size_t)G + 1]();
  int32_t* const order = new (std::nothrow) int32_t[(size_t)N + 1]();
  struct Held {
    int64_t* a;
    int32_t* b;
    ~Held() {
      delete[] a;
      delete[] b;
    }
  } held = {first, order};
  if (!first || !order) return NT_ERR_TOO_LARGE;
  for (int32_t i = 0; i < N; ++i) ++first[tensors[i].group + 1];
  for (int32_t g = 0; g < G; ++g) first[g + 1] += first[g];
  for (int32_t i = 0; i < N; ++i) order[first[tensors[i].group]++] = i;
  // first[g] is now the end of group g
  auto group_begin = [&](int32_t g) { return g ? first[g - 1] : 0; };

  uint32_t per_slab[2] = {0, 0};
  for (int k = 0; k < cuts; ++k) {
    int64_t items = 0;
    for (int32_t i = 0; i < N; ++i) {
      items += pieces_of(tensors[i].rows, tensors[i].cols, sizes[k]).n;
      if (items > (1ll << 31) - 1) return NT_ERR_TOO_LARGE;
    }
    per_slab[k] = slab_items(items);
    int64_t slabs = 0;
    for (int32_t g = 0; g < G; ++g) {
      int64_t here = 0;
      for (int64_t j = group_begin(g); j < first[g]; ++j) here += pieces_of(tensors[order[j]].rows, tensors[order[j]].cols, sizes[k]).n;
      if (here == 0) {
        ++items;
        here = 1;
      }
      slabs += ceil_div(here, per_slab[k]);
    }
    if (items > (1ll << 31) - 1) return NT_ERR_TOO_LARGE;
    p.items[k] = (uint32_t)items;
    p.slabs[k] = (uint32_t)slabs;
  }
  const Layout l = layout_of(p);
  p.bytes = l.bytes;
  p.upload_bytes = l.upload;
  if (image) {
    if (image_bytes < l.upload) return NT_ERR_WORKSPACE_TOO_SMALL;
    char* const b = (char*)image;
    std::memset(b, 0, l.upload);
    for (int32_t i = 0; i < N; ++i) {
      Shape& s = ((Shape*)(b + l.shapes))[i];
      s.rows = tensors[i].rows;
      s.cols = tensors[i].cols;
      for (int k = 0; k < cuts; ++k) {
        const Pieces c = pieces_of(s.rows, s.cols, sizes[k]);
        s.per_row[k] = c.per_row;
        s.rows_per_item[k] = c.rows_per_item;
      }
    }
    for (int k = 0; k < cuts; ++k) {
      Item* items = (Item*)(b + l.items[k]);
      Slab* slabs = (Slab*)(b + l.slabs[k]);
      Group* groups = (Group*)(b + l.groups[k]);
      uint32_t item = 0, slab = 0;
      for (int32_t g = 0; g < G; ++g) {
        groups[g].first = slab;
        const uint32_t begin = item;
        auto put = [&](uint32_t tensor, uint32_t idx, uint32_t count) {
          const uint32_t in = (item - begin) % per_slab[k];
          if (in == 0) slabs[slab++] = {item, 0, (uint32_t)g, 0};
          slabs[slab - 1].n = in + 1;
          items[item++] = {tensor, idx, slab - 1, count};
        };
        for (int64_t j = group_begin(g); j < first[g]; ++j) {
          const nt_tensor& t = tensors[order[j]];
          groups[g].elements += t.rows * t.cols;
          const Pieces c = pieces_of(t.rows, t.cols, sizes[k]);
          for (int64_t idx = 0; idx < c.n; ++idx) {
            int64_t count;
            if (t.rows == 1)
              count = t.cols - idx * sizes[k] < sizes[k] ? t.cols - idx * sizes[k] : sizes[k];
            else if (c.per_row)
              count = 1 | (int64_t)NT_ROWS;
            else
              count = (t.rows - idx * c.rows_per_item < c.rows_per_item ? t.rows - idx * c.rows_per_item : c.rows_per_item) | (int64_t)NT_ROWS;
            put((uint32_t)order[j], (uint32_t)idx, (uint32_t)count);
          }
        }
        if (item == begin) put(0, 0, 0);
        groups[g].n = slab - groups[g].first;
      }
    }
  }
  p.image = plan->image;
  *plan = p;
  return NT_OK;
}

int normtest_list_check(const nt_tensor* list, const nt_tensor* like, int32_t N, uint32_t dtypes) {
  if (N < 0 || (N > 0 && (!list || !like))) return NT_ERR_BAD_ARG;
  for (int32_t i = 0; i < N; ++i) {
    const nt_tensor& t = list[i];
    if (t.dtype < 0 || t.dtype > 2 || !(dtypes >> t.dtype & 1)) return NT_ERR_UNSUPPORTED;
    if (t.rows != like[i].rows || t.cols != like[i].cols || t.rows < 0 || t.cols < 0) return NT_ERR_BAD_ARG;
    if (t.rows == 0 || t.cols == 0) continue;
    if (!t.data || ((uintptr_t)t.data & ((1u << size_shift(t.dtype)) - 1)) || (t.rows > 1 && t.ld < t.cols)) return NT_ERR_BAD_ARG;
  }
  return NT_OK;
}

int normtest_grad_norm(const nt_plan* plan, const nt_tensor* grads, int32_t kind, double max_norm, double grad_scale, nt_norm* norms,
                       void* hip_stream) {
  int rc = check_plan(plan);
  if (rc == NT_OK) rc = check_list(*plan, grads);
  if (rc == NT_OK) rc = check_norm(kind, max_norm, grad_scale, norms);
  if (rc != NT_OK) return rc;
  const Layout l = layout_of(*plan);
  const int k = plan->items[1] ? 1 : 0;
  const uint32_t size = k ? NT_LONG_ITEM : NT_ITEM;
  const NormOut o = {cut_of(*plan, l, k), max_norm, grad_scale, norms};
  ListArgs a = {(const Shape*)((char*)plan->image + l.shapes), o.cut.items, o.cut.slabs, 0};
  hipStream_t st = (hipStream_t)hip_stream;
  return in_launches(plan->items[k], NT_MOST_BLOCKS, [&](uint32_t at, uint32_t n) {
    a.item0 = at;
    if (kind == NT_NORM_L2)
      hipLaunchKernelGGL(k_norm<Square>, dim3(n), dim3(NT_NORM_THREADS), 0, st, a, grads, k, size, o);
    else
      hipLaunchKernelGGL(k_norm<Largest>, dim3(n), dim3(NT_NORM_THREADS), 0, st, a, grads, k, size, o);
  });
}

int normtest_clip_grads(const nt_plan* plan, const nt_tensor* grads, const nt_tensor* out, const nt_norm* norms, void* hip_stream) {
  int rc = check_plan(plan);
  if (rc == NT_OK) rc = check_list(*plan, grads);
  if (rc != NT_OK) return rc;
  if (!norms || misaligned8(norms) || misaligned8(out)) return NT_ERR_BAD_ARG;
  UpdateArgs u = {out ? out : grads, grads, norms, 1.0, 0.f, !out || out == grads};
  NormOut o;
  std::memset(&o, 0, sizeof(o));
  return enqueue_update<false>(*plan, layout_of(*plan), u, 0, o, (hipStream_t)hip_stream);
}

int normtest_accumulate(const nt_plan* plan, const nt_tensor* dst, const nt_tensor* src, double beta, double scale,
                        const nt_norm* src_norms, int32_t kind, double max_norm, double grad_scale, nt_norm* dst_norms,
                        void* hip_stream) {
  int rc = check_plan(plan);
  if (rc == NT_OK) rc = check_list(*plan, dst);
  if (rc == NT_OK) rc = check_list(*plan, src);
  if (rc == NT_OK && dst_norms) rc = check_norm(kind, max_norm, grad_scale, dst_norms);
  if (rc != NT_OK) return rc;
  if (!std::isfinite(beta) || !std::isfinite(scale) || misaligned8(src_norms)) return NT_ERR_BAD_ARG;
  const Layout l = layout_of(*plan);
  const UpdateArgs u = {dst, src, src_norms, scale, (float)beta, 0};
  NormOut o;
  std::memset(&o, 0, sizeof(o));
  if (dst_norms) o = {cut_of(*plan, l, 0), max_norm, grad_scale, dst_norms};
  return beta == 0.0 ? enqueue_update<false>(*plan, l, u, kind, o, (hipStream_t)hip_stream)
                     : enqueue_update<true>(*plan, l, u, kind, o, (hipStream_t)hip_stream);
}

int normtest_adamw_tensors(const nt_plan* plan, const nt_tensor* grads, const nt_tensor* w, const nt_tensor* m, const nt_tensor* v,
                           const nt_tensor* copy, const nt_hyper* hyper, double grad_scale, const nt_norm* norms, uint32_t flags,
                           void* hip_stream) {
  int rc = check_plan(plan);
  for (const nt_tensor* list : {grads, w, m, v})
    if (rc == NT_OK) rc = check_list(*plan, list);
  if (rc != NT_OK) return rc;
  if (!hyper || !std::isfinite(grad_scale) || misaligned8(copy) || misaligned8(norms) || (flags & ~(uint32_t)NT_SKIP_NONFINITE) ||
      ((flags & NT_SKIP_NONFINITE) && !norms))
    return NT_ERR_BAD_ARG;
  if (hyper->step < 1 || !(hyper->lr >= 0.0) || !std::isfinite(hyper->lr) || !(hyper->beta1 >= 0.0 && hyper->beta1 < 1.0) ||
      !(hyper->beta2 >= 0.0 && hyper->beta2 < 1.0) || !(hyper->eps >= 0.0) || !std::isfinite(hyper->eps) ||
      !(hyper->weight_decay >= 0.0) || !std::isfinite(hyper->weight_decay))
    return NT_ERR_BAD_ARG;
  const double bc1 = 1.0 - std::pow(hyper->beta1, (double)hyper->step), bc2 = 1.0 - std::pow(hyper->beta2, (double)hyper->step);
  const AdamwArgs u = {grads, w, m, v, copy, norms, grad_scale, flags,
                       (float)hyper->beta1, (float)(1.0 - hyper->beta1), (float)hyper->beta2, (float)(1.0 - hyper->beta2),
                       (float)(1.0 - hyper->lr * hyper->weight_decay), (float)(hyper->lr / bc1), (float)(1.0 / std::sqrt(bc2)),
                       (float)hyper->eps};
  const Layout l = layout_of(*plan);
  const Cut cut = cut_of(*plan, l, 0);
  ListArgs a = {(const Shape*)((char*)plan->image + l.shapes), cut.items, cut.slabs, 0};
  hipStream_t st = (hipStream_t)hip_stream;
  return in_launches(plan->items[0], NT_MOST_BLOCKS, [&](uint32_t at, uint32_t n) {
    a.item0 = at;
    hipLaunchKernelGGL(k_adamw, dim3(n), dim3(NT_THREADS), 0, st, a, u);
  });
}

}  // extern "C"
