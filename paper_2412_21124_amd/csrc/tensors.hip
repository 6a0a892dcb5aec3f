// Norms, clipping, accumulation and AdamW over lists of tensors, hand-written for gfx950 (MI355X).
//
// A list is cut into items, pieces of one tensor each, by a plan that the host makes once (normtest_plan_make): for the calls that
// write, items of NT_ITEM elements, one for each block, 4 to 16 elements a thread; for the norm alone, which only reads, longer ones, of
// which a block takes several.  Which tensor an item belongs to and where it begins is one 16-byte record, the tensor's address a second one.
// All of it is bound by memory (2 operations a byte), so nothing here is a matrix product; short lists are bound by the way from a launch
// over the two records to the elements and back (some 4 us), and a norm by the counting and adding up behind it (1 to 2 us more).  Measured:
// norm of 1.5e9 bf16 433 us, 6.9 TB/s (a plain read of the same bytes 400); accumulation of 304.6M bf16 296 us, 6.2 TB/s; norm and clipped
// AdamW of 1.1e9 bf16 with a bf16 copy 5.7 ms, 5.8 TB/s with the gradients read twice (an arithmetic-free mix of the kind 5.6 to 5.9).
//
// Norms.  x^2 is formed and summed in fp64, so no finite value overflows and no rounding of the sum is seen; the largest
// magnitude is the largest |x| by its bits as an integer, where a NaN is larger than infinity and so survives.  A block leaves
// one partial for every group that it meets; the blocks of a slab of partials count themselves, the last one adds the slab up, and the
// last slab of a group the group's slabs, and writes its record: one launch, no floating-point atomics, sums in an order that the plan
// alone fixes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <initializer_list>
#include <memory>
#include <new>

#include "normtest.h"

// Sizes and shapes.  Each was chosen between the neighbours it was timed against; times are of whole calls, in us, of lists that the
// cache below may hold from one pass to the next.
#define NT_ITEM 4096               // elements of an item of the kernels that write (8192: AdamW of 1M elements 14.8 -> 16.0, else the same)
#define NT_UPDATE_THREADS 256      // threads of a block of the update (512: clip of 124M bf16 116 -> 146)
#define NT_TOTAL_THREADS 512       // and where it forms a norm (256: 100k elements 5.3 -> 6.0, 124M 201 -> 208, 304.6M 297 -> 305)
#define NT_ADAMW_THREADS 512       // threads of a block of AdamW (256: 16M elements 79 -> 104; 1024: the same)
// Elements from which AdamW's blocks are kept in step: an item in one sweep, one block of a CU (it asks for more than half of the LDS), a
// launch per 2^26 elements.  Blocks that start together load together and store together, which memory serves faster: 64M elements 320 ->
// 307, 137.5M 864 -> 754, 1.1e9 6139 -> 5758; 32M 149 -> 150.  Not where rows are walked (100M elements in slices 602 -> 631).
#define NT_STEP_LIST (5ll << 23)
#define NT_STEP_THREADS 1024
#define NT_STEP_LDS 82000
#define NT_STEP_ITEMS 16384        // (8192: 124M elements 613 -> 625)
#define NT_NORM_THREADS 256        // threads of a block of the norm's kernel (512: 1.5e9 bf16 429 -> 479)
#define NT_NORM_FLIGHT 4           // 16-byte loads that a thread of it has in flight
#define NT_LONG_LIST (1ll << 21)   // elements from which the norm has longer items (4.5M bf16 8.0 -> 6.5, 30M 20.3 -> 14.5; 1M the same)
#define NT_LONG_ITEM 8192          // elements of those (1.5e9 bf16: 418; 4096 535, 16384 429; all without the ends)
#define NT_LONG_BLOCKS 1024        // blocks that walk a long list (1.5e9 bf16 432; 512 488, 2048 469, a block per item 463)
#define NT_RUN 2                   // items of a block in a long list of many groups (75 groups, 30M fp16 14.7; 1 15.5, 4 15.8; of rows 1: 3M bf16 8.5 -> 7.2)
#define NT_MOST_BLOCKS (1u << 20)  // blocks of one launch
// Elements from which loads (and stores) go past the 256 MB cache that the chip's memory has, because what they touch would not stay in it
// until it is needed again.
// What is only read, gradients, which the norm's kernel leaves there for the next call: norm of 1.5e9 bf16 510 -> 471, of 400M 145 -> 135;
// from 2^26 on, norm and clip of 124M 117 -> 124.
#define NT_STREAM_READ (1ll << 27)
#define NT_STREAM_UPDATE (3ll << 23)   // what an update writes: accumulation of 32M bf16 into fp32 59 -> 51, 64M 122 -> 96; 16M the same
#define NT_STREAM_ADAMW (1ll << 23)    // weights and moments: 16M elements 93 -> 80, 64M 364 -> 308; 8M 44 -> 45
#define NT_PLAN_MAGIC 0x4e54504cu
#define NT_PLAN_ROWS 1u         // most elements are in tensors with rows
#define NT_FEW_SLOTS 1024       // partials of a group that the last block adds up by itself (none: 1M elements 6.2 -> 7.1; 4096: 16M 32 -> 35)
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
  uint32_t tensor, idx, group, count;
};
__device__ inline Item item_at(const Item* items, uint32_t i) {
  return __builtin_bit_cast(Item, ((const u32x4 NT_CONST*)(uintptr_t)items)[i]);
}
// A group's items are consecutive, and so are the partials (slots) that the blocks leave for it.  A block that takes a run of items is
// the (b - item0 / run)-th to meet a group whose items begin at item0.  One that walks items b, b + blocks, ... meets it first at the item that is
// ((b - item0) mod blocks) further on.  That number is its slot in the group.  A slab is a power of two of a group's slots.
struct Group {
  uint32_t item0, slot0, slots, slab0;
  int64_t elements, pad;
};
struct Shape {
  int64_t rows, cols;
  uint32_t per_row[2], rows_per_item[2];   // at both item sizes; per_row 0: whole rows
};

// One way of cutting a list: items of one size, and what adds up their partials.
struct Cut {
  const Item* items;
  const Group* groups;
  uint32_t* counters;   // of the slabs, then of the groups; zero before and after every launch
  double* partials;     // one per slot
  double* sums;         // one per slab
  uint32_t nitems, nslabs;
  uint32_t blocks;      // a power of two: block b takes items b, b + blocks, ...
  uint32_t run;         // or, if not zero: items b run .. b run + run - 1
  int shift;            // a slab is up to 1 << shift slots
};
struct Layout {
  size_t shapes, items[2], groups[2], counters[2], upload, partials[2], sums[2], bytes;
};
// Who takes a cut's items: of the first cut, a block each.  The norm's kernel walks a long list with few blocks, unless its groups are so
// short that a block would meet another one, and end a part, with almost every item: then a block takes a run of items, as long as makes
// one launch of them (a grid ends at 2^32 threads; an offset in the kernel, for further launches, made the norm of each of 75 tensors
// 13.9 -> 14.4 us).
uint32_t run_of(const nt_plan& p, int k) {
  if (k == 0) return 1;
  if (p.items[1] >= (int64_t)p.groups * NT_LONG_BLOCKS) return 0;
  const uint32_t run = p.flags & NT_PLAN_ROWS ? 1 : NT_RUN, least = (p.items[1] - 1) / NT_MOST_BLOCKS + 1;
  return run < least ? least : run;
}
// parts of a group that begins with item `begin`
int64_t slots_of(uint32_t run, int64_t begin, int64_t items) {
  if (run) return (begin + items - 1) / run - begin / run + 1;
  return items < NT_LONG_BLOCKS ? items : NT_LONG_BLOCKS;
}
constexpr int64_t SIZES[2] = {NT_ITEM, NT_LONG_ITEM};
// A slab is all slots, or about as many as there are slabs, so that neither counter is counted up often: a counter takes some 10 ns
// per block, a second one some 0.7 us (one of 512 slots: 1M elements 6.2 -> 8.0 us).
int slab_shift(uint32_t slots) {
  if (slots <= 128) return 7;
  int shift = 4;
  while (shift < 8 && slots >> (2 * shift)) ++shift;
  return shift;
}
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
    l.groups[k] = take(p.items[k] ? sizeof(Group) * (size_t)p.groups : 0);
    l.counters[k] = take(p.items[k] ? 4 * NT_COUNTER_WORDS * ((size_t)p.slabs[k] + p.groups) : 0);
  }
  l.upload = at;
  for (int k = 0; k < 2; ++k) {
    l.partials[k] = take(sizeof(double) * (size_t)p.slots[k]);
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

// The elements of an item that is not a whole one of a tensor of one row, four at a time: quad c of the item's row r.  A thread takes
// every THREADS-th quad; only its first place takes a division by the row's quads, which differ from tensor to tensor.
template <int THREADS>
struct Walk {
  int64_t row0, col0;                 // of the item
  uint32_t rows, width, quads;        // of the item
  uint32_t r, c, dr, dc;
  bool wrapped;
  // `width` elements of a tensor of one row from column `col` on
  __device__ inline Walk(int64_t col, uint32_t n) {
    row0 = 0;
    col0 = col;
    rows = 1;
    width = n;
    quads = 1u << 30;   // more than there are: no other row follows
    r = dr = 0;
    c = threadIdx.x;
    dc = THREADS;
  }
  __device__ inline Walk(const Item& it, const Shape* shapes, int level, uint32_t size) : Walk((int64_t)it.idx * size, it.count) {
    if (it.count & NT_ROWS) {
      const Shape NT_CONST* s = constant(shapes) + it.tensor;
      const uint32_t per_row = s->per_row[level];
      row0 = per_row ? it.idx / per_row : (int64_t)it.idx * s->rows_per_item[level];
      col0 = per_row ? (int64_t)(it.idx % per_row) * size : 0;
      rows = it.count & ~NT_ROWS;
      const int64_t left = s->cols - col0;
      width = left < size ? (uint32_t)left : size;
      quads = (width + 3) / 4;
      r = threadIdx.x / quads;
      c = threadIdx.x % quads;
      dr = THREADS / quads;
      dc = THREADS % quads;
    }
  }
  // how many elements there are at this place: 0 past the item's end
  __device__ inline int here() const {
    const int left = (int)width - 4 * (int)c;
    return r < rows && left > 0 ? (left < 4 ? left : 4) : 0;
  }
  __device__ inline void step() {
    r += dr;
    c += dc;
    wrapped = c >= quads;
    if (wrapped) {
      c -= quads;
      ++r;
    }
  }
};
// The walk's place in one tensor, in bytes from the item's first element; it steps behind the walk.
template <int DTYPE>
struct Place {
  char NT_GLOBAL* base;      // of the item, the same for the whole block
  uint64_t off, by, wrap;    // by: of a step; wrap: more where it goes on to another row
  template <class W>
  __device__ inline Place(const nt_tensor NT_CONST* t, const W& at) {
    const uint64_t ld = t->ld;
    constexpr int shift = DTYPE == NT_F32 ? 2 : 1;
    base = (char NT_GLOBAL*)t->data + ((at.row0 * (int64_t)ld + at.col0) << shift);
    off = (at.r * ld + 4 * at.c) << shift;
    by = (at.dr * ld + 4 * at.dc) << shift;
    wrap = (ld - 4 * (uint64_t)at.quads) << shift;
  }
  template <class W>
  __device__ inline void step(const W& at) {
    off += at.wrapped ? by + wrap : by;
  }
  // The n elements here.  A row's last one to three are loaded with the same instruction as four, from four before the row's end on, and
  // settle() moves them down; what else it loads is its neighbour's, which may have been written by then, and is moved out.  Element by
  // element they were a chain of loads in every wave that meets a row's end.  (Two functions, so that several loads are under way.)
  template <class W>
  __device__ inline u32x4 load(const W& at, int n) const {
    u32x4 x = {0u, 0u, 0u, 0u};
    if (at.width < 4)
      x = load_part(DTYPE, base + off, n);
    else if (n > 0)
      x = load4(DTYPE, base + (off - ((uint64_t)(uint32_t)(4 - n) << size_shift(DTYPE))));
    return x;
  }
  template <class W>
  __device__ static inline u32x4 settle(const W& at, const u32x4& x, int n) {
    if (n == 4 || at.width < 4) return x;
    const int back = 4 - n;   // 4: no element, and zeros already
    if (DTYPE == NT_F32) {
      const u32x4 y = back & 1 ? u32x4{x[1], x[2], x[3], 0u} : x;
      return back & 2 ? u32x4{y[2], y[3], 0u, 0u} : y;
    }
    const uint64_t y = ((uint64_t)x[1] << 32 | x[0]) >> (16 * back & 63);
    return u32x4{(uint32_t)y, (uint32_t)(y >> 32), 0u, 0u};
  }
};
__device__ inline void store_n(int dtype, char NT_GLOBAL* p, const u32x4& x, int n) {
  if (n == 4)
    store4(dtype, p, x);
  else
    store_part(dtype, p, x, n);
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
// Total over the wave, in its first lane, on the vector unit: register halves and then rows of 16 lanes change places, and within a row
// values move up by 8, 4, 2 and 1 lanes (zeros come in, which add nothing).  By permutes through LDS a norm of 100k elements took 4.6 us instead of 4.3.
struct Words {
  uint32_t lo, hi;
};
template <class K>
__device__ inline typename K::T wave_total(typename K::T x) {
  typedef typename K::T T;
  Words w = __builtin_bit_cast(Words, x);
  auto lo = __builtin_amdgcn_permlane32_swap(w.lo, w.lo, false, false);
  auto hi = __builtin_amdgcn_permlane32_swap(w.hi, w.hi, false, false);
  x = K::join(__builtin_bit_cast(T, (Words{lo[0], hi[0]})), __builtin_bit_cast(T, (Words{lo[1], hi[1]})));
  w = __builtin_bit_cast(Words, x);
  lo = __builtin_amdgcn_permlane16_swap(w.lo, w.lo, false, false);
  hi = __builtin_amdgcn_permlane16_swap(w.hi, w.hi, false, false);
  x = K::join(__builtin_bit_cast(T, (Words{lo[0], hi[0]})), __builtin_bit_cast(T, (Words{lo[1], hi[1]})));
#define NT_UP(LANES)                                                                                       \
  w = __builtin_bit_cast(Words, x);                                                                        \
  x = K::join(x, __builtin_bit_cast(T, (Words{(uint32_t)__builtin_amdgcn_mov_dpp((int)w.lo, 0x100 + LANES, 0xf, 0xf, true), \
                                              (uint32_t)__builtin_amdgcn_mov_dpp((int)w.hi, 0x100 + LANES, 0xf, 0xf, true)})))
  NT_UP(8);
  NT_UP(4);
  NT_UP(2);
  NT_UP(1);
#undef NT_UP
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

// A value that another block will read goes through this XCD's L2 to memory, and the count follows it.  Both are relaxed on purpose, since
// a release would write back all of the L2 in every block: on gfx950 a store of agent scope is written through, s_waitcnt vmcnt(0) returns
// once it has reached the memory that all XCDs share, and the same wave counts behind it.  The last one's acquire drops what its caches hold.
// Nobody waits for another block.
template <class T>
__device__ inline void hand_over(T value, double* to) {
  if ((threadIdx.x & 63) == 0) {
    __hip_atomic_store((uint64_t*)to, __builtin_bit_cast(uint64_t, value), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
}
// Counts; true in the whole wave for the last of n, which puts the counter back.
__device__ inline bool last_of(uint32_t* counter, uint32_t n) {
  uint32_t before = 0;
  if ((threadIdx.x & 63) == 0) before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if ((uint32_t)__builtin_amdgcn_readfirstlane((int)before) != n - 1) return false;
  if ((threadIdx.x & 63) == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}
// total of n values that were handed over, in the first lane
template <class K>
__device__ inline typename K::T total_of(const double* from, uint32_t n) {
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
  typename K::T t = 0;
#pragma unroll 4
  for (uint32_t i = threadIdx.x & 63; i < n; i += 64) t = K::join(t, __builtin_bit_cast(typename K::T, from[i]));
  return wave_total<K>(t);
}
// A block's part of group g, which its lanes hold: stored in its slot, counted, and added up by whoever comes last.  Few slots are counted in
// slabs but added up at once: 1M elements 7.1 -> 6.2 us, as a slab's sum costs another trip to memory and back.  A block that meets
// several groups alternates `half`, so that the first wave has read one half before another wave writes it again.
template <class K, int THREADS>
__device__ inline void end_part(const NormOut& o, uint32_t block, uint32_t g, typename K::T acc, int half = 0) {
  __shared__ typename K::T red[2][THREADS / 64];
  acc = wave_total<K>(acc);
  if ((threadIdx.x & 63) == 0) red[half][threadIdx.x >> 6] = acc;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  typename K::T total = red[half][0];
#pragma unroll
  for (int w = 1; w < THREADS / 64; ++w) total = K::join(total, red[half][w]);
  const Group NT_CONST* group = constant(o.cut.groups) + g;
  const uint32_t slot0 = group->slot0, slots = group->slots, slab0 = group->slab0;
  if (slots > 1) {
    const uint32_t slot = o.cut.run ? block - group->item0 / o.cut.run : (block - group->item0) & (o.cut.blocks - 1);
    const uint32_t slab = slot >> o.cut.shift;
    const uint32_t slabs = ((slots - 1) >> o.cut.shift) + 1, first = slab << o.cut.shift;
    const uint32_t here = slots - first < (1u << o.cut.shift) ? slots - first : 1u << o.cut.shift;
    uint32_t* const counters = o.cut.counters;
    hand_over(total, o.cut.partials + slot0 + slot);
    if (here > 1 && !last_of(counters + (size_t)NT_COUNTER_WORDS * (slab0 + slab), here)) return;
    uint32_t* const of_group = counters + (size_t)NT_COUNTER_WORDS * (o.cut.nslabs + g);
    if (slots <= NT_FEW_SLOTS) {
      if (slabs > 1 && !last_of(of_group, slabs)) return;
      total = total_of<K>(o.cut.partials + slot0, slots);
    } else {
      hand_over(total_of<K>(o.cut.partials + slot0 + first, here), o.cut.sums + slab0 + slab);
      if (!last_of(of_group, slabs)) return;
      total = total_of<K>(o.cut.sums + slab0, slabs);
    }
  }
  if (threadIdx.x == 0) write_norm<K>(o, g, group->elements, total);
}

// ---------------------------------------------------------------------------------------------
// Kernels
// ---------------------------------------------------------------------------------------------
struct ListArgs {
  const Shape* shapes;
  const Item* items;
  uint32_t item0;       // of this launch
};

// Values of a type known at compile time, N of them in N * size bytes.
template <int DTYPE, int N>
struct Vec {
  static constexpr int SIZE = DTYPE == NT_F32 ? 4 : 2, WORDS = N * SIZE / 4;
  typedef uint32_t raw_t __attribute__((ext_vector_type(WORDS)));
  typedef uint32_t any_t __attribute__((ext_vector_type(WORDS), aligned(SIZE)));
  template <bool STREAM = false>
  __device__ static inline raw_t load(const char NT_GLOBAL* p) {
    if constexpr (STREAM) return __builtin_nontemporal_load((const any_t NT_GLOBAL*)p);
    return *(const any_t NT_GLOBAL*)p;
  }
  template <bool STREAM = false>
  __device__ static inline void store(char NT_GLOBAL* p, const raw_t& r) {
    if constexpr (STREAM)
      __builtin_nontemporal_store((any_t)r, (any_t NT_GLOBAL*)p);
    else
      *(any_t NT_GLOBAL*)p = r;
  }
  __device__ static inline float value(const raw_t& r, int e) {
    if constexpr (DTYPE == NT_F32) return __builtin_bit_cast(float, (uint32_t)r[e]);
    const uint32_t w = r[e >> 1];
    if constexpr (DTYPE == NT_BF16) return __builtin_bit_cast(float, (e & 1) ? (w & 0xffff0000u) : (w << 16));
    return (float)__builtin_bit_cast(_Float16, (uint16_t)((e & 1) ? w >> 16 : w));
  }
  __device__ static inline void put(raw_t& r, int e, float x) {   // rounded to nearest even; elements in ascending order
    if constexpr (DTYPE == NT_F32) {
      r[e] = __builtin_bit_cast(uint32_t, x);
    } else {
      uint16_t h;
      if constexpr (DTYPE == NT_BF16)
        h = __builtin_bit_cast(uint16_t, (__bf16)x);
      else
        h = __builtin_bit_cast(uint16_t, (_Float16)x);
      r[e >> 1] = (e & 1) ? (r[e >> 1] | (uint32_t)h << 16) : h;
    }
  }
};
template <int D>
struct Dtype {
  static constexpr int value = D;
};
// BODY(Dtype<the type>); the same for the whole block
template <class BODY>
__device__ inline void by_type(int dtype, BODY body) {
  if (dtype == NT_F32)
    body(Dtype<NT_F32>());
  else if (dtype == NT_BF16)
    body(Dtype<NT_BF16>());
  else
    body(Dtype<NT_F16>());
}

// n elements from p on, in 16-byte loads of which NT_NORM_FLIGHT are in flight; what is left over one by one.
template <class K, int DTYPE, bool STREAM>
__device__ inline void norm_flat(const char NT_GLOBAL* p, uint32_t n, typename K::T& total) {
  constexpr int PER = DTYPE == NT_F32 ? 4 : 8, FLIGHT = NT_NORM_FLIGHT;
  typedef Vec<DTYPE, PER> V;
  typename K::T acc[2] = {total, 0};
  auto take = [&](const typename V::raw_t& r) {
#pragma unroll
    for (int e = 0; e < PER; ++e) K::add(acc[e & 1], V::value(r, e));
  };
  const uint32_t whole = n / PER;
  uint32_t i = threadIdx.x;
  for (; i + (FLIGHT - 1) * NT_NORM_THREADS < whole; i += FLIGHT * NT_NORM_THREADS) {
    typename V::raw_t r[FLIGHT];
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) r[k] = V::template load<STREAM>(p + 16 * (i + k * NT_NORM_THREADS));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) take(r[k]);
  }
  if (i < whole) {
    typename V::raw_t r[FLIGHT - 1];
#pragma unroll
    for (int k = 0; k < FLIGHT - 1; ++k) {
      r[k] = typename V::raw_t{};
      if (i + k * NT_NORM_THREADS < whole) r[k] = V::template load<STREAM>(p + 16 * (i + k * NT_NORM_THREADS));
    }
#pragma unroll
    for (int k = 0; k < FLIGHT - 1; ++k) take(r[k]);
  }
  if (threadIdx.x < n % PER) {
    const uint32_t at = whole * PER + threadIdx.x;
    if constexpr (DTYPE == NT_F32)
      K::add(acc[0], __builtin_bit_cast(float, ((const uint32_t NT_GLOBAL*)p)[at]));
    else
      K::add(acc[0], Vec<DTYPE, 2>::value(typename Vec<DTYPE, 2>::raw_t{((const uint16_t NT_GLOBAL*)p)[at]}, 0));
  }
  total = K::join(acc[0], acc[1]);
}
// An item of a tensor with rows, four elements at a time.
template <class K, int DTYPE>
__device__ inline void norm_rows(const nt_tensor NT_CONST* t, const Item& it, const Shape* shapes, int level, uint32_t size,
                                 typename K::T& acc) {
  constexpr int FLIGHT = 8;
  Walk<NT_NORM_THREADS> at(it, shapes, level, size);
  Place<DTYPE> place(t, at);
  for (uint32_t done = 0; done < at.rows * at.quads; done += FLIGHT * NT_NORM_THREADS) {
    u32x4 x[FLIGHT];
    int n[FLIGHT];
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) {
      n[k] = at.here();
      x[k] = place.load(at, n[k]);
      at.step();
      place.step(at);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) {
      const f32x4 v = values(DTYPE, place.settle(at, x[k], n[k]));   // zeros, which add nothing, where there are no elements
#pragma unroll
      for (int e = 0; e < 4; ++e) K::add(acc, v[e]);
    }
  }
}
// A block that walks every blocks-th item: the chip as a whole reads a long list from front to back, and neither the way to an item's address
// nor the end of a part is met more often than need be.  The next item's record and address are fetched beside this one's elements.
template <class K, bool STREAM>
__global__ __launch_bounds__(NT_NORM_THREADS) void k_norm(ListArgs a, const nt_tensor* list, int level, NormOut o) {
  const uint32_t size = level ? NT_LONG_ITEM : NT_ITEM;
  const uint32_t step = o.cut.run ? 1 : o.cut.blocks;
  uint32_t item = o.cut.run ? blockIdx.x * o.cut.run : blockIdx.x;
  const uint32_t end = o.cut.run && o.cut.nitems - item > o.cut.run ? item + o.cut.run : o.cut.nitems;
  Item it = item_at(a.items, item);
  const nt_tensor NT_CONST* t = constant(list) + it.tensor;
  const char NT_GLOBAL* data = nullptr;
  int dtype = NT_F32, half = 0;
  if (it.count) {
    data = (const char NT_GLOBAL*)t->data;
    dtype = t->dtype;
  }
  typename K::T acc = 0;
  for (;;) {
    const uint32_t next = item + step;
    const bool more = next < end;
    const char NT_GLOBAL* const from = data + ((uint64_t)it.idx * size << size_shift(dtype));
    const int type = dtype;
    Item nx = it;
    const nt_tensor NT_CONST* nt = t;
    if (more) {
      nx = item_at(a.items, next);
      nt = constant(list) + nx.tensor;
      if (nx.count) {
        data = (const char NT_GLOBAL*)nt->data;
        dtype = nt->dtype;
      }
    }
    if (it.count & NT_ROWS)
      by_type(type, [&](auto d) { norm_rows<K, decltype(d)::value>(t, it, a.shapes, level, size, acc); });
    else if (it.count)
      by_type(type, [&](auto d) { norm_flat<K, decltype(d)::value, STREAM>(from, it.count, acc); });
    if (!more || nx.group != it.group) {
      end_part<K, NT_NORM_THREADS>(o, blockIdx.x, it.group, acc, half);
      if (!more) return;
      half ^= 1;
      acc = 0;
    }
    item = next;
    it = nx;
    t = nt;
  }
}

struct UpdateArgs {
  const nt_tensor* dst;
  const nt_tensor* src;
  const nt_norm* norms;   // of src, may be null
  double scale;
  float beta;
  int in_place;           // dst is src, and nothing is to be done where the factor is 1
};
// What of a call goes past the caches: nothing, what it writes (and reads there), or what it only reads too.
enum { KEEP = 0, STREAM_WRITTEN = 1, STREAM_ALL = 2 };

// A whole item of a tensor of one row: all loads, then all stores.
template <bool READ, class K, int STREAM, int THREADS, int XT, int YT, class ACC>
__device__ inline void update_flat(const char NT_GLOBAL* x, char NT_GLOBAL* y, float scale, float beta, ACC& acc) {
  constexpr int PER = XT != NT_F32 && YT != NT_F32 ? 8 : 4, SWEEPS = NT_ITEM / (PER * THREADS);
  static_assert(SWEEPS * PER * THREADS == NT_ITEM, "an item is whole sweeps");
  typedef Vec<XT, PER> X;
  typedef Vec<YT, PER> Y;
  typename X::raw_t xr[SWEEPS];
  typename Y::raw_t yr[SWEEPS];
  const uint32_t lane = PER * threadIdx.x;
#pragma unroll
  for (int k = 0; k < SWEEPS; ++k) {
    xr[k] = X::template load<STREAM == STREAM_ALL>(x + X::SIZE * (lane + k * PER * THREADS));
    if constexpr (READ) yr[k] = Y::template load<STREAM != KEEP>(y + Y::SIZE * (lane + k * PER * THREADS));
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int k = 0; k < SWEEPS; ++k) {
    typename Y::raw_t z;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const float v = X::value(xr[k], e);
      Y::put(z, e, READ ? __builtin_fmaf(scale, v, beta * Y::value(yr[k], e)) : scale * v);
    }
    Y::template store<STREAM != KEEP>(y + Y::SIZE * (lane + k * PER * THREADS), z);
    if constexpr (!__is_same(K, void)) {
#pragma unroll
      for (int e = 0; e < PER; ++e) K::add(acc, Y::value(z, e));
    }
  }
}
// Any other item.
template <bool READ, class K, int THREADS, int XT, int YT, class ACC>
__device__ inline void update_walk(const nt_tensor NT_CONST* x, const nt_tensor NT_CONST* y, const Item& it, const Shape* shapes, float scale,
                                   float beta, ACC& acc) {
  constexpr int SWEEPS = NT_ITEM / (4 * THREADS);
  Walk<THREADS> at(it, shapes, 0, NT_ITEM);
  Place<XT> from(x, at);
  Place<YT> to(y, at);
  u32x4 xr[SWEEPS], yr[SWEEPS];
  uint64_t off[SWEEPS];
  int n[SWEEPS];
#pragma unroll
  for (int k = 0; k < SWEEPS; ++k) {
    n[k] = at.here();
    off[k] = to.off;
    xr[k] = from.load(at, n[k]);
    if constexpr (READ) yr[k] = to.load(at, n[k]);
    at.step();
    from.step(at);
    to.step(at);
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int k = 0; k < SWEEPS; ++k) {
    const f32x4 xv = values(XT, from.settle(at, xr[k], n[k]));
    f32x4 yv = {0.f, 0.f, 0.f, 0.f}, z;
    if constexpr (READ) yv = values(YT, to.settle(at, yr[k], n[k]));
#pragma unroll
    for (int e = 0; e < 4; ++e) z[e] = READ ? __builtin_fmaf(scale, xv[e], beta * yv[e]) : scale * xv[e];
    const u32x4 zr = rounded(YT, z);
    store_n(YT, to.base + off[k], zr, n[k]);
    if constexpr (!__is_same(K, void)) {
      const f32x4 v = values(YT, zr);
#pragma unroll
      for (int e = 0; e < 4; ++e) K::add(acc, e < n[k] ? v[e] : 0.f);
    }
  }
}
template <class K>
struct Partial {
  typedef typename K::T T;
};
template <>
struct Partial<void> {
  typedef int T;
};
// dst <- beta dst + scale factor src
template <bool READ, class K, int STREAM, int THREADS>
__global__ __launch_bounds__(THREADS) void k_update(ListArgs a, UpdateArgs u, NormOut o) {
  const uint32_t item = a.item0 + blockIdx.x;
  const Item it = item_at(a.items, item);
  typename Partial<K>::T acc = 0;
  if (it.count) {
    const nt_tensor NT_CONST* x = constant(u.src) + it.tensor;
    const nt_tensor NT_CONST* y = constant(u.dst) + it.tensor;
    float scale = (float)u.scale;
    if (u.norms) {
      const float factor = (constant(u.norms) + it.group)->factor;
      if (u.in_place && factor == 1.f) return;
      scale = (float)(u.scale * (double)factor);
    }
    const int xt = x->dtype, yt = y->dtype;
    if (it.count == NT_ITEM) {
      const uint64_t at = (uint64_t)it.idx * NT_ITEM;
      const char NT_GLOBAL* from = (const char NT_GLOBAL*)x->data + (at << size_shift(xt));
      char NT_GLOBAL* to = (char NT_GLOBAL*)y->data + (at << size_shift(yt));
      by_type(xt, [&](auto dx) {
        by_type(yt, [&](auto dy) { update_flat<READ, K, STREAM, THREADS, decltype(dx)::value, decltype(dy)::value>(from, to, scale, u.beta, acc); });
      });
    } else {
      by_type(xt, [&](auto dx) {
        by_type(yt, [&](auto dy) { update_walk<READ, K, THREADS, decltype(dx)::value, decltype(dy)::value>(x, y, it, a.shapes, scale, u.beta, acc); });
      });
    }
  }
  if constexpr (!__is_same(K, void)) end_part<K, THREADS>(o, item, it.group, acc);
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
// A whole item of a tensor of one row.
template <int GT, int STREAM, int THREADS>
__device__ inline void adamw_flat(const AdamwArgs& u, const char NT_GLOBAL* gp, char NT_GLOBAL* wp, char NT_GLOBAL* mp, char NT_GLOBAL* vp,
                                  char NT_GLOBAL* cp, int copy_type, float scale) {
  constexpr int SWEEPS = NT_ITEM / (4 * THREADS);
  constexpr bool S = STREAM != KEEP;
  typedef Vec<GT, 4> G;
  typedef Vec<NT_F32, 4> F;
  typename G::raw_t g[SWEEPS];
  u32x4 w[SWEEPS], m[SWEEPS], v[SWEEPS];
  const uint32_t lane = 4 * threadIdx.x;
#pragma unroll
  for (int k = 0; k < SWEEPS; ++k) {
    const uint32_t at = lane + k * 4 * THREADS;
    g[k] = G::template load<STREAM == STREAM_ALL>(gp + G::SIZE * at);
    w[k] = F::template load<S>(wp + 4 * at);
    m[k] = F::template load<S>(mp + 4 * at);
    v[k] = F::template load<S>(vp + 4 * at);
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int k = 0; k < SWEEPS; ++k) {
    const uint32_t at = lane + k * 4 * THREADS;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float we = F::value(w[k], e), me = F::value(m[k], e), ve = F::value(v[k], e);
      adamw_element(u, scale * G::value(g[k], e), we, me, ve);
      F::put(w[k], e, we);
      F::put(m[k], e, me);
      F::put(v[k], e, ve);
    }
    F::template store<S>(wp + 4 * at, w[k]);
    F::template store<S>(mp + 4 * at, m[k]);
    F::template store<S>(vp + 4 * at, v[k]);
    // the copy is what the next forward pass reads first
    if (cp) store4(copy_type, cp + ((uint64_t)at << size_shift(copy_type)), rounded(copy_type, __builtin_bit_cast(f32x4, w[k])));
  }
}
// Any other item.
template <int GT, int THREADS>
__device__ inline void adamw_walk(const AdamwArgs& u, const nt_tensor NT_CONST* gt, const nt_tensor NT_CONST* wt, const nt_tensor NT_CONST* mt,
                                  const nt_tensor NT_CONST* vt, const nt_tensor NT_CONST* ct, Walk<THREADS> at, float scale) {
  constexpr int SWEEPS = NT_ITEM / (4 * THREADS);
  Place<GT> gp(gt, at);
  Place<NT_F32> wp(wt, at), mp(mt, at), vp(vt, at);
  u32x4 gr[SWEEPS], wr[SWEEPS], mr[SWEEPS], vr[SWEEPS];
  uint64_t wo[SWEEPS], mo[SWEEPS], vo[SWEEPS];
  uint32_t r[SWEEPS], c[SWEEPS];
  int n[SWEEPS];
#pragma unroll
  for (int k = 0; k < SWEEPS; ++k) {
    n[k] = at.here();
    r[k] = at.r;
    c[k] = at.c;
    wo[k] = wp.off;
    mo[k] = mp.off;
    vo[k] = vp.off;
    gr[k] = gp.load(at, n[k]);
    wr[k] = wp.load(at, n[k]);
    mr[k] = mp.load(at, n[k]);
    vr[k] = vp.load(at, n[k]);
    at.step();
    gp.step(at);
    wp.step(at);
    mp.step(at);
    vp.step(at);
  }
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int k = 0; k < SWEEPS; ++k) {
    if (n[k] == 0) continue;
    const f32x4 g = values(GT, gp.settle(at, gr[k], n[k]));
    f32x4 w = values(NT_F32, wp.settle(at, wr[k], n[k])), m = values(NT_F32, mp.settle(at, mr[k], n[k])),
          v = values(NT_F32, vp.settle(at, vr[k], n[k]));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float we = w[e], me = m[e], ve = v[e];
      adamw_element(u, scale * g[e], we, me, ve);
      w[e] = we;
      m[e] = me;
      v[e] = ve;
    }
    store_n(NT_F32, wp.base + wo[k], __builtin_bit_cast(u32x4, w), n[k]);
    store_n(NT_F32, mp.base + mo[k], __builtin_bit_cast(u32x4, m), n[k]);
    store_n(NT_F32, vp.base + vo[k], __builtin_bit_cast(u32x4, v), n[k]);
    if (ct) {
      const int type = ct->dtype;
      const uint64_t at_copy = (at.row0 + r[k]) * ct->ld + at.col0 + 4 * c[k];
      store_n(type, (char NT_GLOBAL*)ct->data + (at_copy << size_shift(type)), rounded(type, w), n[k]);
    }
  }
}
template <int STREAM, int THREADS>
__global__ __launch_bounds__(THREADS) void k_adamw(ListArgs a, AdamwArgs u) {
  const Item it = item_at(a.items, a.item0 + blockIdx.x);
  if (!it.count) return;
  const nt_tensor NT_CONST* gt = constant(u.grads) + it.tensor;
  const nt_tensor NT_CONST* wt = constant(u.w) + it.tensor;
  const nt_tensor NT_CONST* mt = constant(u.m) + it.tensor;
  const nt_tensor NT_CONST* vt = constant(u.v) + it.tensor;
  const nt_tensor NT_CONST* ct = u.copy ? constant(u.copy) + it.tensor : nullptr;
  float scale = (float)u.grad_scale;
  if (u.norms) {
    const nt_norm NT_CONST* n = constant(u.norms) + it.group;
    if ((u.flags & NT_SKIP_NONFINITE) && (n->status & NT_STATUS_NONFINITE)) return;
    scale = (float)u.grad_scale * n->factor;
  }
  const int dtype = gt->dtype;
  if (it.count & NT_ROWS) {
    by_type(dtype, [&](auto d) {
      adamw_walk<decltype(d)::value, THREADS>(u, gt, wt, mt, vt, ct, Walk<THREADS>(it, a.shapes, 0, NT_ITEM), scale);
    });
    return;
  }
  // In lists that stream, items begin where w has a whole line of memory, and what lies before the first one's begin goes with it: tensors one
  // right behind the other, 137.5M elements 757 -> 714 us.  In short lists it costs more than it gives (1M elements 12.7 -> 13.5).
  const int64_t n = wt->cols;
  const uint32_t ahead = STREAM != KEEP && n > NT_ITEM ? (0u - (uint32_t)((uintptr_t)wt->data >> 2)) % 32 : 0;
  const int64_t begin = (int64_t)it.idx * NT_ITEM + ahead;
  const int64_t count = n - begin < NT_ITEM ? n - begin : NT_ITEM;
  for (bool before = STREAM != KEEP && it.idx == 0 && ahead > 0;; before = false) {
    if (before || count < NT_ITEM) {
      if (before || count > 0)
        by_type(dtype, [&](auto d) {
          adamw_walk<decltype(d)::value, THREADS>(u, gt, wt, mt, vt, ct, Walk<THREADS>(before ? 0 : begin, before ? ahead : (uint32_t)count), scale);
        });
    } else {
      const int copy_type = ct ? ct->dtype : 0;
      const char NT_GLOBAL* gp = (const char NT_GLOBAL*)gt->data + (begin << size_shift(dtype));
      char NT_GLOBAL* cp = ct ? (char NT_GLOBAL*)ct->data + (begin << size_shift(copy_type)) : nullptr;
      by_type(dtype, [&](auto d) {
        adamw_flat<decltype(d)::value, STREAM, THREADS>(u, gp, (char NT_GLOBAL*)wt->data + 4 * begin, (char NT_GLOBAL*)mt->data + 4 * begin,
                                                       (char NT_GLOBAL*)vt->data + 4 * begin, cp, copy_type, scale);
      });
    }
    if (!before) break;
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
Cut cut_of(const nt_plan& p, const Layout& l, int k) {
  char* const b = (char*)p.image;
  return {(const Item*)(b + l.items[k]), (const Group*)(b + l.groups[k]), (uint32_t*)(b + l.counters[k]), (double*)(b + l.partials[k]),
          (double*)(b + l.sums[k]), p.items[k], p.slabs[k], NT_LONG_BLOCKS, run_of(p, k), slab_shift(p.slots[k])};
}

// Where a tensor's elements lie, in bytes: rows of `width`, `stride` apart (dense tensors: one row).
struct Span {
  uint64_t begin, end, rows, width, stride;
};
// whether b's row from `at` on, `width` bytes, has bytes of a; at >= a.begin
bool meets(const Span& a, uint64_t at, uint64_t width) {
  const uint64_t row = (at - a.begin) / a.stride, in = (at - a.begin) % a.stride;
  return row < a.rows && (in < a.width || (row + 1 < a.rows && a.stride - in < width));
}
// a.begin <= b.begin < a.end
bool share(const Span& a, const Span& b) {
  if (a.rows == 1) return true;
  // rows that are as far apart as a's lie in each of a's as b's first does; others are looked at one by one, as far as a reaches
  const uint64_t looked_at = a.stride == b.stride ? 1 : b.rows;
  for (uint64_t r = 0; r < looked_at && b.begin + r * b.stride < a.end; ++r)
    if (meets(a, b.begin + r * b.stride, b.width)) return true;
  return false;
}
// whether two of n spans, in ascending order of begin, share memory; open: room for n
bool any_share(const Span* spans, int32_t n, int32_t* open) {
  int32_t nopen = 0;   // those that reach to the present one or beyond it
  for (int32_t i = 0; i < n; ++i) {
    int32_t kept = 0;
    for (int32_t j = 0; j < nopen; ++j)
      if (spans[open[j]].end > spans[i].begin) {
        if (share(spans[open[j]], spans[i])) return true;
        open[kept++] = open[j];
      }
    open[kept++] = i;
    nopen = kept;
  }
  return false;
}

int check_plan(const nt_plan* p) {
  if (!p || p->magic != NT_PLAN_MAGIC || !p->image || ((uintptr_t)p->image & 15u) || p->groups < 1 || p->tensors < 0) return NT_ERR_BAD_ARG;
  return NT_OK;
}
int check_list(const nt_plan& p, const nt_tensor* list) {
  return (p.tensors > 0 && !list) || misaligned8(list) ? NT_ERR_BAD_ARG : NT_OK;
}
// the kernels multiply in fp32, where a larger double would be infinite and make NaN of a zero
bool finite_in_fp32(double x) { return std::isfinite((float)x); }
int check_norm(int32_t kind, double max_norm, double grad_scale, const nt_norm* norms) {
  if ((kind != NT_NORM_L2 && kind != NT_NORM_MAX) || std::isnan(max_norm) || !finite_in_fp32(grad_scale)) return NT_ERR_BAD_ARG;
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

template <bool READ, int STREAM>
int enqueue_update(const nt_plan& p, const Layout& l, const UpdateArgs& u, int kind, const NormOut& o, hipStream_t st) {
  ListArgs a = {(const Shape*)((char*)p.image + l.shapes), cut_of(p, l, 0).items, 0};
  return in_launches(p.items[0], NT_MOST_BLOCKS, [&](uint32_t at, uint32_t n) {
    a.item0 = at;
    if (!o.norms)
      hipLaunchKernelGGL((k_update<READ, void, STREAM, NT_UPDATE_THREADS>), dim3(n), dim3(NT_UPDATE_THREADS), 0, st, a, u, o);
    else if (kind == NT_NORM_L2)
      hipLaunchKernelGGL((k_update<READ, Square, STREAM, NT_TOTAL_THREADS>), dim3(n), dim3(NT_TOTAL_THREADS), 0, st, a, u, o);
    else
      hipLaunchKernelGGL((k_update<READ, Largest, STREAM, NT_TOTAL_THREADS>), dim3(n), dim3(NT_TOTAL_THREADS), 0, st, a, u, o);
  });
}
template <bool READ>
int enqueue_update(const nt_plan& p, const Layout& l, const UpdateArgs& u, int kind, const NormOut& o, hipStream_t st) {
  if (p.elements < NT_STREAM_UPDATE) return enqueue_update<READ, KEEP>(p, l, u, kind, o, st);
  return p.elements < NT_STREAM_READ ? enqueue_update<READ, STREAM_WRITTEN>(p, l, u, kind, o, st)
                                     : enqueue_update<READ, STREAM_ALL>(p, l, u, kind, o, st);
}

}  // namespace

extern "C" {

int normtest_plan_make(const nt_tensor* tensors, int32_t N, int32_t G, nt_plan* plan, void* image, size_t image_bytes) {
  if (!plan || N < 0 || G < 1 || (N > 0 && !tensors) || misaligned8(image)) return NT_ERR_BAD_ARG;
  nt_plan p;
  std::memset(&p, 0, sizeof(p));
  int64_t elements = 0, in_rows = 0;
  for (int32_t i = 0; i < N; ++i) {
    const nt_tensor& t = tensors[i];
    if (t.rows < 0 || t.cols < 0 || t.group < 0 || t.group >= G) return NT_ERR_BAD_ARG;
    if (t.rows > 1 && t.ld < t.cols) return NT_ERR_BAD_ARG;
    int64_t n;
    if (__builtin_mul_overflow(t.rows, t.cols, &n) || __builtin_add_overflow(elements, n, &elements) || elements > (1ll << 43))
      return NT_ERR_TOO_LARGE;
    if (t.rows > 1) in_rows += n;
  }
  p.elements = elements;
  p.flags = in_rows > elements / 2 ? NT_PLAN_ROWS : 0;
  p.tensors = N;
  p.groups = G;
  p.magic = NT_PLAN_MAGIC;
  const int cuts = elements >= NT_LONG_LIST || G > (int32_t)NT_MOST_BLOCKS ? 2 : 1;

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

  auto items_of = [&](int32_t g, int k) {   // at least the empty one
    int64_t n = 0;
    for (int64_t j = group_begin(g); j < first[g]; ++j) n += pieces_of(tensors[order[j]].rows, tensors[order[j]].cols, SIZES[k]).n;
    return n ? n : 1;
  };
  for (int k = 0; k < cuts; ++k) {
    int64_t items = 0, slots = 0, slabs = 0;
    for (int32_t g = 0; g < G; ++g) {
      items += items_of(g, k);
      if (items > (1ll << 31) - 1) return NT_ERR_TOO_LARGE;
    }
    p.items[k] = (uint32_t)items;
    for (int32_t g = 0, at = 0; g < G; at += items_of(g, k), ++g) slots += slots_of(run_of(p, k), at, items_of(g, k));
    const int shift = slab_shift((uint32_t)slots);
    for (int32_t g = 0, at = 0; g < G; at += items_of(g, k), ++g) slabs += ceil_div(slots_of(run_of(p, k), at, items_of(g, k)), 1ll << shift);
    p.slots[k] = (uint32_t)slots;
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
        const Pieces c = pieces_of(s.rows, s.cols, SIZES[k]);
        s.per_row[k] = c.per_row;
        s.rows_per_item[k] = c.rows_per_item;
      }
    }
    for (int k = 0; k < cuts; ++k) {
      Item* const items = (Item*)(b + l.items[k]);
      Group* const groups = (Group*)(b + l.groups[k]);
      const int shift = slab_shift(p.slots[k]);
      uint32_t item = 0, slot = 0, slab = 0;
      for (int32_t g = 0; g < G; ++g) {
        const uint32_t begin = item;
        int64_t held_elements = 0;
        for (int64_t j = group_begin(g); j < first[g]; ++j) {
          const nt_tensor& t = tensors[order[j]];
          held_elements += t.rows * t.cols;
          const Pieces c = pieces_of(t.rows, t.cols, SIZES[k]);
          for (int64_t idx = 0; idx < c.n; ++idx) {
            int64_t count = 1;   // of a part of a row
            if (t.rows == 1)
              count = t.cols - idx * SIZES[k] < SIZES[k] ? t.cols - idx * SIZES[k] : SIZES[k];
            else if (!c.per_row)
              count = t.rows - idx * c.rows_per_item < c.rows_per_item ? t.rows - idx * c.rows_per_item : c.rows_per_item;
            items[item++] = {(uint32_t)order[j], (uint32_t)idx, (uint32_t)g, (uint32_t)count | (t.rows == 1 ? 0u : NT_ROWS)};
          }
        }
        if (item == begin) items[item++] = {0, 0, (uint32_t)g, 0};
        const uint32_t slots = (uint32_t)slots_of(run_of(p, k), begin, item - begin);
        groups[g] = {begin, slot, slots, slab, held_elements, 0};
        slot += slots;
        slab += (uint32_t)ceil_div(slots, 1ll << shift);
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
  if (N < 2) return NT_OK;
  const std::unique_ptr<Span[]> spans(new (std::nothrow) Span[N]);
  const std::unique_ptr<int32_t[]> open(new (std::nothrow) int32_t[N]);
  if (!spans || !open) return NT_ERR_TOO_LARGE;
  int32_t n = 0;
  for (int32_t i = 0; i < N; ++i) {
    const nt_tensor& t = list[i];
    if (t.rows == 0 || t.cols == 0) continue;
    Span s = {(uintptr_t)t.data, 0, (uint64_t)t.rows, (uint64_t)t.cols, (uint64_t)(t.rows > 1 ? t.ld : t.cols)};
    if (s.width == s.stride) {
      if (__builtin_mul_overflow(s.rows, s.width, &s.width)) return NT_ERR_BAD_ARG;
      s.rows = 1;
      s.stride = s.width;
    }
    uint64_t size = 0;   // from the first element to the last
    if (__builtin_mul_overflow(s.width, 1ull << size_shift(t.dtype), &s.width) || __builtin_mul_overflow(s.stride, 1ull << size_shift(t.dtype), &s.stride) ||
        __builtin_mul_overflow(s.rows - 1, s.stride, &size) || __builtin_add_overflow(size, s.width, &size) ||
        __builtin_add_overflow(s.begin, size, &s.end))
      return NT_ERR_BAD_ARG;
    spans[n++] = s;
  }
  std::sort(spans.get(), spans.get() + n, [](const Span& a, const Span& b) { return a.begin < b.begin; });
  return any_share(spans.get(), n, open.get()) ? NT_ERR_SHARED_MEMORY : NT_OK;
}

int normtest_grad_norm(const nt_plan* plan, const nt_tensor* grads, int32_t kind, double max_norm, double grad_scale, nt_norm* norms,
                       void* hip_stream) {
  int rc = check_plan(plan);
  if (rc == NT_OK) rc = check_list(*plan, grads);
  if (rc == NT_OK) rc = check_norm(kind, max_norm, grad_scale, norms);
  if (rc != NT_OK) return rc;
  const Layout l = layout_of(*plan);
  const int k = plan->items[1] ? 1 : 0;
  const NormOut o = {cut_of(*plan, l, k), max_norm, grad_scale, norms};
  const ListArgs a = {(const Shape*)((char*)plan->image + l.shapes), o.cut.items, 0};
  const uint32_t blocks = o.cut.run ? (o.cut.nitems - 1) / o.cut.run + 1 : o.cut.nitems < o.cut.blocks ? o.cut.nitems : o.cut.blocks;
  const bool stream = plan->elements >= NT_STREAM_READ;
  auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(blocks), dim3(NT_NORM_THREADS), 0, (hipStream_t)hip_stream, a, grads, k, o);
    return hip_code(hipGetLastError());
  };
  if (kind == NT_NORM_L2) return stream ? launch(k_norm<Square, true>) : launch(k_norm<Square, false>);
  return stream ? launch(k_norm<Largest, true>) : launch(k_norm<Largest, false>);
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
  if (!finite_in_fp32(beta) || !finite_in_fp32(scale) || misaligned8(src_norms)) return NT_ERR_BAD_ARG;
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
  if (!hyper || !finite_in_fp32(grad_scale) || misaligned8(copy) || misaligned8(norms) || (flags & ~(uint32_t)NT_SKIP_NONFINITE) ||
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
  if (!std::isfinite(u.decay) || !std::isfinite(u.step_size)) return NT_ERR_BAD_ARG;
  const Layout l = layout_of(*plan);
  const Cut cut = cut_of(*plan, l, 0);
  ListArgs a = {(const Shape*)((char*)plan->image + l.shapes), cut.items, 0};
  hipStream_t st = (hipStream_t)hip_stream;
  const bool step = plan->elements >= NT_STEP_LIST && !(plan->flags & NT_PLAN_ROWS);
  return in_launches(plan->items[0], step ? NT_STEP_ITEMS : NT_MOST_BLOCKS, [&](uint32_t at, uint32_t n) {
    a.item0 = at;
    auto launch = [&](auto kernel, int threads, int lds) { hipLaunchKernelGGL(kernel, dim3(n), dim3(threads), lds, st, a, u); };
    if (plan->elements < NT_STREAM_ADAMW)
      launch(k_adamw<KEEP, NT_ADAMW_THREADS>, NT_ADAMW_THREADS, 0);
    else if (!step && plan->elements < NT_STREAM_READ)
      launch(k_adamw<STREAM_WRITTEN, NT_ADAMW_THREADS>, NT_ADAMW_THREADS, 0);
    else if (!step)
      launch(k_adamw<STREAM_ALL, NT_ADAMW_THREADS>, NT_ADAMW_THREADS, 0);
    else if (plan->elements < NT_STREAM_READ)
      launch(k_adamw<STREAM_WRITTEN, NT_STEP_THREADS>, NT_STEP_THREADS, NT_STEP_LDS);
    else
      launch(k_adamw<STREAM_ALL, NT_STEP_THREADS>, NT_STEP_THREADS, NT_STEP_LDS);
  });
}

}  // extern "C"
