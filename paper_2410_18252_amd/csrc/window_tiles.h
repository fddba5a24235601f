// Tiles of rows in LDS for the windowed attention's matrix products, and who sees whom.
#pragma once
#include "window.h"

typedef short s16x4 __attribute__((ext_vector_type(4)));

// A tile keeps rows of HD 16-bit values one behind the other; what varies is where a row's 16-byte chunk c sits: at c ^ chunk_swap(row).
// LDS has 64 banks, so 256 bytes in a row of addresses never conflict.  Two kinds of read have to be spread: fragments with the row
// in the lane (16 lanes read chunk c of 16 rows) and transposed ones (32 lanes read 64 bytes of four rows 4 i .. 4 i + 3).  Rows whose
// start falls on the same place modulo 256 bytes get different low bits of the chunk, neighbours first the bit that changes the 64 bytes.
template <int HD> __host__ __device__ constexpr int chunk_swap(int row) {
  if constexpr (HD % 128 == 0) return ((row & 3) << 2) | ((row >> 2) & 3);
  else if constexpr (HD % 64 == 0) return ((row & 2) << 1) | ((row >> 2) & 3);
  else if constexpr (HD % 32 == 0) return (row >> 2) & 3;
  else return (row >> 3) & 1;
}

// Bits of a chunk's number that chunk_swap changes, and what it changes between a row and the one eight below
template <int HD> constexpr int SWAP_MASK = HD % 128 == 0 ? 15 : HD % 64 == 0 ? 7 : HD % 32 == 0 ? 3 : 1;
template <int HD> constexpr int SWAP_EIGHT = HD % 32 == 0 ? 2 : 1;

// sixteen zeros for the chunks of a tile row past the head's dims
static __device__ const u32x4 zero_chunk = {0, 0, 0, 0};

typedef uint32_t lds_t;                  // byte address in LDS
__device__ __forceinline__ lds_t lds_address(const void* p) { return (lds_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }

// Fragment of 32 rows x 16 dims with the row in the lane: lane (c = lane % 32, g = lane / 32) holds row row0 + c, dims 16 step + 8 g .. + 7.
// A lane's address differs from step to step in the swapped bits (an exclusive or: the tile's rows are multiples of what they span)
// and in a constant; row0 is a multiple of 16.
template <int HD> __device__ __forceinline__ lds_t row_base(int lane) {
  const int c = lane & 31, g = lane >> 5;
  return c * HD * 2 + ((g ^ chunk_swap<HD>(c)) << 4);
}
template <int HD, class V8> __device__ __forceinline__ V8 row_frag(lds_t base, int row0, int step) {
  constexpr int M = SWAP_MASK<HD>;
  return *(__attribute__((address_space(3))) const V8*)(uintptr_t)((base ^ (((2 * step) & M) << 4)) + (((2 * step) & ~M) << 4) + row0 * HD * 2);
}
// The transposed one, 32 dims x 16 rows: lane (c, g) holds dim 32 t + c and the rows row0 + 4 g .. + 3 and row0 + 8 + 4 g .. + 3, which
// are the rows whose products a 32x32 result leaves in that lane group's registers 8 u .. 8 u + 7 (u = row0 / 16).
// The instruction gives lane i of 16 column i of the 4 x 16 values whose 8-byte pieces lanes 4 r + q (row r, columns 4 q .. + 3) point at.
// A last 16 dims alone (odd HD / 16) are read twice: the results of the second are not kept.
template <int HD> struct ColumnBase { lds_t all, last; };
template <int HD> __device__ __forceinline__ ColumnBase<HD> column_base(int lane) {
  constexpr int M = SWAP_MASK<HD>;
  const int i = lane & 15, b = (lane >> 4) & 1, row = 4 * (lane >> 5) + (i >> 2), sw = chunk_swap<HD>(row);
  ColumnBase<HD> r;
  const int chunk = 2 * b + ((i & 3) >> 1), chunk0 = (i & 3) >> 1;
  r.all = row * HD * 2 + ((chunk & ~M) << 4) + (((chunk & M) ^ sw) << 4) + 8 * (i & 1);
  r.last = HD % 32 ? row * HD * 2 + ((chunk0 & ~M) << 4) + (((chunk0 & M) ^ sw) << 4) + 8 * (i & 1) : r.all;
  return r;
}
template <int HD, class V8> __device__ __forceinline__ V8 column_frag(ColumnBase<HD> base, int row0, int t) {
  constexpr int M = SWAP_MASK<HD>;
  const lds_t b = HD % 32 && 32 * t + 16 >= HD ? base.last : base.all;
  union { s16x4 half[2]; V8 whole; } r;
#pragma unroll
  for (int j = 0; j < 2; ++j)
    r.half[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)(
        (b ^ ((((4 * t) & M) ^ (j * SWAP_EIGHT<HD>)) << 4)) + (((4 * t) & ~M) << 4) + (row0 + 8 * j) * HD * 2));
  return r.whole;
}

// Requests of a tile straight into LDS, a kilobyte of it at a time dealt to the WAVES waves of the block: piece n of a wave is the 64 chunks from
// (WAVES n + wave) 64 on, as they lie in the tile.  Rows lie `stride` elements apart behind a base common to the block, so a lane keeps one
// 32-bit offset a piece for the whole loop; the buffer's range check turns what lies past the last row into zeros, and
// so it does with chunks past the head's dims, which are given an offset beyond any range.
constexpr uint32_t OUT_OF_RANGE = 0x80000000u;
template <int HD, int ROWS, int WAVES = 4> struct Pieces {
  static constexpr int CPR = HD / 8, ALL = ROWS * CPR / 64, PER = (ALL + WAVES - 1) / WAVES;
  uint32_t off[PER];
  static __device__ __forceinline__ void place(int n, int wave, int lane, int& row, int& dim) {
    const int at = (n * WAVES + wave) * 64 + lane;
    row = at / CPR;
    dim = ((at % CPR) ^ chunk_swap<HD>(row)) * 8;
  }
};
struct Buffer { const void* base; int bytes; };
// `rows` rows of one kv head (of `width` elements in all) `step` rows behind `first`, the latter at most what is left
struct RowSource {
  const uint16_t* first;
  uint32_t row_bytes;                      // (strides are at most 2^23 elements, tiles at most 128 rows)
  int width_bytes;
  __device__ __forceinline__ Buffer tile(int step, int rows) const {
    return {(const char*)first + (uint64_t)(uint32_t)step * row_bytes, (rows - 1) * (int)row_bytes + width_bytes};
  }
};
__device__ __forceinline__ RowSource row_source(const void* base, int row0, long long stride, int head, int heads, int h) {
  return {(const uint16_t*)base + (long long)row0 * stride + (long long)head * h, (uint32_t)stride * 2, heads * h * 2};
}
template <int HD, int ROWS, int WAVES = 4> __device__ __forceinline__ Pieces<HD, ROWS, WAVES> piece_offsets(int wave, int lane, long long stride, int h) {
  Pieces<HD, ROWS, WAVES> p;
#pragma unroll
  for (int n = 0; n < p.PER; ++n) {
    int row, dim;
    p.place(n, wave, lane, row, dim);
    p.off[n] = dim < h ? (uint32_t)(row * (int)stride + dim) * 2 : OUT_OF_RANGE;
  }
  return p;
}
// Rows of the axis that queries and heads make: row rem + r of the tile is token (rem + r) / G, head (rem + r) % G behind the base's
template <int HD, int ROWS, int WAVES = 4>
__device__ __forceinline__ Pieces<HD, ROWS, WAVES> flat_offsets(int wave, int lane, long long stride, int h, int G, int rem) {
  Pieces<HD, ROWS, WAVES> p;
#pragma unroll
  for (int n = 0; n < p.PER; ++n) {
    int row, dim;
    p.place(n, wave, lane, row, dim);
    const int tok = (rem + row) / G, head = rem + row - tok * G;
    p.off[n] = dim < h ? (uint32_t)(tok * (int)stride + head * h + dim) * 2 : OUT_OF_RANGE;
  }
  return p;
}
// Requests into LDS: lane i's 16 (4) bytes go 16 (4) i behind `to`, which the wave has in common.  Written as instructions because in front
// of every LDS read the compiler waits for all requests that it knows to write LDS, those of the next tile among them; the barrier
// that a tile begins with waits for them instead.  They have no output register, so none can be overwritten by a late answer, and m0 is
// used by nothing else in these kernels.
__device__ __forceinline__ void request(Buffer from, uint32_t offset, lds_t to) {
  u32x4 d;
  d[0] = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)from.base);
  d[1] = __builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)from.base >> 32) & 0xffffu);
  d[2] = __builtin_amdgcn_readfirstlane(from.bytes);
  d[3] = 0x00027000;
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(d), "s"(__builtin_amdgcn_readfirstlane(to)) : "memory");
}
__device__ __forceinline__ void request(const void* from, lds_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(__builtin_amdgcn_readfirstlane(to)) : "memory");
}
__device__ __forceinline__ void request_word(const float* from, lds_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(__builtin_amdgcn_readfirstlane(to)) : "memory");
}
template <int HD, int ROWS, int WAVES>
__device__ __forceinline__ void request_pieces(Buffer from, const Pieces<HD, ROWS, WAVES>& p, lds_t tile, int wave) {
#pragma unroll
  for (int n = 0; n < p.PER; ++n)
    if (p.ALL % WAVES == 0 || n * WAVES + wave < p.ALL) request(from, p.off[n], tile + (n * WAVES + wave) * 1024);
}

// Has the wave wait for fragments that it loaded itself: in front of a loop, or the compiler waits inside it, where requests of the next
// tile are on their way too.
template <class V8, int N> __device__ __forceinline__ void settle(V8 (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    u32x4 w = __builtin_bit_cast(u32x4, f[i]);
    asm volatile("" : "+v"(w));
    f[i] = __builtin_bit_cast(V8, w);
  }
}

template <class W, int N> __device__ __forceinline__ void settle_words(W (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(v[i]));
}

// In front of a loop: scalar loads of what went before have landed.  They count with the LDS reads but come back in any order, so while the
// compiler takes one to be on its way it waits for all reads in front of the first product instead of for that product's own.
__device__ __forceinline__ void scalars_landed() { __builtin_amdgcn_s_waitcnt(0xc07f); }      // lgkmcnt(0) alone

// Row of register i of a 32x32 result in lane group g (its column is lane % 32)
__device__ __forceinline__ constexpr int acc_row(int i, int g) { return (i >> 2) * 8 + 4 * g + (i & 3); }

// The larger (the sum) of a lane's value and that of its partner in the other half of the wave: the instruction exchanges the upper
// half of one register with the lower half of another, no pass through LDS.
__device__ __forceinline__ float max_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Orders the scheduler's work on a run of products whose operands come from LDS: READS reads ahead, then for every AT_ONCE products
// as many further reads (a product's own reads are then as far ahead; left to itself the scheduler asks for each pair and waits).
template <int READS_EACH, int AHEAD, int PRODUCTS> __device__ __forceinline__ void order_products() {
  constexpr int READS = READS_EACH * PRODUCTS, FIRST = AHEAD * READS_EACH < READS ? AHEAD * READS_EACH : READS;
  __builtin_amdgcn_sched_group_barrier(0x100, FIRST, 0);
#pragma unroll
  for (int i = 0; i < PRODUCTS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if ((i + AHEAD + 1) * READS_EACH <= READS) __builtin_amdgcn_sched_group_barrier(0x100, READS_EACH, 0);
  }
}

// Who is seen, as bits: of the 32 keys from first_key on, those that a query at pos sees (first_key is common to the wave).  A lane group's
// share of them, for the registers of a 32x32 result, is what group_bits leaves; element i's bit is then acc_row(i, 0).
__device__ __forceinline__ uint32_t seen_keys(int pos, int first_key, int window, int sinks) {
  const int hi = pos - first_key, lo = hi - window + 1, n = sinks - first_key;
  const uint32_t up = hi < 0 ? 0u : hi >= 31 ? ~0u : (2u << hi) - 1u;
  const uint32_t down = window == 0 || lo <= 0 ? ~0u : lo > 31 ? 0u : ~0u << lo;
  return up & (down | (n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u));
}
__device__ __forceinline__ uint32_t group_bits(uint32_t seen, int g) { return seen >> (4 * g); }
__device__ __forceinline__ uint32_t element_mask(uint32_t bits, int i) { return (uint32_t)__builtin_amdgcn_sbfe((int)bits, acc_row(i, 0), 1); }
__device__ __forceinline__ float or_else(float v, uint32_t mask, uint32_t other) { return __uint_as_float((__float_as_uint(v) & mask) | (~mask & other)); }

// Writes the transposed result of a wave, x[t] dims 32 t .. of the row in each lane's column, times f, as the row's 16-bit values: a lane
// has four dims of every eight and its partner in the other half of the wave the other four, so they exchange and store 16 bytes each.
template <class T, int DT> __device__ __forceinline__ void store_row(uint16_t* row, const f32x16 (&x)[DT], float f, int h, int g, bool live) {
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int i = 8 * j + 2 * e;
        const auto r = __builtin_amdgcn_permlane32_swap(T::pack(x[t][i] * f, x[t][i + 1] * f), T::pack(x[t][i + 4] * f, x[t][i + 5] * f), false, false);
        w[e] = r[0];
        w[2 + e] = r[1];
      }
      if (live && 32 * t + 16 * j < h) *(u32x4*)(row + 32 * t + 16 * j + 8 * g) = w;
    }
}

// One sequence of a call: its rows, its keys and the position of its first row.
struct Seq { int row0, n, total, ctx; };
__device__ __forceinline__ Seq load_seq(const WindowArgs& a, int s, bool paged) {
  Seq q;
  q.row0 = min(max(a.row_starts[s], 0), a.rows);
  q.n = min(max(a.row_starts[s + 1], q.row0), a.rows) - q.row0;
  q.total = q.n;
  if (paged) q.total = (int)min((long long)max(a.total_lens[s], 0), (long long)a.table_stride << a.page_shift);
  q.ctx = q.total - q.n;
  q.n = min(q.n, a.max_new);           // (grids and workspaces are sized by the caller's bound)
  return q;
}
// Block -> unit (sequence and kv head) and its job.  Blocks go round the eight XCDs, each with an L2 of its own: the jobs of one unit, which
// read the same rows, stay on one XCD.  Jobs are numbered from the longest on.  Where an XCD has up to eight of them for each of its 32 CUs its
// units go job by job, job 0 of each first, so that the launch ends with short ones (keys' side of three sequences of 1500 to 4000 tokens
// on 8 kv heads 362 -> 329 us); with more of them one unit goes behind the other, which L2 is glad of (24 sequences of 257 to 576 tokens, 32
// heads of size 80: forward 82 us, 89 job by job).
__host__ __device__ inline int units_at_once(int units, int jobs) {
  const int on_xcd = (units + 7) / 8;
  return (long long)on_xcd * jobs <= 256 ? on_xcd : 1;
}
__device__ __forceinline__ bool map_block(int id, int units, int jobs, int& unit, int& job) {
  const int at_once = units_at_once(units, jobs), x = id & 7, y = id >> 3, group = y / (at_once * jobs), r = y - group * at_once * jobs;
  job = r / at_once;
  unit = (group * at_once + r - job * at_once) * 8 + x;
  return unit < units;
}
inline long long mapped_blocks(long long units, long long jobs) { return (units + 7) / 8 * 8 * jobs; }      // (at_once is all or one)

// The sign of a scale goes to the queries (their sign bits, exactly), so that the largest product has the largest score; a scale of zero
// becomes one that every score vanishes under, since -infinity stands for masked scores.
template <class V8> __device__ __forceinline__ V8 signed_query(V8 q, float scale) {
  u32x4 w = __builtin_bit_cast(u32x4, q);
  w ^= (__float_as_uint(scale) >> 31) * 0x80008000u;
  return __builtin_bit_cast(V8, w);
}
__device__ __forceinline__ float score_factor(float scale) { return fmaxf(fabsf(scale) * 1.4426950408889634f, 1e-37f); }
