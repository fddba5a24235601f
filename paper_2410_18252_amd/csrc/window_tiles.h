// Tiles of rows in LDS for the windowed attention's matrix products, and who sees whom.
#pragma once
#include "window.h"

typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;
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

// sixteen zeros for the chunks of a tile row past the head's dims
static __device__ const u32x4 zero_chunk = {0, 0, 0, 0};

// Fragment of 32 rows x 16 dims with the row in the lane: lane (c = lane % 32, g = lane / 32) holds row row0 + c, dims 16 step + 8 g .. + 7
template <int HD, class V8> __device__ __forceinline__ V8 row_frag(const uint16_t* tile, int row, int step, int g) {
  return *(const V8*)(tile + row * HD + (((2 * step + g) ^ chunk_swap<HD>(row)) << 3));
}
// The transposed one, 32 dims x 16 rows: lane (c, g) holds dim 32 t + c and the rows row0 + 4 g .. + 3 and row0 + 8 + 4 g .. + 3, which
// are the rows whose products a 32x32 result leaves in that lane group's registers 8 u .. 8 u + 7 (u = row0 / 16).
// The instruction gives lane i of 16 column i of the 4 x 16 values whose 8-byte pieces lanes 4 r + q (row r, columns 4 q .. + 3) point at.
template <int HD, class V8> __device__ __forceinline__ V8 column_frag(const uint16_t* tile, int row0, int t, int lane) {
  const int i = lane & 15, b = (lane >> 4) & 1, g = lane >> 5;
  const int dim = 32 * t + (32 * t + 16 < HD ? 16 * b : 0) + 4 * (i & 3);      // (dims past an odd last 16 repeat it: their results are not kept)
  union { s16x4 half[2]; V8 whole; } r;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int row = row0 + 8 * j + 4 * g + (i >> 2);
    const uint16_t* p = tile + row * HD + (((dim >> 3) ^ chunk_swap<HD>(row)) << 3) + (dim & 7);
    r.half[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
  }
  return r.whole;
}

// Row of register i of a 32x32 result in lane group g (its column is lane % 32)
__device__ __forceinline__ constexpr int acc_row(int i, int g) { return (i >> 2) * 8 + 4 * g + (i & 3); }

// lane exchange across the two halves of a wave
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, WAVE); }

__device__ __forceinline__ bool visible(int pos, int key, int window, int sinks) {
  return (key <= pos) & ((window == 0) | (key > pos - window) | (key < sinks));
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
  return q;
}
// Block -> (sequence, kv head) and tile.  Blocks go round the eight XCDs, each with an L2 of its own: the tiles of one unit, which read the
// same keys, stay on one XCD.  Late tiles first where they see more.
__device__ __forceinline__ bool map_block(int id, int units, int tiles, int& unit, int& tile) {
  const int x = id & 7, y = id >> 3;
  unit = y / tiles * 8 + x;
  tile = tiles - 1 - y % tiles;
  return unit < units;
}
inline unsigned mapped_blocks(long long units, long long tiles) { return (unsigned)((units + 7) / 8 * 8 * tiles); }
