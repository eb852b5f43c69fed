// The paged key-value cache: pages of 64 tokens, one record per page and kv
// head, and what the kernels over it share.
//
// A record holds K and V of 64 tokens of one kv head in the register layout of
// the matrix instructions, so that attention reads it straight into operands
// with one 16-byte load per lane, a whole KiB per wave.  Lane l = 16k + n.
//
// HIF4 (4608 G bytes, G = D/64): K's part, then V's, 2304 G bytes each, G
// tiles of 64 rows by 64 values along the contraction (one HIF4 group a row).
//   K: tile = channel group g, row = key, values = the group's channels; key
//      16a + 4t + b is row 16t + 4a + b, so that the scores that a lane gets
//      from the four products of a page (rows 4k .. 4k+3 of each) are those of
//      16 consecutive keys.
//   V: tile = 64 channels, row = channel, values = the page's keys.
//   codes [G][t/2][lane][t%2][c] words: of row 16t + n the words w = 2k + c,
//      word w = values 8w .. 8w+7, value i in nibble i (sign << 3 | u);
//   then per lane the E3 bits [lane][2G bytes]: a byte for the first halves of
//      the words and one for the second, bit 2t + c (G >= 2: the low bytes of
//      two tiles, then their high bytes);
//   the E2 bits [lane][G bytes], bit 2t + c;
//   the bases [n/4][G][t][n%4] bytes: the rows whose products a lane holds.
// FP16 (256 D bytes): K [t][D/32][lane][8 channels], channels 32 cc + 8k + i of
//   the key in row 16t + n (rows as above); V [D/16][c][lane][8 keys], keys
//   16k + 8c + i of channel 16 ct + n.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace hifa4 {

typedef _Float16 half_t;

constexpr int kPage = 64;

struct PagedCache {
  uint8_t* pool;
  const int* table;       // [batch, max_pages]
  const int* lens;        // [batch]
  half_t* tail;           // [batch, 64, hkv, D]: V of each sequence's last page (HIF4)
  int batch, hkv, D, num_pages, max_pages;
  bool fp16;
};

__host__ __device__ constexpr size_t paged_record_bytes(int D, bool fp16) {
  return fp16 ? (size_t)256 * D : (size_t)72 * D;
}

// Offsets in the K or V part of a HIF4 record (part = 2304 G bytes).
__host__ __device__ constexpr int hif4_part(int G) { return 2304 * G; }
__host__ __device__ constexpr int hif4_code_at(int tile, int t, int lane, int c) {
  return 2048 * tile + 1024 * (t >> 1) + 16 * lane + 8 * (t & 1) + 4 * c;
}
__host__ __device__ constexpr int hif4_e3_at(int G, int tile, int lane, int half) {
  return 2048 * G + 2 * G * lane + (G == 1 ? half : 4 * (tile >> 1) + 2 * half + (tile & 1));
}
__host__ __device__ constexpr int hif4_e2_at(int G, int tile, int lane) { return 2176 * G + G * lane + tile; }
__host__ __device__ constexpr int hif4_base_at(int G, int tile, int t, int n) {
  return 2240 * G + 16 * G * (n >> 2) + 16 * tile + 4 * t + (n & 3);
}
// Row 16t + n of a key's row; t and n of key, and back.
__host__ __device__ constexpr int key_t(int key) { return (key >> 2) & 3; }
__host__ __device__ constexpr int key_n(int key) { return 4 * (key >> 4) + (key & 3); }
__host__ __device__ constexpr int key_of(int t, int n) { return 16 * (n >> 2) + 4 * t + (n & 3); }

// Cached tokens of a row of the batch.  Lengths outside the table are outside
// the contract; clamping them keeps every access inside the caller's buffers.
__device__ __forceinline__ int paged_len(const PagedCache& c, int b) {
  return max(0, min(c.lens[b], c.max_pages * kPage));
}
// The record of (sequence, page place, head), or NULL where the table names no
// page of the pool.
__device__ __forceinline__ uint8_t* paged_record(const PagedCache& c, int b, int place, int head) {
  const int page = c.table[(size_t)b * c.max_pages + place];
  if ((unsigned)page >= (unsigned)c.num_pages) return nullptr;
  return c.pool + ((size_t)page * c.hkv + head) * paged_record_bytes(c.D, c.fp16);
}

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);     // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);    // lane 15 of each row to the next
  return x + __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
}

struct PagedAppend {
  PagedCache c;
  const half_t *k, *v;
  const float* s;
  const int* cu;          // [batch + 1], or NULL: one token a sequence
  int total, max_new;
};
struct PagedGather {
  PagedCache c;
  const int *cu, *starts; // starts may be NULL: 0
  half_t *k, *v;
  int total, max_tokens;
};
struct PagedEvict {
  int batch, max_pages, budget, first, last;
  const int *table, *lens;
  const float* w;
  int *out_table, *out_lens, *freed, *num_freed;
  float* out_w;
};
struct PagedDecode {
  PagedCache c;
  int hq;
  const half_t* q;
  const float* s;
  half_t* o;
  float* lse;
  const float* w_in;      // page weights, or NULL
  float* w_out;
  float decay, scale;     // scale = log2(e) / sqrt(D)
  uint8_t* ws;
};

// Workgroups that one launch may have (fewer than this): HIP counts the threads
// of a grid in 32 bits.
constexpr size_t kMaxGrid = (size_t)1 << 24;
constexpr size_t max_grid(int threads) { return threads <= 256 ? kMaxGrid : ((size_t)1 << 32) / threads; }
// Threads of a workgroup of the append: HIF4 a wave per tile of K and per tile of V.
constexpr int paged_append_threads(int D, bool fp16) { return fp16 ? 256 : 2 * D; }

// Whether the pages can be counted and the join's grid is a launch.
bool paged_decode_fits(const PagedCache& c, int hq, bool weights);
size_t paged_decode_workspace(const PagedCache& c, int hq, bool weights);

hipError_t launch_paged_append(const PagedAppend& a, hipStream_t st);
hipError_t launch_paged_gather(const PagedGather& a, hipStream_t st);
hipError_t launch_paged_evict(const PagedEvict& a, hipStream_t st);
hipError_t launch_paged_decode(const PagedDecode& a, hipStream_t st);

}  // namespace hifa4
