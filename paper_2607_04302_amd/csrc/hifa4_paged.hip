// The paged key-value cache (records and layouts: hifa4_paged.h): appending new
// tokens, reading tokens back, and the eviction of pages by the attention
// weight that they have drawn.
//
// Paper: the cache holds K^ and V^ as Algorithm 1 quantizes them (Smooth-QK
// step, HIF4 of K along the channels and of V along 64 tokens); pages, their
// table and the eviction are this library's.
#include "hifa4_paged.h"
#include "hifa4_words.h"

namespace hifa4 {

// New tokens of row b: [begin, begin + count) of the input go to the places
// [first, first + count) of the sequence, whose last tokens they are.  What is
// outside the contract is left out, so that no access leaves a buffer: rows
// behind the input, tokens in front of the sequence (more new ones than it
// holds) and behind max_new.
struct NewTokens {
  int begin, count, first;
};
__device__ __forceinline__ NewTokens new_tokens(const int* cu, int b, int total, int max_new, int len) {
  NewTokens t;
  t.begin = cu ? min(max(cu[b], 0), total) : b;
  const int end = cu ? min(max(cu[b + 1], t.begin), total) : min(b + 1, total);
  t.begin = max(t.begin, end - len);
  t.first = len - (end - t.begin);
  t.count = min(end - t.begin, max_new);
  return t;
}

// One workgroup's share of a call: (sequence, page, head), `blocks` pages a
// sequence.
struct PageItem {
  int b, blk, head;
};
__device__ __forceinline__ PageItem page_item(int hkv, int blocks) {
  const int i = blockIdx.x / hkv;
  return PageItem{i / blocks, i % blocks, (int)blockIdx.x % hkv};
}
__device__ __forceinline__ uint32_t max_pair16(uint32_t p, uint32_t q) {
  return __builtin_bit_cast(uint32_t,
                            __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, p), __builtin_bit_cast(u16x2_t, q)));
}
// Rows of four halves (8 bytes) of eight keys <-> eight halves of each of four channels.
__device__ __forceinline__ void keys_to_channels(const uint2 (&x)[8], uint4 (&y)[4]) {
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = c < 2 ? __builtin_amdgcn_perm(x[2 * i + 1].x, x[2 * i].x, sel)
                   : __builtin_amdgcn_perm(x[2 * i + 1].y, x[2 * i].y, sel);
    y[c] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
__device__ __forceinline__ void channels_to_keys(const uint4 (&y)[4], uint2 (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t sel = i & 1 ? 0x07060302u : 0x05040100u;
    uint32_t w[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) w[c] = i < 2 ? y[c].x : i < 4 ? y[c].y : i < 6 ? y[c].z : y[c].w;
    x[i] = make_uint2(__builtin_amdgcn_perm(w[1], w[0], sel), __builtin_amdgcn_perm(w[3], w[2], sel));
  }
}

// ---------------------------------------------------------------------------
// Append, HIF4.  One workgroup per (sequence, page that the new tokens touch,
// head).  K~ = fp16(k/s) is quantized along the channels, a key's words written
// to its row of the record; V is quantized along the 64 tokens of the page,
// from the new tokens and, before them in the page, from the fp16 rows that
// the tail keeps of the open page, places behind the last token zero: the page
// holds at any time what quantizing the whole sequence would give.
// One wave per tile of K and one per tile of V.  A lane of K is the record's
// lane: 16 channels of the keys of its four rows, so its codes and its bytes of
// metadata are whole and a group's maximum is a matter of four lanes, two rows
// at a time.  A lane of V takes 16 keys of four neighbouring channels, that its
// loads are 8 bytes wide; its codes go through LDS into 16-byte pieces, the
// bits of the four rows of a lane of the record are joined across the wave.
// 16 prompts of 512 to 2048 tokens, 8 heads, D=128, smoothed (107 MB): 30.9 us,
// where the copy rate would take 23.  What is left is the wait for a page's
// loads at its start: six waves per SIMD hide most of it, so K fetches its
// scales from LDS for every row and is scheduled row by row (79 registers; with
// 111, four waves, 41 us; seven with spills 35).
__device__ __forceinline__ int padded(int at) { return at + (at >> 8) * 16; }

// The codes of four pairs of values, a pair in the two halves of a register,
// as nibbles (sign << 3 | u) in the low halves of bytes 0, 1 and 2, 3: those of
// y0's and y1's values.  `sel` orders the four; x: the values, for their signs.
__device__ __forceinline__ uint32_t nibble_bytes(uint32_t y0, uint32_t y1, h2_t x0, h2_t x1, uint32_t sel) {
  const uint32_t u = __builtin_amdgcn_perm(y1, y0, sel) & 0x07070707u;
  const uint32_t s = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, x1), __builtin_bit_cast(uint32_t, x0), sel + 0x01010101u);
  const uint32_t v = u | ((u + 0x07070707u) & ((s >> 4) & 0x08080808u));      // a zero code has no sign
  return v | v >> 4;                       // bytes 0 and 2: two nibbles each
}
// Nothing is scheduled across: fewer registers at a time.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0); }
__device__ __forceinline__ uint32_t max_rows16(uint32_t v) {          // over the four lanes 16 apart, per half
  const Pair32 p = pair32(v);
  v = max_pair16(p.x, p.y);
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return max_pair16(r[0], r[1]);
}
__device__ __forceinline__ uint32_t or_rows(uint32_t v) {
  const Pair32 p = pair32(v);
  v = p.x | p.y;
  const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  return r[0] | r[1];
}

// K: the lane's metadata into `meta` (LDS), its codes into the record.  s: the
// scales of the tile's 64 channels, or NULL; they and their reciprocals wait in
// LDS (`scales`), where every row fetches its lane's 16.
template <int G>
__device__ __forceinline__ void append_k(const uint4 (&in)[4][2], const float* s, float* scales, uint8_t* rec,
                                         uint8_t* meta, int tile, int lane, int lo, int hi) {
  const int n = lane & 15, k = lane >> 4;
  if (s) {
    scales[lane] = s[lane];
    scales[64 + lane] = 1.0f / scales[lane];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  uint32_t e2 = 0, e3 = 0, bases = 0;      // E2 and E3 (halves: of the words' halves) by bit 2t + c; a base a byte
#pragma unroll
  for (int i = 0; i < 2; ++i) {            // rows t = 2i and 2i + 1
    const int key = key_of(2 * i, n);
    const bool na = key >= lo && key < hi, nb = key + 4 >= lo && key + 4 < hi;
    if (!__builtin_amdgcn_ballot_w64(na || nb)) continue;
    h2_t x[2][8], a4[2][2];
    u16x2_t a8[2][2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const uint4 w0 = in[2 * i + r][0], w1 = in[2 * i + r][1];
      const uint32_t w[8] = {w0.x, w0.y, w0.z, w0.w, w1.x, w1.y, w1.z, w1.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) x[r][e] = __builtin_bit_cast(h2_t, w[e]);
      if (s) {
        asm volatile("" ::: "memory");     // (fetched again: registers for more waves are worth more)
        divide_pairs(x[r], scales + 16 * k, scales + 64 + 16 * k);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        a4[r][c] = hmax_pairs(hmax2(habs2(x[r][4 * c]), habs2(x[r][4 * c + 1])),
                              hmax2(habs2(x[r][4 * c + 2]), habs2(x[r][4 * c + 3])));
        a8[r][c] = __builtin_elementwise_max(as_u16(a4[r][c]), __builtin_shufflevector(as_u16(a4[r][c]), as_u16(a4[r][c]), 1, 0));
      }
      keep_order();
    }
    const u16x2_t t0 = __builtin_elementwise_max(a8[0][0], a8[0][1]), t1 = __builtin_elementwise_max(a8[1][0], a8[1][1]);
    const h2_t top = __builtin_bit_cast(h2_t, max_rows16(__builtin_bit_cast(uint32_t, u16x2_t{t0[0], t1[1]})));
    uint32_t word[2][2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const uint32_t base = e6m2_ceil((float)top[r]);
      const float R = hif4_rcp_step(base);
      const h2_t thr = range_floors(e6m2_value(base));
      bases |= base << (8 * (2 * i + r));
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        u16x2_t lv, ne2;
        block_levels(a4[r][c], __builtin_bit_cast(h2_t, a8[r][c]), h2_t{thr[0], thr[0]}, h2_t{thr[1], thr[1]}, lv, ne2);
        uint32_t y[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const unsigned short ne = lv[q];
          const h2_t u = x[r][4 * c + 2 * q], v = x[r][4 * c + 2 * q + 1];
          y[q] = nibble_bytes(codes2(habs2(u), R, R, u16x2_t{ne, ne}), codes2(habs2(v), R, R, u16x2_t{ne, ne}), u, v,
                              0x06040200u);
        }
        word[r][c] = __builtin_amdgcn_perm(y[1], y[0], 0x06040200u);
        const int bit = 2 * (2 * i + r) + c;
        e2 |= (1u - ne2[0]) << bit;
        e3 |= __builtin_bit_cast(uint32_t, u16x2_t{1, 1} + ne2 - lv) << bit;
      }
      keep_order();
    }
    if (rec) {
      uint8_t* at = rec + 2048 * tile + 1024 * i + 16 * lane;
      if (na && nb)
        *reinterpret_cast<uint4*>(at) = make_uint4(word[0][0], word[0][1], word[1][0], word[1][1]);
      else if (na)
        *reinterpret_cast<uint2*>(at) = make_uint2(word[0][0], word[0][1]);
      else if (nb)
        *reinterpret_cast<uint2*>(at + 8) = make_uint2(word[1][0], word[1][1]);
    }
  }
  const int a3 = hif4_e3_at(G, tile, lane, 0) - 2048 * G, b3 = hif4_e3_at(G, tile, lane, 1) - 2048 * G;
  const int a2 = hif4_e2_at(G, tile, lane) - 2048 * G, ab = hif4_base_at(G, tile, k, n) - 2048 * G;    // base: of row t = k
  uint32_t base = bases >> (8 * k) & 0xFFu;
  if (lo > 0 || hi < kPage) {              // the keys before lo keep what they have, those from hi on have nothing
    uint32_t mine = 0, old = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int key = key_of(t, n);
      if (key < lo)
        old |= 3u << (2 * t);
      else if (key < hi)
        mine |= 3u << (2 * t);
    }
    e2 &= mine;
    e3 &= mine * 0x00010001u;
    if (!(mine >> (2 * k) & 1u)) base = 0;
    if (lo > 0 && rec) {
      const uint8_t* was = rec + 2048 * G;
      e2 |= was[a2] & old;
      e3 |= (was[a3] & old) | (was[b3] & old) << 16;
      if (old >> (2 * k) & 1u) base = was[ab];
    }
  }
  meta[a3] = (uint8_t)e3;
  meta[b3] = (uint8_t)(e3 >> 16);
  meta[a2] = (uint8_t)e2;
  meta[ab] = (uint8_t)base;
}

// V: codes and metadata of a lane's 16 keys of four channels into LDS.
template <int G>
__device__ __forceinline__ void append_v(const uint2 (&in)[16], uint8_t* codes, uint8_t* meta, int tile, int lane) {
  const int k = lane & 3, n = lane & 12, t = lane >> 4;          // channels 64 tile + 16 t + n ..
  uint32_t e2[2], ea[2], eb[2], bases = 0;                       // E2; E3 of the words' first and second halves
#pragma unroll
  for (int p = 0; p < 2; ++p) {            // channels n + 2p and n + 2p + 1, in the two halves
    h2_t x[16], a4[4];
#pragma unroll
    for (int e = 0; e < 16; ++e) x[e] = __builtin_bit_cast(h2_t, p ? in[e].y : in[e].x);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      a4[q] = hmax2(hmax2(habs2(x[4 * q]), habs2(x[4 * q + 1])), hmax2(habs2(x[4 * q + 2]), habs2(x[4 * q + 3])));
    const u16x2_t a8[2] = {__builtin_elementwise_max(as_u16(a4[0]), as_u16(a4[1])),
                           __builtin_elementwise_max(as_u16(a4[2]), as_u16(a4[3]))};
    uint32_t all = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(a8[0], a8[1]));
    all = max_pair16(all, (uint32_t)__builtin_amdgcn_mov_dpp((int)all, 0xB1, 0xF, 0xF, true));
    all = max_pair16(all, (uint32_t)__builtin_amdgcn_mov_dpp((int)all, 0x4E, 0xF, 0xF, true));
    const h2_t top = __builtin_bit_cast(h2_t, all);
    const uint32_t base[2] = {e6m2_ceil((float)top[0]), e6m2_ceil((float)top[1])};
    const float r0 = hif4_rcp_step(base[0]), r1 = hif4_rcp_step(base[1]);
    const h2_t f0 = range_floors(e6m2_value(base[0])), f1 = range_floors(e6m2_value(base[1]));
    bases |= (base[0] | base[1] << 8) << (16 * p);
    uint32_t word[2][2];                   // [channel][c]
    e2[p] = ea[p] = eb[p] = 0;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      uint32_t y[4];                       // two keys' nibbles of either channel
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        u16x2_t lv, ne2;
        block_levels(a4[2 * c + q], __builtin_bit_cast(h2_t, a8[c]), h2_t{f0[0], f1[0]}, h2_t{f0[1], f1[1]}, lv, ne2);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const h2_t u = x[8 * c + 4 * q + 2 * e], v = x[8 * c + 4 * q + 2 * e + 1];
          y[2 * q + e] = nibble_bytes(codes2(habs2(u), r0, r1, lv), codes2(habs2(v), r0, r1, lv), u, v, 0x06020400u);
        }
        const uint32_t e3 = __builtin_bit_cast(uint32_t, u16x2_t{1, 1} + ne2 - lv);
        (q ? eb[p] : ea[p]) |= e3 << c;
        if (q == 0) e2[p] |= __builtin_bit_cast(uint32_t, u16x2_t{1, 1} - ne2) << c;
      }
      const uint32_t lo = __builtin_amdgcn_perm(y[1], y[0], 0x06020400u), hi = __builtin_amdgcn_perm(y[3], y[2], 0x06020400u);
      word[0][c] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
      word[1][c] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e)
      *reinterpret_cast<uint2*>(codes + padded(hif4_code_at(tile, t, 16 * k + n + 2 * p + e, 0))) =
          make_uint2(word[e][0], word[e][1]);
  }
  // a byte a channel, the bits of its row t; joined, the bytes of the record's four lanes n .. n+3
  const auto join = [&](const uint32_t (&x)[2]) { return or_rows(__builtin_amdgcn_perm(x[1], x[0], 0x06040200u) << (2 * t)) >> (8 * t); };
  const int to = 16 * k + n + t;
  meta[hif4_e2_at(G, tile, to) - 2048 * G] = (uint8_t)join(e2);
  meta[hif4_e3_at(G, tile, to, 0) - 2048 * G] = (uint8_t)join(ea);
  meta[hif4_e3_at(G, tile, to, 1) - 2048 * G] = (uint8_t)join(eb);
  if (k == 0) *reinterpret_cast<uint32_t*>(meta + hif4_base_at(G, tile, t, n) - 2048 * G) = bases;
}

template <int G>
__global__ void __launch_bounds__(128 * G) k_paged_append(PagedAppend a, int blocks) {
  constexpr int D = 64 * G, kThreads = 128 * G, kMeta = 256 * G;
  __shared__ __align__(16) uint8_t meta[2][kMeta];
  __shared__ __align__(16) uint8_t codes[2048 * G + 8 * G * 16];
  __shared__ __align__(16) float scales[2 * D];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), tile = wave % G;
  const PageItem it = page_item(a.c.hkv, blocks);
  const int len = paged_len(a.c, it.b);
  const NewTokens nt = new_tokens(a.cu, it.b, a.total, a.max_new, len);
  const int place = nt.first / kPage + it.blk, p0 = place * kPage;
  const int stop = nt.first + nt.count;
  if (nt.count == 0 || p0 >= stop) return;
  const int lo = max(nt.first - p0, 0), hi = min(stop - p0, kPage);    // new keys of the page: [lo, hi)
  uint8_t* rec = paged_record(a.c, it.b, place, it.head);
  const size_t row = (size_t)a.c.hkv * D;
  // the new token at key 0 of the page (it may lie before the input: only keys >= lo are read)
  const long t0 = (long)nt.begin + p0 - nt.first;
  half_t* tail = a.c.tail + ((size_t)it.b * kPage * a.c.hkv + it.head) * D;

  if (wave < G) {
    const size_t at = (size_t)it.head * D + 64 * tile + 16 * (lane >> 4);
    uint4 in[4][2];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int key = min(max(key_of(t, lane & 15), lo), hi - 1);
      const uint4* from = reinterpret_cast<const uint4*>(a.k + (size_t)(t0 + key) * row + at);
      in[t][0] = from[0];
      in[t][1] = from[1];
    }
    append_k<G>(in, a.s ? a.s + (size_t)it.head * D + 64 * tile : nullptr, scales + 128 * tile, rec, meta[0], tile, lane, lo, hi);
  } else {
    const int key0 = 16 * (lane & 3), ch = 64 * tile + 4 * (lane >> 2);
    uint2 in[16];
    if (lo == 0 && hi == kPage) {
      const half_t* from = a.v + (size_t)(t0 + key0) * row + (size_t)it.head * D + ch;
#pragma unroll
      for (int e = 0; e < 16; ++e) in[e] = *reinterpret_cast<const uint2*>(from + e * row);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = key0 + e;
        in[e] = make_uint2(0, 0);
        if (key < hi)
          in[e] = *reinterpret_cast<const uint2*>(
              key >= lo ? a.v + (size_t)(t0 + key) * row + (size_t)it.head * D + ch : tail + (size_t)key * row + ch);
      }
    }
    append_v<G>(in, codes, meta[1], tile, lane);
  }
  __syncthreads();
  if (rec) {
    uint8_t* vp = rec + hif4_part(G);
    *reinterpret_cast<uint4*>(vp + 16 * tid) = *reinterpret_cast<const uint4*>(codes + padded(16 * tid));
    if (tid < 2 * kMeta / 16) {
      const int part = tid / (kMeta / 16), at = 16 * (tid % (kMeta / 16));
      *reinterpret_cast<uint4*>((part ? vp : rec) + 2048 * G + at) = *reinterpret_cast<const uint4*>(&meta[part][at]);
    }
  }
  // The tail gets the last page's new rows.  The workgroup of the first page
  // writes them: it alone reads the tail, and has done so before the barrier.
  if (it.blk == 0) {
    const int last = (stop - 1) / kPage * kPage;              // place of the last page's first token
    const int from = max(nt.first - last, 0), to = stop - last;
    const long l0 = (long)nt.begin + last - nt.first;
    for (int i = tid; i < (to - from) * (D / 8); i += kThreads) {
      const int key = from + i / (D / 8), ch = 8 * (i % (D / 8));
      *reinterpret_cast<uint4*>(tail + (size_t)key * row + ch) =
          *reinterpret_cast<const uint4*>(a.v + (size_t)(l0 + key) * row + (size_t)it.head * D + ch);
    }
  }
}

// Place, in halves, of key `key`'s channels 8 oct .. 8 oct + 7 in an FP16
// record's K, and of the keys 8w .. 8w+7 of channel ch in its V.
__device__ __forceinline__ int fp16_k_at(int D, int key, int oct) {
  return ((key_t(key) * (D / 32) + oct / 4) * 64 + 16 * (oct & 3) + key_n(key)) * 8;
}
__device__ __forceinline__ int fp16_v_at(int D, int w, int ch) {
  return 64 * D + ((ch / 16 * 2 + (w & 1)) * 64 + 16 * (w >> 1) + (ch & 15)) * 8;
}

// Append, FP16: the new tokens' K~ and V go to their places in the record.  A
// thread takes eight channels of a key of K, and eight keys of four channels
// of V, which it transposes in registers: all accesses but those of a page's
// unfinished sets of eight keys are 16 bytes wide (8 for V's rows).  Bound by
// HBM: 16 prompts of 512 to 2048 tokens, 8 heads, D=256 (342 MB) in 81 us, 4.2
// TB/s.
template <int G>
__global__ void __launch_bounds__(256) k_paged_append16(PagedAppend a, int blocks) {
  constexpr int D = 64 * G, kK = 2 * G, kV = (G + 1) / 2;
  const int tid = threadIdx.x;
  const PageItem it = page_item(a.c.hkv, blocks);
  const int len = paged_len(a.c, it.b);
  const NewTokens nt = new_tokens(a.cu, it.b, a.total, a.max_new, len);
  const int place = nt.first / kPage + it.blk, p0 = place * kPage;
  const int stop = nt.first + nt.count;
  if (nt.count == 0 || p0 >= stop) return;
  const int lo = max(nt.first - p0, 0), hi = min(stop - p0, kPage);
  uint8_t* rec = paged_record(a.c, it.b, place, it.head);
  if (!rec) return;
  const size_t row = (size_t)a.c.hkv * D;
  const long t0 = (long)nt.begin + p0 - nt.first;
  const half_t* src_v = a.v + (size_t)it.head * D;
  half_t* dst = reinterpret_cast<half_t*>(rec);
  const int oct = tid % (8 * G), key0 = lo + tid / (8 * G);
  uint4 in_k[kK];
#pragma unroll
  for (int i = 0; i < kK; ++i)
    in_k[i] = *reinterpret_cast<const uint4*>(a.k + (size_t)(t0 + min(key0 + i * (32 / G), hi - 1)) * row +
                                              (size_t)it.head * D + 8 * oct);
  uint2 in_v[kV][8];
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int item = tid + 256 * i, w = item / (16 * G), ch = 4 * (item % (16 * G));
#pragma unroll
    for (int e = 0; e < 8; ++e)
      in_v[i][e] = *reinterpret_cast<const uint2*>(src_v + (size_t)(t0 + min(max(8 * w + e, lo), hi - 1)) * row + ch);
  }
  float sc[8], rc[8];
  if (a.s) {
    const float4* sp = reinterpret_cast<const float4*>(a.s + (size_t)it.head * D + 8 * oct);
    const float4 s0 = sp[0], s1 = sp[1];
    const float s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sc[e] = s[e];
      rc[e] = 1.0f / s[e];
    }
  }
#pragma unroll
  for (int i = 0; i < kK; ++i) {
    const int key = key0 + i * (32 / G);
    if (key >= hi) break;
    h2_t x[4] = {__builtin_bit_cast(h2_t, in_k[i].x), __builtin_bit_cast(h2_t, in_k[i].y),
                 __builtin_bit_cast(h2_t, in_k[i].z), __builtin_bit_cast(h2_t, in_k[i].w)};
    if (a.s) divide_pairs(x, sc, rc);
    *reinterpret_cast<uint4*>(dst + fp16_k_at(D, key, oct)) =
        make_uint4(__builtin_bit_cast(uint32_t, x[0]), __builtin_bit_cast(uint32_t, x[1]),
                   __builtin_bit_cast(uint32_t, x[2]), __builtin_bit_cast(uint32_t, x[3]));
  }
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int item = tid + 256 * i, w = item / (16 * G), ch = 4 * (item % (16 * G));
    if (w >= 8 || 8 * w + 8 <= lo || 8 * w >= hi) continue;
    uint4 y[4];
    keys_to_channels(in_v[i], y);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      half_t* at = dst + fp16_v_at(D, w, ch + c);
      if (8 * w >= lo && 8 * w + 8 <= hi) {
        *reinterpret_cast<uint4*>(at) = y[c];
      } else {
        const uint32_t z[4] = {y[c].x, y[c].y, y[c].z, y[c].w};
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (8 * w + e >= lo && 8 * w + e < hi)
            reinterpret_cast<uint16_t*>(at)[e] = (uint16_t)(z[e / 2] >> (16 * (e & 1)));
      }
    }
  }
}

hipError_t launch_paged_append(const PagedAppend& a, hipStream_t st) {
  // pages that max_new tokens can touch from any place in a page
  const int blocks = (a.max_new + kPage - 2) / kPage + 1;
  const dim3 grid((unsigned)((size_t)a.c.batch * blocks * a.c.hkv));
  const int threads = paged_append_threads(a.c.D, a.c.fp16);
  if (a.c.fp16) {
    if (a.c.D == 64)
      k_paged_append16<1><<<grid, threads, 0, st>>>(a, blocks);
    else if (a.c.D == 128)
      k_paged_append16<2><<<grid, threads, 0, st>>>(a, blocks);
    else
      k_paged_append16<4><<<grid, threads, 0, st>>>(a, blocks);
  } else {
    if (a.c.D == 64)
      k_paged_append<1><<<grid, threads, 0, st>>>(a, blocks);
    else if (a.c.D == 128)
      k_paged_append<2><<<grid, threads, 0, st>>>(a, blocks);
    else
      k_paged_append<4><<<grid, threads, 0, st>>>(a, blocks);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Gather: tokens [start, start + n) of each sequence as fp16 rows.  One
// workgroup per (sequence, page, head).  Tokens behind the sequence's end and
// tokens of places without a page are zeros.  HIF4: the record goes to LDS in
// one sweep, padded by 16 bytes per 256 so that the four lanes of a row and
// the tiles lie in different banks; a thread makes eight channels of a key of
// K from one word, eight keys of four channels of V from four.  A value is
// u b/4 2^-(E2+E3), whole in fp32, rounded once.  Bound by HBM, mostly the
// writes: 32 sequences of 300 to 8192 tokens, 8 heads, D=128, HIF4 (750 MB) in
// 153 us, 4.9 TB/s.

// The eight values of word (lane, c) of row (t, n) of a part in LDS, in fp32.
template <int G>
__device__ __forceinline__ void word_values(const uint8_t* part, int tile, int t, int n, int w, float (&x)[8]) {
  const int lane = 16 * (w >> 1) + n, bit = 2 * t + (w & 1);
  const uint32_t word = *reinterpret_cast<const uint32_t*>(part + padded(hif4_code_at(tile, t, lane, w & 1)));
  const uint32_t e2 = (part[padded(hif4_e2_at(G, tile, lane))] >> bit) & 1u;
  const uint32_t ea = (part[padded(hif4_e3_at(G, tile, lane, 0))] >> bit) & 1u;
  const uint32_t eb = (part[padded(hif4_e3_at(G, tile, lane, 1))] >> bit) & 1u;
  const uint32_t base = ((uint32_t)part[padded(hif4_base_at(G, tile, t, n))] << 21) + 0x2F000000u;      // b/4
  const float s0 = __uint_as_float(base - ((e2 + ea) << 23)), s1 = __uint_as_float(base - ((e2 + eb) << 23));
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float u = (float)((word >> (4 * i)) & 7u) * (i < 4 ? s0 : s1);
    x[i] = __uint_as_float(__float_as_uint(u) | ((word << (28 - 4 * i)) & 0x80000000u));
  }
}
__device__ __forceinline__ uint32_t pack_rn16(float a, float b) {
  typedef float f2_t __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2_t{a, b}, h2_t));
}

template <int G, bool kFp16>
__global__ void __launch_bounds__(256) k_paged_gather(PagedGather a, int blocks) {
  constexpr int D = 64 * G, kK = 2 * G, kV = (G + 1) / 2;
  __shared__ __align__(16) uint8_t lds[kFp16 ? 16 : 72 * D + 72 * D / 256 * 16];
  const int tid = threadIdx.x;
  const PageItem it = page_item(a.c.hkv, blocks);
  const int begin = min(max(a.cu[it.b], 0), a.total);
  const int count = min(min(max(a.cu[it.b + 1], begin), a.total) - begin, a.max_tokens);
  const int start = a.starts ? max(a.starts[it.b], 0) : 0;
  const int place = start / kPage + it.blk;
  const long p0 = (long)place * kPage;
  const int lo = (int)max((long)start - p0, 0L), hi = (int)min((long)start + count - p0, (long)kPage);
  if (hi <= lo) return;
  const int held = (int)min(max((long)paged_len(a.c, it.b) - p0, 0L), (long)kPage);      // keys of the page that exist
  const uint8_t* rec = held > 0 ? paged_record(a.c, it.b, place, it.head) : nullptr;
  const int there = rec ? held : 0;
  const size_t row = (size_t)a.c.hkv * D;
  // rows of the output: key `key` of the page is row o0 + key
  const long o0 = (long)begin + p0 - start;
  if (!kFp16 && rec) {
#pragma unroll
    for (int i = 0; i < (72 * D / 16 + 255) / 256; ++i) {
      const int at = 16 * (tid + 256 * i);
      if (at < 72 * D) *reinterpret_cast<uint4*>(lds + padded(at)) = *reinterpret_cast<const uint4*>(rec + at);
    }
  }
  __syncthreads();
  const half_t* src = reinterpret_cast<const half_t*>(rec);
#pragma unroll
  for (int i = 0; i < kK; ++i) {
    const int oct = tid % (8 * G), key = tid / (8 * G) + i * (32 / G);
    if (key < lo || key >= hi) continue;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (key < there) {
      if (kFp16) {
        x = *reinterpret_cast<const uint4*>(src + fp16_k_at(D, key, oct));
      } else {
        float y[8];
        word_values<G>(lds, oct >> 3, key_t(key), key_n(key), oct & 7, y);
        x = make_uint4(pack_rn16(y[0], y[1]), pack_rn16(y[2], y[3]), pack_rn16(y[4], y[5]), pack_rn16(y[6], y[7]));
      }
    }
    *reinterpret_cast<uint4*>(a.k + (size_t)(o0 + key) * row + (size_t)it.head * D + 8 * oct) = x;
  }
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int item = tid + 256 * i, w = item / (16 * G), ch = 4 * (item % (16 * G));
    if (w >= 8 || 8 * w + 8 <= lo || 8 * w >= hi) continue;
    uint2 x[8];
    if (8 * w < there) {
      if (kFp16) {
        uint4 y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = *reinterpret_cast<const uint4*>(src + fp16_v_at(D, w, ch + c));
        channels_to_keys(y, x);
      } else {
        float y[4][8];
#pragma unroll
        for (int c = 0; c < 4; ++c)
          word_values<G>(lds + padded(hif4_part(G)), ch >> 6, (ch >> 4) & 3, (ch & 15) + c, w, y[c]);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = make_uint2(pack_rn16(y[0][e], y[1][e]), pack_rn16(y[2][e], y[3][e]));
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int key = 8 * w + e;
      if (key >= lo && key < hi)
        *reinterpret_cast<uint2*>(a.v + (size_t)(o0 + key) * row + (size_t)it.head * D + ch) =
            key < there ? x[e] : make_uint2(0, 0);
    }
  }
}

hipError_t launch_paged_gather(const PagedGather& a, hipStream_t st) {
  const int blocks = (a.max_tokens + kPage - 2) / kPage + 1;
  const dim3 grid((unsigned)((size_t)a.c.batch * blocks * a.c.hkv));
  if (a.c.fp16) {
    if (a.c.D == 64)
      k_paged_gather<1, true><<<grid, 256, 0, st>>>(a, blocks);
    else if (a.c.D == 128)
      k_paged_gather<2, true><<<grid, 256, 0, st>>>(a, blocks);
    else
      k_paged_gather<4, true><<<grid, 256, 0, st>>>(a, blocks);
  } else {
    if (a.c.D == 64)
      k_paged_gather<1, false><<<grid, 256, 0, st>>>(a, blocks);
    else if (a.c.D == 128)
      k_paged_gather<2, false><<<grid, 256, 0, st>>>(a, blocks);
    else
      k_paged_gather<4, false><<<grid, 256, 0, st>>>(a, blocks);
  }
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Eviction.  One workgroup per sequence.  Of the pages between the first and
// the last ones that stay, the budget's remaining places go to the largest
// weights, equal ones to the lowest place.  The weight at the border is found
// digit by digit (8 bits at a time, by counts in LDS), then one pass over the
// places moves what stays and lists what leaves, both in order.  The first
// 2048 places' weights and pages are read once, into registers.  Bound by
// latency: four counts and one pass, three barriers each, 5.6 us for 8 sequences
// of 512 pages, 7.0 for 64 of up to 2048.  Of longer rows the counts and the pass
// read the rest anew, out of the caches: 64 sequences of 8192 pages 17.8 us.
constexpr int kEvictThreads = 1024, kEvictHeld = 2;

// Order of the weights as unsigned integers; NaN below everything, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ void __launch_bounds__(kEvictThreads) k_paged_evict(PagedEvict a) {
  __shared__ uint32_t hist[256], sums[kEvictThreads / 64], found[3];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const size_t row = (size_t)b * a.max_pages;
  const int len = max(0, min(a.lens[b], a.max_pages * kPage));
  const int pages = (len + kPage - 1) / kPage;
  const int lo = a.first, hi = pages - a.last;               // contenders: [lo, hi)
  float w_held[kEvictHeld];
  int page_held[kEvictHeld];
#pragma unroll
  for (int c = 0; c < kEvictHeld; ++c) {
    const int i = tid + c * kEvictThreads;
    w_held[c] = i < pages ? a.w[row + i] : 0.0f;
    page_held[c] = i < pages ? a.table[row + i] : -1;
  }
  // keys above the border stay, of those equal to it the first `ties` (in all there are `equals`)
  uint32_t border = 0xFFFFFFFFu;
  int ties = 0, equals = 0;
  const int room = a.budget - a.first - a.last;
  if (pages > a.budget && room > 0) {
    border = 0;
    int left = room;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      const auto count = [&](int i, float w) {
        const uint32_t k = weight_key(w);
        if (i >= lo && i < hi && (shift == 24 || ((k ^ border) >> (shift + 8)) == 0)) atomicAdd(&hist[(k >> shift) & 255u], 1u);
      };
#pragma unroll
      for (int c = 0; c < kEvictHeld; ++c) count(tid + c * kEvictThreads, w_held[c]);
      for (int i = tid + kEvictHeld * kEvictThreads; i < hi; i += kEvictThreads) count(i, a.w[row + i]);
      __syncthreads();
      if (wave == 0) {                     // lane l: digits 255 - 4l and the three below
        uint32_t n[4], sum = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += n[e] = hist[255 - 4 * lane - e];
        uint32_t above = (uint32_t)wave_scan((int)sum) - sum;
        if (above < (uint32_t)left && above + sum >= (uint32_t)left) {
          int e = 0;
          while (above + n[e] < (uint32_t)left) above += n[e++];
          found[0] = (uint32_t)(255 - 4 * lane - e);
          found[1] = (uint32_t)left - above;
          found[2] = n[e];
        }
      }
      __syncthreads();
      border |= found[0] << shift;
      left = (int)found[1];
      equals = (int)found[2];
    }
    ties = left;
  }
  // one pass in order; what is written lies at or before what has been read
  int kept = 0, gone = 0, tied = 0;
  for (int c = 0; c * kEvictThreads < pages; ++c) {
    const int i = tid + c * kEvictThreads;
    const bool there = i < pages;
    float w = 0.0f;
    int page = -1;
    if (c == 0) {
      w = w_held[0];
      page = page_held[0];
    } else if (c == 1) {
      w = w_held[1];
      page = page_held[1];
    } else if (there) {
      w = a.w[row + i];
      page = a.table[row + i];
    }
    const uint32_t k = weight_key(w);
    const bool fixed = pages <= a.budget || i < lo || i >= hi;
    const bool equal = there && !fixed && k == border;
    bool keep = there && (fixed || k > border || equal);
    if (ties < equals) {                   // some of the equal ones leave: their order counts
      const unsigned long long same = __builtin_amdgcn_ballot_w64(equal);
      if (lane == 0) sums[wave] = (uint32_t)__popcll(same);
      __syncthreads();
      const int upto = wave_scan(lane < kEvictThreads / 64 ? (int)sums[lane] : 0);
      const int before = tied + (wave ? __builtin_amdgcn_readlane(upto, wave - 1) : 0) +
                         __popcll(same & ((1ull << lane) - 1));
      if (equal && before >= ties) keep = false;
      tied += __builtin_amdgcn_readlane(upto, 63);
      __syncthreads();
    }
    const unsigned long long stay = __builtin_amdgcn_ballot_w64(keep), leave = __builtin_amdgcn_ballot_w64(there && !keep);
    if (lane == 0) sums[wave] = (uint32_t)__popcll(stay) | (uint32_t)__popcll(leave) << 16;
    __syncthreads();
    const uint32_t upto = (uint32_t)wave_scan(lane < kEvictThreads / 64 ? (int)sums[lane] : 0);
    const uint32_t before = wave ? (uint32_t)__builtin_amdgcn_readlane((int)upto, wave - 1) : 0;
    const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    if (keep) {
      const size_t to = row + kept + (before & 0xFFFFu) + __popcll(stay & ((1ull << lane) - 1));
      a.out_table[to] = page;
      a.out_w[to] = w;
    } else if (there) {
      a.freed[row + gone + (before >> 16) + __popcll(leave & ((1ull << lane) - 1))] = page;
    }
    kept += (int)(all & 0xFFFFu);
    gone += (int)(all >> 16);
    __syncthreads();
  }
  for (int i = kept + tid; i < a.max_pages; i += kEvictThreads) {
    a.out_table[row + i] = -1;
    a.out_w[row + i] = 0.0f;
  }
  for (int i = gone + tid; i < a.max_pages; i += kEvictThreads) a.freed[row + i] = -1;
  if (tid == 0) {
    a.out_lens[b] = len - kPage * gone;
    a.num_freed[b] = gone;
  }
}

hipError_t launch_paged_evict(const PagedEvict& a, hipStream_t st) {
  k_paged_evict<<<dim3((unsigned)a.batch), kEvictThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace hifa4
