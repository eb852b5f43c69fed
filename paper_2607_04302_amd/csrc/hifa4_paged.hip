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

// New tokens of row b: [begin, begin + count) of the input, at the places
// [len - count, len) of the sequence.  Counts outside the contract are cut to
// the input, to max_new and to the sequence, so that no access leaves a buffer.
struct NewTokens {
  int begin, count, first;
};
__device__ __forceinline__ NewTokens new_tokens(const int* cu, int b, int total, int max_new, int len) {
  NewTokens t;
  t.begin = cu ? min(max(cu[b], 0), total) : b;
  const int end = cu ? min(max(cu[b + 1], t.begin), total) : min(b + 1, total);
  t.count = min(min(max(end - t.begin, 0), max_new), len);
  t.first = len - t.count;
  return t;
}

// ---------------------------------------------------------------------------
// Append, HIF4.  One workgroup per (sequence, page that the new tokens touch,
// head).  K~ = fp16(k/s) is quantized along the channels, a key's words written
// to its row of the record; V is quantized along the 64 tokens of the page,
// from the new tokens and, before them in the page, from the fp16 rows that
// the tail keeps of the open page, places behind the last token zero: the page
// holds at any time what quantizing the whole sequence would give.
// Metadata bits are gathered in LDS and the page's parts written whole.
template <int G>
__global__ void __launch_bounds__(256) k_paged_append(PagedAppend a, int blocks) {
  constexpr int D = 64 * G, kMeta = 256 * G;
  __shared__ uint32_t meta_k[kMeta / 4], meta_v[kMeta / 4];
  __shared__ __align__(16) uint32_t codes_v[2048 * G / 4];
  const int tid = threadIdx.x;
  const int head = blockIdx.x % a.c.hkv;
  const int blk = (blockIdx.x / a.c.hkv) % blocks, b = blockIdx.x / a.c.hkv / blocks;
  const int len = paged_len(a.c, b);
  const NewTokens nt = new_tokens(a.cu, b, a.total, a.max_new, len);
  const int place = nt.first / kPage + blk, p0 = place * kPage;
  if (nt.count == 0 || p0 >= len) return;
  const int lo = max(nt.first - p0, 0), hi = min(len - p0, kPage);     // new keys of the page: [lo, hi)
  uint8_t* rec = paged_record(a.c, b, place, head);
  const size_t row = (size_t)a.c.hkv * D;
  // the new token at key 0 of the page (it may lie before the input: only keys >= lo are read)
  const long t0 = (long)nt.begin + p0 - nt.first;
  half_t* tail = a.c.tail + ((size_t)b * kPage * a.c.hkv + head) * D;

  // metadata: K's as it stands for the keys before lo, nothing for the others
  for (int i = tid; i < kMeta / 4; i += 256) {
    uint32_t w = 0;
    if (lo > 0 && rec) {
      w = reinterpret_cast<const uint32_t*>(rec + 2048 * G)[i];
      uint32_t keep = 0;
      for (int j = 0; j < 4; ++j) {
        const int at = 4 * i + j;
        if (at < 192 * G) {                                  // E3 or E2: bits 2t + c of a lane
          const int n = (at < 128 * G ? at / (2 * G) : (at - 128 * G) / G) & 15;
          for (int t = 0; t < 4; ++t)
            if (key_of(t, n) < lo) keep |= 3u << (8 * j + 2 * t);
        } else {
          const int x = at - 192 * G, n = 4 * (x / (16 * G)) + (x & 3), t = (x >> 2) & 3;
          if (key_of(t, n) < lo) keep |= 0xFFu << (8 * j);
        }
      }
      w &= keep;
    }
    meta_k[i] = w;
    meta_v[i] = 0;
  }
  __syncthreads();

  // K: eight lanes a group
  for (int i = tid; i < (hi - lo) * 8 * G; i += 256) {
    const int key = lo + i / (8 * G), g = (i >> 3) % G, w = i & 7;
    const uint4 in = *reinterpret_cast<const uint4*>(a.k + (size_t)(t0 + key) * row + (size_t)head * D + 64 * g + 8 * w);
    h2_t x[4] = {__builtin_bit_cast(h2_t, in.x), __builtin_bit_cast(h2_t, in.y), __builtin_bit_cast(h2_t, in.z),
                 __builtin_bit_cast(h2_t, in.w)};
    if (a.s) {
      const float* sp = a.s + (size_t)head * D + 64 * g + 8 * w;
      float sc[8], rc[8];
      for (int e = 0; e < 8; ++e) {
        sc[e] = sp[e];
        rc[e] = 1.0f / sc[e];
      }
      divide_pairs(x, sc, rc);
    }
    h2_t m[4];
    for (int e = 0; e < 4; ++e) m[e] = habs2(x[e]);
    const h2_t a4 = hmax_pairs(hmax2(m[0], m[1]), hmax2(m[2], m[3]));
    const u16x2_t a8u = __builtin_elementwise_max(as_u16(a4), __builtin_shufflevector(as_u16(a4), as_u16(a4), 1, 0));
    const uint32_t gm = reduce8(__builtin_bit_cast(uint32_t, a8u), [](uint32_t p, uint32_t q) {
      return __builtin_bit_cast(
          uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, p), __builtin_bit_cast(u16x2_t, q)));
    });
    const uint32_t base = e6m2_ceil((float)__builtin_bit_cast(h2_t, gm)[0]);
    const float R = hif4_rcp_step(base);
    const h2_t thr = range_floors(e6m2_value(base));
    u16x2_t lv, ne2;
    block_levels(a4, __builtin_bit_cast(h2_t, a8u), h2_t{thr[0], thr[0]}, h2_t{thr[1], thr[1]}, lv, ne2);
    uint32_t word = 0;
    for (int e = 0; e < 4; ++e) {
      const unsigned short ne = lv[e >> 1];
      const uint32_t nib = nibbles2(codes2(m[e], R, R, u16x2_t{ne, ne}), x[e]);
      word |= ((nib | (nib >> 12)) & 0xFFu) << (8 * e);
    }
    const int t = key_t(key), n = key_n(key), lane = 16 * (w >> 1) + n, bit = 2 * t + (w & 1);
    if (rec) *reinterpret_cast<uint32_t*>(rec + hif4_code_at(g, t, lane, w & 1)) = word;
    const uint32_t e2 = 1u - ne2[0], e3a = 2u - lv[0] - e2, e3b = 2u - lv[1] - e2;
    const int a3 = hif4_e3_at(G, g, lane, 0) - 2048 * G, b3 = hif4_e3_at(G, g, lane, 1) - 2048 * G;
    const int a2 = hif4_e2_at(G, g, lane) - 2048 * G, ab = hif4_base_at(G, g, t, n) - 2048 * G;
    atomicOr(&meta_k[a3 >> 2], e3a << (8 * (a3 & 3) + bit));
    atomicOr(&meta_k[b3 >> 2], e3b << (8 * (b3 & 3) + bit));
    atomicOr(&meta_k[a2 >> 2], e2 << (8 * (a2 & 3) + bit));
    if (w == 0) atomicOr(&meta_k[ab >> 2], base << (8 * (ab & 3)));
  }

  // V: a lane takes 8 keys of 4 channels, eight lanes a group
  for (int i = tid; i < 128 * G; i += 256) {
    const int w = i & 7, ch = 4 * (i >> 3);
    h2_t x[8][2];
    for (int e = 0; e < 8; ++e) {
      const int key = 8 * w + e;
      uint2 in = make_uint2(0, 0);
      if (key < hi)
        in = key >= lo ? *reinterpret_cast<const uint2*>(a.v + (size_t)(t0 + key) * row + (size_t)head * D + ch)
                       : *reinterpret_cast<const uint2*>(tail + (size_t)key * row + ch);
      x[e][0] = __builtin_bit_cast(h2_t, in.x);
      x[e][1] = __builtin_bit_cast(h2_t, in.y);
    }
    for (int p = 0; p < 2; ++p) {
      h2_t a4[2];
      for (int q = 0; q < 2; ++q)
        a4[q] = hmax2(hmax2(habs2(x[4 * q][p]), habs2(x[4 * q + 1][p])),
                      hmax2(habs2(x[4 * q + 2][p]), habs2(x[4 * q + 3][p])));
      const u16x2_t a8u = __builtin_elementwise_max(as_u16(a4[0]), as_u16(a4[1]));
      const uint32_t gm = reduce8(__builtin_bit_cast(uint32_t, a8u), [](uint32_t y, uint32_t z) {
        return __builtin_bit_cast(
            uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, y), __builtin_bit_cast(u16x2_t, z)));
      });
      const h2_t top = __builtin_bit_cast(h2_t, gm);
      const uint32_t base[2] = {e6m2_ceil((float)top[0]), e6m2_ceil((float)top[1])};
      const float r0 = hif4_rcp_step(base[0]), r1 = hif4_rcp_step(base[1]);
      const h2_t f0 = range_floors(e6m2_value(base[0])), f1 = range_floors(e6m2_value(base[1]));
      uint32_t acc[2] = {0, 0};            // four keys' nibbles per channel, in the two halves
      uint32_t e2 = 0, e3[2];
      for (int q = 0; q < 2; ++q) {
        u16x2_t lv, ne2;
        block_levels(a4[q], __builtin_bit_cast(h2_t, a8u), h2_t{f0[0], f1[0]}, h2_t{f0[1], f1[1]}, lv, ne2);
        for (int e = 0; e < 4; ++e)
          acc[q] |= nibbles2(codes2(habs2(x[4 * q + e][p]), r0, r1, lv), x[4 * q + e][p]) << (4 * e);
        e2 = 0x00010001u - __builtin_bit_cast(uint32_t, ne2);
        e3[q] = 0x00020002u - __builtin_bit_cast(uint32_t, lv) - e2;
      }
      for (int e = 0; e < 2; ++e) {
        const int c = ch + 2 * p + e, tile = c >> 6, t = (c >> 4) & 3, n = c & 15;
        const int lane = 16 * (w >> 1) + n, bit = 2 * t + (w & 1);
        const uint32_t word = e ? (acc[0] >> 16) | (acc[1] & 0xFFFF0000u) : (acc[0] & 0xFFFFu) | (acc[1] << 16);
        codes_v[hif4_code_at(tile, t, lane, w & 1) >> 2] = word;
        const int a3 = hif4_e3_at(G, tile, lane, 0) - 2048 * G, b3 = hif4_e3_at(G, tile, lane, 1) - 2048 * G;
        const int a2 = hif4_e2_at(G, tile, lane) - 2048 * G, ab = hif4_base_at(G, tile, t, n) - 2048 * G;
        atomicOr(&meta_v[a3 >> 2], ((e3[0] >> (16 * e)) & 1u) << (8 * (a3 & 3) + bit));
        atomicOr(&meta_v[b3 >> 2], ((e3[1] >> (16 * e)) & 1u) << (8 * (b3 & 3) + bit));
        atomicOr(&meta_v[a2 >> 2], ((e2 >> (16 * e)) & 1u) << (8 * (a2 & 3) + bit));
        if (w == 0) atomicOr(&meta_v[ab >> 2], base[e] << (8 * (ab & 3)));
      }
    }
  }
  __syncthreads();
  if (rec) {
    uint8_t* vp = rec + hif4_part(G);
    for (int i = tid; i < 2048 * G / 16; i += 256)
      reinterpret_cast<uint4*>(vp)[i] = reinterpret_cast<const uint4*>(codes_v)[i];
    for (int i = tid; i < kMeta / 4; i += 256) {
      reinterpret_cast<uint32_t*>(rec + 2048 * G)[i] = meta_k[i];
      reinterpret_cast<uint32_t*>(vp + 2048 * G)[i] = meta_v[i];
    }
  }
  // The tail gets the last page's new rows.  The workgroup of the first page
  // writes them: it alone reads the tail, and has done so before the barrier.
  if (blk == 0) {
    const int last = (len - 1) / kPage * kPage;               // place of the last page's first token
    const int from = max(nt.first - last, 0), to = len - last;
    const long l0 = (long)nt.begin + last - nt.first;
    for (int i = tid; i < (to - from) * (D / 8); i += 256) {
      const int key = from + i / (D / 8), ch = 8 * (i % (D / 8));
      *reinterpret_cast<uint4*>(tail + (size_t)key * row + ch) =
          *reinterpret_cast<const uint4*>(a.v + (size_t)(l0 + key) * row + (size_t)head * D + ch);
    }
  }
}

// Append, FP16: the new tokens' K~ and V go to their places in the record.
__global__ void __launch_bounds__(256) k_paged_append16(PagedAppend a, int blocks) {
  const int tid = threadIdx.x, D = a.c.D;
  const int head = blockIdx.x % a.c.hkv;
  const int blk = (blockIdx.x / a.c.hkv) % blocks, b = blockIdx.x / a.c.hkv / blocks;
  const int len = paged_len(a.c, b);
  const NewTokens nt = new_tokens(a.cu, b, a.total, a.max_new, len);
  const int place = nt.first / kPage + blk, p0 = place * kPage;
  if (nt.count == 0 || p0 >= len) return;
  const int lo = max(nt.first - p0, 0), hi = min(len - p0, kPage);
  uint8_t* rec = paged_record(a.c, b, place, head);
  if (!rec) return;
  const size_t row = (size_t)a.c.hkv * D;
  const long t0 = (long)nt.begin + p0 - nt.first;
  half_t* rk = reinterpret_cast<half_t*>(rec);
  half_t* rv = rk + 64 * D;
  for (int i = tid; i < (hi - lo) * (D / 8); i += 256) {
    const int key = lo + i / (D / 8), ch = 8 * (i % (D / 8));
    const size_t at = (size_t)(t0 + key) * row + (size_t)head * D + ch;
    alignas(16) half_t x[8], y[8];
    *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(a.k + at);
    *reinterpret_cast<uint4*>(y) = *reinterpret_cast<const uint4*>(a.v + at);
    if (a.s)
      for (int e = 0; e < 8; ++e) x[e] = div_rn16((float)x[e], a.s[(size_t)head * D + ch + e]);
    const int t = key_t(key), n = key_n(key);
    *reinterpret_cast<uint4*>(rk + (((size_t)t * (D / 32) + ch / 32) * 64 + 16 * (ch / 8 % 4) + n) * 8) =
        *reinterpret_cast<uint4*>(x);
    for (int e = 0; e < 8; ++e) {
      const int c = ch + e;
      rv[(((size_t)(c / 16) * 2 + (key >> 3 & 1)) * 64 + 16 * (key >> 4) + (c & 15)) * 8 + (key & 7)] = y[e];
    }
  }
}

hipError_t launch_paged_append(const PagedAppend& a, hipStream_t st) {
  // pages that max_new tokens can touch from any place in a page
  const int blocks = (a.max_new + kPage - 2) / kPage + 1;
  const dim3 grid((unsigned)((size_t)a.c.batch * blocks * a.c.hkv));
  if (a.c.fp16)
    k_paged_append16<<<grid, 256, 0, st>>>(a, blocks);
  else if (a.c.D == 64)
    k_paged_append<1><<<grid, 256, 0, st>>>(a, blocks);
  else if (a.c.D == 128)
    k_paged_append<2><<<grid, 256, 0, st>>>(a, blocks);
  else
    k_paged_append<4><<<grid, 256, 0, st>>>(a, blocks);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Gather: tokens [start, start + n) of each sequence as fp16 rows.  One
// workgroup per (sequence, page, head).  Tokens behind the sequence's end and
// tokens of places without a page are zeros.
__device__ __forceinline__ float hif4_value(const uint8_t* part, int G, int tile, int t, int n, int elem) {
  const int w = elem >> 3, i = elem & 7, lane = 16 * (w >> 1) + n, bit = 2 * t + (w & 1);
  const uint32_t nib = (part[hif4_code_at(tile, t, lane, w & 1) + (i >> 1)] >> (4 * (i & 1))) & 15u;
  const int sh = ((part[hif4_e2_at(G, tile, lane)] >> bit) & 1) + ((part[hif4_e3_at(G, tile, lane, i >> 2)] >> bit) & 1);
  const float x = (float)(nib & 7u) * e6m2_value(part[hif4_base_at(G, tile, t, n)]) * (sh == 0 ? 0.25f : sh == 1 ? 0.125f : 0.0625f);
  return nib & 8u ? -x : x;
}

__global__ void __launch_bounds__(256) k_paged_gather(PagedGather a, int blocks) {
  const int tid = threadIdx.x, D = a.c.D, G = D / 64;
  const int head = blockIdx.x % a.c.hkv;
  const int blk = (blockIdx.x / a.c.hkv) % blocks, b = blockIdx.x / a.c.hkv / blocks;
  const int begin = min(max(a.cu[b], 0), a.total);
  const int count = min(min(max(a.cu[b + 1], begin), a.total) - begin, a.max_tokens);
  const int start = a.starts ? max(a.starts[b], 0) : 0;
  const int place = start / kPage + blk;
  const long p0 = (long)place * kPage;
  const int lo = (int)max((long)start - p0, 0L), hi = (int)min((long)start + count - p0, (long)kPage);
  if (hi <= lo) return;
  const int held = (int)min(max((long)paged_len(a.c, b) - p0, 0L), (long)kPage);      // keys of the page that exist
  const uint8_t* rec = held > 0 ? paged_record(a.c, b, place, head) : nullptr;
  const size_t row = (size_t)a.c.hkv * D;
  for (int i = tid; i < (hi - lo) * (D / 8); i += 256) {
    const int key = lo + i / (D / 8), ch = 8 * (i % (D / 8));
    const int t = key_t(key), n = key_n(key);
    alignas(16) half_t x[8], y[8];
    for (int e = 0; e < 8; ++e) {
      x[e] = y[e] = (half_t)0;
      if (!rec || key >= held) continue;
      const int c = ch + e;
      if (a.c.fp16) {
        const half_t* rk = reinterpret_cast<const half_t*>(rec);
        x[e] = rk[(((size_t)t * (D / 32) + c / 32) * 64 + 16 * (c / 8 % 4) + n) * 8 + (c & 7)];
        y[e] = rk[64 * D + (((size_t)(c / 16) * 2 + (key >> 3 & 1)) * 64 + 16 * (key >> 4) + (c & 15)) * 8 + (key & 7)];
      } else {
        x[e] = (half_t)hif4_value(rec, G, c >> 6, t, n, c & 63);
        y[e] = (half_t)hif4_value(rec + hif4_part(G), G, c >> 6, (c >> 4) & 3, c & 15, key);
      }
    }
    const size_t at = (size_t)(begin + p0 + key - start) * row + (size_t)head * D + ch;
    *reinterpret_cast<uint4*>(a.k + at) = *reinterpret_cast<uint4*>(x);
    *reinterpret_cast<uint4*>(a.v + at) = *reinterpret_cast<uint4*>(y);
  }
}

hipError_t launch_paged_gather(const PagedGather& a, hipStream_t st) {
  const int blocks = (a.max_tokens + kPage - 2) / kPage + 1;
  k_paged_gather<<<dim3((unsigned)((size_t)a.c.batch * blocks * a.c.hkv)), 256, 0, st>>>(a, blocks);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Eviction.  One workgroup per sequence.  Of the pages between the first and
// the last ones that stay, the budget's remaining places go to the largest
// weights, equal ones to the lowest place.  The weight at the border is found
// digit by digit (8 bits at a time, by counts), then one pass over the places
// moves what stays and lists what leaves, both in order.
constexpr int kEvictThreads = 1024;

// Order of the weights as unsigned integers; NaN below everything, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Inclusive sum over the workgroup of a count per thread (< 2^16 in all), in
// two 16-bit halves.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* sums, uint32_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
  for (int i = 0; i < kEvictThreads / 64; ++i) {
    if (i < wave) before += sums[i];
    total += sums[i];
  }
  return x + before;
}

__global__ void __launch_bounds__(kEvictThreads) k_paged_evict(PagedEvict a) {
  __shared__ uint32_t hist[256], sums[kEvictThreads / 64], found[2];
  const int b = blockIdx.x, tid = threadIdx.x;
  const size_t row = (size_t)b * a.max_pages;
  const int len = max(0, min(a.lens[b], a.max_pages * kPage));
  const int pages = (len + kPage - 1) / kPage;
  const int lo = a.first, hi = pages - a.last;               // contenders: [lo, hi)
  uint32_t border = 0;                                       // keys above stay, keys equal to it while `ties` last
  int left = a.budget - a.first - a.last, ties = 0x7FFFFFFF;
  if (pages > a.budget) {
    if (left == 0) {
      border = 0xFFFFFFFFu;
      ties = 0;
    } else {
      for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i = lo + tid; i < hi; i += kEvictThreads) {
          const uint32_t k = weight_key(a.w[row + i]);
          if (shift == 24 || (k >> (shift + 8)) == (border >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (tid == 0) {
          int need = left, d = 255;
          while (d > 0 && (int)hist[d] < need) need -= (int)hist[d--];
          found[0] = (uint32_t)d;
          found[1] = (uint32_t)need;
        }
        __syncthreads();
        border |= found[0] << shift;
        left = (int)found[1];
      }
      ties = left;
    }
  }
  // one pass in order; what is written lies at or before what has been read
  int kept = 0, gone = 0, tied = 0;
  for (int i0 = 0; i0 < pages; i0 += kEvictThreads) {
    const int i = i0 + tid;
    int page = -1;
    float w = 0.0f;
    bool there = i < pages, fixed = false, equal = false, above = false;
    if (there) {
      page = a.table[row + i];
      w = a.w[row + i];
      const uint32_t k = weight_key(w);
      fixed = pages <= a.budget || i < lo || i >= hi;
      equal = !fixed && k == border;
      above = !fixed && k > border;
    }
    uint32_t total;
    const uint32_t before = block_scan(equal, sums, total) - equal;
    const bool keep = there && (fixed || above || (equal && tied + (int)before < ties));
    tied += (int)total;
    const uint32_t gone_here = there && !keep;
    const uint32_t at = block_scan((uint32_t)keep | (gone_here << 16), sums, total);
    if (keep) {
      const size_t to = row + kept + (at & 0xFFFFu) - 1;
      a.out_table[to] = page;
      a.out_w[to] = w;
    } else if (gone_here) {
      a.freed[row + gone + (at >> 16) - 1] = page;
    }
    kept += (int)(total & 0xFFFFu);
    gone += (int)(total >> 16);
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
