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
__device__ __forceinline__ uint32_t or_pair(uint32_t v) {            // with the neighbouring lane
  return v | (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);
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
// A thread holds whole words (eight channels of a key of K, eight keys of four
// channels of V), eight lanes a group; all its loads are issued before the
// first is used.  Metadata bits are gathered in LDS (the two words of a lane of
// the record are neighbours: one of them writes for both) and the page's parts
// written whole.
// Bound by HBM: 16 prompts of 512 to 2048 tokens, 8 heads, D=128 (107 MB).
template <int G>
__global__ void __launch_bounds__(256) k_paged_append(PagedAppend a, int blocks) {
  constexpr int D = 64 * G, kMeta = 256 * G, kWordsK = 2 * G, kItemsV = (G + 1) / 2;
  __shared__ uint32_t meta_k[kMeta / 4], meta_v[kMeta / 4];
  __shared__ __align__(16) uint32_t codes_k[2048 * G / 4], codes_v[2048 * G / 4];
  const int tid = threadIdx.x;
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

  // K: word w of group g of the keys key0, key0 + 32 / G, ...
  const int w = tid & 7, g = (tid >> 3) % G, key0 = lo + tid / (8 * G);
  uint4 in_k[kWordsK];
#pragma unroll
  for (int i = 0; i < kWordsK; ++i) {
    const int key = min(key0 + i * (32 / G), hi - 1);
    in_k[i] = *reinterpret_cast<const uint4*>(a.k + (size_t)(t0 + key) * row + (size_t)it.head * D + 64 * g + 8 * w);
  }
  // V: keys 8w .. 8w+7 of four channels
  uint2 in_v[kItemsV][8];
#pragma unroll
  for (int i = 0; i < kItemsV; ++i) {
    const int ch = 4 * (tid >> 3) + 128 * i;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int key = 8 * w + e;
      in_v[i][e] = make_uint2(0, 0);
      if (key < hi && ch < D)
        in_v[i][e] = key >= lo ? *reinterpret_cast<const uint2*>(a.v + (size_t)(t0 + key) * row + (size_t)it.head * D + ch)
                               : *reinterpret_cast<const uint2*>(tail + (size_t)key * row + ch);
    }
  }
  // metadata: K's as it stands for the keys before lo, nothing for the others
  for (int i = tid; i < kMeta / 4; i += 256) {
    uint32_t x = 0;
    if (lo > 0 && rec) {
      x = reinterpret_cast<const uint32_t*>(rec + 2048 * G)[i];
      uint32_t keep = 0;
      for (int j = 0; j < 4; ++j) {
        const int at = 4 * i + j;
        if (at < 192 * G) {                                  // E3 or E2: bits 2t + c of a lane
          const int n = (at < 128 * G ? at / (2 * G) : (at - 128 * G) / G) & 15;
          for (int t = 0; t < 4; ++t)
            if (key_of(t, n) < lo) keep |= 3u << (8 * j + 2 * t);
        } else {
          const int y = at - 192 * G, n = 4 * (y / (16 * G)) + (y & 3), t = (y >> 2) & 3;
          if (key_of(t, n) < lo) keep |= 0xFFu << (8 * j);
        }
      }
      x &= keep;
    }
    meta_k[i] = x;
    meta_v[i] = 0;
  }
  __syncthreads();
  uint8_t* bytes_k = reinterpret_cast<uint8_t*>(meta_k);
  uint8_t* bytes_v = reinterpret_cast<uint8_t*>(meta_v);

  {
    float sc[8], rc[8];
    if (a.s) {
      const float4* sp = reinterpret_cast<const float4*>(a.s + (size_t)it.head * D + 64 * g + 8 * w);
      const float4 s0 = sp[0], s1 = sp[1];
      const float s[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sc[e] = s[e];
        rc[e] = 1.0f / s[e];
      }
    }
#pragma unroll
    for (int i = 0; i < kWordsK; ++i) {
      const int key = key0 + i * (32 / G);
      if (key >= hi) break;                                  // whole sets of eight lanes
      h2_t x[4] = {__builtin_bit_cast(h2_t, in_k[i].x), __builtin_bit_cast(h2_t, in_k[i].y),
                   __builtin_bit_cast(h2_t, in_k[i].z), __builtin_bit_cast(h2_t, in_k[i].w)};
      if (a.s) divide_pairs(x, sc, rc);
      h2_t m[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) m[e] = habs2(x[e]);
      const h2_t a4 = hmax_pairs(hmax2(m[0], m[1]), hmax2(m[2], m[3]));
      const u16x2_t a8u = __builtin_elementwise_max(as_u16(a4), __builtin_shufflevector(as_u16(a4), as_u16(a4), 1, 0));
      const uint32_t gm = reduce8(__builtin_bit_cast(uint32_t, a8u), max_pair16);
      const uint32_t base = e6m2_ceil((float)__builtin_bit_cast(h2_t, gm)[0]);
      const float R = hif4_rcp_step(base);
      const h2_t thr = range_floors(e6m2_value(base));
      u16x2_t lv, ne2;
      block_levels(a4, __builtin_bit_cast(h2_t, a8u), h2_t{thr[0], thr[0]}, h2_t{thr[1], thr[1]}, lv, ne2);
      uint32_t word = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned short ne = lv[e >> 1];
        const uint32_t nib = nibbles2(codes2(m[e], R, R, u16x2_t{ne, ne}), x[e]);
        word |= ((nib | (nib >> 12)) & 0xFFu) << (8 * e);
      }
      const int t = key_t(key), n = key_n(key), lane = 16 * (w >> 1) + n, bit = 2 * t + (w & 1);
      codes_k[hif4_code_at(g, t, lane, w & 1) >> 2] = word;
      const uint32_t e2 = 1u - ne2[0], e3 = (2u - lv[0] - e2) | (2u - lv[1] - e2) << (G == 1 ? 8 : 16);
      const int a3 = hif4_e3_at(G, g, lane, 0) - 2048 * G, a2 = hif4_e2_at(G, g, lane) - 2048 * G;
      const uint32_t b3 = or_pair(e3 << (8 * (a3 & 3) + bit)), b2 = or_pair(e2 << (8 * (a2 & 3) + bit));
      if ((w & 1) == 0) {
        atomicOr(&meta_k[a3 >> 2], b3);
        atomicOr(&meta_k[a2 >> 2], b2);
      }
      if (w == 0) bytes_k[hif4_base_at(G, g, t, n) - 2048 * G] = (uint8_t)base;
    }
  }

#pragma unroll
  for (int i = 0; i < kItemsV; ++i) {
    const int ch = 4 * (tid >> 3) + 128 * i;
    if (ch >= D) break;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      h2_t x[8], a4[2];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = __builtin_bit_cast(h2_t, p ? in_v[i][e].y : in_v[i][e].x);
#pragma unroll
      for (int q = 0; q < 2; ++q)
        a4[q] = hmax2(hmax2(habs2(x[4 * q]), habs2(x[4 * q + 1])), hmax2(habs2(x[4 * q + 2]), habs2(x[4 * q + 3])));
      const u16x2_t a8u = __builtin_elementwise_max(as_u16(a4[0]), as_u16(a4[1]));
      const h2_t top = __builtin_bit_cast(h2_t, reduce8(__builtin_bit_cast(uint32_t, a8u), max_pair16));
      const uint32_t base[2] = {e6m2_ceil((float)top[0]), e6m2_ceil((float)top[1])};
      const float r0 = hif4_rcp_step(base[0]), r1 = hif4_rcp_step(base[1]);
      const h2_t f0 = range_floors(e6m2_value(base[0])), f1 = range_floors(e6m2_value(base[1]));
      uint32_t acc[2] = {0, 0};            // four keys' nibbles per channel, in the two halves
      uint32_t e2 = 0, e3[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        u16x2_t lv, ne2;
        block_levels(a4[q], __builtin_bit_cast(h2_t, a8u), h2_t{f0[0], f1[0]}, h2_t{f0[1], f1[1]}, lv, ne2);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[q] |= nibbles2(codes2(habs2(x[4 * q + e]), r0, r1, lv), x[4 * q + e]) << (4 * e);
        e2 = 0x00010001u - __builtin_bit_cast(uint32_t, ne2);
        e3[q] = 0x00020002u - __builtin_bit_cast(uint32_t, lv) - e2;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int c = ch + 2 * p + e, tile = c >> 6, t = (c >> 4) & 3, n = c & 15;
        const int lane = 16 * (w >> 1) + n, bit = 2 * t + (w & 1);
        codes_v[hif4_code_at(tile, t, lane, w & 1) >> 2] =
            __builtin_amdgcn_perm(acc[1], acc[0], e ? 0x07060302u : 0x05040100u);
        const int a3 = hif4_e3_at(G, tile, lane, 0) - 2048 * G, a2 = hif4_e2_at(G, tile, lane) - 2048 * G;
        const uint32_t both = ((e3[0] >> (16 * e)) & 1u) | ((e3[1] >> (16 * e)) & 1u) << (G == 1 ? 8 : 16);
        const uint32_t b3 = or_pair(both << (8 * (a3 & 3) + bit));
        const uint32_t b2 = or_pair(((e2 >> (16 * e)) & 1u) << (8 * (a2 & 3) + bit));
        if ((w & 1) == 0) {
          atomicOr(&meta_v[a3 >> 2], b3);
          atomicOr(&meta_v[a2 >> 2], b2);
        }
        if (w == 0) bytes_v[hif4_base_at(G, tile, t, n) - 2048 * G] = (uint8_t)base[e];
      }
    }
  }
  __syncthreads();
  if (rec) {
    uint8_t* vp = rec + hif4_part(G);
#pragma unroll
    for (int i = tid; i < 2048 * G / 16; i += 256) {
      reinterpret_cast<uint4*>(vp)[i] = reinterpret_cast<const uint4*>(codes_v)[i];
      // of K the words of the new keys: 16 bytes are two keys' (t even, t odd)
      const uint4 x = reinterpret_cast<const uint4*>(codes_k)[i];
      const int t = 2 * ((i >> 6) & 1), ka = key_of(t, i & 15), kb = key_of(t + 1, i & 15);
      const bool na = ka >= lo && ka < hi, nb = kb >= lo && kb < hi;
      if (na && nb)
        reinterpret_cast<uint4*>(rec)[i] = x;
      else if (na)
        reinterpret_cast<uint2*>(rec)[2 * i] = make_uint2(x.x, x.y);
      else if (nb)
        reinterpret_cast<uint2*>(rec)[2 * i + 1] = make_uint2(x.z, x.w);
    }
    for (int i = tid; i < kMeta / 4; i += 256) {
      reinterpret_cast<uint32_t*>(rec + 2048 * G)[i] = meta_k[i];
      reinterpret_cast<uint32_t*>(vp + 2048 * G)[i] = meta_v[i];
    }
  }
  // The tail gets the last page's new rows.  The workgroup of the first page
  // writes them: it alone reads the tail, and has done so before the barrier.
  if (it.blk == 0) {
    const int last = (stop - 1) / kPage * kPage;              // place of the last page's first token
    const int from = max(nt.first - last, 0), to = stop - last;
    const long l0 = (long)nt.begin + last - nt.first;
    for (int i = tid; i < (to - from) * (D / 8); i += 256) {
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
// unfinished sets of eight keys are 16 bytes wide (8 for V's rows).
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
  if (a.c.fp16) {
    if (a.c.D == 64)
      k_paged_append16<1><<<grid, 256, 0, st>>>(a, blocks);
    else if (a.c.D == 128)
      k_paged_append16<2><<<grid, 256, 0, st>>>(a, blocks);
    else
      k_paged_append16<4><<<grid, 256, 0, st>>>(a, blocks);
  } else {
    if (a.c.D == 64)
      k_paged_append<1><<<grid, 256, 0, st>>>(a, blocks);
    else if (a.c.D == 128)
      k_paged_append<2><<<grid, 256, 0, st>>>(a, blocks);
    else
      k_paged_append<4><<<grid, 256, 0, st>>>(a, blocks);
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
// u b/4 2^-(E2+E3), whole in fp32, rounded once.  Bound by HBM: mostly the
// writes.
__device__ __forceinline__ int padded(int at) { return at + (at >> 8) * 16; }

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
// latency: four counts and one pass, three barriers each.
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
