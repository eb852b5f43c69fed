// Attention of each sequence's last tokens over the paged cache (records:
// hifa4_paged.h): chunks of prompts, drafted tokens, one token of each, mixed.
//
// Sequence b holds L tokens, its n new ones among them; query i < n stands at
// position L - n + i and sees the keys up to it:
//   S_j = (q~ . k_j) / sqrt(D),  p_j = exp(S_j - m) / l,  o = sum_j p_j v_j,
//   LSE = m + ln l,  with m = max S_j and l = sum_j exp(S_j - m).
// q~ = fp16(q s) under Smooth-QK.  The products run on fp16 operands with sums in
// fp32: q~ is fp16, and so is a cached HIF4 value (six significant bits; below
// 2^-14 it is rounded by up to 2^-24).  Scores, softmax state and o are held in
// fp32; p is rounded to fp16 for the second product, relative to the heaviest key
// so far (2^7 to 2^15), and o is divided by the sum of the rounded p: a row that
// rests on one key has exactly that key's value.  LSE takes the sum of p itself.
//
// The rows of a sequence, (token, query head of the kv head), are cut into tiles,
// and a tile's pages into runs where there are too few tiles to fill the chip; a
// second kernel joins the runs of a row.  Lengths and counts are read on the
// device, so a captured call follows them.
#include "hifa4_paged_device.h"

#include <algorithm>

namespace hifa4 {

typedef half_t h4v_t __attribute__((ext_vector_type(4)));

// What the heaviest key so far counts: between 2^kTop and 2^(kTop + kSlack), below
// fp16's range; the softmax's reference moves when a score passes that.
constexpr float kTop = 7.0f, kSlack = 8.0f;
constexpr float kNoRef = -1e30f;        // before any key

// ---------------------------------------------------------------------------
// The plan: items (sequence, tile of rows, run of pages), the same for every kv head.
// Sequences of few rows and of many are cut apart, each kind by its own kernel's sizes.
constexpr int kMinRun = 4;              // pages that a run has at least, on average

// How one kind's work is cut: rows a tile, items aimed at, and its bounds (per kv head).
// A tile of P pages has at most 1 + P / per runs and, where it is split, fewer than
// 2 P / per; sum P / per over the tiles is at most the target (in fp32: and one more).
struct ChunkCut {
  int rows, target;
  int above, upto;                      // sequences of more than `above` rows and at most `upto`
  int items, slots, joins;              // items, runs of split tiles, split tiles: at most
};
struct ChunkSeq {
  int first, n;                         // row of q, new tokens (those that the launch holds)
  int len, base;                        // cached tokens, position of the first new one
};
struct Item {
  int b, tile, run, runs;
  int begin, end;                       // pages
  int slot, join;                       // of the tile's first run, and its place among the split tiles; -1: not split
  ChunkSeq seq;
};

// Counts outside the contract are cut, so that no access leaves q, o and lse.
__device__ __forceinline__ ChunkSeq chunk_seq(const PagedChunk& a, int b) {
  ChunkSeq s = {0, 0, 0, 0};
  if (b < a.c.batch) {
    s.first = max(0, min(a.cu[b], a.total));
    const int n = max(0, min(a.cu[b + 1], a.total) - s.first);
    s.n = min(n, a.max_new);
    s.len = paged_len(a.c, b);
    s.base = s.len - n;
  }
  return s;
}
__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }
__device__ __forceinline__ int tiles_of(const ChunkSeq& s, int group, const ChunkCut& cut) {
  const int rows = s.n * group;
  return rows > cut.above && rows <= cut.upto ? ceil_div(rows, cut.rows) : 0;
}
// Pages that the rows of a tile see.
__device__ __forceinline__ int tile_pages(const ChunkSeq& s, int group, const ChunkCut& cut, int tile) {
  const int last = min(s.n - 1, ((tile + 1) * cut.rows - 1) / group);
  return max(0, s.base + last + kPage) / kPage;
}
// Sum over the wave, the same bits in every lane.
template <int kCtrl, int kRowMask, bool kBound>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), kCtrl, kRowMask, 0xF, kBound));
}
__device__ __forceinline__ float wave_sum(float x) {
  x = add_dpp<0x111, 0xF, true>(x);      // row_shr 1, 2, 4, 8
  x = add_dpp<0x112, 0xF, true>(x);
  x = add_dpp<0x114, 0xF, true>(x);
  x = add_dpp<0x118, 0xF, true>(x);
  x = add_dpp<0x142, 0xA, false>(x);     // lane 15 of each row to the next
  x = add_dpp<0x143, 0xC, false>(x);
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), 63));
}

// The item numbered r (found by a whole wave); false: no such item.  `joins`: the
// split tiles.  There are no items at all where the counts are no prefix sums of
// `total` (more rows than the launch and the workspace were sized for).
__device__ __forceinline__ bool find_item(const PagedChunk& a, int group, const ChunkCut& cut, int r, int lane, Item& it, int& joins) {
  const ChunkSeq held = chunk_seq(a, lane);                 // the first 64 sequences are read once
  const auto seq = [&](int b) { return b < 64 ? held : chunk_seq(a, b); };
  float work = 0.0f, tokens = 0.0f;
  for (int b = lane; b < a.c.batch; b += 64) {
    const ChunkSeq s = seq(b);
    tokens += (float)s.n;
    work += (float)tiles_of(s, group, cut) * (float)ceil_div(s.len, kPage);
  }
  joins = 0;
  if (wave_sum(tokens) > (float)a.total * 1.001f) return false;
  const int per = max(kMinRun, (int)ceilf(fminf(wave_sum(work) / (float)cut.target, 0x1p25f)));
  const auto runs_of = [per](const ChunkSeq& s) { return max(1, ceil_div(ceil_div(s.len, kPage), per)); };
  int items = 0, tiles = 0, slots = 0;
  for (int b = lane; b < a.c.batch; b += 64) {
    const ChunkSeq s = seq(b);
    const int t = tiles_of(s, group, cut), n = runs_of(s);
    items += t * n;
    if (n > 1) {
      tiles += t;
      slots += t * n;
    }
  }
  const int upto = wave_scan(items), upto_tiles = wave_scan(tiles), upto_slots = wave_scan(slots);
  if (__builtin_amdgcn_readlane(upto, 63) > cut.items || __builtin_amdgcn_readlane(upto_slots, 63) > cut.slots ||
      __builtin_amdgcn_readlane(upto_tiles, 63) > cut.joins)
    return false;
  joins = __builtin_amdgcn_readlane(upto_tiles, 63);
  const unsigned long long who = __builtin_amdgcn_ballot_w64(r < upto);
  if (!who) return false;
  const int src = __builtin_ctzll(who);
  int at = __builtin_amdgcn_readlane(upto - items, src);
  it.join = __builtin_amdgcn_readlane(upto_tiles - tiles, src);
  it.slot = __builtin_amdgcn_readlane(upto_slots - slots, src);
  for (int b = src; b < a.c.batch; b += 64) {
    ChunkSeq s = held;
    if (b >= 64) s = chunk_seq(a, b);
    const int from = b < 64 ? src : 0;                      // (the same in every lane: kept in scalar registers)
    s.first = __builtin_amdgcn_readlane(s.first, from);
    s.n = __builtin_amdgcn_readlane(s.n, from);
    s.len = __builtin_amdgcn_readlane(s.len, from);
    s.base = __builtin_amdgcn_readlane(s.base, from);
    const int t = tiles_of(s, group, cut), n = runs_of(s);
    if (r < at + t * n) {
      // a sequence's first pages first, of those the tiles that see most
      it.b = b;
      it.seq = s;
      it.run = (r - at) / t;
      it.tile = t - 1 - (r - at) % t;
      it.runs = n;
      const long pages = tile_pages(s, group, cut, it.tile);
      it.begin = __builtin_amdgcn_readfirstlane((int)(pages * it.run / n));
      it.end = __builtin_amdgcn_readfirstlane((int)(pages * (it.run + 1) / n));
      it.join = n > 1 ? it.join + it.tile : -1;
      it.slot = n > 1 ? it.slot + it.tile * n : -1;
      it.run = __builtin_amdgcn_readfirstlane(it.run);
      it.tile = __builtin_amdgcn_readfirstlane(it.tile);
      it.runs = __builtin_amdgcn_readfirstlane(n);
      it.join = __builtin_amdgcn_readfirstlane(it.join);
      it.slot = __builtin_amdgcn_readfirstlane(it.slot);
      return true;
    }
    at += t * n;
    if (n > 1) {
      it.join += t;
      it.slot += t * n;
    }
  }
  return false;
}

// Workspace of a kind: o [slots][hkv][rows][D], then (m, l, l^, -) [slots][hkv][rows],
// then the split tiles, then their number.  Sequences of many rows come first.
struct Split {
  int b, tile, slot, runs;
};
struct ChunkWs {
  float* o;
  float4* ml;
  Split* split;
  int* joins;
};
__host__ __device__ __forceinline__ size_t chunk_ws_bytes(const PagedCache& c, const ChunkCut& cut) {
  return (size_t)cut.slots * c.hkv * cut.rows * (c.D + 4) * 4 + cut.joins * sizeof(Split) + 16;
}
__device__ __forceinline__ ChunkWs chunk_ws(uint8_t* ws, const PagedCache& c, const ChunkCut& cut) {
  const size_t rows = (size_t)cut.slots * c.hkv * cut.rows;
  ChunkWs w;
  w.o = reinterpret_cast<float*>(ws);
  w.ml = reinterpret_cast<float4*>(w.o + rows * c.D);
  w.split = reinterpret_cast<Split*>(w.ml + rows);
  w.joins = reinterpret_cast<int*>(w.split + cut.joins);
  return w;
}

// ---------------------------------------------------------------------------
// HIF4 words as fp16 operands.  A magnitude u/4 has the high byte of its fp16 alone
// (three significant bits), so one byte permutation looks up four of them; the sign
// bits are put in, the bytes are spread to halves, and a packed product by
// b 2^-(E2 + E3) makes the values, exactly where they are normal fp16 numbers.
// The eight values come as the pairs (0,4), (1,5), (2,6), (3,7): each half of a
// register has its own E3, and no register needs a second multiplier.
__device__ __forceinline__ h8v_t hif4_operand(uint32_t w, h2_t by) {
  constexpr uint32_t kLow = 0x3A383400u, kHigh = 0x3F3E3D3Cu;      // 0, .25, .5, .75; 1, 1.25, 1.5, 1.75
  const uint32_t even = __builtin_amdgcn_perm(kHigh, kLow, w & 0x07070707u) | ((w << 4) & 0x80808080u);
  const uint32_t odd = __builtin_amdgcn_perm(kHigh, kLow, (w >> 4) & 0x07070707u) | (w & 0x80808080u);
  const h2_t p0 = __builtin_bit_cast(h2_t, __builtin_amdgcn_perm(even, even, 0x020C000Cu)) * by;
  const h2_t p1 = __builtin_bit_cast(h2_t, __builtin_amdgcn_perm(odd, odd, 0x020C000Cu)) * by;
  const h2_t p2 = __builtin_bit_cast(h2_t, even & 0xFF00FF00u) * by;
  const h2_t p3 = __builtin_bit_cast(h2_t, odd & 0xFF00FF00u) * by;
  return h8v_t{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// K's or V's part of a record in a lane's registers.
template <int G>
struct HifPart {
  uint4 code[2 * G];                    // [tile][t/2]: (t even: words 0, 1), (t odd: words 0, 1)
  uint32_t e3[(G + 1) / 2];
  uint32_t e2;
  uint4 base[G];                        // [tile]: byte n % 4 of word t is row (t, n)'s
};
template <int G>
__device__ __forceinline__ void load_hif4(HifPart<G>& p, const uint8_t* part, int lane) {
  typedef unsigned u4v_t __attribute__((ext_vector_type(4)));
  typedef unsigned u2v_t __attribute__((ext_vector_type(2)));
  const global_ptr meta = scalar_address(part + 2048 * G);
#pragma unroll
  for (int h = 0; h < (G + 1) / 2; ++h) {
    const global_ptr code = scalar_address(part + 4096 * h);
#pragma unroll
    for (int i = 0; i < (G == 1 ? 2 : 4); ++i)
      p.code[4 * h + i] = __builtin_bit_cast(uint4, load_at<u4v_t>(code, 16 * lane + 1024 * i));
  }
  if (G == 1) {
    p.e3[0] = load_at<uint16_t>(meta, 2 * lane);
    p.e2 = load_at<uint8_t>(meta, lane + 128);
  } else if (G == 2) {
    p.e3[0] = load_at<uint32_t>(meta, 4 * lane);
    p.e2 = load_at<uint16_t>(meta, 2 * lane + 256);
  } else {
    const u2v_t x = load_at<u2v_t>(meta, 8 * lane);
    p.e3[0] = x[0];
    p.e3[G == 4 ? 1 : 0] = x[1];
    p.e2 = load_at<uint32_t>(meta, 4 * lane + 512);
  }
#pragma unroll
  for (int g = 0; g < G; ++g)
    p.base[g] = __builtin_bit_cast(uint4, load_at<u4v_t>(meta, 192 * G + 16 * G * ((lane & 15) >> 2) + 16 * g));
}
// Bit `bit` of both halves of x at the place of fp16's exponent.
__device__ __forceinline__ uint32_t exponent_bit(uint32_t x, int bit) {
  return (bit <= 10 ? x << (10 - bit) : x >> (bit - 10)) & 0x04000400u;
}
// The operand of word (t, c) of a tile.
template <int G>
__device__ __forceinline__ h8v_t part_operand(const HifPart<G>& p, int tile, int t, int c, int lane) {
  const uint4 w = p.code[2 * tile + (t >> 1)];
  const uint32_t word = t & 1 ? (c ? w.w : w.z) : (c ? w.y : w.x);
  const uint32_t e3 = G == 1 ? (p.e3[0] & 0xFFu) | ((p.e3[0] & 0xFF00u) << 8) : p.e3[tile / 2];
  const uint32_t e2 = (p.e2 >> (8 * tile) & 0xFFu) * 0x10001u;
  const uint32_t two = 0x3C003C00u - exponent_bit(e3, 8 * (tile & 1) + 2 * t + c) - exponent_bit(e2, 2 * t + c);
  const uint32_t bases = t == 0 ? p.base[tile].x : t == 1 ? p.base[tile].y : t == 2 ? p.base[tile].z : p.base[tile].w;
  const half_t b = (half_t)__uint_as_float(((bases >> (8 * (lane & 3)) & 0xFFu) << 21) + 0x30000000u);
  return hif4_operand(word, h2_t{b, b} * __builtin_bit_cast(h2_t, two));
}

// ---------------------------------------------------------------------------
// Rows: 16 columns of a matrix product, one a lane (lane 16k + n holds column n's share k).
struct Row {
  int limit;                            // the last key that it sees; -1: none, -2: no such row
  int at;                               // row of q and o (token, query head)
};
__device__ __forceinline__ Row row_of(const PagedChunk& a, const Item& it, int group, int head, int row) {
  const int token = row / group, g = row - token * group;
  if (token >= it.seq.n) return Row{-2, 0};
  return Row{max(-1, it.seq.base + token), (it.seq.first + token) * a.hq + head * group + g};
}

// The query's operands: step c's channels of lane k, in the order of the keys'.
template <int G, bool kFp16>
__device__ __forceinline__ void load_query(h8v_t (&q)[2 * G], const PagedChunk& a, const Row& r, int head, int k) {
#pragma unroll
  for (int c = 0; c < 2 * G; ++c) {
    const int ch = kFp16 ? 32 * c + 8 * k : 64 * (c >> 1) + 16 * k + 8 * (c & 1);
    h8v_t x = {0, 0, 0, 0, 0, 0, 0, 0};
    if (r.limit > -2) {
      x = *reinterpret_cast<const h8v_t*>(a.q + (size_t)r.at * (64 * G) + ch);
      if (a.s) {
        const f4v_t* s = reinterpret_cast<const f4v_t*>(a.s + (size_t)head * (64 * G) + ch);
        const f4v_t s0 = s[0], s1 = s[1];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = round_product(x[i], i < 4 ? s0[i & 3] : s1[i & 3]);
      }
    }
    q[c] = kFp16 ? x : __builtin_shufflevector(x, x, 0, 4, 1, 5, 2, 6, 3, 7);
  }
}

// The state of 16 rows' softmax, and their sums.
template <int G>
struct Rows16 {
  float ref, l;                         // p = 2^(score - ref), scores in log2 units; l: the lane's share
  f4v_t sum;                            // of the rounded p
  f4v_t o[4 * G];                       // channels 16 ct + 4k + v
};
template <int G>
__device__ __forceinline__ void start(Rows16<G>& x) {
  const f4v_t z = {0.0f, 0.0f, 0.0f, 0.0f};
  x.ref = kNoRef;
  x.l = 0.0f;
  x.sum = z;
#pragma unroll
  for (int c = 0; c < 4 * G; ++c) x.o[c] = z;
}

// A page's scores (s[t][v]: key 16k + 4t + v, before the scale) to the second product's
// operands; keys behind `seen` (the row's limit in the page) do not count.
template <int G, bool kFp16>
__device__ __forceinline__ void soften(Rows16<G>& x, f4v_t (&s)[4], h8v_t (&p)[2], float scale, bool masked, int seen, int k) {
  if (masked) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (16 * k + 4 * t + v > seen) s[t][v] = -INFINITY;
  }
  float top = s[0][0];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int v = 0; v < 4; ++v) top = fmaxf(top, s[t][v]);
  top *= scale;
  if (__builtin_amdgcn_ballot_w64(top - x.ref > kTop + kSlack)) {
    const float to = fmaxf(x.ref, max_across_rows(top) - kTop), f = __builtin_amdgcn_exp2f(x.ref - to);
    x.ref = to;
    x.l *= f;
    x.sum *= f;
#pragma unroll
    for (int c = 0; c < 4 * G; ++c) x.o[c] *= f;
  }
  // The exponent in one operation, the product not rounded; of scores over 2^20 it is
  // rounded as the reference's was (half a step there is more than p's range).
  float by = scale;
  if (__builtin_amdgcn_ballot_w64(fabsf(x.ref) > 0x1p20f && x.ref != kNoRef)) {
    by = 1.0f;
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] *= scale;
  }
  float l = 0.0f;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      s[t][v] = __builtin_amdgcn_exp2f(fmaf(s[t][v], by, -x.ref));
      l += s[t][v];
    }
  x.l += l;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const h4v_t a = __builtin_convertvector(s[2 * c], h4v_t), b = __builtin_convertvector(s[2 * c + 1], h4v_t);
    p[c] = kFp16 ? __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7) : __builtin_shufflevector(a, b, 0, 4, 1, 5, 2, 6, 3, 7);
  }
}

__device__ __forceinline__ f4v_t product(h8v_t a, h8v_t b, f4v_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ h8v_t ones() { return h8v_t{1, 1, 1, 1, 1, 1, 1, 1}; }

// Values of FP16 pages that some rows of a tile must not see: 0 times them has to be 0
// also where they are infinite or NaN.  Of the keys that no row sees they are cleared;
// of the others what is not finite is counted, per sign, over the keys that a row sees
// (products of ones; NaN under both signs), added where it counts, and cleared.
typedef uint32_t u4v_t __attribute__((ext_vector_type(4)));
// Bit 15 of each half that is not finite.
__device__ __forceinline__ u4v_t not_finite(u4v_t x) { return ((x & 0x7C007C00u) + 0x04000400u) & 0x80008000u; }
__device__ __forceinline__ bool any(u4v_t x) { return (x[0] | x[1] | x[2] | x[3]) != 0; }
// All bits of the halves whose bit 15 is set, and 1.0 in them.
__device__ __forceinline__ u4v_t whole(u4v_t x) { return (x - (x >> 15)) | x; }
__device__ __forceinline__ u4v_t one(u4v_t x) { return (x >> 1) - (x >> 5); }
// All bits of the first `n` halves (cut to 0 .. 8).
__device__ __forceinline__ u4v_t first_halves(int n) {
  u4v_t m;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    const int some = max(0, min(2, n - 2 * d));
    m[d] = (uint32_t)(0xFFFFFFFFull << (16 * some) >> 32);
  }
  return m;
}
template <int G>
__device__ __forceinline__ void add_not_finite(Rows16<G>& x, const u4v_t (&v)[2], int ct, int seen, int k) {
  f4v_t up = {0.0f, 0.0f, 0.0f, 0.0f}, down = up;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const u4v_t odd = not_finite(v[c]), nan = ((v[c] & 0x03FF03FFu) + 0x7FFF7FFFu), minus = v[c];
    const h8v_t who = __builtin_bit_cast(h8v_t, first_halves(seen + 1 - 16 * k - 8 * c) & 0x3C003C00u);
    up = product(__builtin_bit_cast(h8v_t, one(odd & (nan | ~minus))), who, up);
    down = product(__builtin_bit_cast(h8v_t, one(odd & (nan | minus))), who, down);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x.o[ct][i] += up[i] > 0.0f ? INFINITY : 0.0f;
    x.o[ct][i] -= down[i] > 0.0f ? INFINITY : 0.0f;
  }
}

// Leaves 16 rows of an item: rounded and divided, or as a run's share.
template <int G>
__device__ __forceinline__ void finish(const PagedChunk& a, const ChunkWs& ws, const Item& it, Rows16<G>& x, const Row& r, int head,
                                       int tile_rows, int row_in_tile, int k) {
  constexpr int D = 64 * G;
  const float l = sum_across_rows(x.l);
  if (r.limit == -2) return;
  if (it.runs == 1) {
    const float by = x.sum[0] == 0.0f ? 0.0f : 1.0f / x.sum[0];
#pragma unroll
    for (int c = 0; c < 4 * G; ++c)
      *reinterpret_cast<h4v_t*>(a.o + (size_t)r.at * D + 16 * c + 4 * k) = __builtin_convertvector(x.o[c] * by, h4v_t);
    if (k == 0) {
      const int token = r.at / a.hq;
      a.lse[(size_t)(r.at - token * a.hq) * a.total + token] =
          l == 0.0f ? -INFINITY : (float)(((double)x.ref + (double)__log2f(l)) * 0.6931471805599453);
    }
    return;
  }
  const size_t at = ((size_t)(it.slot + it.run) * a.c.hkv + head) * tile_rows + row_in_tile;
#pragma unroll
  for (int c = 0; c < 4 * G; ++c) *reinterpret_cast<f4v_t*>(ws.o + at * D + 16 * c + 4 * k) = x.o[c];
  if (k == 0) ws.ml[at] = make_float4(l == 0.0f ? -INFINITY : x.ref, l, x.sum[0], 0.0f);
}

// ---------------------------------------------------------------------------
// Few rows over HIF4 pages.
// One wave per (item, kv head): 16 NB rows; the operands are made of a page's record
// in registers, one 16-byte load a lane for each KiB.  K of the next page is fetched once
// this one's has been used, V while the scores are made.
template <int G, int NB>
__device__ __forceinline__ void chunk_rows(const PagedChunk& a, const ChunkCut& cut, uint8_t* ws_at, int item, int head, int lane) {
  constexpr int D = 64 * G, kRows = 16 * NB;
  const int n = lane & 15, k = lane >> 4, group = a.hq / a.c.hkv;
  Item it;
  int joins;
  const bool there = find_item(a, group, cut, item, lane, it, joins);
  const ChunkWs ws = chunk_ws(ws_at, a.c, cut);
  if (item == 0 && head == 0 && lane == 0) *ws.joins = joins;
  if (!there) return;
  if (it.runs > 1 && it.run == 0 && head == 0 && lane == 0) ws.split[it.join] = Split{it.b, it.tile, it.slot, it.runs};

  // the pages of the run that are some
  Pages pg;
  pg.base = it.begin - 64;
  int page_at = 0;
  const auto next = [&](int j) {
    for (; j < it.end; ++j) {
      if (j - pg.base >= 64) load_pages(pg, a.c, it.b, j, it.end - 1, lane);
      page_at = __builtin_amdgcn_readlane(pg.mine, j - pg.base);
      if ((unsigned)page_at < (unsigned)a.c.num_pages) break;
    }
    return __builtin_amdgcn_readfirstlane(j);
  };
  const auto record = [&] {
    const size_t at = (size_t)__builtin_amdgcn_readfirstlane(page_at) * a.c.hkv + head;
    return a.c.pool + at * paged_record_bytes(D, false);
  };
  int j = next(it.begin);

  Row row[NB];
  Rows16<G> x[NB];
  h8v_t q[NB][2 * G];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    row[i] = row_of(a, it, group, head, it.tile * kRows + 16 * i + n);
    load_query<G, false>(q[i], a, row[i], head, k);
    start(x[i]);
  }
  const int first_token = it.tile * kRows / group;          // every row of the tile sees the keys up to its
  const int all_see = it.seq.base + first_token;

  const uint8_t* rec = record();
  HifPart<G> k4, v4;
  if (j < it.end) load_hif4<G>(k4, rec, lane);
  while (j < it.end) {
    const int now = j;
    const bool masked = now * kPage + kPage - 1 > all_see;
    keep_order();
    load_hif4<G>(v4, rec + 2304 * G, lane);
    keep_order();
    f4v_t s[NB][4];
    h8v_t p[NB][2];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int t = 0; t < 4; ++t) s[i][t] = f4v_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < 2 * G; ++c)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const h8v_t kr = part_operand<G>(k4, c >> 1, t, c & 1, lane);
#pragma unroll
        for (int i = 0; i < NB; ++i) s[i][t] = product(kr, q[i][c], s[i][t]);
      }
    keep_order();
    j = next(j + 1);
    rec = record();
    if (j < it.end) load_hif4<G>(k4, rec, lane);
    keep_order();
#pragma unroll
    for (int i = 0; i < NB; ++i) soften<G, false>(x[i], s[i], p[i], a.scale, masked, row[i].limit - now * kPage, k);
    keep_order();
#pragma unroll
    for (int u = 0; u < 4 * G; ++u)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const h8v_t vr = part_operand<G>(v4, u >> 2, u & 3, c, lane);
#pragma unroll
        for (int i = 0; i < NB; ++i) x[i].o[u] = product(vr, p[i][c], x[i].o[u]);
      }
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c) x[i].sum = product(ones(), p[i][c], x[i].sum);
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) finish<G>(a, ws, it, x[i], row[i], head, kRows, 16 * i + n, k);
}

template <int G, int NB>
__global__ void __launch_bounds__(64, G == 4 ? 1 : 2) k_chunk_rows(PagedChunk a, ChunkCut cut, int few_ws) {
  chunk_rows<G, NB>(a, cut, a.ws + few_ws, blockIdx.x / a.c.hkv, blockIdx.x % a.c.hkv, threadIdx.x);
}

// ---------------------------------------------------------------------------
// Many rows: kWaves waves of 16 NB rows each share a page, whose operands they make in
// LDS (two pages' room: the next one is made while this one is used).  A record's KiB
// unit of fp16 operands is what a wave reads for one operand of a product, 16 bytes a
// lane in lane order, so neither reads nor writes have bank conflicts.  Over FP16 pages
// a few rows are a workgroup of one wave.
// Units of a page: K [t][c], then V [channels / 16][c].
constexpr int kMatrix = 0x008, kDsRead = 0x100;      // kinds of instructions to the scheduler

// A quarter of a tile's part of a HIF4 record: the words (t, c) of two t.
struct HifQuad {
  uint4 code;
  uint32_t e3, e2;
  uint2 base;
};
template <int G>
__device__ __forceinline__ void load_quad(HifQuad& q, const uint8_t* rec, int at, int lane) {
  typedef unsigned u4v_t __attribute__((ext_vector_type(4)));
  typedef unsigned u2v_t __attribute__((ext_vector_type(2)));
  const int tile = at / 2 % G, half = at & 1;
  const uint8_t* part = rec + at / (2 * G) * (2304 * G);
  const global_ptr code = (global_ptr)(part + 2048 * tile + 1024 * half);
  const global_ptr meta = (global_ptr)(part + 2048 * G);
  q.code = __builtin_bit_cast(uint4, load_at<u4v_t>(code, 16 * lane));
  if (G == 1)
    q.e3 = load_at<uint16_t>(meta, 2 * lane);
  else
    q.e3 = load_at<uint32_t>(meta, 2 * G * lane + 4 * (tile >> 1));
  q.e2 = load_at<uint8_t>(meta, 128 * G + G * lane + tile);
  q.base = __builtin_bit_cast(uint2, load_at<u2v_t>(meta, 192 * G + 16 * G * ((lane & 15) >> 2) + 16 * tile + 8 * half));
}
template <int G>
__device__ __forceinline__ void store_quad(h8v_t* page, const HifQuad& q, int at, int lane) {
  const int tile = at / 2 % G, half = at & 1;
  const bool is_v = at >= 2 * G;
  const uint32_t e3 = (G == 1 ? (q.e3 & 0xFFu) | ((q.e3 & 0xFF00u) << 8) : q.e3) >> (8 * (tile & 1) + 4 * half);
  const uint32_t e2 = (q.e2 * 0x10001u) >> (4 * half);
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const half_t b = (half_t)__uint_as_float((((u ? q.base.y : q.base.x) >> (8 * (lane & 3)) & 0xFFu) << 21) + 0x30000000u);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const uint32_t word = u ? (c ? q.code.w : q.code.z) : (c ? q.code.y : q.code.x);
      const uint32_t two = 0x3C003C00u - exponent_bit(e3, 2 * u + c) - exponent_bit(e2, 2 * u + c);
      const int t = 2 * half + u, unit = is_v ? 8 * G + (4 * tile + t) * 2 + c : t * 2 * G + 2 * tile + c;
      page[64 * unit + lane] = hif4_operand(word, h2_t{b, b} * __builtin_bit_cast(h2_t, two));
    }
  }
}

// What a wave fetches of a HIF4 page, and puts into LDS as operands.
template <int G, int kWaves>
struct HifShare {
  static constexpr int kAll = 4 * G, kMine = (kAll + kWaves - 1) / kWaves;
  HifQuad quad[kMine];
  __device__ __forceinline__ void load(const uint8_t* rec, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) load_quad<G>(quad[i], rec, wave + kWaves * i, lane);
  }
  __device__ __forceinline__ void store(h8v_t* page, int wave, int lane) const {
#pragma unroll
    for (int i = 0; i < kMine; ++i) store_quad<G>(page, quad[i], wave + kWaves * i, lane);
  }
};
// A wave's share of an FP16 page, which is operands as it stands: copied to LDS past
// the registers.  M0 and the copy that takes its LDS address from it are one statement:
// the compiler keeps no value of its own in M0.
template <int kBytes, int kStep>
struct CopyPieces {
  static __device__ __forceinline__ void run(uint64_t from, uint32_t to, uint32_t lane_bytes) {
    if constexpr (kBytes > 0) {
      CopyPieces<kBytes - kStep, kStep>::run(from, to, lane_bytes);
      asm volatile("s_add_u32 m0, %2, %3\n\tglobal_load_lds_dwordx4 %0, %1"
                   :
                   : "v"(lane_bytes + (kBytes - kStep)), "s"(from), "s"(to), "n"(kBytes - kStep)
                   : "memory", "m0", "scc");
    }
  }
};
__device__ __forceinline__ uint32_t scalar(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
template <int G, int kWaves>
__device__ __forceinline__ void copy_share(h8v_t* page, const uint8_t* rec, int wave, int lane) {
  const uint64_t from = (uint64_t)(uintptr_t)(rec + 16384 * G / kWaves * wave);
  const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)(page + 1024 * G / kWaves * wave);
  CopyPieces<16384 * G / kWaves, 1024>::run((uint64_t)scalar((uint32_t)from) | (uint64_t)scalar((uint32_t)(from >> 32)) << 32, scalar(to),
                                            16 * lane);
}
__device__ __forceinline__ void wait_copies() { __builtin_amdgcn_s_waitcnt(0x0F70); }     // vmcnt(0)

template <int G, bool kFp16, int kWaves, int NB>
__global__ void __launch_bounds__(64 * kWaves, G == 4 ? 1 : 2) k_chunk_wide(PagedChunk a, ChunkCut cut, ChunkCut few, int few_ws) {
  constexpr int D = 64 * G, kMine = 16 * NB, kRows = kMine * kWaves, kUnits = 16 * G;
  static_assert(16 * G % kWaves == 0 && 4 * G % kWaves == 0, "equal shares");
  extern __shared__ __align__(16) uint8_t smem[];
  h8v_t* const pages = reinterpret_cast<h8v_t*>(smem);
  const int lane = threadIdx.x & 63, n = lane & 15, k = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int head = blockIdx.x % a.c.hkv, group = a.hq / a.c.hkv, number = blockIdx.x / a.c.hkv;
  if constexpr (!kFp16) {
    if (number >= cut.items) {            // behind the sequences of many rows those of few, an item a wave
      const int item = (number - cut.items) * kWaves + wave;
      if (item < few.items) chunk_rows<G, 1>(a, few, a.ws + few_ws, item, head, lane);
      return;
    }
  }
  Item it;
  int joins;
  const bool there = find_item(a, group, cut, number, lane, it, joins);
  const ChunkWs ws = chunk_ws(a.ws, a.c, cut);
  if (blockIdx.x == 0 && threadIdx.x == 0) *ws.joins = joins;
  if (!there) return;
  if (it.runs > 1 && it.run == 0 && head == 0 && threadIdx.x == 0) ws.split[it.join] = Split{it.b, it.tile, it.slot, it.runs};

  // pages from here on that are some; the table's entries 64 at a time, one a lane
  Pages pg;
  pg.base = it.begin - 64;
  int page_at = 0;                        // the page that next() has found
  const auto next = [&](int j) {
    for (; j < it.end; ++j) {
      if (j - pg.base >= 64) load_pages(pg, a.c, it.b, j, it.end - 1, lane);
      page_at = __builtin_amdgcn_readlane(pg.mine, j - pg.base);
      if ((unsigned)page_at < (unsigned)a.c.num_pages) break;
    }
    return __builtin_amdgcn_readfirstlane(j);
  };
  const auto record = [&] {
    const size_t at = (size_t)__builtin_amdgcn_readfirstlane(page_at) * a.c.hkv + head;
    return a.c.pool + at * paged_record_bytes(D, kFp16);
  };
  HifShare<G, kWaves> share;
  int j = next(it.begin);
  if (j < it.end) {
    if constexpr (kFp16)
      copy_share<G, kWaves>(pages, record(), wave, lane);
    else
      share.load(record(), wave, lane);
  }

  const int row0 = it.tile * kRows + wave * kMine;      // the wave's first row
  Row row[NB];
  Rows16<G> x[NB];
  h8v_t q[NB][2 * G];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    row[i] = row_of(a, it, group, head, row0 + 16 * i + n);
    load_query<G, kFp16>(q[i], a, row[i], head, k);
    start(x[i]);
  }
  // keys that every row of the wave sees, and that any of them sees: up to these
  const int first_token = row0 / group, last_token = min(it.seq.n - 1, (row0 + kMine - 1) / group);
  const int all_see = it.seq.base + first_token, some_see = first_token < it.seq.n ? it.seq.base + last_token : -1;

  int ahead = next(j + 1), at = 0;
  if constexpr (kFp16) {
    wait_copies();
  } else {
    if (j < it.end) share.store(pages, wave, lane);
    if (ahead < it.end) share.load(record(), wave, lane);
  }
  __syncthreads();
  while (j < it.end) {
    const h8v_t* page = pages + 64 * kUnits * at + lane;
    const int now = j;
    j = ahead;
    if (j < it.end) {
      h8v_t* const other = pages + 64 * kUnits * (at ^ 1);
      if constexpr (kFp16) {
        copy_share<G, kWaves>(other, record(), wave, lane);
        ahead = next(j + 1);
      } else {
        share.store(other, wave, lane);
        ahead = next(j + 1);
        if (ahead < it.end) share.load(record(), wave, lane);
      }
    }
    if (now * kPage <= some_see) {
      const bool masked = now * kPage + kPage - 1 > all_see;
      f4v_t s[NB][4];
      h8v_t p[NB][2];
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) s[i][t] = f4v_t{0.0f, 0.0f, 0.0f, 0.0f};
      // Operands come four units ahead of their products: a wave's own products have to
      // cover LDS's latency, there are two waves a SIMD.
      h8v_t next4[2][4];
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int t = 0; t < 4; ++t) next4[0][t] = page[64 * (t * 2 * G)];
#pragma unroll
      for (int c = 0; c < 2 * G; ++c) {
        if (c + 1 < 2 * G)
#pragma unroll
          for (int t = 0; t < 4; ++t) next4[(c + 1) & 1][t] = page[64 * (t * 2 * G + c + 1)];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < NB; ++i) s[i][t] = product(next4[c & 1][t], q[i][c], s[i][t]);
      }
      __builtin_amdgcn_sched_group_barrier(kDsRead, 4, 0);
#pragma unroll
      for (int c = 0; c < 2 * G; ++c) {
        if (c + 1 < 2 * G) __builtin_amdgcn_sched_group_barrier(kDsRead, 4, 0);
        __builtin_amdgcn_sched_group_barrier(kMatrix, 4 * NB, 0);
      }
      keep_order();
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int u = 0; u < 4; ++u) next4[0][u] = page[64 * (8 * G + u)];
#pragma unroll
      for (int i = 0; i < NB; ++i) soften<G, kFp16>(x[i], s[i], p[i], a.scale, masked, row[i].limit - now * kPage, k);
      keep_order();
      const bool odd_values = kFp16 && masked;
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) x[i].sum = product(ones(), p[i][c], x[i].sum);
      if (odd_values) {
#pragma unroll
        for (int u = 0; u < 4 * G; ++u) {
          keep_order();
          u4v_t v[2];
#pragma unroll
          for (int c = 0; c < 2; ++c)
            v[c] = __builtin_bit_cast(u4v_t, page[64 * (8 * G + 2 * u + c)]) & first_halves(some_see - now * kPage + 1 - 16 * k - 8 * c);
          if (__builtin_amdgcn_ballot_w64(any(not_finite(v[0]) | not_finite(v[1])))) {
#pragma unroll
            for (int i = 0; i < NB; ++i) add_not_finite<G>(x[i], v, u, row[i].limit - now * kPage, k);
#pragma unroll
            for (int c = 0; c < 2; ++c) v[c] &= ~whole(not_finite(v[c]));
          }
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < NB; ++i) x[i].o[u] = product(__builtin_bit_cast(h8v_t, v[c]), p[i][c], x[i].o[u]);
        }
      } else {
#pragma unroll
        for (int g = 0; g < 2 * G; ++g) {
          if (g + 1 < 2 * G)
#pragma unroll
            for (int u = 0; u < 4; ++u) next4[(g + 1) & 1][u] = page[64 * (8 * G + 4 * g + 4 + u)];
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < NB; ++i) x[i].o[2 * g + u / 2] = product(next4[g & 1][u], p[i][u & 1], x[i].o[2 * g + u / 2]);
        }
#pragma unroll
        for (int g = 0; g < 2 * G; ++g) {
          if (g + 1 < 2 * G) __builtin_amdgcn_sched_group_barrier(kDsRead, 4, 0);
          __builtin_amdgcn_sched_group_barrier(kMatrix, 4 * NB, 0);
        }
        keep_order();
      }
      __builtin_amdgcn_s_setprio(0);
    }
    at ^= 1;
    if constexpr (kFp16) wait_copies();
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) finish<G>(a, ws, it, x[i], row[i], head, kRows, wave * kMine + 16 * i + n, k);
}

// ---------------------------------------------------------------------------
// Joining the runs of a split tile's rows: with m the largest of their references,
// o = sum o_i 2^(m_i - m) / sum l^_i 2^(m_i - m), l = sum l_i 2^(m_i - m), in a fixed
// order.  kFew: a workgroup takes 32 channels of a row, its threads share out the runs
// (many, where there are few rows); else a wave takes a row.  The workgroups go
// through the split tiles that there are.
constexpr int kChunkJoin = 256;

struct Joined {
  float m, l, sum;
  f4v_t o;
};
__device__ __forceinline__ void join_pair(Joined& x, const Joined& y) {
  const float to = fmaxf(x.m, y.m), ref = to == -INFINITY ? 0.0f : to;
  const float f = __builtin_amdgcn_exp2f(x.m - ref), g = __builtin_amdgcn_exp2f(y.m - ref);
  x.m = to;
  x.l = x.l * f + y.l * g;
  x.sum = x.sum * f + y.sum * g;
  x.o = x.o * f + y.o * g;
}

template <int G, bool kFew>
__device__ __forceinline__ void join_tiles(const PagedChunk& a, const ChunkCut& cut, uint8_t* ws_at, Joined* part) {
  constexpr int D = 64 * G, kCols = kFew ? 8 : D / 4, kSets = (kFew ? kChunkJoin : 64) / kCols, kAhead = 4;
  const int lane = threadIdx.x & 63, at_set = kFew ? threadIdx.x : lane, col = at_set % kCols, set = at_set / kCols;
  const ChunkWs ws = chunk_ws(ws_at, a.c, cut);
  const int group = a.hq / a.c.hkv, slices = kFew ? D / 32 : 1, rows = *ws.joins * a.c.hkv * cut.rows;
  const int step = kFew ? gridDim.x : 4 * gridDim.x;
  for (int item = kFew ? blockIdx.x : 4 * blockIdx.x + (threadIdx.x >> 6); item < rows * slices; item += step) {
    const int at = item / slices, row_in_tile = at % cut.rows, head = at / cut.rows % a.c.hkv;
    const Split sp = ws.split[at / cut.rows / a.c.hkv];
    const int ch = (item % slices) * 32 + 4 * col;
    Item it;
    it.seq = chunk_seq(a, sp.b);
    const Row row = row_of(a, it, group, head, sp.tile * cut.rows + row_in_tile);
    if (row.limit == -2) continue;
    Joined x = {-INFINITY, 0.0f, 0.0f, {0.0f, 0.0f, 0.0f, 0.0f}};
    for (int i = set; i < sp.runs; i += kAhead * kSets) {
      float4 ml[kAhead];
      f4v_t y[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const size_t from = ((size_t)(sp.slot + min(i + u * kSets, sp.runs - 1)) * a.c.hkv + head) * cut.rows + row_in_tile;
        ml[u] = ws.ml[from];
        y[u] = *reinterpret_cast<const f4v_t*>(ws.o + from * D + ch);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i + u * kSets < sp.runs) join_pair(x, Joined{ml[u].x, ml[u].y, ml[u].z, y[u]});
    }
    if constexpr (kFew) {
      part[threadIdx.x] = x;
      __syncthreads();
      if (set == 0) {
#pragma unroll 4
        for (int i = 1; i < kSets; ++i) join_pair(x, part[i * kCols + col]);
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int d = kCols; d < 64; d <<= 1) {
        Joined y;
        y.m = __shfl_xor(x.m, d);
        y.l = __shfl_xor(x.l, d);
        y.sum = __shfl_xor(x.sum, d);
#pragma unroll
        for (int v = 0; v < 4; ++v) y.o[v] = __shfl_xor(x.o[v], d);
        join_pair(x, y);
      }
    }
    if (set) continue;
    *reinterpret_cast<h4v_t*>(a.o + (size_t)row.at * D + ch) = __builtin_convertvector(x.o * (x.sum == 0.0f ? 0.0f : 1.0f / x.sum), h4v_t);
    if (ch == 0) {
      const int token = row.at / a.hq;
      a.lse[(size_t)(row.at - token * a.hq) * a.total + token] =
          x.l == 0.0f ? -INFINITY : (float)(((double)x.m + (double)__log2f(x.l)) * 0.6931471805599453);
    }
  }
}
template <int G, bool kFew>
__global__ void __launch_bounds__(kChunkJoin) k_chunk_join(PagedChunk a, ChunkCut cut, ChunkCut few, int few_ws) {
  __shared__ Joined part[kFew ? kChunkJoin : 1];
  if (cut.joins) join_tiles<G, kFew>(a, cut, a.ws, part);
  if (few.joins) join_tiles<G, kFew>(a, few, a.ws + few_ws, part);
}

// ---------------------------------------------------------------------------
// Rows (of one sequence and kv head) up to which a wave of its own takes them.
constexpr int kFewRows = 32;

// Waves of a workgroup that share a page.
constexpr int wide_waves(int D) { return D == 128 ? 8 : 4; }

// Sizes of one kind: sequences of more than `above` rows, of which there are at most
// `most`, with `all` rows in total.
static bool cut_kind(const PagedCache& c, size_t all, size_t most, size_t batch, ChunkCut* cut) {
  const size_t tiles = std::min(batch * ((most + cut->rows - 1) / cut->rows), all / cut->rows + batch);
  const size_t runs = std::max<size_t>(1, ((size_t)c.max_pages + kMinRun - 1) / kMinRun);
  const size_t items = std::min(tiles * runs, tiles + cut->target + 1);
  const size_t joins = runs == 1 ? 0 : std::min(tiles, (size_t)cut->target + 1);
  if (items * c.hkv >= kMaxGrid || joins * c.hkv * cut->rows >= kMaxGrid) return false;
  cut->items = (int)items;
  cut->joins = (int)joins;
  cut->slots = runs == 1 ? 0 : (int)std::min(tiles * runs, (size_t)2 * cut->target + 2);
  return true;
}
struct ChunkCuts {
  int waves;                            // of a workgroup that takes many rows; 1: there are but few
  ChunkCut many, few;
  int few_ws;                           // offset in the workspace
  size_t blocks, joined, bytes;         // workgroups, rows that may be joined
};
static bool chunk_cuts(const PagedCache& c, int hq, int total, int max_new, ChunkCuts* x) {
  const size_t group = hq / c.hkv, most = max_new * group, all = (size_t)total * group;
  if (most >= (size_t)1 << 30) return false;
  const bool wide = most > kFewRows;
  x->waves = wide ? wide_waves(c.D) : 1;
  x->many = ChunkCut{wide ? 32 * x->waves : 0, 0, c.fp16 ? 0 : kFewRows, 1 << 30, 0, 0, 0};
  x->few = ChunkCut{16, 0, 0, kFewRows, 0, 0, 0};
  const int waves = 1024 * (c.D == 256 ? 1 : 2);            // that the chip holds
  if (c.fp16) {
    if (!wide) x->many.rows = most <= 16 ? 16 : 32;
    x->many.target = std::max(1, waves / x->waves / c.hkv);
    if (!cut_kind(c, all, most, c.batch, &x->many)) return false;
  } else {
    if (!wide && most > 16 && c.D != 256) x->few.rows = 32;
    x->few.target = std::max(1, waves / (wide ? 2 : 1) / c.hkv);
    if (!cut_kind(c, all, std::min(most, (size_t)kFewRows), c.batch, &x->few)) return false;
    x->many.target = std::max(1, waves / x->waves / c.hkv);
    if (wide && !cut_kind(c, all, most, std::min((size_t)c.batch, all / (kFewRows + 1)), &x->many)) return false;
  }
  const size_t many = (chunk_ws_bytes(c, x->many) + 255) / 256 * 256;
  x->few_ws = (int)many;
  x->bytes = many + chunk_ws_bytes(c, x->few);
  x->blocks = (x->many.items + ((size_t)x->few.items + x->waves - 1) / x->waves) * c.hkv;
  x->joined = ((size_t)x->many.joins * x->many.rows + (size_t)x->few.joins * x->few.rows) * c.hkv;
  return many < (size_t)1 << 31 && x->blocks < max_grid(64 * x->waves);
}

bool paged_chunk_fits(const PagedCache& c, int hq, int total, int max_new) {
  ChunkCuts x;
  return chunk_cuts(c, hq, total, max_new, &x);
}
size_t paged_chunk_workspace(const PagedCache& c, int hq, int total, int max_new) {
  ChunkCuts x;
  return chunk_cuts(c, hq, total, max_new, &x) ? x.bytes : 0;
}

template <int G, bool kFp16, int kWaves, int NB>
static hipError_t launch_wide(const PagedChunk& a, const ChunkCuts& x, hipStream_t st) {
  constexpr size_t kLds = (size_t)2 * 16 * G * 1024;
  const auto kernel = k_chunk_wide<G, kFp16, kWaves, NB>;
  if (kLds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds);
    if (e != hipSuccess) return e;
  }
  kernel<<<dim3((unsigned)x.blocks), 64 * kWaves, kLds, st>>>(a, x.many, x.few, x.few_ws);
  return hipGetLastError();
}
template <int G>
static hipError_t launch_chunk(const PagedChunk& a, const ChunkCuts& x, hipStream_t st) {
  hipError_t e;
  if (a.c.fp16) {
    e = x.waves > 1            ? launch_wide<G, true, wide_waves(64 * G), 2>(a, x, st)
        : x.many.rows == 16 ? launch_wide<G, true, 1, 1>(a, x, st)
                            : launch_wide<G, true, 1, 2>(a, x, st);
  } else if (x.waves > 1) {
    e = launch_wide<G, false, wide_waves(64 * G), 2>(a, x, st);
  } else {
    if (G == 4 || x.few.rows == 16)
      k_chunk_rows<G, 1><<<dim3((unsigned)x.blocks), 64, 0, st>>>(a, x.few, x.few_ws);
    else
      k_chunk_rows<G == 4 ? 1 : G, 2><<<dim3((unsigned)x.blocks), 64, 0, st>>>(a, x.few, x.few_ws);
    e = hipGetLastError();
  }
  if (e != hipSuccess || x.joined == 0) return e;
  if (x.joined <= 2048)
    k_chunk_join<G, true><<<dim3((unsigned)(x.joined * (2 * G))), kChunkJoin, 0, st>>>(a, x.many, x.few, x.few_ws);
  else
    k_chunk_join<G, false><<<dim3((unsigned)std::min<size_t>(2048, x.joined / 4)), kChunkJoin, 0, st>>>(a, x.many, x.few, x.few_ws);
  return hipGetLastError();
}

hipError_t launch_paged_chunk(const PagedChunk& a, hipStream_t st) {
  ChunkCuts x;
  if (!chunk_cuts(a.c, a.hq, a.total, a.max_new, &x)) return hipErrorInvalidValue;
  return a.c.D == 64 ? launch_chunk<1>(a, x, st) : a.c.D == 128 ? launch_chunk<2>(a, x, st) : launch_chunk<4>(a, x, st);
}

}  // namespace hifa4
