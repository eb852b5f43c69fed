// Attention of each sequence's last tokens over the paged cache (records:
// hifa4_paged.h): chunks of prompts, drafted tokens, one token of each, mixed.
//
// Sequence b holds L tokens, its n new ones among them; query i < n stands at
// position L - n + i and sees the keys up to it:
//   S_j = (q~ . k_j) / sqrt(D),  p_j = exp(S_j - m) / l,  o = sum_j p_j v_j,
//   LSE = m + ln l,  with m = max S_j and l = sum_j exp(S_j - m).
// q~ = fp16(q s) under Smooth-QK.  The products run on fp16 operands with sums in
// fp32: q~ is fp16, and so is a cached HIF4 value (six significant bits; below
// 2^-14 it is rounded, by up to 1.125 2^-24: the base, its product with 2^-(E2 + E3)
// and that with the magnitude, over all that an append writes).  Scores, softmax
// state and o are held in fp32; p is rounded to fp16 for the second product,
// relative to the heaviest key so far (2^7 to 2^15), and o is divided by the sum of
// the rounded p: a row that rests on one key has exactly that key's value.  LSE
// takes the sum of p itself.
//
// The rows of a sequence, (token, query head of the kv head), are cut into tiles.
// All tiles' pages, one after another, are cut into equal shares, one for each
// workgroup that the chip holds: a share ends where it ends, inside a tile too, and
// a second kernel joins the parts of the tiles that were cut.  Lengths and counts
// are read on the device, so a captured call follows them.
//
// Bounds and times (MI355X, Hq=32, Hkv=8, D=128, HIF4 pages unless stated).  Few rows
// read each page once and make its values in registers: 32 sequences of 300 to 8192
// tokens, 5 new ones each, 65 us (57, and 10 in the join), of which the bytes take 33.  No
// unit is full: the VALU is busy 58% of the cycles, the matrix cores 13%, and a wave waits
// 15% of its own; the one-token decode reads the same records with fewer vector
// instructions, as FP4 operands.  Many rows are bound by the matrix instructions with the
// VALU beside them: 2048 tokens over 32768 in 1015 us, 1.05 PFLOP/s, where a matrix product
// of this library's speed (1.3) takes 819; without the softmax's exponentials and the
// making of operands it took 811.  16 prompts of 512 to 2048 tokens: 377 us, 7 us of each
// tile's beginning and end among 21 of its pages (a wave a tile, runs of pages of one
// length instead of equal shares: 712).
#include "hifa4_paged_device.h"

#include <algorithm>
#include <type_traits>

namespace hifa4 {

typedef half_t h4v_t __attribute__((ext_vector_type(4)));

// What the heaviest key so far counts: between 2^kTop and 2^(kTop + kSlack), below
// fp16's range; the softmax's reference moves when a score passes that.
constexpr float kTop = 7.0f, kSlack = 8.0f;
constexpr float kNoRef = -1e30f;        // before any key

// ---------------------------------------------------------------------------
// The plan, the same for every kv head.  Sequences of few rows and of many are two
// kinds of work, each with its own tiles and shares.
struct ChunkCut {
  int rows;                             // of a tile
  int above, upto;                      // sequences of more than `above` rows and at most `upto`
  int shares;                           // at most
  int tile_cost, least, whole;          // in pages: what a tile costs beside its own; the least share; a tile's
                                        // part of fewer than `whole` is left with the rest of it
};
struct ChunkSeq {
  int first, n;                         // row of q, new tokens (those that the launch holds)
  int len, base;                        // cached tokens, position of the first new one
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
__device__ __forceinline__ int scalar(int x) { return __builtin_amdgcn_readfirstlane(x); }
// The same in scalar registers.
__device__ __forceinline__ ChunkSeq seq_of(const PagedChunk& a, int b) {
  const ChunkSeq s = chunk_seq(a, scalar(b));
  return ChunkSeq{scalar(s.first), scalar(s.n), scalar(s.len), scalar(s.base)};
}
__device__ __forceinline__ ChunkSeq lane_seq(const ChunkSeq& s, int lane) {
  return ChunkSeq{__builtin_amdgcn_readlane(s.first, lane), __builtin_amdgcn_readlane(s.n, lane), __builtin_amdgcn_readlane(s.len, lane),
                  __builtin_amdgcn_readlane(s.base, lane)};
}
__device__ __forceinline__ int tiles_of(const ChunkSeq& s, int group, const ChunkCut& cut) {
  const int rows = s.n * group;
  return rows > cut.above && rows <= cut.upto ? (rows + cut.rows - 1) / cut.rows : 0;
}
// Pages that the rows of a tile see.
__device__ __forceinline__ int tile_pages(const ChunkSeq& s, int group, const ChunkCut& cut, int tile) {
  const int last = min(s.n - 1, ((tile + 1) * cut.rows - 1) / group);
  return max(0, s.base + last + kPage) / kPage;
}
// Cost of a sequence's first `tiles` tiles, counted in 1/group of a key: tile t's is
// tile_cost pages and the keys that it sees, about base + (t + 1) rows / group (with base
// near 2^31 beyond 31 bits).  Whole numbers in fp64; where they are too large for it,
// every wave still rounds alike.
__device__ __forceinline__ double tiles_cost(const ChunkSeq& s, int group, const ChunkCut& cut, int tiles) {
#pragma clang fp contract(off)
  const double t = tiles;
  return t * ((double)group * ((double)(kPage * cut.tile_cost) + (double)max(0, s.base))) + (double)cut.rows * (t * (t + 1.0) * 0.5);
}

// Sequences are in the order of the lanes that count them: b, b + 64, ..., then b + 1.
struct ChunkPlan {
  double before, upto, all;             // cost of the lanes before this one, up to it, of all
};
__device__ __forceinline__ int next_sequence(const PagedChunk& a, int b) {
  if (b + 64 < a.c.batch) return b + 64;
  b = (b & 63) + 1;
  return b < 64 && b < a.c.batch ? b : -1;
}
template <int kCtrl, int kRowMask, bool kBound>
__device__ __forceinline__ double add_dpp(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, kCtrl, kRowMask, 0xF, kBound);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), kCtrl, kRowMask, 0xF, kBound);
  return x + __builtin_bit_cast(double, (uint64_t)lo | (uint64_t)hi << 32);
}
__device__ __forceinline__ double lane_value(double x, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane) |
                                        (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane) << 32);
}
__device__ __forceinline__ void count_costs(ChunkPlan& p, const PagedChunk& a, const ChunkSeq& first, int group, const ChunkCut& cut, int lane) {
#pragma clang fp contract(off)
  double mine = tiles_cost(first, group, cut, tiles_of(first, group, cut));
  for (int b = lane + 64; b < a.c.batch; b += 64) {
    const ChunkSeq s = chunk_seq(a, b);
    mine += tiles_cost(s, group, cut, tiles_of(s, group, cut));
  }
  double sum = mine;
  sum = add_dpp<0x111, 0xF, true>(sum);      // row_shr 1, 2, 4, 8
  sum = add_dpp<0x112, 0xF, true>(sum);
  sum = add_dpp<0x114, 0xF, true>(sum);
  sum = add_dpp<0x118, 0xF, true>(sum);
  sum = add_dpp<0x142, 0xA, false>(sum);     // lane 15 of each row to the next
  sum = add_dpp<0x143, 0xC, false>(sum);
  p.before = sum - mine;
  p.upto = sum;
  p.all = lane_value(sum, 63);
}

// A place between two pages of the work: before page `page` of a tile, which is not
// behind its last one; tile may be the number of the sequence's tiles.  b < 0: the end.
struct Place {
  int b, tile, page;
};
__device__ __forceinline__ bool same_tile(const Place& x, const Place& y) { return x.b == y.b && x.tile == y.tile; }
// (`first`: lane l's sequence l)
__device__ __forceinline__ Place place_at(const ChunkPlan& p, const PagedChunk& a, const ChunkSeq& first, int group, const ChunkCut& cut,
                                          double x) {
#pragma clang fp contract(off)
  const unsigned long long who = __builtin_amdgcn_ballot_w64(x < p.upto);
  if (!who) return Place{-1, 0, 0};
  const int src = __builtin_ctzll(who);
  x -= lane_value(p.before, src);
  for (int b = src; b < a.c.batch; b += 64) {
    const ChunkSeq s = b < 64 ? lane_seq(first, b) : seq_of(a, b);
    const int tiles = tiles_of(s, group, cut);
    const double cost = tiles_cost(s, group, cut, tiles);
    if (!(x < cost) && b + 64 < a.c.batch) {
      x -= cost;
      continue;
    }
    if (tiles == 0) return Place{b, 0, 0};
    int t = 0, behind = tiles;           // the tile with cost(t) <= x < cost(t + 1)
    while (behind - t > 1) {
      const int mid = (t + behind) / 2;
      if (scalar((int)(tiles_cost(s, group, cut, mid) <= x)))
        t = mid;
      else
        behind = mid;
    }
    const double from = tiles_cost(s, group, cut, t), to = tiles_cost(s, group, cut, t + 1);
    const int pages = tile_pages(s, group, cut, t);
    const int page = max(0, min(pages, scalar((int)((x - from) / (to - from) * (double)pages))));
    if (page < cut.whole) return Place{b, t, 0};
    if (pages - page < cut.whole) return Place{b, t + 1, 0};
    return Place{b, t, page};
  }
  return Place{-1, 0, 0};
}

// A share of the work, walked tile by tile.
struct Share {
  Place at, to;                         // pages from at.page on
  ChunkSeq seq;
  int tiles, end;                       // of the sequence; the tile's last page (behind it) in the share
  bool ends;                            // the tile ends in the share
};
__device__ __forceinline__ Share share_of(const ChunkPlan& p, const PagedChunk& a, const ChunkSeq& first, int group, const ChunkCut& cut,
                                          int number, int shares) {
#pragma clang fp contract(off)
  Share s;
  // equal parts: at least `least` pages and a tile's cost
  const double least = (double)group * (double)(kPage * (cut.least + cut.tile_cost));
  const int parts = scalar((int)fmax(1.0, fmin((double)min(shares, cut.shares), floor(p.all / least))));
  s.at = s.to = Place{-1, 0, 0};
  if (number >= parts || p.all == 0.0) return s;
  const double each = p.all / (double)parts;
  s.at = place_at(p, a, first, group, cut, each * (double)number);
  if (number + 1 < parts) s.to = place_at(p, a, first, group, cut, each * (double)(number + 1));
  if (s.at.b >= 0) {
    s.seq = s.at.b < 64 ? lane_seq(first, s.at.b) : seq_of(a, s.at.b);
    s.tiles = tiles_of(s.seq, group, cut);
  }
  return s;
}
// The tile at s.at, or the next that there is; false: the share is over.
__device__ __forceinline__ bool enter_tile(Share& s, const PagedChunk& a, int group, const ChunkCut& cut) {
  for (;;) {
    if (s.at.b < 0 || (same_tile(s.at, s.to) && s.at.page >= s.to.page)) return false;
    if (s.at.tile < s.tiles) break;
    s.at = Place{next_sequence(a, s.at.b), 0, 0};
    if (s.at.b < 0) return false;
    s.seq = seq_of(a, s.at.b);
    s.tiles = tiles_of(s.seq, group, cut);
  }
  s.ends = !same_tile(s.at, s.to);
  s.end = s.ends ? tile_pages(s.seq, group, cut, s.at.tile) : s.to.page;
  return true;
}
__device__ __forceinline__ void leave_tile(Share& s) {
  if (s.ends)
    s.at = Place{s.at.b, s.at.tile + 1, 0};
  else
    s.at.page = s.end;
}
// The pages of a tile that are some: the table's entries 64 at a time, one a lane.
struct TilePages {
  Pages pg;
  int b, end, page;                     // `page`: of the pool, the one found last
};
__device__ __forceinline__ TilePages pages_of_tile(const Share& s) { return TilePages{Pages{0, s.at.page - 64}, s.at.b, s.end, 0}; }
// The first at or behind place j, or `end`.
__device__ __forceinline__ int next_page(TilePages& x, const PagedChunk& a, int j, int lane) {
  for (; j < x.end; ++j) {
    if (j - x.pg.base >= 64) load_pages(x.pg, a.c, x.b, j, x.end - 1, lane);
    x.page = __builtin_amdgcn_readlane(x.pg.mine, j - x.pg.base);
    if ((unsigned)x.page < (unsigned)a.c.num_pages) break;
  }
  return scalar(j);
}
template <int D, bool kFp16>
__device__ __forceinline__ const uint8_t* record_of(const TilePages& x, const PagedChunk& a, int head) {
  return a.c.pool + ((size_t)scalar(x.page) * a.c.hkv + head) * paged_record_bytes(D, kFp16);
}

// Workspace of a kind: o [shares][2][hkv][rows][D], then (m, l, l^, -) [shares][2][hkv]
// [rows], then what the shares cut.  A share leaves the part of a tile that began
// before it in its first place, that of one that goes on behind it in its second.
enum { kCutAfter = 1, kCutBefore = 2, kWithin = 4 };      // a tile goes on behind the share; began before it; both
struct Split {
  int how, tile;                        // the tile that begins in the share and goes on behind it
  ChunkSeq seq;
};
struct ChunkWs {
  float* o;
  float4* ml;
  Split* split;
};
__host__ __device__ __forceinline__ size_t chunk_ws_bytes(const PagedCache& c, const ChunkCut& cut) {
  return (size_t)2 * cut.shares * c.hkv * cut.rows * (c.D + 4) * 4 + cut.shares * sizeof(Split);
}
__device__ __forceinline__ ChunkWs chunk_ws(uint8_t* ws, const PagedCache& c, const ChunkCut& cut) {
  const size_t rows = (size_t)2 * cut.shares * c.hkv * cut.rows;
  ChunkWs w;
  w.o = reinterpret_cast<float*>(ws);
  w.ml = reinterpret_cast<float4*>(w.o + rows * c.D);
  w.split = reinterpret_cast<Split*>(w.ml + rows);
  return w;
}
__device__ __forceinline__ Split split_of(const PagedChunk& a, const Share& s) {
  Split x = {0, 0, {0, 0, 0, 0}};
  const bool before = s.at.b >= 0 && s.at.page > 0, within = before && same_tile(s.at, s.to);
  if (before) x.how = within ? kWithin : kCutBefore;
  if (s.to.b >= 0 && s.to.page > 0 && !within) x = Split{x.how | kCutAfter, s.to.tile, chunk_seq(a, s.to.b)};
  return x;
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
// E2 + E3 of words in both halves of a register, two bits each: of the words (t, 0) in
// `even`, of the words (t, 1) in `odd`, from bits 2t on (of E2's and E3's own 2t + c).
struct Exponents {
  uint32_t even, odd;
};
__device__ __forceinline__ Exponents add_exponents(uint32_t e3, uint32_t e2) {
  constexpr uint32_t kEven = 0x55555555u;
  return Exponents{(e3 & kEven) + (e2 & kEven), (e3 >> 1 & kEven) + (e2 >> 1 & kEven)};
}
// 2^-(E2 + E3) in both halves, from bit `bit` on.
__device__ __forceinline__ h2_t powers(uint32_t x, int bit) {
  return __builtin_bit_cast(h2_t, 0x3C003C00u - ((bit <= 10 ? x << (10 - bit) : x >> (bit - 10)) & 0x0C000C00u));
}
// The exponents of tile and tile ^ 1, and the operand of word (t, c) of a tile.
template <int G>
__device__ __forceinline__ Exponents exponents_of(const HifPart<G>& p, int tile) {
  const uint32_t e3 = G == 1 ? (p.e3[0] & 0xFFu) | ((p.e3[0] & 0xFF00u) << 8) : p.e3[tile / 2];
  return add_exponents(e3, (p.e2 >> (16 * (tile / 2)) & 0xFFFFu) * 0x10001u);
}
template <int G>
__device__ __forceinline__ h8v_t part_operand(const HifPart<G>& p, const Exponents& x, int tile, int t, int c, int lane) {
  const uint4 w = p.code[2 * tile + (t >> 1)];
  const uint32_t word = t & 1 ? (c ? w.w : w.z) : (c ? w.y : w.x);
  const uint32_t bases = t == 0 ? p.base[tile].x : t == 1 ? p.base[tile].y : t == 2 ? p.base[tile].z : p.base[tile].w;
  const half_t b = (half_t)__uint_as_float(((bases >> (8 * (lane & 3)) & 0xFFu) << 21) + 0x30000000u);
  return hif4_operand(word, h2_t{b, b} * powers(c ? x.odd : x.even, 8 * (tile & 1) + 2 * t));
}

// ---------------------------------------------------------------------------
// Rows: 16 columns of a matrix product, one a lane (lane 16k + n holds column n's share k).
struct Row {
  int limit;                            // the last key that it sees; -1: none, -2: no such row
  int at;                               // row of q and o (token, query head)
};
__device__ __forceinline__ Row row_of(const PagedChunk& a, const ChunkSeq& s, int group, int head, int row) {
  const int token = row / group, g = row - token * group;
  if (token >= s.n) return Row{-2, 0};
  return Row{max(-1, s.base + token), (s.first + token) * a.hq + head * group + g};
}

// q s of eight channels, the exact products rounded once.  The fp32 products rounded to
// fp16 are that but where one lies half way between fp16 numbers (normal ones: its low 13
// bits are 1 and zeros) or below them: seldom, and then all eight take the longer way
// (12 instructions each in place of 4).
__device__ __forceinline__ h8v_t round_products(const h8v_t& q, const f4v_t (&s)[2]) {
  float x[8];
  int half_way = 0;
  float least = INFINITY;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[e] = (float)q[e] * s[e >> 2][e & 3];
    half_way = min(half_way, (int)(__float_as_uint(x[e]) << 19));
    least = fminf(least, fabsf(x[e]));
  }
  h8v_t to;
  if (__builtin_amdgcn_ballot_w64(half_way == (int)0x80000000 || !(least >= 0x1p-14f))) {
#pragma unroll
    for (int e = 0; e < 8; ++e) to[e] = round_product(q[e], s[e >> 2][e & 3]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) to[e] = (half_t)x[e];
  }
  return to;
}

// The queries' operands: step c's channels of lane k, in the order of the keys'.  All
// loads are on their way before the first is used.
template <int G, bool kFp16, int NB>
__device__ __forceinline__ void load_queries(h8v_t (&q)[NB][2 * G], const PagedChunk& a, const Row (&r)[NB], int head, int k) {
  const auto channel = [k](int c) { return kFp16 ? 32 * c + 8 * k : 64 * (c >> 1) + 16 * k + 8 * (c & 1); };
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const half_t* row = a.q + (size_t)r[i].at * (64 * G);      // (the first row where there is none)
#pragma unroll
    for (int c = 0; c < 2 * G; ++c) q[i][c] = *reinterpret_cast<const h8v_t*>(row + channel(c));
  }
  if (a.s) {
    f4v_t s[2 * G][2];
#pragma unroll
    for (int c = 0; c < 2 * G; ++c) {
      const f4v_t* from = reinterpret_cast<const f4v_t*>(a.s + (size_t)head * (64 * G) + channel(c));
      s[c][0] = from[0];
      s[c][1] = from[1];
    }
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int c = 0; c < 2 * G; ++c)
        q[i][c] = round_products(q[i][c], s[c]);
  }
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int c = 0; c < 2 * G; ++c) {
      if (r[i].limit == -2) q[i][c] = h8v_t{0, 0, 0, 0, 0, 0, 0, 0};
      if (!kFp16) q[i][c] = __builtin_shufflevector(q[i][c], q[i][c], 0, 4, 1, 5, 2, 6, 3, 7);
    }
}

// The state of 16 rows' softmax, and their sums.
// The sum of p as it was rounded is a lane's share, by dot products; or, where the vector
// instructions have more to do than the matrix instructions, the whole sum by a product.
template <int G, bool kDot>
struct Rows16 {
  float ref, l;                         // p = 2^(score - ref), scores in log2 units; l: the lane's share of its sum
  std::conditional_t<kDot, float, f4v_t> sum;
  f4v_t o[4 * G];                       // channels 16 ct + 4k + v
};
template <int G, bool kDot>
__device__ __forceinline__ void start(Rows16<G, kDot>& x) {
  const f4v_t z = {0.0f, 0.0f, 0.0f, 0.0f};
  x.ref = kNoRef;
  x.l = 0.0f;
  x.sum = {};
#pragma unroll
  for (int c = 0; c < 4 * G; ++c) x.o[c] = z;
}

// A page's scores (s[t][v]: key 16k + 4t + v, before the scale) to the second product's
// operands; keys behind `seen` (the row's limit in the page) do not count.
template <int G, bool kFp16, bool kDot>
__device__ __forceinline__ void soften(Rows16<G, kDot>& x, f4v_t (&s)[4], h8v_t (&p)[2], float scale, bool masked, int seen, int k) {
  if (masked) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (4 * t + v > seen - 16 * k) s[t][v] = -INFINITY;
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
    if constexpr (kDot)
#pragma unroll
      for (int i = 0; i < 8; i += 2) x.sum = __builtin_amdgcn_fdot2(h2_t{p[c][i], p[c][i + 1]}, h2_t{1, 1}, x.sum, false);
  }
}

__device__ __forceinline__ f4v_t product(h8v_t a, h8v_t b, f4v_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Values of FP16 pages that some rows of a tile must not see: 0 times them has to be 0
// also where they are infinite or NaN.  Of the keys that no row sees they are cleared;
// of the others what is not finite is counted, per sign, over the keys that a row sees
// (products of ones; NaN under both signs), and cleared: what it makes of the row's sums
// is added when the tile ends.
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
// Bits 0 to 3: the lane's channels to which an infinity or NaN comes, 4 to 7: to which a
// negative infinity or NaN does.
__device__ __forceinline__ int count_not_finite(const u4v_t (&v)[2], int seen, int k) {
  f4v_t up = {0.0f, 0.0f, 0.0f, 0.0f}, down = up;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const u4v_t odd = not_finite(v[c]), nan = ((v[c] & 0x03FF03FFu) + 0x7FFF7FFFu), minus = v[c];
    const h8v_t who = __builtin_bit_cast(h8v_t, first_halves(seen + 1 - 16 * k - 8 * c) & 0x3C003C00u);
    up = product(__builtin_bit_cast(h8v_t, one(odd & (nan | ~minus))), who, up);
    down = product(__builtin_bit_cast(h8v_t, one(odd & (nan | minus))), who, down);
  }
  int bits = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) bits |= (up[i] > 0.0f ? 1 << i : 0) | (down[i] > 0.0f ? 16 << i : 0);
  return bits;
}

// Leaves 16 rows of a tile: rounded and divided, or (`part` >= 0, a place of the
// workspace) as a share's part.
template <int G, bool kDot>
__device__ __forceinline__ void finish(const PagedChunk& a, const ChunkWs& ws, long part, Rows16<G, kDot>& x, const Row& r, int head,
                                       int tile_rows, int row_in_tile, int k) {
  constexpr int D = 64 * G;
  const float l = sum_across_rows(x.l);
  float sum;
  if constexpr (kDot)
    sum = sum_across_rows(x.sum);
  else
    sum = x.sum[0];
  if (r.limit == -2) return;
  if (part < 0) {
    const float by = sum == 0.0f ? 0.0f : 1.0f / sum;
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
  const size_t at = ((size_t)part * a.c.hkv + head) * tile_rows + row_in_tile;
#pragma unroll
  for (int c = 0; c < 4 * G; ++c) *reinterpret_cast<f4v_t*>(ws.o + at * D + 16 * c + 4 * k) = x.o[c];
  if (k == 0) ws.ml[at] = make_float4(l == 0.0f ? -INFINITY : x.ref, l, sum, 0.0f);
}
// The place of a share's part of its present tile; -1: the whole tile is the share's.
__device__ __forceinline__ long part_of(const Share& s, int number) {
  return s.at.page > 0 ? 2L * number : s.ends ? -1L : 2L * number + 1;
}

// ---------------------------------------------------------------------------
// Few rows over HIF4 pages.
// One wave per (share, kv head): tiles of 16 NB rows; the operands are made of a page's
// record in registers, one 16-byte load a lane for each KiB: no barrier, and 8 waves a CU
// hide each other's loads.  About 21 vector instructions make the eight values of a word
// (E2 + E3 as one field: 2.5 fewer, 74 to 72 us for the 32 sequences above).  K of the next page is
// fetched once this one's has been used, V while the scores are made.
template <int G, int NB>
__device__ __forceinline__ void chunk_rows(const PagedChunk& a, const ChunkCut& cut, uint8_t* ws_at, const ChunkPlan& plan,
                                           const ChunkSeq& first, int number, int shares, int head, int lane) {
  constexpr int D = 64 * G, kRows = 16 * NB;
  const int n = lane & 15, k = lane >> 4, group = a.hq / a.c.hkv;
  const ChunkWs ws = chunk_ws(ws_at, a.c, cut);
  Share s = share_of(plan, a, first, group, cut, number, shares);
  if (head == 0 && lane == 0) ws.split[number] = split_of(a, s);
  HifPart<G> k4, v4;
  for (; enter_tile(s, a, group, cut); leave_tile(s)) {
    TilePages tp = pages_of_tile(s);
    int j = next_page(tp, a, s.at.page, lane);
    const uint8_t* rec = record_of<D, false>(tp, a, head);
    if (j < s.end) load_hif4<G>(k4, rec, lane);
    Row row[NB];
    Rows16<G, true> x[NB];
    h8v_t q[NB][2 * G];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      row[i] = row_of(a, s.seq, group, head, s.at.tile * kRows + 16 * i + n);
      start(x[i]);
    }
    load_queries<G, false, NB>(q, a, row, head, k);
    const int all_see = s.seq.base + s.at.tile * kRows / group;     // every row of the tile sees the keys up to this one
    while (j < s.end) {
      const int key0 = j * kPage;
      const bool masked = key0 + kPage - 1 > all_see;
      keep_order();
      load_hif4<G>(v4, rec + 2304 * G, lane);
      keep_order();
      f4v_t sc[NB][4];
      h8v_t p[NB][2];
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) sc[i][t] = f4v_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < 2 * G; ++c) {
        const Exponents e = exponents_of(k4, c >> 1);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const h8v_t kr = part_operand<G>(k4, e, c >> 1, t, c & 1, lane);
#pragma unroll
          for (int i = 0; i < NB; ++i) sc[i][t] = product(kr, q[i][c], sc[i][t]);
        }
      }
      keep_order();
      j = next_page(tp, a, j + 1, lane);
      rec = record_of<D, false>(tp, a, head);
      if (j < s.end) load_hif4<G>(k4, rec, lane);
      keep_order();
#pragma unroll
      for (int i = 0; i < NB; ++i) soften<G, false, true>(x[i], sc[i], p[i], a.scale, masked, row[i].limit - key0, k);
      keep_order();
#pragma unroll
      for (int u = 0; u < 4 * G; ++u) {
        const Exponents e = exponents_of(v4, u >> 2);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const h8v_t vr = part_operand<G>(v4, e, u >> 2, u & 3, c, lane);
#pragma unroll
          for (int i = 0; i < NB; ++i) x[i].o[u] = product(vr, p[i][c], x[i].o[u]);
        }
      }
    }
    const long part = part_of(s, number);
#pragma unroll
    for (int i = 0; i < NB; ++i) finish(a, ws, part, x[i], row[i], head, kRows, 16 * i + n, k);
  }
}

template <int G, int NB>
__global__ void __launch_bounds__(64, G == 4 ? 1 : 2) k_chunk_rows(PagedChunk a, ChunkCut cut) {
  ChunkPlan plan;
  const ChunkSeq first = chunk_seq(a, threadIdx.x);         // the first 64 sequences are read once
  count_costs(plan, a, first, a.hq / a.c.hkv, cut, threadIdx.x);
  chunk_rows<G, NB>(a, cut, a.ws, plan, first, blockIdx.x / a.c.hkv, cut.shares, blockIdx.x % a.c.hkv, threadIdx.x);
}

// ---------------------------------------------------------------------------
// Many rows: kWaves waves of 16 NB rows each share a page, whose operands they make in
// LDS (two pages' room: the next one is made while this one is used).  A record's KiB
// unit of fp16 operands is what a wave reads for one operand of a product, 16 bytes a
// lane in lane order, so neither reads nor writes have bank conflicts.  Over FP16 pages
// a few rows are a workgroup of one wave.  A page of HIF4 operands takes a workgroup 4700
// cycles, of which the matrix instructions are 2180: making the operands costs the eight
// waves 15% (1038 to 889 us without, 2048 tokens over 32768), the exponentials 8%.  FP16
// pages are copied past the registers; D=256 has one wave a SIMD and no other to fill
// its waits: 4 x 201 tokens over 1000 to 8192, Hq=16, 175 to 178 us (floor 50).
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
  const Exponents x = add_exponents((G == 1 ? (q.e3 & 0xFFu) | ((q.e3 & 0xFF00u) << 8) : q.e3) >> (8 * (tile & 1) + 4 * half),
                                    (q.e2 * 0x10001u) >> (4 * half));
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const half_t b = (half_t)__uint_as_float((((u ? q.base.y : q.base.x) >> (8 * (lane & 3)) & 0xFFu) << 21) + 0x30000000u);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const uint32_t word = u ? (c ? q.code.w : q.code.z) : (c ? q.code.y : q.code.x);
      const int t = 2 * half + u, unit = is_v ? 8 * G + (4 * tile + t) * 2 + c : t * 2 * G + 2 * tile + c;
      page[64 * unit + lane] = hif4_operand(word, h2_t{b, b} * powers(c ? x.odd : x.even, 2 * u));
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
// the compiler keeps no value of its own in M0, and puts no wait between the two.
template <int G, int kWaves>
__device__ __forceinline__ void copy_share(h8v_t* page, const uint8_t* rec, int wave, int lane) {
  const uint64_t from = (uint64_t)(uintptr_t)(rec + 16384 * G / kWaves * wave);
  const uint64_t at = (uint64_t)(uint32_t)scalar((int)from) | (uint64_t)(uint32_t)scalar((int)(from >> 32)) << 32;
  uint32_t to = (uint32_t)scalar((int)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)(page + 1024 * G / kWaves * wave));
  uint32_t offset = 16 * lane;            // (goes along in one register: eight or more kept for the loop would be spilled)
#pragma unroll
  for (int i = 0; i < 16 * G / kWaves; ++i)
    asm volatile("s_mov_b32 m0, %1\n\t" HIFA4_M0_WAIT
                 "global_load_lds_dwordx4 %0, %2\n\tv_add_u32 %0, 0x400, %0\n\ts_add_u32 %1, %1, 0x400"
                 : "+v"(offset), "+s"(to)
                 : "s"(at)
                 : "memory", "m0", "scc");
}
__device__ __forceinline__ void wait_copies() { __builtin_amdgcn_s_waitcnt(0x0F70); }     // vmcnt(0)

// How many of a head's workgroups take the sequences of many rows where there are both
// kinds: by the time that their pages take.  A page of 16 rows on one of a workgroup's
// waves counts kFewTime of one of 256 rows on all of them (prompts and single tokens in
// one batch of 35: 155 us, with 0.14 210, with 0.28 167; of 256: 368, 431, 366).
constexpr float kFewTime = 0.2f;
__device__ __forceinline__ int many_shares(double many, double few, int shares) {
  if (few == 0.0) return shares;
  if (many == 0.0) return 0;
  const float m = (float)many, f = kFewTime * (float)few;
  return max(1, min(shares - 1, (int)((float)shares * m / (m + f) + 0.5f)));
}

template <int G, bool kFp16, int kWaves, int NB>
__global__ void __launch_bounds__(64 * kWaves, G == 4 || kWaves == 1 ? 1 : 2) k_chunk_wide(PagedChunk a, ChunkCut cut, ChunkCut few, size_t few_ws) {
  constexpr int D = 64 * G, kMine = 16 * NB, kRows = kMine * kWaves, kUnits = 16 * G;
  static_assert(16 * G % kWaves == 0 && 4 * G % kWaves == 0, "equal shares");
  extern __shared__ __align__(16) uint8_t smem[];
  h8v_t* const pages = reinterpret_cast<h8v_t*>(smem);
  const int lane = threadIdx.x & 63, n = lane & 15, k = lane >> 4;
  const int wave = scalar((int)(threadIdx.x >> 6));
  const int head = blockIdx.x % a.c.hkv, group = a.hq / a.c.hkv, number = blockIdx.x / a.c.hkv;
  const ChunkWs ws = chunk_ws(a.ws, a.c, cut);
  ChunkPlan plan;
  const ChunkSeq first = chunk_seq(a, lane);                // the first 64 sequences are read once
  count_costs(plan, a, first, group, cut, lane);
  int shares = cut.shares;
  if constexpr (!kFp16) {
    ChunkPlan other;
    count_costs(other, a, first, group, few, lane);
    shares = scalar(many_shares(plan.all, other.all, cut.shares));
    const int rest = cut.shares - shares;
    Split* const split = chunk_ws(a.ws + few_ws, a.c, few).split;
    if (number >= shares) {               // the rest of the workgroups: a share a wave
      if (head == 0 && threadIdx.x == 0) ws.split[number] = Split{};
      chunk_rows<G, 1>(a, few, a.ws + few_ws, other, first, wave * rest + number - shares, rest * kWaves, head, lane);
      return;
    }
    if (head == 0 && lane == 0) split[rest * kWaves + number * kWaves + wave] = Split{};
  }
  Share s = share_of(plan, a, first, group, cut, number, shares);
  if (head == 0 && threadIdx.x == 0) ws.split[number] = split_of(a, s);
  HifShare<G, kWaves> share;
  // what is not finite and comes to the lane's sums: [channels / 16][lane][16 rows]
  uint8_t* const odd_sums = smem + 2 * 1024 * kUnits + (wave * 4 * G * 64 + lane) * NB;
  for (; enter_tile(s, a, group, cut); leave_tile(s)) {
    // page j is in LDS, page `ahead` on its way (HIF4) or next to be copied
    TilePages tp = pages_of_tile(s);
    int j = next_page(tp, a, s.at.page, lane), at = 0;
    if (j < s.end) {
      if constexpr (kFp16)
        copy_share<G, kWaves>(pages, record_of<D, true>(tp, a, head), wave, lane);
      else
        share.load(record_of<D, false>(tp, a, head), wave, lane);
    }
    const int row0 = s.at.tile * kRows + wave * kMine;      // the wave's first row
    Row row[NB];
    Rows16<G, kFp16> x[NB];
    h8v_t q[NB][2 * G];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      row[i] = row_of(a, s.seq, group, head, row0 + 16 * i + n);
      start(x[i]);
    }
    load_queries<G, kFp16, NB>(q, a, row, head, k);
    // keys that every row of the wave sees, and that any of them sees: up to these
    const int first_token = row0 / group, last_token = min(s.seq.n - 1, (row0 + kMine - 1) / group);
    const int all_see = s.seq.base + first_token, some_see = first_token < s.seq.n ? s.seq.base + last_token : -1;
    bool any_odd = false;
    int ahead = next_page(tp, a, j + 1, lane);
    if constexpr (kFp16) {
      wait_copies();
    } else {
      if (j < s.end) share.store(pages, wave, lane);
      if (ahead < s.end) share.load(record_of<D, false>(tp, a, head), wave, lane);
    }
    __syncthreads();
    while (j < s.end) {
      const h8v_t* page = pages + 64 * kUnits * at + lane;
      const int key0 = j * kPage;
      j = ahead;
      if (j < s.end) {
        h8v_t* const other = pages + 64 * kUnits * (at ^ 1);
        if constexpr (kFp16) {
          copy_share<G, kWaves>(other, record_of<D, true>(tp, a, head), wave, lane);
          ahead = next_page(tp, a, j + 1, lane);
        } else {
          share.store(other, wave, lane);
          ahead = next_page(tp, a, j + 1, lane);
          if (ahead < s.end) share.load(record_of<D, false>(tp, a, head), wave, lane);
        }
      }
      if (key0 <= some_see) {
        const bool masked = key0 + kPage - 1 > all_see;
        f4v_t sc[NB][4];
        h8v_t p[NB][2];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int t = 0; t < 4; ++t) sc[i][t] = f4v_t{0.0f, 0.0f, 0.0f, 0.0f};
        // Operands come some units ahead of their products: a wave's own products have to
        // cover LDS's latency, there are two waves a SIMD (one at D=256, where four units
        // ahead spill: 769 us for 2 x 1000 tokens over 8000, with two 757).
        constexpr int kAhead = G == 4 ? 2 : 4, kGroups = 8 * G / kAhead;
        h8v_t next[2][kAhead];
        const auto k_unit = [&](int e) { return page[64 * (e % 4 * 2 * G + e / 4)]; };
        const auto v_unit = [&](int e) { return page[64 * (8 * G + e)]; };
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int e = 0; e < kAhead; ++e) next[0][e] = k_unit(e);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          if (g + 1 < kGroups)
#pragma unroll
            for (int e = 0; e < kAhead; ++e) next[(g + 1) & 1][e] = k_unit((g + 1) * kAhead + e);
#pragma unroll
          for (int e = 0; e < kAhead; ++e) {
            const int at_unit = g * kAhead + e, c = at_unit / 4, t = at_unit % 4;
#pragma unroll
            for (int i = 0; i < NB; ++i) sc[i][t] = product(next[g & 1][e], q[i][c], sc[i][t]);
          }
        }
        __builtin_amdgcn_sched_group_barrier(kDsRead, kAhead, 0);
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          if (g + 1 < kGroups) __builtin_amdgcn_sched_group_barrier(kDsRead, kAhead, 0);
          __builtin_amdgcn_sched_group_barrier(kMatrix, kAhead * NB, 0);
        }
        keep_order();
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int e = 0; e < kAhead; ++e) next[0][e] = v_unit(e);
#pragma unroll
        for (int i = 0; i < NB; ++i) soften<G, kFp16, kFp16>(x[i], sc[i], p[i], a.scale, masked, row[i].limit - key0, k);
        keep_order();
        const bool odd_values = kFp16 && masked;
        __builtin_amdgcn_s_setprio(1);
        if constexpr (!kFp16)
#pragma unroll
          for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int c = 0; c < 2; ++c) x[i].sum = product(h8v_t{1, 1, 1, 1, 1, 1, 1, 1}, p[i][c], x[i].sum);
        if (odd_values) {
          bool odd = false;
#pragma unroll 1
          for (int u = 0; u < 8 * G; ++u)
            odd |= any(not_finite(__builtin_bit_cast(u4v_t, page[64 * (8 * G + u)]) & first_halves(some_see - key0 + 1 - 16 * k - 8 * (u & 1))));
          const bool found = __builtin_amdgcn_ballot_w64(odd) != 0;
          if (found) {
#pragma unroll 1
            for (int u = 0; u < 4 * G; ++u) {
              u4v_t v[2];
#pragma unroll
              for (int c = 0; c < 2; ++c)
                v[c] = __builtin_bit_cast(u4v_t, page[64 * (8 * G + 2 * u + c)]) & first_halves(some_see - key0 + 1 - 16 * k - 8 * c);
#pragma unroll
              for (int i = 0; i < NB; ++i) {
                uint8_t* const bits = odd_sums + u * 64 * NB + i;
                *bits = (uint8_t)(count_not_finite(v, row[i].limit - key0, k) | (any_odd ? *bits : 0));
              }
            }
            any_odd = true;
          }
#pragma unroll
          for (int u = 0; u < 4 * G; ++u)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              u4v_t v = __builtin_bit_cast(u4v_t, page[64 * (8 * G + 2 * u + c)]) & first_halves(some_see - key0 + 1 - 16 * k - 8 * c);
              if (found) v &= ~whole(not_finite(v));
#pragma unroll
              for (int i = 0; i < NB; ++i) x[i].o[u] = product(__builtin_bit_cast(h8v_t, v), p[i][c], x[i].o[u]);
            }
        } else {
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            if (g + 1 < kGroups)
#pragma unroll
              for (int e = 0; e < kAhead; ++e) next[(g + 1) & 1][e] = v_unit((g + 1) * kAhead + e);
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
              const int at_unit = g * kAhead + e, u = at_unit / 2, c = at_unit % 2;
#pragma unroll
              for (int i = 0; i < NB; ++i) x[i].o[u] = product(next[g & 1][e], p[i][c], x[i].o[u]);
            }
          }
#pragma unroll
          for (int g = 0; g < kGroups; ++g) {
            if (g + 1 < kGroups) __builtin_amdgcn_sched_group_barrier(kDsRead, kAhead, 0);
            __builtin_amdgcn_sched_group_barrier(kMatrix, kAhead * NB, 0);
          }
          keep_order();
        }
        __builtin_amdgcn_s_setprio(0);
      }
      at ^= 1;
      if constexpr (kFp16) wait_copies();
      __syncthreads();
    }
    if (any_odd) {
#pragma unroll
      for (int u = 0; u < 4 * G; ++u)
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          const int bits = odd_sums[u * 64 * NB + i];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[i].o[u][e] += bits >> e & 1 ? INFINITY : 0.0f;
            x[i].o[u][e] -= bits >> (4 + e) & 1 ? INFINITY : 0.0f;
          }
        }
    }
    const long part = part_of(s, number);
#pragma unroll
    for (int i = 0; i < NB; ++i) finish(a, ws, part, x[i], row[i], head, kRows, wave * kMine + 16 * i + n, k);
  }
}

// ---------------------------------------------------------------------------
// Joining the parts of a row that several shares hold: with m the largest of their
// references, o = sum o_i 2^(m_i - m) / sum l^_i 2^(m_i - m), l = sum l_i 2^(m_i - m), in
// the shares' order.  kFew: a workgroup takes 32 channels of a row, its threads share out
// the parts (many, where there are few rows); else a wave takes a row.  A workgroup reads
// once what the shares have cut and goes through its part of it.  Bound by the latency of
// dependent loads: 7 to 14 us, 29 after 2048 tokens over 32768 (64 parts of 256 rows a
// head at most: 104 MB).
constexpr int kChunkJoin = 256, kMostShares = 2048;

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

constexpr int kJoinRows = 4;           // of a workgroup where a wave takes a row

template <int G, bool kFew>
__device__ __forceinline__ void join_tiles(const PagedChunk& a, const ChunkCut& cut, uint8_t* ws_at, Joined* part, uint8_t* how,
                                           short* cuts, int* counts) {
  constexpr int D = 64 * G, kCols = kFew ? 8 : D / 4, kSets = (kFew ? kChunkJoin : 64) / kCols, kAhead = 4;
  const int tid = threadIdx.x, lane = tid & 63, at_set = kFew ? tid : lane, col = at_set % kCols, set = at_set / kCols;
  const ChunkWs ws = chunk_ws(ws_at, a.c, cut);
  const int group = a.hq / a.c.hkv;
  // the shares behind which a tile goes on, in order
  int found = 0;
  for (int i0 = 0; i0 < cut.shares; i0 += kChunkJoin) {
    const int i = i0 + tid, h = i < cut.shares ? ws.split[i].how : 0;
    if (i < cut.shares) how[i] = (uint8_t)h;
    const unsigned long long who = __builtin_amdgcn_ballot_w64(h & kCutAfter);
    if (lane == 0) counts[tid >> 6] = __popcll(who);
    __syncthreads();
    int to = found + __popcll(who & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < kChunkJoin / 64; ++w) {
      if (w < tid >> 6) to += counts[w];
      found += counts[w];
    }
    if (h & kCutAfter) cuts[to] = (short)i;
    __syncthreads();
  }
  // of such a share and a head: kFew rows times slices of 32 channels, else sets of kJoinRows rows
  const int per = kFew ? cut.rows * (D / 32) : cut.rows / kJoinRows;
  for (int block = blockIdx.x; block < found * a.c.hkv * per; block += gridDim.x) {
    const int first = cuts[block / per / a.c.hkv], head = block / per % a.c.hkv;
    const Split sp = ws.split[first];
    int parts = 2;                       // the shares that lie within the tile, then the one that it ends in
    for (int from = first + 1; from < cut.shares; from += 64) {
      const bool goes_on = from + lane < cut.shares && (how[from + lane] & kWithin);
      const unsigned long long stops = ~__builtin_amdgcn_ballot_w64(goes_on);
      parts += stops ? __builtin_ctzll(stops) : 64;
      if (stops) break;
    }
    const int ch = (kFew ? block % per % (D / 32) * 32 : 0) + 4 * col;
#pragma unroll
    for (int r = 0; r < (kFew ? 1 : kJoinRows / 4); ++r) {
      const int row_in_tile = kFew ? block % per / (D / 32) : block % per * kJoinRows + 4 * r + (int)(threadIdx.x >> 6);
      const Row row = row_of(a, sp.seq, group, head, sp.tile * cut.rows + row_in_tile);
      if (row.limit == -2) continue;
      Joined x = {-INFINITY, 0.0f, 0.0f, {0.0f, 0.0f, 0.0f, 0.0f}};
      for (int i = set; i < parts; i += kAhead * kSets) {
        float4 ml[kAhead];
        f4v_t y[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int share = first + min(i + u * kSets, parts - 1);
          const size_t from = (((size_t)2 * share + (share == first)) * a.c.hkv + head) * cut.rows + row_in_tile;
          ml[u] = ws.ml[from];
          y[u] = *reinterpret_cast<const f4v_t*>(ws.o + from * D + ch);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (i + u * kSets < parts) join_pair(x, Joined{ml[u].x, ml[u].y, ml[u].z, y[u]});
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
}
template <int G, bool kFew>
__global__ void __launch_bounds__(kChunkJoin) k_chunk_join(PagedChunk a, ChunkCut cut, ChunkCut few, size_t few_ws) {
  __shared__ Joined part[kFew ? kChunkJoin : 1];
  __shared__ uint8_t how[kMostShares];
  __shared__ short cuts[kMostShares];
  __shared__ int counts[kChunkJoin / 64];
  if (cut.shares > 1) join_tiles<G, kFew>(a, cut, a.ws, part, how, cuts, counts);
  __syncthreads();
  if (few.shares > 1) join_tiles<G, kFew>(a, few, a.ws + few_ws, part, how, cuts, counts);
}

// ---------------------------------------------------------------------------
// Rows (of one sequence and kv head) up to which a wave of its own takes them.  Of 32
// sequences of 300 to 8192 tokens 20 rows each: 65 us, by the workgroups of 256 rows 143;
// 32 rows: 68 and 143 (D=64: 43 and 78).  The workgroups take 40 and 64 rows in 147 and 148
// us (D=64 92), a wave's tiles of 32 would in 102 and 105 (67 and 69): between 33 and about
// 128 rows there is no kind of their own.
constexpr int kFewRows = 32;
// Waves of a workgroup that share a page.  At D=128 eight, two a SIMD: 16 prompts 377 us,
// with four 605.  D=64 has four shares of a page and two workgroups a CU; at D=256 two
// waves a SIMD do not hold 32 rows' sums.
constexpr int wide_waves(int D) { return D == 128 ? 8 : 4; }
// Workgroups that the chip holds at once: by the registers of their waves, or by their
// LDS where one wave copies FP16 pages.
constexpr int resident(int D, bool fp16, int waves) {
  return waves > 1 ? (D == 64 ? 512 : 256) : fp16 ? (D == 64 ? 1024 : D == 128 ? 512 : 256) : D == 256 ? 1024 : 2048;
}

struct ChunkCuts {
  int waves;                            // of a workgroup
  ChunkCut many, few;
  size_t few_ws, blocks, joined, bytes; // offset in the workspace; workgroups; rows that may be joined
};
// tile_cost, least, whole of many rows over HIF4: 4, 4 and 10 pages.  16 prompts: 377 us,
// with a tile's cost at 1 425, with parts of six pages kept apart 383; `least` says
// only how small a share of small calls may be (16: no difference there).
// Shares of a kind: those that `most` workgroups (or waves) of a head take, if there can be as many.
static int most_shares(const PagedCache& c, const ChunkCut& cut, size_t tiles, size_t most) {
  const size_t all = tiles * ((size_t)c.max_pages + cut.tile_cost) / (cut.least + cut.tile_cost) + 1;
  return (int)std::min(all, most);
}
static bool chunk_cuts(const PagedCache& c, int hq, int total, int max_new, ChunkCuts* x) {
  const size_t group = hq / c.hkv, most = max_new * group, all = (size_t)total * group, batch = c.batch;
  if (most >= (size_t)1 << 30) return false;
  const bool wide = most > kFewRows, both = wide && !c.fp16;
  x->waves = wide ? wide_waves(c.D) : 1;
  const size_t per_head = std::max<size_t>(both ? 2 : 1, resident(c.D, c.fp16, x->waves) / c.hkv);
  x->many = ChunkCut{wide ? 32 * x->waves : most <= 16 ? 16 : 32, c.fp16 ? 0 : kFewRows, 1 << 30, 0, wide ? 4 : 1, wide ? 4 : 2, wide ? 10 : 1};
  x->few = ChunkCut{!wide && most > 16 && c.D != 256 ? 32 : 16, 0, kFewRows, 0, 1, 2, 1};
  const auto tiles = [&](const ChunkCut& cut, size_t seqs, size_t rows) {
    return std::min(seqs * ((rows + cut.rows - 1) / cut.rows), all / cut.rows + seqs);
  };
  if (both) {                             // the few's waves come in the same workgroups
    x->many.shares = (int)per_head;
    x->few.shares = (int)per_head * x->waves;
  } else if (c.fp16) {
    x->many.shares = most_shares(c, x->many, tiles(x->many, batch, most), per_head);
  } else {
    x->few.shares = most_shares(c, x->few, tiles(x->few, batch, most), per_head);
  }
  const size_t many = x->many.shares ? (chunk_ws_bytes(c, x->many) + 255) / 256 * 256 : 0;
  x->few_ws = many;
  x->bytes = many + chunk_ws_bytes(c, x->few) + 16;
  x->blocks = (size_t)(x->many.shares ? x->many.shares : x->few.shares) * c.hkv;
  x->joined = ((size_t)(x->many.shares > 1 ? x->many.shares : 0) * x->many.rows +
               (size_t)(x->few.shares > 1 ? x->few.shares : 0) * x->few.rows) * c.hkv;
  return std::max(x->many.shares, x->few.shares) <= kMostShares && x->blocks < max_grid(64 * x->waves) && x->joined < (size_t)1 << 26;
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
  constexpr size_t kLds = (size_t)2 * 16 * G * 1024 + (kFp16 ? kWaves * 4 * G * 64 * NB : 0);
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
    e = x.waves > 1         ? launch_wide<G, true, wide_waves(64 * G), 2>(a, x, st)
        : x.many.rows == 16 ? launch_wide<G, true, 1, 1>(a, x, st)
                            : launch_wide<G, true, 1, 2>(a, x, st);
  } else if (x.waves > 1) {
    e = launch_wide<G, false, wide_waves(64 * G), 2>(a, x, st);
  } else {
    if (G == 4 || x.few.rows == 16)
      k_chunk_rows<G, 1><<<dim3((unsigned)x.blocks), 64, 0, st>>>(a, x.few);
    else
      k_chunk_rows<G == 4 ? 1 : G, 2><<<dim3((unsigned)x.blocks), 64, 0, st>>>(a, x.few);
    e = hipGetLastError();
  }
  if (e != hipSuccess || x.joined == 0) return e;
  // few rows in many parts: their parts shared out among a workgroup's threads.  One token,
  // one kv head: over 16384 cached ones (86 shares) 18.0 us, a wave a row 25.2; over 4096
  // (22 shares) 17.6 by either; over 2048 (11) 16.5 and 15.0.
  if (x.joined <= 2048 && std::max(x.many.shares, x.few.shares) > 24)
    k_chunk_join<G, true><<<dim3((unsigned)(x.joined * (2 * G))), kChunkJoin, 0, st>>>(a, x.many, x.few, x.few_ws);
  else
    k_chunk_join<G, false><<<dim3(2048), kChunkJoin, 0, st>>>(a, x.many, x.few, x.few_ws);
  return hipGetLastError();
}

hipError_t launch_paged_chunk(const PagedChunk& a, hipStream_t st) {
  ChunkCuts x;
  if (!chunk_cuts(a.c, a.hq, a.total, a.max_new, &x)) return hipErrorInvalidValue;
  return a.c.D == 64 ? launch_chunk<1>(a, x, st) : a.c.D == 128 ? launch_chunk<2>(a, x, st) : launch_chunk<4>(a, x, st);
}

}  // namespace hifa4
