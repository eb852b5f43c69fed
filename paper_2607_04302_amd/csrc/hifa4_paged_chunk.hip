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
constexpr int kMinRun = 4;              // pages that a run has at least, on average

// How a launch cuts its work: rows a tile, items aimed at, and its bounds (per kv head).
// A tile of P pages has at most 1 + P / per runs and, where it is split, fewer than
// 2 P / per; sum P / per over the tiles is at most the target (in fp32: and one more).
struct ChunkCut {
  int rows, target;
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
__device__ __forceinline__ int tiles_of(const ChunkSeq& s, int group, const ChunkCut& cut) { return ceil_div(s.n * group, cut.rows); }
// Pages that the rows of a tile see.
__device__ __forceinline__ int tile_pages(const ChunkSeq& s, int group, const ChunkCut& cut, int tile) {
  const int last = min(s.n - 1, ((tile + 1) * cut.rows - 1) / group);
  return max(0, s.base + last + kPage) / kPage;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return x;
}

// The item numbered r (found by a whole wave); false: no such item.  `joins`: the
// split tiles.  There are no items at all where the counts are no prefix sums of
// `total` (more rows than the launch and the workspace were sized for).
__device__ __forceinline__ bool find_item(const PagedChunk& a, int group, const ChunkCut& cut, int r, int lane, Item& it, int& joins) {
  float work = 0.0f, tokens = 0.0f;
  for (int b = lane; b < a.c.batch; b += 64) {
    const ChunkSeq s = chunk_seq(a, b);
    tokens += (float)s.n;
    work += (float)tiles_of(s, group, cut) * (float)ceil_div(s.len, kPage);
  }
  joins = 0;
  if (wave_sum(tokens) > (float)a.total * 1.001f) return false;
  const int per = max(kMinRun, (int)ceilf(fminf(wave_sum(work) / (float)cut.target, 0x1p25f)));
  const auto runs_of = [per](const ChunkSeq& s) { return max(1, ceil_div(ceil_div(s.len, kPage), per)); };
  int items = 0, tiles = 0, slots = 0;
  for (int b = lane; b < a.c.batch; b += 64) {
    const ChunkSeq s = chunk_seq(a, b);
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
    const ChunkSeq s = chunk_seq(a, b);
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
      it.seq.first = __builtin_amdgcn_readfirstlane(s.first);      // (the same in every lane: kept in scalar registers)
      it.seq.n = __builtin_amdgcn_readfirstlane(s.n);
      it.seq.len = __builtin_amdgcn_readfirstlane(s.len);
      it.seq.base = __builtin_amdgcn_readfirstlane(s.base);
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

// Workspace: o [slots][hkv][rows][D], then (m, l, l^, -) [slots][hkv][rows], then the
// split tiles, then their number.
struct Split {
  int b, tile, slot, runs;
};
struct ChunkWs {
  float* o;
  float4* ml;
  Split* split;
  int* joins;
};
__host__ __device__ __forceinline__ ChunkWs chunk_ws(uint8_t* ws, const PagedCache& c, const ChunkCut& cut) {
  const size_t rows = (size_t)cut.slots * c.hkv * cut.rows;
  ChunkWs w;
  w.o = reinterpret_cast<float*>(ws);
  w.ml = reinterpret_cast<float4*>(w.o + rows * c.D);
  w.split = reinterpret_cast<Split*>(w.ml + rows);
  w.joins = reinterpret_cast<int*>(w.split + cut.joins);
  return w;
}
static size_t chunk_ws_bytes(const PagedCache& c, const ChunkCut& cut) {
  return (size_t)cut.slots * c.hkv * cut.rows * (c.D + 4) * 4 + cut.joins * sizeof(Split) + 16;
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
__device__ __forceinline__ bool any_not_finite(const h8v_t& v) {
  typedef uint32_t u4v_t __attribute__((ext_vector_type(4)));
  const u4v_t x = (__builtin_bit_cast(u4v_t, v) & 0x7C007C00u) + 0x04000400u;
  return ((x[0] | x[1] | x[2] | x[3]) & 0x80008000u) != 0;
}
__device__ __forceinline__ h8v_t seen_keys(int seen, int first) {
  h8v_t x;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = first + i <= seen ? (half_t)1 : (half_t)0;
  return x;
}
template <int G>
__device__ __forceinline__ void add_not_finite(Rows16<G>& x, const h8v_t (&v)[2], int ct, int seen, int k) {
  const half_t inf = (half_t)INFINITY;
  f4v_t up = {0.0f, 0.0f, 0.0f, 0.0f}, down = up;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    h8v_t is_up, is_down;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      is_up[i] = v[c][i] < inf ? (half_t)0 : (half_t)1;
      is_down[i] = v[c][i] > -inf ? (half_t)0 : (half_t)1;
    }
    const h8v_t who = seen_keys(seen, 16 * k + 8 * c);
    up = product(is_up, who, up);
    down = product(is_down, who, down);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (up[i] > 0.0f) x.o[ct][i] += INFINITY;
    if (down[i] > 0.0f) x.o[ct][i] -= INFINITY;
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
// Waves a SIMD whose registers the compiler may use, for tiles of 16 nb rows.
constexpr int chunk_waves(int D, bool fp16, int nb) { return D == 256 || (fp16 && D == 128 && nb == 2) ? 1 : 2; }

// One wave per (item, kv head): 16 NB rows; a page's operands come straight from its
// record, one 16-byte load a lane for each KiB.
template <int G, bool kFp16, int NB>
__global__ void __launch_bounds__(64, chunk_waves(64 * G, kFp16, NB)) k_chunk_rows(PagedChunk a, ChunkCut cut) {
  constexpr int D = 64 * G, kRows = 16 * NB;
  const int lane = threadIdx.x, n = lane & 15, k = lane >> 4;
  const int head = blockIdx.x % a.c.hkv, group = a.hq / a.c.hkv;
  Item it;
  int joins;
  const bool there = find_item(a, group, cut, blockIdx.x / a.c.hkv, lane, it, joins);
  const ChunkWs ws = chunk_ws(a.ws, a.c, cut);
  if (blockIdx.x == 0 && lane == 0) *ws.joins = joins;
  if (!there) return;
  if (it.runs > 1 && it.run == 0 && head == 0 && lane == 0) ws.split[it.join] = Split{it.b, it.tile, it.slot, it.runs};

  Row row[NB];
  Rows16<G> x[NB];
  h8v_t q[NB][2 * G];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    row[i] = row_of(a, it, group, head, it.tile * kRows + 16 * i + n);
    load_query<G, kFp16>(q[i], a, row[i], head, k);
    start(x[i]);
  }
  // keys that every row of the tile sees, and that any of them sees: up to these
  const int first_token = it.tile * kRows / group, last_token = min(it.seq.n - 1, (it.tile * kRows + kRows - 1) / group);
  const int all_see = it.seq.base + first_token, some_see = it.seq.base + last_token;

  Pages pg;
  load_pages(pg, a.c, it.b, it.begin, it.end - 1, lane);
  for (int j = it.begin; j < it.end; ++j) {
    if (j - pg.base >= 64) load_pages(pg, a.c, it.b, j, it.end - 1, lane);
    const int page = __builtin_amdgcn_readlane(pg.mine, j - pg.base);
    if ((unsigned)page >= (unsigned)a.c.num_pages) continue;
    const uint8_t* rec = a.c.pool + ((size_t)page * a.c.hkv + head) * paged_record_bytes(D, kFp16);
    const bool masked = j * kPage + kPage - 1 > all_see;
    f4v_t s[NB][4];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int t = 0; t < 4; ++t) s[i][t] = f4v_t{0.0f, 0.0f, 0.0f, 0.0f};
    h8v_t p[NB][2];
    if constexpr (kFp16) {
      h8v_t kr[8 * G], vr[8 * G];       // K [t][D/32], V [D/16][c]
      load_operands<8 * G, 1024>(kr, rec, lane);
#pragma unroll
      for (int c = 0; c < 2 * G; ++c)
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < NB; ++i) s[i][t] = product(kr[2 * G * t + c], q[i][c], s[i][t]);
      keep_order();
      load_operands<8 * G, 1024>(vr, rec + 128 * D, lane);
      keep_order();
#pragma unroll
      for (int i = 0; i < NB; ++i) soften<G, kFp16>(x[i], s[i], p[i], a.scale, masked, row[i].limit - j * kPage, k);
      if (masked) {
        bool odd_values = false;
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (j * kPage + 16 * k + 8 * c + i > some_see)
#pragma unroll
              for (int u = 0; u < 4 * G; ++u) vr[2 * u + c][i] = (half_t)0;
#pragma unroll
        for (int u = 0; u < 8 * G; ++u) odd_values |= any_not_finite(vr[u]);
        if (__builtin_amdgcn_ballot_w64(odd_values)) {
#pragma unroll
          for (int u = 0; u < 4 * G; ++u) {
            const h8v_t v[2] = {vr[2 * u], vr[2 * u + 1]};
#pragma unroll
            for (int i = 0; i < NB; ++i) add_not_finite<G>(x[i], v, u, row[i].limit - j * kPage, k);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int i = 0; i < 8; ++i)
                if (!(v[c][i] < (half_t)INFINITY && v[c][i] > -(half_t)INFINITY)) vr[2 * u + c][i] = (half_t)0;
          }
        }
      }
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int u = 0; u < 4 * G; ++u)
#pragma unroll
          for (int i = 0; i < NB; ++i) x[i].o[u] = product(vr[2 * u + c], p[i][c], x[i].o[u]);
    } else {
      HifPart<G> kp, vp;
      load_hif4<G>(kp, rec, lane);
#pragma unroll
      for (int c = 0; c < 2 * G; ++c)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const h8v_t kr = part_operand<G>(kp, c >> 1, t, c & 1, lane);
#pragma unroll
          for (int i = 0; i < NB; ++i) s[i][t] = product(kr, q[i][c], s[i][t]);
        }
      keep_order();
      load_hif4<G>(vp, rec + 2304 * G, lane);
      keep_order();
#pragma unroll
      for (int i = 0; i < NB; ++i) soften<G, kFp16>(x[i], s[i], p[i], a.scale, masked, row[i].limit - j * kPage, k);
#pragma unroll
      for (int u = 0; u < 4 * G; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const h8v_t vr = part_operand<G>(vp, u >> 2, u & 3, c, lane);
#pragma unroll
          for (int i = 0; i < NB; ++i) x[i].o[u] = product(vr, p[i][c], x[i].o[u]);
        }
    }
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c) x[i].sum = product(ones(), p[i][c], x[i].sum);
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) finish<G>(a, ws, it, x[i], row[i], head, kRows, 16 * i + n, k);
}

// ---------------------------------------------------------------------------
// Many rows: kWaves waves of 32 rows each share a page, whose operands they make in
// LDS (two pages' room: the next one is made while this one is used).  A record's KiB
// unit of fp16 operands is what a wave reads for one operand of a product, 16 bytes a
// lane in lane order, so neither reads nor writes have bank conflicts.
// Units of a page: K [t][c], then V [channels / 16][c].
constexpr int kWideRows = 32;           // of a wave
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

// What a wave fetches of a page, and puts into LDS.
template <int G, bool kFp16, int kWaves>
struct WideShare {
  static constexpr int kAll = kFp16 ? 16 * G : 4 * G, kMine = (kAll + kWaves - 1) / kWaves;
  h8v_t unit[kFp16 ? kMine : 1];
  HifQuad quad[kFp16 ? 1 : kMine];
  __device__ __forceinline__ void load(const uint8_t* rec, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int at = wave + kWaves * i;
      if (kAll % kWaves && at >= kAll) break;
      if constexpr (kFp16)
        unit[i] = load_at<h8v_t>((global_ptr)(rec + 1024 * at), 16 * lane);
      else
        load_quad<G>(quad[i], rec, at, lane);
    }
  }
  __device__ __forceinline__ void store(h8v_t* page, int wave, int lane) const {
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int at = wave + kWaves * i;
      if (kAll % kWaves && at >= kAll) break;
      if constexpr (kFp16)
        page[64 * at + lane] = unit[i];
      else
        store_quad<G>(page, quad[i], at, lane);
    }
  }
};

template <int G, bool kFp16, int kWaves>
__global__ void __launch_bounds__(64 * kWaves, G == 4 ? 1 : 2) k_chunk_wide(PagedChunk a, ChunkCut cut) {
  constexpr int D = 64 * G, kRows = kWideRows * kWaves, NB = 2, kUnits = 16 * G;
  extern __shared__ __align__(16) uint8_t smem[];
  h8v_t* const pages = reinterpret_cast<h8v_t*>(smem);
  const int lane = threadIdx.x & 63, n = lane & 15, k = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int head = blockIdx.x % a.c.hkv, group = a.hq / a.c.hkv;
  Item it;
  int joins;
  const bool there = find_item(a, group, cut, blockIdx.x / a.c.hkv, lane, it, joins);
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
  WideShare<G, kFp16, kWaves> share;
  int j = next(it.begin);
  if (j < it.end) share.load(record(), wave, lane);

  const int row0 = it.tile * kRows + wave * kWideRows;      // the wave's first row
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
  const int first_token = row0 / group, last_token = min(it.seq.n - 1, (row0 + kWideRows - 1) / group);
  const int all_see = it.seq.base + first_token, some_see = first_token < it.seq.n ? it.seq.base + last_token : -1;

  const bool late = false;
  int ahead = next(j + 1), at = 0;
  if (j < it.end) share.store(pages, wave, lane);
  if (ahead < it.end) share.load(record(), wave, lane);
  __syncthreads();
  while (j < it.end) {
    const h8v_t* page = pages + 64 * kUnits * at + lane;
    const int now = j;
    j = ahead;
    const auto make_next = [&] {
      if (j < it.end) {
        share.store(pages + 64 * kUnits * (at ^ 1), wave, lane);
        ahead = next(j + 1);
        if (ahead < it.end) share.load(record(), wave, lane);
      }
    };
    if (!late) make_next();
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
          h8v_t v[2] = {page[64 * (8 * G + 2 * u)], page[64 * (8 * G + 2 * u + 1)]};
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (now * kPage + 16 * k + 8 * c + e > some_see) v[c][e] = (half_t)0;
          if (__builtin_amdgcn_ballot_w64(any_not_finite(v[0]) || any_not_finite(v[1]))) {
#pragma unroll
            for (int i = 0; i < NB; ++i) add_not_finite<G>(x[i], v, u, row[i].limit - now * kPage, k);
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (!(v[c][e] < (half_t)INFINITY && v[c][e] > -(half_t)INFINITY)) v[c][e] = (half_t)0;
          }
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < NB; ++i) x[i].o[u] = product(v[c], p[i][c], x[i].o[u]);
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
    if (late) make_next();
    at ^= 1;
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < NB; ++i) finish<G>(a, ws, it, x[i], row[i], head, kRows, wave * kWideRows + 16 * i + n, k);
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
__global__ void __launch_bounds__(kChunkJoin) k_chunk_join(PagedChunk a, ChunkCut cut) {
  constexpr int D = 64 * G, kCols = kFew ? 8 : D / 4, kSets = (kFew ? kChunkJoin : 64) / kCols, kAhead = 4;
  __shared__ Joined part[kFew ? kChunkJoin : 1];
  const int lane = threadIdx.x & 63, at_set = kFew ? threadIdx.x : lane, col = at_set % kCols, set = at_set / kCols;
  const ChunkWs ws = chunk_ws(a.ws, a.c, cut);
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

// Waves of a workgroup that share a page.
constexpr int wide_waves(int D, bool fp16) { return D == 128 ? 8 : 4; }

static bool chunk_cut(const PagedCache& c, int hq, int total, int max_new, ChunkCut* cut) {
  const size_t group = hq / c.hkv;
  const size_t most = max_new * group;
  cut->rows = most <= 16 ? 16 : most <= 32 ? (c.D == 256 ? 16 : 32) : kWideRows * wide_waves(c.D, c.fp16);
  if (cut->rows <= 32)
    cut->target = std::max(1, 1024 * chunk_waves(c.D, c.fp16, cut->rows / 16) / c.hkv);
  else
    cut->target = std::max(1, 1024 * (c.D == 256 ? 1 : 2) / wide_waves(c.D, c.fp16) / c.hkv);
  const size_t tiles = std::min((size_t)c.batch * ((max_new * group + cut->rows - 1) / cut->rows),
                                (size_t)total * group / cut->rows + c.batch);
  const size_t runs = std::max<size_t>(1, ((size_t)c.max_pages + kMinRun - 1) / kMinRun);
  const size_t items = std::min(tiles * runs, tiles + cut->target + 1);
  const size_t joins = runs == 1 ? 0 : std::min(tiles, (size_t)cut->target + 1);
  if (items * c.hkv >= kMaxGrid || joins * c.hkv * cut->rows >= kMaxGrid) return false;
  cut->items = (int)items;
  cut->joins = (int)joins;
  cut->slots = runs == 1 ? 0 : (int)std::min(tiles * runs, (size_t)2 * cut->target + 2);
  return true;
}

bool paged_chunk_fits(const PagedCache& c, int hq, int total, int max_new) {
  ChunkCut cut;
  return chunk_cut(c, hq, total, max_new, &cut);
}
size_t paged_chunk_workspace(const PagedCache& c, int hq, int total, int max_new) {
  ChunkCut cut;
  return chunk_cut(c, hq, total, max_new, &cut) ? chunk_ws_bytes(c, cut) : 0;
}

template <int G, bool kFp16>
static hipError_t launch_rows(const PagedChunk& a, const ChunkCut& cut, hipStream_t st) {
  const dim3 grid((unsigned)((size_t)cut.items * a.c.hkv));
  if (cut.rows > 32) {
    constexpr int kWaves = wide_waves(64 * G, kFp16);
    constexpr size_t kLds = (size_t)2 * 16 * G * 1024;
    if (kLds > 65536) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_chunk_wide<G, kFp16, kWaves>),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds);
      if (e != hipSuccess) return e;
    }
    k_chunk_wide<G, kFp16, kWaves><<<grid, 64 * kWaves, kLds, st>>>(a, cut);
  } else if (G == 4 || cut.rows == 16)
    k_chunk_rows<G, kFp16, 1><<<grid, 64, 0, st>>>(a, cut);
  else
    k_chunk_rows<G == 4 ? 1 : G, kFp16, 2><<<grid, 64, 0, st>>>(a, cut);
  return hipGetLastError();
}

template <int G>
static void launch_join(const PagedChunk& a, const ChunkCut& cut, hipStream_t st) {
  const size_t rows = (size_t)cut.joins * a.c.hkv * cut.rows;
  if (rows <= 2048)
    k_chunk_join<G, true><<<dim3((unsigned)(rows * (2 * G))), kChunkJoin, 0, st>>>(a, cut);
  else
    k_chunk_join<G, false><<<dim3((unsigned)std::min<size_t>(2048, rows / 4)), kChunkJoin, 0, st>>>(a, cut);
}

hipError_t launch_paged_chunk(const PagedChunk& a, hipStream_t st) {
  ChunkCut cut;
  if (!chunk_cut(a.c, a.hq, a.total, a.max_new, &cut)) return hipErrorInvalidValue;
  hipError_t e;
  if (a.c.fp16)
    e = a.c.D == 64 ? launch_rows<1, true>(a, cut, st) : a.c.D == 128 ? launch_rows<2, true>(a, cut, st) : launch_rows<4, true>(a, cut, st);
  else
    e = a.c.D == 64 ? launch_rows<1, false>(a, cut, st) : a.c.D == 128 ? launch_rows<2, false>(a, cut, st) : launch_rows<4, false>(a, cut, st);
  if (e != hipSuccess || !cut.joins) return e;
  if (a.c.D == 64)
    launch_join<1>(a, cut, st);
  else if (a.c.D == 128)
    launch_join<2>(a, cut, st);
  else
    launch_join<4>(a, cut, st);
  return hipGetLastError();
}

}  // namespace hifa4
