// One new token's attention over the paged cache (records: hifa4_paged.h).
//
// For query row h of sequence b over its L cached tokens:
//   S_j = (q~ . k_j) / sqrt(D),  p_j = exp(S_j - m) / l,  o = sum_j p_j v_j,
//   LSE = m + ln l,  with m = max S_j and l = sum_j exp(S_j - m);
//   page weights w'[page] = decay w[page] + sum over the heads and the page's
//   tokens of p_j.
// q~ = fp16(q s) under Smooth-QK (the cache holds k/s); keys and values are
// what the cache holds; scores, m, l, the page weights and o are held in fp32
// and o is rounded once to fp16.  In the products p has 22 bits (FP16 pages) or,
// like q~, 19 under the largest of its 64 (HIF4 pages): the operands that the
// matrix instructions take, in two and four pieces.
//
// The pages of all sequences are cut into runs of about equal length, as many
// as fill the chip: a run leaves (m, l, o) of its rows, and a second kernel
// joins the runs of a row.  Lengths are read on the device, so a captured call
// follows them.
#include "hifa4_device.h"
#include "hifa4_packed.h"
#include "hifa4_paged.h"
#include "hifa4_paged_device.h"
#include "hifa4_words.h"

#include <algorithm>

namespace hifa4 {

typedef int i8v_t __attribute__((ext_vector_type(8)));
typedef short s2v_t __attribute__((ext_vector_type(2)));

// Query heads that a wave takes: the 16 columns of a matrix product, four for
// each query on HIF4 pages.
__host__ __device__ __forceinline__ int query_tiles(int hq, int hkv, bool fp16) {
  const int per = fp16 ? 16 : 4;
  return (hq / hkv + per - 1) / per;
}
// How the pages are cut: into as many runs as give every SIMD the waves that
// its registers hold (a page's K and V and, on their way, the next one's).
// More runs than that wait for a place and are short: 8 x 32768 tokens, HIF4,
// D=128, 63.7 us with two waves' runs a SIMD, 71, 73 and 77 with 3, 4 and 6;
// fewer registers a wave for three waves spill (81).  At D=256 one wave: 4 x 16384
// tokens, 16 query heads, 37.7 us, for which two, with spills, take 47.0.  Every
// sequence is cut into equal parts of at most ceil(units / target), numbered
// densely over the sequences: at most target + batch runs.
__host__ __device__ __forceinline__ int run_target(int hq, int hkv, int D, bool fp16) {
  const int waves = fp16 ? (D == 64 ? 3 : D == 128 ? 2 : 1) : (D == 256 ? 1 : D == 128 ? 2 : 3);
  const int each = hkv * query_tiles(hq, hkv, fp16);
  return (1024 * waves + each - 1) / each;
}
// Units of a page that runs are cut into: FP16 pages of D = 256 (64 KiB a head,
// few a wave) in halves, keys 16k + 8c .. 16k + 8c + 7 in half c: 3 sequences
// of 2000 tokens 19.0 to 16.9 us, 4 of 1000 to 8192 39.9 to 38.9.  At D=128 the
// second half's turn costs more than the balance gives: 13.2 to 14.4 us.
__host__ __device__ constexpr int page_units(int D, bool fp16) { return fp16 && D == 256 ? 2 : 1; }
__host__ __device__ __forceinline__ size_t run_slots(const PagedCache& c, int target) {
  const size_t all = (size_t)c.batch * c.max_pages * page_units(c.D, c.fp16), most = (size_t)target + c.batch;
  return all < most ? all : most;
}
struct Run {
  int b, begin, end;              // units [begin, end) of sequence b; b < 0: no such run
  int first, count;               // the sequence's runs: [first, first + count)
};

// The sequences are dealt to the lanes of a wave (b, b + 64, ...), the units of
// a lane's first kHeldSeqs in registers.
constexpr int kHeldSeqs = 4;
struct Dealt {
  int n[kHeldSeqs];
};
// Sum of f(units) over the sequences of each lane.
template <int kUnits, typename F>
__device__ __forceinline__ int lane_sum(const PagedCache& c, const Dealt& d, int lane, F f) {
  int sum = f(d.n[0]);
#pragma unroll
  for (int i = 1; i < kHeldSeqs; ++i)
    if (c.batch > 64 * i) sum += f(d.n[i]);
  for (int b = 64 * kHeldSeqs + lane; b < c.batch; b += 64) sum += f(kUnits * pages_of(c, b));
  return sum;
}
// The run numbered r (found by a whole wave).  Runs are numbered lane by lane of the above.
template <int kUnits>
__device__ __forceinline__ Run find_run(const PagedCache& c, int target, int r, int lane) {
  Dealt d;
#pragma unroll
  for (int i = 0; i < kHeldSeqs; ++i) d.n[i] = kUnits * pages_of(c, 64 * i + lane);
  int mine = lane_sum<kUnits>(c, d, lane, [](int n) { return n; }), upto = wave_scan(mine), per = 1;
  const int total = __builtin_amdgcn_readlane(upto, 63);
  if (total > target) {
    per = (total + target - 1) / target;
    // the last runs of the sequences are shorter: longer runs until all fit into one round (or nearly)
    for (int i = 0;; ++i) {
      mine = lane_sum<kUnits>(c, d, lane, [per](int n) { return (n + per - 1) / per; });
      upto = wave_scan(mine);
      const int runs = __builtin_amdgcn_readlane(upto, 63);
      if (runs <= target || i == 6 || c.batch >= target) break;
      per += max(1, (int)((long)per * (runs - target) / target));
    }
  }
  Run out = {-1, 0, 0, 0, 0};
  const unsigned long long who = __builtin_amdgcn_ballot_w64(r < upto);
  if (!who) return out;
  const int src = __builtin_ctzll(who);
  out.first = __builtin_amdgcn_readlane(upto - mine, src);
  for (int b = src, i = 0; b < c.batch; b += 64, ++i) {
    const int n = i == 0   ? __builtin_amdgcn_readlane(d.n[0], src)
                  : i == 1 ? __builtin_amdgcn_readlane(d.n[1], src)
                  : i == 2 ? __builtin_amdgcn_readlane(d.n[2], src)
                  : i == 3 ? __builtin_amdgcn_readlane(d.n[3], src)
                           : __builtin_amdgcn_readfirstlane(kUnits * pages_of(c, b));
    out.count = (n + per - 1) / per;
    if (r < out.first + out.count) {
      const int k = r - out.first, some = n / out.count, more = n % out.count;
      out.b = b;                       // the first runs get one unit more where the count does not divide
      out.begin = k * some + min(k, more);
      out.end = out.begin + some + (k < more);
      return out;
    }
    out.first += out.count;
  }
  return out;
}

// Workspace: o [slots][hq][D], then (m, l) [slots][hq], the runs (first, count)
// of each sequence that has any, then with page weights (m, sum)
// [batch][max_pages * units][hq]; m in log2 units.
struct DecodeWs {
  float* o;
  float2* ml;
  int2* runs;
  float2* page;
};
__host__ __device__ __forceinline__ DecodeWs decode_ws(uint8_t* ws, const PagedCache& c, int target, int hq) {
  const size_t slots = run_slots(c, target);
  DecodeWs w;
  w.o = reinterpret_cast<float*>(ws);
  w.ml = reinterpret_cast<float2*>(w.o + slots * hq * c.D);
  w.runs = reinterpret_cast<int2*>(w.ml + slots * hq);
  w.page = reinterpret_cast<float2*>(w.runs + c.batch);
  return w;
}
size_t paged_decode_workspace(const PagedCache& c, int hq, bool weights) {
  const size_t slots = run_slots(c, run_target(hq, c.hkv, c.D, c.fp16));
  return slots * hq * (c.D + 2) * 4 + (size_t)c.batch * 8 + (weights ? (size_t)c.batch * c.max_pages * page_units(c.D, c.fp16) * hq * 8 : 0);
}

// ---------------------------------------------------------------------------
// HIF4 pages.  One wave per (run, kv head, four query heads).
//
// A cache word of eight codes is a matrix operand as it stands: a magnitude u
// is (u & 3) + (u & 4), both parts are FP4 codes (of half their value) under
// the code's own sign bit, so two masks make two registers of it, and two more
// with the half-words of E3 = 1 cleared make their sum u 2^-E3.  E2 is the
// lane's E8M0 scale; the bases multiply the products in fp32.
// The other operand has 8 bits.  The instruction adds the products of sixteen
// neighbouring slots on one grid, 13 binades below the largest (measured: 2^1
// is lost beside 2^15 - 2^15, 2^2 is not), so operands of few bits and one
// scale are the ones whose sums are exact: a value is written in base 32 with
// digits -16 .. 16, whole numbers that FP8 (E4M3) holds, relative to the
// largest of its 64; four digits (19 bits below that largest value), each in a
// column of its own with the scale 32^-k.  Products are multiples of 1/2 up to
// 32: every digit's sum over a group is exact.  So a product of 16 columns is
// four queries, and four neighbouring lanes add up to the score in fp32.  The
// weights p of a page are cut the same way, relative to the page's largest:
// light pages keep their bits, and a key that is light beside another of its
// page is rounded by up to 2^-19 of that one's weight (half a step of 2^-15
// where the largest lies between 8 and 16).
//
// Slots of v_mfma_scale_f32_16x16x128_f8f6f4 (measured): FP4 operand lane
// 16k + n holds K 32k .. 32k+31, its four registers in order; FP8 operand lane
// 16k + n holds K 16k .. 16k+15 in its first four registers and 64 + 16k .. in
// the others.  So FP8 lanes k = 2j, 2j+1 meet FP4 lanes j and 2 + j: they hold
// the words of both, each twice.  V is read with its lanes k = 1 and 2
// exchanged, which makes the words of FP4 lanes j and 2 + j the keys whose
// scores lanes 2j and 2j + 1 have: one exchange between neighbouring rows of
// 16 lanes brings p into place.
//
// Bound by the reads of the pages: 8 x 32768 tokens, 8 kv heads, D=128 (302
// MB) in 60 us, 5.1 TB/s, where a plain read of as much reaches 5.6.  Mixed
// lengths (32 of 300 to 8192, 165 MB) take 39 us, 4.2 TB/s: about 3 us until
// the first page is there, and 10% for runs of unequal length.
constexpr int kFp4 = 4, kFp8 = 0;            // operand formats of the instruction
// The reference of the softmax is a whole power of two and moves only when a
// page's largest score passes it by this many binades: fp32 sums do not mind.
constexpr float kSlack = 16.0f;
// Row of p's digits in LDS, padded so that the four rows of lanes write to different banks.
constexpr int kDigitRow = 68;
// E8M0 byte of the FP4 side without E2: 2^(94 - E2).  The bases enter as the
// float whose bits are byte << 21 = b 2^-96, and an operand's sum is 4 values.
constexpr uint32_t kUnit = 127 + 94;

// over the four pieces of a query (the same bits in each of the four lanes)
__device__ __forceinline__ float sum_pieces(float v) {
  v += __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0xB1, 0xF, 0xF, true));
  return v + __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x4E, 0xF, 0xF, true));
}

__device__ __forceinline__ float max_quad(float v) {
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0xB1, 0xF, 0xF, true)));
  return fmaxf(v, __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x4E, 0xF, 0xF, true)));
}
// mine + the neighbour's other (quad permutation kPerm)
template <int kPerm>
__device__ __forceinline__ float add_xor(float mine, float other) {
  return mine + __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(other), kPerm, 0xF, 0xF, true));
}

// The digits of x (|x| <= 16): R_k = rint(32^k x), digit k = R_k - 32 R_(k-1),
// between -16 and 16; they add up to R_3 / 32^3.
__device__ __forceinline__ void digits(float x, float (&d)[4]) {
  const float r0 = __builtin_rintf(x), r1 = __builtin_rintf(x * 32.0f), r2 = __builtin_rintf(x * 1024.0f),
              r3 = __builtin_rintf(x * 32768.0f);
  d[0] = r0;
  d[1] = fmaf(-32.0f, r0, r1);
  d[2] = fmaf(-32.0f, r1, r2);
  d[3] = fmaf(-32.0f, r2, r3);
}
__device__ __forceinline__ uint32_t fp8x4(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

// K's or V's part of a record in a lane's registers.
template <int G>
struct Part {
  uint4 code[2 * G];       // [tile][t/2]: (t even: words 0, 1), (t odd: words 0, 1)
  uint32_t e3[(G + 1) / 2];
  uint32_t e2;
  uint32_t base;           // G bytes of the 64 G, in the record's order
};
template <int G>
__device__ __forceinline__ void load_part(Part<G>& p, const uint8_t* part, uint32_t lane, uint32_t base_lane) {
  typedef unsigned u4v_t __attribute__((ext_vector_type(4)));
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
    typedef unsigned u2v_t __attribute__((ext_vector_type(2)));
    const u2v_t x = load_at<u2v_t>(meta, 8 * lane);
    p.e3[0] = x[0];
    p.e3[G == 4 ? 1 : 0] = x[1];
    p.e2 = load_at<uint32_t>(meta, 4 * lane + 512);
  }
  if (G == 1)
    p.base = load_at<uint8_t>(meta, base_lane + 192);
  else if (G == 2)
    p.base = load_at<uint16_t>(meta, 2 * base_lane + 384);
  else
    p.base = load_at<uint32_t>(meta, 4 * base_lane + 768);
}

// 0xFFFF in each half-word of word (t, c) of `tile` with E3 = 0; x: the
// complement of its E3 bits, one half of the word in each 16 bits.
template <int G>
__device__ __forceinline__ uint32_t e3_keep(uint32_t x, int tile, int t, int c) {
  const int bit = 8 * (tile & 1) + 2 * t + c;
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(s2v_t, x << (15 - bit)) >> (short)15);
}
// E8M0 bytes of a tile's words (t, c), t = 0..3 in bytes 0..3.
__device__ __forceinline__ uint32_t e2_scales(uint32_t e2, int tile, int c) {
  const uint32_t bits = (e2 >> (8 * tile + c)) & 0x55u;
  return kUnit * 0x01010101u - (__umul24(bits, 0x41041u) & 0x01010101u);
}
template <int T>
__device__ __forceinline__ f4v_t mfma_word(uint32_t w, uint32_t keep, uint32_t scale, const i8v_t& b, uint32_t b_scale,
                                           f4v_t c) {
  const uint32_t lo = w & 0xBBBBBBBBu, hi = w & 0xCCCCCCCCu;
  const i8v_t a = {(int)lo, (int)hi, (int)(lo & keep), (int)(hi & keep), 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, kFp4, kFp8, T, (int)scale, 0, (int)b_scale);
}
template <int G>
__device__ __forceinline__ uint32_t e3_halves(const Part<G>& p, int tile) {
  const uint32_t x = ~p.e3[tile / 2];
  return G == 1 ? (x & 0xFFu) | ((x & 0xFF00u) << 8) : x;
}
// Between a wave's accesses of LDS that hand data from lane to lane: the hardware
// keeps their order, the compiler would only where one lane's meet.
__device__ __forceinline__ void lds_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local"); }
// A lane's bases to LDS as floats (b 2^-96), for the lanes that hold their rows' products.
template <int G>
__device__ __forceinline__ void spread_bases(float* to, uint32_t base, int lane) {
#pragma unroll
  for (int i = 0; i < G; ++i) to[G * lane + i] = __uint_as_float((base >> (8 * i) & 0xFFu) << 21);
}
// use(tile, t, products, bases): products of a tile's rows 16 t + 4k + v with
// the columns of the other operand, which get(tile, b0, b1, scale) fetches
// (its two words' parts).  `spread`: 64 G floats of LDS for the bases.
template <int G, typename Get, typename Use>
__device__ __forceinline__ void products(const Part<G>& p, float* spread, int lane, Get get, Use use) {
  spread_bases<G>(spread, p.base, lane);
  lds_order();
#pragma unroll
  for (int tile = 0; tile < G; ++tile) {
    const uint32_t x = e3_halves<G>(p, tile), s0 = e2_scales(p.e2, tile, 0), s1 = e2_scales(p.e2, tile, 1);
    i8v_t b0, b1;
    uint32_t scale;
    get(tile, b0, b1, scale);
    const uint4 w0 = p.code[2 * tile], w1 = p.code[2 * tile + 1];
    const f4v_t z = {0.0f, 0.0f, 0.0f, 0.0f};
    // four chains of two, side by side
    f4v_t c0 = mfma_word<0>(w0.x, e3_keep<G>(x, tile, 0, 0), s0, b0, scale, z);
    f4v_t c1 = mfma_word<1>(w0.z, e3_keep<G>(x, tile, 1, 0), s0, b0, scale, z);
    f4v_t c2 = mfma_word<2>(w1.x, e3_keep<G>(x, tile, 2, 0), s0, b0, scale, z);
    f4v_t c3 = mfma_word<3>(w1.z, e3_keep<G>(x, tile, 3, 0), s0, b0, scale, z);
    c0 = mfma_word<0>(w0.y, e3_keep<G>(x, tile, 0, 1), s1, b1, scale, c0);
    c1 = mfma_word<1>(w0.w, e3_keep<G>(x, tile, 1, 1), s1, b1, scale, c1);
    c2 = mfma_word<2>(w1.y, e3_keep<G>(x, tile, 2, 1), s1, b1, scale, c2);
    c3 = mfma_word<3>(w1.w, e3_keep<G>(x, tile, 3, 1), s1, b1, scale, c3);
    const f4v_t* b = reinterpret_cast<const f4v_t*>(spread + 16 * G * (lane >> 4) + 16 * tile);
    use(tile, 0, c0, b[0]);
    use(tile, 1, c1, b[1]);
    use(tile, 2, c2, b[2]);
    use(tile, 3, c3, b[3]);
  }
}
// The FP8 operand of two words, each twice (x: the FP4 lane j's, y: lane 2 + j's).
__device__ __forceinline__ i8v_t fp8_operand(uint4 x, uint4 y) {
  return i8v_t{(int)x.x, (int)x.y, (int)x.z, (int)x.w, (int)y.x, (int)y.y, (int)y.z, (int)y.w};
}

// The digits of four query heads' rows (q: the first of them, `rows` exist) in
// LDS: [channel group][c][FP4 lane][column 4 query + digit][8 channels]; and
// the exponent that each group of 64 was scaled by.
template <int G>
struct QueryDigits {
  uint4 word[G][2][4][16];             // a word's eight bytes, twice
  int exponent[G][4];
};
// The rows as they come, eight channels of a row per lane and step (they are
// fetched before the first page's loads, so that only they are waited for).
template <int G>
struct QueryRows {
  uint4 q[(G + 1) / 2];
  f4v_t s[(G + 1) / 2][2];
};
template <int G>
__device__ __forceinline__ void load_query(QueryRows<G>& in, const half_t* q, int rows, const float* s, int lane) {
#pragma unroll
  for (int k = 0; k < (G + 1) / 2; ++k) {
    const int i = lane + 64 * k, row = i / (8 * G), at = 8 * (i % (8 * G));
    in.q[k] = make_uint4(0, 0, 0, 0);
    if (row < min(rows, 4)) in.q[k] = *reinterpret_cast<const uint4*>(q + (size_t)row * 64 * G + at);
    if (s) {
      in.s[k][0] = *reinterpret_cast<const f4v_t*>(s + at);
      in.s[k][1] = *reinterpret_cast<const f4v_t*>(s + at + 4);
    }
  }
}
template <int G>
__device__ __forceinline__ void query_digits(QueryDigits<G>& out, const QueryRows<G>& in, bool smooth, int lane) {
#pragma unroll
  for (int step = 0; step < (G + 1) / 2; ++step) {
    const int i = lane + 64 * step, row = i / (8 * G), g = i / 8 % G, w = i & 7;
    if (row >= 4) break;               // (half of the lanes with one group)
    const uint4 q = in.q[step];
    const h2_t y[4] = {__builtin_bit_cast(h2_t, q.x), __builtin_bit_cast(h2_t, q.y), __builtin_bit_cast(h2_t, q.z),
                       __builtin_bit_cast(h2_t, q.w)};
    float x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const half_t z = y[u >> 1][u & 1];
      x[u] = smooth ? (float)round_product(z, in.s[step][u >> 2][u & 3]) : (float)z;
    }
    float top = 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) top = fmaxf(top, fabsf(x[u]));
    top = __uint_as_float(reduce8(__float_as_uint(top), [](uint32_t a, uint32_t b) {
      return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }));
    // 2^e <= top < 2^(e+1): 2^(3-e) x lies below 16
    const int e = top > 0.0f ? (int)(__float_as_uint(top) >> 23) - 127 : 0;
    const float up = __uint_as_float((uint32_t)(127 + 3 - e) << 23);
    if (w == 0) out.exponent[g][row] = e;
    float d[8][4];
#pragma unroll
    for (int u = 0; u < 8; ++u) digits(x[u] * up, d[u]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t d0 = fp8x4(d[0][k], d[1][k], d[2][k], d[3][k]), d1 = fp8x4(d[4][k], d[5][k], d[6][k], d[7][k]);
      out.word[g][w & 1][w >> 1][4 * row + k] = make_uint4(d0, d1, d0, d1);
    }
  }
}

template <int G>
__global__ void __launch_bounds__(64, G == 4 ? 1 : G == 2 ? 2 : 3) k_runs_hif4(PagedDecode a, int tiles) {
  constexpr int D = 64 * G;
  __shared__ QueryDigits<G> qd;
  __shared__ __align__(16) uint32_t pd[4][kDigitRow];      // [k][query][digit][t]: four keys' digits of p
  __shared__ __align__(16) float spread_k[64 * G], spread_v[64 * G];
  const int lane = threadIdx.x, n = lane & 15, k = lane >> 4, piece = n & 3;
  const int head = blockIdx.x % a.c.hkv, group = a.hq / a.c.hkv;
  const int tile = blockIdx.x / a.c.hkv % tiles, r = blockIdx.x / a.c.hkv / tiles;
  const int target = run_target(a.hq, a.c.hkv, D, false);
  const Run run = find_run<page_units(D, false)>(a.c, target, r, lane);
  if (run.b < 0) return;
  const int len = __builtin_amdgcn_readfirstlane(paged_len(a.c, run.b));
  const DecodeWs ws = decode_ws(a.ws, a.c, target, a.hq);
  if (r == run.first && head == 0 && tile == 0 && lane == 0) ws.runs[run.b] = make_int2(run.first, run.count);
  const size_t rec_bytes = (size_t)72 * D;
  const int v_lane = 16 * ((k & 1) * 2 + (k >> 1)) + n;        // lanes k = 1, 2 exchanged
  const int q_in = 4 * tile + (n >> 2), h = head * group + q_in;

  Pages pg;
  load_pages(pg, a.c, run.b, run.begin, run.end - 1, lane);
  bool has, has_next = false;
  // The record of page j; of a page that is none the pool's first, whose keys are all masked then.
  const auto record = [&](int j, bool& there) -> const uint8_t* {
    if (j - pg.base >= 64) {
      load_pages(pg, a.c, run.b, j, run.end - 1, lane);
      asm volatile("" : "+v"(pg.mine));  // waited for here: else every page's look-up would wait for all loads
    }
    const int page = __builtin_amdgcn_readlane(pg.mine, j - pg.base);
    there = (unsigned)page < (unsigned)a.c.num_pages;
    return a.c.pool + ((size_t)(there ? page : 0) * a.c.hkv + head) * rec_bytes;
  };
  QueryRows<G> rows;
  load_query<G>(rows, a.q + ((size_t)run.b * a.hq + head * group + 4 * tile) * D, group - 4 * tile,
                a.s ? a.s + (size_t)head * D : nullptr, lane);
  keep_order();
  Part<G> kp[2], vp[2];
  const uint8_t* rec = record(run.begin, has);
  load_part<G>(kp[0], rec, lane, lane);
  keep_order();
  load_part<G>(vp[0], rec + 2304 * G, v_lane, lane);
  keep_order();
  query_digits<G>(qd, rows, a.s != nullptr, lane);
  __syncthreads();
  uint32_t q_scale[G];
#pragma unroll
  for (int g = 0; g < G; ++g) q_scale[g] = (uint32_t)(127 - 3 - 5 * piece + qd.exponent[g][n >> 2]);

  // sums are of p = 2^(score - ref), ref a whole number
  const bool odd = piece & 1, high = piece & 2;
  float ref = -1e30f, l = 0.0f;
  f4v_t o[G][4];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int t = 0; t < 4; ++t) o[g][t] = f4v_t{0.0f, 0.0f, 0.0f, 0.0f};

  // One page from kc and vc, while the next one's parts are loaded into kn and
  // vn (the last page's own again at the end, which nothing waits for).
  const auto page = [&](const Part<G>& kc, const Part<G>& vc, Part<G>& kn, Part<G>& vn, int j) __attribute__((always_inline)) {
    // The waves of a SIMD issue oldest first: one with more of its run left
    // goes before, so that they end together (8 x 32768 tokens: 65.8 to 63.9 us).
    const int some = run.end - run.begin, rem = 4 * (run.end - j);
    if (rem > 3 * some)
      __builtin_amdgcn_s_setprio(3);
    else if (rem > 2 * some)
      __builtin_amdgcn_s_setprio(2);
    else if (rem > some)
      __builtin_amdgcn_s_setprio(1);
    else
      __builtin_amdgcn_s_setprio(0);
    const uint8_t* next = record(min(j + 1, run.end - 1), has_next);
    keep_order();
    load_part<G>(kn, next, lane, lane);
    keep_order();
    f4v_t s[4];
    asm volatile("" ::: "memory");       // the query's operands come from LDS in every page, not from registers
    products<G>(kc, spread_k, lane, [&](int g, i8v_t& b0, i8v_t& b1, uint32_t& scale) {
      const int j2 = k >> 1;
      b0 = fp8_operand(qd.word[g][0][j2][n], qd.word[g][0][2 + j2][n]);
      b1 = fp8_operand(qd.word[g][1][j2][n], qd.word[g][1][2 + j2][n]);
      scale = q_scale[g];
    }, [&](int g, int t, f4v_t d, f4v_t b) {
#pragma unroll
      for (int v = 0; v < 4; ++v) s[t][v] = g == 0 ? d[v] * b[v] : fmaf(d[v], b[v], s[t][v]);
    });
    keep_order();
    load_part<G>(vn, next + 2304 * G, v_lane, lane);
    keep_order();
    // The scores: a lane adds up the digits' products of its share, the four
    // keys 4 piece .. 4 piece + 3 of its 16; log2 units from here on.
    float x[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float a01 = add_xor<0xB1>(odd ? s[1][v] : s[0][v], odd ? s[0][v] : s[1][v]);
      const float a23 = add_xor<0xB1>(odd ? s[3][v] : s[2][v], odd ? s[2][v] : s[3][v]);
      x[v] = add_xor<0x4E>(high ? a23 : a01, high ? a01 : a23) * a.scale;
    }
    const int held = has ? len - j * kPage : 0;
    if (held < kPage) {
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (16 * k + 4 * piece + v >= held) x[v] = -INFINITY;
    }
    const float top = max_across_rows(max_quad(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]))));
    // the page's own reference: the next whole number above its largest score
    // (far below ref, where nothing of the page counts, 100 binades are enough)
    const float own = fmaxf(ceilf(top), ref - 100.0f);
    // 2^low counts 1 in the page's sums; beside numbers over 2^26 it may be own
    // or own - 8 (p, a power of two there, is then at most 1 or 256)
    const float low = own - 4.0f;
    if (__builtin_amdgcn_ballot_w64(own - ref > kSlack)) {
      const float to = fmaxf(ref, own), f = __builtin_amdgcn_exp2f(ref - to);
      ref = to;
      l *= f;
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int t = 0; t < 4; ++t) o[g][t] *= f;
    }
    float sum = 0.0f, d[4][4];
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float p = __builtin_amdgcn_exp2f(x[v] - low);      // 16 p, at most 16
      sum += p;
      digits(p, d[v]);
    }
    // every lane's digits to the lanes that need them: of its query's 16 keys and of the next row's
#pragma unroll
    for (int i = 0; i < 4; ++i) pd[k][16 * (n >> 2) + 4 * i + piece] = fp8x4(d[0][i], d[1][i], d[2][i], d[3][i]);
    lds_order();
    // 2^up: what the page's sums count (ref - 100 may lie 128 below ref)
    const int up = max((int)(low - ref), -104);
    l = fmaf(sum, __uint_as_float((uint32_t)(127 + up) << 23), l);
    const uint32_t p_scale = (uint32_t)(127 + up - 5 * piece);
    if (a.w_in) {
      const float all = sum_across_rows(sum_pieces(sum));
      if (k == 0 && piece == 0 && q_in < group)
        ws.page[((size_t)run.b * a.c.max_pages + j) * a.hq + h] = make_float2(low, all);
    }
    const uint4 pe = *reinterpret_cast<const uint4*>(&pd[k & 2][4 * n]);
    const uint4 po = *reinterpret_cast<const uint4*>(&pd[(k & 2) + 1][4 * n]);
    const i8v_t pa[2] = {fp8_operand(make_uint4(pe.x, pe.y, pe.x, pe.y), make_uint4(po.x, po.y, po.x, po.y)),
                         fp8_operand(make_uint4(pe.z, pe.w, pe.z, pe.w), make_uint4(po.z, po.w, po.z, po.w))};
    products<G>(vc, spread_v, lane, [&](int, i8v_t& b0, i8v_t& b1, uint32_t& scale) {
      b0 = pa[0];
      b1 = pa[1];
      scale = p_scale;
    }, [&](int g, int t, f4v_t d, f4v_t b) {
#pragma unroll
      for (int v = 0; v < 4; ++v) o[g][t][v] = fmaf(d[v], b[v], o[g][t][v]);
    });
    keep_order();
    has = has_next;
  };
  for (int j = run.begin; j < run.end; j += 2) {
    page(kp[0], vp[0], kp[1], vp[1], j);
    if (j + 1 == run.end) break;
    page(kp[1], vp[1], kp[0], vp[0], j + 1);
  }

  l = sum_across_rows(sum_pieces(l));
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) o[g][t][v] = sum_pieces(o[g][t][v]);
  if (q_in >= group) return;
  const size_t slot = (size_t)r * a.hq + h;
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (t == piece) *reinterpret_cast<f4v_t*>(ws.o + slot * D + 64 * g + 16 * t + 4 * k) = o[g][t];
  if (k == 0 && piece == 0) ws.ml[slot] = make_float2(l == 0.0f ? -INFINITY : ref, l);
}

// ---------------------------------------------------------------------------
// FP16 pages.  One wave per (run, kv head, 16 query heads): the record's KiB
// pieces are the operands of v_mfma_f32_16x16x32_f16 as they are loaded, the
// scores of a lane (16 keys of its query) its operand of the second product.
// p enters that product as the sum of two fp16 values (22 bits; one alone
// would round a row that rests on one key by 2^-12 more than its output is
// rounded anyway), scaled so that the heaviest key so far lies between 2^7 and
// 2^15: small weights stay above fp16's subnormals down to 2^-21 of it.  What p
// counts from is held itself, not the score 7 binades above it: of scores over
// 2^24 that difference is no number, and p would pass fp16's range.
// Bound by the reads: D=128, 8 x 8192 tokens (268 MB) in 51 us, 5.2 TB/s.
typedef half_t h4v_t __attribute__((ext_vector_type(4)));
constexpr float kTop16 = 7.0f, kSlack16 = 8.0f;

template <int G>
__global__ void __launch_bounds__(64, G == 1 ? 3 : G == 2 ? 2 : 1) k_runs_fp16(PagedDecode a, int tiles) {
  constexpr int D = 64 * G, kUnits = page_units(D, true), kT = 4 / kUnits, kC = 2 / kUnits;
  const int lane = threadIdx.x, n = lane & 15, k = lane >> 4;
  const int head = blockIdx.x % a.c.hkv, group = a.hq / a.c.hkv;
  const int tile = blockIdx.x / a.c.hkv % tiles, r = blockIdx.x / a.c.hkv / tiles;
  const int target = run_target(a.hq, a.c.hkv, D, true);
  const Run run = find_run<kUnits>(a.c, target, r, lane);
  if (run.b < 0) return;
  const int len = __builtin_amdgcn_readfirstlane(paged_len(a.c, run.b));
  const DecodeWs ws = decode_ws(a.ws, a.c, target, a.hq);
  if (r == run.first && head == 0 && tile == 0 && lane == 0) ws.runs[run.b] = make_int2(run.first, run.count);
  const int q_in = 16 * tile + n, h = head * group + q_in;

  const int last = (run.end - 1) / kUnits;
  Pages pg;
  load_pages(pg, a.c, run.b, run.begin / kUnits, last, lane);
  bool has, has_next = false;
  const auto record = [&](int unit, bool& there) -> const uint8_t* {
    const int j = unit / kUnits;
    if (j - pg.base >= 64) {
      load_pages(pg, a.c, run.b, j, last, lane);
      asm volatile("" : "+v"(pg.mine));  // waited for here: else every page's look-up would wait for all loads
    }
    const int page = __builtin_amdgcn_readlane(pg.mine, j - pg.base);
    there = (unsigned)page < (unsigned)a.c.num_pages;
    return a.c.pool + ((size_t)(there ? page : 0) * a.c.hkv + head) * (size_t)(256 * D);
  };
  h8v_t q[2 * G];
  const float* s = a.s + (size_t)head * D + 8 * k;
#pragma unroll
  for (int c = 0; c < 2 * G; ++c) {
    q[c] = h8v_t{0, 0, 0, 0, 0, 0, 0, 0};
    if (q_in < group) q[c] = *reinterpret_cast<const h8v_t*>(a.q + ((size_t)run.b * a.hq + h) * D + 32 * c + 8 * k);
  }
  if (a.s)
#pragma unroll
    for (int c = 0; c < 2 * G; ++c) {
      const f4v_t s0 = *reinterpret_cast<const f4v_t*>(s + 32 * c), s1 = *reinterpret_cast<const f4v_t*>(s + 32 * c + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) q[c][i] = round_product(q[c][i], i < 4 ? s0[i & 3] : s1[i & 3]);
    }
  h8v_t kr[2 * G * kT], vr[4 * G * kC];    // K [t][D/32], V [D/16][c]
  const uint8_t* rec = record(run.begin, has);
  // a unit's part of a record: half of K's rows, every other KiB of V
  const auto load_k = [&](const uint8_t* from, int j) {
    load_operands<2 * G * kT, 1024>(kr, from + j % kUnits * 64 * D, lane);
  };
  const auto load_v = [&](const uint8_t* from, int j) {
    load_operands<4 * G * kC, 1024 * kUnits>(vr, from + 128 * D + j % kUnits * 1024, lane);
  };
  load_k(rec, run.begin);
  load_v(rec, run.begin);
  float ref = -1e30f, l = 0.0f;            // p = 2^(score - ref), scores in log2 units
  f4v_t o[4 * G];
#pragma unroll
  for (int c = 0; c < 4 * G; ++c) o[c] = f4v_t{0.0f, 0.0f, 0.0f, 0.0f};

  for (int j = run.begin; j < run.end; ++j) {
    f4v_t s[kT];
#pragma unroll
    for (int t = 0; t < kT; ++t) s[t] = f4v_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < 2 * G; ++c)
#pragma unroll
      for (int t = 0; t < kT; ++t) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kr[2 * G * t + c], q[c], s[t], 0, 0, 0);
    const int j2 = min(j + 1, run.end - 1);
    const uint8_t* next = record(j2, has_next);
    load_k(next, j2);
#pragma unroll
    for (int t = 0; t < kT; ++t) s[t] *= a.scale;
    const int held = has ? len - j / kUnits * kPage : 0;
    const int first = 16 * k + 8 * (j % kUnits);     // the lane's first key in the page
    if (held < kPage) {
      asm volatile("");                  // (kept a branch)
#pragma unroll
      for (int t = 0; t < kT; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (first + 4 * t + v >= held) s[t][v] = -INFINITY;
      // what lies in the page behind the last token may be anything: 0 times it has to be 0
#pragma unroll
      for (int c = 0; c < kC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (first + 8 * c + i >= held)
#pragma unroll
            for (int u = 0; u < 4 * G; ++u) vr[kC * u + c][i] = (half_t)0;
    }
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < kT; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) top = fmaxf(top, s[t][v]);
    if (__builtin_amdgcn_ballot_w64(top - ref > kTop16 + kSlack16)) {
      const float to = fmaxf(ref, max_across_rows(top) - kTop16), f = __builtin_amdgcn_exp2f(ref - to);
      ref = to;
      l *= f;
#pragma unroll
      for (int c = 0; c < 4 * G; ++c) o[c] *= f;
    }
    float sum = 0.0f;
    h8v_t hi[kC], lo[kC];
#pragma unroll
    for (int t = 0; t < kT; ++t) {
      f4v_t p;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        p[v] = __builtin_amdgcn_exp2f(s[t][v] - ref);
        sum += p[v];
      }
      const h4v_t a4 = __builtin_convertvector(p, h4v_t);
      const h4v_t b4 = __builtin_convertvector(p - __builtin_convertvector(a4, f4v_t), h4v_t);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        hi[t / 2][4 * (t & 1) + v] = a4[v];
        lo[t / 2][4 * (t & 1) + v] = b4[v];
      }
    }
    l += sum;
    if (a.w_in) {
      const float all = sum_across_rows(sum);
      if (k == 0 && q_in < group)
        ws.page[((size_t)run.b * a.c.max_pages * kUnits + j) * a.hq + h] = make_float2(ref, all);
    }
#pragma unroll
    for (int c = 0; c < kC; ++c)
#pragma unroll
      for (int u = 0; u < 4 * G; ++u) {
        o[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vr[kC * u + c], lo[c], o[u], 0, 0, 0);
        o[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vr[kC * u + c], hi[c], o[u], 0, 0, 0);
      }
    load_v(next, j2);
    has = has_next;
  }

  l = sum_across_rows(l);
  if (q_in >= group) return;
  const size_t slot = (size_t)r * a.hq + h;
#pragma unroll
  for (int c = 0; c < 4 * G; ++c) *reinterpret_cast<f4v_t*>(ws.o + slot * D + 16 * c + 4 * k) = o[c];
  if (k == 0) ws.ml[slot] = make_float2(l == 0.0f ? -INFINITY : ref, l);
}

// ---------------------------------------------------------------------------
// Joining the runs of a row: with m the largest of their references,
// o = sum o_i 2^(m_i - m) / l, l = sum l_i 2^(m_i - m).  One workgroup per row
// and kWidth channels (a row's channels are shared out where there are few
// rows); behind those, with page weights, one per 16 pages of a sequence.
// Bound by latency: 4 to 5 us, most of it the launch, two dependent reads and
// the sets' sum (as a part of the runs' kernel, by the last wave of a row, it
// took longer: one wave then walks all of them).
constexpr int kJoin = 256, kPagesJoined = 16, kShare = kJoin / kPagesJoined;

// (first, count) of a sequence's runs; the runs kernel wrote those of sequences with pages.
__device__ __forceinline__ int2 sequence_runs(const PagedCache& c, const DecodeWs& ws, int b) {
  const int2 r = ws.runs[b];
  return paged_len(c, b) ? r : make_int2(0, 0);
}

// Two partial sums over runs as one, in the first's place.
__device__ __forceinline__ void join_pair(float& m, float& l, f4v_t& o, float m2, float l2, f4v_t o2) {
  const float to = fmaxf(m, m2), ref = to == -INFINITY ? 0.0f : to;
  const float f = __builtin_amdgcn_exp2f(m - ref), f2 = __builtin_amdgcn_exp2f(m2 - ref);
  m = to;
  l = l * f + l2 * f2;
  o = o * f + o2 * f2;
}

template <int kWidth>
__global__ void __launch_bounds__(kJoin) k_paged_join(PagedDecode a, int rows) {
  constexpr int kCols = kWidth / 4, kSets = kJoin / kCols;
  __shared__ f4v_t part[kSets][kCols];
  __shared__ float2 part_ml[kSets];
  __shared__ float2 joined[4][64];
  const int tid = threadIdx.x, lane = tid & 63, D = a.c.D;
  const int target = run_target(a.hq, a.c.hkv, D, a.c.fp16);
  const DecodeWs ws = decode_ws(a.ws, a.c, target, a.hq);
  if ((int)blockIdx.x < rows) {
    // a set of threads takes every kSets-th run, (m, l) and o in one go; then the sets are joined in order
    const int slices = D / kWidth, row = blockIdx.x / slices, d0 = blockIdx.x % slices * kWidth;
    const int b = row / a.hq, h = row % a.hq;
    const int2 run = sequence_runs(a.c, ws, b);
    const int col = tid % kCols, set = tid / kCols;
    f4v_t o = {0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, l = 0.0f;
    constexpr int kAhead = 4;
    for (int i = set; i < run.y; i += kAhead * kSets) {
      float2 x[kAhead];
      f4v_t y[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const size_t slot = (size_t)(run.x + min(i + u * kSets, run.y - 1)) * a.hq + h;
        x[u] = ws.ml[slot];
        y[u] = *reinterpret_cast<const f4v_t*>(ws.o + slot * D + d0 + 4 * col);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i + u * kSets < run.y) join_pair(m, l, o, x[u].x, x[u].y, y[u]);
    }
    part[set][col] = o;
    if (col == 0) part_ml[set] = make_float2(m, l);
    __syncthreads();
    if (tid < kWidth) {
      float top = -INFINITY, sum = 0.0f, all = 0.0f;
      for (int i = 0; i < kSets; ++i) top = fmaxf(top, part_ml[i].x);
      if (top == -INFINITY) top = 0.0f;
#pragma unroll 8
      for (int i = 0; i < kSets; ++i) {
        const float f = __builtin_amdgcn_exp2f(part_ml[i].x - top);
        all += part_ml[i].y * f;
        sum += part[i][tid / 4][tid & 3] * f;
      }
      a.o[(size_t)row * D + d0 + tid] = (half_t)(all == 0.0f ? 0.0f : sum / all);
      if (tid == 0 && d0 == 0)
        a.lse[(size_t)h * a.c.batch + b] =
            all == 0.0f ? -INFINITY : (float)(((double)top + (double)__log2f(all)) * 0.6931471805599453);
    }
    return;
  }
  // page weights: (m, l) of 64 heads at a time, then the pages, sixteen threads each, whose sums are
  // fetched meanwhile
  const int chunks = (a.c.max_pages + kPagesJoined - 1) / kPagesJoined, at = blockIdx.x - rows;
  const int b = at / chunks, j0 = kPagesJoined * (at % chunks), wave = tid >> 6;
  const int pages = pages_of(a.c, b), j = j0 + tid / kShare;
  const int units = page_units(D, a.c.fp16);
  const size_t place = (size_t)b * a.c.max_pages + min(j, a.c.max_pages - 1);
  const float before = a.w_in[place];
  float w = 0.0f;
  if (j0 < pages) {
    const int2 run = sequence_runs(a.c, ws, b);
    for (int h0 = 0; h0 < a.hq; h0 += 64) {
      float2 y[64 / kShare];
#pragma unroll
      for (int i = 0; i < 64 / kShare; ++i) {
        const int h = h0 + tid % kShare + kShare * i;
        y[i] = j < pages && h < a.hq ? ws.page[place * units * a.hq + h] : make_float2(0.0f, 0.0f);
      }
      float m = -INFINITY, l = 0.0f;
      if (h0 + lane < a.hq)
        for (int i = wave; i < run.y; i += 4) {
          const float2 x = ws.ml[(size_t)(run.x + i) * a.hq + h0 + lane];
          const float to = fmaxf(m, x.x), ref = to == -INFINITY ? 0.0f : to;
          l = l * __builtin_amdgcn_exp2f(m - ref) + x.y * __builtin_amdgcn_exp2f(x.x - ref);
          m = to;
        }
      joined[wave][lane] = make_float2(m, l);
      __syncthreads();
      if (wave == 0) {
        float2 x[4];
        for (int i = 0; i < 4; ++i) x[i] = joined[i][lane];
        m = fmaxf(fmaxf(x[0].x, x[1].x), fmaxf(x[2].x, x[3].x));
        if (m == -INFINITY) m = 0.0f;
        l = 0.0f;
        for (int i = 0; i < 4; ++i) l += x[i].y * __builtin_amdgcn_exp2f(x[i].x - m);
        joined[0][lane] = make_float2(m, l == 0.0f ? 0.0f : 1.0f / l);
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 64 / kShare; ++i) {
        const float2 x = joined[0][tid % kShare + kShare * i];
        w += y[i].y * __builtin_amdgcn_exp2f(y[i].x - x.x) * x.y;
        const int h = h0 + tid % kShare + kShare * i;
        if (units == 2 && j < pages && h < a.hq) {
          const float2 z = ws.page[(place * 2 + 1) * a.hq + h];
          w += z.y * __builtin_amdgcn_exp2f(z.x - x.x) * x.y;
        }
      }
      __syncthreads();
    }
  }
  for (int d = 1; d < kShare; d <<= 1) w += __shfl_xor(w, d);
  if (tid % kShare == 0 && j < a.c.max_pages) a.w_out[place] = j < pages ? a.decay * before + w : before;
}

// Workgroups of the join: those of the rows (their channels shared out while
// there are fewer rows than compute units) and those of the page weights.
static int join_rows(const PagedCache& c, int hq) {
  const int rows = c.batch * hq;
  return rows < 256 ? rows * (c.D / 32) : rows;
}
static int join_pages(const PagedCache& c) { return c.batch * ((c.max_pages + kPagesJoined - 1) / kPagesJoined); }

bool paged_decode_fits(const PagedCache& c, int hq, bool weights) {
  return (size_t)c.batch * c.max_pages * page_units(c.D, c.fp16) < (size_t)1 << 30 &&      // find_run counts in 32 bits
         (size_t)join_rows(c, hq) + (weights ? join_pages(c) : 0) < kMaxGrid;
}

hipError_t launch_paged_decode(const PagedDecode& a, hipStream_t st) {
  const int tiles = query_tiles(a.hq, a.c.hkv, a.c.fp16);
  const size_t runs = run_slots(a.c, run_target(a.hq, a.c.hkv, a.c.D, a.c.fp16));
  const dim3 grid((unsigned)(runs * a.c.hkv * tiles));
  if (a.c.fp16) {
    if (a.c.D == 64)
      k_runs_fp16<1><<<grid, 64, 0, st>>>(a, tiles);
    else if (a.c.D == 128)
      k_runs_fp16<2><<<grid, 64, 0, st>>>(a, tiles);
    else
      k_runs_fp16<4><<<grid, 64, 0, st>>>(a, tiles);
  } else {
    if (a.c.D == 64)
      k_runs_hif4<1><<<grid, 64, 0, st>>>(a, tiles);
    else if (a.c.D == 128)
      k_runs_hif4<2><<<grid, 64, 0, st>>>(a, tiles);
    else
      k_runs_hif4<4><<<grid, 64, 0, st>>>(a, tiles);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int groups = join_rows(a.c, a.hq);
  const bool few = groups != a.c.batch * a.hq;
  const dim3 join((unsigned)(groups + (a.w_in ? join_pages(a.c) : 0)));
  if (few)
    k_paged_join<32><<<join, kJoin, 0, st>>>(a, groups);
  else if (a.c.D == 64)
    k_paged_join<64><<<join, kJoin, 0, st>>>(a, groups);
  else if (a.c.D == 128)
    k_paged_join<128><<<join, kJoin, 0, st>>>(a, groups);
  else
    k_paged_join<256><<<join, kJoin, 0, st>>>(a, groups);
  return hipGetLastError();
}

}  // namespace hifa4
