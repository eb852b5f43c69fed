// One new token's attention over the paged cache (records: hifa4_paged.h).
//
// For query row h of sequence b over its L cached tokens:
//   S_j = (q~ . k_j) / sqrt(D),  p_j = exp(S_j - m) / l,  o = sum_j p_j v_j,
//   LSE = m + ln l,  with m = max S_j and l = sum_j exp(S_j - m);
//   page weights w'[page] = decay w[page] + sum over the heads and the page's
//   tokens of p_j.
// q~ = fp16(q s) under Smooth-QK (the cache holds k/s); keys and values are
// what the cache holds; scores, m, l, the weights p and o are held in fp32 and
// o is rounded once to fp16.
//
// The pages of all sequences are cut into runs of about equal length, as many
// as fill the chip: a run leaves (m, l, o) of its rows, and a second kernel
// joins the runs of a row.  Lengths are read on the device, so a captured call
// follows them.
#include "hifa4_device.h"
#include "hifa4_packed.h"
#include "hifa4_paged.h"

#include <algorithm>

namespace hifa4 {

constexpr int kWaves = 2048;      // waves that share the work of a call

// How the pages are cut: a run has at most `per` pages, every sequence is cut
// into equal parts, and all of them are numbered densely: at most
// run_slots() runs.
__host__ __device__ __forceinline__ int run_target(int hkv) { return (kWaves + hkv - 1) / hkv; }
__host__ __device__ __forceinline__ size_t run_slots(int batch, int hkv, int max_pages) {
  const size_t all = (size_t)batch * max_pages, most = (size_t)run_target(hkv) + batch;
  return all < most ? all : most;
}
struct Run {
  int b, begin, end;              // pages [begin, end) of sequence b; b < 0: no such run
  int first, count;               // the sequence's runs: [first, first + count)
};

__device__ __forceinline__ int wave_sum(int x) {
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ int pages_of(const PagedCache& c, int b) {
  return b < c.batch ? (paged_len(c, b) + kPage - 1) / kPage : 0;
}
__device__ __forceinline__ int pages_per_run(const PagedCache& c, int lane) {
  int total = 0;
  for (int b0 = 0; b0 < c.batch; b0 += 64) total += pages_of(c, b0 + lane);
  total = wave_sum(total);
  const int target = run_target(c.hkv);
  return max(1, (total + target - 1) / target);
}
// The run numbered r (found by a whole wave), or with r < 0 the runs of
// sequence `want`.
__device__ __forceinline__ Run find_run(const PagedCache& c, int r, int want, int lane) {
  const int per = pages_per_run(c, lane);
  Run out = {-1, 0, 0, 0, 0};
  int before = 0;
  for (int b0 = 0; b0 < c.batch; b0 += 64) {
    const int b = b0 + lane, n = pages_of(c, b), cnt = (n + per - 1) / per;
    int upto = cnt;
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(upto, d);
      if (lane >= d) upto += y;
    }
    const int mine = before + upto - cnt;
    const bool hit = r >= 0 ? (r >= mine && r < mine + cnt) : b == want;
    const unsigned long long who = __ballot(hit);
    if (who) {
      const int src = __ffsll(who) - 1;
      out.b = b0 + src;
      out.first = __shfl(mine, src);
      out.count = __shfl(cnt, src);
      const int pages = __shfl(n, src);
      if (r >= 0) {
        out.begin = (int)((long)(r - out.first) * pages / out.count);
        out.end = (int)((long)(r - out.first + 1) * pages / out.count);
      }
      return out;
    }
    before += __shfl(upto, 63);
  }
  return out;
}

// Workspace: o [slots][hq][D], then (m, l) [slots][hq], then with page weights
// (m, sum) [batch][max_pages][hq]; m in log2 units.
struct DecodeWs {
  float* o;
  float2* ml;
  float2* page;
};
__host__ __device__ __forceinline__ DecodeWs decode_ws(uint8_t* ws, int batch, int hq, int hkv, int D, int max_pages) {
  const size_t slots = run_slots(batch, hkv, max_pages);
  DecodeWs w;
  w.o = reinterpret_cast<float*>(ws);
  w.ml = reinterpret_cast<float2*>(w.o + slots * hq * D);
  w.page = w.ml + slots * hq;
  return w;
}
size_t paged_decode_workspace(int batch, int hq, int hkv, int D, int max_pages, bool weights) {
  const size_t slots = run_slots(batch, hkv, max_pages);
  return slots * hq * (D + 2) * 4 + (weights ? (size_t)batch * max_pages * hq * 8 : 0);
}

// fp16(q s): the exact product rounded once.
__device__ __forceinline__ half_t smoothed_q(const PagedDecode& a, int b, int h, int d) {
  const half_t q = a.q[((size_t)b * a.hq + h) * a.c.D + d];
  if (!a.s) return q;
  return rn16_from_f64((double)q * (double)a.s[(size_t)(h / (a.hq / a.c.hkv)) * a.c.D + d]);
}

__device__ __forceinline__ float record_value(const uint8_t* rec, int D, bool fp16, bool v, int key, int ch) {
  const int t = key_t(key), n = key_n(key), G = D / 64;
  if (fp16) {
    const half_t* x = reinterpret_cast<const half_t*>(rec);
    return v ? (float)x[64 * D + (((size_t)(ch / 16) * 2 + (key >> 3 & 1)) * 64 + 16 * (key >> 4) + (ch & 15)) * 8 + (key & 7)]
             : (float)x[(((size_t)t * (D / 32) + ch / 32) * 64 + 16 * (ch / 8 % 4) + n) * 8 + (ch & 7)];
  }
  const uint8_t* part = v ? rec + hif4_part(G) : rec;
  const int tile = ch >> 6, rt = v ? (ch >> 4) & 3 : t, rn = v ? ch & 15 : n, elem = v ? key : ch & 63;
  const int w = elem >> 3, i = elem & 7, lane = 16 * (w >> 1) + rn, bit = 2 * rt + (w & 1);
  const uint32_t nib = (part[hif4_code_at(tile, rt, lane, w & 1) + (i >> 1)] >> (4 * (i & 1))) & 15u;
  const int sh = ((part[hif4_e2_at(G, tile, lane)] >> bit) & 1) + ((part[hif4_e3_at(G, tile, lane, i >> 2)] >> bit) & 1);
  const float x = (float)(nib & 7u) * e6m2_value(part[hif4_base_at(G, tile, rt, rn)]) *
                  (sh == 0 ? 0.25f : sh == 1 ? 0.125f : 0.0625f);
  return nib & 8u ? -x : x;
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
// page is rounded to 2^-20 of that one's weight.
//
// Slots of v_mfma_scale_f32_16x16x128_f8f6f4 (measured): FP4 operand lane
// 16k + n holds K 32k .. 32k+31, its four registers in order; FP8 operand lane
// 16k + n holds K 16k .. 16k+15 in its first four registers and 64 + 16k .. in
// the others.  So FP8 lanes k = 2j, 2j+1 meet FP4 lanes j and 2 + j: they hold
// the words of both, each twice.  V is read with its lanes k = 1 and 2
// exchanged, which makes the words of FP4 lanes j and 2 + j the keys whose
// scores lanes 2j and 2j + 1 have: one exchange between neighbouring rows of
// 16 lanes brings p into place.
typedef int i8v_t __attribute__((ext_vector_type(8)));
typedef float f4v_t __attribute__((ext_vector_type(4)));
typedef short s2v_t __attribute__((ext_vector_type(2)));

constexpr int kFp4 = 4, kFp8 = 0;            // operand formats of the instruction
// The reference of the softmax is a whole power of two and moves only when a
// page's largest score passes it by this many binades: fp32 sums do not mind.
constexpr float kSlack = 16.0f;
// E8M0 byte of the FP4 side without E2: 2^(94 - E2).  The bases enter as the
// float whose bits are byte << 21 = b 2^-96, and an operand's sum is 4 values.
constexpr uint32_t kUnit = 127 + 94;

// x and y lane values of (own, partner) exchanges
__device__ __forceinline__ float max_across_rows(float v) {      // over the four lanes of a column
  const Pair32 p = pair32(__float_as_uint(v));
  v = fmaxf(__uint_as_float(p.x), __uint_as_float(p.y));
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_across_rows(float v) {
  v = add_with_partner(v);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// over the four pieces of a query (the same bits in each of the four lanes)
__device__ __forceinline__ float sum_pieces(float v) {
  v += __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0xB1, 0xF, 0xF, true));
  return v + __uint_as_float(__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), 0x4E, 0xF, 0xF, true));
}

// Digit k of x (|x| <= 16): rint(32^k x) - 32 rint(32^(k-1) x), between -16 and
// 16; digits 0..3 add up to rint(32^3 x) / 32^3.
struct DigitScale {
  float now, before;       // 32^k and, for k > 0, 32^(k-1)
};
__device__ __forceinline__ DigitScale digit_scale(int k) {
  return DigitScale{__uint_as_float((uint32_t)(127 + 5 * k) << 23), k ? __uint_as_float((uint32_t)(122 + 5 * k) << 23) : 0.0f};
}
__device__ __forceinline__ float digit(float x, const DigitScale& s) {
  return fmaf(-32.0f, __builtin_rintf(x * s.before), __builtin_rintf(x * s.now));
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
  uint4 base[G];           // word t: the four rows whose products the lane holds
};
template <int G>
__device__ __forceinline__ void load_part(Part<G>& p, const uint8_t* part, int lane, int k) {
#pragma unroll
  for (int i = 0; i < 2 * G; ++i) p.code[i] = *reinterpret_cast<const uint4*>(part + 1024 * i + 16 * lane);
  const uint8_t* e3 = part + 2048 * G + 2 * G * lane;
  const uint8_t* e2 = part + 2176 * G + G * lane;
  if (G == 1) {
    p.e3[0] = *reinterpret_cast<const uint16_t*>(e3);
    p.e2 = *e2;
  } else if (G == 2) {
    p.e3[0] = *reinterpret_cast<const uint32_t*>(e3);
    p.e2 = *reinterpret_cast<const uint16_t*>(e2);
  } else {
    const uint2 x = *reinterpret_cast<const uint2*>(e3);
    p.e3[0] = x.x;
    p.e3[G == 4 ? 1 : 0] = x.y;
    p.e2 = *reinterpret_cast<const uint32_t*>(e2);
  }
#pragma unroll
  for (int i = 0; i < G; ++i) p.base[i] = *reinterpret_cast<const uint4*>(part + 2240 * G + 16 * G * k + 16 * i);
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
// Products of a tile's rows 16 T + 4k + v with the columns of b (both words).
template <int G, int T>
__device__ __forceinline__ f4v_t tile_product(const Part<G>& p, int tile, uint32_t x, uint32_t s0, uint32_t s1,
                                              const i8v_t& b0, const i8v_t& b1, uint32_t b_scale) {
  const uint4 w = p.code[2 * tile + T / 2];
  f4v_t c = {0.0f, 0.0f, 0.0f, 0.0f};
  c = mfma_word<T>(T & 1 ? w.z : w.x, e3_keep<G>(x, tile, T, 0), s0, b0, b_scale, c);
  return mfma_word<T>(T & 1 ? w.w : w.y, e3_keep<G>(x, tile, T, 1), s1, b1, b_scale, c);
}
template <int G>
__device__ __forceinline__ uint32_t e3_halves(const Part<G>& p, int tile) {
  const uint32_t x = ~p.e3[tile / 2];
  return G == 1 ? (x & 0xFFu) | ((x & 0xFF00u) << 8) : x;
}
__device__ __forceinline__ f4v_t bases(uint32_t w) {
  return f4v_t{__uint_as_float((w & 0xFFu) << 21), __uint_as_float((w >> 8 & 0xFFu) << 21),
               __uint_as_float((w >> 16 & 0xFFu) << 21), __uint_as_float((w >> 24) << 21)};
}
template <int G, typename F>
__device__ __forceinline__ void products(const Part<G>& p, const i8v_t* b0, const i8v_t* b1, const uint32_t* b_scale, F use) {
#pragma unroll
  for (int tile = 0; tile < G; ++tile) {
    const uint32_t x = e3_halves<G>(p, tile), s0 = e2_scales(p.e2, tile, 0), s1 = e2_scales(p.e2, tile, 1);
    const uint4 bw = p.base[tile];
    use(tile, 0, tile_product<G, 0>(p, tile, x, s0, s1, b0[tile], b1[tile], b_scale[tile]), bases(bw.x));
    use(tile, 1, tile_product<G, 1>(p, tile, x, s0, s1, b0[tile], b1[tile], b_scale[tile]), bases(bw.y));
    use(tile, 2, tile_product<G, 2>(p, tile, x, s0, s1, b0[tile], b1[tile], b_scale[tile]), bases(bw.z));
    use(tile, 3, tile_product<G, 3>(p, tile, x, s0, s1, b0[tile], b1[tile], b_scale[tile]), bases(bw.w));
  }
}

// The pages of a run, as their records: 64 table entries at a time, one a lane.
struct Pages {
  int mine, base;
};
__device__ __forceinline__ void load_pages(Pages& p, const PagedCache& c, const Run& r, int from, int lane) {
  p.base = from;
  p.mine = from + lane < r.end ? c.table[(size_t)r.b * c.max_pages + from + lane] : -1;
}

template <int G>
__global__ void __launch_bounds__(64) k_runs_hif4(PagedDecode a, int tiles) {
  constexpr int D = 64 * G;
  const int lane = threadIdx.x, n = lane & 15, k = lane >> 4, piece = n & 3;
  const int head = blockIdx.x % a.c.hkv, group = a.hq / a.c.hkv;
  const int tile = blockIdx.x / a.c.hkv % tiles, r = blockIdx.x / a.c.hkv / tiles;
  const Run run = find_run(a.c, r, 0, lane);
  if (run.b < 0) return;
  const int len = paged_len(a.c, run.b);
  const DecodeWs ws = decode_ws(a.ws, a.c.batch, a.hq, a.c.hkv, D, a.c.max_pages);
  const size_t rec_bytes = (size_t)72 * D;
  const int v_lane = 16 * ((k & 1) * 2 + (k >> 1)) + n;        // lanes k = 1, 2 exchanged

  Pages pg;
  load_pages(pg, a.c, run, run.begin, lane);
  bool has, has_next = false;
  // The record of page j; of a page that is none the pool's first, whose keys are all masked then.
  const auto record = [&](int j, bool& there) -> const uint8_t* {
    if (j - pg.base >= 64) load_pages(pg, a.c, run, j, lane);
    const int page = __builtin_amdgcn_readlane(pg.mine, j - pg.base);
    there = (unsigned)page < (unsigned)a.c.num_pages;
    return a.c.pool + ((size_t)(there ? page : 0) * a.c.hkv + head) * rec_bytes;
  };
  Part<G> kp, vp;
  const uint8_t* rec = record(run.begin, has);
  load_part<G>(kp, rec, lane, k);
  load_part<G>(vp, rec + 2304 * G, v_lane, k);

  // the query's pieces
  const int q_in = 4 * tile + (n >> 2), h = head * group + q_in;
  const DigitScale ds = digit_scale(piece);
  i8v_t qa[G], qb[G];
  uint32_t q_scale[G];
  {
    const int j = k >> 1;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float x[2][2][8];                // [c][FP4 lane j, 2 + j][value]
      float top = 0.0f;
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const int ch = 64 * g + 8 * (2 * (j + 2 * f) + c);
          uint4 in = make_uint4(0, 0, 0, 0);
          if (q_in < group) in = *reinterpret_cast<const uint4*>(a.q + ((size_t)run.b * a.hq + h) * D + ch);
          const h2_t y[4] = {__builtin_bit_cast(h2_t, in.x), __builtin_bit_cast(h2_t, in.y),
                             __builtin_bit_cast(h2_t, in.z), __builtin_bit_cast(h2_t, in.w)};
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            half_t z = y[i >> 1][i & 1];
            if (a.s) z = rn16_from_f64((double)z * (double)a.s[(size_t)head * D + ch + i]);
            x[c][f][i] = (float)z;
            top = fmaxf(top, fabsf((float)z));
          }
        }
      top = max_across_rows(top);
      // 2^e <= top < 2^(e+1): 2^(3-e) x lies below 16
      const int e = top > 0.0f ? (int)(__float_as_uint(top) >> 23) - 127 : 0;
      const float up = __uint_as_float((uint32_t)(127 + 3 - e) << 23);
      q_scale[g] = (uint32_t)(127 + e - 3 - 5 * piece);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        int w[2][2];
#pragma unroll
        for (int f = 0; f < 2; ++f)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) y[u] = digit(x[c][f][4 * i + u] * up, ds);
            w[f][i] = (int)fp8x4(y[0], y[1], y[2], y[3]);
          }
        (c ? qb : qa)[g] = i8v_t{w[0][0], w[0][1], w[0][0], w[0][1], w[1][0], w[1][1], w[1][0], w[1][1]};
      }
    }
  }

  // scores in log2 units; sums are of p = 2^(score - ref), ref a whole number
  float ref = -1e30f, l = 0.0f;
  f4v_t o[G][4];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int t = 0; t < 4; ++t) o[g][t] = f4v_t{0.0f, 0.0f, 0.0f, 0.0f};

  for (int j = run.begin; j < run.end; ++j) {
    f4v_t s[4];
    products<G>(kp, qa, qb, q_scale, [&](int g, int t, f4v_t d, f4v_t b) {
#pragma unroll
      for (int v = 0; v < 4; ++v) s[t][v] = g == 0 ? d[v] * b[v] : fmaf(d[v], b[v], s[t][v]);
    });
    // the next page's K loads while this page's softmax and V go on
    const uint8_t* next = nullptr;
    if (j + 1 < run.end) {
      next = record(j + 1, has_next);
      load_part<G>(kp, next, lane, k);
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) s[t][v] = sum_pieces(s[t][v]) * a.scale;
    const int held = has ? len - j * kPage : 0;
    if (held < kPage) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (16 * k + 4 * t + v >= held) s[t][v] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int v = 0; v < 4; ++v) top = fmaxf(top, s[t][v]);
    // the page's own reference: the next whole number above its largest score
    // (far below ref, where nothing of the page counts, 100 binades are enough)
    const float own = fmaxf(ceilf(max_across_rows(top)), ref - 100.0f);
    if (__builtin_amdgcn_ballot_w64(own > ref + kSlack)) {
      const float to = fmaxf(ref, own), f = __builtin_amdgcn_exp2f(ref - to);
      ref = to;
      l *= f;
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int t = 0; t < 4; ++t) o[g][t] *= f;
    }
    float sum = 0.0f;
    uint32_t pw[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      float y[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float p = __builtin_amdgcn_exp2f(s[t][v] - (own - 4.0f));      // 16 p, at most 16
        sum += p;
        y[v] = digit(p, ds);
      }
      pw[t] = fp8x4(y[0], y[1], y[2], y[3]);
    }
    // 2^(own - ref - 4): what the page's sums count
    const int up = (int)(own - ref) - 4;
    l = fmaf(sum, __uint_as_float((uint32_t)(127 + up) << 23), l);
    const uint32_t p_scale = (uint32_t)(127 + up - 5 * piece);
    if (a.w_in) {
      const float all = sum_across_rows(sum);
      if (k == 0 && piece == 0 && q_in < group)
        ws.page[((size_t)run.b * a.c.max_pages + j) * a.hq + h] = make_float2(own - 4.0f, all);
    }
    i8v_t pa[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const auto x = __builtin_amdgcn_permlane16_swap(pw[2 * c], pw[2 * c], false, false);
      const auto y = __builtin_amdgcn_permlane16_swap(pw[2 * c + 1], pw[2 * c + 1], false, false);
      pa[c] = i8v_t{(int)x[0], (int)y[0], (int)x[0], (int)y[0], (int)x[1], (int)y[1], (int)x[1], (int)y[1]};
    }
    i8v_t p0[G], p1[G];
    uint32_t ps[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      p0[g] = pa[0];
      p1[g] = pa[1];
      ps[g] = p_scale;
    }
    products<G>(vp, p0, p1, ps, [&](int g, int t, f4v_t d, f4v_t b) {
#pragma unroll
      for (int v = 0; v < 4; ++v) o[g][t][v] = fmaf(d[v], b[v], o[g][t][v]);
    });
    if (next) load_part<G>(vp, next + 2304 * G, v_lane, k);
    has = has_next;
  }

  l = sum_across_rows(l);
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

// FP16 pages.  One wave per (run, query head).
__global__ void __launch_bounds__(64) k_runs_fp16(PagedDecode a) {
  __shared__ float qs[256], ps[64];
  const int lane = threadIdx.x, D = a.c.D;
  const int h = blockIdx.x % a.hq, r = blockIdx.x / a.hq;
  const Run run = find_run(a.c, r, 0, lane);
  if (run.b < 0) return;
  const int len = paged_len(a.c, run.b), head = h / (a.hq / a.c.hkv);
  const DecodeWs ws = decode_ws(a.ws, a.c.batch, a.hq, a.c.hkv, D, a.c.max_pages);
  for (int d = lane; d < D; d += 64) qs[d] = (float)smoothed_q(a, run.b, h, d);
  float m = -INFINITY, l = 0.0f, o[4] = {0, 0, 0, 0};
  __syncthreads();
  for (int j = run.begin; j < run.end; ++j) {
    const uint8_t* rec = paged_record(a.c, run.b, j, head);
    float s = -INFINITY;
    if (rec && j * kPage + lane < len) {
      s = 0.0f;
      for (int d = 0; d < D; ++d) s = fmaf(qs[d], record_value(rec, D, a.c.fp16, false, lane, d), s);
      s *= a.scale;
    }
    float top = s;
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    const float m_new = fmaxf(m, top), ref = m_new == -INFINITY ? 0.0f : m_new;
    const float p = exp2f(s - ref), f = exp2f(m - ref);
    float sum = p;
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    l = l * f + sum;
    m = m_new;
    if (a.w_in && lane == 0)
      ws.page[((size_t)run.b * a.c.max_pages + j) * a.hq + h] = make_float2(m, sum);
    ps[lane] = p;
    __syncthreads();
    for (int i = 0; i < D / 64; ++i) {
      o[i] *= f;
      if (rec)
        for (int key = 0; key < kPage; ++key)
          if (ps[key] != 0.0f) o[i] = fmaf(ps[key], record_value(rec, D, a.c.fp16, true, key, 64 * i + lane), o[i]);
    }
    __syncthreads();
  }
  const size_t slot = (size_t)r * a.hq + h;
  for (int i = 0; i < D / 64; ++i) ws.o[slot * D + 64 * i + lane] = o[i];
  if (lane == 0) ws.ml[slot] = make_float2(m, l);
}

// LSE (log2) of row (b, h) from its runs.
__device__ __forceinline__ float2 row_lse(const DecodeWs& ws, int hq, const Run& run, int h, int lane) {
  float m = -INFINITY;
  for (int i = lane; i < run.count; i += 64) m = fmaxf(m, ws.ml[(size_t)(run.first + i) * hq + h].x);
  for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  const float ref = m == -INFINITY ? 0.0f : m;
  float l = 0.0f;
  for (int i = lane; i < run.count; i += 64) {
    const float2 x = ws.ml[(size_t)(run.first + i) * hq + h];
    l += x.y * exp2f(x.x - ref);
  }
  for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d);
  return make_float2(ref, l);
}

// One wave per row (b, h); behind them one wave per 64 pages of a sequence.
__global__ void __launch_bounds__(64) k_paged_join(PagedDecode a, int rows) {
  const int lane = threadIdx.x, D = a.c.D;
  const DecodeWs ws = decode_ws(a.ws, a.c.batch, a.hq, a.c.hkv, D, a.c.max_pages);
  if ((int)blockIdx.x < rows) {
    const int b = blockIdx.x / a.hq, h = blockIdx.x % a.hq;
    const Run run = find_run(a.c, -1, b, lane);
    const float2 x = row_lse(ws, a.hq, run, h, lane);
    for (int d = lane; d < D; d += 64) {
      float o = 0.0f;
      for (int i = 0; i < run.count; ++i) {
        const size_t slot = (size_t)(run.first + i) * a.hq + h;
        o += ws.o[slot * D + d] * exp2f(ws.ml[slot].x - x.x);
      }
      a.o[(size_t)blockIdx.x * D + d] = (half_t)(x.y == 0.0f ? 0.0f : o / x.y);
    }
    if (lane == 0)
      a.lse[(size_t)h * a.c.batch + b] = x.y == 0.0f ? -INFINITY : (float)((x.x + log2f(x.y)) * 0.6931471805599453);
    return;
  }
  const int chunks = (a.c.max_pages + 63) / 64, at = blockIdx.x - rows;
  const int b = at / chunks, j = 64 * (at % chunks) + lane;
  const Run run = find_run(a.c, -1, b, lane);
  const int pages = pages_of(a.c, b);
  if (j - lane >= a.c.max_pages) return;
  float w = 0.0f;
  for (int h = 0; h < a.hq && pages > j - lane; ++h) {
    const float2 x = row_lse(ws, a.hq, run, h, lane);
    if (j < pages && x.y != 0.0f) {
      const float2 y = ws.page[((size_t)b * a.c.max_pages + j) * a.hq + h];
      w += y.y * exp2f(y.x - x.x) / x.y;
    }
  }
  if (j < a.c.max_pages) {
    const size_t i = (size_t)b * a.c.max_pages + j;
    a.w_out[i] = j < pages ? a.decay * a.w_in[i] + w : a.w_in[i];
  }
}

hipError_t launch_paged_decode(const PagedDecode& a, hipStream_t st) {
  const size_t runs = run_slots(a.c.batch, a.c.hkv, a.c.max_pages);
  const int tiles = (a.hq / a.c.hkv + 3) / 4;
  const dim3 grid((unsigned)(a.c.fp16 ? runs * a.hq : runs * a.c.hkv * tiles));
  if (a.c.fp16)
    k_runs_fp16<<<grid, 64, 0, st>>>(a);
  else if (a.c.D == 64)
    k_runs_hif4<1><<<grid, 64, 0, st>>>(a, tiles);
  else if (a.c.D == 128)
    k_runs_hif4<2><<<grid, 64, 0, st>>>(a, tiles);
  else
    k_runs_hif4<4><<<grid, 64, 0, st>>>(a, tiles);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int rows = a.c.batch * a.hq;
  const size_t extra = a.w_in ? (size_t)a.c.batch * ((a.c.max_pages + 63) / 64) : 0;
  k_paged_join<<<dim3((unsigned)(rows + extra)), 64, 0, st>>>(a, rows);
  return hipGetLastError();
}

}  // namespace hifa4
