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

// One wave per (run, query head).
__global__ void __launch_bounds__(64) k_paged_runs(PagedDecode a) {
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
  const size_t runs = run_slots(a.c.batch, a.c.hkv, a.c.max_pages) * a.hq;
  if (runs) {
    k_paged_runs<<<dim3((unsigned)runs), 64, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int rows = a.c.batch * a.hq;
  const size_t extra = a.w_in ? (size_t)a.c.batch * ((a.c.max_pages + 63) / 64) : 0;
  k_paged_join<<<dim3((unsigned)(rows + extra)), 64, 0, st>>>(a, rows);
  return hipGetLastError();
}

}  // namespace hifa4
