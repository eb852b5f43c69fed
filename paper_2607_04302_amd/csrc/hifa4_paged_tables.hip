// The paged cache's tables: pages dealt out of a stack of free ones and put back.
//
// Row b holds L tokens and gets n more: the places ceil(L/64) .. ceil((L+n)/64) - 1
// of its table need a page.  With u_b the running sum of those over the rows, the
// j-th new page of row b is free[top - 1 - (u_b + j)]: which page goes where follows
// from sums alone, so every workgroup finds its own pages and no order is left to
// chance.  A release is the mirror image: the entry of rank r of T (row by row, place
// by place) goes to free[top + T - 1 - r], so that it undoes an extension.
#include "hifa4_paged.h"
#include "hifa4_paged_tables.h"

#include <algorithm>

namespace hifa4 {

constexpr int kExtendThreads = 1024;
// kFillTokens: what one workgroup of the second kernel takes.  kExtendAlone: the new
// tokens (of all rows) up to which the first kernel fills everything in by itself.  All of
// it is latency: a launch and chains of three loads.  32 rows of a token: 2.7 us, a call
// 8.5 to 9.7 (by two kernels 11.1 to 12.7); 64 prompts of 1.08 million tokens in all: 3.5
// and 7.3 us, a call 11.3 to 13.0 (512 or 8192 tokens a workgroup: 11.3 to 13.2 and 16.4
// to 17.1), 2.6 of them the bytes.
constexpr int kExtendAlone = 4096;

__device__ __forceinline__ int extend_len(const PagedExtend& a, int b) {
  return max(0, min(a.lens[b], a.max_pages * kPage));
}
// Tokens that row b asks for: none where they are more than its table or the launch holds.
__device__ __forceinline__ int extend_asked(const PagedExtend& a, int b, int len) {
  const int n = max(0, a.counts[b]);
  return n <= min(a.max_new, a.max_pages * kPage - len) ? n : 0;
}
__device__ __forceinline__ int pages_in(int tokens) { return (tokens + kPage - 1) / kPage; }

// New tokens of row b, `len` tokens before them; the row's first new page is the one
// below stack place `top`.
struct RowPlan {
  int b, len, top;
};
// Page of the row's i-th new token.
__device__ __forceinline__ int page_of(const PagedExtend& a, const RowPlan& r, int i) {
  const int place = (r.len + i) / kPage, have = pages_in(r.len);
  return place < have ? a.table[(size_t)r.b * a.max_pages + place] : a.free[r.top - 1 - (place - have)];
}
// The token, t-th of all, is put down; the first of a new page puts down the page.
__device__ __forceinline__ void place_token(const PagedExtend& a, const RowPlan& r, int i, int t, int page, int shift) {
  const int at = r.len + i, place = at / kPage;
  if (place >= pages_in(r.len) && (i == 0 || at % kPage == 0)) a.table[(size_t)r.b * a.max_pages + place] = page;
  a.positions[t] = at + shift;
  a.slots[t] = page < 0 ? -1 : (int64_t)page * kPage + at % kPage;
}

// Sums over the workgroup's threads before this one, and over all (64 bits: 2^30
// pages of 64 tokens).
struct Sums {
  long tokens, pages;
};
template <int kCtrl, int kRowMask, bool kBound>
__device__ __forceinline__ long add_dpp(long x) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, kCtrl, kRowMask, 0xF, kBound);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), kCtrl, kRowMask, 0xF, kBound);
  return x + (long)((uint64_t)lo | (uint64_t)hi << 32);
}
__device__ __forceinline__ long wave_scan(long x) {
  x = add_dpp<0x111, 0xF, true>(x);      // row_shr 1, 2, 4, 8
  x = add_dpp<0x112, 0xF, true>(x);
  x = add_dpp<0x114, 0xF, true>(x);
  x = add_dpp<0x118, 0xF, true>(x);
  x = add_dpp<0x142, 0xA, false>(x);     // lane 15 of each row to the next
  return add_dpp<0x143, 0xC, false>(x);
}
__device__ __forceinline__ Sums scan_sums(Sums x, Sums* waves, Sums& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Sums s = {wave_scan(x.tokens), wave_scan(x.pages)};
  if (lane == 63) waves[wave] = s;
  __syncthreads();
  all = Sums{0, 0};
  Sums before = {s.tokens - x.tokens, s.pages - x.pages};
  for (int w = 0; w < (int)blockDim.x / 64; ++w) {
    const Sums y = waves[w];
    if (w < wave) {
      before.tokens += y.tokens;
      before.pages += y.pages;
    }
    all.tokens += y.tokens;
    all.pages += y.pages;
  }
  __syncthreads();
  return before;
}

// What every row gets: one workgroup over the batch, a row a thread.  With kAlone
// (few tokens, at most a row a thread) it also fills in pages, positions and slots,
// which saves a launch.
template <bool kAlone>
__global__ void __launch_bounds__(kExtendThreads) k_paged_extend(PagedExtend a) {
  __shared__ Sums waves[kExtendThreads / 64];
  __shared__ int first[kExtendThreads + 1], lens[kExtendThreads], stacks[kExtendThreads];
  const int tid = threadIdx.x;
  const int top = max(0, min(a.num_free[0], a.capacity));
  Sums upto = {0, 0};                    // asked for by the rows before
  long given = 0;
  int taken = 0;
  for (int b0 = 0; b0 < a.batch; b0 += blockDim.x) {
    const int b = b0 + tid;
    const bool there = b < a.batch;
    const int len = there ? extend_len(a, b) : 0, asked = there ? extend_asked(a, b, len) : 0;
    const int need = pages_in(len + asked) - pages_in(len);
    Sums all;
    const Sums before = scan_sums(Sums{asked, need}, waves, all);
    const bool fits = upto.tokens + before.tokens + asked <= a.max_total &&
                      (need == 0 || upto.pages + before.pages + need <= top);
    const int n = fits ? asked : 0, pages = fits ? need : 0;
    Sums got = all, mine = before;
    if (upto.tokens + all.tokens > a.max_total || upto.pages + all.pages > top) mine = scan_sums(Sums{n, pages}, waves, got);
    const int t0 = (int)(given + mine.tokens), stack = top - taken - (int)mine.pages;
    if (there) {
      a.cu[b] = t0;
      a.out_lens[b] = len + n;
      if (kAlone) {
        first[b] = t0;
        lens[b] = len;
        stacks[b] = stack;
      }
    }
    upto.tokens += all.tokens;
    upto.pages += all.pages;
    given += got.tokens;
    taken += (int)got.pages;
  }
  if (tid == 0) {
    a.cu[a.batch] = (int)given;
    a.out_free[0] = top - taken;
  }
  if (!kAlone) return;
  if (tid == 0) first[a.batch] = (int)given;
  __syncthreads();
  for (int t = tid; t < a.max_total; t += blockDim.x) {
    if (t >= (int)given) {
      a.positions[t] = -1;
      a.slots[t] = -1;
      continue;
    }
    int b = 0, behind = a.batch;         // first[b] <= t < first[behind]
    while (behind - b > 1) {
      const int mid = (b + behind) / 2;
      if (first[mid] <= t)
        b = mid;
      else
        behind = mid;
    }
    const RowPlan r = {b, lens[b], stacks[b]};
    place_token(a, r, t - first[b], t, page_of(a, r, t - first[b]), a.shift ? a.shift[b] : 0);
  }
}

// Pages, positions and slots of up to kFillTokens new tokens of one row.
__global__ void __launch_bounds__(kFillThreads) k_paged_extend_fill(PagedExtend a, int chunks) {
  __shared__ int sums[2][kFillThreads / 64];
  const int b = blockIdx.x / chunks, i0 = blockIdx.x % chunks * kFillTokens, tid = threadIdx.x;
  // (all loads that hang on nothing first)
  const int total = a.cu[a.batch], t0 = a.cu[b], n = a.cu[b + 1] - t0, has = a.out_lens[b], left = a.out_free[0];
  const int shift = a.shift ? a.shift[b] : 0;
  int before = 0, all = 0;
  for (int r = tid; r < a.batch; r += kFillThreads) {
    const int len = a.out_lens[r], pages = pages_in(len) - pages_in(len - (a.cu[r + 1] - a.cu[r]));
    all += pages;
    if (r < b) before += pages;
  }
  for (int64_t t = tail_first(total, blockIdx.x, tid); t < a.max_total; t += tail_step(gridDim.x)) {
    a.positions[t] = -1;
    a.slots[t] = -1;
  }
  if (i0 >= n) return;
  // pages that the rows before this one took, and all rows: what is left says where the stack began
  before = wave_scan(before);
  all = wave_scan(all);
  if ((tid & 63) == 63) {
    sums[0][tid >> 6] = before;
    sums[1][tid >> 6] = all;
  }
  __syncthreads();
  before = all = 0;
#pragma unroll
  for (int w = 0; w < kFillThreads / 64; ++w) {
    before += sums[0][w];
    all += sums[1][w];
  }
  const RowPlan row = {b, has - n, left + all - before};
  const int end = fill_end(n, i0);
  constexpr int kMine = kFillTokens / kFillThreads;
  int page[kMine];
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    const int i = i0 + tid + u * kFillThreads;
    page[u] = i < end ? page_of(a, row, i) : 0;
  }
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    const int i = i0 + tid + u * kFillThreads;
    if (i < end) place_token(a, row, i, t0 + i, page[u], shift);
  }
}

hipError_t launch_paged_extend(const PagedExtend& a, hipStream_t st) {
  if (a.max_total <= kExtendAlone && a.batch <= kExtendThreads) {
    // a thread for each row and, up to a point, for each token: fewer waves meet sooner
    const int threads = std::max(a.batch, std::min(a.max_total, kExtendThreads));
    k_paged_extend<true><<<dim3(1), (threads + 63) / 64 * 64, 0, st>>>(a);
    return hipGetLastError();
  }
  k_paged_extend<false><<<dim3(1), kExtendThreads, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.max_total == 0) return e;
  const int chunks = extend_chunks(a.max_new);
  k_paged_extend_fill<<<dim3((unsigned)(a.batch * chunks)), kFillThreads, 0, st>>>(a, chunks);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Release: the rows' entries are counted, then placed by their rank.
constexpr int kReleaseThreads = 256;

__device__ __forceinline__ int2 released(const PagedRelease& a, int b) {
  return make_int2(a.first ? release_first(a.first[b], a.max_pages) : 0, release_end(a.to[b], a.max_pages));
}

__global__ void __launch_bounds__(kReleaseThreads) k_paged_release_count(PagedRelease a) {
  __shared__ int sums[kReleaseThreads / 64];
  const int b = blockIdx.x, tid = threadIdx.x;
  const int2 r = released(a, b);
  const int* row = a.table + (size_t)b * a.max_pages;
  int n = 0;
  for (int j = r.x + tid; j < r.y; j += kReleaseThreads) n += row[j] >= 0;
  n = wave_scan(n);
  if ((tid & 63) == 63) sums[tid >> 6] = n;
  __syncthreads();
  if (tid == 0) {
    a.ws[b] = sums[0] + sums[1] + sums[2] + sums[3];
    if (b == 0) a.ws[a.batch] = max(0, min(a.num_free[0], a.capacity));
  }
}

__global__ void __launch_bounds__(kReleaseThreads) k_paged_release(PagedRelease a) {
  __shared__ int sums[2][kReleaseThreads / 64], counts[kReleaseThreads / 64];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int before = 0, all = 0;
  for (int i = tid; i < a.batch; i += kReleaseThreads) {
    const int n = a.ws[i];
    all += n;
    if (i < b) before += n;
  }
  before = wave_scan(before);
  all = wave_scan(all);
  if (lane == 63) {
    sums[0][wave] = before;
    sums[1][wave] = all;
  }
  __syncthreads();
  before = all = 0;
#pragma unroll
  for (int w = 0; w < kReleaseThreads / 64; ++w) {
    before += sums[0][w];
    all += sums[1][w];
  }
  const int top = a.ws[a.batch];
  const int2 r = released(a, b);
  const int* row = a.table + (size_t)b * a.max_pages;
  for (int j0 = r.x; j0 < r.y; j0 += kReleaseThreads) {
    const int j = j0 + tid, page = j < r.y ? row[j] : -1;
    const unsigned long long who = __builtin_amdgcn_ballot_w64(page >= 0);
    if (lane == 0) counts[wave] = __popcll(who);
    __syncthreads();
    int rank = before + __popcll(who & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < kReleaseThreads / 64; ++w) {
      if (w < wave) rank += counts[w];
      before += counts[w];
    }
    const long to = (long)top + all - 1 - rank;
    if (page >= 0 && to < a.capacity) a.free[to] = page;
    __syncthreads();
  }
  if (b == 0 && tid == 0) a.out_free[0] = (int)min((long)a.capacity, (long)top + all);
}

// Few places in all: one workgroup reads them once, the entries in registers.  32 rows of
// 128: 3.4 us, a call 7.5 to 8.3 (by two kernels 10.1 to 10.8); more do not fit its
// registers.
constexpr int kReleaseFew = 4096, kFewThreads = 1024, kFewHeld = kReleaseFew / kFewThreads;

__global__ void __launch_bounds__(kFewThreads) k_paged_release_few(PagedRelease a) {
  constexpr int kWaves = kFewThreads / 64;
  __shared__ int counts[kFewHeld * kWaves];
  static_assert(kFewHeld * kWaves == 64, "a count a lane");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, places = a.batch * a.max_pages;
  const int top = max(0, min(a.num_free[0], a.capacity));
  int page[kFewHeld];
  unsigned long long who[kFewHeld];
#pragma unroll
  for (int u = 0; u < kFewHeld; ++u) {
    const int i = u * kFewThreads + tid, b = i / a.max_pages, place = i - b * a.max_pages;
    page[u] = -1;
    if (i < places) {
      const int2 r = released(a, b);
      const int x = a.table[i];
      if (place >= r.x && place < r.y) page[u] = x;
    }
    who[u] = __builtin_amdgcn_ballot_w64(page[u] >= 0);
    if (lane == 0) counts[u * kWaves + wave] = __popcll(who[u]);
  }
  __syncthreads();
  const int mine = counts[lane], upto = wave_scan(mine), all = __builtin_amdgcn_readlane(upto, 63);
#pragma unroll
  for (int u = 0; u < kFewHeld; ++u) {
    const int rank = __builtin_amdgcn_readlane(upto - mine, u * kWaves + __builtin_amdgcn_readfirstlane(wave)) +
                     __popcll(who[u] & ((1ull << lane) - 1));
    const long to = (long)top + all - 1 - rank;
    if (page[u] >= 0 && to < a.capacity) a.free[to] = page[u];
  }
  __syncthreads();
  if (tid == 0) a.out_free[0] = (int)min((long)a.capacity, (long)top + all);
}

hipError_t launch_paged_release(const PagedRelease& a, hipStream_t st) {
  if ((long)a.batch * a.max_pages <= kReleaseFew) {
    k_paged_release_few<<<dim3(1), kFewThreads, 0, st>>>(a);
    return hipGetLastError();
  }
  k_paged_release_count<<<dim3((unsigned)a.batch), kReleaseThreads, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_paged_release<<<dim3((unsigned)a.batch), kReleaseThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace hifa4
