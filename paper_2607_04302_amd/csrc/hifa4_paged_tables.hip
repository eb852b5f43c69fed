// The paged cache's tables: pages dealt out of a stack of free ones and put back.
//
// Row b holds L tokens and gets n more: the places ceil(L/64) .. ceil((L+n)/64) - 1
// of its table need a page.  With u_b the running sum of those over the rows, the
// j-th new page of row b is free[top - 1 - (u_b + j)]: which page goes where follows
// from sums alone, so every workgroup finds its own pages and no order is left to
// chance.  A release is the mirror image: the entry of rank r of T (row by row, place
// by place) goes to free[top + T - 1 - r], so that it undoes an extension.
#include "hifa4_paged.h"

#include <algorithm>

namespace hifa4 {

constexpr int kExtendThreads = 1024, kFillThreads = 256;
// New tokens that one workgroup of the second kernel takes, and up to which (of all
// rows) the first kernel fills everything in by itself.
constexpr int kFillTokens = 2048, kExtendAlone = 4096;

__device__ __forceinline__ int extend_len(const PagedExtend& a, int b) {
  return max(0, min(a.lens[b], a.max_pages * kPage));
}
// Tokens that row b asks for: none where they are more than its table or the launch holds.
__device__ __forceinline__ int extend_asked(const PagedExtend& a, int b, int len) {
  const int n = max(0, a.counts[b]);
  return n <= min(a.max_new, a.max_pages * kPage - len) ? n : 0;
}
__device__ __forceinline__ int pages_in(int tokens) { return (tokens + kPage - 1) / kPage; }

// One new token of row b: i-th of the row, t-th of all, `len` tokens before them;
// the row's first new page is the one below stack place `top`.
__device__ __forceinline__ void place_token(const PagedExtend& a, int b, int len, int i, int t, int top) {
  const int at = len + i, place = at / kPage, have = pages_in(len);
  int* entry = a.table + (size_t)b * a.max_pages + place;
  const int page = place < have ? *entry : a.free[top - 1 - (place - have)];
  if (place >= have && (i == 0 || at % kPage == 0)) *entry = page;
  a.positions[t] = at + (a.shift ? a.shift[b] : 0);
  a.slots[t] = page < 0 ? -1 : (int64_t)page * kPage + at % kPage;
}

// Sums over the workgroup's threads before this one, and over all (64 bits: 2^30
// pages of 64 tokens).
struct Sums {
  long tokens, pages;
};
__device__ __forceinline__ Sums scan_sums(Sums x, Sums* waves, Sums& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Sums s = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long t = __shfl_up(s.tokens, d), p = __shfl_up(s.pages, d);
    if (lane >= d) {
      s.tokens += t;
      s.pages += p;
    }
  }
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
  for (int b0 = 0; b0 < a.batch; b0 += kExtendThreads) {
    const int b = b0 + tid;
    const bool there = b < a.batch;
    const int len = there ? extend_len(a, b) : 0, asked = there ? extend_asked(a, b, len) : 0;
    const int need = pages_in(len + asked) - pages_in(len);
    Sums all;
    const Sums before = scan_sums(Sums{asked, need}, waves, all);
    const bool fits = upto.tokens + before.tokens + asked <= a.max_total &&
                      (need == 0 || upto.pages + before.pages + need <= top);
    const int n = fits ? asked : 0, pages = fits ? need : 0;
    Sums got;
    const Sums mine = scan_sums(Sums{n, pages}, waves, got);
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
  for (int t = tid; t < a.max_total; t += kExtendThreads) {
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
    place_token(a, b, lens[b], t - first[b], t, stacks[b]);
  }
}

// Pages, positions and slots of up to kFillTokens new tokens of one row.
__global__ void __launch_bounds__(kFillThreads) k_paged_extend_fill(PagedExtend a, int chunks) {
  __shared__ int sums[2][kFillThreads / 64];
  const int b = blockIdx.x / chunks, i0 = blockIdx.x % chunks * kFillTokens, tid = threadIdx.x;
  const int total = a.cu[a.batch];
  for (int t = total + blockIdx.x * kFillThreads + tid; t < a.max_total; t += gridDim.x * kFillThreads) {
    a.positions[t] = -1;
    a.slots[t] = -1;
  }
  const int t0 = a.cu[b], n = a.cu[b + 1] - t0;
  if (i0 >= n) return;
  // pages that the rows before this one took, and all rows: what is left says where the stack began
  int before = 0, all = 0;
  for (int r = tid; r < a.batch; r += kFillThreads) {
    const int len = a.out_lens[r], pages = pages_in(len) - pages_in(len - (a.cu[r + 1] - a.cu[r]));
    all += pages;
    if (r < b) before += pages;
  }
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
  const int len = a.out_lens[b] - n, stack = a.out_free[0] + all - before;
  const int end = min(n, i0 + kFillTokens);
  for (int i = i0 + tid; i < end; i += kFillThreads) place_token(a, b, len, i, t0 + i, stack);
}

hipError_t launch_paged_extend(const PagedExtend& a, hipStream_t st) {
  if (a.max_total <= kExtendAlone && a.batch <= kExtendThreads) {
    k_paged_extend<true><<<dim3(1), kExtendThreads, 0, st>>>(a);
    return hipGetLastError();
  }
  k_paged_extend<false><<<dim3(1), kExtendThreads, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int chunks = extend_chunks(a.max_new);
  k_paged_extend_fill<<<dim3((unsigned)(a.batch * chunks)), kFillThreads, 0, st>>>(a, chunks);
  return hipGetLastError();
}

int extend_chunks(int max_new) { return max_new / kFillTokens + (max_new % kFillTokens != 0); }

// ---------------------------------------------------------------------------
// Release: the rows' entries are counted, then placed by their rank.
constexpr int kReleaseThreads = 256;

__device__ __forceinline__ int2 released(const PagedRelease& a, int b) {
  const int from = a.first ? max(0, a.first[b]) : 0;
  return make_int2(from, min(a.to[b], a.max_pages));
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

hipError_t launch_paged_release(const PagedRelease& a, hipStream_t st) {
  k_paged_release_count<<<dim3((unsigned)a.batch), kReleaseThreads, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_paged_release<<<dim3((unsigned)a.batch), kReleaseThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace hifa4
