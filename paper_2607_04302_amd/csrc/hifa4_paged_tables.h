// Index arithmetic of the page tables' kernels, which needs nothing of the GPU:
// plain C++ that the kernels, the launcher and a host compiler all accept.
#pragma once

#include <cstdint>

#ifndef HIFA4_HD
#ifdef __HIPCC__
#define HIFA4_HD __host__ __device__ __forceinline__
#else
#define HIFA4_HD inline
#endif
#endif

namespace hifa4 {

// Threads of a workgroup of the fill, and new tokens of one row that it takes.
constexpr int kFillThreads = 256, kFillTokens = 2048;

// Workgroups that a row's new tokens are cut into: one also where there are none, since
// the entries behind the last token are theirs.
HIFA4_HD int extend_chunks(int max_new) { return max_new / kFillTokens + (max_new % kFillTokens != 0 || max_new == 0); }

// The entries behind the last new token, dealt out to every thread of the fill: a
// thread's first one, and how far it is to its next.  In 64 bits: a launch has up to
// 2^32 threads, and the entries up to 2^31 places.
HIFA4_HD int64_t tail_first(int total, uint32_t block, int thread) { return total + (int64_t)block * kFillThreads + thread; }
HIFA4_HD int64_t tail_step(uint32_t blocks) { return (int64_t)blocks * kFillThreads; }

// Where the part of a row's n new tokens ends that begins at i0 < n (n up to 2^31 - 64:
// i0 + kFillTokens may pass 31 bits).
HIFA4_HD int fill_end(int n, int i0) { return n - i0 < kFillTokens ? n : i0 + kFillTokens; }

// The places [first, to) of a row that a release takes, cut to the row: both at most
// max_pages (below 2^25), so that a thread's steps from there stay within 31 bits.
HIFA4_HD int release_first(int first, int max_pages) { return first < 0 ? 0 : first < max_pages ? first : max_pages; }
HIFA4_HD int release_end(int to, int max_pages) { return to < max_pages ? to : max_pages; }

}  // namespace hifa4
