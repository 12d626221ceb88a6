// Pages of a pool for the caches of requests that come and go (alpaserve_ops.h):
// which pages new tokens lie on, where every packed token goes, and pages given
// back, from lengths that stay on the device.
//
// Sums over the sequences in their order, then work that does not depend on order.
// What they move is nothing; a call is launches and the latency of a few loads and
// barriers.  One workgroup makes the sums: 5 us for 48 sequences, 6 for a thousand, and
// 3 for every further thousand.
#include "ops_common.hpp"

using as_host::fail;

namespace as_ops {

constexpr int kPageThreads = 1024, kPageWaves = kPageThreads / 64;
constexpr int32_t kRefused = INT32_MIN;

// Sums over the workgroup's threads before this one; total: of all.
__device__ __forceinline__ int64_t sum_before(int64_t x, int64_t* waves, int64_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t upto = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(upto, o);
    if (lane >= o) upto += y;
  }
  lds_barrier();
  if (lane == 63) waves[wave] = upto;
  lds_barrier();
  int64_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPageWaves; ++w) {
    if (w < wave) before += waves[w];
    total += waves[w];
  }
  return before + upto - x;
}

// Slots of a page, 32 m of them, and what quotients by m follow from: n / m is the
// upper half of n ceil(2^32 / m), exact for n (m - 1) < 2^32, and n is below
// 2^25 + 127 here and m at most 128.  (A division takes some 30 instructions; one
// workgroup makes all of them.)
struct Page {
  int32_t slots, blocks;
  uint64_t inverse;
};
__device__ __forceinline__ int page_at(const Page& p, int slot) { return (int)((uint32_t)(slot >> 5) * p.inverse >> 32); }
__device__ __forceinline__ int pages_of(const Page& p, int64_t tokens) {  // tokens: at most 2^30
  return (int)((uint32_t)(((int)tokens + 31 >> 5) + p.blocks - 1) * p.inverse >> 32);
}

struct ReserveArgs {
  const int32_t *stack, *count, *length, *add;
  int32_t *new_count, *new_length, *table, *offsets, *seq, *slot;
  int32_t* base;  // [n_seqs] place in the stack of a sequence's first new page; [n_seqs] its length before
  int32_t n_pages, n_seqs, max_pages, n_tokens;
  Page page;
};

// What every sequence needs and gets, in their order.  One workgroup.
__device__ __forceinline__ void reserve_scan(const ReserveArgs& p, int32_t* offsets, int32_t* base, int32_t* lengths) {
  __shared__ int64_t waves[kPageWaves];
  __shared__ int32_t taken;
  const int tid = threadIdx.x;
  const int64_t count = min(max(p.count[0], 0), p.n_pages), cap = (int64_t)p.max_pages * p.page.slots;
  if (tid == 0) taken = 0;
  int64_t tokens = 0, pages = 0;  // of the sequences before this run of them
  for (int first = 0; first < p.n_seqs; first += kPageThreads) {
    const int b = first + tid;
    const bool there = b < p.n_seqs;
    const int64_t length = there ? min((int64_t)max(p.length[b], 0), cap) : 0;
    const int64_t add = there ? max(p.add[b], 0) : 0;
    int64_t total;
    const int64_t at = tokens + sum_before(add, waves, total);
    tokens += total;
    const bool room = length + add <= cap && at + add <= p.n_tokens;
    const int64_t need = add && room ? pages_of(p.page, length + add) - pages_of(p.page, length) : 0;
    const int64_t upto = pages + sum_before(need, waves, total) + need;
    pages += total;
    const bool fits = (add == 0 || room) && (need == 0 || upto <= count);
    if (there) {
      offsets[b] = (int32_t)min(at, (int64_t)p.n_tokens);
      p.new_length[b] = (int32_t)(fits ? length + add : length);
      lengths[b] = (int32_t)length;
      base[b] = fits ? (int32_t)(count - 1 - (upto - need)) : kRefused;
      if (fits && need) atomicMax(&taken, (int32_t)upto);
    }
  }
  lds_barrier();
  if (tid == 0) {
    offsets[p.n_seqs] = (int32_t)min(tokens, (int64_t)p.n_tokens);
    p.new_count[0] = (int32_t)count - taken;
  }
}

// A packed token's sequence and slot; the token that begins a page writes it into
// the table.
__device__ __forceinline__ void reserve_fill(const ReserveArgs& p, const int32_t* offsets, const int32_t* base,
                                             const int32_t* lengths, int t) {
  int32_t seq = -1, slot = -1;
  if (t < offsets[p.n_seqs]) {
    int lo = 0, hi = p.n_seqs - 1;  // the first sequence that ends behind t
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (offsets[mid + 1] > t)
        hi = mid;
      else
        lo = mid + 1;
    }
    const int from = base[lo];
    if (from != kRefused) {
      const int length = lengths[lo];
      seq = lo;
      slot = length + (t - offsets[lo]);
      const int index = page_at(p.page, slot);
      if (index * p.page.slots == slot)
        p.table[(int64_t)lo * p.max_pages + index] = p.stack[from - (index - pages_of(p.page, length))];
    }
  }
  p.seq[t] = seq;
  p.slot[t] = slot;
}

__global__ __launch_bounds__(kPageThreads) void reserve_sequences(ReserveArgs p) {
  reserve_scan(p, p.offsets, p.base, p.base + p.n_seqs);
}

__global__ __launch_bounds__(256) void reserve_tokens(ReserveArgs p) {
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (t < p.n_tokens) reserve_fill(p, p.offsets, p.base, p.base + p.n_seqs, (int)t);
}

// Few sequences and tokens: both in one launch, what lies between in LDS.  In one
// launch and in two, on the device and for a call in a loop: 48 sequences of a token
// 4.8 and 5.9 us, 9 and 12; 4800 tokens 9.0 and 8.5, 9 and 12; 8000 of 1000 sequences
// 12.4 and 9.4, 12 and 12 (one workgroup's searches).
constexpr int kOnceSeqs = kPageThreads, kOnceTokens = 4 * kPageThreads;

__global__ __launch_bounds__(kPageThreads) void reserve_once(ReserveArgs p) {
  __shared__ int32_t offsets[kOnceSeqs + 1], base[kOnceSeqs], lengths[kOnceSeqs];
  reserve_scan(p, offsets, base, lengths);
  lds_barrier();
  for (int b = threadIdx.x; b <= p.n_seqs; b += kPageThreads) p.offsets[b] = offsets[b];
  for (int t = threadIdx.x; t < p.n_tokens; t += kPageThreads) reserve_fill(p, offsets, base, lengths, t);
}

struct ReleaseArgs {
  int32_t* stack;
  const int32_t *count, *table, *length;
  const uint8_t* which;
  int32_t *new_count, *new_length;
  int32_t n_pages, n_seqs, max_pages;
  Page page;
};

// Pages of the sequences that end, in their order, behind the free ones.  One
// workgroup.
__global__ __launch_bounds__(kPageThreads) void release_pages(ReleaseArgs p) {
  __shared__ int64_t waves[kPageWaves];
  __shared__ int32_t begin[kPageThreads];
  const int tid = threadIdx.x;
  const int64_t count = min(max(p.count[0], 0), p.n_pages), cap = (int64_t)p.max_pages * p.page.slots;
  int64_t at = count;
  for (int first = 0; first < p.n_seqs; first += kPageThreads) {
    const int b = first + tid;
    const bool there = b < p.n_seqs, ends = there && p.which[b] != 0;
    const int64_t length = there ? min((int64_t)max(p.length[b], 0), cap) : 0;
    const int64_t pages = ends ? pages_of(p.page, length) : 0;
    int64_t total;
    const int64_t before = sum_before(pages, waves, total);
    // more pages than the pool has: lengths that no reservation gave
    const int64_t room = max((int64_t)0, min(total, (int64_t)p.n_pages - at));
    begin[tid] = (int32_t)min(before, room);
    if (there) p.new_length[b] = ends ? 0 : (int32_t)length;
    lds_barrier();
    for (int64_t i = tid; i < room; i += kPageThreads) {
      int lo = 0, hi = kPageThreads - 1;  // the last sequence that begins at or before i
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (begin[mid] <= i)
          lo = mid;
        else
          hi = mid - 1;
      }
      p.stack[at + i] = p.table[(int64_t)(first + lo) * p.max_pages + (i - begin[lo])];
    }
    at += room;
  }
  lds_barrier();
  if (tid == 0) p.new_count[0] = (int32_t)at;
}

Page page_args(int32_t page) {
  const int32_t blocks = page / 32;
  return {page, blocks, ((uint64_t(1) << 32) + blocks - 1) / blocks};
}

// Sizes of both calls.
int check_pages(const char* name, int32_t n_pages, int32_t n_seqs, int32_t max_pages, int32_t page) {
  if (n_pages < 0 || n_seqs < 0 || max_pages < 0)
    return fail(AS_E_INVALID_ARG, "%s: %d pages, %d sequences of %d pages", name, n_pages, n_seqs, max_pages);
  if (page < 32 || page > 4096 || page % 32)
    return fail(AS_E_LIMITS, "%s: pages of %d slots (a multiple of 32, at most 4096)", name, page);
  if ((int64_t)max_pages * page > (1 << 30))
    return fail(AS_E_LIMITS, "%s: sequences of %lld slots (at most 2^30)", name, (long long)max_pages * page);
  if (n_seqs > (1 << 20)) return fail(AS_E_LIMITS, "%s: %d sequences (at most 2^20)", name, n_seqs);
  return AS_OK;
}

}  // namespace as_ops

using namespace as_ops;

extern "C" {

int64_t as_pages_reserve_workspace(int32_t n_seqs) { return n_seqs > 0 ? round_up((int64_t)n_seqs * 8, 256) : 0; }

int as_pages_reserve(const int32_t* stack, const int32_t* count, int32_t n_pages, int32_t* page_table, int32_t n_seqs,
                     int32_t max_pages, int32_t page, const int32_t* length, const int32_t* add, int64_t n_tokens,
                     int32_t* new_count, int32_t* new_length, int32_t* offsets, int32_t* seq, int32_t* slot,
                     void* workspace, int64_t workspace_bytes, void* stream) {
  const int rc = check_pages("pages_reserve", n_pages, n_seqs, max_pages, page);
  if (rc != AS_OK) return rc;
  if (n_tokens < 0) return fail(AS_E_INVALID_ARG, "pages_reserve: %lld tokens", (long long)n_tokens);
  if (n_tokens > (1 << 30)) return fail(AS_E_LIMITS, "pages_reserve: %lld tokens (at most 2^30)", (long long)n_tokens);
  if (!count || !new_count || !offsets || (n_pages && !stack) || (n_tokens && (!seq || !slot)) ||
      (n_seqs && (!length || !add || !new_length || (max_pages && !page_table))))
    return fail(AS_E_INVALID_ARG, "pages_reserve: null pointer");
  const int64_t need = as_pages_reserve_workspace(n_seqs);
  if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 256))))
    return fail(AS_E_INVALID_ARG, "pages_reserve: workspace of %lld bytes, %lld needed (aligned to 256)",
                (long long)workspace_bytes, (long long)need);
  const ReserveArgs p{stack,  count, length,     add,
                      new_count, new_length, page_table, offsets, seq, slot,
                      reinterpret_cast<int32_t*>(workspace),
                      n_pages, n_seqs, max_pages, (int32_t)n_tokens, page_args(page)};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (n_seqs <= kOnceSeqs && n_tokens <= kOnceTokens) {
    hipLaunchKernelGGL(reserve_once, dim3(1), dim3(kPageThreads), 0, s, p);
    return launched("pages_reserve");
  }
  hipLaunchKernelGGL(reserve_sequences, dim3(1), dim3(kPageThreads), 0, s, p);
  if (n_tokens) hipLaunchKernelGGL(reserve_tokens, dim3((unsigned)((n_tokens + 255) / 256)), dim3(256), 0, s, p);
  return launched("pages_reserve");
}

int as_pages_release(int32_t* stack, const int32_t* count, int32_t n_pages, const int32_t* page_table, int32_t n_seqs,
                     int32_t max_pages, int32_t page, const int32_t* length, const uint8_t* which, int32_t* new_count,
                     int32_t* new_length, void* stream) {
  const int rc = check_pages("pages_release", n_pages, n_seqs, max_pages, page);
  if (rc != AS_OK) return rc;
  if (!count || !new_count || (n_pages && !stack) ||
      (n_seqs && (!length || !which || !new_length || (max_pages && !page_table))))
    return fail(AS_E_INVALID_ARG, "pages_release: null pointer");
  const ReleaseArgs p{stack, count, page_table, length, which, new_count, new_length, n_pages, n_seqs, max_pages,
                      page_args(page)};
  hipLaunchKernelGGL(release_pages, dim3(1), dim3(kPageThreads), 0, reinterpret_cast<hipStream_t>(stream), p);
  return launched("pages_release");
}

}  // extern "C"
