// Pages of a pool for the caches of requests that come and go (alpaserve_ops.h):
// which pages new tokens lie on, where every packed token goes, and pages given
// back, from lengths that stay on the device.
//
// Sums over the sequences in their order, then work that does not depend on order.
// What they move is nothing; a call is launches and the latency of a few loads and
// barriers.  One workgroup makes the sums: 3.2 us for 48 sequences, 4.1 for a thousand.
#include "ops_common.hpp"

using as_host::fail;

namespace as_ops {

constexpr int kPageThreads = 1024, kPageWaves = kPageThreads / 64;
constexpr int32_t kRefused = INT32_MIN;

// Sums that stop at `most` (below 2^31): of as many lanes as rows of 16 or all.
template <bool ROW>
__device__ __forceinline__ uint32_t scan_capped(uint32_t x, uint32_t most) {
#define AS_ADD_DPP(ctrl, rows) \
  x = min(x + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, false), most)
  AS_ADD_DPP(0x111, 0xf);  // row_shr:1
  AS_ADD_DPP(0x112, 0xf);
  AS_ADD_DPP(0x114, 0xf);
  AS_ADD_DPP(0x118, 0xf);
  if (!ROW) {
    AS_ADD_DPP(0x142, 0xa);  // row_bcast:15
    AS_ADD_DPP(0x143, 0xc);  // row_bcast:31
  }
#undef AS_ADD_DPP
  return x;
}

// The sum over the workgroup's threads before this one, at most `most`, as x is;
// total: of all, likewise.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t most, uint32_t* waves, uint32_t& total) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t upto = scan_capped<false>(x, most);
  const uint32_t own = __builtin_amdgcn_update_dpp(0, (int)upto, 0x138, 0xf, 0xf, false);  // of the lane before
  lds_barrier();
  if (lane == 63) waves[wave] = upto;
  lds_barrier();
  const uint32_t all = scan_capped<true>(waves[lane & 15], most);
  total = (uint32_t)__builtin_amdgcn_readlane((int)all, 15);
  return min(own + (wave ? (uint32_t)__builtin_amdgcn_readlane((int)all, wave - 1) : 0u), most);
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

// What every sequence needs and gets, in their order.  One workgroup, a sequence to a
// thread at a time (2, 4 and 8 were slower).  Sums of tokens stop behind n_tokens; those
// of pages are below 2^30 / 32 and one for each sequence.
__device__ __forceinline__ void reserve_scan(const ReserveArgs& p, int32_t* offsets, int32_t* base, int32_t* lengths) {
  __shared__ uint32_t waves[kPageWaves];
  __shared__ int32_t taken;
  const int tid = threadIdx.x;
  const int count = min(max(p.count[0], 0), p.n_pages), cap = p.max_pages * p.page.slots;
  const uint32_t beyond = (uint32_t)p.n_tokens + 1;
  if (tid == 0) taken = 0;
  uint32_t tokens = 0, pages = 0, total;  // of the sequences before this run of them
  int most = 0;                           // pages up to the last sequence that gets any
  for (int b = tid; b - tid < p.n_seqs; b += kPageThreads) {
    const bool there = b < p.n_seqs;
    const int length = there ? min(max(p.length[b], 0), cap) : 0, add = there ? max(p.add[b], 0) : 0;
    const uint32_t more = min((uint32_t)add, beyond), at = min(tokens + sum_before(more, beyond, waves, total), beyond);
    tokens = min(tokens + total, beyond);
    const bool room = (uint32_t)length + (uint32_t)add <= (uint32_t)cap && at + more < beyond;
    const int need = add && room ? pages_of(p.page, length + add) - pages_of(p.page, length) : 0;
    const int before = (int)(pages + sum_before((uint32_t)need, 0x7fffffffu, waves, total));
    pages += total;
    const bool fits = (add == 0 || room) && (need == 0 || before + need <= count);
    if (there) {
      offsets[b] = (int)min(at, (uint32_t)p.n_tokens);
      p.new_length[b] = fits ? length + add : length;
      lengths[b] = length;
      base[b] = fits ? count - 1 - before : kRefused;
      if (fits && need) most = before + need;
    }
  }
  lds_barrier();
  if (most) atomicMax(&taken, most);
  lds_barrier();
  if (tid == 0) {
    offsets[p.n_seqs] = (int)min(tokens, (uint32_t)p.n_tokens);
    p.new_count[0] = count - taken;
  }
}

// The first sequence from lo on that ends behind t: all of lo.. do before n.
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int lo, int n, int64_t t) {
  int hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid + 1] > t)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo;
}

// A packed token's slot, from its sequence's first row, first new page's place in
// the stack and length; the token that begins a page writes it into the table.
__device__ __forceinline__ void reserve_token(const ReserveArgs& p, int t, int seq, int row, int from, int length) {
  int slot = -1;
  if (seq >= 0 && from != kRefused) {
    slot = length + (t - row);
    const int index = page_at(p.page, slot);
    if (index * p.page.slots == slot)
      p.table[(int64_t)seq * p.max_pages + index] = p.stack[from - (index - pages_of(p.page, length))];
  } else {
    seq = -1;
  }
  p.seq[t] = seq;
  p.slot[t] = slot;
}

__global__ __launch_bounds__(kPageThreads) void reserve_sequences(ReserveArgs p) {
  reserve_scan(p, p.offsets, p.base, p.base + p.n_seqs);
}

// A wavefront takes kRun tokens.  It finds the first one's sequence, among 64 places at
// once, and has that and the 63 behind it in registers: a token's own is found among
// those, in memory only where it is none of them.  (A search in memory for every token
// is 11 loads one after the other for 2000 sequences: 2000 of 350 tokens 22.4 us in
// all, so 13.)
constexpr int kRun = 256;
__global__ __launch_bounds__(256) void reserve_tokens(ReserveArgs p) {
  const int lane = threadIdx.x & 63;
  const int64_t t0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * kRun;
  if (t0 >= p.n_tokens) return;
  const int64_t end = p.offsets[p.n_seqs];
  int first = 0;
  for (int n = p.n_seqs; n > 1;) {  // it is one of first..first + n - 1, if any
    const int step = (n + 63) / 64, at = (lane + 1) * step;
    const int before = __popcll(__ballot(at < n && p.offsets[first + min(at, n)] <= t0));
    first += before * step;
    n = min(step, n - before * step);
  }
  const bool any = p.n_seqs > 0;
  const int mine = min(first + lane, p.n_seqs - 1);
  const int row = any ? p.offsets[mine] : 0, stop = any ? p.offsets[mine + 1] : 0;
  const int from = any ? p.base[mine] : kRefused, length = any ? p.base[p.n_seqs + mine] : 0;
  const int last = __builtin_amdgcn_readlane(stop, 63);
  for (int i = 0; i < kRun; i += 64) {  // (all lanes: they read from each other)
    const int64_t t = t0 + i + lane;
    int j = 0;  // sequences in registers that end at or before t
#pragma unroll
    for (int bit = 32; bit; bit >>= 1)
      if (__shfl(stop, j + bit - 1) <= t) j += bit;
    int u = first + j, r = __shfl(row, j), f = __shfl(from, j), l = __shfl(length, j);
    if (t >= p.n_tokens) continue;
    if (t >= last && t < end) {
      u = sequence_of(p.offsets, min(first + 63, p.n_seqs - 1), p.n_seqs, t);
      r = p.offsets[u], f = p.base[u], l = p.base[p.n_seqs + u];
    }
    reserve_token(p, (int)t, t < end ? u : -1, r, f, l);
  }
}

// Few sequences and tokens: both in one launch, what lies between in LDS.  In one
// launch and in two, on the device and for a call in a loop: 48 sequences of a token
// 3.3 and 5.3 us, 9 and 12; 8 of 1000 tokens 7.5 and 7.0, 9 and 12; 1000 of 8 11.1 and
// 7.7 (one workgroup's searches), 11 and 12.  The rule goes by the call: in a replayed
// graph, where the device's time counts, thousands of tokens of many sequences would be
// faster in two.
constexpr int kOnceSeqs = kPageThreads, kOnceTokens = 8 * kPageThreads;

__global__ __launch_bounds__(kPageThreads) void reserve_once(ReserveArgs p) {
  __shared__ int32_t offsets[kOnceSeqs + 1], base[kOnceSeqs], lengths[kOnceSeqs];
  reserve_scan(p, offsets, base, lengths);
  lds_barrier();
  for (int b = threadIdx.x; b <= p.n_seqs; b += kPageThreads) p.offsets[b] = offsets[b];
  for (int t = threadIdx.x; t < p.n_tokens; t += kPageThreads) {
    const int seq = t < offsets[p.n_seqs] ? sequence_of(offsets, 0, p.n_seqs, t) : -1, at = max(seq, 0);
    reserve_token(p, t, seq, offsets[at], base[at], lengths[at]);
  }
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
  __shared__ uint32_t waves[kPageWaves];
  __shared__ int32_t begin[kPageThreads];
  const int tid = threadIdx.x;
  const int cap = p.max_pages * p.page.slots;
  int at = min(max(p.count[0], 0), p.n_pages);
  for (int first = 0; first < p.n_seqs; first += kPageThreads) {
    const int b = first + tid;
    const bool there = b < p.n_seqs, ends = there && p.which[b] != 0;
    const int length = there ? min(max(p.length[b], 0), cap) : 0;
    // more pages than the pool has: lengths that no reservation gave
    const uint32_t most = (uint32_t)(p.n_pages - at), pages = ends ? pages_of(p.page, length) : 0;
    uint32_t room;
    begin[tid] = (int)sum_before(min(pages, most), most, waves, room);
    if (there) p.new_length[b] = ends ? 0 : length;
    lds_barrier();
    // Four pages a thread at a time: their searches' steps, loads and stores do not wait
    // for one another (100 of 2000 sequences with up to 141 pages 9.2 us one by one, so 6.0).
    constexpr int kAtOnce = 4;
    for (uint32_t i0 = tid; i0 < room; i0 += kAtOnce * kPageThreads) {
      int lo[kAtOnce] = {}, page[kAtOnce];  // the last sequence that begins at or before the page
#pragma unroll
      for (int half = kPageThreads / 2; half; half /= 2)
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
          if ((uint32_t)begin[lo[j] + half] <= i0 + j * kPageThreads) lo[j] += half;
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const uint32_t i = i0 + j * kPageThreads;
        page[j] = i < room ? p.table[(int64_t)(first + lo[j]) * p.max_pages + ((int)i - begin[lo[j]])] : 0;
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
        if (i0 + j * kPageThreads < room) p.stack[at + (int)(i0 + j * kPageThreads)] = page[j];
    }
    at += (int)room;
  }
  if (tid == 0) p.new_count[0] = at;
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
  if (n_tokens) hipLaunchKernelGGL(reserve_tokens, dim3((unsigned)((n_tokens + 4 * kRun - 1) / (4 * kRun))),
                                   dim3(256), 0, s, p);
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
