// The 4-bit cache of a served model (alpaserve_ops.h): checks, appending a
// step's tokens, and cutting it to a budget by accumulated attention weight.
#include "ops_common.hpp"

using as_host::fail;

namespace as_ops {

int check_cache(const as_cache_t* c, const char* name, bool need_pos, bool need_acc) {
  if (!c) return fail(AS_E_INVALID_ARG, "%s: null cache", name);
  if (c->dim != 64 && c->dim != 128) return fail(AS_E_LIMITS, "%s: heads of %d channels (64 or 128)", name, c->dim);
  if ((c->group != 32 && c->group != 64 && c->group != 128) || c->group > c->dim)
    return fail(AS_E_LIMITS, "%s: %d channels to a scale (32, 64 or 128, at most the head's %d)", name, c->group,
                c->dim);
  if (c->page < 32 || c->page > 4096 || c->page % 32)
    return fail(AS_E_LIMITS, "%s: pages of %d slots (a multiple of 32, at most 4096)", name, c->page);
  if (c->n_heads < 1 || c->n_heads > 1024) return fail(AS_E_LIMITS, "%s: %d heads (1 to 1024)", name, c->n_heads);
  if (c->n_pages < 0 || c->n_seqs < 0 || c->max_pages < 0 || c->reserved != 0)
    return fail(AS_E_INVALID_ARG, "%s: %d pages, %d sequences of %d pages, reserved %d", name, c->n_pages, c->n_seqs,
                c->max_pages, c->reserved);
  if ((int64_t)c->max_pages * c->page > (1 << 30))
    return fail(AS_E_LIMITS, "%s: sequences of %lld slots (at most 2^30)", name, (long long)c->max_pages * c->page);
  if ((int64_t)c->n_seqs * c->n_heads > (1 << 20))
    return fail(AS_E_LIMITS, "%s: %d sequences of %d heads (at most 2^20 in all)", name, c->n_seqs, c->n_heads);
  if (c->n_seqs == 0) return AS_OK;
  if (c->max_pages > 0 && !c->page_table) return fail(AS_E_INVALID_ARG, "%s: null page table", name);
  if (c->n_pages > 0 && (!c->k || !c->v || !c->k_par || !c->v_par))
    return fail(AS_E_INVALID_ARG, "%s: null codes or scales", name);
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_par, 16) || !aligned(c->v_par, 16))
    return fail(AS_E_INVALID_ARG, "%s: codes and scales have to be aligned to 16 bytes", name);
  if (c->n_pages > 0 && ((need_pos && !c->pos) || (need_acc && !c->acc)))
    return fail(AS_E_INVALID_ARG, "%s: positions and accumulated weights are needed", name);
  return AS_OK;
}

CacheArgs cache_args(const as_cache_t* c) {
  return CacheArgs{c->k,       c->v,       reinterpret_cast<uint32_t*>(c->k_par), reinterpret_cast<uint32_t*>(c->v_par),
                   c->pos,     c->acc,     c->page_table,
                   c->n_pages, c->n_heads, c->dim,
                   c->group,   c->page,    c->n_seqs,
                   c->max_pages};
}

// ------------------------------------------------------------------- append

struct AppendArgs {
  CacheArgs c;
  const uint16_t *k, *v;
  int64_t k_seq, k_token, v_seq, v_token;
  const int32_t *start, *first_pos;
  float *held_k, *held_v;
  int32_t n_tokens;
};

// Bits of element e of a word.
__device__ __forceinline__ int nibble(int e) { return 4 * ((e >> 1) + 4 * (e & 1)); }

// One workgroup per (sequence, head, block of 32 slots).  DIM/8 lanes quantise
// a token's key or value, 8 channels each: a word of K as it is; V's codes
// change direction (a word holds 8 tokens of one channel), through LDS, and a
// word that keeps older tokens is read first.  No other workgroup has this
// block's words, so nothing races.  Latency bounds a step of one token: 5.6 us
// for 40 sequences of 8 heads, a load that depends on two others and a store.
template <int TYPE, int DIM, int GROUP>
__global__ __launch_bounds__(256) void append(AppendArgs p) {
  constexpr int kLanes = DIM / 8;       // lanes of one token's key or value
  constexpr int kShare = GROUP / 8;     // of them, those that share a scale
  constexpr int kWords = DIM / 8;
  __shared__ v2u v_codes[32][kLanes];   // a byte per channel
  const int b = blockIdx.y / p.c.n_heads, h = blockIdx.y % p.c.n_heads;
  const int64_t cap = (int64_t)p.c.max_pages * p.c.page;
  const int64_t start = p.start[b];
  const int64_t first = (start >> 5) * 32 + (int64_t)blockIdx.x * 32;  // the block's first slot
  if (first >= start + p.n_tokens || first + 32 <= 0 || first >= cap) return;
  const int64_t row = cache_row(p.c, b, h, (int)(first / p.c.page));
  if (row < 0) return;
  const int in_page = (int)(first % p.c.page);
  const int lane = threadIdx.x % kLanes;
  // the block's new slots
  const int lo = (int)max((int64_t)0, start - first);
  const int hi = (int)min((int64_t)32, start + p.n_tokens - first);
  for (int j = threadIdx.x / kLanes; j < 2 * (hi - lo); j += 256 / kLanes) {
    const bool is_v = j >= hi - lo;
    const int s = lo + (is_v ? j - (hi - lo) : j);
    const int64_t t = first + s - start;
    const uint16_t* x = (is_v ? p.v + b * p.v_seq + t * p.v_token : p.k + b * p.k_seq + t * p.k_token) +
                        (int64_t)h * DIM + lane * 8;
    float f[8];
    float low = kInf, high = -kInf;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      f[e] = to_f32<TYPE>(x[e]);
      bad |= f[e] != f[e];
      f[e] = fminf(fmaxf(f[e], -65504.0f), 65504.0f);
      low = fminf(low, f[e]);
      high = fmaxf(high, f[e]);
    }
    int any = bad;
#pragma unroll
    for (int o = 1; o < kShare; o <<= 1) {
      low = fminf(low, __shfl_xor(low, o));
      high = fmaxf(high, __shfl_xor(high, o));
      any |= __shfl_xor(any, o);
    }
    const _Float16 base = any ? (_Float16)__builtin_nanf("") : (_Float16)low;
    const _Float16 step = any ? (_Float16)__builtin_nanf("") : (_Float16)((high - low) / 15.0f);
    const float m = (float)base, d = (float)step;
    uint32_t word = 0, bytes[2] = {0, 0};
    float* held = is_v ? p.held_v : p.held_k;
    if (held) held += (((int64_t)b * p.n_tokens + t) * p.c.n_heads + h) * DIM + lane * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // x - m is exact for 16-bit x and m of like size, so the quotient rounds
      // as in exact arithmetic
      const float q = rintf((f[e] - m) / d);
      const uint32_t code = d > 0.0f ? (uint32_t)fminf(fmaxf(q, 0.0f), 15.0f) : 0u;
      word |= code << nibble(e);
      bytes[e >> 2] |= code << (8 * (e & 3));
      if (held) held[e] = (float)code * d + m;
    }
    const int at = in_page + s;
    if (is_v) {
      v_codes[s][lane] = v2u{bytes[0], bytes[1]};
    } else {
      // channels 8 lane..: word [g = lane%4][i = lane/4] of the token
      p.c.k[(row * p.c.page + at) * kWords + (lane & 3) * (DIM / 32) + (lane >> 2)] = word;
    }
    if (lane % kShare == 0) {
      uint32_t* par = is_v ? p.c.v_par : p.c.k_par;
      par[(row * (DIM / GROUP) + lane / kShare) * p.c.page + at] =
          (uint32_t)__builtin_bit_cast(uint16_t, step) | (uint32_t)__builtin_bit_cast(uint16_t, base) << 16;
    }
    if (is_v && lane == 0) {
      if (p.c.pos) p.c.pos[row * p.c.page + at] = (int32_t)(p.first_pos ? p.first_pos[b] + t : first + s);
      if (p.c.acc) p.c.acc[row * p.c.page + at] = 0.0f;
    }
  }
  __syncthreads();
  const uint8_t* codes = reinterpret_cast<const uint8_t*>(v_codes);
  uint32_t* v = p.c.v + (row * p.c.page + in_page) * kWords;
  for (int w = threadIdx.x; w < 32 * kWords; w += 256) {
    const int i = w % (DIM / 16), c = w / (DIM / 16) % 16, g = w / DIM;
    uint32_t mask = 0, word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int s = 16 * (e >> 2) + 4 * g + (e & 3);
      if (s >= lo && s < hi) {
        word |= (uint32_t)codes[s * DIM + 16 * i + c] << nibble(e);
        mask |= 15u << nibble(e);
      }
    }
    if (mask == 0xffffffffu)
      v[w] = word;
    else if (mask)
      v[w] = (v[w] & ~mask) | word;
  }
}

template <int TYPE>
void launch_append(const AppendArgs& p, hipStream_t s) {
  const dim3 g((unsigned)((p.n_tokens + 31) / 32 + 1), (unsigned)(p.c.n_seqs * p.c.n_heads)), t(256);
  if (p.c.dim == 64 && p.c.group == 32) hipLaunchKernelGGL((append<TYPE, 64, 32>), g, t, 0, s, p);
  if (p.c.dim == 64 && p.c.group == 64) hipLaunchKernelGGL((append<TYPE, 64, 64>), g, t, 0, s, p);
  if (p.c.dim == 128 && p.c.group == 32) hipLaunchKernelGGL((append<TYPE, 128, 32>), g, t, 0, s, p);
  if (p.c.dim == 128 && p.c.group == 64) hipLaunchKernelGGL((append<TYPE, 128, 64>), g, t, 0, s, p);
  if (p.c.dim == 128 && p.c.group == 128) hipLaunchKernelGGL((append<TYPE, 128, 128>), g, t, 0, s, p);
}

// ----------------------------------------------------------------- eviction

struct EvictArgs {
  CacheArgs src, dst;
  const int32_t *length, *total;
  int32_t* out_length;
  int32_t* kept;  // [n_seqs * n_heads][keep] slots of src
  int32_t keep, recent;
  uint32_t src_mul, dst_mul;  // page_magic of the caches' pages
  bool vec;                   // src.pos and src.acc aligned to 16 bytes
};

// Order of a token among those to keep: the newest positions first, then by
// weight; NaN last, and -0 as 0.
__device__ __forceinline__ uint32_t order_key(int pos, float acc, int newest) {
  const uint32_t u = __float_as_uint(acc + 0.0f);
  uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);  // all bits of a negative number, else the sign
  k = acc != acc ? 0u : k;
  return pos >= newest ? 0xffffffffu : k;
}

__device__ __forceinline__ int evict_length(const EvictArgs& p, int b) {
  const int64_t cap = (int64_t)p.src.max_pages * p.src.page;
  return (int)max((int64_t)0, min((int64_t)p.length[b], cap));
}

// Which slots stay, one workgroup per (sequence, head).  The keys are read once
// and stay in registers, four neighbouring slots to a thread (sequences longer
// than the registers are read again in every step).  The keep-th largest key is
// found by three rounds of 11, 11 and 10 bits: a histogram in LDS of the keys
// that agree with the digits found so far, and a sum over its bins from the
// top.  11 bits hold an fp32 number's sign, exponent and two more bits: weights
// that spread over powers of two spread over the bins, so few lanes add to the
// same one.  Then every slot above the key, and as many equal ones as there is
// room for, lowest slot first, is written at its place, which the counts of the
// wavefronts before it give.  Bound by the rounds' latency, barriers and LDS
// atomics: 10 us for 1300 tokens, 37 us for 65,000.
constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;

// Exclusive sum over the workgroup of one number a thread; total: of all.
__device__ __forceinline__ uint32_t scan_threads(uint32_t x, uint32_t* waves, uint32_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t sum = scan_lanes(x);
  __syncthreads();
  if (lane == 63) waves[wave] = sum;
  __syncthreads();
  uint32_t before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) {
    if (w < wave) before += waves[w];
    total += waves[w];
  }
  return before + sum - x;
}

template <int QUADS>
__global__ __launch_bounds__(kSelThreads) void evict_select(EvictArgs p) {
  constexpr int kSeg = QUADS * 4 * kSelThreads;  // slots that the registers hold
  __shared__ uint32_t hist[2048];
  __shared__ uint32_t waves[kSelWaves];
  __shared__ uint32_t found[2];  // digit, keys still to take among those that have it
  __shared__ uint32_t sums[2][QUADS * kSelWaves];
  const int b = blockIdx.x / p.src.n_heads, h = blockIdx.x % p.src.n_heads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = evict_length(p, b);
  if (h == 0 && tid == 0) p.out_length[b] = min(n, p.keep);
  int32_t* kept = p.kept + (int64_t)blockIdx.x * p.keep;
  if (n <= p.keep) {
    for (int s = tid; s < n; s += kSelThreads) kept[s] = s;
    return;
  }
  const int newest = p.total[b] - p.recent;
  const int segs = (n + kSeg - 1) / kSeg;
  uint32_t key[QUADS][4];
  // Slots seg * kSeg + (j * threads + tid) * 4 + e.  Those beyond n get the
  // lowest key, 0; they are never kept: more than `keep` slots before them are
  // at least as high, and equal ones are taken from the lowest slot up.
  // A slot without a page reads the pool's first one and gets key 0 too.
  auto load = [&](int seg) {
    if (p.src.n_pages == 0) {
#pragma unroll
      for (int j = 0; j < QUADS; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) key[j][e] = 0;
      return;
    }
    const int32_t* table = p.src.page_table + (int64_t)b * p.src.max_pages;
    int page[QUADS];
#pragma unroll
    for (int j = 0; j < QUADS; ++j) {
      const int s = min(seg * kSeg + (j * kSelThreads + tid) * 4, n - 1);
      page[j] = table[page_index(s >> 5, p.src_mul)];
    }
    __builtin_amdgcn_sched_barrier(0);
    constexpr int kBatch = QUADS < 4 ? QUADS : 4;  // loads in flight: two a quad
#pragma unroll
    for (int j0 = 0; j0 < QUADS; j0 += kBatch) {
      v4i pos[kBatch];
      v4f acc[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int s = min(seg * kSeg + ((j0 + j) * kSelThreads + tid) * 4, (n - 1) & ~3);
        const int64_t row = (unsigned)page[j0 + j] < (unsigned)p.src.n_pages ? (int64_t)page[j0 + j] * p.src.n_heads + h : h;
        const int64_t i = row * p.src.page + s - page_index(s >> 5, p.src_mul) * p.src.page;
        if (p.vec) {
          pos[j] = *reinterpret_cast<const v4i*>(p.src.pos + i);
          acc[j] = *reinterpret_cast<const v4f*>(p.src.acc + i);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) pos[j][e] = p.src.pos[i + e], acc[j][e] = p.src.acc[i + e];
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int s = seg * kSeg + ((j0 + j) * kSelThreads + tid) * 4;
        const bool there = (unsigned)page[j0 + j] < (unsigned)p.src.n_pages;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          key[j0 + j][e] = there && s + e < n ? order_key(pos[j][e], acc[j][e], newest) : 0u;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  uint32_t prefix = 0, want = (uint32_t)p.keep;
#pragma nounroll
  for (int round = 0; round < 3; ++round) {
    const int shift = round == 0 ? 21 : round == 1 ? 10 : 0;
    const uint32_t digits = round == 2 ? 1023u : 2047u;
    const uint32_t known = round == 0 ? 0u : round == 1 ? ~0u << 21 : ~0u << 10;
    for (int i = tid; i < 2048; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int seg = 0; seg < segs; ++seg) {
      if (round == 0 || segs > 1) load(seg);
#pragma unroll
      for (int j = 0; j < QUADS; ++j) {
        if (seg * kSeg + j * 4 * kSelThreads >= n) break;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (((key[j][e] ^ prefix) & known) == 0) atomicAdd(&hist[key[j][e] >> shift & digits], 1u);
      }
    }
    __syncthreads();
    // two bins a thread, from the top
    const int bin = 2047 - 2 * tid;
    const uint32_t c1 = hist[bin], c0 = hist[bin - 1];
    uint32_t all;
    const uint32_t before = scan_threads(c1 + c0, waves, all);
    if (before < want && want <= before + c1 + c0) {
      const bool upper = want <= before + c1;
      found[0] = (uint32_t)(upper ? bin : bin - 1);
      found[1] = want - before - (upper ? 0 : c1);
    }
    __syncthreads();
    prefix |= (uint32_t)__builtin_amdgcn_readfirstlane((int)found[0]) << shift;
    want = (uint32_t)__builtin_amdgcn_readfirstlane((int)found[1]);
  }

  uint32_t base_above = 0, base_equal = 0;
  for (int seg = 0; seg < segs; ++seg) {
    if (segs > 1) load(seg);
    // Counts, keys above the threshold in the low half and equal ones in the
    // high half: of the lanes before in 256 neighbouring slots, then of the
    // wavefronts and quads before.
    uint32_t lanes[QUADS];
#pragma unroll
    for (int j = 0; j < QUADS; ++j) {
      uint32_t c = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) c += (key[j][e] > prefix ? 1u : 0u) + (key[j][e] == prefix ? 0x10000u : 0u);
      const uint32_t sum = scan_lanes(c);
      lanes[j] = sum - c;
      if (lane == 63) sums[0][j * kSelWaves + wave] = sum & 0xffffu, sums[1][j * kSelWaves + wave] = sum >> 16;
      __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
    const uint32_t xa = tid < QUADS * kSelWaves ? sums[0][tid] : 0, xe = tid < QUADS * kSelWaves ? sums[1][tid] : 0;
    uint32_t all_a, all_e;
    const uint32_t sa = scan_threads(xa, waves, all_a);
    const uint32_t se = scan_threads(xe, waves, all_e);
    if (tid < QUADS * kSelWaves) sums[0][tid] = sa, sums[1][tid] = se;
    __syncthreads();
    // (the same number again, so that the compiler compares once more rather
    // than keep the results of all comparisons)
    uint32_t limit = prefix;
    asm volatile("" : "+s"(limit));
#pragma unroll
    for (int j = 0; j < QUADS; ++j) {
      const int s = seg * kSeg + (j * kSelThreads + tid) * 4;
      uint32_t na = base_above + sums[0][j * kSelWaves + wave] + (lanes[j] & 0xffffu);
      uint32_t ne = base_equal + sums[1][j * kSelWaves + wave] + (lanes[j] >> 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool up = key[j][e] > limit, eq = key[j][e] == limit;
        if (up || (eq && ne < want)) kept[na + min(ne, want)] = s + e;
        na += up;
        ne += eq;
      }
    }
    base_above += all_a;
    base_equal += all_e;
    __syncthreads();
  }
}

// The kept tokens to dst, one workgroup per (sequence, head, block of 32 slots
// of dst), everything read before anything is written.  K's words, scales,
// positions and weights move as they are, 16 bytes to a thread; a word of V is
// put together from 8 tokens' nibbles.  A kept token's nibbles lie in words that
// it shares with 7 others, and its scales, position and weight in sectors that
// it shares with 15: where few tokens stay, that is what bounds it (12 sequences
// of 8 heads, 6000 of 20,000 to 65,000 tokens: 83 us for 448 MB of lines, 5.4
// TB/s, of which the kept tokens' own bytes are 175 MB).
template <int DIM>
__global__ __launch_bounds__(256, 4) void evict_move(EvictArgs p) {
  constexpr int kWords = DIM / 8;
  __shared__ int64_t from_row[32];
  __shared__ int from_at[32];
  const int bh = blockIdx.y, b = bh / p.src.n_heads, h = bh % p.src.n_heads, tid = threadIdx.x;
  const int first = blockIdx.x * 32;
  const int count = min(evict_length(p, b), p.keep);
  if (first >= count) return;
  const int to_page = page_index(first >> 5, p.dst_mul), in_page = first - to_page * p.dst.page;
  const int64_t to = cache_row(p.dst, b, h, to_page);
  if (to < 0) return;
  if (tid < 32) {
    int64_t row = -1;
    int at = 0;
    if (first + tid < count) {
      const int s = p.kept[(int64_t)bh * p.keep + first + tid];
      const int pi = page_index(s >> 5, p.src_mul);
      at = s - pi * p.src.page;
      row = cache_row(p.src, b, h, pi);
    }
    from_row[tid] = row;
    from_at[tid] = at;
  }
  __syncthreads();
  if (tid < DIM) {
    // four words of V: channels (c, i) = 4 ci.. of slots 16 (e/4) + 4 g + e%4
    const int g = tid / (DIM / 4), ci = tid % (DIM / 4) * 4;
    v4u x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int s = 16 * (e >> 2) + 4 * g + (e & 3);
      const int64_t row = from_row[s];
      const int at = from_at[s];
      x[e] = v4u{0, 0, 0, 0};
      if (row >= 0)
        x[e] = *reinterpret_cast<const v4u*>(p.src.v + (row * p.src.page + (at & ~31)) * kWords + (at >> 2 & 3) * DIM +
                                             ci);
    }
    v4u word = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int at = from_at[16 * (e >> 2) + 4 * g + (e & 3)] & 31;
      word |= ((x[e] >> nibble(4 * (at >> 4) + (at & 3))) & 15u) << nibble(e);
    }
    *reinterpret_cast<v4u*>(p.dst.v + (to * p.dst.page + in_page) * kWords + g * DIM + ci) = word;
  } else {
    // the other threads: K's words 16 bytes each, then a word of every slot's
    // scales, position and weight
    const int t = tid - DIM, groups = p.src.dim / p.src.group;
    const int others = 256 - DIM;
    for (int i = t; i < 32 * kWords / 4; i += others) {
      const int s = i / (kWords / 4), w = i % (kWords / 4) * 4;
      if (from_row[s] >= 0)
        *reinterpret_cast<v4u*>(p.dst.k + (to * p.dst.page + in_page + s) * kWords + w) =
            *reinterpret_cast<const v4u*>(p.src.k + (from_row[s] * p.src.page + from_at[s]) * kWords + w);
    }
    for (int i = t; i < 32 * (2 * groups + 2); i += others) {
      const int s = i & 31, what = i >> 5, g = what >> 1;
      if (from_row[s] < 0) continue;
      if (g < groups) {
        const int64_t f = (from_row[s] * groups + g) * p.src.page + from_at[s];
        const int64_t o = (to * groups + g) * p.dst.page + in_page + s;
        if (what & 1)
          p.dst.v_par[o] = p.src.v_par[f];
        else
          p.dst.k_par[o] = p.src.k_par[f];
      } else {
        const int64_t f = from_row[s] * p.src.page + from_at[s], o = to * p.dst.page + in_page + s;
        if (what & 1)
          p.dst.acc[o] = p.src.acc[f];
        else
          p.dst.pos[o] = p.src.pos[f];
      }
    }
  }
}

}  // namespace as_ops

using namespace as_ops;

extern "C" {

int as_cache_append(const as_cache_t* cache, const void* k, const void* v, int32_t type, int32_t n_tokens,
                    int64_t k_seq, int64_t k_token, int64_t v_seq, int64_t v_token, const int32_t* start,
                    const int32_t* first_pos, float* held_k, float* held_v, void* stream) {
  const int rc = check_cache(cache, "cache_append", false, false);
  if (rc != AS_OK) return rc;
  if (type != AS_BF16 && type != AS_F16) return fail(AS_E_INVALID_ARG, "cache_append: type %d", type);
  if (n_tokens < 0) return fail(AS_E_INVALID_ARG, "cache_append: %d tokens", n_tokens);
  if (n_tokens > (1 << 24)) return fail(AS_E_LIMITS, "cache_append: %d tokens (at most 2^24)", n_tokens);
  if ((int64_t)cache->n_seqs * cache->n_heads > 65535)
    return fail(AS_E_LIMITS, "cache_append: %d sequences of %d heads (at most 65535 in all)", cache->n_seqs,
                cache->n_heads);
  if (n_tokens == 0 || cache->n_seqs == 0) return as_host::ok();
  if (!k || !v || !start) return fail(AS_E_INVALID_ARG, "cache_append: null pointer");
  const AppendArgs p{cache_args(cache), reinterpret_cast<const uint16_t*>(k), reinterpret_cast<const uint16_t*>(v),
                     k_seq, k_token, v_seq, v_token, start, first_pos, held_k, held_v, n_tokens};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (type == AS_BF16)
    launch_append<AS_BF16>(p, s);
  else
    launch_append<AS_F16>(p, s);
  return launched("cache_append");
}

int64_t as_cache_evict_workspace(const as_cache_t* src, int32_t keep) {
  if (!src || keep < 1 || src->n_seqs < 1 || src->n_heads < 1) return 0;
  return round_up((int64_t)src->n_seqs * src->n_heads * keep * 4, 256);
}

int as_cache_evict(const as_cache_t* src, const as_cache_t* dst, const int32_t* length, const int32_t* total,
                   int32_t keep, int32_t recent, int32_t* out_length, void* workspace, int64_t workspace_bytes,
                   void* stream) {
  int rc = check_cache(src, "cache_evict", true, true);
  if (rc != AS_OK) return rc;
  rc = check_cache(dst, "cache_evict", true, true);
  if (rc != AS_OK) return rc;
  if (src->n_heads != dst->n_heads || src->dim != dst->dim || src->group != dst->group || src->n_seqs != dst->n_seqs)
    return fail(AS_E_INVALID_ARG, "cache_evict: the caches differ in heads, channels or sequences");
  if (keep < 1 || recent < 0 || recent > keep || keep > (int64_t)dst->max_pages * dst->page)
    return fail(AS_E_INVALID_ARG, "cache_evict: keep %d (the destination has room for %lld), recent %d", keep,
                (long long)dst->max_pages * dst->page, recent);
  // a workgroup of 256 for 32 of them, fewer than 2^32 threads a launch
  if (keep > (1 << 29) - 32) return fail(AS_E_LIMITS, "cache_evict: keep %d (at most 2^29 - 32)", keep);
  if ((int64_t)src->n_seqs * src->n_heads > 65535)
    return fail(AS_E_LIMITS, "cache_evict: %d sequences of %d heads (at most 65535 in all)", src->n_seqs,
                src->n_heads);
  if (src->n_seqs == 0) return as_host::ok();
  if (!length || !total || !out_length) return fail(AS_E_INVALID_ARG, "cache_evict: null pointer");
  const uintptr_t out = (uintptr_t)out_length, n = (uintptr_t)src->n_seqs * 4;
  for (const int32_t* read : {length, total})
    if (out < (uintptr_t)read + n && (uintptr_t)read < out + n)
      return fail(AS_E_INVALID_ARG, "cache_evict: out_length overlaps length or total");
  const int64_t need = as_cache_evict_workspace(src, keep);
  if (workspace_bytes < need || !workspace || !aligned(workspace, 256))
    return fail(AS_E_INVALID_ARG, "cache_evict: workspace of %lld bytes, %lld needed (aligned to 256)",
                (long long)workspace_bytes, (long long)need);
  const EvictArgs p{cache_args(src), cache_args(dst), length, total, out_length, reinterpret_cast<int32_t*>(workspace),
                    keep, recent, page_magic(src->page), page_magic(dst->page),
                    aligned(src->pos, 16) && aligned(src->acc, 16)};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const unsigned rows = (unsigned)(src->n_seqs * src->n_heads);
  const int64_t cap = (int64_t)src->max_pages * src->page;
  // registers for the longest sequence that the table has room for
  if (cap <= 4 * kSelThreads)
    hipLaunchKernelGGL((evict_select<1>), dim3(rows), dim3(kSelThreads), 0, s, p);
  else if (cap <= 16 * kSelThreads)
    hipLaunchKernelGGL((evict_select<4>), dim3(rows), dim3(kSelThreads), 0, s, p);
  else
    hipLaunchKernelGGL((evict_select<16>), dim3(rows), dim3(kSelThreads), 0, s, p);
  const dim3 g((unsigned)((keep + 31) / 32), rows);
  if (src->dim == 64)
    hipLaunchKernelGGL((evict_move<64>), g, dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((evict_move<128>), g, dim3(256), 0, s, p);
  return launched("cache_evict");
}

}  // extern "C"
