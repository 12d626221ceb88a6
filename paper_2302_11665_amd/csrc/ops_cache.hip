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
// block's words, so nothing races.  Latency bounds a step of one token.
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
};

constexpr int kSelThreads = 1024;

// Order of a token among those to keep: the newest positions first, then by
// weight; NaN last, and -0 as 0.
__device__ __forceinline__ uint32_t order_key(const EvictArgs& p, int b, int h, int slot, int total) {
  const int64_t row = cache_row(p.src, b, h, slot / p.src.page);
  if (row < 0) return 0;
  const int64_t at = row * p.src.page + slot % p.src.page;
  if (p.src.pos[at] >= total - p.recent) return 0xffffffffu;
  const float a = p.src.acc[at];
  if (a != a) return 0;
  const uint32_t u = __float_as_uint(a + 0.0f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int evict_length(const EvictArgs& p, int b) {
  const int64_t cap = (int64_t)p.src.max_pages * p.src.page;
  return (int)max((int64_t)0, min((int64_t)p.length[b], cap));
}

// Which slots stay, one workgroup per (sequence, head): the keep-th largest key
// by four rounds of 8 bits (a histogram of the keys that agree with the digits
// found so far), then one pass in slot order that writes the slots above it and
// as many equal ones as there is room for, lowest first.
__global__ __launch_bounds__(kSelThreads) void evict_select(EvictArgs p) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t found[2];  // digits found, keys still to take among the equal ones
  __shared__ uint32_t sums[kSelThreads / 64][2];
  const int b = blockIdx.x / p.src.n_heads, h = blockIdx.x % p.src.n_heads;
  const int n = evict_length(p, b);
  if (h == 0 && threadIdx.x == 0) p.out_length[b] = min(n, p.keep);
  int32_t* kept = p.kept + (int64_t)blockIdx.x * p.keep;
  if (n <= p.keep) {
    for (int s = threadIdx.x; s < n; s += kSelThreads) kept[s] = s;
    return;
  }
  const int total = p.total[b];
  uint32_t prefix = 0, want = (uint32_t)p.keep;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (threadIdx.x < 256) hist[threadIdx.x] = 0;
    __syncthreads();
    for (int s = threadIdx.x; s < n; s += kSelThreads) {
      const uint32_t key = order_key(p, b, h, s, total);
      if (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t above = 0;
      int d = 255;
      while (d > 0 && above + hist[d] < want) above += hist[d--];
      found[0] = prefix | (uint32_t)d << shift;
      found[1] = want - above;
    }
    __syncthreads();
    prefix = found[0];
    want = found[1];
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t base = 0, ties = 0;  // slots written, equal keys met
  for (int s0 = 0; s0 < n; s0 += kSelThreads) {
    const int s = s0 + threadIdx.x;
    const uint32_t key = s < n ? order_key(p, b, h, s, total) : 0;
    const bool above = s < n && key > prefix, equal = s < n && key == prefix;
    const uint64_t ma = __ballot(above), me = __ballot(equal);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    __syncthreads();
    if (lane == 0) {
      sums[wave][0] = (uint32_t)__popcll(ma);
      sums[wave][1] = (uint32_t)__popcll(me);
    }
    __syncthreads();
    uint32_t a0 = 0, e0 = 0, a1 = 0, e1 = 0;
#pragma unroll
    for (int w = 0; w < kSelThreads / 64; ++w) {
      if (w < wave) a0 += sums[w][0], e0 += sums[w][1];
      a1 += sums[w][0], e1 += sums[w][1];
    }
    const uint32_t met = ties + e0 + (uint32_t)__popcll(me & below);  // equal keys before this slot
    const uint32_t at = base + a0 + (uint32_t)__popcll(ma & below) + min(met, want) - min(ties, want);
    if (above || (equal && met < want)) kept[at] = s;
    base += a1 + min(ties + e1, want) - min(ties, want);
    ties += e1;
  }
}

// Words of one row (page and head) of a token, by cache_row's index.
__device__ __forceinline__ int64_t token_row(const CacheArgs& c, int b, int h, int slot, int& in_page) {
  in_page = slot % c.page;
  return cache_row(c, b, h, slot / c.page);
}

// The kept tokens to dst, one workgroup per (sequence, head, block of 32 slots
// of dst).  K words, scales, positions and weights move as they are; a word of V
// is put together from 8 tokens' nibbles.
__global__ __launch_bounds__(256) void evict_move(EvictArgs p) {
  __shared__ int64_t from_row[32];
  __shared__ int from_at[32];
  const int bh = blockIdx.y, b = bh / p.src.n_heads, h = bh % p.src.n_heads;
  const int first = blockIdx.x * 32;
  const int count = min(evict_length(p, b), p.keep);
  if (first >= count) return;
  int in_page;
  const int64_t to = token_row(p.dst, b, h, first, in_page);
  if (to < 0) return;
  if (threadIdx.x < 32) {
    const int j = first + threadIdx.x;
    from_row[threadIdx.x] = -1;
    if (j < count) {
      int at;
      from_row[threadIdx.x] = token_row(p.src, b, h, p.kept[(int64_t)bh * p.keep + j], at);
      from_at[threadIdx.x] = at;
    }
  }
  __syncthreads();
  const int words = p.src.dim / 8, groups = p.src.dim / p.src.group;
  for (int w = threadIdx.x; w < 32 * words; w += 256) {
    const int s = w / words, c = w % words;
    if (from_row[s] >= 0)
      p.dst.k[(to * p.dst.page + in_page + s) * words + c] =
          p.src.k[(from_row[s] * p.src.page + from_at[s]) * words + c];
  }
  for (int w = threadIdx.x; w < 32 * groups; w += 256) {
    const int s = w & 31, g = w >> 5;
    if (from_row[s] >= 0) {
      const int64_t i = (from_row[s] * groups + g) * p.src.page + from_at[s];
      const int64_t o = (to * groups + g) * p.dst.page + in_page + s;
      p.dst.k_par[o] = p.src.k_par[i];
      p.dst.v_par[o] = p.src.v_par[i];
    }
  }
  if (threadIdx.x < 32 && from_row[threadIdx.x] >= 0) {
    const int64_t i = from_row[threadIdx.x] * p.src.page + from_at[threadIdx.x];
    const int64_t o = to * p.dst.page + in_page + threadIdx.x;
    p.dst.pos[o] = p.src.pos[i];
    p.dst.acc[o] = p.src.acc[i];
  }
  // a word of V: channel (c, i) of slots 16 (e/4) + 4 g + e%4
  const int dim = p.src.dim;
  for (int w = threadIdx.x; w < 4 * dim; w += 256) {
    const int g = w / dim, ci = w % dim;
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int s = 16 * (e >> 2) + 4 * g + (e & 3);
      if (from_row[s] < 0) continue;
      const int at = from_at[s] & 31;
      const int64_t block = (from_row[s] * p.src.page + (from_at[s] & ~31)) * words;
      const uint32_t x = p.src.v[block + ((at >> 2) & 3) * dim + ci];
      word |= ((x >> nibble(4 * (at >> 4) + (at & 3))) & 15u) << nibble(e);
    }
    p.dst.v[(to * p.dst.page + in_page) * words + w] = word;
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
  if ((int64_t)src->n_seqs * src->n_heads > 65535)
    return fail(AS_E_LIMITS, "cache_evict: %d sequences of %d heads (at most 65535 in all)", src->n_seqs,
                src->n_heads);
  if (src->n_seqs == 0) return as_host::ok();
  if (!length || !total || !out_length) return fail(AS_E_INVALID_ARG, "cache_evict: null pointer");
  const int64_t need = as_cache_evict_workspace(src, keep);
  if (workspace_bytes < need || !workspace || !aligned(workspace, 256))
    return fail(AS_E_INVALID_ARG, "cache_evict: workspace of %lld bytes, %lld needed (aligned to 256)",
                (long long)workspace_bytes, (long long)need);
  const EvictArgs p{cache_args(src), cache_args(dst), length, total, out_length,
                    reinterpret_cast<int32_t*>(workspace), keep, recent};
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const unsigned rows = (unsigned)(src->n_seqs * src->n_heads);
  hipLaunchKernelGGL(evict_select, dim3(rows), dim3(kSelThreads), 0, s, p);
  hipLaunchKernelGGL(evict_move, dim3((unsigned)((keep + 31) / 32), rows), dim3(256), 0, s, p);
  return launched("cache_evict");
}

}  // extern "C"
