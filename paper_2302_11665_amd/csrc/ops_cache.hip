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

// What 8 channels of one token and head become, on one of the DIM/8 lanes that
// hold it: their codes as a word of K and as a byte each, the group's scale, and
// the values that they stand for.
struct Quantised {
  uint32_t word, bytes[2];
  _Float16 step, base;
  float value[8];
};

// Codes are those of (x - m) / d rounded to fp32: the quotient is taken with the
// reciprocal and corrected once by its remainder, which leaves it 2^-46 of itself
// off before the last rounding.  d has 11 bits, so no quotient is that near to the
// middle between two fp32 numbers without being there, and the result is the
// division's.  x - m is exact for 16-bit x and m of like size.  Adding 1.5 * 2^23
// rounds to whole numbers, ties to even.
__device__ __forceinline__ v4u read8(const uint16_t* x) {
  v4u raw;
  __builtin_memcpy(&raw, x, 16);
  return raw;
}

// The value of the lane at the other end of a pair, of four lanes, of 8 and of 16,
// or in the other pair: exchanges within a row of 16.
template <int CTRL>
__device__ __forceinline__ int row_exchange(int x) {
  return __builtin_amdgcn_update_dpp(x, x, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ void group_step(float& low, float& high, int& any) {
  low = fminf(low, __int_as_float(row_exchange<CTRL>(__float_as_int(low))));
  high = fmaxf(high, __int_as_float(row_exchange<CTRL>(__float_as_int(high))));
  any |= row_exchange<CTRL>(any);
}

template <int TYPE, int GROUP>
__device__ __forceinline__ Quantised quantise8(const v4u& raw) {
  float f[8];
  float low = kInf, high = -kInf;
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    f[e] = to_f32<TYPE>(e & 1 ? raw[e >> 1] >> 16 : raw[e >> 1] & 0xffffu);
    bad |= f[e] != f[e];
    f[e] = __builtin_amdgcn_fmed3f(f[e], -65504.0f, 65504.0f);  // (finite, a NaN too)
    low = fminf(low, f[e]);
    high = fmaxf(high, f[e]);
  }
  int any = bad;
  static_assert(GROUP == 32 || GROUP == 64 || GROUP == 128, "4, 8 or 16 lanes to a group");
  group_step<0xb1>(low, high, any);   // lanes 1, 0, 3, 2 of four
  group_step<0x4e>(low, high, any);   // 2, 3, 0, 1
  if (GROUP >= 64) group_step<0x141>(low, high, any);   // 8 lanes mirrored: the other four's
  if (GROUP >= 128) group_step<0x140>(low, high, any);  // 16: the other 8's
  Quantised z{};
  z.base = any ? (_Float16)__builtin_nanf("") : (_Float16)low;
  z.step = any ? (_Float16)__builtin_nanf("") : (_Float16)((high - low) / 15.0f);
  const float m = (float)z.base, d = (float)z.step;
  const bool some = d > 0.0f;  // (not NaN)
  const float by = some ? 1.0f / d : 0.0f, from = some ? m : 0.0f, step = some ? d : 0.0f;
  uint32_t r[8];  // the code in the lowest byte
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float y = f[e] - from;
    float q = y * by;
    q = fmaf(fmaf(-q, step, y), by, q);
    const float whole = __builtin_amdgcn_fmed3f(q, 0.0f, 15.0f) + 12582912.0f;
    r[e] = __float_as_uint(whole);
    z.value[e] = (whole - 12582912.0f) * d + m;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)  // elements 2 i and 2 i + 1: nibbles i and 4 + i
    z.word |= __builtin_amdgcn_perm(r[2 * i + 1], r[2 * i], 0x0c040c00) << (4 * i);
#pragma unroll
  for (int i = 0; i < 2; ++i)
    z.bytes[i] = __builtin_amdgcn_perm(r[4 * i + 1], r[4 * i], 0x0c0c0400) |
                 __builtin_amdgcn_perm(r[4 * i + 3], r[4 * i + 2], 0x04000c0c);
  return z;
}

// Puts one lane's 8 channels of a key or value at place `at` of a page and head
// (row); V's codes go to v_codes, the token's row in LDS.
template <int DIM, int GROUP>
__device__ __forceinline__ void put8(const CacheArgs& c, int64_t row, int at, int lane, bool is_v, const Quantised& z,
                                     v2u* v_codes) {
  if (is_v)
    v_codes[lane] = v2u{z.bytes[0], z.bytes[1]};
  else
    // channels 8 lane..: word [g = lane%4][i = lane/4] of the token
    c.k[(row * c.page + at) * (DIM / 8) + (lane & 3) * (DIM / 32) + (lane >> 2)] = z.word;
  if (lane % (GROUP / 8) == 0) {
    uint32_t* par = is_v ? c.v_par : c.k_par;
    par[(row * (DIM / GROUP) + lane / (GROUP / 8)) * c.page + at] =
        (uint32_t)__builtin_bit_cast(uint16_t, z.step) | (uint32_t)__builtin_bit_cast(uint16_t, z.base) << 16;
  }
}

// Word w of a block of 32 slots of V from the codes of its slots lo..hi-1, a row of
// DIM each; the other slots' bits stay.
template <int DIM>
__device__ __forceinline__ void put_v_word(uint32_t* v, int w, const uint8_t* codes, int lo, int hi) {
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

// A wavefront's part of a block of 32 slots of V, the words of slots 4 g.. and 16 + 4 g..,
// from rows of codes, row 0 being slot 0's; only `slots` are the call's.  Others
// may write the other slots' bits of a word meanwhile.  The slots' own bits are nobody
// else's: one atomic clears them and one sets them, neither of which is waited for (a
// read and an exclusive or of what has to change: 64 single tokens 9.0 us, so 6.9).
// Rows of other slots are read and left out, so that no read waits for another.
template <int DIM>
__device__ __forceinline__ void put_v_words(uint32_t* v, int g, uint32_t slots, const uint8_t* codes) {
  const int lane = threadIdx.x & 63;
  uint32_t mask = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) mask |= (slots >> (16 * (e >> 2) + 4 * g + (e & 3)) & 1u) * (15u << nibble(e));
#pragma unroll
  for (int w = lane; w < DIM; w += 64) {
    const int i = w % (DIM / 16), c = w / (DIM / 16);
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      word |= (uint32_t)(codes[(16 * (e >> 2) + 4 * g + (e & 3)) * DIM + 16 * i + c] & 15) << nibble(e);
    uint32_t* to = v + g * DIM + w;
    if (mask == 0xffffffffu)
      *to = word;
    else
      atomicAnd(to, ~mask), atomicOr(to, word & mask);
  }
}

// One workgroup per (sequence, head, block of 32 slots).  DIM/8 lanes quantise
// a token's key or value, 8 channels each: a word of K as it is; V's codes
// change direction (a word holds 8 tokens of one channel), through LDS, and a
// word that keeps older tokens is read first.  No other workgroup has this
// block's words, so nothing races.  Latency bounds a step of one token: 4.3 us
// for 40 sequences of 8 heads, a load that depends on two others and a store.
template <int TYPE, int DIM, int GROUP>
__global__ __launch_bounds__(256) void append(AppendArgs p) {
  constexpr int kLanes = DIM / 8;       // lanes of one token's key or value
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
    float* held = is_v ? p.held_v : p.held_k;
    if (held) held += (((int64_t)b * p.n_tokens + t) * p.c.n_heads + h) * DIM + lane * 8;
    const int at = in_page + s;
    const Quantised z = quantise8<TYPE, GROUP>(read8(x));
    put8<DIM, GROUP>(p.c, row, at, lane, is_v, z, v_codes[s]);
    if (held) __builtin_memcpy(held, z.value, 32);
    if (is_v && lane == 0) {
      if (p.c.pos) p.c.pos[row * p.c.page + at] = (int32_t)(p.first_pos ? p.first_pos[b] + t : first + s);
      if (p.c.acc) p.c.acc[row * p.c.page + at] = 0.0f;
    }
  }
  __syncthreads();
  uint32_t* v = p.c.v + (row * p.c.page + in_page) * kWords;
  for (int w = threadIdx.x; w < 32 * kWords; w += 256)
    put_v_word<DIM>(v, w, reinterpret_cast<const uint8_t*>(v_codes), lo, hi);
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

// ------------------------------------------------------------ packed append

struct PackedArgs {
  CacheArgs c;
  const uint16_t *k, *v;
  int64_t k_token, v_token;
  const int32_t *seq, *slot, *pos;
  float *held_k, *held_v;
  int32_t n_tokens, n_blocks, tile;  // blocks of 32 tokens; tokens whose runs a workgroup takes, at most 32
};

// Writes one token's values from its DIM/8 lanes, 8 channels each, past the caches, 4
// channels side by side to a lane at a time (`own`: LDS of the token).
template <int DIM>
__device__ __forceinline__ void put_held(float* held, int lane, const float (&value)[8], v4f* own) {
  own[2 * lane] = v4f{value[0], value[1], value[2], value[3]};
  own[2 * lane + 1] = v4f{value[4], value[5], value[6], value[7]};
  __builtin_amdgcn_wave_barrier();
  typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int i = 0; i < 2; ++i)
    __builtin_nontemporal_store((v4f_any)own[i * (DIM / 8) + lane], reinterpret_cast<v4f_any*>(held) + i * (DIM / 8) + lane);
  __builtin_amdgcn_wave_barrier();
}

// One workgroup per (tile of packed tokens, head).  Neighbouring tokens of one
// sequence on neighbouring slots of one block of 32 are a run; a workgroup takes
// the runs that begin in its tile, whole, so that most words of V are written
// in one store.  First all of its tokens are quantised side by side, then V's words
// are written, a quarter of a run's block (the words of 8 of its slots) to a
// wavefront at a time.  Few tokens cost a launch and a chain of loads (places, page,
// values): 39 of 8 heads of 128 channels 4.9 us.  Many are bound by what they read and
// write and by the quantisation's instructions, some ten a value, which take about as
// long: 64,590 of 8 heads of 64 channels 54 us, with the values held 70.
template <int TYPE, int DIM, int GROUP>
__global__ __launch_bounds__(256) void append_packed(PackedArgs p) {
  constexpr int kLanes = DIM / 8, kWords = DIM / 8, kAtOnce = 256 / kLanes;
  // places for values; then V's codes of the tile's tokens and as many behind them
  constexpr int kValues = kAtOnce * kLanes * 32;
  static_assert(kValues >= 31 * DIM, "rows up to 31 before the first are read, and left out");
  __shared__ __attribute__((aligned(16))) uint8_t lds[kValues + 64 * DIM];
  auto v_codes = reinterpret_cast<v2u (*)[kLanes]>(lds + kValues);
  __shared__ int64_t rows[64];         // page and head of each, -1: none
  __shared__ int32_t places[64];       // in the page
  const int wide = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Within a long run one tile in 32 / tile begins a block and has work, the others
  // none: such tiles of all heads are neighbours in the grid, which deals workgroups
  // to the XCDs in turn.  (With tiles in the order of their tokens, those that had work
  // were on two XCDs: 1305 tokens of 8 heads 15.2 us, so 9.)
  const int h = blockIdx.x / p.n_blocks % p.c.n_heads, part = blockIdx.x / p.n_blocks / p.c.n_heads;
  const int64_t t0 = (int64_t)(blockIdx.x % p.n_blocks) * 32 + part * p.tile;
  // every wavefront looks at the tile's tokens and those behind them
  const int64_t t = t0 + wide;
  int seq = -1, slot = -1;
  if (t < p.n_tokens) seq = p.seq[t], slot = p.slot[t];
  int before = __shfl_up(seq, 1), slot_before = __shfl_up(slot, 1);
  if (wide == 0 && t > 0 && t < p.n_tokens) before = p.seq[t - 1], slot_before = p.slot[t - 1];
  const bool real = (unsigned)seq < (unsigned)p.c.n_seqs && slot >= 0;
  const bool follows = real && t > 0 && slot % 32 != 0 && before == seq && slot_before == slot - 1;
  const uint64_t in_run = __ballot(follows), tile = (uint64_t(1) << p.tile) - 1;
  uint64_t begins = __ballot(real && !follows) & tile;
  if (!begins) return;
  // from its first beginning on, the tile's tokens are its own, and behind the
  // tile those that go on with its last run (at most 31)
  const uint64_t own_from = ~uint64_t(0) << __builtin_ctzll(begins);
  uint64_t own = __ballot(real) & tile & own_from;
  if (own >> (p.tile - 1) & 1) own |= ((uint64_t(1) << __builtin_ctzll(~(in_run >> p.tile))) - 1) << p.tile;
  if (wave == 0) {
    const bool mine = own >> wide & 1;
    rows[wide] = mine ? cache_row(p.c, seq, h, slot / p.c.page) : -1;
    places[wide] = slot % p.c.page;
  }
  lds_barrier();
  const int lane = threadIdx.x % kLanes, last = 63 - __builtin_clzll(own);
  for (int i0 = __builtin_ctzll(own) + threadIdx.x / kLanes; i0 <= last; i0 += 2 * kAtOnce) {
    v4u raw[2][2];  // of two tokens, all on their way at once
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = i0 + j * kAtOnce;
      if (i > last || rows[i] < 0) continue;
      const int64_t u = t0 + i, from = (int64_t)h * DIM + lane * 8;
      raw[j][0] = read8(p.k + u * p.k_token + from);
      raw[j][1] = read8(p.v + u * p.v_token + from);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = i0 + j * kAtOnce;
      if (i > last) continue;
      const int64_t row = rows[i], u = t0 + i, held = (u * p.c.n_heads + h) * DIM;
      if (row < 0) continue;
      const int at = places[i];
      const Quantised k = quantise8<TYPE, GROUP>(raw[j][0]), v = quantise8<TYPE, GROUP>(raw[j][1]);
      v4f* own = reinterpret_cast<v4f*>(lds) + threadIdx.x / kLanes * 2 * kLanes;
      if (p.held_k) put_held<DIM>(p.held_k + held, lane, k.value, own);
      if (p.held_v) put_held<DIM>(p.held_v + held, lane, v.value, own);
      put8<DIM, GROUP>(p.c, row, at, lane, false, k, nullptr);
      put8<DIM, GROUP>(p.c, row, at, lane, true, v, v_codes[i]);
      if (lane == 0) {
        if (p.c.pos) p.c.pos[row * p.c.page + at] = p.pos ? p.pos[u] : p.slot[u];
        if (p.c.acc) p.c.acc[row * p.c.page + at] = 0.0f;
      }
    }
  }
  lds_barrier();
  for (; begins; begins &= begins - 1) {
    const int i = __builtin_ctzll(begins);
    const int n = 1 + (i < 63 ? (int)__builtin_ctzll(~(in_run >> (i + 1))) : 0);  // at most 32
    const int64_t row = rows[i];
    const int at = __builtin_amdgcn_readfirstlane(places[i]), lo = at % 32;
    const uint32_t slots = (n < 32 ? (1u << n) - 1 : ~0u) << lo;
    if (row < 0 || !(slots & 0x000f000fu << (4 * wave))) continue;  // slots 4 wave.. and 16 + 4 wave..
    put_v_words<DIM>(p.c.v + (row * p.c.page + at - lo) * kWords, wave, slots, lds + kValues + (i - lo) * DIM);
  }
}

template <int TYPE>
void launch_packed(const PackedArgs& p, hipStream_t s) {
  const dim3 g((unsigned)(p.n_blocks * (32 / p.tile) * p.c.n_heads)), t(256);
  if (p.c.dim == 64 && p.c.group == 32) hipLaunchKernelGGL((append_packed<TYPE, 64, 32>), g, t, 0, s, p);
  if (p.c.dim == 64 && p.c.group == 64) hipLaunchKernelGGL((append_packed<TYPE, 64, 64>), g, t, 0, s, p);
  if (p.c.dim == 128 && p.c.group == 32) hipLaunchKernelGGL((append_packed<TYPE, 128, 32>), g, t, 0, s, p);
  if (p.c.dim == 128 && p.c.group == 64) hipLaunchKernelGGL((append_packed<TYPE, 128, 64>), g, t, 0, s, p);
  if (p.c.dim == 128 && p.c.group == 128) hipLaunchKernelGGL((append_packed<TYPE, 128, 128>), g, t, 0, s, p);
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

int as_cache_append_packed(const as_cache_t* cache, const void* k, const void* v, int32_t type, int64_t n_tokens,
                           int64_t k_token, int64_t v_token, const int32_t* seq, const int32_t* slot, const int32_t* pos,
                           float* held_k, float* held_v, void* stream) {
  const int rc = check_cache(cache, "cache_append_packed", false, false);
  if (rc != AS_OK) return rc;
  if (type != AS_BF16 && type != AS_F16) return fail(AS_E_INVALID_ARG, "cache_append_packed: type %d", type);
  if (n_tokens < 0) return fail(AS_E_INVALID_ARG, "cache_append_packed: %lld tokens", (long long)n_tokens);
  // (a workgroup of 256 threads to 32 tokens and a head, fewer than 2^32 threads)
  if (n_tokens > (1 << 28) || (n_tokens + 31) / 32 * cache->n_heads >= (1 << 24))
    return fail(AS_E_LIMITS, "cache_append_packed: %lld tokens of %d heads (tokens times heads below 2^29)",
                (long long)n_tokens, cache->n_heads);
  if (n_tokens == 0 || cache->n_seqs == 0) return as_host::ok();
  if (!k || !v || !seq || !slot) return fail(AS_E_INVALID_ARG, "cache_append_packed: null pointer");
  PackedArgs p{cache_args(cache), reinterpret_cast<const uint16_t*>(k), reinterpret_cast<const uint16_t*>(v),
               k_token, v_token, seq, slot, pos, held_k, held_v, (int32_t)n_tokens, (int32_t)((n_tokens + 31) / 32), 4};
  // Single tokens are a run each: few of them to a workgroup as long as there are not
  // too many workgroups.  Tiles of 4 and of 32 tokens, 8 heads of 128 channels: 39 single
  // tokens 4.9 and 10.6 us, 38 and a prompt of 1305 8.9 and 11.7, a prompt of 8000 23 and 18.
  while (p.tile < 32 && p.n_blocks * (32 / p.tile) * (int64_t)cache->n_heads > 16 * (int64_t)as_host::compute_units())
    p.tile *= 2;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (type == AS_BF16)
    launch_packed<AS_BF16>(p, s);
  else
    launch_packed<AS_F16>(p, s);
  return launched("cache_append_packed");
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
