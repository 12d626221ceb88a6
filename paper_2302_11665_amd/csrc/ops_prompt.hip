// Causal attention over packed prompts (alpaserve_ops.h): every token of a
// sequence attends to the tokens of its sequence up to itself.
//
//   o_t = sum_s p_ts v_s,  p_ts = exp(scale q_t.k_s) / sum_s' exp(scale q_t.k_s')
//
// The products are made transposed, S^T = K Q^T and O^T = V^T P^T, in tiles of
// 32x32x16: lane l then holds scores of one query (column l % 32) alone, so the
// softmax's maximum and sum stay within a lane and its partner l ^ 32, a query's
// rescaling is one factor per lane, and P^T is in the order in which the second
// product takes it.  There a lane has keys 8 (r / 4) + 4 (l / 32) + r % 4 of 32;
// V's operand takes the same order of keys, four of one channel at a time, from
// rows in LDS by transposing reads.
//
// What bounds it: 4 dim operations a head and pair of tokens, which the matrix units
// would do in 0.96 ms for 12,001 tokens of 32 heads of 128 channels, and an exponential
// for each pair, whose vector instructions take about half as long as the products.
// The kernel takes 1.07 to 1.11 ms (1063 to 1103 TFLOP/s, of the pairs that count; the matrix units
// busy for 54 % of the cycles, at 1.75 GHz under this load), 0.97 ms without the
// softmax.  Heads of 64 channels have half the products for as many exponentials, and matrix
// and vector instructions follow one another (30 and 61 % of the cycles): 32 of them 0.67 to 0.69 ms.
#include <algorithm>
#include <type_traits>

#include "ops_common.hpp"

using as_host::fail;

namespace as_ops {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));

struct PromptArgs {
  const uint16_t *q, *k, *v;
  uint16_t* out;
  int64_t q_token, k_token, v_token;  // strides in elements
  const int32_t* offsets;
  int32_t n_tokens, n_seqs, n_heads, group;  // key/value heads; query heads to each
  float factor;                              // scale log2 e
  int32_t part_tiles, n_parts;               // of a split block (below)
  float* parts;
  int32_t second;  // blocks from here on are taken in the opposite order
};

template <int TYPE>
__device__ __forceinline__ v16f multiply(v8s a, v8s b, v16f c) {
  if constexpr (TYPE == AS_BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// Two numbers rounded to the type, the first in the low half.
template <int TYPE>
__device__ __forceinline__ uint32_t pack_two(float a, float b) {
  if constexpr (TYPE == AS_BF16) return pack_bf16(a, b);
  return __builtin_bit_cast(uint32_t, v2h{(_Float16)a, (_Float16)b});
}

__device__ __forceinline__ float max_halves(float x) {
  const v2u p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const v2u p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// A sequence's tokens, clipped to those that there are, and its blocks of ROWS rows
// (a row: one query of one head of the group).
struct Sequence {
  int begin, length;
};
__device__ __forceinline__ Sequence sequence(const PromptArgs& p, int b) {
  const int begin = min(max(p.offsets[b], 0), p.n_tokens);
  return {begin, min(max(p.offsets[b + 1], begin), p.n_tokens) - begin};
}
template <int ROWS>
__device__ __forceinline__ int blocks_of(const PromptArgs& p, int length) {
  return (int)((uint32_t)(length * p.group + ROWS - 1) / ROWS);
}

// Tiles of 64 keys that a block's rows see.
constexpr int kKeys = 64;
template <int ROWS>
__device__ __forceinline__ int tiles_of(const PromptArgs& p, int length, int block) {
  return min(block * ROWS + ROWS - 1, length * p.group - 1) / p.group / kKeys + 1;
}

// What a workgroup works on: a block of a sequence.
struct Item {
  int begin, length, block, none;
};

__device__ __forceinline__ uint32_t sum_lanes(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_readlane((int)scan_lanes(x), 63);
}

// The item-th block of at most 64 sequences, those with the most keys first:
// blocks begin at their sequence's first token, so the j-th of every sequence has
// as much work, and items are in order of falling j, then of sequences.  False where
// there are fewer items.  A wavefront's work: a lane to a sequence, and j is found
// by halving.
template <int ROWS>
__device__ __forceinline__ bool find_block(const PromptArgs& p, uint32_t item, Item& found) {
  const int lane = threadIdx.x & 63;
  Sequence s{0, 0};
  if (lane < p.n_seqs) s = sequence(p, lane);
  const int blocks = blocks_of<ROWS>(p, s.length);
  auto beyond = [&](int j) { return sum_lanes((uint32_t)max(0, blocks - j)); };  // items of blocks j and later
  if (beyond(0) <= item) return false;
  int lo = 0, hi = 1;  // beyond(lo) > item >= beyond(hi)
  while (beyond(hi) > item) lo = hi, hi *= 2;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (beyond(mid) > item)
      lo = mid;
    else
      hi = mid;
  }
  const uint32_t rank = item - beyond(lo + 1);  // among the sequences that have this block
  const uint64_t have = __ballot(blocks > lo);
  const bool here = (have >> lane & 1) && (uint32_t)__popcll(have & ((uint64_t(1) << lane) - 1)) == rank;
  const int at = __builtin_ctzll(__ballot(here));
  found = Item{__builtin_amdgcn_readlane(s.begin, at), __builtin_amdgcn_readlane(s.length, at), lo, 0};
  return true;
}

// The same for many sequences, once for all workgroups: the blocks of all
// sequences, listed by classes of their numbers of blocks (four to a power of two),
// the largest first, and within a sequence the last one first.  One workgroup: the
// classes are counted, then every sequence takes its place in its class (in no
// certain order, which changes nothing but when a block is worked on), then wavefronts write
// the sequences' blocks.  (200 prompts of 700 tokens, heads of 64 channels: 461 us where
// every workgroup went over the sequences to find its block, 281 with the list.)
// Offsets that make no sense may give each of 2^20 sequences 2^23 blocks: blocks are
// counted in 64 bits, and those behind the list's end neither written nor gone over.
constexpr int kPlanThreads = 1024;

template <int ROWS>
__global__ __launch_bounds__(kPlanThreads) void prompt_plan(PromptArgs p, Item* items, int n_items) {
  __shared__ unsigned long long classes[128];
  __shared__ Item part[kPlanThreads];  // block: how many; none: the first one's place
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto class_of = [](int blocks) { return 127 - min(127, (int)(__float_as_uint((float)blocks) >> 21) - (127 << 2)); };
  if (tid < 128) classes[tid] = 0;
  __syncthreads();
  for (int b = tid; b < p.n_seqs; b += kPlanThreads) {
    const int blocks = blocks_of<ROWS>(p, sequence(p, b).length);
    if (blocks) atomicAdd(&classes[class_of(blocks)], (unsigned long long)blocks);
  }
  __syncthreads();
  if (wave == 0) {  // where every class begins (n_items is below 2^24: the sum of 128 is below 2^31)
    const unsigned long long most = n_items;
    const uint32_t a = (uint32_t)min(classes[2 * lane], most), z = (uint32_t)min(classes[2 * lane + 1], most);
    const uint32_t upto = scan_lanes(a + z);
    classes[2 * lane] = upto - a - z;
    classes[2 * lane + 1] = upto - z;
    if (lane == 63) part[0].none = (int)upto;
  }
  __syncthreads();
  for (int i = part[0].none + tid; i < n_items; i += kPlanThreads) items[i] = Item{0, 0, 0, 1};
  __syncthreads();
  for (int first = 0; first < p.n_seqs; first += kPlanThreads) {
    Item mine{0, 0, 0, 0};
    if (first + tid < p.n_seqs) {
      const Sequence s = sequence(p, first + tid);
      const int blocks = blocks_of<ROWS>(p, s.length);
      mine = Item{s.begin, s.length, blocks, 0};
      if (blocks) {
        const unsigned long long at = atomicAdd(&classes[class_of(blocks)], (unsigned long long)blocks);
        mine.none = (int)min(at, (unsigned long long)n_items);
      }
    }
    part[tid] = mine;
    __syncthreads();
    for (int i = wave; i < min(kPlanThreads, p.n_seqs - first); i += kPlanThreads / 64) {
      const Item s = part[i];
      for (int j = lane; j < min(s.block, n_items - s.none); j += 64)
        items[s.none + j] = Item{s.begin, s.length, s.block - 1 - j, 0};
    }
    __syncthreads();
  }
}

// Rows of a stage lie in LDS as in memory, in pieces of 16 bytes whose order is
// swapped around by key: 16 keys at one piece (K's operand) and 4 keys at two
// pieces side by side (V's) then fall on different banks.
template <int DIM>
__device__ __forceinline__ int swizzle(int key) {
  return DIM == 128 ? (key & 3) << 2 | (key >> 2 & 3) : (key >> 1 & 1) << 2 | (key >> 2 & 3);
}

// Bits of a 16-bit value that is not finite.
template <int TYPE>
__device__ __forceinline__ bool not_finite(uint16_t u) {
  return TYPE == AS_BF16 ? (u & 0x7f80u) == 0x7f80u : (u & 0x7c00u) == 0x7c00u;
}
template <int TYPE>
constexpr uint16_t kOne = TYPE == AS_BF16 ? 0x3f80 : 0x3c00;
template <int TYPE>
constexpr uint16_t kInfinity = TYPE == AS_BF16 ? 0x7f80 : 0x7c00;

// A workgroup takes 32 rows a wavefront of one key/value head (rows: queries and
// the heads of their group, queries in order) over the keys that they see, 64 at
// a time, which come into two stages of LDS straight from memory.  All heads of a group
// share a tile of keys, and queries stay in registers.  8 wavefronts a workgroup or
// stages of 32 keys were slower: more rows of a block wait for its last keys, or there
// are more barriers to a key.
//
// Masked scores give p = 0, but 0 times an infinity or NaN in V is NaN.  A block
// whose results are all finite met none; otherwise (false is returned, and nothing
// written) it is done again, CAREFUL: at keys that some of its rows do not see,
// values that are not finite are left out of the product and reach the rows that see
// them by products of their marks with a mask.
//
// Values of bf16 times weights that are not divided by their sum yet can also pass fp32's
// range where the result does not (1e38).  Where the block's keys have finite values of
// kLarge or more, CAREFUL takes the reference and the sum of weights that the first pass
// found and divides each weight by that sum before it is rounded: what is added up then
// stays below the largest value, but for roundings.  (fp16's sums cannot get there.)
//
// SPLIT: its tiles of keys from first to end; sums, the reference of the weights and
// their sums go to `part`, the sum of weights with its sign turned where the sums are
// divided by it.
constexpr uint16_t kLarge = 0x4d80;  // 2^28, in bf16: 2^26 weights of 2^8, off by 2^64 for the largest logits
struct Weights {
  float reference, total;  // of a row's exponents; sum of its weights
};
template <int TYPE, int DIM, int WAVES, bool CAREFUL, bool SPLIT>
__device__ __forceinline__ bool attend_block(const PromptArgs& p, uint8_t (*lds)[2][kKeys * DIM * 2], int head, int begin,
                                             int length, int block, int first, int end, float* part, Weights& found) {
  constexpr int kRows = 32 * WAVES, kRowBytes = DIM * 2, kTile = kKeys * kRowBytes;
  constexpr int kLoads = kTile / 1024 / WAVES;  // of K and of V, by a wavefront, a stage
  constexpr int kPieces = kRowBytes / 16, kPerLoad = 1024 / kRowBytes;  // keys of a load
  constexpr int kSteps = DIM / 16, kDimTiles = DIM / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int rows = length * p.group, row0 = block * kRows + wave * 32;
  // rows behind the last one do its work again
  const int row = min(row0 + col, rows - 1), pos = row / p.group, member = row - pos * p.group;
  // tiles that all rows of the block see whole, that this wavefront's rows see, and
  // that any row does
  if (!SPLIT) first = 0, end = INT32_MAX;
  const int open = min((block * kRows / p.group + 1) / kKeys, end);
  const int mine = min(min(row0 + 31, rows - 1) / p.group / kKeys + 1, end);
  const int tiles = min(tiles_of<kRows>(p, length, block), end);

  v8s q[kSteps];
  {
    const uint16_t* at = p.q + (int64_t)(begin + pos) * p.q_token + (int64_t)(head * p.group + member) * DIM + half * 8;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) q[i] = *reinterpret_cast<const v8s*>(at + i * 16);
  }

  // Stages come in by loads of 1 KiB, kPerLoad keys each, of which the wavefront
  // brings every WAVES-th.  A lane has the same piece of all of its keys, so its
  // place is one offset from an address that is the wavefront's.
  const int in_load = wave * kPerLoad + lane / kPieces, piece = (lane % kPieces) ^ swizzle<DIM>(in_load);
  const uint32_t k_lane = (uint32_t)(lane / kPieces * (int)p.k_token * 2 + piece * 16);
  const uint32_t v_lane = (uint32_t)(lane / kPieces * (int)p.v_token * 2 + piece * 16);
  const uint8_t* k0 = reinterpret_cast<const uint8_t*>(p.k + (int64_t)begin * p.k_token + (int64_t)head * DIM);
  const uint8_t* v0 = reinterpret_cast<const uint8_t*>(p.v + (int64_t)begin * p.v_token + (int64_t)head * DIM);
  auto bring = [&](uint8_t* to, const uint8_t* from, int64_t token, uint32_t offset, int tile) {
    auto load = [&](int j, const uint8_t* at) {
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)at,
                                       (__attribute__((address_space(3))) void*)(to + (wave + j * WAVES) * 1024), 16, 0,
                                       0);
    };
    const int key = tile * kKeys + wave * kPerLoad;  // of the first lane and load
    if ((tile + 1) * kKeys <= length) {
      const uint8_t* at = from + (int64_t)key * token * 2;
#pragma unroll
      for (int j = 0; j < kLoads; ++j) load(j, at + j * (int64_t)(WAVES * kPerLoad) * token * 2 + offset);
    } else {  // keys behind the last one are it again: masked, and no other sequence's
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        load(j, from + (int64_t)min(key + j * WAVES * kPerLoad + lane / kPieces, length - 1) * token * 2 + piece * 16);
    }
  };
  auto bring_k = [&](int tile) { bring(lds[tile & 1][0], k0, p.k_token, k_lane, tile); };
  auto bring_v = [&](int tile) { bring(lds[tile & 1][1], v0, p.v_token, v_lane, tile); };

  v16f o[kDimTiles];
  float reference, total;  // of the exponents; sum of this lane's keys' p
  bool divided = false;
  if (CAREFUL && TYPE == AS_BF16) {
    uint32_t top = 0;
    const int from = first * kKeys, keys = min(tiles * kKeys, length) - from;
    for (int64_t i = threadIdx.x; i < (int64_t)keys * kPieces; i += 64 * WAVES) {
      const v4u eight = *reinterpret_cast<const v4u*>(v0 + ((from + i / kPieces) * p.v_token + i % kPieces * 8) * 2);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t u = (e & 1 ? eight[e >> 1] >> 16 : eight[e >> 1]) & 0x7fffu;
        if (u < kInfinity<TYPE>) top = max(top, u);
      }
    }
    uint32_t* marks = reinterpret_cast<uint32_t*>(lds[1][0]);
    const bool any = __any(top >= kLarge);
    if (lane == 0) marks[wave] = any;
    lds_barrier();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) divided |= marks[i] != 0;
    lds_barrier();  // all have read it before tiles come in there
    divided = divided && found.total > 0x1p-100f && found.total < 0x1p100f;
  }
  const float share = divided ? 1.0f / found.total : 1.0f;

  // Places of the operands: the pieces' order changes by exclusive ors of bits that
  // nothing else in an address has, so a lane's places follow from one.
  const uint32_t k_place = col * kRowBytes + ((half ^ swizzle<DIM>(col)) << 4);
  const int v_key = half * 4 + (lane & 15) / 4;
  const uint32_t v_place = v_key * kRowBytes + (((lane >> 4 & 1) * 2 + (lane >> 1 & 1) ^ swizzle<DIM>(v_key)) << 4) + (lane & 1) * 8;
  auto scores = [&](int tile, v16f (&s)[2]) {
    const uint32_t at = (uint32_t)(tile & 1) * (2 * kTile) + k_place;
#pragma unroll
    for (int h = 0; h < 2; ++h) s[h] = v16f{};
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)  // keys 32 h.., channels 16 i..
        s[h] = multiply<TYPE>(*reinterpret_cast<const v8s*>(lds[0][0] + (at ^ 32 * i) + h * 32 * kRowBytes), q[i], s[h]);
  };
  // The reference of a query's exponents follows its maximum when it is passed by 2^8.
  auto follow = [&](const v16f (&s)[2]) {
    float top = s[0][0];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[h][r]);
    top = max_halves(top) * p.factor;
    if (__any(top > reference + 8.0f)) {
      const float now = top > reference + 8.0f ? top : reference, by = __builtin_amdgcn_exp2f(reference - now);
      reference = now;
      total *= by;
#pragma unroll
      for (int i = 0; i < kDimTiles; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] *= by;
    }
  };
  // The matrix instructions take weights of the type: each is rounded to it, and their sum
  // is of what they were before.  (Two numbers of the type to a weight would keep its bits
  // for half as many products again.)
  auto weigh = [&](const v16f (&s)[2], v8s (&weights)[4]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float e = __builtin_amdgcn_exp2f(fmaf(s[h][r], p.factor, -reference));
        if (CAREFUL) e *= share;
        total += e;
        weights[h * 2 + (r >> 3)][r & 7] = (short)from_f32<TYPE>(e);
      }
  };
  // V's operand: channels 32 i.. of keys 16 z..
  auto values = [&](int tile, int i, int z) {
    const uint32_t at = (uint32_t)(tile & 1) * (2 * kTile) + v_place;
    v8s v;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const v4s four = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) v4s*)(lds[0][1] + (at ^ (64 * i | 32 * j)) + (z * 16 + j * 8) * kRowBytes));
#pragma unroll
      for (int e = 0; e < 4; ++e) v[j * 4 + e] = four[e];
    }
    return v;
  };
  auto add = [&](int tile, const v8s (&weights)[4]) {
#pragma unroll
    for (int z = 0; z < 4; ++z)
#pragma unroll
      for (int i = 0; i < kDimTiles; ++i) o[i] = multiply<TYPE>(values(tile, i, z), weights[z], o[i]);
  };
  // The same where some rows do not see some keys and values may not be finite:
  // for each of NaN and the two infinities, the count of those that a row sees.
  auto add_careful = [&](int tile, const v8s (&weights)[4]) {
#pragma unroll
    for (int i = 0; i < kDimTiles; ++i) {
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        v8s v = values(tile, i, z);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = not_finite<TYPE>((uint16_t)v[e]) ? (short)0 : v[e];
        o[i] = multiply<TYPE>(v, weights[z], o[i]);
      }
#pragma unroll 1
      for (int kind = 0; kind < 3; ++kind) {
        const uint16_t wanted = kind == 0 ? kInfinity<TYPE> : kInfinity<TYPE> | 0x8000;
        v16f count = {};
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          v8s v = values(tile, i, z), seen;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const uint16_t u = (uint16_t)v[e];
            const bool is = kind == 2 ? not_finite<TYPE>(u) && (u & 0x7fff) != kInfinity<TYPE> : u == wanted;
            v[e] = (short)(is ? kOne<TYPE> : 0);
            const int key = tile * kKeys + z * 16 + 8 * (e >> 2) + 4 * half + (e & 3);
            seen[e] = (short)(key <= pos ? kOne<TYPE> : 0);
          }
          count = multiply<TYPE>(v, seen, count);
        }
        const float what = kind == 0 ? kInf : kind == 1 ? -kInf : __builtin_nanf("");
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] += count[r] > 0.0f ? what : 0.0f;
      }
    }
  };

#pragma unroll
  for (int i = 0; i < kDimTiles; ++i) o[i] = v16f{};
  reference = divided ? found.reference : -1e30f, total = 0.0f;
  bring_k(first);
  if (first + 1 < tiles) bring_k(first + 1);
  bring_v(first);
  // V of this tile and K of the one behind the next are there, and all are done with
  // V of the last tile and K of the next.
  auto turn = [&] {
    wait_loads<0>();
    lds_barrier();
  };
  // In their places, when V of this tile has been read: reads that transpose are made
  // to wait for all loads on their way.
  auto bring_next = [&](int tile) {
    if (tile + 1 < tiles) bring_v(tile + 1);
    if (tile + 3 < tiles) bring_k(tile + 3);
  };
  v16f s[2], next[2];
  v8s weights[4];
  int tile = first;
  if (first + 1 < tiles)
    wait_loads<2 * kLoads>();
  else
    wait_loads<kLoads>();
  lds_barrier();  // K of the first tile is there
  scores(first, s);
  wait_loads<kLoads>();
  lds_barrier();  // and of the second, and all are done with the first
  if (first + 2 < tiles) bring_k(first + 2);
  // A wavefront makes the scores of a tile while it turns the last one's into
  // weights, so that its matrix and vector instructions overlap.  Where heads have 64
  // channels, three wavefronts a SIMD overlap instead, which have no registers for two
  // tiles' scores (16 prompts of 512: 91 us with two wavefronts and the scores ahead, 67).  (Behind the last tile, scores are those of what lies in LDS, and
  // not used.)
  auto step = [&](v16f (&now)[2], v16f (&then)[2]) {
    follow(now);
    if (DIM == 128) scores(tile + 1, then);
    weigh(now, weights);
    if (DIM == 64) scores(tile + 1, then);
    turn();
    add(tile, weights);
    bring_next(tile);
    ++tile;
  };
  if (!CAREFUL && DIM == 128) {
    while (tile + 1 < open) {
      step(s, next);
      step(next, s);
    }
    if (tile < open) {
      step(s, next);
      s[0] = next[0], s[1] = next[1];
    }
  } else if (!CAREFUL) {
    while (tile < open) step(s, s);
  }
  // the tiles that some rows do not see whole, or not at all
  for (; tile < tiles; ++tile) {
    if (tile < mine) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (tile * kKeys + h * 32 + 8 * (r >> 2) + 4 * half + (r & 3) > pos) s[h][r] = -kInf;
      follow(s);
      weigh(s, weights);
      if (tile + 1 < mine) scores(tile + 1, s);
    }
    turn();
    if (tile < mine) {
      if (CAREFUL && tile >= open)
        add_careful(tile, weights);
      else
        add(tile, weights);
    }
    bring_next(tile);
  }
  total = sum_halves(total);

  lds_barrier();  // all are done with the tiles
  if (!CAREFUL) {
    bool fine = true;
#pragma unroll
    for (int i = 0; i < kDimTiles; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) fine &= fabsf(o[i][r]) < kInf;
    uint32_t* marks = reinterpret_cast<uint32_t*>(lds[1][0]);
    const bool any = __any(!fine);
    if (lane == 0) marks[wave] = any;
    lds_barrier();
    uint32_t all = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) all |= marks[i];
    if (__builtin_amdgcn_readfirstlane(all)) {
      lds_barrier();  // all have read it before the next pass writes there
      found = Weights{reference, total};
      return false;
    }
  }
  if (SPLIT) {  // channels 4 c.. of row r at [c][r]
#pragma unroll
    for (int i = 0; i < kDimTiles; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        reinterpret_cast<v4f*>(part)[(i * 8 + r / 2 + half) * kRows + wave * 32 + col] =
            v4f{o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
    if (half == 0) {
      part[DIM * kRows + wave * 32 + col] = reference;
      part[(DIM + 1) * kRows + wave * 32 + col] = divided ? -found.total : total;
    }
    return true;
  }
  // Rows go through LDS, where a row's lanes leave them 8 bytes each, and out as
  // whole lines.
  int late = lane;  // (what follows from it is computed here, not kept in registers all along)
  asm volatile("" : "+v"(late));
  const int row_in = late & 31, upper = late >> 5;
  uint8_t* own = lds[0][0] + wave * 32 * kRowBytes;
  const float by = 1.0f / total;
#pragma unroll
  for (int i = 0; i < kDimTiles; ++i)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const v2u four = {pack_two<TYPE>(o[i][r] * by, o[i][r + 1] * by), pack_two<TYPE>(o[i][r + 2] * by, o[i][r + 3] * by)};
      const int byte = i * 64 + r * 4 + upper * 8;
      *reinterpret_cast<v2u*>(own + row_in * kRowBytes + (((byte >> 4) ^ swizzle<DIM>(row_in)) << 4) + (byte & 8)) = four;
    }
#pragma unroll
  for (int i = 0; i < 32 / kPerLoad; ++i) {
    const int in = i * kPerLoad + late / kPieces, at = row0 + in;
    const v4u eight = *reinterpret_cast<const v4u*>(own + in * kRowBytes + (((late % kPieces) ^ swizzle<DIM>(in)) << 4));
    if (at >= rows) continue;
    const int query = at / p.group;
    uint16_t* to = p.out + ((int64_t)(begin + query) * p.n_heads * p.group + head * p.group + at - query * p.group) * DIM;
    *reinterpret_cast<v2u*>(to + late % kPieces * 8) = v2u{eight[0], eight[1]};
    *reinterpret_cast<v2u*>(to + late % kPieces * 8 + 4) = v2u{eight[2], eight[3]};
  }
  return true;
}

// (a function of its own: what it keeps in registers costs the ordinary case none)
template <int TYPE, int DIM, int WAVES, bool SPLIT>
__device__ __attribute__((noinline)) void attend_block_again(PromptArgs p, uint8_t (*lds)[2][kKeys * DIM * 2],
                                                             int head, int begin, int length, int block, int first,
                                                             int end, float* part, Weights found) {
  attend_block<TYPE, DIM, WAVES, true, SPLIT>(p, lds, head, begin, length, block, first, end, part, found);
}

// How a workgroup finds its block: in the list, or among few sequences; SPLIT: the
// same, and a part of it.
enum { kListed, kSearched, kSplit };

// Floats of a part: its rows' sums, references and sums of weights.
template <int DIM, int ROWS>
constexpr int64_t kPart = (DIM + 2) * ROWS;

// Two or three wavefronts a SIMD, heads of 64 channels: 29 ragged prompts 352 and 332 us,
// 12,001 tokens 721 and 691, 33 tokens 8.5 and 6.7.  Those of 128 channels have registers
// for two.
template <int TYPE, int DIM, int WAVES, int HOW>
__global__ __launch_bounds__(64 * WAVES, DIM == 64 ? 3 : 2) void prompt_attention(PromptArgs p, const Item* items) {
  // of two tiles: K, V.  (Memory of a size given at the launch: reads of an array of
  // the kernel's own are made to wait for all loads on their way to it, those of the
  // next tiles among them.)
  extern __shared__ __attribute__((aligned(1024))) uint8_t stages[];
  auto lds = reinterpret_cast<uint8_t (*)[2][kKeys * DIM * 2]>(stages);
  constexpr int kRows = 32 * WAVES;
  constexpr bool kParts = HOW == kSplit;
  const int head = blockIdx.x % p.n_heads;
  int at = blockIdx.x / p.n_heads;
  if (HOW == kSearched && at >= p.second) at = p.second + (int)gridDim.x / p.n_heads - 1 - at;
  const int n_items = kParts ? gridDim.x / p.n_heads / p.n_parts : 0, which = kParts ? at / n_items : 0;
  Item item;
  if (HOW == kListed) {
    item = items[at];
    if (item.none) return;
  } else if (!find_block<kRows>(p, kParts ? at % n_items : at, item)) {
    return;
  }
  const int first = which * p.part_tiles;
  const int end = which + 1 < p.n_parts ? first + p.part_tiles : INT32_MAX;  // (the last one takes the rest)
  float* part = nullptr;
  if (kParts) {
    if (first >= tiles_of<kRows>(p, item.length, item.block)) return;
    part = p.parts + ((int64_t)(at % n_items * p.n_heads + head) * p.n_parts + which) * kPart<DIM, kRows>;
  }
  Weights found;
  if (!attend_block<TYPE, DIM, WAVES, false, kParts>(p, lds, head, item.begin, item.length, item.block, first, end, part, found))
    attend_block_again<TYPE, DIM, WAVES, kParts>(p, lds, head, item.begin, item.length, item.block, first, end, part, found);
}

// Joins the parts of a block: sums and sums of weights, brought to the largest
// reference.  A workgroup per 32 rows, 8 of them a wavefront, a row to 8 lanes, which
// have 4 channels of 32 each.
template <int TYPE, int DIM, int WAVES>
__global__ __launch_bounds__(256) void prompt_join(PromptArgs p) {
  constexpr int kRows = 32 * WAVES, kTimes = DIM / 32;
  const int at = blockIdx.x / WAVES, head = at % p.n_heads, lane = threadIdx.x & 63;
  const int in = blockIdx.x % WAVES * 32 + (threadIdx.x >> 6) * 8 + lane % 8;
  Item item;
  if (!find_block<kRows>(p, at / p.n_heads, item)) return;
  const int row = item.block * kRows + in;
  if (row >= item.length * p.group) return;
  const int parts = min((tiles_of<kRows>(p, item.length, item.block) + p.part_tiles - 1) / p.part_tiles, p.n_parts);
  const float* from = p.parts + (int64_t)at * p.n_parts * kPart<DIM, kRows> + in;
  float top = from[DIM * kRows];
#pragma unroll 4
  for (int i = 1; i < parts; ++i) top = fmaxf(top, from[i * kPart<DIM, kRows> + DIM * kRows]);
  v4f sum[kTimes];
  float total, share = 1.0f;
  // What the parts' sums are multiplied by, and their sums of weights; share: of all.
  auto add_up = [&] {
#pragma unroll
    for (int k = 0; k < kTimes; ++k) sum[k] = v4f{};
    total = 0.0f;
#pragma unroll 2
    for (int i = 0; i < parts; ++i) {
      const float* x = from + i * kPart<DIM, kRows>;
      const float weights = x[(DIM + 1) * kRows], by = __builtin_amdgcn_exp2f(x[DIM * kRows] - top);
      total = fmaf(fabsf(weights), by, total);
      const float times = (weights < 0.0f ? -weights * by : by) * share;
#pragma unroll
      for (int k = 0; k < kTimes; ++k) {
        const v4f four = *reinterpret_cast<const v4f*>(x - in + ((int64_t)(k * 8 + lane / 8) * kRows + in) * 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[k][e] = fmaf(four[e], times, sum[k][e]);
      }
    }
  };
  add_up();
  const float by = 1.0f / total;
  bool fine = true;
#pragma unroll
  for (int k = 0; k < kTimes; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      fine &= fabsf(sum[k][e]) < kInf;
      sum[k][e] *= by;
    }
  if (TYPE == AS_BF16 && !fine) {  // as in a block's second pass: divided before they are added up
    v4f before[kTimes];
#pragma unroll
    for (int k = 0; k < kTimes; ++k) before[k] = sum[k];
    share = by;
    add_up();
#pragma unroll
    for (int k = 0; k < kTimes; ++k)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (fabsf(before[k][e]) < kInf) sum[k][e] = before[k][e];
  }
  const int query = row / p.group;
  uint16_t* to =
      p.out + ((int64_t)(item.begin + query) * p.n_heads * p.group + head * p.group + row - query * p.group) * DIM;
#pragma unroll
  for (int k = 0; k < kTimes; ++k)
    *reinterpret_cast<v2u*>(to + (k * 8 + lane / 8) * 4) =
        v2u{pack_two<TYPE>(sum[k][0], sum[k][1]), pack_two<TYPE>(sum[k][2], sum[k][3])};
}

constexpr int kPromptWaves = 4;

// Blocks that there can be at most: a part of one for each sequence.
int64_t prompt_items(int64_t n_tokens, int64_t n_seqs, int64_t group) {
  return n_tokens * group / (32 * kPromptWaves) + std::min(n_seqs, n_tokens);
}

// A list costs a launch and takes any number; without one a wavefront finds its block
// among 64 sequences in registers.  With the list and without, one prompt of 33 tokens
// 9.0 and 6.7 us, 8 of 200 20.1 and 16.3, 64 of 700 81 and 74, 29 ragged ones 324 and 332.
bool prompt_planned(int64_t n_seqs) { return n_seqs > 64; }

// Where there are few blocks, the longest of which take much longer than all of them
// would together, they are split into parts of so many tiles of keys, and joined by
// another launch.  Lengths are on the device: the host counts as if all tokens were one
// prompt's, or the longest of several nearly twice as long as they are on average.  Not split,
// a block takes 9 us and 1.1 for each of its tiles; split, all take 22 us and 2 for each of a
// workgroup's share of all tiles.  Not split and split, heads of 128 channels: 12,000 tokens
// of one head 208 and 63 us, of 6000 of 4 in a group 109 and 64, 1500 of 8 heads 36 and 28;
// of 2048 tokens of 32 heads in groups of 4 52 and 59, which the rule leaves whole.
struct Split {
  int tiles, parts;  // 0: not split
};
Split prompt_split(int64_t n_tokens, int64_t n_seqs, int64_t n_heads, int64_t group) {
  if (prompt_planned(n_seqs)) return {0, 0};
  const int64_t room = 2 * as_host::compute_units(), blocks = (n_tokens * group + 127) / 128;
  const int64_t longest = (2 * n_tokens / (n_seqs + 1) + kKeys - 1) / kKeys;
  const int64_t share = (n_heads * blocks * (longest + 1) / 2 + room - 1) / room;
  if (11 * longest <= 130 + 20 * share) return {0, 0};
  const int64_t tiles = std::max<int64_t>(4, share + share / 3 + 2);
  return {(int)tiles, (int)((longest + tiles - 1) / tiles)};
}

template <int TYPE, int DIM>
void launch_prompt(PromptArgs p, void* workspace, hipStream_t s) {
  const int n = (int)prompt_items(p.n_tokens, p.n_seqs, p.group);
  const dim3 g((unsigned)(n * p.n_heads)), t(64 * kPromptWaves);
  constexpr size_t kLds = 4 * kKeys * DIM * 2;
  static_assert(kLds <= 64 * 1024, "more has to be allowed for a kernel");
  const Split split = prompt_split(p.n_tokens, p.n_seqs, p.n_heads, p.group);
  if (prompt_planned(p.n_seqs)) {
    Item* items = reinterpret_cast<Item*>(workspace);
    hipLaunchKernelGGL((prompt_plan<32 * kPromptWaves>), dim3(1), dim3(kPlanThreads), 0, s, p, items, n);
    hipLaunchKernelGGL((prompt_attention<TYPE, DIM, kPromptWaves, kListed>), g, t, kLds, s, p, items);
  } else if (split.tiles) {
    p.part_tiles = split.tiles, p.n_parts = split.parts, p.parts = reinterpret_cast<float*>(workspace);
    hipLaunchKernelGGL((prompt_attention<TYPE, DIM, kPromptWaves, kSplit>), dim3(g.x * split.parts), t, kLds, s, p, nullptr);
    hipLaunchKernelGGL((prompt_join<TYPE, DIM, kPromptWaves>), dim3(g.x * kPromptWaves), dim3(256), 0, s, p);
  } else {
    // Where all blocks run at once, two to a compute unit, the second ones are taken in
    // the opposite order, so that the longest are with the shortest (heads of 128 channels
    // in groups of 4 or 8: 1500 tokens 42.3 us and so 40.3, 2000 56 and 53, 1000 of 64 heads
    // 32.8 and 31.5; of 64 channels, three to a unit, 2048 37.4 and 37.8).
    const int64_t cus = as_host::compute_units();
    p.second = DIM == 128 && g.x > cus && g.x <= 2 * cus + 64 ? (int)(cus / p.n_heads) : INT32_MAX;
    hipLaunchKernelGGL((prompt_attention<TYPE, DIM, kPromptWaves, kSearched>), g, t, kLds, s, p, nullptr);
  }
}

}  // namespace as_ops

using namespace as_ops;

extern "C" {

int64_t as_attention_prompt_workspace(int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t n_seqs) {
  if (n_tokens < 1 || n_kv_heads < 1 || n_q_heads < n_kv_heads || n_seqs < 1) return 0;
  const int64_t group = n_q_heads / n_kv_heads, n = prompt_items(n_tokens, n_seqs, group);
  if (prompt_planned(n_seqs)) return round_up(n * (int64_t)sizeof(Item), 256);
  const Split split = prompt_split(n_tokens, n_seqs, n_kv_heads, group);
  return round_up(n * n_kv_heads * split.parts * kPart<128, 32 * kPromptWaves> * (int64_t)sizeof(float), 256);
}

int as_attention_prompt(const void* q, const void* k, const void* v, int32_t type, int64_t n_tokens,
                        int32_t n_q_heads, int32_t n_kv_heads, int32_t dim, int64_t q_token, int64_t k_token,
                        int64_t v_token, const int32_t* offsets, int32_t n_seqs, float scale, void* out, void* workspace,
                        int64_t workspace_bytes, void* stream) {
  if (type != AS_BF16 && type != AS_F16) return fail(AS_E_INVALID_ARG, "attention_prompt: type %d", type);
  if (dim != 64 && dim != 128) return fail(AS_E_LIMITS, "attention_prompt: heads of %d channels (64 or 128)", dim);
  if (n_tokens < 0 || n_seqs < 0 || n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % n_kv_heads)
    return fail(AS_E_INVALID_ARG, "attention_prompt: %lld tokens, %d sequences, %d query heads of %d key/value heads",
                (long long)n_tokens, n_seqs, n_q_heads, n_kv_heads);
  if (q_token < 0 || k_token < 0 || v_token < 0 || q_token % 8 || k_token % 8 || v_token % 8)
    return fail(AS_E_INVALID_ARG, "attention_prompt: strides %lld, %lld and %lld (multiples of 8)", (long long)q_token,
                (long long)k_token, (long long)v_token);
  if (!(scale > 0.0f) || scale > 2e38f) return fail(AS_E_INVALID_ARG, "attention_prompt: scale %g", (double)scale);
  const int group = n_q_heads / n_kv_heads;
  // (a workgroup of 256 threads each, fewer than 2^32 in all)
  if (n_tokens > (1 << 26) || n_seqs > (1 << 20) || n_q_heads > 4096 || n_tokens * n_q_heads > (1 << 30) ||
      prompt_items(n_tokens, n_seqs, group) * n_kv_heads >= (1 << 24) ||
      k_token > (1 << 26) || v_token > (1 << 26))
    return fail(AS_E_LIMITS, "attention_prompt: %lld tokens of %d heads in %d sequences, keys and values %lld and %lld apart",
                (long long)n_tokens, n_q_heads, n_seqs, (long long)k_token, (long long)v_token);
  if (n_tokens == 0 || n_seqs == 0) return as_host::ok();
  if (!q || !k || !v || !offsets || !out) return fail(AS_E_INVALID_ARG, "attention_prompt: null pointer");
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 8))
    return fail(AS_E_INVALID_ARG, "attention_prompt: queries, keys and values aligned to 16 bytes, outputs to 8");
  const int64_t need = as_attention_prompt_workspace(n_tokens, n_q_heads, n_kv_heads, n_seqs);
  if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 256))))
    return fail(AS_E_INVALID_ARG, "attention_prompt: workspace of %lld bytes, %lld needed (aligned to 256)",
                (long long)workspace_bytes, (long long)need);
  const uintptr_t out0 = (uintptr_t)out, out1 = out0 + (uintptr_t)(n_tokens * n_q_heads * dim * 2);
  auto meets = [&](const void* x, int64_t token, int heads) {
    return (uintptr_t)x < out1 && out0 < (uintptr_t)x + (uintptr_t)(((n_tokens - 1) * token + (int64_t)heads * dim) * 2);
  };
  if (meets(q, q_token, n_q_heads) || meets(k, k_token, n_kv_heads) || meets(v, v_token, n_kv_heads))
    return fail(AS_E_INVALID_ARG, "attention_prompt: outputs share memory with queries, keys or values");
  PromptArgs p{};
  p.q = reinterpret_cast<const uint16_t*>(q);
  p.k = reinterpret_cast<const uint16_t*>(k);
  p.v = reinterpret_cast<const uint16_t*>(v);
  p.out = reinterpret_cast<uint16_t*>(out);
  p.q_token = q_token;
  p.k_token = k_token;
  p.v_token = v_token;
  p.offsets = offsets;
  p.n_tokens = (int32_t)n_tokens;
  p.n_seqs = n_seqs;
  p.n_heads = n_kv_heads;
  p.group = group;
  p.factor = scale * 1.44269504f;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (type == AS_BF16)
    dim == 64 ? launch_prompt<AS_BF16, 64>(p, workspace, s) : launch_prompt<AS_BF16, 128>(p, workspace, s);
  else
    dim == 64 ? launch_prompt<AS_F16, 64>(p, workspace, s) : launch_prompt<AS_F16, 128>(p, workspace, s);
  return launched("attention_prompt");
}

}  // extern "C"
