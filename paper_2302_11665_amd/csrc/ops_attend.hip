// Attention of a step's queries over a cache held in 4 bits, and the attention
// weight that every cached token gets (alpaserve_ops.h).
//
// A group's value is code * d + m, so with codes c
//   q.k     = sum over groups of  d (sum q c) + m (sum q)
//   sum p v = sum over tokens of  (p d) c + p m
// and the codes enter v_mfma_f32_16x16x32 as 16 + c, which a shift, a mask and
// an or make of 4 bits (bf16 holds 16..31 in steps of 1/8, fp16 in steps of
// 1/64); the 16 is taken out in fp32: the first product starts from -16 sum q.
// Queries are exact in the first product; p d enters the second as two bf16
// numbers, whose sum P is p d but for the last 7 of its 24 bits.  With 23.5 the
// mean of 16 + c,
//   sum p v = sum P (16 + c) - 23.5 sum P + sum p (m + 7.5 d):
// what P leaves is multiplied by c - 7.5 rather than 16 + c, and the last sum's
// terms are near the group's mean, so it loses nothing.  The matrix instructions
// make the second sum too, from the same operands.  The first grows with the
// slots and not with the result, hence it is kept for 8 blocks only, and its sum
// for a group of channels brought back by the other two (kRebase below).
//
// The products are K q^T and V^T p^T: the queries that share a key/value head
// are the 16 columns.  A lane of the first product's result then holds, for one
// query, the slots 4 g + 0..3 (g = lane / 16) of each 16, which are the slots
// that the same lane has to supply to the second: p never leaves its lane, and a
// word of V holds the channel's codes for just those 8 slots.  A query's running
// maximum is the same in its four lanes, its sum is kept per lane.
#include <type_traits>

#include "ops_common.hpp"

using as_host::fail;

namespace as_ops {

constexpr int kWaves = 4;
constexpr float kFloor = -1e30f;  // running maximum before any slot was seen

struct AttArgs {
  CacheArgs c;
  const uint16_t* q;
  int64_t q_seq, q_token;
  const int32_t* length;
  void* out;
  float* part_o;   // [workgroups][2][16 tiles][dim], not normalised
  float* part_ml;  // [workgroups][2][16 tiles][2]: maximum (log2 units), sum
  float* row_ml;   // [n_seqs * n_heads][rows][2] for the weights: maximum, 1 / sum
  const float* acc_in;
  float* acc_out;
  float c_log2;      // scale * log2(e)
  uint32_t page_mul; // page_magic of the cache's pages
  int32_t n_queries, per, rows;
  int32_t row_groups, row_span;  // parts of 16 tiles query rows
  int32_t workgroups, weigh_workgroups;
  int32_t round, weigh_round;  // log2 of a round's blocks
  int32_t least;               // rounds of a share, at least
};

// ---------------------------------------------------------------- 4-bit codes

// 16 + c of a word's eight codes, as bf16 or fp16 pairs.  The two constants are
// made once, out of the compiler's sight: with their values unknown, mask and
// or become one instruction.
template <int TYPE>
struct Expand {
  uint32_t sixteen = TYPE == AS_BF16 ? 0x41804180u : 0x4c004c00u;
  uint32_t mask = TYPE == AS_BF16 ? 0x00780078u : 0x03c003c0u;
  __device__ __forceinline__ Expand() {
    asm("" : "+v"(sixteen));
    asm("" : "+s"(mask));
  }
  __device__ __forceinline__ v4u operator()(uint32_t w) const {
    if (TYPE == AS_BF16)
      return v4u{((w << 3) & mask) | sixteen, ((w >> 1) & mask) | sixteen, ((w >> 5) & mask) | sixteen,
                 ((w >> 9) & mask) | sixteen};
    return v4u{((w << 6) & mask) | sixteen, ((w << 2) & mask) | sixteen, ((w >> 2) & mask) | sixteen,
               ((w >> 6) & mask) | sixteen};
  }
};

template <int TYPE>
__device__ __forceinline__ v4f mfma(v4u a, v4u b, v4f c) {
  if (TYPE == AS_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0,
                                                   0);
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// fma(x, y, z) in fp32 with y the scale (low half) or the minimum (high half)
// of a word; the conversion is part of the instruction.
__device__ __forceinline__ float fma_d(float x, uint32_t w, float z) {
  return fmaf(x, (float)__builtin_bit_cast(v2h, w)[0], z);
}
__device__ __forceinline__ float fma_m(float x, uint32_t w, float z) {
  return fmaf(x, (float)__builtin_bit_cast(v2h, w)[1], z);
}

// Row (page and head) of a block of 32 slots of a sequence, or -1; at: its
// first slot's place on the page.
__device__ __forceinline__ int64_t block_row(const AttArgs& p, int b, int h, int blk, int& at) {
  const int pb = page_index(blk, p.page_mul);
  at = blk * 32 - pb * p.c.page;
  return cache_row(p.c, b, h, pb);
}

// A wavefront's ring in LDS: each stage takes 32 slots of a head, which come
// straight from memory.  A lane's words lie 64 bytes from its neighbour's in
// K, and the scales are the same for 16 lanes: as loads into registers these
// cost the vector cache several times the cycles of a contiguous KiB, so the
// lanes take them out of LDS instead.  The 16-byte pieces of K's slots are
// turned by the slot's number, which spreads a read of one piece of many slots
// over the banks.
template <int DIM, int GROUP, bool WITH_V>
struct Stage {
  static constexpr int kNG = DIM / GROUP;
  static constexpr int kWords = 32 * DIM / 2;                    // bytes of 32 slots' codes
  static constexpr int kParAt = WITH_V ? 2 * kWords : kWords;
  static constexpr int kBytes = kParAt + (WITH_V ? 2 : 1) * kNG * 128;
  static constexpr int kLoads = kParAt / 1024 + (WITH_V ? 2 : 1);

  // Load 16 bytes a lane from a place that all lanes share plus the lane's own offset.
  __device__ static __forceinline__ void load16(const void* base, uint32_t offset, uint8_t* dst) {
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) void*)(reinterpret_cast<const uint8_t*>(base) + offset),
        (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
  }

  // Start the loads of a block; row < 0 (no such page) loads the pool's first
  // one, which is not used.
  __device__ static __forceinline__ void bring(const AttArgs& p, int64_t row, int at, uint32_t lane, uint8_t* lds) {
    if (row < 0) row = 0, at = 0;
    const int64_t words = (row * p.c.page + at) * (DIM / 8), pars = row * kNG * p.c.page + at;
#pragma unroll
    for (int j = 0; j < kWords / 1024; ++j) {
      const uint32_t piece = 64 * j + lane;
      load16(p.c.k + words, (DIM == 128 ? piece ^ (piece >> 3 & 3) : piece) * 16, lds + j * 1024);
    }
    if (WITH_V) {
#pragma unroll
      for (int j = 0; j < kWords / 1024; ++j)
        load16(p.c.v + words, j * 1024 + lane * 16, lds + kWords + j * 1024);
    }
    if (lane < kNG * 8) {
      const uint32_t offset = (lane >> 3) * (uint32_t)p.c.page * 4 + (lane & 7) * 16;
      load16(p.c.k_par + pars, offset, lds + kParAt);
      if (WITH_V) load16(p.c.v_par + pars, offset, lds + kParAt + kNG * 128);
    }
  }

  // A lane's words of K of slot 16 t + lane % 16, and the scales of group n of
  // slots 16 t + 4 (lane / 16) + 0..3.
  __device__ static __forceinline__ void keys(const uint8_t* lds, int lane, int t, uint32_t (&k)[DIM / 32]) {
    const int s = 16 * t + (lane & 15), g = lane >> 4;
    if (DIM == 128) {
      const v4u w = *reinterpret_cast<const v4u*>(lds + s * 64 + (g ^ (s >> 1 & 3)) * 16);
#pragma unroll
      for (int i = 0; i < DIM / 32; ++i) k[i] = w[i];
    } else {
      const v2u w = *reinterpret_cast<const v2u*>(lds + s * 32 + g * 8);
#pragma unroll
      for (int i = 0; i < DIM / 32; ++i) k[i] = w[i];
    }
  }
  __device__ static __forceinline__ v4u key_scales(const uint8_t* lds, int lane, int t, int n) {
    return *reinterpret_cast<const v4u*>(lds + kParAt + n * 128 + t * 64 + (lane >> 4) * 16);
  }
  // A lane's words of V: channels 16 i + lane % 16 for the i of group n.
  __device__ static __forceinline__ void values(const uint8_t* lds, int lane, int n, uint32_t (&v)[GROUP / 16]) {
    const uint8_t* at = lds + kWords + lane * (DIM / 4) + n * (GROUP / 4);
    if (GROUP == 32) {
      const v2u w = *reinterpret_cast<const v2u*>(at);
      v[0] = w[0], v[1] = w[1];
    } else {
#pragma unroll
      for (int j = 0; j < GROUP / 64; ++j) {
        const v4u w = *reinterpret_cast<const v4u*>(at + 16 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[4 * j + i] = w[i];
      }
    }
  }
  __device__ static __forceinline__ v4u value_scales(const uint8_t* lds, int lane, int t, int n) {
    return key_scales(lds, lane, t, kNG + n);
  }
};

// Sixteen queries as the second operand of K q^T: lane's channels 32 i + 8 g +
// 0..7 of query row lane % 16; the sums over each group's channels.
template <int TYPE, int DIM, int GROUP>
struct Queries {
  v4u q[DIM / 32];
  float sum[DIM / GROUP];
  int limit;  // slots that the query sees
};

template <int TYPE, int DIM, int GROUP>
__device__ __forceinline__ void load_queries(const AttArgs& p, int b, int h, int row, int n, int lane,
                                             Queries<TYPE, DIM, GROUP>& x) {
  const int t = row / p.per;
  const uint16_t* q = p.q + b * p.q_seq + t * p.q_token + (int64_t)(h * p.per + row - t * p.per) * DIM + (lane >> 4) * 8;
  // rows beyond the last are zero and see what the last sees; they are not stored
  x.limit = n - p.n_queries + (row < p.rows ? t : p.n_queries - 1) + 1;
#pragma unroll
  for (int i = 0; i < DIM / 32; ++i)
    x.q[i] = row < p.rows ? *reinterpret_cast<const v4u*>(q + 32 * i) : v4u{0, 0, 0, 0};
}
// The sums, once the loads are under way and others after them.
template <int TYPE, int DIM, int GROUP>
__device__ __forceinline__ void sum_queries(Queries<TYPE, DIM, GROUP>& x) {
#pragma unroll
  for (int g = 0; g < DIM / GROUP; ++g) {
    float s = 0.0f;
#pragma unroll
    for (int i = g * (GROUP / 32); i < (g + 1) * (GROUP / 32); ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s += to_f32<TYPE>(x.q[i][j] & 0xffffu) + to_f32<TYPE>(x.q[i][j] >> 16);
    x.sum[g] = sum_over_rows(s);
  }
}

// q.k of the lane's query and 2 x 4 slots.
template <int TYPE, int DIM, int GROUP>
__device__ __forceinline__ void scores(const v4u (&kf)[DIM / 32], const v4u (&par)[DIM / GROUP],
                                       const Queries<TYPE, DIM, GROUP>& q, float (&s)[4]) {
#pragma unroll
  for (int g = 0; g < DIM / GROUP; ++g) {
    const float c = -16.0f * q.sum[g];
    v4f a = {c, c, c, c};
#pragma unroll
    for (int i = g * (GROUP / 32); i < (g + 1) * (GROUP / 32); ++i) a = mfma<TYPE>(kf[i], q.q[i], a);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[r] = fma_m(q.sum[g], par[g][r], g == 0 ? 0.0f : s[r]);
      s[r] = fma_d(a[r], par[g][r], s[r]);
    }
  }
}

__device__ __forceinline__ int clamped_length(const AttArgs& p, int b) {
  const int64_t cap = (int64_t)p.c.max_pages * p.c.page;
  return (int)max((int64_t)0, min((int64_t)p.length[b], cap));
}

// ---------------------------------------------------------------- attention

// The compiler's scheduler stays on its side of this: a block's steps one after
// the other need half the registers that they take when mixed, and the other
// wavefronts of the SIMD fill the gaps.
__device__ __forceinline__ void phase() { __builtin_amdgcn_sched_barrier(0); }

// Sums over the slots that a wavefront has seen, for 16 NT queries.
template <int DIM, int GROUP, int NT>
struct Sums {
  v4f o[NT][DIM / 16];
  float shift[NT][DIM / GROUP];  // a quarter of -23.5 sum P, plus the lane's slots' sum of p (m + 7.5 d)
  float mref[NT], sum[NT];       // reference of the exponents (log2 units), sum of p over the lane's slots
};

template <int DIM, int GROUP, int NT>
__device__ __forceinline__ void clear(Sums<DIM, GROUP, NT>& a, int t) {
  a.mref[t] = kFloor;
  a.sum[t] = 0.0f;
#pragma unroll
  for (int g = 0; g < DIM / GROUP; ++g) a.shift[t][g] = 0.0f;
#pragma unroll
  for (int i = 0; i < DIM / 16; ++i) a.o[t][i] = v4f{0, 0, 0, 0};
}

// o as it is without the 16 of the codes: the four lanes' shifts are added to it.
// Once in kRebase blocks (6 instructions a group and one a register of o): its
// own rounding then stays that of a sum of 256 slots, not of all.  Nearly flat
// attention of one wavefront over 65,536 slots is off by 2.6e-3 of the result
// without this, by 1e-5 so, and by 3e-6 with every block's sum.
constexpr int kRebase = 8;

template <int DIM, int GROUP, int NT>
__device__ __forceinline__ void rebase(Sums<DIM, GROUP, NT>& a) {
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int g = 0; g < DIM / GROUP; ++g) {
      const float add = sum_over_rows(a.shift[t][g]);
#pragma unroll
      for (int i = g * (GROUP / 16); i < (g + 1) * (GROUP / 16); ++i) a.o[t][i] += add;
      a.shift[t][g] = 0.0f;
    }
}

// A quarter of -23.5 times the sum of a block's P, in every lane of a query.
__device__ __forceinline__ float mean_shift(v4u hi, v4u lo) {
  constexpr uint32_t kMean = 0xc0bcc0bcu;  // -5.875, exact in bf16
  const v4u mean = {kMean, kMean, kMean, kMean};
  return mfma<AS_BF16>(mean, lo, mfma<AS_BF16>(mean, hi, v4f{0, 0, 0, 0}))[0];
}

// The q.k of a lane's 8 slots of a block to p, the sums so far scaled where the
// reference moves.
template <int TYPE, int DIM, int GROUP, int NT, bool RAGGED>
__device__ __forceinline__ void softmax_block(const AttArgs& p, int slot0, int limit, int u, float (&s)[8],
                                              Sums<DIM, GROUP, NT>& a) {
  if (RAGGED) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (slot0 + 16 * (e >> 2) + (e & 3) >= limit) s[e] = -kInf;
  }
  const float top = p.c_log2 * fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])),
                                     fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
  // The reference follows the maximum only where it is passed by a factor of
  // 2^8: sums and products stay far from fp32's range, and the sums so far are
  // hardly ever scaled.
  if (__any(top > a.mref[u] + 8.0f)) {
    const float m = fmaxf(a.mref[u], max_over_rows(top));
    const float f = __builtin_amdgcn_exp2f(a.mref[u] - m);
    a.mref[u] = m;
    a.sum[u] *= f;
#pragma unroll
    for (int g = 0; g < DIM / GROUP; ++g) a.shift[u][g] *= f;
#pragma unroll
    for (int i = 0; i < DIM / 16; ++i) a.o[u][i] *= f;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], p.c_log2, -a.mref[u]));
    a.sum[u] += s[e];
  }
}

// Two numbers as pairs of bf16: the nearest, and the nearest to what it leaves.
__device__ __forceinline__ v2u split_bf16(float x, float y) {
  const uint32_t hi = pack_bf16(x, y);
  return v2u{hi, pack_bf16(x - __uint_as_float(hi << 16), y - __uint_as_float(hi & 0xffff0000u))};
}

// 32 slots more; RAGGED: some are not seen by some query.
template <int TYPE, int DIM, int GROUP, int NT, bool RAGGED>
__device__ __forceinline__ void attend_block(const AttArgs& p, int blk, int lane,
                                             const Queries<TYPE, DIM, GROUP> (&q)[NT], const uint8_t* lds,
                                             const Expand<TYPE>& key_codes, const Expand<AS_BF16>& value_codes,
                                             Sums<DIM, GROUP, NT>& a) {
  constexpr int NG = DIM / GROUP;
  typedef Stage<DIM, GROUP, true> S;
  float s[NT][8];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    uint32_t k[DIM / 32];
    S::keys(lds, lane, t, k);
    v4u kf[DIM / 32], par[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) par[g] = S::key_scales(lds, lane, t, g);
#pragma unroll
    for (int i = 0; i < DIM / 32; ++i) kf[i] = key_codes(k[i]);
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      float x[4];
      scores<TYPE, DIM, GROUP>(kf, par, q[u], x);
#pragma unroll
      for (int r = 0; r < 4; ++r) s[u][4 * t + r] = x[r];
    }
    phase();
  }
  const int slot0 = blk * 32 + (lane >> 4) * 4;
#pragma unroll
  for (int u = 0; u < NT; ++u) softmax_block<TYPE, DIM, GROUP, NT, RAGGED>(p, slot0, q[u].limit, u, s[u], a);
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    phase();
    v4u par[2], hi[NT], lo[NT];
#pragma unroll
    for (int t = 0; t < 2; ++t) par[t] = S::value_scales(lds, lane, t, g);
    uint32_t v[GROUP / 16];
    S::values(lds, lane, g, v);
#pragma unroll
    for (int u = 0; u < NT; ++u) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float pd[2];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int e = 2 * j + z;
          uint32_t w = par[e >> 2][e & 3];
          // a slot that is not seen may hold anything, infinities and NaN too
          if (RAGGED && slot0 + 16 * (e >> 2) + (e & 3) >= q[u].limit) w = 0;
          pd[z] = fma_d(s[u][e], w, 0.0f);
          a.shift[u][g] = fma_m(s[u][e], w, a.shift[u][g]);
          a.shift[u][g] = fmaf(7.5f, pd[z], a.shift[u][g]);
        }
        const v2u two = split_bf16(pd[0], pd[1]);
        hi[u][j] = two[0], lo[u][j] = two[1];
      }
      a.shift[u][g] += mean_shift(hi[u], lo[u]);
    }
#pragma unroll
    for (int i = 0; i < GROUP / 16; ++i) {
      if (i % 4 == 0) phase();
      const v4u vf = value_codes(v[i]);
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        v4f& o = a.o[u][g * (GROUP / 16) + i];
        o = mfma<AS_BF16>(vf, hi[u], o);
        o = mfma<AS_BF16>(vf, lo[u], o);
      }
    }
  }
}

// ----------------------------------------------------------------- the shares

// A segment is what 16 NT query rows of one head see of one sequence, in blocks
// of 32 slots, and a round what a workgroup does of it at once: a block for each
// wavefront, or one block that all of them work at.  The rounds of all sequences,
// heads and row groups, one after the other, are dealt to the workgroups in
// shares of one size, whatever the lengths.  All workgroups run at once: there is
// no tail, and none is started for slots that a table has room for but a sequence
// does not use.  A segment that lies within a share is finished there; of another
// one, each workgroup leaves its part: in place 1 the one that begins it, in
// place 0 the others.  (Shares of blocks rather than rounds put the last block
// of one segment and the first of the next into one share, which then takes two
// rounds: 10 us for 8 segments of 129 blocks, a round each.)
struct Segment {
  int b, h, rg, n;
  int blk, seen;  // first block of the share, blocks of the segment
};

// Blocks that the rows of group rg see; least: slots that the first row sees.
__device__ __forceinline__ int seen_blocks(const AttArgs& p, int n, int rg, int& least) {
  const int row0 = rg * p.row_span;
  const int last = min(n, n - p.n_queries + min(row0 + p.row_span - 1, p.rows - 1) / p.per + 1);
  least = n - p.n_queries + row0 / p.per + 1;
  return max(0, (last + 31) / 32);
}

// Rounds of so many blocks.  WEIGH: one segment of all rows.
template <bool WEIGH>
__device__ __forceinline__ uint32_t rounds(const AttArgs& p, int blocks) {
  const int log2 = WEIGH ? p.weigh_round : p.round;
  return (uint32_t)(blocks + (1 << log2) - 1) >> log2;
}

// Rounds of all segments of one head of a sequence.
template <bool WEIGH>
__device__ __forceinline__ uint32_t head_rounds(const AttArgs& p, int n) {
  if (WEIGH || p.row_groups == 1) return rounds<WEIGH>(p, (n + 31) / 32);
  uint32_t sum = 0;
  int least;
  for (int rg = 0; rg < p.row_groups; ++rg) sum += rounds<false>(p, seen_blocks(p, n, rg, least));
  return sum;
}

// 64 sequences from b0 on: the lane's length, and the sum of the rounds of the
// sequences up to and with the lane's.
struct Sequences {
  int n;
  uint32_t sum;
};
template <bool WEIGH>
__device__ __forceinline__ Sequences scan_sequences(const AttArgs& p, int b0, int lane) {
  const int b = b0 + lane;
  Sequences s;
  s.n = b < p.c.n_seqs ? clamped_length(p, b) : 0;
  s.sum = scan_lanes(head_rounds<WEIGH>(p, s.n) * (uint32_t)p.c.n_heads);
  return s;
}
__device__ __forceinline__ uint32_t all_rounds(const Sequences& s) {
  return (uint32_t)__builtin_amdgcn_readlane((int)s.sum, 63);
}

// Rounds in all, and the size of a share.  first: the scan of the first 64
// sequences.
template <bool WEIGH>
__device__ __forceinline__ uint32_t share_size(const AttArgs& p, int lane, Sequences& first, uint32_t& total) {
  first = scan_sequences<WEIGH>(p, 0, lane);
  total = all_rounds(first);
  for (int b0 = 64; b0 < p.c.n_seqs; b0 += 64) total += all_rounds(scan_sequences<WEIGH>(p, b0, lane));
  const uint32_t groups = (uint32_t)(WEIGH ? p.weigh_workgroups : p.workgroups);
  return max((total + groups - 1) / groups, WEIGH ? 1u : (uint32_t)p.least);
}

// This workgroup's share's number, or -1.  Neighbouring workgroup numbers go to
// different XCDs; each XCD gets a run of shares, which mostly read the same
// slots where a head has several row groups.
__device__ __forceinline__ int64_t share_number(uint32_t total, uint32_t size) {
  const uint32_t shares = (total + size - 1) / size, per_xcd = (shares + 7) / 8;
  const uint32_t at = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  return (blockIdx.x >> 3) < per_xcd && at < shares ? (int64_t)at : -1;
}

// The segment that holds round `unit` of all.
template <bool WEIGH>
__device__ __forceinline__ Segment locate(const AttArgs& p, uint32_t unit, int lane, const Sequences& first) {
  uint32_t before = 0;
  Sequences q = first;
  int b0 = 0;
  while (unit >= before + all_rounds(q) && b0 + 64 < p.c.n_seqs) {
    before += all_rounds(q);
    q = scan_sequences<WEIGH>(p, b0 += 64, lane);
  }
  const uint64_t past = __ballot(before + q.sum > unit);
  const int i = past ? __builtin_ctzll(past) : 0;
  if (i > 0) before += (uint32_t)__builtin_amdgcn_readlane((int)q.sum, i - 1);
  Segment s;
  s.b = b0 + i;
  s.n = __builtin_amdgcn_readlane(q.n, i);
  const uint32_t per_head = max(1u, head_rounds<WEIGH>(p, s.n));
  uint32_t off = unit - before;
  s.h = (int)(off / per_head);
  off -= (uint32_t)s.h * per_head;
  s.rg = 0;
  int least;
  s.seen = WEIGH ? (s.n + 31) / 32 : seen_blocks(p, s.n, 0, least);
  while (!WEIGH && s.rg + 1 < p.row_groups && off >= rounds<false>(p, s.seen)) {
    off -= rounds<false>(p, s.seen);
    s.seen = seen_blocks(p, s.n, ++s.rg, least);
  }
  s.blk = (int)(off << (WEIGH ? p.weigh_round : p.round));
  return s;
}

// The next segment that is not empty; there is one.
template <bool WEIGH>
__device__ __forceinline__ void advance(const AttArgs& p, Segment& s) {
  int least;
  do {
    if (WEIGH || ++s.rg == p.row_groups) {
      s.rg = 0;
      if (++s.h == p.c.n_heads) {
        s.h = 0;
        if (++s.b >= p.c.n_seqs) return;
        s.n = clamped_length(p, s.b);
      }
    }
    s.seen = WEIGH ? (s.n + 31) / 32 : seen_blocks(p, s.n, s.rg, least);
  } while (s.seen == 0);
  s.blk = 0;
}

// ------------------------------------------------------------------ the kernels

// Where a row's output is.
__device__ __forceinline__ int64_t out_index(const AttArgs& p, int b, int h, int row, int dim) {
  const int t = row / p.per;
  return (((int64_t)b * p.n_queries + t) * p.c.n_heads * p.per + h * p.per + row - t * p.per) * dim;
}

template <int TYPE>
__device__ __forceinline__ void store_row(const AttArgs& p, int64_t at, v4f x, float l) {
  const float inv = 1.0f / l;
  uint16_t* out = reinterpret_cast<uint16_t*>(p.out) + at;
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float lo = l == 0.0f ? 0.0f : x[2 * i] * inv, hi = l == 0.0f ? 0.0f : x[2 * i + 1] * inv;
    w[i] = (uint32_t)from_f32<TYPE>(lo) | (uint32_t)from_f32<TYPE>(hi) << 16;
  }
  *reinterpret_cast<v2u*>(out) = v2u{w[0], w[1]};
}

__device__ __forceinline__ void store_row_ml(const AttArgs& p, int b, int h, int row, float m, float l) {
  float* to = p.row_ml + (((int64_t)b * p.c.n_heads + h) * p.rows + row) * 2;
  to[0] = m;
  to[1] = l == 0.0f ? 0.0f : 1.0f / l;
}

constexpr int kStages = 2;
template <int DIM, int GROUP>
constexpr int attend_lds(int waves) {
  constexpr int ring = kStages * Stage<DIM, GROUP, true>::kBytes, part = 16 * (DIM + 4) * 4;
  return waves * (ring > part ? ring : part);
}

template <int TYPE, int DIM, int GROUP, int NT, int NW>
__device__ __forceinline__ void attend_segment(const AttArgs& p, const Segment& s, int take, int share, int lane,
                                               int wave, uint8_t* lds, float (*ml)[16][2]) {
  constexpr int NG = DIM / GROUP;
  typedef Stage<DIM, GROUP, true> S;
  constexpr int kRing = kStages * S::kBytes;
  const int b = s.b, h = s.h, n = s.n, row0 = s.rg * 16 * NT, end = s.blk + take;
  int least;
  seen_blocks(p, n, s.rg, least);
  uint8_t* ring = lds + wave * kRing;
  Queries<TYPE, DIM, GROUP> q[NT];
  Sums<DIM, GROUP, NT> a;
#pragma unroll
  for (int t = 0; t < NT; ++t) load_queries<TYPE, DIM, GROUP>(p, b, h, row0 + 16 * t + (lane & 15), n, lane, q[t]);
  int blk = s.blk + wave;
  uint32_t valid = 0;  // bit j: the block j turns on has a page
#pragma unroll
  for (int j = 0; j < kStages; ++j) {
    if (blk + j * NW >= end) break;
    int at;
    const int64_t row = block_row(p, b, h, blk + j * NW, at);
    valid |= (uint32_t)(row >= 0) << j;
    if (p.c.n_pages > 0) S::bring(p, row, at, lane, ring + j * S::kBytes);
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    sum_queries(q[t]);
    clear(a, t);
  }
  const Expand<TYPE> key_codes;
  const Expand<AS_BF16> value_codes;
  int slot = 0, since = 0;
  // Blocks up to `to`, all of one kind.
  auto blocks = [&](int to, auto ragged) {
    for (; blk < to; blk += NW) {
      int at = 0;
      int64_t row = -1;
      const bool more = blk + kStages * NW < end;
      if (more) row = block_row(p, b, h, blk + kStages * NW, at);
      if (blk + (kStages - 1) * NW < end)
        wait_loads<(kStages - 1) * S::kLoads>();
      else
        wait_loads<0>();
      uint8_t* here = ring + slot * S::kBytes;
      if (valid & 1)
        attend_block<TYPE, DIM, GROUP, NT, decltype(ragged)::value>(p, blk, lane, q, here, key_codes, value_codes, a);
      valid = valid >> 1 | (uint32_t)(row >= 0) << (kStages - 1);
      if (more) {
        wait_reads();
        if (p.c.n_pages > 0) S::bring(p, row, at, lane, here);
      }
      slot = slot + 1 == kStages ? 0 : slot + 1;
      if (++since == kRebase) rebase(a), since = 0;
    }
  };
  blocks(min(end, least >> 5), std::false_type());  // all 32 slots seen by all queries
  blocks(end, std::true_type());

  // Join the wavefronts, 16 rows at a time.
  float* part = reinterpret_cast<float*>(lds);  // [NW][16][DIM + 4]
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    const float total = sum_over_rows(a.sum[u]);
    __syncthreads();  // the rings, and the rows before, are done with
    if (lane < 16) {
      ml[wave][lane][0] = a.mref[u];
      ml[wave][lane][1] = total;
    }
    __syncthreads();
    float m = kFloor;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, ml[w][lane & 15][0]);
    const float f = __builtin_amdgcn_exp2f(a.mref[u] - m);
    float add[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) add[g] = sum_over_rows(a.shift[u][g]);
#pragma unroll
    for (int i = 0; i < DIM / 16; ++i)
      *reinterpret_cast<v4f*>(part + (wave * 16 + (lane & 15)) * (DIM + 4) + 16 * i + (lane >> 4) * 4) =
          (a.o[u][i] + add[i * 16 / GROUP]) * f;
    __syncthreads();
    for (int j = threadIdx.x; j < 16 * DIM / 4; j += 64 * NW) {
      const int r = j / (DIM / 4), d = j % (DIM / 4) * 4;
      const int row = row0 + 16 * u + r;
      if (row >= p.rows) continue;
      v4f x = {0, 0, 0, 0};
      float top = kFloor, l = 0.0f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        x += *reinterpret_cast<const v4f*>(part + (w * 16 + r) * (DIM + 4) + d);
        top = fmaxf(top, ml[w][r][0]);
      }
#pragma unroll
      for (int w = 0; w < NW; ++w) l += ml[w][r][1] * __builtin_amdgcn_exp2f(ml[w][r][0] - top);
      if (take == s.seen) {
        store_row<TYPE>(p, out_index(p, b, h, row, DIM) + d, x, l);
        if (p.row_ml && d == 0) store_row_ml(p, b, h, row, top, l);
      } else {
        const int64_t at = ((int64_t)share * 2 + (s.blk == 0)) * (16 * NT) + 16 * u + r;
        *reinterpret_cast<v4f*>(p.part_o + at * DIM + d) = x;
        if (d == 0) *reinterpret_cast<float2*>(p.part_ml + at * 2) = make_float2(top, l);
      }
    }
  }
  __syncthreads();  // the next segment's rings
}

// One workgroup per share; its four wavefronts take a segment's blocks in turn,
// each with a ring of its own in LDS so that none waits for another, and join
// their results at the segment's end.  Bound by memory where rows are few (128
// channels in groups of 64, 8 rows: 1.04 GB of long contexts in 212 us, 4.9 TB/s;
// 403 MB of 40 ragged ones in 96 us, 4.2), by the vector instructions of codes and
// softmax above some 16 rows, and by a round's latency, 8 us, for one short
// sequence.
// (Segments of 32 rows, so that codes are expanded once for both halves, took as
// long, 77 us for 9 sequences of up to 90,000 slots, 2 heads of 20 rows each, or
// longer: 57 us, 49 in segments of 16, for 40 rows; they leave half the wavefronts.)
template <int TYPE, int DIM, int GROUP>
__global__ __launch_bounds__(64 * kWaves, DIM == 4 * GROUP ? 3 : 4) void attend(AttArgs p) {
  __shared__ float ml[kWaves][16][2];
  extern __shared__ __align__(16) uint8_t lds[];  // the rings, then the parts to be joined
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Sequences first;
  uint32_t total;
  const uint32_t size = share_size<false>(p, lane, first, total);
  const int64_t share = share_number(total, size);
  if (share < 0) return;
  const uint32_t unit = (uint32_t)share * size;
  int left = (int)min(size, total - unit);
  Segment g = locate<false>(p, unit, lane, first);
  for (;;) {
    const int take = min(left << p.round, g.seen - g.blk);
    attend_segment<TYPE, DIM, GROUP, 1, kWaves>(p, g, take, (int)share, lane, wave, lds, ml);
    left -= (int)rounds<false>(p, take);
    if (left == 0) return;
    advance<false>(p, g);
  }
}

// Many rows: every wavefront has 32 rows of its own and all slots of the
// segment, and the four expand each block's codes together, a quarter each, into
// operands in LDS that all of them multiply with: 128 rows share the work at the
// codes, which otherwise takes half of the vector instructions.  The words of the
// next block are on their way, and the operands of the one after this are written
// while this one is multiplied; one barrier a block.  1200 rows a head of two
// sequences of up to 12,000 slots take 201 us, 0.47 PFLOP/s as the formula counts,
// 0.77 with V's second product and the means'.  Neither unit bounds it alone: the
// vector instructions take 53 % of the cycles and the matrix instructions 32 %,
// hardly ever at once, since K q^T, softmax and V p^T follow each other and a SIMD
// has two wavefronts.
constexpr int kManyRows = 128;

template <int DIM, int GROUP>
struct Operands {
  static constexpr int kNG = DIM / GROUP, kWords = DIM / 32;  // words of a lane's quarter
  static constexpr int kV = 2 * kWords * 1024;                // K's operands: [2][kWords], then V's [2 kWords]
  static constexpr int kKeyPar = 2 * kV;                      // words [kNG][32]
  static constexpr int kValuePar = kKeyPar + kNG * 128;       // words [kNG][32]
  static constexpr int kValueMean = kValuePar + kNG * 128;    // m + 7.5 d, fp32 [kNG][32]
  static constexpr int kBytes = kValueMean + kNG * 128;

  uint32_t words[kWords], par;  // this wavefront's quarter of a block

  __device__ __forceinline__ void fetch(const AttArgs& p, int64_t row, int at, int lane, int wave) {
    if (row < 0) row = 0, at = 0;
    const uint32_t* from = wave < 2 ? p.c.k + (row * p.c.page + at + 16 * wave + (lane & 15)) * (DIM / 8) + (lane >> 4) * kWords
                                    : p.c.v + (row * p.c.page + at) * (DIM / 8) + lane * (2 * kWords) + (wave - 2) * kWords;
    if (kWords == 4) {
      const v4u w = *reinterpret_cast<const v4u*>(from);
#pragma unroll
      for (int i = 0; i < kWords; ++i) words[i] = w[i];
    } else {
      const v2u w = *reinterpret_cast<const v2u*>(from);
#pragma unroll
      for (int i = 0; i < kWords; ++i) words[i] = w[i];
    }
    const int i = (wave & 1) * 16 * kNG + lane;  // of the 32 kNG words of K's (wave < 2) or V's scales
    if (lane < 16 * kNG)
      par = (wave < 2 ? p.c.k_par : p.c.v_par)[(row * kNG + (i >> 5)) * p.c.page + at + (i & 31)];
  }

  template <int TYPE>
  __device__ __forceinline__ void store(uint8_t* lds, int lane, int wave, const Expand<TYPE>& key_codes,
                                        const Expand<AS_BF16>& value_codes) const {
    uint8_t* to = lds + wave * kWords * 1024 + lane * 16;  // (K's tiles of 16 slots, V's halves)
#pragma unroll
    for (int i = 0; i < kWords; ++i)
      *reinterpret_cast<v4u*>(to + i * 1024) = wave < 2 ? key_codes(words[i]) : value_codes(words[i]);
    const int i = (wave & 1) * 16 * kNG + lane;
    if (lane < 16 * kNG) {
      *reinterpret_cast<uint32_t*>(lds + (wave < 2 ? kKeyPar : kValuePar) + i * 4) = par;
      if (wave >= 2) *reinterpret_cast<float*>(lds + kValueMean + i * 4) = fma_m(1.0f, par, fma_d(7.5f, par, 0.0f));
    }
  }
};

template <int TYPE, int DIM, int GROUP, bool RAGGED>
__device__ __forceinline__ void many_block(const AttArgs& p, int blk, int lane,
                                           const Queries<TYPE, DIM, GROUP> (&q)[2], const uint8_t* lds,
                                           Sums<DIM, GROUP, 2>& a) {
  typedef Operands<DIM, GROUP> O;
  constexpr int NG = DIM / GROUP;
  float s[2][8];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    v4u kf[DIM / 32], par[NG];
#pragma unroll
    for (int i = 0; i < DIM / 32; ++i)
      kf[i] = *reinterpret_cast<const v4u*>(lds + (t * (DIM / 32) + i) * 1024 + lane * 16);
#pragma unroll
    for (int g = 0; g < NG; ++g)
      par[g] = *reinterpret_cast<const v4u*>(lds + O::kKeyPar + g * 128 + t * 64 + (lane >> 4) * 16);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      float x[4];
      scores<TYPE, DIM, GROUP>(kf, par, q[u], x);
#pragma unroll
      for (int r = 0; r < 4; ++r) s[u][4 * t + r] = x[r];
    }
  }
  const int slot0 = blk * 32 + (lane >> 4) * 4;
#pragma unroll
  for (int u = 0; u < 2; ++u) softmax_block<TYPE, DIM, GROUP, 2, RAGGED>(p, slot0, q[u].limit, u, s[u], a);
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    v4u par[2], hi[2], lo[2];
    v4f mean[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      par[t] = *reinterpret_cast<const v4u*>(lds + O::kValuePar + g * 128 + t * 64 + (lane >> 4) * 16);
      mean[t] = *reinterpret_cast<const v4f*>(lds + O::kValueMean + g * 128 + t * 64 + (lane >> 4) * 16);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float pd[2];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int e = 2 * j + z;
          uint32_t w = par[e >> 2][e & 3];
          float m = mean[e >> 2][e & 3];
          // a slot that is not seen may hold anything, infinities and NaN too
          if (RAGGED && slot0 + 16 * (e >> 2) + (e & 3) >= q[u].limit) w = 0, m = 0.0f;
          pd[z] = fma_d(s[u][e], w, 0.0f);
          a.shift[u][g] = fmaf(s[u][e], m, a.shift[u][g]);
        }
        const v2u two = split_bf16(pd[0], pd[1]);
        hi[u][j] = two[0], lo[u][j] = two[1];
      }
      a.shift[u][g] += mean_shift(hi[u], lo[u]);
    }
    // (the two products of one sum apart, so that neither waits for the other)
    constexpr int kRun = GROUP / 16 < 4 ? GROUP / 16 : 4;
#pragma unroll
    for (int i0 = 0; i0 < GROUP / 16; i0 += kRun) {
        v4u vf[kRun];
#pragma unroll
      for (int i = 0; i < kRun; ++i)
        vf[i] = *reinterpret_cast<const v4u*>(lds + O::kV + (g * (GROUP / 16) + i0 + i) * 1024 + lane * 16);
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < kRun; ++i)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            v4f& o = a.o[u][g * (GROUP / 16) + i0 + i];
            o = mfma<AS_BF16>(vf[i], half ? lo[u] : hi[u], o);
          }
    }
  }
}

template <int TYPE, int DIM, int GROUP>
__device__ __forceinline__ void many_segment(const AttArgs& p, const Segment& s, int take, int share, int lane,
                                             int wave, uint8_t* lds) {
  constexpr int NG = DIM / GROUP;
  typedef Operands<DIM, GROUP> O;
  const int b = s.b, h = s.h, n = s.n, row0 = s.rg * kManyRows + wave * 32, end = s.blk + take;
  int least;
  seen_blocks(p, n, s.rg, least);
  Queries<TYPE, DIM, GROUP> q[2];
  Sums<DIM, GROUP, 2> a;
#pragma unroll
  for (int t = 0; t < 2; ++t) load_queries<TYPE, DIM, GROUP>(p, b, h, row0 + 16 * t + (lane & 15), n, lane, q[t]);
  const Expand<TYPE> key_codes;
  const Expand<AS_BF16> value_codes;
  O quarter;
  int blk = s.blk, half = 0, since = 0;
  bool valid[2];  // of this block and the next
  auto fetch = [&](int i, bool& ok) {
    int at;
    const int64_t row = block_row(p, b, h, i, at);
    ok = row >= 0;
    if (p.c.n_pages > 0) quarter.fetch(p, row, at, lane, wave);
  };
  valid[0] = valid[1] = false;
  if (blk < end) {
    fetch(blk, valid[0]);
    quarter.store(lds, lane, wave, key_codes, value_codes);
  }
  if (blk + 1 < end) fetch(blk + 1, valid[1]);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    sum_queries(q[t]);
    clear(a, t);
  }
  lds_barrier();
  auto blocks = [&](int to, auto ragged) {
    for (; blk < to; ++blk, half ^= 1) {
      const bool here = valid[0];
      valid[0] = valid[1];
      if (blk + 1 < end) quarter.store(lds + (half ^ 1) * O::kBytes, lane, wave, key_codes, value_codes);
      if (blk + 2 < end) fetch(blk + 2, valid[1]);
      if (here) many_block<TYPE, DIM, GROUP, decltype(ragged)::value>(p, blk, lane, q, lds + half * O::kBytes, a);
      if (++since == kRebase) rebase(a), since = 0;
      lds_barrier();
    }
  };
  blocks(min(end, least >> 5), std::false_type());
  blocks(end, std::true_type());
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int in = wave * 32 + 16 * u + (lane & 15), row = s.rg * kManyRows + in, g = lane >> 4;
    const float l = sum_over_rows(a.sum[u]);
    float add[NG];
#pragma unroll
    for (int k = 0; k < NG; ++k) add[k] = sum_over_rows(a.shift[u][k]);
    if (row >= p.rows) continue;
    const int64_t at = ((int64_t)share * 2 + (s.blk == 0)) * kManyRows + in;
#pragma unroll
    for (int i = 0; i < DIM / 16; ++i) {
      const v4f x = a.o[u][i] + add[i * 16 / GROUP];
      if (take == s.seen)
        store_row<TYPE>(p, out_index(p, b, h, row, DIM) + 16 * i + 4 * g, x, l);
      else
        *reinterpret_cast<v4f*>(p.part_o + at * DIM + 16 * i + 4 * g) = x;
    }
    if (g == 0 && take == s.seen && p.row_ml) store_row_ml(p, b, h, row, a.mref[u], l);
    if (g == 0 && take != s.seen) *reinterpret_cast<float2*>(p.part_ml + at * 2) = make_float2(a.mref[u], l);
  }
}

// ALONE: a segment to a workgroup.
template <int TYPE, int DIM, int GROUP, bool ALONE>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_many(AttArgs p) {
  extern __shared__ __align__(16) uint8_t lds[];  // two blocks' operands
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (ALONE) {
    // the longest segments, which a step's last rows have, first
    const int heads = p.c.n_seqs * p.c.n_heads, bh = blockIdx.x % heads;
    Segment g;
    g.rg = p.row_groups - 1 - blockIdx.x / heads;
    g.b = bh / p.c.n_heads, g.h = bh % p.c.n_heads;
    g.n = clamped_length(p, g.b);
    g.blk = 0;
    int least;
    g.seen = seen_blocks(p, g.n, g.rg, least);
    many_segment<TYPE, DIM, GROUP>(p, g, g.seen, 0, lane, wave, lds);
    return;
  }
  Sequences first;
  uint32_t total;
  const uint32_t size = share_size<false>(p, lane, first, total);
  const int64_t share = share_number(total, size);
  if (share < 0) return;
  const uint32_t unit = (uint32_t)share * size;
  int left = (int)min(size, total - unit);
  Segment g = locate<false>(p, unit, lane, first);
  for (;;) {
    const int take = min(left << p.round, g.seen - g.blk);
    many_segment<TYPE, DIM, GROUP>(p, g, take, (int)share, lane, wave, lds);
    left -= (int)rounds<false>(p, take);
    if (left == 0) return;
    advance<false>(p, g);
  }
}

// Joins the parts of the segments that several workgroups had, four channels to
// a thread.  ROWS = 1: a workgroup joins one row, its parts side by side (few
// rows, and a long segment may have hundreds of parts); otherwise a workgroup
// joins ROWS rows of a segment, or 16.  Bound by latency: 3.6 us for 32 rows of 33
// parts, 5.4 for 320 segments of 3 parts (7.6 with a workgroup to a row), 14 for
// 1200 rows of 16 heads.
template <int TYPE, int DIM, int ROWS, int THREADS>
__global__ __launch_bounds__(THREADS) void join(AttArgs p) {
  constexpr int kSide = THREADS / (DIM / 4) / ROWS;
  __shared__ float mls[kSide][2];
  __shared__ v4f sums[kSide][DIM / 4];
  const int tid = threadIdx.x, lane = tid & 63;
  constexpr int kRun = ROWS == 1 ? 1 : 16;  // rows of a workgroup
  const int across = (p.rows + kRun - 1) / kRun;
  const int bh = blockIdx.x / across, in = blockIdx.x % across * kRun;
  const int rg = in / p.row_span;
  const int b = bh / p.c.n_heads, h = bh % p.c.n_heads;
  const int n = clamped_length(p, b);
  int least;
  const int seen = seen_blocks(p, n, rg, least);
  const int d = tid % (DIM / 4), side = tid / (DIM / 4) % kSide;
  int row = ROWS == 1 ? in : in + tid / (DIM / 4);
  const int end = min(p.rows, in + kRun);
  if (seen == 0) {  // in no workgroup's share
    if (side) return;
    for (; row < end; row += ROWS) {
      store_row<TYPE>(p, out_index(p, b, h, row, DIM) + 4 * d, v4f{0, 0, 0, 0}, 0.0f);
      if (p.row_ml && d == 0) store_row_ml(p, b, h, row, kFloor, 0.0f);
    }
    return;
  }
  // the segment's first round among all
  Sequences first;
  uint32_t total;
  const uint32_t size = share_size<false>(p, lane, first, total);
  uint32_t start = 0;
  for (int b0 = 0; b0 < b; b0 += 64) {
    if (b0) first = scan_sequences<false>(p, b0, lane);
    start += (uint32_t)__builtin_amdgcn_readlane((int)first.sum, min(63, b - 1 - b0));
  }
  start += (uint32_t)h * head_rounds<false>(p, n);
  for (int r = 0; r < rg; ++r) start += rounds<false>(p, seen_blocks(p, n, r, least));
  const int share = (int)(start / size), parts = (int)((start + rounds<false>(p, seen) - 1) / size) - share + 1;
  if (parts == 1) return;  // finished where it was
  for (; row < end; row += ROWS) {
    auto at = [&](int s) { return ((int64_t)(share + s) * 2 + (s == 0)) * p.row_span + row - rg * p.row_span; };
    float m = kFloor, l = 0.0f;
    v4f x = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = side; s < parts; s += kSide) {
      const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + at(s) * 2);
      const v4f o = *reinterpret_cast<const v4f*>(p.part_o + at(s) * DIM + 4 * d);
      const float top = fmaxf(m, ml.x), was = __builtin_amdgcn_exp2f(m - top), f = __builtin_amdgcn_exp2f(ml.x - top);
      m = top;
      l = fmaf(l, was, ml.y * f);
      x = x * was + o * f;
    }
    if (kSide > 1) {
      if (d == 0) mls[side][0] = m, mls[side][1] = l;
      sums[side][d] = x;
      __syncthreads();
      if (side) return;  // (one row to a workgroup)
#pragma unroll
      for (int s = 1; s < kSide; ++s) m = fmaxf(m, mls[s][0]);
      l = 0.0f;
      x = v4f{0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < kSide; ++s) {
        const float f = __builtin_amdgcn_exp2f(mls[s][0] - m);
        l = fmaf(mls[s][1], f, l);
        x += sums[s][d] * f;
      }
    }
    store_row<TYPE>(p, out_index(p, b, h, row, DIM) + 4 * d, x, l);
    if (p.row_ml && d == 0) store_row_ml(p, b, h, row, m, l);
  }
}

// The tokens' weights, from the keys once more now that every query's maximum
// and sum are known; shares as before, all rows of a head in one segment.  The
// product is q K^T here, so that a lane has one slot and four queries: a slot's
// sum over the queries stays in the lane but for two steps across rows of lanes.
// 61 us for 225 MB of keys and weights (40 sequences of 8 heads, 8 rows): 3.7 TB/s,
// memory and vector instructions about even; three blocks on their way to each
// wavefront, three workgroups a compute unit (four spill: 64 us).
constexpr int kWeighStages = 3;

template <int TYPE, int DIM, int GROUP, int NW>
__device__ __forceinline__ void weigh_segment(const AttArgs& p, const Segment& s, int take, int lane, int wave,
                                              uint8_t* lds) {
  constexpr int NG = DIM / GROUP;
  typedef Stage<DIM, GROUP, false> S;
  constexpr int kStage = S::kBytes + 128;
  const int b = s.b, h = s.h, n = s.n, end = s.blk + take, g = lane >> 4;
  int blk = s.blk + wave;
  const Expand<TYPE> key_codes;
  uint8_t* ring = lds + wave * kWeighStages * kStage;
  int64_t rows[kWeighStages];
  int places[kWeighStages];
  // a block's keys, and the weights that its slots had (anything without them)
  auto bring = [&](int z) {
    uint8_t* to = ring + z * kStage;
    S::bring(p, rows[z], places[z], lane, to);
    const int64_t i = max(rows[z], (int64_t)0) * p.c.page + (rows[z] < 0 ? 0 : places[z]);
    const float* was = p.acc_in ? p.acc_in + i : reinterpret_cast<const float*>(p.c.k);
    if (lane < 32)
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(was + lane),
                                       (__attribute__((address_space(3))) void*)(to + S::kBytes), 4, 0, 0);
  };
#pragma unroll
  for (int j = 0; j < kWeighStages; ++j) {
    rows[j] = -1;
    if (blk + j * NW >= end) continue;
    rows[j] = block_row(p, b, h, blk + j * NW, places[j]);
    if (p.c.n_pages > 0) bring(j);
  }
  // Queries r0.. : the operand, and of the lane's four rows 4 g + r the sums
  // over the groups, the maximum, 1 / sum (0 for rows beyond the last) and the
  // slots that it sees.
  v4u q[DIM / 32];
  v4f start[NG], qsum[NG];
  float m[4], inv[4];
  int limit[4];
  auto queries = [&](int r0) {
    Queries<TYPE, DIM, GROUP> x;
    load_queries<TYPE, DIM, GROUP>(p, b, h, r0 + (lane & 15), n, lane, x);
    sum_queries(x);
#pragma unroll
    for (int i = 0; i < DIM / 32; ++i) q[i] = x.q[i];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = r0 + 4 * g + r;
      const float* ml = p.row_ml + (((int64_t)b * p.c.n_heads + h) * p.rows + min(row, p.rows - 1)) * 2;
      m[r] = ml[0];
      inv[r] = row < p.rows ? ml[1] : 0.0f;
      limit[r] = row < p.rows ? n - p.n_queries + row / p.per + 1 : 0;
#pragma unroll
      for (int k = 0; k < NG; ++k) {
        qsum[k][r] = __shfl(x.sum[k], 4 * g + r);
        start[k][r] = -16.0f * qsum[k][r];
      }
    }
  };
  queries(0);
  while (blk < end) {
#pragma unroll
    for (int z = 0; z < kWeighStages; ++z) {
      if (blk >= end) break;
      const int64_t here = rows[z];
      const int place = places[z];
      const bool more = blk + kWeighStages * NW < end;
      if (more) rows[z] = block_row(p, b, h, blk + kWeighStages * NW, places[z]);
      // (a store of weights after those loads only makes this wait longer)
      if (blk + (kWeighStages - 1) * NW < end)
        wait_loads<(kWeighStages - 1) * (S::kLoads + 1)>();
      else
        wait_loads<0>();
      uint32_t k[2][DIM / 32], par[2][NG];
      const uint8_t* at = ring + z * kStage;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        S::keys(at, lane, t, k[t]);
#pragma unroll
        for (int i = 0; i < NG; ++i)
          par[t][i] = *reinterpret_cast<const uint32_t*>(at + S::kParAt + i * 128 + (16 * t + (lane & 15)) * 4);
      }
      const float was = *reinterpret_cast<const float*>(at + S::kBytes + (lane & 31) * 4);
      if (more) {
        wait_reads();
        if (p.c.n_pages > 0) bring(z);
      }
      if (here >= 0) {
        float w[2] = {0.0f, 0.0f};
        v4u kf[2][DIM / 32];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < DIM / 32; ++i) kf[t][i] = key_codes(k[t][i]);
        for (int r0 = 0; r0 < p.rows; r0 += 16) {
          if (p.rows > 16) queries(r0);  // (in attend_whole alone)
          const bool ragged = blk * 32 + 32 > n - p.n_queries + 1;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            float x[4];
#pragma unroll
            for (int i = 0; i < NG; ++i) {
              v4f a = start[i];
#pragma unroll
              for (int c = i * (GROUP / 32); c < (i + 1) * (GROUP / 32); ++c) a = mfma<TYPE>(q[c], kf[t][c], a);
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                x[r] = fma_m(qsum[i][r], par[t][i], i == 0 ? 0.0f : x[r]);
                x[r] = fma_d(a[r], par[t][i], x[r]);
              }
            }
            const int slot = blk * 32 + 16 * t + (lane & 15);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float e = __builtin_amdgcn_exp2f(fmaf(x[r], p.c_log2, -m[r])) * inv[r];
              // (rows beyond the last have 0 / sum, but may be NaN)
              if (ragged || p.rows % 16) e = slot < limit[r] ? e : 0.0f;
              w[t] += e;
            }
          }
        }
        const float w0 = sum_over_rows(w[0]), w1 = sum_over_rows(w[1]);
        const float x = (lane & 16) ? w1 : w0;
        const int place_s = place + (lane & 31);
        if (lane < 32 && blk * 32 + (lane & 31) < n) p.acc_out[here * p.c.page + place_s] = (p.acc_in ? was : 0.0f) + x;
      }
      blk += NW;
    }
  }
}

// More than 16 rows: a wavefront keeps the expanded keys of BLOCKS blocks in
// registers and goes over the rows, 16 at a time; the other wavefronts of the
// workgroup read the same rows at about the same time.  The sums of q come from
// the matrix instructions too, as a product with ones.  Bound by the exponentials
// and sums, 1200 rows over two sequences of up to 12,000 slots take 180 us.
template <int TYPE, int DIM, int GROUP, int BLOCKS>
__device__ __forceinline__ void weigh_rows(const AttArgs& p, const Segment& s, int take, int lane, int wave) {
  constexpr int NG = DIM / GROUP;
  const int b = s.b, h = s.h, n = s.n, end = s.blk + take, g = lane >> 4, in = lane & 15;
  const Expand<TYPE> key_codes;
  const uint32_t one = TYPE == AS_BF16 ? 0x3f803f80u : 0x3c003c00u;
  const v4u ones = {one, one, one, one};
  const float* row_ml = p.row_ml + ((int64_t)b * p.c.n_heads + h) * p.rows * 2;
  for (int blk0 = s.blk + wave * BLOCKS; blk0 < end; blk0 += kWaves * BLOCKS) {
    v4u kf[BLOCKS][2][DIM / 32];
    uint32_t par[BLOCKS][2][NG];
    int64_t slots[BLOCKS];  // of the block's first slot in a pool of one value a slot, or -1
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
      slots[i] = -1;
      if (blk0 + i >= end) continue;
      int at;
      const int64_t row = block_row(p, b, h, blk0 + i, at);
      if (row < 0) continue;
      slots[i] = row * p.c.page + at;
      const uint32_t* k = p.c.k + (slots[i] + in) * (DIM / 8) + g * (DIM / 32);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (DIM == 128) {
          const v4u w = *reinterpret_cast<const v4u*>(k + t * 16 * (DIM / 8));
#pragma unroll
          for (int c = 0; c < DIM / 32; ++c) kf[i][t][c] = key_codes(w[c]);
        } else {
          const v2u w = *reinterpret_cast<const v2u*>(k + t * 16 * (DIM / 8));
#pragma unroll
          for (int c = 0; c < DIM / 32; ++c) kf[i][t][c] = key_codes(w[c]);
        }
#pragma unroll
        for (int c = 0; c < NG; ++c) par[i][t][c] = p.c.k_par[(row * NG + c) * p.c.page + at + 16 * t + in];
      }
    }
    float w[BLOCKS][2] = {};
    const bool ragged = (blk0 + BLOCKS) * 32 > n - p.n_queries + 1;
    for (int r0 = 0; r0 < p.rows; r0 += 16) {
      const int row = min(r0 + in, p.rows - 1), t = row / p.per;
      const uint16_t* from = p.q + b * p.q_seq + t * p.q_token + (int64_t)(h * p.per + row - t * p.per) * DIM + g * 8;
      v4u q[DIM / 32];
#pragma unroll
      for (int c = 0; c < DIM / 32; ++c) q[c] = *reinterpret_cast<const v4u*>(from + 32 * c);
      v4f qsum[NG], start[NG];
      float m[4], inv[4];
      int limit[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int at = r0 + 4 * g + r;
        const float2 ml = *reinterpret_cast<const float2*>(row_ml + (int64_t)min(at, p.rows - 1) * 2);
        m[r] = ml.x;
        inv[r] = ml.y;
      }
      const bool masked = ragged || r0 + 16 > p.rows;
      if (masked) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int at = r0 + 4 * g + r;
          limit[r] = at < p.rows ? n - p.n_queries + at / p.per + 1 : 0;
        }
      }
#pragma unroll
      for (int k = 0; k < NG; ++k) {
        qsum[k] = v4f{0, 0, 0, 0};
#pragma unroll
        for (int c = k * (GROUP / 32); c < (k + 1) * (GROUP / 32); ++c) qsum[k] = mfma<TYPE>(q[c], ones, qsum[k]);
        start[k] = qsum[k] * -16.0f;
      }
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          float x[4];
#pragma unroll
          for (int k = 0; k < NG; ++k) {
            v4f a = start[k];
#pragma unroll
            for (int c = k * (GROUP / 32); c < (k + 1) * (GROUP / 32); ++c) a = mfma<TYPE>(q[c], kf[i][t][c], a);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              x[r] = fma_m(qsum[k][r], par[i][t][k], k == 0 ? 0.0f : x[r]);
              x[r] = fma_d(a[r], par[i][t][k], x[r]);
            }
          }
          const int slot = (blk0 + i) * 32 + 16 * t + in;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float e = __builtin_amdgcn_exp2f(fmaf(x[r], p.c_log2, -m[r])) * inv[r];
            if (masked) e = slot < limit[r] ? e : 0.0f;
            w[i][t] += e;
          }
        }
    }
#pragma unroll
    for (int i = 0; i < BLOCKS; ++i) {
      const float w0 = sum_over_rows(w[i][0]), w1 = sum_over_rows(w[i][1]);
      const int slot = lane & 31;
      if (slots[i] >= 0 && lane < 32 && (blk0 + i) * 32 + slot < n)
        p.acc_out[slots[i] + slot] = (p.acc_in ? p.acc_in[slots[i] + slot] : 0.0f) + ((lane & 16) ? w1 : w0);
    }
  }
}

template <int TYPE, int DIM, int GROUP, bool MANY>
__global__ __launch_bounds__(64 * kWaves, MANY ? 2 : 3) void weigh(AttArgs p) {
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Sequences first;
  uint32_t total;
  const uint32_t size = share_size<true>(p, lane, first, total);
  const int64_t share = share_number(total, size);
  if (share < 0) return;
  const uint32_t unit = (uint32_t)share * size;
  int left = (int)min(size, total - unit);
  Segment g = locate<true>(p, unit, lane, first);
  for (;;) {
    const int take = min(left << p.weigh_round, g.seen - g.blk);
    if (MANY)
      weigh_rows<TYPE, DIM, GROUP, 256 / DIM>(p, g, take, lane, wave);
    else
      weigh_segment<TYPE, DIM, GROUP, kWaves>(p, g, take, lane, wave, lds);
    left -= (int)rounds<true>(p, take);
    if (left == 0) return;
    advance<true>(p, g);
  }
}

// Short sequences: a workgroup has a whole segment, so that nothing is left to
// be joined, and the weights too, where all rows are in one segment: one launch,
// where a launch costs more than the work.  Very short ones take four
// wavefronts, others as many as their registers allow.
constexpr int whole_waves(int dim, int group, int nt) { return nt == 1 && dim < 4 * group ? 16 : 8; }

template <int TYPE, int DIM, int GROUP, int NT, int NW>
__global__ __launch_bounds__(64 * NW) void attend_whole(AttArgs p) {
  __shared__ float ml[NW][16][2];
  extern __shared__ __align__(16) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Segment s;
  const int bh = blockIdx.x / p.row_groups;
  s.rg = blockIdx.x % p.row_groups;
  s.b = bh / p.c.n_heads, s.h = bh % p.c.n_heads;
  s.n = clamped_length(p, s.b);
  s.blk = 0;
  int least;
  s.seen = seen_blocks(p, s.n, s.rg, least);
  attend_segment<TYPE, DIM, GROUP, NT, NW>(p, s, s.seen, 0, lane, wave, lds, ml);
  if (!p.acc_out || p.row_groups > 1) return;
  s.seen = (s.n + 31) / 32;
  weigh_segment<TYPE, DIM, GROUP, NW>(p, s, s.seen, lane, wave, lds);
}

struct Plan {
  bool many;
  int whole;   // wavefronts of attend_whole, kWaves or more, or 0
  bool alone;  // attend_many with a segment to a workgroup
  int per, rows, tiles, row_groups, workgroups, weigh_workgroups;
  int round, weigh_round, least;  // as in AttArgs
  int64_t parts;  // of a segment, at most, where all have one length
  int64_t o_bytes, ml_bytes, row_bytes;
};

// attend_whole takes tables of up to kShortBlocks blocks with four wavefronts
// (64 sequences of 8 heads, up to 10 blocks, with weights: 37 us on the device in
// three launches of shares and 14 there), and of up to kWholeBlocks with more
// wavefronts where every segment has a compute unit.  One compute unit works 0.2 us at a
// block: 12 heads of up to 60 blocks with weights took 17 us on the device
// there, 17 us in shares, and 22 us a step against 35; 8 heads of 129 blocks 28
// us there and 14 us in shares.
constexpr int kShortBlocks = 16, kWholeBlocks = 64;

// Workgroups that a compute unit runs at once: the launch bounds of the kernels.
Plan make_plan(const as_cache_t* c, int n_queries, int n_q_heads, bool weights) {
  Plan pl;
  pl.per = n_q_heads / c->n_heads;
  pl.rows = pl.per * n_queries;
  // attend_many takes 4/5 as long for a row, empty ones of its 128 included (128
  // channels in groups of 64, 9 sequences of up to 30,000 slots, 2 heads: 98 us
  // against 109 for 100 rows, 156 against 122 for 130, 225 against 211 for 260), but
  // longer with groups of a fourth of the channels, whose sums leave room for one
  // wavefront a SIMD: 390 us against 261 for 260 rows.
  const bool wide = c->dim == 4 * c->group;
  pl.many = !wide && round_up(pl.rows, kManyRows) * 4 <= round_up(pl.rows, 16) * 5;
  auto set_tiles = [&](int tiles) {
    pl.tiles = tiles;
    pl.row_groups = (pl.rows + 16 * tiles - 1) / (16 * tiles);
  };
  set_tiles(pl.many ? kManyRows / 16 : pl.rows > 16 ? 2 : 1);
  const int64_t heads = (int64_t)c->n_seqs * c->n_heads;
  const int64_t blocks = (int64_t)c->max_pages * c->page / 32;
  pl.whole = 0;
  if (!pl.many) {
    if (blocks <= kShortBlocks)
      pl.whole = kWaves;
    else if (blocks <= kWholeBlocks && heads * pl.row_groups <= as_host::compute_units())
      pl.whole = whole_waves(c->dim, c->group, pl.tiles);
  }
  if (!pl.many && !pl.whole) set_tiles(1);
  // Many rows of short tables: shares would only add parts to be joined, unless
  // some segments are long and there are few.  15 sequences of up to 500 slots,
  // 226 new tokens, 20 heads of 64 channels: 36 us so, 54 in shares and joined; 300
  // tokens of 2 and of 15 such sequences, 32 heads of 128: 32 us against 45, 79
  // against 154.
  pl.alone = pl.many && (blocks <= kShortBlocks ||
                         (blocks <= kWholeBlocks && heads * pl.row_groups >= 2 * (int64_t)as_host::compute_units()));
  const int resident = pl.many ? 2 : wide ? 3 : 4;
  pl.round = pl.many ? 0 : 2;
  pl.least = pl.many ? kWaves : 1;
  pl.weigh_round = pl.rows <= 16 ? 2 : c->dim == 128 ? 3 : 4;
  static_assert(kWaves == 4, "rounds");
  // As many as run at once, but no more than there can be shares (starting a
  // workgroup takes about 4 ns, those without a share included).
  auto groups = [&](int64_t segments, int64_t in_share, int64_t running) {
    const int64_t most = segments * ((blocks + in_share - 1) / in_share);
    return (int)round_up(most > running ? running : most < 1 ? 1 : most, 8);
  };
  const int cus = as_host::compute_units();
  pl.workgroups = groups(heads * pl.row_groups, kWaves, (int64_t)cus * resident);
  pl.weigh_workgroups = groups(heads, 1 << pl.weigh_round, (int64_t)cus * (pl.rows > 16 ? 2 : 3));
  pl.parts = pl.workgroups / (heads * pl.row_groups);
  if (pl.parts > blocks / kWaves) pl.parts = blocks / kWaves;
  const int64_t places = (int64_t)pl.workgroups * 2 * 16 * pl.tiles;
  pl.o_bytes = pl.whole || pl.alone ? 0 : round_up(places * c->dim * 4, 256);
  pl.ml_bytes = pl.whole || pl.alone ? 0 : round_up(places * 8, 256);
  pl.row_bytes = weights ? round_up(heads * pl.rows * 8, 256) : 0;
  return pl;
}

int check_queries(const as_cache_t* c, int32_t n_queries, int32_t n_q_heads) {
  if (n_queries < 0 || n_q_heads < 1 || n_q_heads % c->n_heads)
    return fail(AS_E_INVALID_ARG, "attention_kv4: %d queries of %d heads over %d key/value heads", n_queries,
                n_q_heads, c->n_heads);
  if (n_queries > 65536 || n_q_heads > 65536)
    return fail(AS_E_LIMITS, "attention_kv4: %d queries of %d heads (at most 65536 each)", n_queries, n_q_heads);
  if ((int64_t)c->n_seqs * c->n_heads > 65535)
    return fail(AS_E_LIMITS, "attention_kv4: %d sequences of %d heads (at most 65535 in all)", c->n_seqs, c->n_heads);
  if ((int64_t)c->n_seqs * n_queries * n_q_heads > (1 << 26))
    return fail(AS_E_LIMITS, "attention_kv4: %d sequences, %d queries, %d heads (at most 2^26 rows in all)", c->n_seqs,
                n_queries, n_q_heads);
  const int64_t spans = ((int64_t)n_q_heads / c->n_heads * n_queries + 15) / 16;
  if ((int64_t)c->n_seqs * c->n_heads * spans * ((int64_t)c->max_pages * c->page / 32) > 0x7fffffff)
    return fail(AS_E_LIMITS, "attention_kv4: at most 2^31 blocks of 32 slots over all sequences, heads and 16 rows");
  return AS_OK;
}

template <int TYPE, int DIM, int GROUP, int NT, int NW>
int launch_whole(const AttArgs& p, hipStream_t s) {
  typedef Stage<DIM, GROUP, false> KeyStage;
  size_t lds = attend_lds<DIM, GROUP>(NW);
  const size_t weigh_lds = (size_t)NW * kWeighStages * (KeyStage::kBytes + 128);
  if (p.acc_out && weigh_lds > lds) lds = weigh_lds;
  const int rc = allow_lds<&attend_whole<TYPE, DIM, GROUP, NT, NW>>(lds, "attention_kv4");
  if (rc != AS_OK) return rc;
  hipLaunchKernelGGL((attend_whole<TYPE, DIM, GROUP, NT, NW>),
                     dim3((unsigned)(p.c.n_seqs * p.c.n_heads * p.row_groups)), dim3(64 * NW), lds, s, p);
  return launched("attention_kv4");
}

template <int TYPE, int DIM, int GROUP>
int launch_attention(const AttArgs& p, const Plan& pl, hipStream_t s) {
  const int64_t heads = (int64_t)p.c.n_seqs * p.c.n_heads;
  const dim3 t(64 * kWaves);
  if (pl.whole) {
    int rc;
    if (pl.whole == kWaves)
      rc = pl.tiles == 1 ? launch_whole<TYPE, DIM, GROUP, 1, kWaves>(p, s)
                         : launch_whole<TYPE, DIM, GROUP, 2, kWaves>(p, s);
    else
      rc = pl.tiles == 1 ? launch_whole<TYPE, DIM, GROUP, 1, whole_waves(DIM, GROUP, 1)>(p, s)
                         : launch_whole<TYPE, DIM, GROUP, 2, whole_waves(DIM, GROUP, 2)>(p, s);
    if (rc != AS_OK || p.row_groups == 1) return rc;
  } else {
    typedef Operands<DIM, GROUP> OperandSet;
    if constexpr (DIM < 4 * GROUP) {
      const size_t lds = 2 * OperandSet::kBytes;
      if (pl.alone)
        hipLaunchKernelGGL((attend_many<TYPE, DIM, GROUP, true>), dim3((unsigned)(heads * p.row_groups)), t, lds, s, p);
      else if (pl.many)
        hipLaunchKernelGGL((attend_many<TYPE, DIM, GROUP, false>), dim3((unsigned)pl.workgroups), t, lds, s, p);
    }
    const size_t lds = attend_lds<DIM, GROUP>(kWaves);
    if (!pl.many)
      hipLaunchKernelGGL((attend<TYPE, DIM, GROUP>), dim3((unsigned)pl.workgroups), t, lds, s, p);
  }
  if (!pl.whole && !pl.alone) {
    const dim3 by_row((unsigned)(heads * p.rows));
    if (pl.many || pl.parts < 8)
      hipLaunchKernelGGL((join<TYPE, DIM, 1024 / DIM, 256>), dim3((unsigned)(heads * ((p.rows + 15) / 16))), dim3(256),
                         0, s, p);
    else if (pl.parts >= 64)
      hipLaunchKernelGGL((join<TYPE, DIM, 1, 1024>), by_row, dim3(1024), 0, s, p);
    else
      hipLaunchKernelGGL((join<TYPE, DIM, 1, 256>), by_row, dim3(256), 0, s, p);
  }
  typedef Stage<DIM, GROUP, false> KeyStage;
  if (p.acc_out && p.rows > 16)
    hipLaunchKernelGGL((weigh<TYPE, DIM, GROUP, true>), dim3((unsigned)pl.weigh_workgroups), t, 0, s, p);
  else if (p.acc_out)
    hipLaunchKernelGGL((weigh<TYPE, DIM, GROUP, false>), dim3((unsigned)pl.weigh_workgroups), t,
                       (size_t)kWaves * kWeighStages * (KeyStage::kBytes + 128), s, p);
  return launched("attention_kv4");
}

template <int TYPE>
int launch_by_shape(const AttArgs& p, const Plan& pl, hipStream_t s) {
  if (p.c.dim == 64)
    return p.c.group == 32 ? launch_attention<TYPE, 64, 32>(p, pl, s) : launch_attention<TYPE, 64, 64>(p, pl, s);
  if (p.c.group == 32) return launch_attention<TYPE, 128, 32>(p, pl, s);
  if (p.c.group == 64) return launch_attention<TYPE, 128, 64>(p, pl, s);
  return launch_attention<TYPE, 128, 128>(p, pl, s);
}

}  // namespace as_ops

using namespace as_ops;

extern "C" {

int64_t as_attention_kv4_workspace(const as_cache_t* cache, int32_t n_queries, int32_t n_q_heads, int32_t weights) {
  if (check_cache(cache, "attention_kv4", false, false) != AS_OK ||
      check_queries(cache, n_queries, n_q_heads) != AS_OK || cache->n_seqs == 0 || n_queries == 0)
    return 0;
  const Plan pl = make_plan(cache, n_queries, n_q_heads, weights != 0);
  return pl.o_bytes + pl.ml_bytes + pl.row_bytes;
}

int as_attention_kv4(const as_cache_t* cache, const void* q, int32_t type, int32_t n_queries, int32_t n_q_heads,
                     int64_t q_seq, int64_t q_token, const int32_t* length, float scale, void* out,
                     const float* acc_in, float* acc_out, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_cache(cache, "attention_kv4", false, false);
  if (rc != AS_OK) return rc;
  rc = check_queries(cache, n_queries, n_q_heads);
  if (rc != AS_OK) return rc;
  if (type != AS_BF16 && type != AS_F16) return fail(AS_E_INVALID_ARG, "attention_kv4: type %d", type);
  // (its product with log2 e has to be finite)
  if (!(scale > 0.0f) || scale > 2.0e38f) return fail(AS_E_INVALID_ARG, "attention_kv4: scale %g", (double)scale);
  if (cache->n_seqs == 0 || n_queries == 0) return as_host::ok();
  if (!q || !length || !out) return fail(AS_E_INVALID_ARG, "attention_kv4: null pointer");
  if (!aligned(q, 16) || !aligned(out, 8) || q_seq % 8 || q_token % 8)
    return fail(AS_E_INVALID_ARG, "attention_kv4: queries (and outputs, to 8) have to be aligned to 16 bytes, strides a multiple of 8");
  const Plan pl = make_plan(cache, n_queries, n_q_heads, acc_out != nullptr);
  const int64_t need = pl.o_bytes + pl.ml_bytes + pl.row_bytes;
  if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 256))))
    return fail(AS_E_INVALID_ARG, "attention_kv4: workspace of %lld bytes, %lld needed (aligned to 256)",
                (long long)workspace_bytes, (long long)need);
  AttArgs p{};
  p.c = cache_args(cache);
  p.q = reinterpret_cast<const uint16_t*>(q);
  p.q_seq = q_seq;
  p.q_token = q_token;
  p.length = length;
  p.out = out;
  char* ws = reinterpret_cast<char*>(workspace);
  p.part_o = reinterpret_cast<float*>(ws);
  p.part_ml = reinterpret_cast<float*>(ws + pl.o_bytes);
  p.row_ml = pl.row_bytes ? reinterpret_cast<float*>(ws + pl.o_bytes + pl.ml_bytes) : nullptr;
  p.acc_in = acc_in;
  p.acc_out = acc_out;
  p.c_log2 = scale * 1.4426950408889634f;
  p.page_mul = page_magic(cache->page);
  p.n_queries = n_queries;
  p.per = pl.per;
  p.rows = pl.rows;
  p.row_groups = pl.row_groups;
  p.row_span = 16 * pl.tiles;
  p.workgroups = pl.workgroups;
  p.weigh_workgroups = pl.weigh_workgroups;
  p.round = pl.round;
  p.weigh_round = pl.weigh_round;
  p.least = pl.least;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == AS_BF16 ? launch_by_shape<AS_BF16>(p, pl, s) : launch_by_shape<AS_F16>(p, pl, s);
}

}  // extern "C"
