// Attention of a step's queries over a cache held in 4 bits, and the attention
// weight that every cached token gets (alpaserve_ops.h).
//
// A group's value is code * d + m, so with codes c
//   q.k     = sum over groups of  d (sum q c) + m (sum q)
//   sum p v = sum over tokens of  (p d) c + p m
// and the codes enter v_mfma_f32_16x16x32 as 16 + c, which a shift, a mask and
// an or make of 4 bits (bf16 holds 16..31 in steps of 1/8, fp16 in steps of
// 1/64); the 16 is taken out in fp32: the first product starts from -16 sum q,
// the second is corrected by 16 (p d).  Queries are exact in the first product;
// p d enters the second as two bf16 numbers.
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
  float* part_o;   // [n_seqs * n_heads][splits][rows][dim], not normalised
  float* part_ml;  // [n_seqs * n_heads][splits][rows][2]: maximum (log2 units), sum
  float* row_ml;   // [n_seqs * n_heads][rows][2] for the weights: maximum, 1 / sum
  const float* acc_in;
  float* acc_out;
  float c_log2;      // scale * log2(e)
  uint32_t page_mul; // page_magic of the cache's pages
  int32_t n_queries, per, rows, splits, row_groups;
  int32_t chunk, row_span;  // blocks of 32 slots and query rows of a workgroup of attend
  int32_t weigh_chunk;      // blocks of a workgroup of weigh
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

// Wait until at most N of the wavefront's loads are on their way; what is read
// from LDS afterwards is read afterwards.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "six bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
  asm volatile("" ::: "memory");
}
// Wait for the wavefront's LDS reads: their place may be written again.
__device__ __forceinline__ void wait_reads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0), nothing else
  asm volatile("" ::: "memory");
}

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
  for (int g = 0; g < DIM / GROUP; ++g) {
    float s = 0.0f;
#pragma unroll
    for (int i = g * (GROUP / 32); i < (g + 1) * (GROUP / 32); ++i) {
      x.q[i] = row < p.rows ? *reinterpret_cast<const v4u*>(q + 32 * i) : v4u{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 4; ++j) s += to_f32<TYPE>(x.q[i][j] & 0xffffu) + to_f32<TYPE>(x.q[i][j] >> 16);
    }
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
  float shift[NT][DIM / GROUP];  // sum of p m - 16 p d over the lane's slots
  float mref[NT], sum[NT];       // reference of the exponents (log2 units), sum of p over the lane's slots
};

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
  if (RAGGED) {
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (slot0 + 16 * (e >> 2) + (e & 3) >= q[u].limit) s[u][e] = -kInf;
  }
#pragma unroll
  for (int u = 0; u < NT; ++u) {
    const float top = p.c_log2 * fmaxf(fmaxf(fmaxf(s[u][0], s[u][1]), fmaxf(s[u][2], s[u][3])),
                                       fmaxf(fmaxf(s[u][4], s[u][5]), fmaxf(s[u][6], s[u][7])));
    // The reference follows the maximum only where it is passed by a factor
    // of 2^8: sums and products stay far from fp32's range, and the sums so
    // far are hardly ever scaled.
    if (__any(top > a.mref[u] + 8.0f)) {
      const float m = fmaxf(a.mref[u], max_over_rows(top));
      const float f = __builtin_amdgcn_exp2f(a.mref[u] - m);
      a.mref[u] = m;
      a.sum[u] *= f;
#pragma unroll
      for (int g = 0; g < NG; ++g) a.shift[u][g] *= f;
#pragma unroll
      for (int i = 0; i < DIM / 16; ++i) a.o[u][i] *= f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s[u][e] = __builtin_amdgcn_exp2f(fmaf(s[u][e], p.c_log2, -a.mref[u]));
      a.sum[u] += s[u][e];
    }
  }
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
          a.shift[u][g] = fmaf(-16.0f, pd[z], a.shift[u][g]);
        }
        hi[u][j] = pack_bf16(pd[0], pd[1]);
        lo[u][j] = pack_bf16(pd[0] - __uint_as_float(hi[u][j] << 16), pd[1] - __uint_as_float(hi[u][j] & 0xffff0000u));
      }
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

// Blocks of 32 slots that the query rows row0.. (`count` of them) see, and the
// slots that the first of them sees.
__device__ __forceinline__ int seen_blocks(const AttArgs& p, int n, int row0, int count, int& least) {
  const int last = min(n, n - p.n_queries + min(row0 + count - 1, p.rows - 1) / p.per + 1);
  least = n - p.n_queries + row0 / p.per + 1;
  return max(0, (last + 31) / 32);
}

// One workgroup per (sequence, head, run of p.chunk blocks of 32 slots, 16 NT
// query rows); its four wavefronts take the blocks in turn, each with a ring of
// its own in LDS so that none waits for another, and join their results at the
// end.
constexpr int kStages = 2;
template <int DIM, int GROUP>
constexpr int attend_lds() {
  constexpr int ring = kStages * Stage<DIM, GROUP, true>::kBytes, part = 16 * (DIM + 4) * 4;
  return kWaves * (ring > part ? ring : part);
}

template <int TYPE, int DIM, int GROUP, int NT>
__global__ __launch_bounds__(64 * kWaves, (NT == 1 ? 4 : 2) - (DIM == 4 * GROUP)) void attend(AttArgs p) {
  constexpr int NG = DIM / GROUP;
  typedef Stage<DIM, GROUP, true> S;
  constexpr int kRing = kStages * S::kBytes;
  __shared__ float ml[kWaves][16][2];
  extern __shared__ __align__(16) uint8_t lds[];  // the rings, then the parts to be joined
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Neighbouring workgroup numbers go to different XCDs: the row groups of one
  // part, which read the same slots, are a multiple of 8 apart.
  const int unit = (int)(blockIdx.x / (8 * p.row_groups)) * 8 + (int)(blockIdx.x & 7);
  const int rg = (int)(blockIdx.x / 8) % p.row_groups;
  const int bh = unit / p.splits, split = unit % p.splits;
  if (bh >= p.c.n_seqs * p.c.n_heads) return;
  const int b = bh / p.c.n_heads, h = bh % p.c.n_heads;
  const int n = clamped_length(p, b);
  const int row0 = rg * 16 * NT;
  int least;
  const int seen = seen_blocks(p, n, row0, 16 * NT, least);
  const int end = min((split + 1) * p.chunk, seen);
  if (p.splits > 1 && split * p.chunk >= seen) return;

  uint8_t* ring = lds + wave * kRing;
  Queries<TYPE, DIM, GROUP> q[NT];
  Sums<DIM, GROUP, NT> a;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    load_queries<TYPE, DIM, GROUP>(p, b, h, row0 + 16 * t + (lane & 15), n, lane, q[t]);
    a.mref[t] = kFloor;
    a.sum[t] = 0.0f;
#pragma unroll
    for (int g = 0; g < NG; ++g) a.shift[t][g] = 0.0f;
#pragma unroll
    for (int i = 0; i < DIM / 16; ++i) a.o[t][i] = v4f{0, 0, 0, 0};
  }

  const Expand<TYPE> key_codes;
  const Expand<AS_BF16> value_codes;
  int blk = split * p.chunk + wave;
  uint32_t valid = 0;  // bit j: the block j turns on has a page
#pragma unroll
  for (int j = 0; j < kStages; ++j) {
    if (blk + j * kWaves >= end) break;
    int at;
    const int64_t row = block_row(p, b, h, blk + j * kWaves, at);
    valid |= (uint32_t)(row >= 0) << j;
    if (p.c.n_pages > 0) S::bring(p, row, at, lane, ring + j * S::kBytes);
  }
  int slot = 0;
  // Blocks up to `to`, all of one kind.
  auto blocks = [&](int to, auto ragged) {
    for (; blk < to; blk += kWaves) {
      int at = 0;
      int64_t row = -1;
      const bool more = blk + kStages * kWaves < end;
      if (more) row = block_row(p, b, h, blk + kStages * kWaves, at);
      if (blk + (kStages - 1) * kWaves < end)
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
    }
  };
  blocks(min(end, least >> 5), std::false_type());  // all 32 slots seen by all queries
  blocks(end, std::true_type());

  // Join the wavefronts, 16 rows at a time.
  float* part = reinterpret_cast<float*>(lds);  // [kWaves][16][DIM + 4]
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
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ml[w][lane & 15][0]);
    const float f = __builtin_amdgcn_exp2f(a.mref[u] - m);
    float add[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) add[g] = sum_over_rows(a.shift[u][g]);
#pragma unroll
    for (int i = 0; i < DIM / 16; ++i)
      *reinterpret_cast<v4f*>(part + (wave * 16 + (lane & 15)) * (DIM + 4) + 16 * i + (lane >> 4) * 4) =
          (a.o[u][i] + add[i * 16 / GROUP]) * f;
    __syncthreads();
    for (int j = threadIdx.x; j < 16 * DIM / 4; j += 64 * kWaves) {
      const int r = j / (DIM / 4), d = j % (DIM / 4) * 4;
      const int row = row0 + 16 * u + r;
      if (row >= p.rows) continue;
      v4f x = {0, 0, 0, 0};
      float top = kFloor, l = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        x += *reinterpret_cast<const v4f*>(part + (w * 16 + r) * (DIM + 4) + d);
        top = fmaxf(top, ml[w][r][0]);
      }
#pragma unroll
      for (int w = 0; w < kWaves; ++w) l += ml[w][r][1] * __builtin_amdgcn_exp2f(ml[w][r][0] - top);
      const int64_t at = ((int64_t)bh * p.splits + split) * p.rows + row;
      if (p.splits > 1) *reinterpret_cast<v4f*>(p.part_o + at * DIM + d) = x;
      if (p.part_ml && d == 0) {
        p.part_ml[at * 2] = top;
        p.part_ml[at * 2 + 1] = l;
      }
      if (p.splits == 1) {
        const int t = row / p.per;
        uint16_t* out = reinterpret_cast<uint16_t*>(p.out) +
                        (((int64_t)b * p.n_queries + t) * p.c.n_heads * p.per + h * p.per + row - t * p.per) * DIM + d;
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = from_f32<TYPE>(l == 0.0f ? 0.0f : x[e] / l);
      }
    }
  }
}

// Joins the splits, one workgroup per row: every split's factor first, then
// their sums, four channels to a thread and several splits side by side.
constexpr int kMaxSplits = 1024;

template <int TYPE, int DIM>
__global__ __launch_bounds__(256) void join(AttArgs p) {
  constexpr int kSide = 256 / (DIM / 4);
  __shared__ float factor[kMaxSplits];
  __shared__ float red[2][4];
  __shared__ v4f sums[kSide][DIM / 4];
  const int row = blockIdx.x % p.rows, bh = blockIdx.x / p.rows;
  const int b = bh / p.c.n_heads, h = bh % p.c.n_heads, tid = threadIdx.x;
  const int rows_wg = p.row_span;
  int least;
  const int seen = seen_blocks(p, clamped_length(p, b), row / rows_wg * rows_wg, rows_wg, least);
  const int live = p.splits > 1 ? (seen + p.chunk - 1) / p.chunk : 1;
  const int64_t base = (int64_t)bh * p.splits * p.rows + row;
  float m = kFloor;
  for (int s = tid; s < live; s += 256) m = fmaxf(m, p.part_ml[(base + (int64_t)s * p.rows) * 2]);
#pragma unroll
  for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((tid & 63) == 0) red[0][tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
  float l = 0.0f;
  for (int s = tid; s < live; s += 256) {
    const float* ml = p.part_ml + (base + (int64_t)s * p.rows) * 2;
    const float f = __builtin_amdgcn_exp2f(ml[0] - m);
    factor[s] = f;
    l += f * ml[1];
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) l += __shfl_xor(l, o);
  if ((tid & 63) == 0) red[1][tid >> 6] = l;
  __syncthreads();
  l = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
  if (p.row_ml && tid == 0) {
    p.row_ml[((int64_t)bh * p.rows + row) * 2] = m;
    p.row_ml[((int64_t)bh * p.rows + row) * 2 + 1] = l == 0.0f ? 0.0f : 1.0f / l;
  }
  if (p.splits == 1) return;
  const int d = tid % (DIM / 4), side = tid / (DIM / 4);
  v4f x = {0, 0, 0, 0};
#pragma unroll 4
  for (int s = side; s < live; s += kSide)
    x += *reinterpret_cast<const v4f*>(p.part_o + (base + (int64_t)s * p.rows) * DIM + 4 * d) * factor[s];
  sums[side][d] = x;
  __syncthreads();
  if (side) return;
#pragma unroll
  for (int s = 1; s < kSide; ++s) x += sums[s][d];
  const int t = row / p.per;
  uint16_t* out = reinterpret_cast<uint16_t*>(p.out) +
                  (((int64_t)b * p.n_queries + t) * p.c.n_heads * p.per + h * p.per + row - t * p.per) * DIM + 4 * d;
#pragma unroll
  for (int e = 0; e < 4; ++e) out[e] = from_f32<TYPE>(l == 0.0f ? 0.0f : x[e] / l);
}

// The sum of x over the 16 lanes of a row, in every one of them.
__device__ __forceinline__ float sum_in_row(float x) {
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x128, 0xf, 0xf, false));  // row_ror:8
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x124, 0xf, 0xf, false));
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x122, 0xf, 0xf, false));
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x121, 0xf, 0xf, false));
  return x;
}

// The tokens' weights, from the keys once more now that every query's maximum
// and sum are known: one workgroup per run of blocks, whose wavefronts take them
// in turn, all queries of the head.  With at most 16 rows the queries stay in
// registers.
constexpr int kWeighStages = 3;

template <int TYPE, int DIM, int GROUP>
__global__ __launch_bounds__(64 * kWaves, DIM == 4 * GROUP ? 2 : 3) void weigh(AttArgs p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int bh = blockIdx.y, b = bh / p.c.n_heads, h = bh % p.c.n_heads;
  const int n = clamped_length(p, b);
  const int end = min((int)(blockIdx.x + 1) * p.weigh_chunk, (n + 31) / 32);
  int blk = (int)blockIdx.x * p.weigh_chunk + wave;
  if (blk >= end) return;
  const Expand<TYPE> key_codes;
  Queries<TYPE, DIM, GROUP> q;
  float m = 0.0f, inv = 0.0f;
  auto queries = [&](int r0) {
    const int r = r0 + (lane & 15);
    load_queries<TYPE, DIM, GROUP>(p, b, h, r, n, lane, q);
    if (r >= p.rows) q.limit = 0;
    const float* ml = p.row_ml + ((int64_t)bh * p.rows + min(r, p.rows - 1)) * 2;
    m = ml[0], inv = ml[1];
  };
  queries(0);
  typedef Stage<DIM, GROUP, false> S;
  extern __shared__ __align__(16) uint8_t lds[];
  constexpr int kStage = S::kBytes + 128;
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
    if (blk + j * kWaves >= end) continue;
    rows[j] = block_row(p, b, h, blk + j * kWaves, places[j]);
    if (p.c.n_pages > 0) bring(j);
  }
  while (blk < end) {
#pragma unroll
    for (int z = 0; z < kWeighStages; ++z) {
      if (blk >= end) break;
      const int64_t here = rows[z];
      const int place = places[z];
      const bool more = blk + kWeighStages * kWaves < end;
      if (more) rows[z] = block_row(p, b, h, blk + kWeighStages * kWaves, places[z]);
      // (a store of weights after those loads only makes this wait longer)
      if (blk + (kWeighStages - 1) * kWaves < end)
        wait_loads<(kWeighStages - 1) * (S::kLoads + 1)>();
      else
        wait_loads<0>();
      uint32_t k[2][DIM / 32];
      v4u par[2][DIM / GROUP];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        S::keys(ring + z * kStage, lane, t, k[t]);
#pragma unroll
        for (int g = 0; g < DIM / GROUP; ++g) par[t][g] = S::key_scales(ring + z * kStage, lane, t, g);
      }
      const int e8 = lane & 15, s8 = 16 * (e8 >> 2) + (lane >> 4) * 4 + (e8 & 3);  // the slot that lanes e8 < 8 store
      const float was = e8 < 8 ? *reinterpret_cast<const float*>(ring + z * kStage + S::kBytes + s8 * 4) : 0.0f;
      if (more) {
        wait_reads();
        if (p.c.n_pages > 0) bring(z);
      }
      if (here >= 0) {
        v4u kf[2][DIM / 32];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < DIM / 32; ++i) kf[t][i] = key_codes(k[t][i]);
        float w[8] = {};
        const int slot0 = blk * 32 + (lane >> 4) * 4;
        for (int r0 = 0; r0 < p.rows; r0 += 16) {
          if (p.rows > 16) queries(r0);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            float x[4];
            scores<TYPE, DIM, GROUP>(kf[t], par[t], q, x);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (slot0 + 16 * t + e < q.limit) w[4 * t + e] += __builtin_amdgcn_exp2f(fmaf(x[e], p.c_log2, -m)) * inv;
          }
        }
        // lane e of each row of 16 stores its slot e
        float x = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = sum_in_row(w[e]);
          x = (lane & 15) == e ? y : x;
        }
        if (e8 < 8 && blk * 32 + s8 < n) p.acc_out[here * p.c.page + place + s8] = (p.acc_in ? was : 0.0f) + x;
      }
      blk += kWaves;
    }
  }
}

struct Plan {
  int per, rows, tiles, row_groups, splits, chunk, weigh_chunk, weigh_groups;
  int64_t o_bytes, ml_bytes, row_bytes;
};

// Blocks of 32 slots to a workgroup of four wavefronts: at least two for each
// wavefront, and more where that still leaves about 2048 workgroups.  Runs of one
// length balance ragged sequences: those beyond a sequence's end return at once.
int choose_chunk(int64_t blocks, int64_t units, int64_t target) {
  int64_t c = blocks * units / target;
  c = c < 8 ? 8 : round_up(c, 8);
  const int64_t least = (blocks + kMaxSplits - 1) / kMaxSplits;
  return (int)(c > least ? c : round_up(least, 8));
}

Plan make_plan(const as_cache_t* c, int n_queries, int n_q_heads, bool weights) {
  Plan pl;
  pl.per = n_q_heads / c->n_heads;
  pl.rows = pl.per * n_queries;
  pl.tiles = pl.rows > 16 ? 2 : 1;
  pl.row_groups = (pl.rows + 16 * pl.tiles - 1) / (16 * pl.tiles);
  const int64_t heads = (int64_t)c->n_seqs * c->n_heads;
  int64_t blocks = (int64_t)c->max_pages * c->page / 32;
  if (blocks < 1) blocks = 1;
  pl.chunk = choose_chunk(blocks, heads * pl.row_groups, 2048);
  pl.splits = (int)((blocks + pl.chunk - 1) / pl.chunk);
  pl.weigh_chunk = choose_chunk(blocks, heads, 2048);
  pl.weigh_groups = (int)((blocks + pl.weigh_chunk - 1) / pl.weigh_chunk);
  const int64_t rows = heads * pl.rows;
  pl.o_bytes = pl.splits > 1 ? round_up(rows * pl.splits * c->dim * 4, 256) : 0;
  pl.ml_bytes = pl.splits > 1 || weights ? round_up(rows * pl.splits * 8, 256) : 0;
  pl.row_bytes = weights ? round_up(rows * 8, 256) : 0;
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
  return AS_OK;
}

template <int TYPE, int DIM, int GROUP>
int launch_attention(const AttArgs& p, const Plan& pl, hipStream_t s) {
  const int64_t units = round_up((int64_t)p.c.n_seqs * p.c.n_heads * pl.splits, 8) * pl.row_groups;
  const dim3 g((unsigned)units), t(64 * kWaves);
  const size_t lds = attend_lds<DIM, GROUP>();
  if (pl.tiles == 1)
    hipLaunchKernelGGL((attend<TYPE, DIM, GROUP, 1>), g, t, lds, s, p);
  else
    hipLaunchKernelGGL((attend<TYPE, DIM, GROUP, 2>), g, t, lds, s, p);
  if (pl.splits > 1 || p.acc_out)
    hipLaunchKernelGGL((join<TYPE, DIM>), dim3((unsigned)((int64_t)p.c.n_seqs * p.c.n_heads * p.rows)), dim3(256), 0,
                       s, p);
  typedef Stage<DIM, GROUP, false> KeyStage;
  if (p.acc_out)
    hipLaunchKernelGGL((weigh<TYPE, DIM, GROUP>),
                       dim3((unsigned)pl.weigh_groups, (unsigned)(p.c.n_seqs * p.c.n_heads)), t,
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
  if (!(scale > 0.0f) || scale > 3.0e38f) return fail(AS_E_INVALID_ARG, "attention_kv4: scale %g", (double)scale);
  if (cache->n_seqs == 0 || n_queries == 0) return as_host::ok();
  if (!q || !length || !out) return fail(AS_E_INVALID_ARG, "attention_kv4: null pointer");
  if (!aligned(q, 16) || q_seq % 8 || q_token % 8)
    return fail(AS_E_INVALID_ARG, "attention_kv4: queries have to be aligned to 16 bytes, strides a multiple of 8");
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
  p.part_o = pl.o_bytes ? reinterpret_cast<float*>(ws) : nullptr;
  p.part_ml = pl.ml_bytes ? reinterpret_cast<float*>(ws + pl.o_bytes) : nullptr;
  p.row_ml = pl.row_bytes ? reinterpret_cast<float*>(ws + pl.o_bytes + pl.ml_bytes) : nullptr;
  p.acc_in = acc_in;
  p.acc_out = acc_out;
  p.c_log2 = scale * 1.4426950408889634f;
  p.page_mul = page_magic(cache->page);
  p.n_queries = n_queries;
  p.per = pl.per;
  p.rows = pl.rows;
  p.splits = pl.splits;
  p.row_groups = pl.row_groups;
  p.chunk = pl.chunk;
  p.row_span = 16 * pl.tiles;
  p.weigh_chunk = pl.weigh_chunk;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  return type == AS_BF16 ? launch_by_shape<AS_BF16>(p, pl, s) : launch_by_shape<AS_F16>(p, pl, s);
}

}  // extern "C"
