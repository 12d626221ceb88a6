// Linear layers with 8-bit weights and activations quantised per token
// (alpaserve_ops.h): y = (sum_k c_tk w_nk) * s_t * u_n + b_n.
//
// Both operands are stored as the matrix instruction v_mfma_i32_16x16x64_i8
// takes them: a tile of 16 rows x 64 columns is 1 KiB in which lane l's 16
// bytes (row l%16, columns 16 (l/16)..+15) lie at 16 l, so a wavefront's load of
// an operand is one contiguous KiB.
#include "ops_common.hpp"

using as_host::fail;

namespace as_ops {

// ------------------------------------------------------------- quantisation

constexpr int kQThreads = 256;

template <int TYPE>
__device__ __forceinline__ float load_one(const void* x, int64_t i) {
  if (TYPE == AS_F32) return reinterpret_cast<const float*>(x)[i];
  return to_f32<TYPE>(reinterpret_cast<const uint16_t*>(x)[i]);
}

// 16 values from column c of a row; columns beyond n_cols are 0.  Rows may start
// anywhere: memory takes unaligned loads of 16 bytes.
template <int TYPE>
__device__ __forceinline__ void load16(const void* x, int64_t row, int64_t c, int64_t n_cols, float (&f)[16]) {
  if (c + 16 <= n_cols) {
    if (TYPE == AS_F32) {
      const float* p = reinterpret_cast<const float*>(x) + row + c;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v4f v;
        __builtin_memcpy(&v, p + 4 * i, 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[4 * i + j] = v[j];
      }
    } else {
      const uint16_t* p = reinterpret_cast<const uint16_t*>(x) + row + c;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v4u v;
        __builtin_memcpy(&v, p + 8 * i, 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f[8 * i + 2 * j] = to_f32<TYPE>(v[j] & 0xffffu);
          f[8 * i + 2 * j + 1] = to_f32<TYPE>(v[j] >> 16);
        }
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) f[i] = c + i < n_cols ? load_one<TYPE>(x, row + c + i) : 0.0f;
}

// Largest magnitude as ordered bits: infinities above every number, NaN above
// them, so that one integer maximum finds both.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// How a row is quantised, from its largest magnitude.  A power of two takes
// rows of very large or small numbers away from the ends of fp32's range.
template <int TYPE>
struct Quantiser {
  float by, top, inv;  // 127 and the largest magnitude, scaled; 1 / top
  bool none;           // all codes are 0
  __device__ __forceinline__ Quantiser(float a, bool finite) {
    none = !finite || a == 0.0f;
    const float scale = a > 0x1p100f ? 0x1p-64f : a < 0x1p-64f ? 0x1p64f : 1.0f;
    by = 127.0f * scale;
    top = none ? 1.0f : a * scale;
    inv = 1.0f / top;
  }
  // Codes of four values.  127 x is exact for 16-bit x.  Its quotient by top is
  // taken with the reciprocal and corrected once by the exact remainder: off by
  // 2^-46 of itself before the last rounding, so a quotient that ties between
  // two codes comes out exactly, and no other one can reach a tie (the nearest
  // is 2^-19 away).  The codes are therefore those of exact arithmetic.  fp32
  // values are divided.  Adding 1.5 * 2^23 rounds to whole numbers, ties to
  // even, and leaves the code in the low byte.
  __device__ __forceinline__ uint32_t codes4(const float* f) const {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = f[i] * by;
      float q;
      if (TYPE == AS_F32) {
        q = x / top;
      } else {
        q = x * inv;
        q = fmaf(fmaf(-q, top, x), inv, q);
      }
      u[i] = __float_as_uint(q + 12582912.0f);
    }
    const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu);
    return none ? 0u : lo | hi;
  }
};

// One workgroup per row: its largest magnitude, then its codes; the second
// reading comes from the caches.  Bound by latency for few rows, by the bytes
// of x for many: 48 rows of 4096 take 3.3 us, 1187 of 282 5.6 us.
template <int TYPE>
__global__ __launch_bounds__(kQThreads) void quantize_rows(const void* __restrict__ x, int64_t n_cols,
                                                           int64_t row_stride, int64_t padded,
                                                           uint8_t* __restrict__ codes, float* __restrict__ scale) {
  __shared__ uint32_t part[kQThreads / 64];
  const int64_t r = blockIdx.x;
  const int64_t row = r * row_stride;
  uint32_t top = 0;
  for (int64_t c = (int64_t)threadIdx.x * 16; c < n_cols; c += kQThreads * 16) {
    float f[16];
    load16<TYPE>(x, row, c, n_cols, f);
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, magnitude(f[i]));
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kQThreads / 64; ++w) top = max(top, part[w]);
  const bool finite = top < 0x7f800000u;
  const float a = __uint_as_float(top);
  const Quantiser<TYPE> quantiser(a, finite);
  if (threadIdx.x == 0) scale[r] = finite ? a / 127.0f : __builtin_nanf("");
  // byte offset of column c: tiles of 1 KiB, 256 bytes for each 16 columns
  uint8_t* out = codes + (r >> 4) * (padded >> 6) * 1024 + (r & 15) * 16;
  for (int64_t c = (int64_t)threadIdx.x * 16; c < padded; c += kQThreads * 16) {
    v4u q = {0, 0, 0, 0};
    if (!quantiser.none && c < n_cols) {
      float f[16];
      load16<TYPE>(x, row, c, n_cols, f);
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = quantiser.codes4(f + 4 * i);
    }
    *reinterpret_cast<v4u*>(out + (c >> 4) * 256) = q;
  }
}

// Many rows of 16-bit values: a workgroup of 16 wavefronts per 16 rows, a lane of
// which has 16 columns of one row of every 64 x 16th tile and keeps them in
// registers, so that x is read once and the codes are written as contiguous
// tiles.  Bound by the bytes: 4096 rows of 8192 took 47 us with a workgroup per
// row, 32 us with a wavefront per row, whose codes go out 16 bytes at a time, and
// take 21 us so (67 MB read, 34 written: 4.7 TB/s).
template <int TYPE, int TILES>
__global__ __launch_bounds__(1024) void quantize_tiles(const uint16_t* __restrict__ x, int64_t n_rows, int n_cols,
                                                       int64_t row_stride, int k_tiles, uint8_t* __restrict__ codes,
                                                       float* __restrict__ scale) {
  __shared__ uint32_t tops[16][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in = lane & 15;
  const int64_t r = (int64_t)blockIdx.x * 16 + in;
  const uint16_t* row = x + min(r, n_rows - 1) * row_stride;
  v4u raw[TILES][2];
#pragma unroll
  for (int i = 0; i < TILES; ++i) {
    const int c = (i * 16 + wave) * 64 + (lane >> 4) * 16;
    raw[i][0] = raw[i][1] = v4u{0, 0, 0, 0};
    if (c + 16 <= n_cols) {
      __builtin_memcpy(&raw[i][0], row + c, 16);
      __builtin_memcpy(&raw[i][1], row + c + 8, 16);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (c + e < n_cols) raw[i][e >> 3][(e >> 1) & 3] |= (uint32_t)row[c + e] << (16 * (e & 1));
    }
  }
  // magnitudes of 16-bit values are ordered as their bits without the sign
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < TILES; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t w = raw[i][j >> 2][j & 3] & 0x7fff7fffu;
      top = max(top, max(w & 0xffffu, w >> 16));
    }
  top = max(top, (uint32_t)__shfl_xor((int)top, 16));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32));
  if (lane < 16) tops[wave][in] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 16; ++w) top = max(top, tops[w][in]);
  const float a = to_f32<TYPE>(top);
  const bool finite = top < (TYPE == AS_BF16 ? 0x7f80u : 0x7c00u);
  const Quantiser<TYPE> quantiser(a, finite);
  if (threadIdx.x < 16 && r < n_rows) scale[r] = finite ? a / 127.0f : __builtin_nanf("");
  uint8_t* out = codes + (int64_t)blockIdx.x * k_tiles * 1024 + lane * 16;
#pragma unroll
  for (int i = 0; i < TILES; ++i) {
    const int tile = i * 16 + wave;
    if (tile >= k_tiles) break;
    float f[16];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      f[2 * j] = to_f32<TYPE>(raw[i][j >> 2][j & 3] & 0xffffu);
      f[2 * j + 1] = to_f32<TYPE>(raw[i][j >> 2][j & 3] >> 16);
    }
    *reinterpret_cast<v4u*>(out + (int64_t)tile * 1024) =
        v4u{quantiser.codes4(f), quantiser.codes4(f + 4), quantiser.codes4(f + 8), quantiser.codes4(f + 12)};
  }
}

template <int TYPE>
void launch_quantize(const void* x, int64_t rows, int64_t cols, int64_t stride, void* codes, float* scale,
                     hipStream_t s) {
  const int64_t padded = round_up(cols, 128);
  if constexpr (TYPE != AS_F32) {
    // enough rows for half the compute units, 16 to each; rows that fit the registers
    if (rows >= 2048 && cols <= 8192) {
      auto tiles = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + 15) / 16)), dim3(1024), 0, s,
                           reinterpret_cast<const uint16_t*>(x), rows, (int)cols, stride, (int)(padded / 64),
                           (uint8_t*)codes, scale);
      };
      if (cols <= 1024)
        tiles(quantize_tiles<TYPE, 1>);
      else if (cols <= 2048)
        tiles(quantize_tiles<TYPE, 2>);
      else if (cols <= 4096)
        tiles(quantize_tiles<TYPE, 4>);
      else
        tiles(quantize_tiles<TYPE, 8>);
      return;
    }
  }
  hipLaunchKernelGGL((quantize_rows<TYPE>), dim3((unsigned)rows), dim3(kQThreads), 0, s, x, cols, stride, padded,
                     (uint8_t*)codes, scale);
}

// ------------------------------------------------------------------ product

struct LinArgs {
  const uint8_t* a;      // activations' codes, in tiles
  const float* a_scale;  // [n_tokens]
  const uint8_t* w;      // weights' codes, in tiles
  const float* w_scale;  // [n_out]
  const float* bias;     // [n_out] or null
  void* y;
  int64_t y_stride;
  int32_t n_tokens, n_out, k_tiles;
  // activations, where the product quantises them
  const void* x;
  int64_t x_stride;
  int32_t n_in;
};

template <int YTYPE>
__device__ __forceinline__ void store_one(void* y, int64_t i, float v) {
  if (YTYPE == AS_F32)
    reinterpret_cast<float*>(y)[i] = v;
  else
    reinterpret_cast<uint16_t*>(y)[i] = from_f32<YTYPE>(v);
}

// (rows of an odd length are at any address: one store all the same)
template <int YTYPE>
__device__ __forceinline__ void store_four(void* y, int64_t i, const float (&v)[4]) {
  if (YTYPE == AS_F32) {
    __builtin_memcpy(reinterpret_cast<float*>(y) + i, v, 16);
  } else {
    const uint32_t lo = from_f32<YTYPE>(v[0]) | (uint32_t)from_f32<YTYPE>(v[1]) << 16;
    const uint32_t hi = from_f32<YTYPE>(v[2]) | (uint32_t)from_f32<YTYPE>(v[3]) << 16;
    const v2u two = {lo, hi};
    __builtin_memcpy(reinterpret_cast<uint16_t*>(y) + i, &two, 8);
  }
}

// a's upper 32 lanes and b's lower ones change places; then, of each 32 lanes,
// a's upper 16 and b's lower ones.
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
  const v2u p = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = p[0], b = p[1];
}
__device__ __forceinline__ void swap_rows(uint32_t& a, uint32_t& b) {
  const v2u p = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = p[0], b = p[1];
}

// 8 values from column c of a row of 16-bit values; columns beyond n are 0.
template <int TYPE>
__device__ __forceinline__ void load8(const uint16_t* x, int64_t row, int c, int n, float (&f)[8]) {
  if (c + 8 <= n) {
    v4u v;
    __builtin_memcpy(&v, x + row + c, 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f[2 * j] = to_f32<TYPE>(v[j] & 0xffffu);
      f[2 * j + 1] = to_f32<TYPE>(v[j] >> 16);
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = c + i < n ? to_f32<TYPE>(x[row + c + i]) : 0.0f;
}

// Result of one sum.
template <int YTYPE>
__device__ __forceinline__ void finish(const LinArgs& p, int t, int n, int sum, float s) {
  float v = (float)sum * s * p.w_scale[n];
  if (p.bias) v += p.bias[n];
  store_one<YTYPE>(p.y, (int64_t)t * p.y_stride + n, v);
}

// Few tokens: the weights' bytes bound it, each read once.  One workgroup takes
// 16 CT channels and all tokens; its eight wavefronts share out the columns and
// add their sums in LDS (whole numbers: the order does not matter).  Weights go
// from memory to registers, 1 KiB a load, several in flight.
// FUSED (at most 16 tokens): the workgroup quantises the activations itself,
// into LDS, with its first weights already on their way; this repeats little
// work in every workgroup and saves a launch.  1 token 4096 -> 4096: 5.0 us (3.3
// TB/s of weights: a launch, two passes over the token and the last sums are half
// of it), 8.4 us a call by the host; 48 tokens 4096 -> 16384: 16.7 us, 4.0 TB/s.
constexpr int kFewWaves = 8;

template <int YTYPE, int XTYPE, int CT, int TT, bool FUSED>
__global__ __launch_bounds__(64 * kFewWaves) void product_few(LinArgs p) {
  extern __shared__ uint8_t lds[];
  int* sums = reinterpret_cast<int*>(lds);                       // [TT][CT][4][64], as the lanes have them
  uint32_t* tops = reinterpret_cast<uint32_t*>(sums + TT * CT * 256);  // [16]
  uint8_t* rows = reinterpret_cast<uint8_t*>(tops + 16);         // FUSED: [n_tokens][row_bytes]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_ct = (p.n_out + 15) / 16, ct0 = blockIdx.x * CT;
  const int64_t tile_row = (int64_t)p.k_tiles * 1024;
  const int per = (p.k_tiles + kFewWaves - 1) / kFewWaves;
  const int k0 = wave * per, k1 = min(p.k_tiles, k0 + per);
  const uint8_t* w[CT];
#pragma unroll
  for (int i = 0; i < CT; ++i) w[i] = p.w + min(ct0 + i, n_ct - 1) * tile_row + lane * 16;
  constexpr int kAhead = CT <= 2 ? 4 : 2;
  v4i first[kAhead][CT];
#pragma unroll
  for (int j = 0; j < kAhead; ++j)
#pragma unroll
    for (int i = 0; i < CT; ++i)
      first[j][i] = k0 + j < k1 ? *reinterpret_cast<const v4i*>(w[i] + (int64_t)(k0 + j) * 1024) : v4i{0, 0, 0, 0};
  for (int j = tid; j < TT * CT * 256; j += 64 * kFewWaves) sums[j] = 0;
  const int row_bytes = p.k_tiles * 64 + 16;  // 16 rows' words of one column group fall on different banks
  if (FUSED) {
    if (tid < 16) tops[tid] = 0;
    lds_barrier();
    const int chunks = p.k_tiles * 8;  // of 8 columns
    const uint16_t* x = reinterpret_cast<const uint16_t*>(p.x);
    // One or two tokens: all wavefronts at each.  More: a wavefront to a token,
    // so that no token waits for another.
    const bool together = p.n_tokens <= 2;
    const int from = together ? tid : lane, step = together ? 64 * kFewWaves : 64;
    for (int t = together ? 0 : wave; t < p.n_tokens; t += together ? 1 : kFewWaves) {
      uint32_t top = 0;
#pragma unroll 8
      for (int c = from; c < chunks; c += step) {
        float f[8];
        load8<XTYPE>(x, t * p.x_stride, c * 8, p.n_in, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, magnitude(f[i]));
      }
#pragma unroll
      for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
      if (lane == 0) atomicMax(&tops[t], top);
    }
    lds_barrier();
    for (int t = together ? 0 : wave; t < p.n_tokens; t += together ? 1 : kFewWaves) {
      const uint32_t top = tops[t];
      const Quantiser<XTYPE> quantiser(__uint_as_float(top), top < 0x7f800000u);
#pragma unroll 4
      for (int c = from; c < chunks; c += step) {
        float f[8];
        load8<XTYPE>(x, t * p.x_stride, c * 8, p.n_in, f);
        *reinterpret_cast<v2u*>(rows + t * row_bytes + c * 8) = v2u{quantiser.codes4(f), quantiser.codes4(f + 4)};
      }
    }
  }
  lds_barrier();
  const uint8_t* a = FUSED ? rows + min(lane & 15, p.n_tokens - 1) * row_bytes + (lane >> 4) * 16 : p.a + lane * 16;
  const int a_step = FUSED ? 64 : 1024;
  v4i acc[CT][TT] = {};
  for (int k = k0; k < k1; k += kAhead) {
    v4i b[kAhead][TT];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
#pragma unroll
      for (int u = 0; u < TT; ++u)
        b[j][u] = k + j < k1 ? *reinterpret_cast<const v4i*>(a + u * tile_row + (int64_t)(k + j) * a_step)
                             : v4i{0, 0, 0, 0};
    v4i next[kAhead][CT];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
#pragma unroll
      for (int i = 0; i < CT; ++i)
        next[j][i] = k + kAhead + j < k1 ? *reinterpret_cast<const v4i*>(w[i] + (int64_t)(k + kAhead + j) * 1024)
                                         : v4i{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
#pragma unroll
      for (int i = 0; i < CT; ++i) {
#pragma unroll
        for (int u = 0; u < TT; ++u)
          acc[i][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(first[j][i], b[j][u], acc[i][u], 0, 0, 0);
        first[j][i] = next[j][i];
      }
  }
#pragma unroll
  for (int u = 0; u < TT; ++u)
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        atomicAdd(&sums[((u * CT + i) * 4 + r) * 64 + lane], acc[i][u][r]);
  lds_barrier();
  for (int j = tid; j < TT * CT * 256; j += 64 * kFewWaves) {
    const int t = j / (CT * 16), n = ct0 * 16 + j % (CT * 16);
    if (t >= p.n_tokens || n >= p.n_out) continue;
    float s;
    if (FUSED)
      s = tops[t] < 0x7f800000u ? __uint_as_float(tops[t]) / 127.0f : __builtin_nanf("");
    else
      s = p.a_scale[t];
    const int i = j / 16 % CT, c = j % 16;  // channel 4 (lane / 16) + r of the tile, token lane % 16
    finish<YTYPE>(p, t, n, sums[((t / 16 * CT + i) * 4 + (c & 3)) * 64 + (c >> 2) * 16 + (t & 15)], s);
  }
}

// Many tokens: bound by the matrix instructions and what feeds them (the matrix
// units are busy for 53 % of the cycles of tiles of 256 x 256).  A workgroup of WC x WT wavefronts takes
// 16 TC channels x 16 TT tokens, KS tiles of 64 columns at a time: they come
// into a ring of S stages in LDS straight from memory (a tile is a contiguous KiB
// there and in LDS, read back without bank conflicts) while older ones are
// multiplied; one barrier a stage.  Neighbouring workgroup numbers go to different
// XCDs, so each XCD gets a contiguous run of tiles in an order that walks the
// channels in bands of 8: the tiles that run together share rows of both
// operands in its L2.  4096 tokens 8192 -> 8192: 218 us in tiles of 256 x 256, 2.5
// POP/s; 333 tokens 1500 -> 2777: 7 us.
template <int YTYPE, int TC, int TT, int WC, int WT, int KS, int S>
__global__ __launch_bounds__(64 * WC * WT) void product_many(LinArgs p) {
  constexpr int kW = WC * WT, kC = TC / WC, kT = TT / WT, kStage = (TC + TT) * KS, kLoads = kStage / kW;
  static_assert(kStage % kW == 0, "every wavefront brings in as many tiles");
  extern __shared__ uint8_t lds[];  // [S][kStage][1024]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_ct = (p.n_out + 15) / 16, n_tt = (p.n_tokens + 15) / 16;
  const int gc = (n_ct + TC - 1) / TC, gt = (n_tt + TT - 1) / TT;
  const int total = gc * gt, id = blockIdx.x;
  const int share = total / 8, more = total % 8, xcd = id & 7;
  const int at = xcd * share + min(xcd, more) + (id >> 3);
  const int band = at / (8 * gt), wide = min(8, gc - band * 8), in_band = at - band * 8 * gt;
  const int c0 = (band * 8 + in_band % wide) * TC, t0 = in_band / wide * TT;
  const int64_t tile_row = (int64_t)p.k_tiles * 1024;

  // The tiles of a stage that this wavefront brings in: i, i + kW, ..
  const uint8_t* from[kLoads];
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int i = wave + j * kW, r = i / KS;
    from[j] = (r < TC ? p.w + min(c0 + r, n_ct - 1) * tile_row : p.a + min(t0 + r - TC, n_tt - 1) * tile_row) +
              (i % KS) * 1024 + lane * 16;
  }
  auto bring = [&](int slot, int k) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)(from[j] + (int64_t)k * 1024),
          (__attribute__((address_space(3))) void*)(lds + (slot * kStage + wave + j * kW) * 1024), 16, 0, 0);
  };
  const int wc = wave % WC * kC, wt = wave / WC * kT;
  v4i acc[kC][kT] = {};
  const int steps = p.k_tiles / KS;
#pragma unroll
  for (int j = 0; j < S - 1; ++j)
    if (j < steps) bring(j, j * KS);
  int slot = 0;
  for (int i = 0; i < steps; ++i) {
    // stage i is there for this wavefront, then for all; all are done with i - 1
    if (i + S - 2 < steps)
      wait_loads<(S - 2) * kLoads>();
    else
      wait_loads<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int free = slot == 0 ? S - 1 : slot - 1;
    if (i + S - 1 < steps) bring(free, (i + S - 1) * KS);
    const uint8_t* here = lds + slot * kStage * 1024 + lane * 16;
#pragma unroll
    for (int z = 0; z < KS; ++z) {
      v4i a[kC], b[kT];
#pragma unroll
      for (int j = 0; j < kC; ++j) a[j] = *reinterpret_cast<const v4i*>(here + ((wc + j) * KS + z) * 1024);
#pragma unroll
      for (int j = 0; j < kT; ++j) b[j] = *reinterpret_cast<const v4i*>(here + ((TC + wt + j) * KS + z) * 1024);
#pragma unroll
      for (int j = 0; j < kC; ++j)
#pragma unroll
        for (int u = 0; u < kT; ++u) acc[j][u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[j], b[u], acc[j][u], 0, 0, 0);
    }
    wait_reads();
    slot = slot + 1 == S ? 0 : slot + 1;
  }
  float s[kT];
#pragma unroll
  for (int j = 0; j < kT; ++j) s[j] = p.a_scale[min((t0 + wt + j) * 16 + (lane & 15), p.n_tokens - 1)];
  // Where the wavefront has 64 channels side by side, the four lanes of a token
  // exchange theirs: 32 bytes a lane, 128 side by side, not four times 32.
  constexpr bool kSwap = YTYPE != AS_F32 && kC % 4 == 0;
  if (kSwap && (c0 + wc + kC) * 16 <= p.n_out) {
#pragma unroll
    for (int i = 0; i < kC; i += 4) {
      const int n = (c0 + wc + i) * 16 + (lane >> 4) * 4;
      float u[4][4], bias[4][4] = {};
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        __builtin_memcpy(u[z], p.w_scale + n + 16 * z, 16);
        if (p.bias) __builtin_memcpy(bias[z], p.bias + n + 16 * z, 16);
      }
#pragma unroll
      for (int j = 0; j < kT; ++j) {
        const int t = (t0 + wt + j) * 16 + (lane & 15);
        uint32_t w[2][4];  // of tile z: channels 0 and 1, 2 and 3 of the lane's four
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          float v[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            v[r] = (float)acc[i + z][j][r] * s[j] * u[z][r];
            if (p.bias) v[r] += bias[z][r];
          }
#pragma unroll
          for (int h = 0; h < 2; ++h)
            w[h][z] = from_f32<YTYPE>(v[2 * h]) | (uint32_t)from_f32<YTYPE>(v[2 * h + 1]) << 16;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // tile z's quarter g to tile g's quarter z
          swap_halves(w[h][0], w[h][2]);
          swap_halves(w[h][1], w[h][3]);
          swap_rows(w[h][0], w[h][1]);
          swap_rows(w[h][2], w[h][3]);
        }
        if (t >= p.n_tokens) continue;
        uint16_t* y = reinterpret_cast<uint16_t*>(p.y) + (int64_t)t * p.y_stride + (c0 + wc + i + (lane >> 4)) * 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const v4u two = {w[0][2 * h], w[1][2 * h], w[0][2 * h + 1], w[1][2 * h + 1]};
          __builtin_memcpy(y + 8 * h, &two, 16);
        }
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kC; ++i) {
    const int n = (c0 + wc + i) * 16 + (lane >> 4) * 4;
    if (n + 4 <= p.n_out) {
      float u[4], bias[4] = {};
      __builtin_memcpy(u, p.w_scale + n, 16);
      if (p.bias) __builtin_memcpy(bias, p.bias + n, 16);
#pragma unroll
      for (int j = 0; j < kT; ++j) {
        const int t = (t0 + wt + j) * 16 + (lane & 15);
        if (t >= p.n_tokens) continue;
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          v[r] = (float)acc[i][j][r] * s[j] * u[r];
          if (p.bias) v[r] += bias[r];
        }
        store_four<YTYPE>(p.y, (int64_t)t * p.y_stride + n, v);
      }
    } else {
#pragma unroll
      for (int j = 0; j < kT; ++j) {
        const int t = (t0 + wt + j) * 16 + (lane & 15);
        if (t >= p.n_tokens) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (n + r < p.n_out) finish<YTYPE>(p, t, n + r, acc[i][j][r], s[j]);
      }
    }
  }
}

template <int YTYPE, int TC, int TT, int WC, int WT, int KS, int S>
int launch_many(const LinArgs& p, hipStream_t s) {
  const int64_t gc = ((p.n_out + 15) / 16 + TC - 1) / TC, gt = ((p.n_tokens + 15) / 16 + TT - 1) / TT;
  const size_t lds = (size_t)S * (TC + TT) * KS * 1024;
  const int rc = allow_lds<&product_many<YTYPE, TC, TT, WC, WT, KS, S>>(lds, "linear_i8");
  if (rc != AS_OK) return rc;
  hipLaunchKernelGGL((product_many<YTYPE, TC, TT, WC, WT, KS, S>), dim3((unsigned)(gc * gt)), dim3(64 * WC * WT), lds, s, p);
  return launched("linear_i8");
}

template <int YTYPE, int XTYPE, int CT, int TT, bool FUSED>
int launch_few(const LinArgs& p, hipStream_t s) {
  const int n_ct = (p.n_out + 15) / 16;
  size_t lds = (size_t)TT * CT * 1024 + 64;
  if (FUSED) lds += (size_t)p.n_tokens * (p.k_tiles * 64 + 16);
  const int rc = allow_lds<&product_few<YTYPE, XTYPE, CT, TT, FUSED>>(lds, "linear_i8");
  if (rc != AS_OK) return rc;
  hipLaunchKernelGGL((product_few<YTYPE, XTYPE, CT, TT, FUSED>), dim3((unsigned)((n_ct + CT - 1) / CT)),
                     dim3(64 * kFewWaves), lds, s, p);
  return launched("linear_i8");
}

// Channel tiles of a workgroup of product_few: as many as leave every compute
// unit a workgroup.
template <int YTYPE, int XTYPE, int TT, bool FUSED>
int few_by_channels(const LinArgs& p, hipStream_t s) {
  const int n_ct = (p.n_out + 15) / 16, cus = as_host::compute_units();
  if (n_ct >= 8 * cus) return launch_few<YTYPE, XTYPE, 4, TT, FUSED>(p, s);
  if (n_ct >= 4 * cus) return launch_few<YTYPE, XTYPE, 2, TT, FUSED>(p, s);
  return launch_few<YTYPE, XTYPE, 1, TT, FUSED>(p, s);
}

template <int YTYPE>
int launch_product(const LinArgs& p, hipStream_t s) {
  const int n_tt = (p.n_tokens + 15) / 16;
  if (n_tt == 1) return few_by_channels<YTYPE, AS_BF16, 1, false>(p, s);
  if (n_tt == 2) return few_by_channels<YTYPE, AS_BF16, 2, false>(p, s);
  if (n_tt == 3) return few_by_channels<YTYPE, AS_BF16, 3, false>(p, s);
  if (n_tt == 4) return few_by_channels<YTYPE, AS_BF16, 4, false>(p, s);
  // A compute unit runs one workgroup of 256 x 256 or two of 128 x 128, which take
  // 1.15 times as long for as much work (4096 tokens 8192 -> 8192: 296 us against
  // 268) but leave fewer units idle at the end: 1187 tokens 8192 -> 13712 take 3
  // turns of them, 174 us, and 2 of the larger ones, each as long as 1.7 (222 us).
  const int64_t n_ct = (p.n_out + 15) / 16, cus = as_host::compute_units();
  const int64_t large = ((n_ct + 15) / 16) * ((n_tt + 15) / 16), middle = ((n_ct + 7) / 8) * ((n_tt + 7) / 8);
  const int64_t large_turns = (large + cus - 1) / cus, middle_turns = (middle + 2 * cus - 1) / (2 * cus);
  if (large >= cus && large_turns * 200 <= middle_turns * 115) return launch_many<YTYPE, 16, 16, 2, 4, 2, 2>(p, s);
  if (middle >= cus) return launch_many<YTYPE, 8, 8, 2, 4, 2, 2>(p, s);
  // Two workgroups of either of these run on a compute unit; the smaller tiles
  // where all of them run at once (333 tokens 1500 -> 2777: 264 tiles of 64 x 64 took
  // 12.6 us, 484 of 64 x 32 took 9.8).
  if (((n_ct + 3) / 4) * ((n_tt + 1) / 2) > 2 * cus) return launch_many<YTYPE, 4, 4, 2, 2, 2, 4>(p, s);
  return launch_many<YTYPE, 4, 2, 4, 1, 2, 6>(p, s);
}

// Whether the product quantises the activations itself: they fit one tile of
// tokens and leave LDS for another workgroup.
bool fuses(int64_t n_tokens, int64_t n_in) {
  return n_tokens <= 16 && n_tokens * (round_up(n_in, 128) + 16) <= 72 * 1024;
}

template <int XTYPE>
int launch_fused(const LinArgs& p, int y_type, hipStream_t s) {
  if (y_type == AS_BF16) return few_by_channels<AS_BF16, XTYPE, 1, true>(p, s);
  if (y_type == AS_F16) return few_by_channels<AS_F16, XTYPE, 1, true>(p, s);
  return few_by_channels<AS_F32, XTYPE, 1, true>(p, s);
}

constexpr int64_t kMaxRows = (1 << 24) - 1;  // a workgroup of 256 to a row, fewer than 2^32 threads a launch

}  // namespace as_ops

using namespace as_ops;

extern "C" {

int64_t as_i8_bytes(int64_t n_rows, int64_t n_cols) {
  if (n_rows <= 0 || n_cols <= 0 || n_rows > kMaxRows || n_cols > AS_I8_MAX_INPUTS) return 0;
  return round_up(n_rows, 16) * round_up(n_cols, 128);
}

int as_quantize_i8(const void* x, int32_t type, int64_t n_rows, int64_t n_cols, int64_t row_stride, void* codes,
                   float* scale, void* stream) {
  if (type != AS_BF16 && type != AS_F16 && type != AS_F32) return fail(AS_E_INVALID_ARG, "quantize_i8: type %d", type);
  if (n_rows < 0 || n_cols < 1 || row_stride < n_cols)
    return fail(AS_E_INVALID_ARG, "quantize_i8: %lld rows of %lld columns, stride %lld", (long long)n_rows,
                (long long)n_cols, (long long)row_stride);
  if (n_rows > kMaxRows || n_cols > AS_I8_MAX_INPUTS)
    return fail(AS_E_LIMITS, "quantize_i8: at most %lld rows of %d columns", (long long)kMaxRows, AS_I8_MAX_INPUTS);
  if (n_rows == 0) return as_host::ok();
  if (!x || !codes || !scale) return fail(AS_E_INVALID_ARG, "quantize_i8: null pointer");
  if (!aligned(codes, 16)) return fail(AS_E_INVALID_ARG, "quantize_i8: codes not aligned to 16 bytes");
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (type == AS_BF16)
    launch_quantize<AS_BF16>(x, n_rows, n_cols, row_stride, codes, scale, s);
  else if (type == AS_F16)
    launch_quantize<AS_F16>(x, n_rows, n_cols, row_stride, codes, scale, s);
  else
    launch_quantize<AS_F32>(x, n_rows, n_cols, row_stride, codes, scale, s);
  return launched("quantize_i8");
}

int64_t as_linear_i8_workspace(int64_t n_tokens, int64_t n_in, int64_t n_out) {
  (void)n_out;
  const int64_t codes = as_i8_bytes(n_tokens, n_in);
  if (codes && fuses(n_tokens, n_in)) return 0;
  return codes ? codes + round_up(n_tokens * 4, 256) : 0;
}

int as_linear_i8(const void* x, int32_t x_type, int64_t n_tokens, int64_t n_in, int64_t x_stride, const void* w,
                 const float* w_scale, const float* bias, int64_t n_out, void* y, int32_t y_type, int64_t y_stride,
                 void* workspace, int64_t workspace_bytes, void* stream) {
  if (x_type != AS_BF16 && x_type != AS_F16) return fail(AS_E_INVALID_ARG, "linear_i8: x_type %d", x_type);
  if (y_type != AS_BF16 && y_type != AS_F16 && y_type != AS_F32)
    return fail(AS_E_INVALID_ARG, "linear_i8: y_type %d", y_type);
  if (n_tokens < 0 || n_in < 1 || n_out < 1 || x_stride < n_in || y_stride < n_out)
    return fail(AS_E_INVALID_ARG, "linear_i8: %lld tokens, %lld -> %lld, strides %lld and %lld", (long long)n_tokens,
                (long long)n_in, (long long)n_out, (long long)x_stride, (long long)y_stride);
  // (tiles and their threads then fit a launch for every y that fits the memory)
  if (n_tokens > 65535 * 16 || n_out > kMaxRows || n_in > AS_I8_MAX_INPUTS)
    return fail(AS_E_LIMITS, "linear_i8: at most %d tokens, %lld outputs, %d inputs", 65535 * 16, (long long)kMaxRows,
                AS_I8_MAX_INPUTS);
  if (n_tokens == 0) return as_host::ok();
  if (!x || !w || !w_scale || !y) return fail(AS_E_INVALID_ARG, "linear_i8: null pointer");
  if (!aligned(w, 16)) return fail(AS_E_INVALID_ARG, "linear_i8: weights not aligned to 16 bytes");
  const int64_t need = as_linear_i8_workspace(n_tokens, n_in, n_out);
  if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 256))))
    return fail(AS_E_INVALID_ARG, "linear_i8: workspace of %lld bytes, %lld needed (aligned to 256)",
                (long long)workspace_bytes, (long long)need);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  uint8_t* codes = reinterpret_cast<uint8_t*>(workspace);
  float* scale = reinterpret_cast<float*>(codes + as_i8_bytes(n_tokens, n_in));
  LinArgs p{};
  p.a = codes;
  p.a_scale = scale;
  p.w = reinterpret_cast<const uint8_t*>(w);
  p.w_scale = w_scale;
  p.bias = bias;
  p.y = y;
  p.y_stride = y_stride;
  p.n_tokens = (int32_t)n_tokens;
  p.n_out = (int32_t)n_out;
  p.k_tiles = (int32_t)(round_up(n_in, 128) / 64);
  p.x = x;
  p.x_stride = x_stride;
  p.n_in = (int32_t)n_in;
  if (fuses(n_tokens, n_in)) return x_type == AS_BF16 ? launch_fused<AS_BF16>(p, y_type, s) : launch_fused<AS_F16>(p, y_type, s);
  if (x_type == AS_BF16)
    launch_quantize<AS_BF16>(x, n_tokens, n_in, x_stride, codes, scale, s);
  else
    launch_quantize<AS_F16>(x, n_tokens, n_in, x_stride, codes, scale, s);
  if (y_type == AS_BF16) return launch_product<AS_BF16>(p, s);
  if (y_type == AS_F16) return launch_product<AS_F16>(p, s);
  return launch_product<AS_F32>(p, s);
}

}  // extern "C"
