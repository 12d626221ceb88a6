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

// 16 values from column c of a row; columns beyond n_cols are 0.  VEC: the row
// is aligned to 16 bytes.
template <int TYPE, bool VEC>
__device__ __forceinline__ void load16(const void* x, int64_t row, int64_t c, int64_t n_cols, float (&f)[16]) {
  if (VEC && c + 16 <= n_cols) {
    if (TYPE == AS_F32) {
      const v4f* p = reinterpret_cast<const v4f*>(reinterpret_cast<const float*>(x) + row + c);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const v4f v = p[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) f[4 * i + j] = v[j];
      }
    } else {
      const v4u* p = reinterpret_cast<const v4u*>(reinterpret_cast<const uint16_t*>(x) + row + c);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const v4u v = p[i];
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

// Codes of the N values of one row whose largest magnitude is top.  127 x is
// exact for 16-bit x, and its quotient by top cannot round to a tie that it is
// not, so rint(127 x / top) is the code of exact arithmetic.  The quotient is
// first taken with a reciprocal; the remainder 127 x - code * top, exact in one
// fma, shows whether the code is the nearest, and where a remainder is half of
// top or more (a tie, or a reciprocal that misled) all N are divided.
template <int N>
__device__ __forceinline__ void codes_of(const float (&f)[N], float top, float inv, uint32_t (&out)[N / 4]) {
  float q[N], worst = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    q[i] = rintf(f[i] * inv);
    worst = fmaxf(worst, fabsf(fmaf(-q[i], top, f[i] * 127.0f)));
  }
  if (!(worst + worst < top)) {
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = rintf(f[i] * 127.0f / top);
  }
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w |= ((uint32_t)(int)q[4 * i + j] & 0xffu) << (8 * j);
    out[i] = w;
  }
}

// One workgroup per row: its largest magnitude, then its codes; the second
// reading comes from the caches.  Bound by latency for few rows, by the bytes
// of x for many.
template <int TYPE, bool VEC>
__global__ __launch_bounds__(kQThreads) void quantize_rows(const void* __restrict__ x, int64_t n_cols,
                                                           int64_t row_stride, int64_t padded,
                                                           uint8_t* __restrict__ codes, float* __restrict__ scale) {
  __shared__ uint32_t part[kQThreads / 64];
  const int64_t r = blockIdx.x;
  const int64_t row = r * row_stride;
  uint32_t top = 0;
  for (int64_t c = (int64_t)threadIdx.x * 16; c < n_cols; c += kQThreads * 16) {
    float f[16];
    load16<TYPE, VEC>(x, row, c, n_cols, f);
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
  const float a = __uint_as_float(top), inv = 127.0f / a;
  if (threadIdx.x == 0) scale[r] = finite ? a / 127.0f : __builtin_nanf("");
  // byte offset of column c: tiles of 1 KiB, 256 bytes for each 16 columns
  uint8_t* out = codes + (r >> 4) * (padded >> 6) * 1024 + (r & 15) * 16;
  for (int64_t c = (int64_t)threadIdx.x * 16; c < padded; c += kQThreads * 16) {
    v4u q = {0, 0, 0, 0};
    if (finite && top != 0 && c < n_cols) {
      float f[16];
      load16<TYPE, VEC>(x, row, c, n_cols, f);
      uint32_t w[4];
      codes_of<16>(f, a, inv, w);
      q = v4u{w[0], w[1], w[2], w[3]};
    }
    *reinterpret_cast<v4u*>(out + (c >> 4) * 256) = q;
  }
}

template <int TYPE>
void launch_quantize(const void* x, int64_t rows, int64_t cols, int64_t stride, void* codes, float* scale,
                     hipStream_t s) {
  const int64_t padded = round_up(cols, 128);
  const int elt = TYPE == AS_F32 ? 4 : 2;
  const bool vec = aligned(x, 16) && (stride * elt) % 16 == 0;
  const dim3 g((unsigned)rows), t(kQThreads);
  if (vec)
    hipLaunchKernelGGL((quantize_rows<TYPE, true>), g, t, 0, s, x, cols, stride, padded, (uint8_t*)codes, scale);
  else
    hipLaunchKernelGGL((quantize_rows<TYPE, false>), g, t, 0, s, x, cols, stride, padded, (uint8_t*)codes, scale);
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
  bool y_vec;            // four neighbouring channels can be stored at once
  // activations, where the product quantises them
  const void* x;
  int64_t x_stride;
  int32_t n_in;
  bool x_aligned;        // rows aligned to 16 bytes
};

template <int YTYPE>
__device__ __forceinline__ void store_one(void* y, int64_t i, float v) {
  if (YTYPE == AS_F32)
    reinterpret_cast<float*>(y)[i] = v;
  else
    reinterpret_cast<uint16_t*>(y)[i] = from_f32<YTYPE>(v);
}

template <int YTYPE>
__device__ __forceinline__ void store_four(void* y, int64_t i, const float (&v)[4]) {
  if (YTYPE == AS_F32) {
    *reinterpret_cast<v4f*>(reinterpret_cast<float*>(y) + i) = v4f{v[0], v[1], v[2], v[3]};
  } else {
    const uint32_t lo = from_f32<YTYPE>(v[0]) | (uint32_t)from_f32<YTYPE>(v[1]) << 16;
    const uint32_t hi = from_f32<YTYPE>(v[2]) | (uint32_t)from_f32<YTYPE>(v[3]) << 16;
    *reinterpret_cast<v2u*>(reinterpret_cast<uint16_t*>(y) + i) = v2u{lo, hi};
  }
}

// 8 values from column c of a row of 16-bit values; columns beyond n are 0.
template <int TYPE>
__device__ __forceinline__ void load8(const uint16_t* x, int64_t row, int c, int n, bool vec, float (&f)[8]) {
  if (vec && c + 8 <= n) {
    const v4u v = *reinterpret_cast<const v4u*>(x + row + c);
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

// Barrier of a workgroup that orders its LDS accesses alone: loads from memory
// stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Few tokens: the weights' bytes bound it, each read once.  One workgroup takes
// 16 CT channels and all tokens; its eight wavefronts share out the columns and
// add their sums in LDS (whole numbers: the order does not matter).  Weights go
// from memory to registers, 1 KiB a load, several in flight.
// FUSED (at most 16 tokens): the workgroup quantises the activations itself,
// into LDS, with its first weights already on their way; this repeats little
// work in every workgroup and saves a launch.
constexpr int kFewWaves = 8;

template <int YTYPE, int XTYPE, int CT, int TT, bool FUSED>
__global__ __launch_bounds__(64 * kFewWaves) void product_few(LinArgs p) {
  extern __shared__ uint8_t lds[];
  int* sums = reinterpret_cast<int*>(lds);                       // [TT][16 tokens][CT * 16 channels]
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
  constexpr int kAhead = CT == 1 ? 8 : CT == 2 ? 4 : 2;
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
    for (int t = 0; t < p.n_tokens; ++t) {
      uint32_t top = 0;
      for (int c = tid; c < chunks; c += 64 * kFewWaves) {
        float f[8];
        load8<XTYPE>(x, t * p.x_stride, c * 8, p.n_in, p.x_aligned, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, magnitude(f[i]));
      }
#pragma unroll
      for (int o = 32; o; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
      if (lane == 0) atomicMax(&tops[t], top);
    }
    lds_barrier();
    for (int t = 0; t < p.n_tokens; ++t) {
      const uint32_t top = tops[t];
      const bool zero = top == 0 || top >= 0x7f800000u;
      const float a = zero ? 1.0f : __uint_as_float(top), inv = 127.0f / a;
      for (int c = tid; c < chunks; c += 64 * kFewWaves) {
        float f[8];
        load8<XTYPE>(x, t * p.x_stride, c * 8, p.n_in, p.x_aligned, f);
        uint32_t q[2] = {0, 0};
        if (!zero) codes_of<8>(f, a, inv, q);
        *reinterpret_cast<v2u*>(rows + t * row_bytes + c * 8) = v2u{q[0], q[1]};
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
        atomicAdd(&sums[(u * 16 + (lane & 15)) * (CT * 16) + i * 16 + (lane >> 4) * 4 + r], acc[i][u][r]);
  lds_barrier();
  for (int j = tid; j < TT * CT * 256; j += 64 * kFewWaves) {
    const int t = j / (CT * 16), n = ct0 * 16 + j % (CT * 16);
    if (t >= p.n_tokens || n >= p.n_out) continue;
    float s;
    if (FUSED)
      s = tops[t] < 0x7f800000u ? __uint_as_float(tops[t]) / 127.0f : __builtin_nanf("");
    else
      s = p.a_scale[t];
    finish<YTYPE>(p, t, n, sums[j], s);
  }
}

// Many tokens: the matrix rate bounds it.  A workgroup of WC x WT wavefronts takes
// 16 TC channels x 16 TT tokens, two tiles of 64 columns at a time: they come
// into one half of LDS straight from memory (a tile is a contiguous KiB there
// and in LDS, read back without bank conflicts) while the other half is
// multiplied.  Neighbouring workgroup numbers go to different XCDs, so each XCD
// gets a contiguous run of tiles in an order that walks the channels in bands
// of 8: the tiles that run together share rows of both operands in its L2.
template <int YTYPE, int TC, int TT, int WC, int WT>
__global__ __launch_bounds__(64 * WC * WT) void product_many(LinArgs p) {
  constexpr int kW = WC * WT, kC = TC / WC, kT = TT / WT, kStage = (TC + TT) * 2;
  extern __shared__ uint8_t lds[];  // [2][kStage][1024]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_ct = (p.n_out + 15) / 16, n_tt = (p.n_tokens + 15) / 16;
  const int gc = (n_ct + TC - 1) / TC, gt = (n_tt + TT - 1) / TT;
  const int total = gc * gt, id = blockIdx.x;
  const int share = total / 8, more = total % 8, xcd = id & 7;
  const int at = xcd * share + min(xcd, more) + (id >> 3);
  const int band = at / (8 * gt), wide = min(8, gc - band * 8), in_band = at - band * 8 * gt;
  const int c0 = (band * 8 + in_band % wide) * TC, t0 = in_band / wide * TT;
  const int64_t tile_row = (int64_t)p.k_tiles * 1024;

  // The tiles that this wavefront brings in: i, i + kW, ..
  auto bring = [&](int half, int k) {
#pragma unroll
    for (int j = 0; j < kStage / kW; ++j) {
      const int i = wave + j * kW, r = i >> 1;
      const uint8_t* src = r < TC ? p.w + min(c0 + r, n_ct - 1) * tile_row : p.a + min(t0 + r - TC, n_tt - 1) * tile_row;
      src += (int64_t)(k + (i & 1)) * 1024 + lane * 16;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                       (__attribute__((address_space(3))) void*)(lds + (half * kStage + i) * 1024), 16, 0,
                                       0);
    }
  };
  const int wc = wave % WC * kC, wt = wave / WC * kT;
  v4i acc[kC][kT] = {};
  bring(0, 0);
  __syncthreads();
  int half = 0;
  for (int k = 0; k < p.k_tiles; k += 2, half ^= 1) {
    if (k + 2 < p.k_tiles) bring(half ^ 1, k + 2);
    const uint8_t* here = lds + half * kStage * 1024 + lane * 16;
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      v4i a[kC], b[kT];
#pragma unroll
      for (int i = 0; i < kC; ++i) a[i] = *reinterpret_cast<const v4i*>(here + ((wc + i) * 2 + z) * 1024);
#pragma unroll
      for (int i = 0; i < kT; ++i) b[i] = *reinterpret_cast<const v4i*>(here + ((TC + wt + i) * 2 + z) * 1024);
#pragma unroll
      for (int i = 0; i < kC; ++i)
#pragma unroll
        for (int j = 0; j < kT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[i], b[j], acc[i][j], 0, 0, 0);
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < kT; ++j) {
    const int t = (t0 + wt + j) * 16 + (lane & 15);
    if (t >= p.n_tokens) continue;
    const float s = p.a_scale[t];
#pragma unroll
    for (int i = 0; i < kC; ++i) {
      const int n = (c0 + wc + i) * 16 + (lane >> 4) * 4;
      if (p.y_vec && n + 4 <= p.n_out) {
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          v[r] = (float)acc[i][j][r] * s * p.w_scale[n + r];
          if (p.bias) v[r] += p.bias[n + r];
        }
        store_four<YTYPE>(p.y, (int64_t)t * p.y_stride + n, v);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (n + r < p.n_out) finish<YTYPE>(p, t, n + r, acc[i][j][r], s);
      }
    }
  }
}

template <int YTYPE, int TC, int TT, int WC, int WT>
int launch_many(const LinArgs& p, hipStream_t s) {
  const int64_t gc = ((p.n_out + 15) / 16 + TC - 1) / TC, gt = ((p.n_tokens + 15) / 16 + TT - 1) / TT;
  const size_t lds = (size_t)2 * (TC + TT) * 2 * 1024;
  const int rc = allow_lds<&product_many<YTYPE, TC, TT, WC, WT>>(lds, "linear_i8");
  if (rc != AS_OK) return rc;
  hipLaunchKernelGGL((product_many<YTYPE, TC, TT, WC, WT>), dim3((unsigned)(gc * gt)), dim3(64 * WC * WT), lds, s, p);
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
  if (n_ct >= 4 * cus) return launch_few<YTYPE, XTYPE, 4, TT, FUSED>(p, s);
  if (n_ct >= 2 * cus) return launch_few<YTYPE, XTYPE, 2, TT, FUSED>(p, s);
  return launch_few<YTYPE, XTYPE, 1, TT, FUSED>(p, s);
}

template <int YTYPE>
int launch_product(const LinArgs& p, hipStream_t s) {
  const int n_tt = (p.n_tokens + 15) / 16;
  if (n_tt == 1) return few_by_channels<YTYPE, AS_BF16, 1, false>(p, s);
  if (n_tt == 2) return few_by_channels<YTYPE, AS_BF16, 2, false>(p, s);
  if (n_tt == 3) return few_by_channels<YTYPE, AS_BF16, 3, false>(p, s);
  if (n_tt == 4) return few_by_channels<YTYPE, AS_BF16, 4, false>(p, s);
  const int64_t n_ct = (p.n_out + 15) / 16, cus = as_host::compute_units();
  if (((n_ct + 15) / 16) * ((n_tt + 15) / 16) >= cus) return launch_many<YTYPE, 16, 16, 2, 4>(p, s);
  if (((n_ct + 7) / 8) * ((n_tt + 7) / 8) >= cus) return launch_many<YTYPE, 8, 8, 2, 2>(p, s);
  return launch_many<YTYPE, 4, 4, 2, 2>(p, s);
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

constexpr int64_t kMaxRows = 1 << 24;

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
  // rows of 16 tokens are a grid's second dimension
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
  const int y_bytes = y_type == AS_F32 ? 4 : 2;
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
  p.y_vec = aligned(y, 4 * y_bytes) && y_stride % 4 == 0;
  p.x = x;
  p.x_stride = x_stride;
  p.n_in = (int32_t)n_in;
  p.x_aligned = aligned(x, 16) && x_stride % 8 == 0;
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
