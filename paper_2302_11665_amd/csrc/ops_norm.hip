// Rows brought to mean square 1 and held in 8 bits (alpaserve_ops.h): a residual
// added, the root-mean-square norm, a gain, codes and a scale per row.
//
// The code of an element is that of its share of the row's largest magnitude, so
// the norm's root cancels from it: codes are those of t = h g, and only the scale,
// max |t| / (127 sqrt(mean h^2 + eps)), needs the sum of squares.  Both reductions
// therefore run side by side, over values that stay in registers.
#include "ops_quant.hpp"

using as_host::fail;

namespace as_ops {

struct NormArgs {
  const uint16_t *x, *residual;  // residual may be null
  const float* gain;             // [n_cols] or null
  uint16_t* sum;                 // where there is a residual
  uint8_t* codes;
  float *scale, *held;           // held may be null
  int64_t n_tokens, x_stride, residual_stride, sum_stride;
  int32_t n_cols, k_tiles;
  float eps;
  bool past;  // write the sum past the caches
};

// A wavefront takes 1024 / ROWS columns of ROWS rows at a time, lane `at` of a row's
// 64 / ROWS two pieces of 8 columns: from column c + 8 at, and as many lanes further on.
// A load or store then takes a row's columns side by side.
template <int ROWS>
__device__ __forceinline__ int piece_of(int z) {
  return (z * (64 / ROWS) + (threadIdx.x & 63) / ROWS) * 8;
}

typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(2)));  // at any 16-bit value

// A lane's pieces of a row of 16-bit values, two to a word; columns beyond n are 0.
template <int ROWS>
__device__ __forceinline__ void read16(const uint16_t* row, int c, int n, v4u (&w)[2]) {
#pragma unroll
  for (int z = 0; z < 2; ++z) {
    const int at = c + piece_of<ROWS>(z);
    w[z] = v4u{0, 0, 0, 0};
    if (at + 8 <= n) {
      __builtin_memcpy(&w[z], row + at, 16);
    } else if (at < n) {  // all loads at once: one latency, not one after the other
      uint16_t u[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = row[min(at + e, n - 1)];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[z][e >> 1] |= (uint32_t)(at + e < n ? u[e] : 0) << (16 * (e & 1));
    }
  }
}

template <int ROWS>
__device__ __forceinline__ void write16(uint16_t* row, int c, int n, const v4u (&w)[2], bool past) {
#pragma unroll
  for (int z = 0; z < 2; ++z) {
    const int at = c + piece_of<ROWS>(z);
    if (at + 8 <= n && past) {
      __builtin_nontemporal_store((v4u_any)w[z], reinterpret_cast<v4u_any*>(row + at));
    } else if (at + 8 <= n) {
      __builtin_memcpy(row + at, &w[z], 16);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < n) row[at + e] = (uint16_t)(w[z][e >> 1] >> (16 * (e & 1)));
    }
  }
}

template <int TYPE>
__device__ __forceinline__ void unpack16(const v4u (&w)[2], float (&f)[16]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    f[2 * j] = to_f32<TYPE>(w[j >> 2][j & 3] & 0xffffu);
    f[2 * j + 1] = to_f32<TYPE>(w[j >> 2][j & 3] >> 16);
  }
}

// w += r, rounded to the type: the sum that is kept is the one that is normed.
template <int TYPE>
__device__ __forceinline__ void add16(v4u (&w)[2], const v4u (&r)[2]) {
  float a[16], b[16];
  unpack16<TYPE>(w, a);
  unpack16<TYPE>(r, b);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    w[j >> 2][j & 3] = (uint32_t)from_f32<TYPE>(a[2 * j] + b[2 * j]) |
                       (uint32_t)from_f32<TYPE>(a[2 * j + 1] + b[2 * j + 1]) << 16;
}

// The gains of a lane's pieces; 0 beyond n.
template <int ROWS>
__device__ __forceinline__ void gain16(const float* gain, int c, int n, float (&g)[16]) {
#pragma unroll
  for (int z = 0; z < 2; ++z) {
    const int at = c + piece_of<ROWS>(z);
    if (at + 8 <= n) {
      __builtin_memcpy(g + 8 * z, gain + at, 16);
      __builtin_memcpy(g + 8 * z + 4, gain + at + 4, 16);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[8 * z + e] = gain[min(at + e, n - 1)];
#pragma unroll
      for (int e = 0; e < 8; ++e) g[8 * z + e] = at + e < n ? g[8 * z + e] : 0.0f;
    }
  }
}

// A row's scale from its largest |t| and its sum of squares.  One lane's work: in
// 64 bits, since nothing waits for it.
__device__ __forceinline__ float norm_scale(float top, bool finite, double squares, int n_cols, float eps) {
  if (!finite) return __builtin_nanf("");
  if (top == 0.0f) return 0.0f;
  return (float)((double)top / (127.0 * sqrt(squares / n_cols + (double)eps)));
}

// Sums of squares that fp32 holds without loss: beyond them a row is summed again
// in 64 bits (16-bit values reach 3e38 in bf16, whose square does not).
__device__ __forceinline__ bool fp32_holds(float squares) { return squares > 0x1p-60f && squares < 0x1p120f; }

// Largest magnitude and sum of squares of a lane's t and h.
template <bool GAIN>
__device__ __forceinline__ void measure16(const float (&f)[16], const float (&g)[16], uint32_t& top, float& squares) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    squares = fmaf(f[e], f[e], squares);
    top = max(top, magnitude(GAIN ? f[e] * g[e] : f[e]));
  }
}

// Codes of a lane's h (two to a word) go through LDS (`own`, of the wavefront alone) and
// out, 16 columns to a lane as the tiles have them, and where held is not null the values
// that they stand for, 4 columns to a lane at a time.
template <int TYPE, bool GAIN, int ROWS>
__device__ __forceinline__ void put_codes(const NormArgs& p, const Quantiser<GAIN ? AS_F32 : TYPE>& quantiser,
                                          const v4u (&w)[2], int c, uint8_t* tile, float* held, float scale, bool there,
                                          v4u* own) {
  constexpr int kLanes = 64 / ROWS;
  const int lane = threadIdx.x & 63, in = lane % ROWS, at = lane / ROWS;
  float f[16], g[16];
  unpack16<TYPE>(w, f);
  if (GAIN) {
    gain16<ROWS>(p.gain, c, p.n_cols, g);
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] *= g[e];
  }
  v4u* row = own + in * kLanes;
#pragma unroll
  for (int z = 0; z < 2; ++z)
    reinterpret_cast<v2u*>(row)[z * kLanes + at] = v2u{quantiser.codes4(f + 8 * z), quantiser.codes4(f + 8 * z + 4)};
  __builtin_amdgcn_wave_barrier();
  // (rows behind the last one are in its tile's storage)
  if (c + at * 16 < p.k_tiles * 64) *reinterpret_cast<v4u*>(tile + (int64_t)((c >> 4) + at) * 256) = row[at];
  if (held) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t four = reinterpret_cast<const uint32_t*>(row)[i * kLanes + at];
      const int from = c + (i * kLanes + at) * 4;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (float)(int8_t)(four >> (8 * e)) * scale;
      if (!there) continue;
      if (from + 4 <= p.n_cols) {
        typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));
        __builtin_nontemporal_store(v4f_any{v[0], v[1], v[2], v[3]}, reinterpret_cast<v4f_any*>(held + from));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (from + e < p.n_cols) held[from + e] = v[e];
      }
    }
  }
  __builtin_amdgcn_wave_barrier();
}

// One workgroup per row, 16 columns to a thread (KEEP), which stay in registers;
// rows of more than those are gone over twice, the second time from the caches
// (131,072 columns with a residual and a gain: one row 27 us, 48 rows 36, 2048 rows 680, of
// which 370 are the 7 bytes a value that it cannot do without; 16,384, which stay in
// registers, 5.5, 6.3 and 48).
// Latency bounds a few rows: a launch, the loads, two exchanges (4096 columns: one row
// 3.9 us, 48 rows 4.1, 256 rows 5.0, with a residual and a gain).
template <int TYPE, bool GAIN, bool KEEP>
__global__ __launch_bounds__(1024) void norm_rows(NormArgs p) {
  constexpr int kStep = KEEP ? 1 << 30 : 16 * 1024;
  __shared__ uint32_t tops[16];
  __shared__ float sums[16];
  __shared__ double wide[16];
  const int waves = blockDim.x >> 6;
  __shared__ float row_scale;
  __shared__ v4u words[16][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, padded = p.k_tiles * 64;
  const int64_t r = blockIdx.x;
  const uint16_t* x = p.x + r * p.x_stride;
  const uint16_t* add = p.residual ? p.residual + r * p.residual_stride : nullptr;
  uint16_t* sum = p.sum + r * p.sum_stride;
  const uint16_t* h = add ? sum : x;  // what is read again
  uint32_t top = 0;
  float squares = 0.0f;
  v4u kept[2] = {};
  for (int c = wave * 1024; c < padded; c += kStep) {
    v4u w[2], b[2];
    float f[16], g[16];
    read16<1>(x, c, p.n_cols, w);
    if (add) read16<1>(add, c, p.n_cols, b);
    if (GAIN) gain16<1>(p.gain, c, p.n_cols, g);
    if (add) {
      add16<TYPE>(w, b);
      write16<1>(sum, c, p.n_cols, w, p.past);
    }
    unpack16<TYPE>(w, f);
    measure16<GAIN>(f, g, top, squares);
    kept[0] = w[0], kept[1] = w[1];
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    top = max(top, (uint32_t)__shfl_xor((int)top, o));
    squares += __shfl_xor(squares, o);
  }
  if (lane == 0) tops[wave] = top, sums[wave] = squares;
  lds_barrier();
  squares = 0.0f;
  for (int i = 0; i < waves; ++i) {
    top = max(top, tops[i]);
    squares += sums[i];
  }
  const bool finite = top < 0x7f800000u;
  double total = squares;
  if (finite && top != 0 && !fp32_holds(squares)) {
    double d = 0.0;
    for (int c = wave * 1024; c < padded; c += kStep) {
      v4u w[2] = {kept[0], kept[1]};
      float f[16];
      if (!KEEP) read16<1>(h, c, p.n_cols, w);
      unpack16<TYPE>(w, f);
#pragma unroll
      for (int e = 0; e < 16; ++e) d += (double)f[e] * f[e];
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) d += __shfl_xor(d, o);
    if (lane == 0) wide[wave] = d;
    lds_barrier();
    total = 0.0;
    for (int i = 0; i < waves; ++i) total += wide[i];
  }
  if (tid == 0) {
    row_scale = norm_scale(__uint_as_float(top), finite, total, p.n_cols, p.eps);
    p.scale[r] = row_scale;
  }
  if (p.held) lds_barrier();
  const Quantiser<GAIN ? AS_F32 : TYPE> quantiser(__uint_as_float(top), finite);
  uint8_t* out = p.codes + (r >> 4) * p.k_tiles * 1024 + (r & 15) * 16;
  for (int c = wave * 1024; c < padded; c += kStep) {
    v4u w[2] = {kept[0], kept[1]};
    if (!KEEP) read16<1>(h, c, p.n_cols, w);
    put_codes<TYPE, GAIN, 1>(p, quantiser, w, c, out, p.held ? p.held + r * p.n_cols : nullptr, row_scale, true, words[wave]);
  }
}

// Many rows: a workgroup of as many wavefronts as the columns need, up to 8, per
// two rows, a lane of which has 16 columns of one row, TIMES over, in registers.
// Rows are read once, and codes written 32 bytes side by side: 7 bytes a value in all, 11
// with the values held, which bound it (8192 rows of 8192 columns with a residual: 93 us, 5.0
// TB/s, with the values held 129 us, 5.7 TB/s; when a lane had 16 columns side by side, and its
// stores pieces of lines, 111 and 186).  Four rows a workgroup: 102 and 142 us; 16, whose codes
// are whole tiles, half as fast again: they wait for all of their loads at once.
constexpr int kNormRows = 2, kNormWaves = 8;

template <int TYPE, bool GAIN, int TIMES>
__global__ __launch_bounds__(64 * kNormWaves) void norm_pairs(NormArgs p) {
  constexpr int kWide = 16 * 64 / kNormRows;  // columns of a wavefront
  __shared__ uint32_t tops[kNormWaves][kNormRows];
  __shared__ float sums[kNormWaves][kNormRows];
  __shared__ double wide[kNormWaves][kNormRows];
  __shared__ float scales[kNormRows];
  __shared__ v4u words[kNormWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in = lane % kNormRows, waves = blockDim.x >> 6;
  const int64_t r = (int64_t)blockIdx.x * kNormRows + in;
  const bool there = r < p.n_tokens;
  const int64_t row = there ? r : p.n_tokens - 1;
  const uint16_t* x = p.x + row * p.x_stride;
  auto column = [&](int i) { return (i * waves + wave) * kWide; };
  v4u w[TIMES][2];
#pragma unroll
  for (int i = 0; i < TIMES; ++i) read16<kNormRows>(x, column(i), p.n_cols, w[i]);
  if (p.residual) {
    const uint16_t* add = p.residual + row * p.residual_stride;
#pragma unroll
    for (int i = 0; i < TIMES; ++i) {
      v4u b[2];
      read16<kNormRows>(add, column(i), p.n_cols, b);
      add16<TYPE>(w[i], b);
    }
    // (rows behind the last one do its work, which may be over before they read)
    if (there) {
#pragma unroll
      for (int i = 0; i < TIMES; ++i) write16<kNormRows>(p.sum + row * p.sum_stride, column(i), p.n_cols, w[i], p.past);
    }
  }
  uint32_t top = 0;
  float squares = 0.0f;
#pragma unroll
  for (int i = 0; i < TIMES; ++i) {
    float f[16], g[16];
    unpack16<TYPE>(w[i], f);
    if (GAIN) gain16<kNormRows>(p.gain, column(i), p.n_cols, g);
    measure16<GAIN>(f, g, top, squares);
  }
#pragma unroll
  for (int o = kNormRows; o < 64; o <<= 1) {
    top = max(top, (uint32_t)__shfl_xor((int)top, o));
    squares += __shfl_xor(squares, o);
  }
  if (lane < kNormRows) tops[wave][in] = top, sums[wave][in] = squares;
  lds_barrier();
  squares = 0.0f;
  for (int i = 0; i < waves; ++i) {
    top = max(top, tops[i][in]);
    squares += sums[i][in];
  }
  const bool finite = top < 0x7f800000u;
  double total = squares;
  // (a row's lanes agree, the rows of a workgroup need not: two barriers then)
  const bool again = finite && top != 0 && !fp32_holds(squares);
  const bool rare = __any(again);  // every wavefront has lanes of all rows
  if (rare) {
    double d = 0.0;
#pragma unroll
    for (int i = 0; i < TIMES; ++i) {
      float f[16];
      unpack16<TYPE>(w[i], f);
#pragma unroll
      for (int e = 0; e < 16; ++e) d += (double)f[e] * f[e];
    }
#pragma unroll
    for (int o = kNormRows; o < 64; o <<= 1) d += __shfl_xor(d, o);
    if (lane < kNormRows) wide[wave][in] = d;
    lds_barrier();
    if (again) {
      total = 0.0;
      for (int i = 0; i < waves; ++i) total += wide[i][in];
    }
  }
  if (threadIdx.x < kNormRows) {
    scales[in] = norm_scale(__uint_as_float(top), finite, total, p.n_cols, p.eps);
    if (there) p.scale[r] = scales[in];
  }
  if (p.held) lds_barrier();
  const Quantiser<GAIN ? AS_F32 : TYPE> quantiser(__uint_as_float(top), finite);
  uint8_t* out = p.codes + (r >> 4) * p.k_tiles * 1024 + (r & 15) * 16;
#pragma unroll
  for (int i = 0; i < TIMES; ++i)
    put_codes<TYPE, GAIN, kNormRows>(p, quantiser, w[i], column(i), out, p.held ? p.held + r * p.n_cols : nullptr, scales[in],
                                     there, words[wave]);
}

template <int TYPE, bool GAIN>
void launch_norm(const NormArgs& p, hipStream_t s) {
  auto launch = [&](auto kernel, int64_t groups, int threads) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(threads), 0, s, p);
  };
  constexpr int kOnce = 16 * 64 / kNormRows;  // columns of a wavefront at a time
  // (a row to a workgroup and two, 4096 columns: 48 rows 4.1 and 4.5 us, 256 rows 5.0
  // and 4.9, 384 rows 6.2 and 5.3)
  if (p.n_tokens > as_host::compute_units() && p.n_cols <= 4 * kOnce * kNormWaves) {
    const int times = p.n_cols <= kOnce * kNormWaves ? 1 : p.n_cols <= 2 * kOnce * kNormWaves ? 2 : 4;
    const int threads = (p.n_cols + times * kOnce - 1) / (times * kOnce) * 64;
    const int64_t groups = (p.n_tokens + kNormRows - 1) / kNormRows;
    if (times == 1) return launch(norm_pairs<TYPE, GAIN, 1>, groups, threads);
    if (times == 2) return launch(norm_pairs<TYPE, GAIN, 2>, groups, threads);
    return launch(norm_pairs<TYPE, GAIN, 4>, groups, threads);
  }
  if (p.n_cols <= 16384)
    launch(norm_rows<TYPE, GAIN, true>, p.n_tokens, (int)round_up((p.n_cols + 15) / 16, 64));
  else
    launch(norm_rows<TYPE, GAIN, false>, p.n_tokens, 1024);
}

// Whether rows of n elements of 16 bits from a share memory with those from b
// without being them.
bool clashes(const void* a, int64_t a_stride, const void* b, int64_t b_stride, int64_t rows, int64_t n) {
  const int64_t u = (int64_t)((uintptr_t)a / 2), w = (int64_t)((uintptr_t)b / 2);
  if (rows == 1) a_stride = b_stride = n;
  if (u == w && a_stride == b_stride) return (uintptr_t)a != (uintptr_t)b;
  if (u + (rows - 1) * a_stride + n <= w || w + (rows - 1) * b_stride + n <= u) return false;
  if (a_stride != b_stride) return true;
  const int64_t d = ((w - u) % a_stride + a_stride) % a_stride;  // columns of one buffer, side by side
  return d < n || a_stride - d < n;
}

}  // namespace as_ops

using namespace as_ops;

extern "C" int as_norm_i8(const void* x, const void* residual, int32_t type, int64_t n_tokens, int64_t n_cols,
                          int64_t x_stride, int64_t residual_stride, const float* gain, float eps, void* sum,
                          int64_t sum_stride, void* codes, float* scale, float* held, void* stream) {
  if (type != AS_BF16 && type != AS_F16) return fail(AS_E_INVALID_ARG, "norm_i8: type %d", type);
  if (n_tokens < 0 || n_cols < 1 || x_stride < n_cols || (residual && (residual_stride < n_cols || sum_stride < n_cols)))
    return fail(AS_E_INVALID_ARG, "norm_i8: %lld tokens of %lld columns, strides %lld, %lld and %lld",
                (long long)n_tokens, (long long)n_cols, (long long)x_stride, (long long)residual_stride,
                (long long)sum_stride);
  if (!(eps >= 0.0f) || eps > 3.4e38f) return fail(AS_E_INVALID_ARG, "norm_i8: eps %g", (double)eps);
  // (a workgroup of up to 1024 threads to a row, fewer than 2^32 threads a launch)
  if (n_tokens > 65535 * 16 || n_cols > AS_I8_MAX_INPUTS)
    return fail(AS_E_LIMITS, "norm_i8: at most %d tokens of %d columns", 65535 * 16, AS_I8_MAX_INPUTS);
  if (n_tokens == 0) return as_host::ok();
  if (!x || !codes || !scale || (residual != nullptr) != (sum != nullptr))
    return fail(AS_E_INVALID_ARG, "norm_i8: null pointer, or one of residual and sum alone");
  if (!aligned(codes, 16)) return fail(AS_E_INVALID_ARG, "norm_i8: codes not aligned to 16 bytes");
  if (sum && (clashes(sum, sum_stride, x, x_stride, n_tokens, n_cols) ||
              clashes(sum, sum_stride, residual, residual_stride, n_tokens, n_cols)))
    return fail(AS_E_INVALID_ARG, "norm_i8: the sum shares memory with other rows of x or the residual");
  NormArgs p{};
  p.x = reinterpret_cast<const uint16_t*>(x);
  p.residual = reinterpret_cast<const uint16_t*>(residual);
  p.gain = gain;
  p.sum = reinterpret_cast<uint16_t*>(sum);
  p.codes = reinterpret_cast<uint8_t*>(codes);
  p.scale = scale;
  p.held = held;
  p.n_tokens = n_tokens;
  p.x_stride = x_stride;
  p.residual_stride = residual_stride;
  p.sum_stride = sum_stride;
  p.n_cols = (int32_t)n_cols;
  p.k_tiles = (int32_t)(round_up(n_cols, 128) / 64);
  p.eps = eps;
  // What one call reads and writes beyond the last cache's 256 MiB is not found there by the
  // next one, and writing it past the caches is faster (8192 rows of 5000 columns 85 us and
  // 62, of 8192 111 and 93; of 4096, which it holds, 41 and 46).  Held values, which have
  // the most bytes, always are (2048 rows of 8192 columns 32 us and 31, 8192 of 8192 186
  // and 129).
  p.past = n_tokens * n_cols * (held ? 11 : 7) > (int64_t(256) << 20);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (type == AS_BF16)
    gain ? launch_norm<AS_BF16, true>(p, s) : launch_norm<AS_BF16, false>(p, s);
  else
    gain ? launch_norm<AS_F16, true>(p, s) : launch_norm<AS_F16, false>(p, s);
  return launched("norm_i8");
}
