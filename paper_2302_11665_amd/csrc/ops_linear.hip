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

// Codes of 16 values.  127 x is exact for 16-bit x, and its quotient cannot
// round to a tie that it is not, so the codes are those of exact arithmetic.
__device__ __forceinline__ v4u codes16(const float (&f)[16], float top) {
  v4u out;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int q = (int)rintf(f[4 * i + j] * 127.0f / top);
      w |= ((uint32_t)q & 0xffu) << (8 * j);
    }
    out[i] = w;
  }
  return out;
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
  const float a = __uint_as_float(top);
  if (threadIdx.x == 0) scale[r] = finite ? a / 127.0f : __builtin_nanf("");
  // byte offset of column c: tiles of 1 KiB, 256 bytes for each 16 columns
  uint8_t* out = codes + (r >> 4) * (padded >> 6) * 1024 + (r & 15) * 16;
  for (int64_t c = (int64_t)threadIdx.x * 16; c < padded; c += kQThreads * 16) {
    v4u q = {0, 0, 0, 0};
    if (finite && top != 0 && c < n_cols) {
      float f[16];
      load16<TYPE, VEC>(x, row, c, n_cols, f);
      q = codes16(f, a);
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
};

template <int YTYPE>
__device__ __forceinline__ void store_one(void* y, int64_t i, float v) {
  if (YTYPE == AS_F32)
    reinterpret_cast<float*>(y)[i] = v;
  else
    reinterpret_cast<uint16_t*>(y)[i] = from_f32<YTYPE>(v);
}

// One wavefront per 64 channels x 16 tokens, operands straight from memory.
// The weights are the instruction's rows: a lane then holds four neighbouring
// channels of one token.
template <int YTYPE>
__global__ __launch_bounds__(256) void product(LinArgs p) {
  const int lane = threadIdx.x & 63;
  const int ct = (blockIdx.x * 4 + (threadIdx.x >> 6)) * 4;  // first of its four channel tiles
  const int n_ct = (p.n_out + 15) / 16;
  if (ct >= n_ct) return;
  const int64_t tile_row = (int64_t)p.k_tiles * 1024;
  const uint8_t* a = p.a + blockIdx.y * tile_row + lane * 16;
  const uint8_t* w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = p.w + min(ct + i, n_ct - 1) * tile_row + lane * 16;
  v4i acc[4] = {};
  for (int k = 0; k < p.k_tiles; ++k) {
    const v4i b = *reinterpret_cast<const v4i*>(a + (int64_t)k * 1024);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const v4i*>(w[i] + (int64_t)k * 1024), b,
                                                     acc[i], 0, 0, 0);
  }
  const int t = blockIdx.y * 16 + (lane & 15);
  if (t >= p.n_tokens) return;
  const float s = p.a_scale[t];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int n = (ct + i) * 16 + (lane >> 4) * 4 + r;
      if (n < p.n_out) {
        float v = (float)acc[i][r] * s * p.w_scale[n];
        if (p.bias) v += p.bias[n];
        store_one<YTYPE>(p.y, t * p.y_stride + n, v);
      }
    }
}

template <int YTYPE>
void launch_product(const LinArgs& p, hipStream_t s) {
  const dim3 g((unsigned)((p.n_out + 255) / 256), (unsigned)((p.n_tokens + 15) / 16));
  hipLaunchKernelGGL((product<YTYPE>), g, dim3(256), 0, s, p);
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
  if (x_type == AS_BF16)
    launch_quantize<AS_BF16>(x, n_tokens, n_in, x_stride, codes, scale, s);
  else
    launch_quantize<AS_F16>(x, n_tokens, n_in, x_stride, codes, scale, s);
  LinArgs p{codes, scale, reinterpret_cast<const uint8_t*>(w), w_scale, bias, y, y_stride, (int32_t)n_tokens,
            (int32_t)n_out, (int32_t)(round_up(n_in, 128) / 64)};
  if (y_type == AS_BF16)
    launch_product<AS_BF16>(p, s);
  else if (y_type == AS_F16)
    launch_product<AS_F16>(p, s);
  else
    launch_product<AS_F32>(p, s);
  return launched("linear_i8");
}

}  // extern "C"
