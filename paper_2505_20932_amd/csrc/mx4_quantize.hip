// Microscaled 4-bit floating point: quantizer and its inverse.  A block of 32 consecutive values of a row shares a
// power of two 2^e, e = clamp(floor(log2(max |x|)) - 2, -127, 127), stored as the byte e + 127; an element is the E2M1
// number (0, .5, 1, 1.5, 2, 3, 4, 6 with a sign) nearest to x / 2^e, ties to the even code, 6 beyond.
//
// Bound: HBM (2 or 4 bytes read, 17/32 written per value; 16384 x 11008 bf16: 82 us = 5.6 TB/s, the inverse 71).
// A lane takes eight consecutive values, so a wavefront reads 512 values of a row in whole lines; four lanes share a block, whose maximum is two cross-lane steps, and eight codes
// make the word that a lane stores.  The maximum is taken on the bit patterns, as whole numbers: their order is that
// of the magnitudes, a NaN or an infinity comes out on top and its exponent field tells it apart.  Division by 2^e is a multiplication
// by 2^-e: exact, unless the quotient is below 2^-126, where the code is zero either way.
#include "cwac_internal.h"
#include "mx4.h"

namespace cwac {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

// STREAM: past the caches, for values that would only push the codes out of them.
template <bool STREAM, typename V>
__device__ __forceinline__ V load16(const V *p) {
  if constexpr (STREAM)
    return __builtin_nontemporal_load(p);
  else
    return *p;
}

template <bool STREAM, typename V>
__device__ __forceinline__ void store16(V *p, V v) {
  if constexpr (STREAM)
    __builtin_nontemporal_store(v, p);
  else
    *p = v;
}

// Eight consecutive values as they lie in memory, and as fp32.
template <int TYPE>
struct Eight;
template <>
struct Eight<CWAC_OUT_FP32> {
  v4f a, b;
  static constexpr int SIZE = 4;
  template <bool STREAM>
  __device__ __forceinline__ void load(const char *p) {
    a = load16<STREAM>(reinterpret_cast<const v4f *>(p));
    b = load16<STREAM>(reinterpret_cast<const v4f *>(p) + 1);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[i + 4] = b[i];
  }
  template <bool STREAM>
  __device__ static __forceinline__ void store(char *p, const float (&v)[8]) {
    store16<STREAM>(reinterpret_cast<v4f *>(p), v4f{v[0], v[1], v[2], v[3]});
    store16<STREAM>(reinterpret_cast<v4f *>(p) + 1, v4f{v[4], v[5], v[6], v[7]});
  }
};
template <>
struct Eight<CWAC_OUT_FP16> {
  h8 a;
  static constexpr int SIZE = 2;
  template <bool STREAM>
  __device__ __forceinline__ void load(const char *p) { a = load16<STREAM>(reinterpret_cast<const h8 *>(p)); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
  }
  template <bool STREAM>
  __device__ static __forceinline__ void store(char *p, const float (&v)[8]) {
    h8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (_Float16)v[i];
    store16<STREAM>(reinterpret_cast<h8 *>(p), r);
  }
};
template <>
struct Eight<CWAC_OUT_BF16> {
  u4 a;
  static constexpr int SIZE = 2;
  template <bool STREAM>
  __device__ __forceinline__ void load(const char *p) { a = load16<STREAM>(reinterpret_cast<const u4 *>(p)); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(a[i] << 16);
      v[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
  }
  // the numbers of a block have two significant bits: their upper half is all of them (2^-128, the smallest, included)
  template <bool STREAM>
  __device__ static __forceinline__ void store(char *p, const float (&v)[8]) {
    u4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (__float_as_uint(v[2 * i]) >> 16) | (__float_as_uint(v[2 * i + 1]) & 0xffff0000u);
    store16<STREAM>(reinterpret_cast<u4 *>(p), r);
  }
};

constexpr int kThreads = 256;
constexpr int kChunk = 512;  // values of a row that a wavefront takes at a time

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// ROWS consecutive rows x 512 values per wavefront and step: their loads are in flight together, and the scale bytes of a panel's
// rows, which lie side by side, go out in one store.
template <int TYPE, int ROWS, bool STREAM>
__global__ __launch_bounds__(kThreads) void mx4_quantize_kernel(const char *__restrict__ x, int64_t ldx, int64_t rows, int k,
                                                                uint8_t *__restrict__ codes, int64_t ldc,
                                                                uint8_t *__restrict__ scales, int chunks, int64_t tasks) {
  using E = Eight<TYPE>;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  for (int64_t task = (int64_t)blockIdx.x * (kThreads / 64) + wave; task < tasks; task += (int64_t)gridDim.x * (kThreads / 64)) {
    const int64_t r0 = task / chunks * ROWS;
    const int chunk = (int)(task % chunks), col = chunk * kChunk + lane * 8;
    const bool in = col < k;
    const int n = rows - r0 < ROWS ? (int)(rows - r0) : ROWS;
    E raw[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if (in && r < n) raw[r].template load<STREAM>(x + ((r0 + r) * ldx + col) * E::SIZE);
    uint32_t bytes[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      bytes[r] = 0;
      if (r >= n) continue;
      float v[8];
      uint32_t top = 0;
      if (in) {
        raw[r].get(v);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) top = umax(top, __float_as_uint(v[i]) & 0x7fffffffu);
      top = umax(top, dpp<0xb1>(top));  // the other lane of the pair, the other pair of the four
      top = umax(top, dpp<0x4e>(top));
      const uint32_t field = top >> 23;
      const uint32_t code = field == 255u ? 255u : (field > 2u ? field - 2u : 0u);
      const float inv = __uint_as_float((254u - code) << 23);
      uint32_t word = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= inv;
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[0], v[1], 1.0f, 0);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[2], v[3], 1.0f, 1);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[4], v[5], 1.0f, 2);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[6], v[7], 1.0f, 3);
      if (code == 255u) word = 0;
      if (in) *reinterpret_cast<uint32_t *>(codes + (r0 + r) * ldc + col / 2) = word;
      // four blocks' bytes to a word, in every lane of a row of 16
      uint32_t b = (in ? code : 0u) << (8 * ((lane >> 2) & 3));
      b |= dpp<0x124>(b);
      bytes[r] = b | dpp<0x128>(b);
    }
    // lane r of 16 stores row r's word
    uint32_t mine = bytes[0];
#pragma unroll
    for (int r = 1; r < ROWS; ++r) mine = (lane & 15) == r ? bytes[r] : mine;
    const int panel = chunk * (kChunk / kMx4Panel) + (lane >> 5);
    if ((lane & 15) < n && panel * kMx4Panel < k)
      *reinterpret_cast<uint32_t *>(scales + ((int64_t)panel * rows + r0 + (lane & 15)) * 8 + ((lane >> 4) & 1) * 4) = mine;
  }
}

template <int TYPE, int ROWS, bool STREAM>
__global__ __launch_bounds__(kThreads) void mx4_dequantize_kernel(const uint8_t *__restrict__ codes, int64_t ldc,
                                                                  const uint8_t *__restrict__ scales, int64_t rows, int k,
                                                                  char *__restrict__ out, int64_t ldo, int chunks, int64_t tasks) {
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  for (int64_t task = (int64_t)blockIdx.x * (kThreads / 64) + wave; task < tasks; task += (int64_t)gridDim.x * (kThreads / 64)) {
    const int64_t r0 = task / chunks * ROWS;
    const int col = (int)(task % chunks) * kChunk + lane * 8;
    if (col >= k) continue;
    const int n = rows - r0 < ROWS ? (int)(rows - r0) : ROWS;
    uint32_t words[ROWS], scale[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
      if (r < n) {
        words[r] = *reinterpret_cast<const uint32_t *>(codes + (r0 + r) * ldc + col / 2);
        scale[r] = scales[((int64_t)(col / kMx4Panel) * rows + r0 + r) * 8 + (col % kMx4Panel) / kMx4Block];
      }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (r >= n) break;
      const uint32_t word = words[r], code = scale[r];
      const float s = code == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(code ? code << 23 : 0x00400000u);
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // magnitudes 2 m = 0, 1, 2, 3, 4, 6, 8, 12, a nibble each
        const uint32_t c = (word >> (4 * i)) & 15u;
        const float m = 0.5f * (float)((0xc8643210u >> (4 * (c & 7u))) & 15u);
        v[i] = (c & 8u ? -m : m) * s;
      }
      Eight<TYPE>::template store<STREAM>(out + ((r0 + r) * ldo + col) * Eight<TYPE>::SIZE, v);
    }
  }
}

constexpr int64_t kMaxBlocks = 1 << 20;
// values of half the last-level cache and more would leave nothing of the codes in it
constexpr int64_t kStreamBytes = (int64_t)128 << 20;

template <int TYPE>
cwac_status launch_quantize(const void *x, int64_t ldx, int64_t rows, int k, uint8_t *codes, int64_t ldc, uint8_t *scales, hipStream_t st) {
  const int chunks = (int)ceil_div(k, kChunk);
  // eight rows to a wavefront once that still leaves wavefronts for every SIMD; single rows below
  const bool many = rows * chunks >= 8 * 4096;
  const bool stream = many && rows * k * Eight<TYPE>::SIZE >= kStreamBytes;
  const int64_t tasks = (many ? ceil_div(rows, 8) : rows) * chunks;
  const int64_t blocks = ceil_div(tasks, kThreads / 64);
  const dim3 grid((unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks));
  const char *xp = static_cast<const char *>(x);
  if (stream)
    mx4_quantize_kernel<TYPE, 8, true><<<grid, kThreads, 0, st>>>(xp, ldx, rows, k, codes, ldc, scales, chunks, tasks);
  else if (many)
    mx4_quantize_kernel<TYPE, 8, false><<<grid, kThreads, 0, st>>>(xp, ldx, rows, k, codes, ldc, scales, chunks, tasks);
  else
    mx4_quantize_kernel<TYPE, 1, false><<<grid, kThreads, 0, st>>>(xp, ldx, rows, k, codes, ldc, scales, chunks, tasks);
  return launch_status();
}

template <int TYPE>
cwac_status launch_dequantize(const uint8_t *codes, int64_t ldc, const uint8_t *scales, int64_t rows, int k, void *out, int64_t ldo,
                              hipStream_t st) {
  const int chunks = (int)ceil_div(k, kChunk);
  const bool many = rows * chunks >= 8 * 4096;
  const int64_t tasks = (many ? ceil_div(rows, 8) : rows) * chunks, blocks = ceil_div(tasks, kThreads / 64);
  const dim3 grid((unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks));
  const bool stream = many && rows * k * Eight<TYPE>::SIZE >= kStreamBytes;
  if (stream)
    mx4_dequantize_kernel<TYPE, 8, true><<<grid, kThreads, 0, st>>>(codes, ldc, scales, rows, k, static_cast<char *>(out), ldo, chunks, tasks);
  else if (many)
    mx4_dequantize_kernel<TYPE, 8, false><<<grid, kThreads, 0, st>>>(codes, ldc, scales, rows, k, static_cast<char *>(out), ldo, chunks, tasks);
  else
    mx4_dequantize_kernel<TYPE, 1, false><<<grid, kThreads, 0, st>>>(codes, ldc, scales, rows, k, static_cast<char *>(out), ldo, chunks, tasks);
  return launch_status();
}

// The checks that both directions share.
cwac_status check(const void *values, int32_t type, int64_t ldv, int64_t rows, int32_t k, const uint8_t *codes, int64_t ldc,
                  const uint8_t *scales) {
  if (type != CWAC_OUT_FP32 && type != CWAC_OUT_FP16 && type != CWAC_OUT_BF16) return CWAC_E_MODE;
  if (rows < 0 || rows > kMx4MaxRows || k < kMx4Block || k > kMx4MaxK || k % kMx4Block != 0 || ldv < k || ldc < k / 2)
    return CWAC_E_SHAPE;
  if (rows == 0) return CWAC_OK;
  if (!values || !codes || !scales) return CWAC_E_NULL;
  const int64_t size = type == CWAC_OUT_FP32 ? 4 : 2;
  if (!aligned(values, 16) || (ldv * size) % 16 != 0 || !aligned(codes, 16) || ldc % 16 != 0 || !aligned(scales, 8)) return CWAC_E_ALIGN;
  return CWAC_OK;
}

}  // namespace
}  // namespace cwac

using namespace cwac;

extern "C" size_t cwac_mx4_scale_bytes(int64_t rows, int32_t k) {
  if (rows < 1 || rows > kMx4MaxRows || k < 1 || k > kMx4MaxK) return 0;
  return (size_t)ceil_div(k, kMx4Panel) * (size_t)rows * 8;
}

extern "C" cwac_status cwac_mx4_quantize(const void *x, int32_t x_type, int64_t ldx, int64_t rows, int32_t k, uint8_t *codes,
                                         int64_t ldc, uint8_t *scales, void *stream) {
  const cwac_status c = check(x, x_type, ldx, rows, k, codes, ldc, scales);
  if (c != CWAC_OK || rows == 0) return c;
  hipStream_t st = as_stream(stream);
  if (x_type == CWAC_OUT_FP32) return launch_quantize<CWAC_OUT_FP32>(x, ldx, rows, k, codes, ldc, scales, st);
  if (x_type == CWAC_OUT_FP16) return launch_quantize<CWAC_OUT_FP16>(x, ldx, rows, k, codes, ldc, scales, st);
  return launch_quantize<CWAC_OUT_BF16>(x, ldx, rows, k, codes, ldc, scales, st);
}

extern "C" cwac_status cwac_mx4_dequantize(const uint8_t *codes, int64_t ldc, const uint8_t *scales, int64_t rows, int32_t k,
                                           void *out, int32_t out_type, int64_t ldo, void *stream) {
  const cwac_status c = check(out, out_type, ldo, rows, k, codes, ldc, scales);
  if (c != CWAC_OK || rows == 0) return c;
  hipStream_t st = as_stream(stream);
  if (out_type == CWAC_OUT_FP32) return launch_dequantize<CWAC_OUT_FP32>(codes, ldc, scales, rows, k, out, ldo, st);
  if (out_type == CWAC_OUT_FP16) return launch_dequantize<CWAC_OUT_FP16>(codes, ldc, scales, rows, k, out, ldo, st);
  return launch_dequantize<CWAC_OUT_BF16>(codes, ldc, scales, rows, k, out, ldo, st);
}
