// Linear layer on microscaled 4-bit operands (E2M1 codes, a power of two per 32 values of a row) with the CWAC epilogue:
//   y[m, n] = (sum over blocks b of 2^(ex[m, b] + ew[n, b]) * sum_i cx[m, 32 b + i] cw[n, 32 b + i]) * mult[n] + fbias[n].
// The block-scaled matrix instructions take both codes and scale bytes: a lane's operand is 16 bytes of codes = one
// block of one row, and its scale is one byte of a register that the instruction selects.  So the codes' way through the kernel is that of an
// int8 layer of half the K, and the scales ride beside them.
//
// Which block of a K step a lane holds is free as long as both operands agree (the sum has no order), so each lane group takes
// consecutive blocks over the steps of a 256-value panel: its scale bytes are then consecutive bytes of the
// panel's eight, one load for all of the panel's steps.
//
// K that is no multiple of 256: the last panel's codes beyond K are whatever lies there (the next row, the gap between rows, zeros
// behind the last row), finite numbers all of them, and their scale bytes are zero on both sides: at most 224 products of
// 36 * 2^-254, together below 2^-240, far below half an ulp of any fp32 sum that is not zero and zero when rounded to fp32 by themselves.
#include <type_traits>

#include "mx4.h"
#include "mx4_rules.h"
#include "qlinear_common.h"

namespace cwac {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));

#define CWAC_LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))
#define CWAC_GLOBAL_PTR(p) ((const __attribute__((address_space(1))) void *)(p))

struct Mx4Params {
  const uint8_t *x, *w, *xs, *ws;
  int64_t ldx, ldw, ldo, m;
  int n, k;
  const float *mult, *fbias;
  void *out;
  int tiles_m, tiles_n;
  int first;  // tile of the launch's first workgroup (split-K forms)
};

// The operand of an instruction: 32 codes, the lower half of the register block that other formats fill.
__device__ __forceinline__ v8i operand(v4i c) { return __builtin_shufflevector(c, c, 0, 1, 2, 3, -1, -1, -1, -1); }
constexpr int kE2M1 = 4;  // the instruction's code for the element type

template <int STEP>
__device__ __forceinline__ v4f mfma16(v4i w, v4i x, v4f acc, int ws, int xs) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(w), operand(x), acc, kE2M1, kE2M1, STEP, ws, STEP, xs);
}

template <int OUT>
struct OutType;
// (a row of the output starts at any element, which the vector stores of this device take)
template <>
struct OutType<CWAC_OUT_FP32> {
  typedef float T;
  typedef int Any4i __attribute__((ext_vector_type(4), aligned(4)));
  typedef float Any4 __attribute__((ext_vector_type(4), aligned(4)));
  static __device__ __forceinline__ T make(float u) { return u; }
};
template <>
struct OutType<CWAC_OUT_FP16> {
  typedef uint16_t T;
  typedef int Any4i __attribute__((ext_vector_type(4), aligned(2)));
  typedef uint16_t Any4 __attribute__((ext_vector_type(4), aligned(2)));
  static __device__ __forceinline__ T make(float u) { return __builtin_bit_cast(uint16_t, (_Float16)u); }
};
template <>
struct OutType<CWAC_OUT_BF16> {
  typedef uint16_t T;
  typedef int Any4i __attribute__((ext_vector_type(4), aligned(2)));
  typedef uint16_t Any4 __attribute__((ext_vector_type(4), aligned(2)));
  static __device__ __forceinline__ T make(float u) { return __builtin_bit_cast(uint16_t, (__bf16)u); }
};

// ------------------------------------------------------------------------------------------
// Few tokens or few tiles: 16 TN channels x 16 TM tokens per workgroup, K split over its W wavefronts, each of which streams its
// panels through a ring of D units of its own in LDS (no barrier before the sums meet).  Bound: the operands' arrival - HBM for the weights of
// a decoding step (1 x 4096 x 4096: 3.1-4.0 us, 1 x 11008 x 4096 6.7), the round trips of a short K loop.
// ------------------------------------------------------------------------------------------
template <int TN, int TM, int W, int D>
struct Mx4SplitCfg {
  static constexpr int BN = 16 * TN, BM = 16 * TM, NT = 64 * W;
  static constexpr int UK = kMx4Panel / 2;                  // bytes of codes of a row per unit: one panel
  static constexpr int W_BYTES = BN * UK, CODES = (BN + BM) * UK;
  static constexpr int SCALE_LOADS = (BN + BM + 31) / 32;   // 32 rows x 8 bytes each
  static constexpr int UNIT = CODES + SCALE_LOADS * 256;
  static constexpr int LPU = 2 * (TN + TM) + SCALE_LOADS;   // loads per unit; of codes: 8 rows x 128 bytes each
  static constexpr int RING = D * UNIT;
  static constexpr int SLAB = TN * TM * 1024;
  static constexpr int LDS_BYTES = W * RING;
  static_assert(SLAB <= RING && LDS_BYTES <= 160 * 1024 && D * LPU < 64, "LDS budget, 6-bit load counter");
};

// (Outside the kernel template: the host pass drops the stub of a template that passes dependent arguments to these.)
__device__ __forceinline__ void codes_to_lds(__amdgpu_buffer_rsrc_t desc, uint8_t *dst, int offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(desc, CWAC_LDS_PTR(dst), 16, offset, 0, 0, 0);
}
__device__ __forceinline__ void scales_to_lds(const uint8_t *src, uint8_t *dst) {
  __builtin_amdgcn_global_load_lds(CWAC_GLOBAL_PTR(src), CWAC_LDS_PTR(dst), 4, 0, 0);
}

template <int N>
__device__ __forceinline__ void wait_loads() {  // at most N loads of this wavefront outstanding
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ void wait_lds() {  // everything read from LDS is in registers
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(15 | (7 << 4) | (3 << 14));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <int TN, int TM, int W, int D, int OUT>
__global__ __launch_bounds__(64 * W) void mx4_splitk_kernel(const Mx4Params p) {
  using C = Mx4SplitCfg<TN, TM, W, D>;
  using O = OutType<OUT>;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  int tile_m, tile_n;
  tile_of_block(p.first + (int)blockIdx.x, p.tiles_m, p.tiles_n, tile_m, tile_n);
  const int64_t bm0 = (int64_t)tile_m * C::BM;
  const int bn0 = tile_n * C::BN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, quad = lane >> 4;
  const int rows_m = p.m - bm0 < C::BM ? (int)(p.m - bm0) : C::BM;
  const int rows_n = p.n - bn0 < C::BN ? p.n - bn0 : C::BN;
  // rows past the last token or channel lie behind the extent: such lanes touch no memory and bring zeros
  const __amdgpu_buffer_rsrc_t xd = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t *>(p.x + bm0 * p.ldx), 0, (int)((int64_t)(rows_m - 1) * p.ldx + p.k / 2), 0x00020000);
  const __amdgpu_buffer_rsrc_t wd = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t *>(p.w + (int64_t)bn0 * p.ldw), 0, (int)((int64_t)(rows_n - 1) * p.ldw + p.k / 2), 0x00020000);
  // ---- global -> LDS: lane = (row lr, 16-byte slot pc) inside a load of 8 rows; the slot of a chunk is XORed with
  // bits 1-3 of the row (on the global side), so that 16 lanes reading one chunk of 16 rows hit distinct banks
  const int lr = lane >> 3, pc = lane & 7;
  int wv[2 * TN], xv[2 * TM];
#pragma unroll
  for (int j = 0; j < 2 * TN; ++j) wv[j] = (j * 8 + lr) * (int)p.ldw + ((pc ^ (lr >> 1) ^ ((j & 1) << 2)) << 4);
#pragma unroll
  for (int j = 0; j < 2 * TM; ++j) xv[j] = (j * 8 + lr) * (int)p.ldx + ((pc ^ (lr >> 1) ^ ((j & 1) << 2)) << 4);
  // scale bytes: four per lane, rows of the weights first; rows past the end read the last row's (their codes are zeros)
  const uint8_t *sv[C::SCALE_LOADS];
  int64_t sstep[C::SCALE_LOADS];
#pragma unroll
  for (int j = 0; j < C::SCALE_LOADS; ++j) {
    const int row = j * 32 + (lane >> 1);
    const bool is_w = row < C::BN;
    const int r = is_w ? (row < rows_n ? row : rows_n - 1) : (row - C::BN < rows_m ? row - C::BN : rows_m - 1);
    sv[j] = (is_w ? p.ws + (int64_t)(bn0 + r) * 8 : p.xs + (bm0 + r) * 8) + (lane & 1) * 4;
    sstep[j] = is_w ? (int64_t)p.n * 8 : p.m * 8;
  }
  uint8_t *ring = smem + wave * C::RING;
  auto issue = [&](int d, int unit) {
    uint8_t *dst = ring + d * C::UNIT;
#pragma unroll
    for (int j = 0; j < 2 * TN; ++j) codes_to_lds(wd, dst + j * 1024, wv[j] + unit * C::UK);
#pragma unroll
    for (int j = 0; j < 2 * TM; ++j) codes_to_lds(xd, dst + C::W_BYTES + j * 1024, xv[j] + unit * C::UK);
#pragma unroll
    for (int j = 0; j < C::SCALE_LOADS; ++j) scales_to_lds(sv[j] + unit * sstep[j], dst + C::CODES + j * 256);
  };
  // ---- LDS -> operands.  Step s of a panel: lane group `quad` takes block 2 quad + s of its row.
  const int swz = (l16 >> 1) & 7;
  auto read = [&](int d, int s, v4i(&fw)[TN], v4i(&fx)[TM]) {
    const uint8_t *base = ring + d * C::UNIT + l16 * C::UK + (((2 * quad + s) ^ swz) << 4);
#pragma unroll
    for (int a = 0; a < TN; ++a) fw[a] = *reinterpret_cast<const v4i *>(base + a * 16 * C::UK);
#pragma unroll
    for (int b = 0; b < TM; ++b) fx[b] = *reinterpret_cast<const v4i *>(base + C::W_BYTES + b * 16 * C::UK);
  };
  auto read_scales = [&](int d, int(&sw)[TN], int(&sx)[TM]) {
    const uint8_t *base = ring + d * C::UNIT + C::CODES + l16 * 8 + 2 * quad;
#pragma unroll
    for (int a = 0; a < TN; ++a) sw[a] = *reinterpret_cast<const uint16_t *>(base + a * 128);
#pragma unroll
    for (int b = 0; b < TM; ++b) sx[b] = *reinterpret_cast<const uint16_t *>(base + (TN + b) * 128);
  };
  v4f acc[TN][TM];
#pragma unroll
  for (int a = 0; a < TN; ++a)
#pragma unroll
    for (int b = 0; b < TM; ++b) acc[a][b] = v4f{0, 0, 0, 0};
  v4i fw0[TN], fx0[TM], fw1[TN], fx1[TM];
  int sw[TN], sx[TM];
  auto mma = [&]() {
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
      for (int b = 0; b < TM; ++b) acc[a][b] = mfma16<0>(fw0[a], fx0[b], acc[a][b], sw[a], sx[b]);
#pragma unroll
    for (int a = 0; a < TN; ++a)
#pragma unroll
      for (int b = 0; b < TM; ++b) acc[a][b] = mfma16<1>(fw1[a], fx1[b], acc[a][b], sw[a], sx[b]);
  };

  // ---- K: a contiguous range of panels per wavefront, D in flight
  const int units = (p.k + kMx4Panel - 1) / kMx4Panel;
  const int mine = units / W + (wave < units % W ? 1 : 0);
  const int first = wave * (units / W) + (wave < units % W ? wave : units % W);
#pragma unroll
  for (int d = 0; d < D; ++d)
    if (d < mine) issue(d, first + d);
  int d = 0;
#pragma unroll 1
  for (int i = 0; i + D < mine; ++i) {
    wait_loads<(D - 1) * C::LPU>();
    read(d, 0, fw0, fx0);
    read(d, 1, fw1, fx1);
    read_scales(d, sw, sx);
    wait_lds();  // the unit is in registers, its place is free
    issue(d, first + i + D);
    mma();
    settle();  // (the next turn may copy the sums)
    d = d + 1 == D ? 0 : d + 1;
  }
  // Memory operations return in order: with r units issued behind a unit, it is complete at r * LPU outstanding.
  auto last = [&](auto tag) {  // the last D units: nothing more to issue
    constexpr int behind = decltype(tag)::value;
    if (behind >= D || behind >= mine) return;
    wait_loads<(behind < D ? behind * C::LPU : 0)>();
    read(d, 0, fw0, fx0);
    read(d, 1, fw1, fx1);
    read_scales(d, sw, sx);
    mma();
    d = d + 1 == D ? 0 : d + 1;
  };
  static_assert(D <= 4, "one call per slot");
  last(std::integral_constant<int, 3>{});
  last(std::integral_constant<int, 2>{});
  last(std::integral_constant<int, 1>{});
  last(std::integral_constant<int, 0>{});
  asm volatile("" ::: "memory");
  settle();

  // ---- the W partial tiles meet in LDS: slot 16 q + t of a 16 x 16 tile holds channels 4 q .. 4 q + 3 of token t
#pragma unroll
  for (int a = 0; a < TN; ++a)
#pragma unroll
    for (int b = 0; b < TM; ++b) reinterpret_cast<v4f *>(ring + (a * TM + b) * 1024)[lane] = acc[a][b];
  __syncthreads();
  constexpr int GROUPS = C::BM * C::BN / 4;
#pragma unroll
  for (int g0 = 0; g0 < GROUPS; g0 += C::NT) {
    const int g = g0 + tid;
    if (GROUPS % C::NT != 0 && g >= GROUPS) break;
    const int cg = g % (C::BN / 4), row = g / (C::BN / 4);
    const int tile = (cg >> 2) * TM + (row >> 4), at = (cg & 3) * 16 + (row & 15);
    if (row >= rows_m || 4 * cg >= rows_n) continue;
    const uint8_t *part = smem + tile * 1024 + at * 16;
    v4f sum = *reinterpret_cast<const v4f *>(part);
#pragma unroll
    for (int s = 1; s < W; ++s) sum += *reinterpret_cast<const v4f *>(part + s * C::RING);
    const int nn = bn0 + 4 * cg;
    typename O::T u[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int ch = nn + r < p.n ? nn + r : p.n - 1;
      float f = sum[r];
      if (p.mult) f = f * p.mult[ch];
      if (p.fbias) f = f + p.fbias[ch];
      u[r] = O::make(f);
    }
    typename O::T *o = static_cast<typename O::T *>(p.out) + (bm0 + row) * p.ldo + nn;
    if (nn + 3 < p.n) {
      *reinterpret_cast<typename O::Any4 *>(o) = typename O::Any4{u[0], u[1], u[2], u[3]};
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (nn + r < p.n) o[r] = u[r];
    }
  }
}

template <int TN, int TM, int W, int D, int OUT>
cwac_status launch_split_one(Mx4Params p, int64_t tiles, hipStream_t st) {
  constexpr int LDS = Mx4SplitCfg<TN, TM, W, D>::LDS_BYTES;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void *>(&mx4_splitk_kernel<TN, TM, W, D, OUT>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  if (attr != hipSuccess) return CWAC_E_LAUNCH;
  static_assert(64 * W <= 256, "kMx4TilesPerLaunch");
  for (int64_t at = 0; at < tiles; at += kMx4TilesPerLaunch) {
    p.first = (int)at;
    const int64_t blocks = tiles - at < kMx4TilesPerLaunch ? tiles - at : kMx4TilesPerLaunch;
    mx4_splitk_kernel<TN, TM, W, D, OUT><<<(unsigned)blocks, 64 * W, LDS, st>>>(p);
    const cwac_status s = launch_status();
    if (s != CWAC_OK) return s;
  }
  return CWAC_OK;
}

template <int TN, int TM, int W, int D>
cwac_status launch_split(Mx4Params p, int out_kind, hipStream_t st) {
  p.tiles_m = (int)ceil_div(p.m, 16 * TM);
  p.tiles_n = (int)ceil_div(p.n, 16 * TN);
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  if (tiles > 0x3fffffff) return CWAC_E_SHAPE;  // (an output of 2^38 elements or more; a tile's number and that of a tile row's eight stay in 32 bits)
  if (out_kind == CWAC_OUT_FP32) return launch_split_one<TN, TM, W, D, CWAC_OUT_FP32>(p, tiles, st);
  if (out_kind == CWAC_OUT_FP16) return launch_split_one<TN, TM, W, D, CWAC_OUT_FP16>(p, tiles, st);
  return launch_split_one<TN, TM, W, D, CWAC_OUT_BF16>(p, tiles, st);
}

// ------------------------------------------------------------------------------------------
// Many tiles: BM tokens x BN channels at a time, both panels through a ring of NSTAGE stages in LDS, one stage = one panel of 256
// values (128 bytes of codes and 8 scale bytes per row).  Bound: the matrix cores, under the device's power limit: 16384 x 4096 x 11008 bf16
// 305 to 356 us in the profiler, median 350 = 4.2 PFLOP/s (4.8 over K alone), where the instruction by itself sustains 5.2 on random codes; they are busy for 62 % of
// the cycles at 1.63 GHz.  128 x 128 tiles read as many LDS cycles as they multiply and take 0.4 us a stage.
//   * Codes go global -> LDS directly, 8 rows x 128 bytes per load; the 16-byte chunk c of row r lands at position c ^ ((r >> 1) & 7)
//     (applied on the global side), so operand reads are free of bank conflicts.  Buffer loads whose descriptor moves along K with
//     the stages and ends with the matrix: a lane's offset never changes, and what lies beyond reads as zeros, so the last
//     panel needs no case of its own.
//   * A stage is four steps of v_mfma_scale_f32_32x32x64: the half-wave h takes block 4 h + step of its row, so its four scale bytes
//     are one word, read once per stage, and the instruction picks the step's byte.
//   * Operands are double-buffered in registers: the LDS reads of a step run under the matrix instructions of the one before,
//     those of the next stage's first step under this stage's last, behind the only barrier of the stage.
//   * Workgroups are persistent: the first stage of the next tile and its parameters travel under the epilogue, whose slabs lie over the
//     other stages.
// Tiles that reach beyond the matrix are moved inwards: their rows or channels are computed twice, with the same values.
// ------------------------------------------------------------------------------------------
template <int BM_, int BN_, int WM_, int TA_, int NSTAGE_>
struct Mx4TileCfg {
  static constexpr int BM = BM_, BN = BN_, NSTAGE = NSTAGE_, TA = TA_;  // TA: 32-channel tiles per wavefront
  static constexpr int WM = WM_, WN = BN / (32 * TA), NW = WM * WN, NT = 64 * NW;
  static constexpr int TB = BM / (32 * WM);                             // 32-token tiles per wavefront
  static constexpr int BK = kMx4Panel / 2;
  // LDS: codes of the tokens [NSTAGE], of the channels [NSTAGE], their scale bytes [NSTAGE] each, two parameter blocks
  static constexpr int X_BYTES = BM * BK, W_BYTES = BN * BK, W_AT = NSTAGE * X_BYTES, XS_AT = W_AT + NSTAGE * W_BYTES;
  static constexpr int WS_AT = XS_AT + NSTAGE * BM * 8, PARAM = WS_AT + NSTAGE * BN * 8, LDS = PARAM + 2 * 8 * BN;
  static constexpr int XR = BM / NW, WR = BN / NW;                      // rows whose loads a wavefront issues
  static constexpr int LX = XR / 8, LW = WR / 8, SX = XR / 32, SW = WR / 32, LPS = LX + LW + SX + SW;
  // slabs of the epilogue, 8 KiB each, over stage 1 of the tokens (the first half of the wavefronts) and of the channels
  static constexpr int SLAB = 8192;
  static_assert(XR % 32 == 0 && WR % 32 == 0 && LDS <= 160 * 1024 && NSTAGE * BM * BK <= 65536 && NSTAGE * BN * BK <= 65536, "layout");
  static_assert(NW / 2 * SLAB <= X_BYTES && NW / 2 * SLAB <= W_BYTES && NW == BN / 32 && BN * 4 == NW / 2 * 256, "slabs, parameter loads");
};

__device__ __forceinline__ void words_to_lds(__amdgpu_buffer_rsrc_t desc, uint8_t *dst, int offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(desc, CWAC_LDS_PTR(dst), 4, offset, 0, 0, 0);
}
template <int STEP>
__device__ __forceinline__ v16f mfma32(v4i w, v4i x, v16f acc, int ws, int xs) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(w), operand(x), acc, kE2M1, kE2M1, STEP, ws, STEP, xs);
}

// STREAM: the output's stores go past the caches
template <typename C, int OUT, bool STREAM>
__global__ __launch_bounds__(C::NT) void mx4_tile_kernel(const Mx4Params p) {
  using O = OutType<OUT>;
  constexpr int TA = C::TA, TB = C::TB, BK = C::BK, NSTAGE = C::NSTAGE;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wave_m = wave % C::WM, wave_n = wave / C::WM;
  const int total = p.tiles_m * p.tiles_n, stages = (p.k + kMx4Panel - 1) / kMx4Panel;
  if (p.mult == nullptr || p.fbias == nullptr) {  // absent parameters: both blocks filled once
    for (int i = tid; i < 2 * C::BN; i += C::NT) {
      float *block = reinterpret_cast<float *>(smem + C::PARAM) + (i / C::BN) * 2 * C::BN;
      if (!p.mult) block[i % C::BN] = 1.0f;
      if (!p.fbias) block[C::BN + i % C::BN] = 0.0f;
    }
  }
  // ---- global -> LDS.  A lane's place in a load: row lr of 8, chunk pc ^ swizzle; loads with odd number sit 8 rows further, which
  // flips bit 2 of the swizzle (a wavefront's rows start at a multiple of 32)
  const int lr = lane >> 3, pc = lane & 7;
  int xv[C::LX], wv[C::LW];
#pragma unroll
  for (int i = 0; i < C::LX; ++i)
    xv[i] = (int)((uint32_t)(wave * C::XR + 8 * i + lr) * (uint32_t)p.ldx + (uint32_t)((pc ^ (lr >> 1) ^ ((i & 1) << 2)) << 4));
#pragma unroll
  for (int i = 0; i < C::LW; ++i)
    wv[i] = (int)((uint32_t)(wave * C::WR + 8 * i + lr) * (uint32_t)p.ldw + (uint32_t)((pc ^ (lr >> 1) ^ ((i & 1) << 2)) << 4));
  const int xsv = wave * C::XR * 8 + lane * 4, wsv = wave * C::WR * 8 + lane * 4;
  int64_t bm0 = 0;
  int bn0 = 0;
  // where the next stage to be loaded begins, what is left of the matrix from there, and how many stages are; past the last
  // one the extents are zero: such loads touch no memory and bring zeros that nobody reads
  const uint8_t *xg = nullptr, *wg = nullptr, *xsg = nullptr, *wsg = nullptr;
  uint32_t xleft = 0, wleft = 0;
  int xtodo = 0, wtodo = 0;
  // load i of the stage into ring place buf, and the step to the next stage behind the last one
  auto load_x = [&](int i, int buf) {
    if (i < C::LX) {
      const __amdgpu_buffer_rsrc_t d = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(xg), 0, xtodo > 0 ? (int)xleft : 0, 0x00020000);
      codes_to_lds(d, smem + buf * C::X_BYTES + wave * C::XR * BK + i * 8 * BK, xv[i < C::LX ? i : 0]);
    } else {
      const __amdgpu_buffer_rsrc_t d = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(xsg), 0, xtodo > 0 ? C::BM * 8 : 0, 0x00020000);
      words_to_lds(d, smem + C::XS_AT + (buf * C::BM + wave * C::XR + 32 * (i - C::LX)) * 8, xsv + (i - C::LX) * 256);
    }
    if (i == C::LX + C::SX - 1) xg += BK, xleft -= BK, xsg += p.m * 8, --xtodo;
  };
  auto load_w = [&](int i, int buf) {
    if (i < C::LW) {
      const __amdgpu_buffer_rsrc_t d = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(wg), 0, wtodo > 0 ? (int)wleft : 0, 0x00020000);
      codes_to_lds(d, smem + C::W_AT + buf * C::W_BYTES + wave * C::WR * BK + i * 8 * BK, wv[i < C::LW ? i : 0]);
    } else {
      const __amdgpu_buffer_rsrc_t d = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(wsg), 0, wtodo > 0 ? C::BN * 8 : 0, 0x00020000);
      words_to_lds(d, smem + C::WS_AT + (buf * C::BN + wave * C::WR + 32 * (i - C::LW)) * 8, wsv + (i - C::LW) * 256);
    }
    if (i == C::LW + C::SW - 1) wg += BK, wleft -= BK, wsg += (int64_t)p.n * 8, --wtodo;
  };
  auto issue_x = [&](int buf) {
#pragma unroll
    for (int i = 0; i < C::LX + C::SX; ++i) load_x(i, buf);
  };
  auto issue_w = [&](int buf) {
#pragma unroll
    for (int i = 0; i < C::LW + C::SW; ++i) load_w(i, buf);
  };
  // a tile's origin, its parameters (the first half of the wavefronts the multipliers, the others the constants), its stage 0
  auto open = [&](int id, int block) {
    int tile_m, tile_n;
    tile_of_block(id, p.tiles_m, p.tiles_n, tile_m, tile_n);
    bm0 = (int64_t)tile_m * C::BM;
    if (bm0 > p.m - C::BM) bm0 = p.m - C::BM;
    bn0 = tile_n * C::BN;
    if (bn0 > p.n - C::BN) bn0 = p.n - C::BN;
    xg = p.x + bm0 * p.ldx, wg = p.w + (int64_t)bn0 * p.ldw, xsg = p.xs + bm0 * 8, wsg = p.ws + (int64_t)bn0 * 8;
    xleft = (uint32_t)((uint64_t)(C::BM - 1) * (uint64_t)p.ldx + (uint64_t)(p.k / 2));
    wleft = (uint32_t)((uint64_t)(C::BN - 1) * (uint64_t)p.ldw + (uint64_t)(p.k / 2));
    xtodo = wtodo = stages;
    const float *src = wave < C::NW / 2 ? p.mult : p.fbias;
    if (src)
      scales_to_lds(reinterpret_cast<const uint8_t *>(src + bn0 + (wave % (C::NW / 2)) * 64 + lane),
                    smem + C::PARAM + block * 8 * C::BN + wave * 256);
    issue_x(0);
    issue_w(0);
  };
  // ---- LDS -> operands
  const int swz = (l32 >> 1) & 7;
  const int x_row = (wave_m * 32 * TB + l32) * BK, w_row = C::W_AT + (wave_n * 32 * TA + l32) * BK;
  const int xs_row = C::XS_AT + (wave_m * 32 * TB + l32) * 8 + 4 * half, ws_row = C::WS_AT + (wave_n * 32 * TA + l32) * 8 + 4 * half;
  // operand i of a step (the channels' first), scale word i of a stage
  auto read_one = [&](int i, int buf, int step, v4i(&fw)[TA], v4i(&fx)[TB]) {
    const int chunk = ((4 * half + step) ^ swz) << 4;
    if (i < TA)
      fw[i < TA ? i : 0] = *reinterpret_cast<const v4i *>(smem + w_row + chunk + buf * C::W_BYTES + i * 32 * BK);
    else
      fx[i < TA ? 0 : i - TA] = *reinterpret_cast<const v4i *>(smem + x_row + chunk + buf * C::X_BYTES + (i - TA) * 32 * BK);
  };
  auto read_scale = [&](int i, int buf, int(&sw)[TA], int(&sx)[TB]) {
    if (i < TA)
      sw[i < TA ? i : 0] = *reinterpret_cast<const int *>(smem + ws_row + buf * C::BN * 8 + i * 256);
    else
      sx[i < TA ? 0 : i - TA] = *reinterpret_cast<const int *>(smem + xs_row + buf * C::BM * 8 + (i - TA) * 256);
  };
  v16f acc[TA][TB];
  v4i fwA[TA], fxA[TB], fwB[TA], fxB[TB];
  int sw[TA], sx[TB];
  // One step: its matrix instructions in order, behind each of them a share of `reads` (a callable for LDS read i) and of `loads` (for
  // load i) of n_reads and n_loads.  A load holds up its wavefront while the address unit is busy, so they go out one at a time.
  auto step = [&](auto tag, const v4i(&fw)[TA], const v4i(&fx)[TB], auto n_reads, auto reads, auto n_loads, auto loads) {
    constexpr int MM = TA * TB, NR = decltype(n_reads)::value, NL = decltype(n_loads)::value;
#pragma unroll
    for (int i = 0; i < MM; ++i) {
      const int a = i / TB, b = i % TB;
      acc[a][b] = mfma32<decltype(tag)::value>(fw[a], fx[b], acc[a][b], sw[a], sx[b]);
      // the reads behind the first three quarters, the loads spread over all
#pragma unroll
      for (int r = 0; r < NR; ++r)
        if (r * (MM * 3 / 4) / NR == i) reads(r);
#pragma unroll
      for (int l = 0; l < NL; ++l)
        if (l * MM / NL == i) loads(l);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  using S2 = std::integral_constant<int, 2>;
  using S3 = std::integral_constant<int, 3>;
  using Operands = std::integral_constant<int, TA + TB>;
  // Stage s in ring place buf.  The loads of stage s + NSTAGE go into the place that this stage leaves, behind its barrier: the
  // tokens' under the last step, the channels' under the first step of the next stage.
  auto stage_body = [&](int prev, int buf, int next) {
    auto none = [](int) {};
    step(S0{}, fwA, fxA, Operands{}, [&](int i) { read_one(i, buf, 1, fwB, fxB); }, std::integral_constant<int, C::LW + C::SW>{},
         [&](int i) { load_w(i, prev); });
    step(S1{}, fwB, fxB, Operands{}, [&](int i) { read_one(i, buf, 2, fwA, fxA); }, S0{}, none);
    step(S2{}, fwA, fxA, Operands{}, [&](int i) { read_one(i, buf, 3, fwB, fxB); }, S0{}, none);
    wait_loads<(NSTAGE - 2) * C::LPS>();  // stage s + 1 has landed
    wait_lds();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    int nw[TA], nx[TB];
    step(S3{}, fwB, fxB, std::integral_constant<int, 2 * (TA + TB)>{},
         [&](int i) {
           if (i < TA + TB)
             read_one(i, next, 0, fwA, fxA);
           else
             read_scale(i - TA - TB, next, nw, nx);
         },
         std::integral_constant<int, C::LX + C::SX>{}, [&](int i) { load_x(i, buf); });
#pragma unroll
    for (int a = 0; a < TA; ++a) sw[a] = nw[a];
#pragma unroll
    for (int b = 0; b < TB; ++b) sx[b] = nx[b];
  };

  constexpr int ES = sizeof(typename O::T), AP = ES == 4 ? (TA < 2 ? TA : 2) : TA, ROW = AP * 32 * ES;
  constexpr int LPR = ROW / 16, RPS = 64 / LPR, STORES = TB * (TA / AP) * (32 / RPS);  // lanes per row, rows per store, stores per tile
  constexpr int AHEAD = (NSTAGE - 1) * (C::LX + C::SX) + (NSTAGE - 2) * (C::LW + C::SW);  // loads behind stage 0 when a tile begins
  static_assert(32 * ROW <= C::SLAB && STORES + AHEAD < 64, "slab, 6-bit counter");
  uint8_t *slab = smem + (wave < C::NW / 2 ? C::X_BYTES : C::W_AT + C::W_BYTES) + (wave % (C::NW / 2)) * C::SLAB;
  int id = blockIdx.x, block = 0;
  bool stored = false;  // this wavefront's newest operations before the stages to come are STORES stores
  if (id >= total) return;
  open(id, 0);
  __syncthreads();  // (the filled parameters)
  for (;;) {
    // ---- the tile's first stages.  Operations are counted in order: stage 0 has landed when at most the later ones - and the
    // stores of the tile before, which lie between - are outstanding
#pragma unroll
    for (int s = 1; s < NSTAGE; ++s) {
      issue_x(s);
      if (s + 1 < NSTAGE) issue_w(s);
    }
    if (stored)
      wait_loads<AHEAD + STORES>();
    else
      wait_loads<AHEAD>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int a = 0; a < TA; ++a)
#pragma unroll
      for (int b = 0; b < TB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;
#pragma unroll
    for (int i = 0; i < TA + TB; ++i) {
      read_one(i, 0, 0, fwA, fxA);
      read_scale(i, 0, sw, sx);
    }
    int prev = NSTAGE - 1, buf = 0, next = 1;
#pragma unroll 1
    for (int left = stages; left > 0; --left) {
      stage_body(prev, buf, next);
      const int after = NSTAGE == 2 ? buf : prev;
      prev = buf, buf = next, next = after;
    }
    static_assert(NSTAGE == 2 || NSTAGE == 3, "the rotation above");
    wait_loads<0>();  // the loads past the last stage: their zeros lie where the next tile or the slabs go
    wait_lds();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    settle();
    settle();

    // ---- the ring is free: the next tile's first loads go out, then this one's epilogue.  Element 4 g + r of acc[a][b]: channel
    // 32 a + 8 g + 4 half + r, token 32 b + l32 of the wavefront's tile.
    // A slab is 32 tokens x ROW bytes, the 16-byte chunk c of row r at position c ^ r.
    const int64_t em0 = bm0;
    const int en0 = bn0;
    const float *s_mult = reinterpret_cast<const float *>(smem + C::PARAM + block * 8 * C::BN), *s_fb = s_mult + C::BN;
    id += gridDim.x;
    const bool more = id < total;
    block ^= 1;
    if (more) open(id, block);
#pragma unroll
    for (int b = 0; b < TB; ++b)
#pragma unroll
      for (int a0 = 0; a0 < TA; a0 += AP) {
#pragma unroll
        for (int a = a0; a < a0 + AP; ++a)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int ch = wave_n * 32 * TA + a * 32 + 8 * g + 4 * half;
            const v4f mu = *reinterpret_cast<const v4f *>(s_mult + ch), fb = *reinterpret_cast<const v4f *>(s_fb + ch);
            typename O::T u[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float f = acc[a][b][4 * g + r] * mu[r];
              if (p.fbias) f = f + fb[r];
              u[r] = O::make(f);
            }
            const int byte = ((a - a0) * 32 + 8 * g + 4 * half) * ES;
            uint8_t *at = slab + l32 * ROW + (((byte >> 4) ^ (l32 & (LPR - 1))) << 4) + (byte & 15);
            if constexpr (ES == 4)
              *reinterpret_cast<v4f *>(at) = v4f{u[0], u[1], u[2], u[3]};
            else
              *reinterpret_cast<uint2 *>(at) = make_uint2((uint32_t)u[0] | (uint32_t)u[1] << 16, (uint32_t)u[2] | (uint32_t)u[3] << 16);
          }
        // (a wavefront's own slab: its LDS operations are in order)
        typename O::T *o = static_cast<typename O::T *>(p.out) + (em0 + wave_m * 32 * TB + 32 * b) * p.ldo + en0 + wave_n * 32 * TA + 32 * a0;
#pragma unroll
        for (int i = 0; i < 32 / RPS; ++i) {
          const int row = i * RPS + lane / LPR;
          const v4i v = *reinterpret_cast<const v4i *>(slab + row * ROW + (((lane % LPR) ^ (row & (LPR - 1))) << 4));
          auto *dst = reinterpret_cast<typename O::Any4i *>(o + row * p.ldo + (lane % LPR) * (16 / ES));
          if constexpr (STREAM)
            __builtin_nontemporal_store(v, dst);
          else
            *dst = v;
        }
      }
    if (!more) break;
    stored = true;
    wait_lds();
    __builtin_amdgcn_s_barrier();  // every slab is read: the stages under them are free
    __builtin_amdgcn_sched_barrier(0);
  }
}

template <typename C, int OUT, bool STREAM>
cwac_status launch_tile_one(const Mx4Params &p, unsigned blocks, hipStream_t st) {
  static const hipError_t attr =
      hipFuncSetAttribute(reinterpret_cast<const void *>(&mx4_tile_kernel<C, OUT, STREAM>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
  if (attr != hipSuccess) return CWAC_E_LAUNCH;
  mx4_tile_kernel<C, OUT, STREAM><<<blocks, C::NT, C::LDS, st>>>(p);
  return launch_status();
}
// The large tiles' outputs are larger than the L2s and go past the caches (16384 x 11008 x 4096 394 -> 348 us), unless rows begin inside
// a line: the line that two stores share would cross to memory twice (7567 x 9129 x 896 bf16 87 / 102, fp32 128 / 163).
template <typename C, int OUT>
cwac_status launch_tile_out(const Mx4Params &p, unsigned blocks, hipStream_t st) {
  if constexpr (C::BM == 256) {
    if (aligned(p.out, 64) && p.ldo * (int64_t)sizeof(typename OutType<OUT>::T) % 64 == 0) return launch_tile_one<C, OUT, true>(p, blocks, st);
  }
  return launch_tile_one<C, OUT, false>(p, blocks, st);
}

template <typename C>
cwac_status launch_tile(Mx4Params p, int out_kind, hipStream_t st) {
  p.tiles_m = (int)ceil_div(p.m, C::BM);
  p.tiles_n = (int)ceil_div(p.n, C::BN);
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
  if (tiles > 0x3fffffff) return CWAC_E_SHAPE;
  // as many persistent workgroups as fit the chip (256 compute units); a multiple of 8 keeps a workgroup's tiles on one XCD
  const int64_t fit = 256 * (160 * 1024 / C::LDS);
  const unsigned blocks = (unsigned)(tiles < fit ? tiles : fit);
  if (out_kind == CWAC_OUT_FP32) return launch_tile_out<C, CWAC_OUT_FP32>(p, blocks, st);
  if (out_kind == CWAC_OUT_FP16) return launch_tile_out<C, CWAC_OUT_FP16>(p, blocks, st);
  return launch_tile_out<C, CWAC_OUT_BF16>(p, blocks, st);
}

using Tile256 = Mx4TileCfg<256, 256, 4, 4, 2>;      // eight wavefronts of 64 x 128, one workgroup per compute unit
using Tile128Pair = Mx4TileCfg<128, 128, 2, 2, 2>;  // four of 64 x 64, two workgroups
using Tile128Deep = Mx4TileCfg<128, 128, 2, 2, 3>;  // one workgroup, three stages: a single round with a long K

}  // namespace
}  // namespace cwac

using namespace cwac;

extern "C" cwac_status qlinear_mx4_cwac_forward_ex(const uint8_t *x_codes, int64_t ldx, const uint8_t *x_scales,
                                                   const uint8_t *w_codes, int64_t ldw, const uint8_t *w_scales, int64_t m,
                                                   int32_t n, int32_t k, const float *mult, const float *fbias, int32_t out_kind,
                                                   void *out, int64_t ldo, const cwac_tuning *tuning, void *stream) {
  if (!x_codes || !x_scales || !w_codes || !w_scales || !out) return CWAC_E_NULL;
  if (m < 1 || m > 0x7fffffff || n < 1 || k < kMx4Block || k > kMx4MaxK || k % kMx4Block != 0 || ldx < k / 2 || ldw < k / 2 ||
      ldx > kMx4MaxPitch || ldw > kMx4MaxPitch || ldo < n)
    return CWAC_E_SHAPE;
  Tune tune;
  if ((out_kind != CWAC_OUT_FP32 && out_kind != CWAC_OUT_FP16 && out_kind != CWAC_OUT_BF16) || !tune_from(tuning, tune)) return CWAC_E_MODE;
  const int64_t size = out_kind == CWAC_OUT_FP32 ? 4 : 2;
  if (!aligned(x_codes, 16) || !aligned(w_codes, 16) || ldx % 16 != 0 || ldw % 16 != 0 || !aligned(x_scales, 8) ||
      !aligned(w_scales, 8) || !aligned(out, (size_t)size))
    return CWAC_E_ALIGN;
  Mx4Params p{};
  p.x = x_codes, p.w = w_codes, p.xs = x_scales, p.ws = w_scales;
  p.ldx = ldx, p.ldw = ldw, p.ldo = ldo, p.m = m, p.n = n, p.k = k;
  p.mult = mult, p.fbias = fbias, p.out = out;
  hipStream_t st = as_stream(stream);
  int form = mx4_form(m, n, k);
  if (tune.kernel == CWAC_KERNEL_SPLIT_K) form = mx4_split_form(m, n, k);
  if (tune.kernel == CWAC_KERNEL_DIRECT_LDS) {
    if (tune.shape == CWAC_SHAPE_256_8W && m >= 256 && n >= 256) form = kMx4Tile256;
    if (tune.shape == CWAC_SHAPE_128_PAIR && m >= 128 && n >= 128) form = kMx4Tile128Pair;
    if (tune.shape == CWAC_SHAPE_128_128 && m >= 128 && n >= 128) form = kMx4Tile128Deep;
  }
  switch (form) {
    case kMx4Tile256: return launch_tile<Tile256>(p, out_kind, st);
    case kMx4Tile128Pair: return launch_tile<Tile128Pair>(p, out_kind, st);
    case kMx4Tile128Deep: return launch_tile<Tile128Deep>(p, out_kind, st);
    case kMx4Split64: return launch_split<4, 4, 4, 2>(p, out_kind, st);
    case kMx4Split32: return launch_split<2, 2, 4, 2>(p, out_kind, st);
    case kMx4Split32x16: return launch_split<2, 1, 4, 3>(p, out_kind, st);
    default: return launch_split<1, 1, 4, 4>(p, out_kind, st);
  }
}

extern "C" cwac_status qlinear_mx4_cwac_forward(const uint8_t *x_codes, int64_t ldx, const uint8_t *x_scales,
                                                const uint8_t *w_codes, int64_t ldw, const uint8_t *w_scales, int64_t m,
                                                int32_t n, int32_t k, const float *mult, const float *fbias, int32_t out_kind,
                                                void *out, int64_t ldo, void *stream) {
  return qlinear_mx4_cwac_forward_ex(x_codes, ldx, x_scales, w_codes, ldw, w_scales, m, n, k, mult, fbias, out_kind, out, ldo, nullptr, stream);
}
