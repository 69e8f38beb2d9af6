// Attention of one new token per request over a paged key-value cache:
//   o[b, h] = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale * q[b, h] . k_t - max),  t over the request's visible tokens.
//
// Bound: HBM - every visible key and value is read once, 2 to 32 operations per byte (heads that share a key head share
// the read); 61 requests of up to 8190 tokens, 8 key heads of 128, bf16: 188 us = 5.4 TB/s, int8 with 5 of up to 131072: 165 us, 5.1 TB/s, the
// join of the parts another 5 to 6.  So the kernel is a stream:
//   * a workgroup takes one request, one key head (up to 16 query heads) and a part of the length; its four wavefronts (one,
//     two or eight where they take a short length whole) take turns over tiles of 32 tokens, each on its own: running maximum, sum and output per
//     wavefront, joined through LDS at the end and, where the length is split, by a second small kernel through the workspace (fixed
//     order, no atomics);
//   * keys and values go global -> LDS directly (no registers held while they travel), per 16 tokens one contiguous piece of a page; the
//     buffers of keys and of values are refilled in turn, so one of the two is always in flight, and two workgroups share a
//     compute unit;
//   * S^T = K Q^T and O^T = V^T P^T on the matrix cores: tokens are the rows of S^T, so that a lane ends up with the weights of
//     eight tokens of one head, which is the operand layout of the second product once its sum runs over the tokens in
//     that order - the weights never change lanes.  The values come out of LDS transposed (the transposing reads of this device).
//     One query head uses one of 16 columns; the matrix cores are idle otherwise;
//   * an 8-bit cache is widened to binary16 in registers (exact); the keys' scales multiply the logits, the values' scales the
//     weights, relative to a power of two that follows a head's largest product of the two.  bfloat16 queries become binary16 relative to
//     the head's largest one (what falls below 2^-25 of that is lost).
// Weights meet the values as a sum of two numbers of the matrix instruction's type (off by 2^-17 of a weight in bfloat16; by 2^-20 in
// binary16, whose two are cut off rather than rounded, which is one instruction for a pair).  binary16 has no steps below 2^-24, so the weights take
// its whole range: the largest one (8 bits: weight times scale) is 2^15 (8 bits: 2^10 to 2^15), and what lies far below it is off by up to 2^-39 (2^-34) of
// it.  A power of two above every scale so far would let one token of large values and no weight spoil all others: 0.5 % at
// 2^16 times their scale, 8 % at 2^20.  One binary16 number would be off by
// 2^-11 and lets int8 caches' outputs be 1.7 times as far from the exact ones; the second one's matrix instructions wait for nothing
// (five requests of 30011 to 131072 tokens 173.8 us either way).  Maximum, sum and output are fp32.
// Tokens outside [lo, len), and those of a page whose number is not one, get weight 0, and what the cache holds there is
// replaced by 0, NaN included.
#include <type_traits>

#include "cwac_internal.h"
#include "llm_rules.h"

namespace cwac {
namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

#define CWAC_LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))
#define CWAC_GLOBAL_PTR(p) ((const __attribute__((address_space(1))) void *)(p))

struct PagedParams {
  const char *q, *k, *v;
  const float *ks, *vs;
  const int32_t *table, *lens;
  char *out;
  float *part;       // [batch * q_heads][splits][head_dim], then [batch * q_heads][splits][2]: maximum and sum
  int64_t ldq, ldo, ldt;
  float c;           // |scale| * log2(e), at least 2^-126
  int negate;        // scale < 0: the queries change sign
  int batch, q_heads, kv_heads, group, tiles, shift, cols, n_pages, window;
  int splits, split_tiles;
  int log_waves;     // of a workgroup: 1 << log_waves wavefronts
};

// The part of a request's length that is seen, in tiles, and how many splits it takes.
struct Span {
  int lo, len, first, tiles, used;
  __device__ __forceinline__ Span(const PagedParams &p, int b) {
    const int64_t cap = (int64_t)p.cols << p.shift;
    const int l = p.lens[b];
    len = l < 0 ? 0 : (l > cap ? (int)cap : l);
    lo = p.window > 0 && len > p.window ? len - p.window : 0;
    first = lo / kPagedTile;
    tiles = len > 0 ? (len - 1) / kPagedTile + 1 - first : 0;
    used = (tiles + p.split_tiles - 1) / p.split_tiles;
  }
};

template <int D, bool I8>
struct PagedCfg {
  static constexpr int RB = D * (I8 ? 1 : 2);      // bytes of a row
  static constexpr int CPR = RB / 16;              // 16-byte chunks of it
  static constexpr int LB = RB / 64;               // loads (1 KiB) of 16 rows
  static constexpr int BLOCK = 16 * RB, TILE = 2 * BLOCK;
  static constexpr int SCALES = I8 ? 256 : 0;
  static constexpr int WAVE = 2 * TILE + 2 * SCALES;  // a wavefront's keys, values and their scales
  static constexpr int LOADS = 2 * LB + (I8 ? 1 : 0);
  static constexpr int SLAB = (D + 4) * 4;            // a head's partial output, 16 bytes apart from the next bank round
  static constexpr int JOIN = kPagedHeads * SLAB + kPagedHeads * 8;  // a wavefront's
  static constexpr int LDS = WAVE > JOIN ? WAVE : JOIN;              // a wavefront's
  static constexpr int MOST = LDS * kPagedWide <= 160 * 1024 ? kPagedWide : kPagedWaves;  // wavefronts of a workgroup
  // chunk c of row r lies at position c ^ swz(r): 16 rows of one chunk, and 4 x 32-byte pieces of 16 rows, hit distinct banks
  static constexpr int PER = RB >= 256 ? 1 : 256 / RB;  // rows of a bank round
  __host__ __device__ static constexpr int swz(int r) { return (r / PER) & (CPR < 16 ? CPR - 1 : 15); }
};

__device__ __forceinline__ void to_lds16(const char *src, uint32_t offset, char *dst) {
  __builtin_amdgcn_global_load_lds(CWAC_GLOBAL_PTR(src + offset), CWAC_LDS_PTR(dst), 16, 0, 0);
}
__device__ __forceinline__ void to_lds4(const float *src, char *dst) {
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

// Eight signed bytes as binary16 numbers: 0x6400 | u is 1024 + u for a byte u = code + 128.
__device__ __forceinline__ u4 widen(uint32_t a, uint32_t b) {
  u4 r;
  const uint32_t w[2] = {a ^ 0x80808080u, b ^ 0x80808080u};
  const h2 bias = {(_Float16)1152.0f, (_Float16)1152.0f};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const h2 lo = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w[i], 0x04010400u)) - bias;
    const h2 hi = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w[i], 0x04030402u)) - bias;
    r[2 * i] = __builtin_bit_cast(uint32_t, lo);
    r[2 * i + 1] = __builtin_bit_cast(uint32_t, hi);
  }
  return r;
}
template <bool BF16>
__device__ __forceinline__ v4f mma(u4 a, u4 b, v4f c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
// Over the four lanes l16, l16 + 16, + 32, + 48 that hold one head's tokens: the register swaps hand every lane its
// own value and its partner's.
template <typename F>
__device__ __forceinline__ float over_quads(float x, F op) {
  const uint32_t a = __float_as_uint(x);
  const auto p = __builtin_amdgcn_permlane16_swap(a, a, false, false);
  const uint32_t b = __float_as_uint(op(__uint_as_float(p[0]), __uint_as_float(p[1])));
  const auto q = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  return op(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float quad_max(float x) {
  return over_quads(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float quad_sum(float x) {
  return over_quads(x, [](float a, float b) { return a + b; });
}
// Transposing reads of the values, written out because the compiler puts a wait for ALL loads in flight before the builtin; the wait
// for the reads themselves is part of the block.  `at`: LDS byte address of a lane's piece, `second`: of the other block of 16 tokens.
template <int SECOND>
__device__ __forceinline__ void read_values16(const uint32_t (&at)[4], u4 (&v)[4]) {
  u2 r[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
      "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
      "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "n"(SECOND)
      : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = u4{r[2 * i][0], r[2 * i][1], r[2 * i + 1][0], r[2 * i + 1][1]};
}
__device__ __forceinline__ void read_values8(const uint32_t (&at)[4], u4 (&v)[4]) {
  u2 r[4];
  asm volatile(
      "ds_read_b64_tr_b8 %0, %4\n\tds_read_b64_tr_b8 %1, %5\n\tds_read_b64_tr_b8 %2, %6\n\tds_read_b64_tr_b8 %3, %7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
      : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3])
      : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = u4{r[i][0], r[i][1], 0, 0};
}
__device__ __forceinline__ uint32_t lds_address(const char *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p;
}
template <bool BF16>
__device__ __forceinline__ uint16_t narrow(float f) {
  return BF16 ? __builtin_bit_cast(uint16_t, (__bf16)f) : __builtin_bit_cast(uint16_t, (_Float16)f);
}

template <bool BF16>
__device__ __forceinline__ float wide(uint16_t h) {
  return BF16 ? __uint_as_float((uint32_t)h << 16) : (float)__builtin_bit_cast(_Float16, h);
}

// BF16: the type of the queries and the output, and of a 16-bit cache.
template <int D, bool BF16, bool I8>
__global__ __launch_bounds__((64 * PagedCfg<D, I8>::MOST)) void paged_attention_kernel(const PagedParams p) {
  using C = PagedCfg<D, I8>;
  constexpr int KS = D / 32, DT = D / 16;
  constexpr bool MB = BF16 && !I8;  // the matrix instructions' type
  const int W = 1 << p.log_waves;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  // key heads vary fastest: their workgroups read neighbouring pieces of the same pages at about the same time (16 requests, 8 key
  // heads of 256, pages of 64: 137 us with the splits fastest, 107 so)
  const int split = blockIdx.y, h = blockIdx.x / p.tiles, ht = blockIdx.x % p.tiles, b = blockIdx.z;
  // The pages' numbers need the request's length only for what lies beyond it, so without a window both loads go out together.
  // Lane 2 i + a: block a (16 tokens) of the wavefront's tile 32 n + i
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  auto page_of = [&](int first_tile, int j) {
    const int64_t col = (int64_t)(2 * (first_tile + wave + W * (j + (lane >> 1))) + (lane & 1)) >> (p.shift - 4);
    return col < p.cols ? p.table[b * p.ldt + col] : -1;
  };
  int raw = p.window == 0 ? page_of(split * p.split_tiles, 0) : -1;
  const Span span(p, b);
  const int heads = p.group - ht * kPagedHeads < kPagedHeads ? p.group - ht * kPagedHeads : kPagedHeads;
  const int head0 = h * p.group + ht * kPagedHeads;
  uint16_t *out = reinterpret_cast<uint16_t *>(p.out) + b * p.ldo + (int64_t)head0 * D;
  if (split >= span.used) {
    if (split == 0)  // nothing is seen
      for (int i = tid; i < heads * (D / 4); i += 64 * W) reinterpret_cast<u2 *>(out)[i] = u2{0, 0};
    return;
  }
  // ---- this wavefront's tiles: t0 + wave, + W, ...
  const int t0 = span.first + split * p.split_tiles;
  const int nt = span.tiles - split * p.split_tiles < p.split_tiles ? span.tiles - split * p.split_tiles : p.split_tiles;
  const int mine = (nt - wave + W - 1) >> p.log_waves;  // at least 0
  char *kbuf = smem + wave * C::WAVE, *vbuf = kbuf + C::TILE, *sbuf = vbuf + C::TILE;

  // -1: not a page, or not a token
  int ids = -1;
  auto take_ids = [&](int j) {
    const int blk = 2 * (t0 + wave + W * (j + (lane >> 1))) + (lane & 1);
    ids = (int64_t)blk * 16 < span.len && raw >= 0 && raw < p.n_pages ? raw : -1;
  };
  if (p.window != 0) raw = page_of(t0, 0);
  take_ids(0);

  // ---- queries.  Lane group `quad` holds the dims of its chunk of each step (any order serves, if keys and queries share it)
  u4 fq[KS];
  float c = p.c;  // of this lane's head
  {
    const char *qrow = p.q + (b * p.ldq + (int64_t)(head0 + (l16 < heads ? l16 : 0)) * D) * 2;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int dim = I8 ? 16 * (4 * (s >> 1) + quad) + 8 * (s & 1) : 8 * (4 * s + quad);
      fq[s] = *reinterpret_cast<const u4 *>(qrow + dim * 2);
      if (p.negate) fq[s] ^= 0x80008000u;
      if (l16 >= heads) fq[s] = u4{0, 0, 0, 0};
    }
    if (I8 && BF16) {  // to binary16, relative to 2^e > max |q|
      float top = 0x1p-126f;
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          top = fmaxf(top, fmaxf(fabsf(__uint_as_float(fq[s][i] << 16)), fabsf(__uint_as_float(fq[s][i] & 0xffff0000u))));
      // (c < 2^ec stays finite: queries near the largest bfloat16 number are taken relative to less)
      const int eq = __builtin_amdgcn_frexp_expf(quad_max(top)), ec = __builtin_amdgcn_frexp_expf(c), e = eq < 128 - ec ? eq : 128 - ec;
      c = fmaxf(__builtin_amdgcn_ldexpf(c, e), 0x1p-126f);
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = __builtin_amdgcn_ldexpf(__uint_as_float(fq[s][i] << 16), -e);
          const float y = __builtin_amdgcn_ldexpf(__uint_as_float(fq[s][i] & 0xffff0000u), -e);
          fq[s][i] = (uint32_t)narrow<false>(x) | (uint32_t)narrow<false>(y) << 16;
        }
    }
  }

  // row of the cache [page, head, token] at which 16 tokens start; a missing page's loads go to page 0
  auto row_of = [&](int id, int blk) {
    return (((int64_t)(id < 0 ? 0 : id) * p.kv_heads + h) << p.shift) + ((blk * 16) & ((1 << p.shift) - 1));
  };
  uint32_t voff[C::LB];
#pragma unroll
  for (int i = 0; i < C::LB; ++i) {
    const int r = i * (1024 / C::RB) + lane / C::CPR;
    voff[i] = (uint32_t)(r * C::RB + (((lane % C::CPR) ^ C::swz(r)) << 4));
  }
  auto issue = [&](const char *cache, const float *scales, int64_t ra, int64_t rb, char *dst, char *sdst) {
    const char *src[2] = {cache + ra * C::RB, cache + rb * C::RB};
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int i = 0; i < C::LB; ++i) to_lds16(src[a], voff[i], dst + a * C::BLOCK + i * 1024);
    if (I8) to_lds4(scales + (lane & 16 ? rb : ra) + l16, sdst);
  };
  // a lane's place in the transposing reads.  16 bit: four rows (tokens 4 quad .. + 3 of a block) x 16 dims, lane = row l16 / 4,
  // quarter l16 % 4; 8 bit: eight rows (tokens 4 quad .. + 3 of both blocks) x 16 dims, lane = row l16 / 2, half l16 % 2.
  // Its chunk of dims 16 t .. is 2 t + (l16 % 4) / 2, or t: the part that depends on t is XORed with the rest
  const int v_token = I8 ? ((l16 >> 1) < 4 ? 0 : 16) + 4 * quad + ((l16 >> 1) & 3) : 4 * quad + (l16 >> 2);
  const uint32_t v_at = lds_address(vbuf) + v_token * C::RB + (l16 & 1) * 8;
  const uint32_t v_swz = (uint32_t)((I8 ? 0 : (l16 & 3) >> 1) ^ C::swz(v_token & 15)) << 4;

  v4f acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] = v4f{0, 0, 0, 0};
  float m = -INFINITY, l = 0.0f;  // maximum of the logits before the factor c, sum of the weights of this lane's tokens
  // Binary16 weights, and so acc, are multiplied by a power of two.  8-bit caches: times the value's scale first, whose largest product so far,
  // as much of it as the maximum of the logits leaves, is `peak` in one of a head's four lanes
  float per = I8 ? 0x1p126f : 0x1p15f, peak = 0.0f;

  int idA = -1, idB = -1;
  if (mine > 0) {
    idA = __builtin_amdgcn_readlane(ids, 0);
    idB = __builtin_amdgcn_readlane(ids, 1);
    const int64_t ra = row_of(idA, 2 * (t0 + wave)), rb = row_of(idB, 2 * (t0 + wave) + 1);
    issue(p.k, p.ks, ra, rb, kbuf, sbuf);
    issue(p.v, p.vs, ra, rb, vbuf, sbuf + C::SCALES);
  }
#pragma unroll 1
  for (int j = 0; j < mine; ++j) {
    const int tile = t0 + wave + W * j;
    const bool more = j + 1 < mine;
    const bool okA = idA >= 0, okB = idB >= 0;
    // ---- logits
    wait_loads<C::LOADS>();
    u4 fk[2][KS];
    v4f ksc[2];
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      const char *row = kbuf + a * C::BLOCK + l16 * C::RB;
      if (I8) {
        ksc[a] = *reinterpret_cast<const v4f *>(sbuf + (a * 16 + 4 * quad) * 4);
#pragma unroll
        for (int u = 0; u < KS / 2; ++u) fk[a][u] = *reinterpret_cast<const u4 *>(row + (((4 * u + quad) ^ C::swz(l16)) << 4));
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) fk[a][s] = *reinterpret_cast<const u4 *>(row + (((4 * s + quad) ^ C::swz(l16)) << 4));
      }
    }
    wait_lds();
    int64_t ra = 0, rb = 0;
    int nextA = -1, nextB = -1;
    if (more) {
      const int n = (j + 1) & 31;
      if (n == 0) {
        raw = page_of(t0, j + 1);
        take_ids(j + 1);
      }
      nextA = __builtin_amdgcn_readlane(ids, 2 * n);
      nextB = __builtin_amdgcn_readlane(ids, 2 * n + 1);
      ra = row_of(nextA, 2 * (tile + W));
      rb = row_of(nextB, 2 * (tile + W) + 1);
      issue(p.k, p.ks, ra, rb, kbuf, sbuf);
    }
    v4f s[2] = {v4f{0, 0, 0, 0}, v4f{0, 0, 0, 0}};
#pragma unroll
    for (int a = 0; a < 2; ++a) {
      if (I8) {
#pragma unroll
        for (int u = 0; u < KS / 2; ++u) {
          s[a] = mma<MB>(widen(fk[a][u][0], fk[a][u][1]), fq[2 * u], s[a]);
          s[a] = mma<MB>(widen(fk[a][u][2], fk[a][u][3]), fq[2 * u + 1], s[a]);
        }
      } else {
#pragma unroll
        for (int t = 0; t < KS; ++t) s[a] = mma<MB>(fk[a][t], fq[t], s[a]);
      }
    }
    settle();
    // ---- weights.  Element i of s[a] is token 32 tile + 16 a + 4 quad + i of head l16.
    if (I8) {
#pragma unroll
      for (int a = 0; a < 2; ++a) s[a] *= ksc[a];
    }
    const bool whole = okA && okB && tile * kPagedTile >= span.lo && tile * kPagedTile + kPagedTile <= span.len;
    uint32_t seen = 0xff;  // bit 4 a + i
    if (!whole) {
      seen = 0;
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = tile * kPagedTile + 16 * a + 4 * quad + i;
          const bool ok = (a ? okB : okA) && t >= span.lo && t < span.len;
          seen |= (ok ? 1u : 0u) << (4 * a + i);
          s[a][i] = ok ? s[a][i] : -INFINITY;
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, s[a][i]);
    const float m_new = fmaxf(m, quad_max(top));
    const float base = m_new == -INFINITY ? 0.0f : m_new;
    float alpha = __builtin_amdgcn_exp2f((m - base) * c);
    m = m_new;
    l *= alpha;
    const float shift = -base * c;
    float w[8];
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[4 * a + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[a][i], c, shift));
        l += w[4 * a + i];
      }

    // ---- values
    if (more)
      wait_loads<C::LOADS>();
    else
      wait_loads<0>();
    u4 fv[DT];
    v4f vsc[2];
#pragma unroll
    for (int t0 = 0; t0 < DT; t0 += 4) {
      uint32_t at[4];
      u4 four[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) at[i] = v_at + (((uint32_t)(t0 + i) * (I8 ? 16 : 32)) ^ v_swz);
      if constexpr (I8)
        read_values8(at, four);
      else
        read_values16<C::BLOCK>(at, four);
#pragma unroll
      for (int i = 0; i < 4; ++i) fv[t0 + i] = four[i];
    }
    if (I8) {
#pragma unroll
      for (int a = 0; a < 2; ++a) vsc[a] = *reinterpret_cast<const v4f *>(sbuf + C::SCALES + (a * 16 + 4 * quad) * 4);
    }
    wait_lds();
    if (more) issue(p.v, p.vs, ra, rb, vbuf, sbuf + C::SCALES);
    if (!whole) {  // what lies at tokens that are not seen may be anything
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        if (I8) {
#pragma unroll
          for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int i = 0; i < 4; ++i) fv[t][a] &= (seen >> (4 * a + i)) & 1 ? ~0u : ~(0xffu << (8 * i));
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) fv[t][i >> 1] &= (seen >> i) & 1 ? ~0u : ~(0xffffu << (16 * (i & 1)));
        }
      }
      if (I8) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!((seen >> i) & 1)) vsc[i >> 2][i & 3] = 0.0f;
      }
    }
    if (I8) {
      float big = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[i] *= vsc[i >> 2][i & 3];
        big = fmaxf(big, fabsf(w[i]));
      }
      peak = fmaxf(peak * alpha, big);
      const float at = peak * per;
      const uint64_t over = __builtin_amdgcn_ballot_w64(at > 0x1p15f);
      if (over | __builtin_amdgcn_ballot_w64(alpha != 1.0f)) {  // after the first tiles neither is frequent
        // the heads of which some lane has at least 2^10 (only a new maximum can have lowered it), or that cannot be raised
        const uint64_t lanes = __builtin_amdgcn_ballot_w64(at >= 0x1p10f || per >= 0x1p126f);
        uint32_t fit = (uint32_t)lanes | (uint32_t)(lanes >> 32);
        fit |= fit >> 16;
        if (over || (fit & 0xffff) != 0xffff) {
          peak = quad_max(peak);
          const float next = __builtin_amdgcn_ldexpf(1.0f, 15 - __builtin_amdgcn_frexp_expf(fmaxf(peak, 0x1p-112f)));
          // (at most 2^6: acc was in proportion to the peak that alpha has lowered)
          alpha = __builtin_amdgcn_ldexpf(alpha, __builtin_amdgcn_frexp_expf(next) - __builtin_amdgcn_frexp_expf(per));
          per = next;
        }
#pragma unroll
        for (int t = 0; t < DT; ++t) acc[t] *= alpha;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] *= per;
    } else if (!MB) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] *= 0x1p15f;
    }
    u4 hi, lo;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (MB) {
        const uint16_t a0 = narrow<MB>(w[2 * i]), a1 = narrow<MB>(w[2 * i + 1]);
        hi[i] = (uint32_t)a0 | (uint32_t)a1 << 16;
        lo[i] = (uint32_t)narrow<MB>(w[2 * i] - wide<MB>(a0)) | (uint32_t)narrow<MB>(w[2 * i + 1] - wide<MB>(a1)) << 16;
      } else {
        const auto a = __builtin_amdgcn_cvt_pkrtz(w[2 * i], w[2 * i + 1]);
        hi[i] = __builtin_bit_cast(uint32_t, a);
        lo[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(w[2 * i] - (float)a[0], w[2 * i + 1] - (float)a[1]));
      }
    }
    if (!I8 && __builtin_amdgcn_ballot_w64(alpha != 1.0f)) {  // after the first tiles a maximum seldom moves
#pragma unroll
      for (int t = 0; t < DT; ++t) acc[t] *= alpha;
    }
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const u4 val = I8 ? widen(fv[t][0], fv[t][1]) : fv[t];
      acc[t] = mma<MB>(val, hi, acc[t]);
      acc[t] = mma<MB>(val, lo, acc[t]);
    }
    settle();
    idA = nextA;
    idB = nextB;
  }

  // ---- the wavefronts' parts meet in LDS: [wave][head][D + 4], [wave][head][2]
  l = quad_sum(l);
  __syncthreads();
  float *slab = reinterpret_cast<float *>(smem);
  float *ml = slab + W * kPagedHeads * (D + 4);
  float *mine_at = slab + (wave * kPagedHeads + l16) * (D + 4) + 4 * quad;
#pragma unroll
  for (int t = 0; t < DT; ++t) {
    v4f o = acc[t];
    if (!MB) o *= 1.0f / per;
    *reinterpret_cast<v4f *>(mine_at + 16 * t) = o;
  }
  if (quad == 0) {
    ml[(wave * kPagedHeads + l16) * 2] = m * c;
    ml[(wave * kPagedHeads + l16) * 2 + 1] = l;
  }
  __syncthreads();
  for (int i = tid; i < heads * (D / 4); i += 64 * W) {
    const int head = i / (D / 4), d4 = i % (D / 4) * 4;
    // the wavefronts four at a time (or one or two): their reads are in flight together
    float top = -INFINITY, sum = 0.0f;
    v4f o = {0, 0, 0, 0};
    auto over_waves = [&](auto body) {
      if (W >= 4) {
        for (int s0 = 0; s0 < W; s0 += 4)
#pragma unroll
          for (int s = 0; s < 4; ++s) body(s0 + s);
      } else {
        for (int s = 0; s < W; ++s) body(s);
      }
    };
    over_waves([&](int s) { top = fmaxf(top, ml[(s * kPagedHeads + head) * 2]); });
    const float base = top == -INFINITY ? 0.0f : top;
    over_waves([&](int s) {
      const float f = __builtin_amdgcn_exp2f(ml[(s * kPagedHeads + head) * 2] - base);
      sum += f * ml[(s * kPagedHeads + head) * 2 + 1];
      o += f * *reinterpret_cast<const v4f *>(slab + (s * kPagedHeads + head) * (D + 4) + d4);
    });
    if (span.used == 1) {
      if (sum == 0.0f) sum = 1.0f;  // no token with a page: zeros
      const u2 r = {(uint32_t)narrow<BF16>(o[0] / sum) | (uint32_t)narrow<BF16>(o[1] / sum) << 16,
                    (uint32_t)narrow<BF16>(o[2] / sum) | (uint32_t)narrow<BF16>(o[3] / sum) << 16};
      *reinterpret_cast<u2 *>(out + head * D + d4) = r;
    } else {
      const int64_t at = ((int64_t)b * p.q_heads + head0 + head) * p.splits + split;
      *reinterpret_cast<v4f *>(p.part + at * D + d4) = o;
      if (d4 == 0) {
        float *pml = p.part + (int64_t)p.batch * p.q_heads * p.splits * D + at * 2;
        pml[0] = top;
        pml[1] = sum;
      }
    }
  }
}

// The parts of a split length: one workgroup per request and query head.  Bound: latency; so D / 4 threads read a part in 16-byte
// pieces, the workgroup's 256 D / 4 groups of them take turns over the parts with several loads in flight, and every
// wavefront works out the parts' factors for itself.
template <int D, bool BF16>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedParams p) {
  constexpr int G = 1024 / D;
  constexpr int PER = kPagedMaxSplits / 64;  // parts per lane
  __shared__ float factor[kPagedMaxSplits];
  __shared__ v4f part[G][D / 4];
  const int head = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const Span span(p, b);
  const int n = span.used;
  if (n <= 1) return;
  const int64_t at = ((int64_t)b * p.q_heads + head) * p.splits;
  const float2 *pml = reinterpret_cast<const float2 *>(p.part + (int64_t)p.batch * p.q_heads * p.splits * D) + at;
  float2 x[PER];
  float top = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    x[i] = lane + 64 * i < n ? pml[lane + 64 * i] : make_float2(-INFINITY, 0.0f);
    top = fmaxf(top, x[i].x);
  }
  top = wave_max(top);
  const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const float f = __builtin_amdgcn_exp2f(x[i].x - base);
    sum += f * x[i].y;
    if (tid < 64) factor[lane + 64 * i] = f;
  }
  sum = wave_sum(sum);
  if (sum == 0.0f) sum = 1.0f;  // no token with a page: zeros
  __syncthreads();
  const int d4 = tid % (D / 4), g = tid / (D / 4);
  const v4f *src = reinterpret_cast<const v4f *>(p.part + at * D) + d4;
  v4f o = {0, 0, 0, 0};
#pragma unroll 4
  for (int s = g; s < n; s += G) o += factor[s] * src[(int64_t)s * (D / 4)];
  part[g][d4] = o;
  __syncthreads();
  if (tid < D) {
    float r = 0.0f;
#pragma unroll
    for (int i = 0; i < G; ++i) r += reinterpret_cast<const float *>(part[i])[tid];
    reinterpret_cast<uint16_t *>(p.out)[b * p.ldo + (int64_t)head * D + tid] = narrow<BF16>(r / sum);
  }
}

template <int D, bool BF16, bool I8>
cwac_status launch_paged(const PagedParams &p, hipStream_t st) {
  constexpr int LDS = PagedCfg<D, I8>::LDS, MOST = PagedCfg<D, I8>::MOST * LDS;
  static_assert(MOST <= 160 * 1024, "LDS of a compute unit");
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void *>(&paged_attention_kernel<D, BF16, I8>),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, MOST);
  if (attr != hipSuccess) return CWAC_E_LAUNCH;
  paged_attention_kernel<D, BF16, I8><<<dim3(p.kv_heads * p.tiles, p.splits, p.batch), 64u << p.log_waves, LDS << p.log_waves, st>>>(p);
  const cwac_status s = launch_status();
  if (s != CWAC_OK || p.splits == 1) return s;
  paged_join_kernel<D, BF16><<<dim3(p.q_heads, p.batch), 256, 0, st>>>(p);
  return launch_status();
}
template <int D>
cwac_status launch_width(const PagedParams &p, bool bf16, bool i8, hipStream_t st) {
  if (bf16) return i8 ? launch_paged<D, true, true>(p, st) : launch_paged<D, true, false>(p, st);
  return i8 ? launch_paged<D, false, true>(p, st) : launch_paged<D, false, false>(p, st);
}

bool sizes_ok(int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t cols, int32_t page) {
  if (batch < 1 || batch > 65535 || kv_heads < 1 || kv_heads > 1024 || q_heads < 1 || q_heads > 16384 || q_heads % kv_heads != 0 ||
      (head_dim != 64 && head_dim != 128 && head_dim != 256) || cols < 1)
    return false;
  if (page < 16 || page > 1024 || (page & (page - 1)) != 0) return false;
  return (int64_t)cols * page <= 0x7fffffff - 64;
}

}  // namespace
}  // namespace cwac

using namespace cwac;

extern "C" size_t llm_paged_attention_workspace(int32_t batch, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                                                int32_t table_cols, int32_t page) {
  if (!sizes_ok(batch, q_heads, kv_heads, head_dim, table_cols, page)) return 0;
  const int s = paged_splits(batch, q_heads, kv_heads, (int64_t)table_cols * page);
  return s == 1 ? 16 : (size_t)batch * q_heads * s * (head_dim + 2) * 4;
}

extern "C" cwac_status llm_paged_attention(const void *q, int64_t ldq, int32_t type, const void *k_cache, const void *v_cache,
                                           int32_t cache_type, const float *k_scales, const float *v_scales, int32_t n_pages,
                                           int32_t page, const int32_t *table, int64_t ldt, int32_t table_cols,
                                           const int32_t *lens, int32_t batch, int32_t q_heads, int32_t kv_heads,
                                           int32_t head_dim, float scale, int32_t window, void *out, int64_t ldo,
                                           void *workspace, size_t workspace_bytes, void *stream) {
  if (type != CWAC_OUT_FP16 && type != CWAC_OUT_BF16) return CWAC_E_MODE;
  const bool int8 = cache_type == CWAC_OUT_INT8;
  if (!int8 && cache_type != type) return CWAC_E_MODE;
  if (!sizes_ok(batch, q_heads, kv_heads, head_dim, table_cols, page) || n_pages < 1 || window < 0 || ldt < table_cols ||
      ldq < (int64_t)q_heads * head_dim || ldo < (int64_t)q_heads * head_dim)
    return CWAC_E_SHAPE;
  if (!q || !k_cache || !v_cache || !table || !lens || !out || (int8 && (!k_scales || !v_scales))) return CWAC_E_NULL;
  if (!aligned(q, 16) || ldq % 8 != 0 || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(table, 4) || !aligned(lens, 4) ||
      !aligned(out, 8) || ldo % 4 != 0 || (int8 && (!aligned(k_scales, 4) || !aligned(v_scales, 4))))
    return CWAC_E_ALIGN;
  PagedParams p{};
  const int64_t tokens = paged_span((int64_t)table_cols * page, window);
  p.splits = paged_splits(batch, q_heads, kv_heads, tokens);
  // (eight wavefronts' tiles of 16-bit heads of 256 exceed the LDS)
  const bool wide = (head_dim != 256 || int8) && paged_wide(batch, q_heads, kv_heads, head_dim, tokens);
  if (wide) p.splits = 1;
  const int waves = wide ? kPagedWide : p.splits == 1 ? paged_waves(tokens) : kPagedWaves;
  while ((1 << p.log_waves) < waves) ++p.log_waves;
  const int64_t chunk = paged_chunk(tokens, p.splits);
  p.splits = (int)ceil_div(tokens, chunk);
  p.split_tiles = (int)(chunk / kPagedTile);
  if (p.splits > 1) {
    if (!workspace || workspace_bytes < (size_t)batch * q_heads * p.splits * (head_dim + 2) * 4) return CWAC_E_WORKSPACE;
    if (!aligned(workspace, 16)) return CWAC_E_ALIGN;
  }
  p.q = static_cast<const char *>(q), p.k = static_cast<const char *>(k_cache), p.v = static_cast<const char *>(v_cache);
  p.ks = k_scales, p.vs = v_scales, p.table = table, p.lens = lens, p.out = static_cast<char *>(out);
  p.part = static_cast<float *>(workspace);
  p.ldq = ldq, p.ldo = ldo, p.ldt = ldt, p.c = fabsf(scale) * 1.44269504088896340736f, p.negate = scale < 0.0f;
  if (p.c < 0x1p-126f) p.c = 0x1p-126f;  // a masked logit stays -inf when the scale is zero
  p.batch = batch, p.q_heads = q_heads, p.kv_heads = kv_heads, p.group = q_heads / kv_heads;
  p.tiles = (p.group + kPagedHeads - 1) / kPagedHeads;
  for (p.shift = 4; (1 << p.shift) < page;) ++p.shift;
  p.cols = table_cols, p.n_pages = n_pages, p.window = window;
  hipStream_t st = as_stream(stream);
  if (head_dim == 64) return launch_width<64>(p, type == CWAC_OUT_BF16, int8, st);
  if (head_dim == 128) return launch_width<128>(p, type == CWAC_OUT_BF16, int8, st);
  return launch_width<256>(p, type == CWAC_OUT_BF16, int8, st);
}
