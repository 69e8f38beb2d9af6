// The paged key-value cache of a language model: pages for a step's new tokens, and the tokens' keys and values into them.
#include "cwac_internal.h"
#include "llm_rules.h"

namespace cwac {
namespace {

// ------------------------------------------------------------------------------------------
// Block tables and slots from the requests' lengths.  Bound: latency - two running sums over the requests and one launch.
// Every workgroup computes the sums for all requests (a few KB from the L2) and keeps them in LDS, so that no workgroup
// waits for another; then each fills its share of the table rows and of the slots, a slot to a thread: the chain of one - a search
// through the sums in LDS, one load, one store - is what a launch lasts (500 requests, 64 thousand new tokens: 10.9 us with four
// slots to a thread).  A slot's page is taken from the free
// stack directly when it is new, never read back from the table, so nothing depends on another workgroup's stores.
// Sums saturate at 2^31 - 1 instead of wrapping: no length in device memory can lead a store out of bounds.
// ------------------------------------------------------------------------------------------
constexpr int kThreads = 1024;
constexpr int kMaxBatch = CWAC_KV_MAX_BATCH;
constexpr uint32_t kTop = 0x7fffffffu, kNot = 0xffffffffu;

__device__ __forceinline__ uint32_t sat(uint32_t a, uint32_t b) {  // both at most kTop
  const uint32_t s = a + b;
  return s > kTop ? kTop : s;
}

struct AssignParams {
  const int32_t *old_lens, *new_lens, *free_pages, *n_free;
  int32_t *table, *token_start, *seq_lens, *n_left;
  int64_t *slots;
  int64_t ldt, capacity;
  int batch, shift, free_capacity, cols;
};

struct Request {
  uint32_t old_len, new_len, have, need;
  bool fits;  // the table has columns for it
  __device__ __forceinline__ Request(const AssignParams &p, int b) {
    const int o = p.old_lens[b], n = p.new_lens[b];
    old_len = o < 0 ? 0 : o;
    new_len = n < 0 ? 0 : n;
    const uint32_t mask = (1u << p.shift) - 1;
    have = (old_len + mask) >> p.shift;                       // at most 2^31 + 2^10: no wrap
    const uint64_t end = ((uint64_t)old_len + new_len + mask) >> p.shift;
    fits = end <= (uint64_t)p.cols;
    need = fits ? (uint32_t)end - have : 0;
  }
};

__global__ __launch_bounds__(kThreads) void kv_assign_kernel(const AssignParams p) {
  extern __shared__ uint32_t lds[];
  uint32_t *tok_end = lds;             // [batch] new tokens up to and with request b
  uint32_t *page_at = lds + p.batch;   // [batch] pages of the requests before b; kNot: b is not served
  uint32_t *old_at = page_at + p.batch;  // [batch] tokens in the cache
  __shared__ uint32_t wave_tok[kThreads / 64], wave_page[kThreads / 64], taken_all;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int n_free = *p.n_free;
  n_free = n_free < 0 ? 0 : (n_free > p.free_capacity ? p.free_capacity : n_free);
  if (tid == 0) taken_all = 0;

  // ---- running sums: a thread's consecutive requests, the wavefront, the workgroup
  const int each = (p.batch + kThreads - 1) / kThreads, first = tid * each;
  uint32_t tok = 0, page = 0;
  for (int i = 0; i < each && first + i < p.batch; ++i) {
    const Request r(p, first + i);
    tok = sat(tok, r.new_len);
    page = sat(page, r.need);
  }
  uint32_t tok_sum = tok, page_sum = page;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t a = __shfl_up(tok_sum, o, 64), b = __shfl_up(page_sum, o, 64);
    if (lane >= o) tok_sum = sat(tok_sum, a), page_sum = sat(page_sum, b);
  }
  if (lane == 63) wave_tok[wave] = tok_sum, wave_page[wave] = page_sum;
  // the sums of the lanes before this one (a saturated sum cannot be taken back by subtraction)
  uint32_t tok_before = __shfl_up(tok_sum, 1, 64), page_before = __shfl_up(page_sum, 1, 64);
  if (lane == 0) tok_before = 0, page_before = 0;
  __syncthreads();
  uint32_t t0 = 0, g0 = 0;
  for (int w = 0; w < wave; ++w) t0 = sat(t0, wave_tok[w]), g0 = sat(g0, wave_page[w]);
  t0 = sat(t0, tok_before);
  g0 = sat(g0, page_before);
  uint32_t taken = 0;
  for (int i = 0; i < each && first + i < p.batch; ++i) {
    const int b = first + i;
    const Request r(p, b);
    const uint32_t g1 = sat(g0, r.need);
    // rows without a slot cannot be appended: such a request takes no pages (nor do those behind it, whose rows lie further back)
    const bool rows = r.new_len == 0 || p.capacity == 0 || (uint64_t)t0 + r.new_len <= (uint64_t)(p.capacity < kTop ? p.capacity : kTop);
    const bool served = r.fits && rows && (r.need == 0 || (uint64_t)g0 + r.need <= (uint32_t)n_free);
    page_at[b] = served ? g0 : kNot;
    old_at[b] = r.old_len;
    if (served && r.need) taken = g1;
    if (blockIdx.x == 0) {
      p.token_start[b] = (int32_t)t0;
      p.seq_lens[b] = (int32_t)(served ? r.old_len + r.new_len : r.old_len);
    }
    t0 = sat(t0, r.new_len);
    tok_end[b] = t0;
    g0 = g1;
    if (blockIdx.x == 0 && b == p.batch - 1) p.token_start[p.batch] = (int32_t)t0;
  }
  if (taken) atomicMax(&taken_all, taken);  // the running sum is monotone: the largest is the last one served
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) *p.n_left = n_free - (int32_t)taken_all;

  // ---- table entries of the new pages: a wavefront per request
  for (int b = blockIdx.x * (kThreads / 64) + wave; b < p.batch; b += gridDim.x * (kThreads / 64)) {
    const Request r(p, b);
    const uint32_t at = page_at[b];
    if (at == kNot) continue;
    for (uint32_t i = lane; i < r.need; i += 64) p.table[(int64_t)b * p.ldt + r.have + i] = p.free_pages[n_free - 1 - (int)(at + i)];
  }
  // ---- slots
  const uint32_t total = tok_end[p.batch - 1];
  for (int64_t t = (int64_t)blockIdx.x * kThreads + tid; t < p.capacity; t += (int64_t)gridDim.x * kThreads) {
    int64_t slot = -1;
    if (t < (int64_t)total) {
      int lo = 0, hi = p.batch - 1;  // the first request whose end lies beyond t
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (tok_end[mid] > (uint32_t)t)
          hi = mid;
        else
          lo = mid + 1;
      }
      const uint32_t at = page_at[lo];
      if (at != kNot) {
        const uint32_t old = old_at[lo], start = lo ? tok_end[lo - 1] : 0, mask = (1u << p.shift) - 1;
        const uint32_t pos = old + ((uint32_t)t - start), idx = pos >> p.shift, have = (old + mask) >> p.shift;
        const int pg = idx < have ? p.table[(int64_t)lo * p.ldt + idx] : p.free_pages[n_free - 1 - (int)(at + idx - have)];
        if (pg >= 0) slot = ((int64_t)pg << p.shift) + (pos & mask);
      }
    }
    p.slots[t] = slot;
  }
}

// ------------------------------------------------------------------------------------------
// New keys and values into the cache.  Bound: HBM, each value read and written once.  A thread moves 16 bytes (eight values) of
// TOK tokens; neighbouring lanes take neighbouring pieces of a token's row, which are contiguous within a head on both sides.
// An 8-bit cache keeps code = round(x / s), s = max |x| * (1 / 127) over the token's head: its head_dim / 8 lanes lie in one group of
// 8, 16 or 32 and take the maximum by cross-lane steps.
// ------------------------------------------------------------------------------------------
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
constexpr int kAppendThreads = 256;

// STREAM: past the caches
template <bool STREAM, typename V>
__device__ __forceinline__ void put(V *p, V v) {
  if constexpr (STREAM)
    __builtin_nontemporal_store(v, p);
  else
    *p = v;
}

struct AppendParams {
  const char *k, *v;
  int64_t ldk, ldv;  // bytes
  const int64_t *slots;
  char *k_cache, *v_cache;
  float *k_scales, *v_scales;
  int64_t tokens, n_slots;
  int heads, log_pieces, shift;  // pieces of 16 bytes of a head: 1 << log_pieces
  uint32_t pieces;               // of a row: heads << log_pieces
  uint32_t units;                // of a step's TOK tokens: 2 * pieces, the keys' first
  int64_t first;                 // workgroup of the call that the launch begins with
};

template <bool BF16>
__device__ __forceinline__ void widen(u4 a, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (BF16) {
      f[2 * i] = __uint_as_float(a[i] << 16);
      f[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    } else {
      f[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)a[i]);
      f[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(a[i] >> 16));
    }
  }
}

template <bool INT8, bool BF16, int TOK>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(const AppendParams p) {
  const uint64_t id = (uint64_t)(p.first + blockIdx.x) * kAppendThreads + threadIdx.x;
  const int64_t step = (int64_t)(id / p.units);
  uint32_t piece = (uint32_t)(id % p.units);
  const bool is_v = piece >= p.pieces;
  if (is_v) piece -= p.pieces;
  const int64_t t0 = step * TOK;
  const char *src = is_v ? p.v : p.k;
  const int64_t ld = is_v ? p.ldv : p.ldk;
  char *cache = is_v ? p.v_cache : p.k_cache;
  const int head = (int)(piece >> p.log_pieces), at = (int)(piece & ((1u << p.log_pieces) - 1));
  int64_t slot[TOK];
  u4 val[TOK];
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    slot[i] = t0 + i < p.tokens ? p.slots[t0 + i] : -1;
    val[i] = u4{0, 0, 0, 0};
    if (t0 + i < p.tokens) val[i] = *reinterpret_cast<const u4 *>(src + (t0 + i) * ld + (int64_t)piece * 16);
  }
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    const bool ok = slot[i] >= 0 && slot[i] < p.n_slots;
    const int64_t page = slot[i] >> p.shift;
    const int64_t row = ((page * p.heads + head) << p.shift) + (slot[i] & ((1 << p.shift) - 1));  // of the cache [page, head, token]
    if (!INT8) {
      if (ok) put<(TOK > 1)>(reinterpret_cast<u4 *>(cache + (((row << p.log_pieces) + at) << 4)), val[i]);
    } else {
      float f[8];
      widen<BF16>(val[i], f);
      uint32_t top = 0;  // of the bit patterns: a NaN or an infinity comes out on top
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t b = __float_as_uint(f[j]) & 0x7fffffffu;
        top = b > top ? b : top;
      }
      for (int o = 1; o < (1 << p.log_pieces); o <<= 1) {
        const uint32_t other = __shfl_xor(top, o, 64);
        top = other > top ? other : top;
      }
      const bool finite = top < 0x7f800000u;
      const float s = finite ? fmaxf(__uint_as_float(top) * (1.0f / 127.0f), 0x1p-118f) : __uint_as_float(0x7fc00000u);
      uint32_t w[2] = {0, 0};
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float c = fminf(fmaxf(rintf(__fdiv_rn(f[j], s)), -127.0f), 127.0f);
        if (!finite) c = 0.0f;
        w[j >> 2] |= ((uint32_t)(int)c & 255u) << (8 * (j & 3));
      }
      if (ok) {
        put<(TOK > 1)>(reinterpret_cast<u2 *>(cache + (((row << p.log_pieces) + at) << 3)), u2{w[0], w[1]});
        if (at == 0) (is_v ? p.v_scales : p.k_scales)[row] = s;
      }
    }
  }
}

template <bool INT8, bool BF16>
cwac_status launch_append(AppendParams p, hipStream_t st) {
  // Four tokens to a thread once single ones fill the chip with threads several times.  What those write goes past the caches:
  // 16384 tokens of 8 heads of 128, bf16, 30.4 -> 25.2 us (5.3 TB/s), 4096 tokens (16 MB) 7.5 -> 6.7.  A decoding step's few tokens
  // stay, for the attention behind it.
  const bool many = p.tokens * p.units >= 4 * 262144;
  const int64_t steps = many ? ceil_div(p.tokens, 4) : p.tokens;
  const int64_t blocks = ceil_div(steps * p.units, kAppendThreads);
  static_assert(kAppendThreads == 256, "kAppendBlocksPerLaunch");
  for (p.first = 0; p.first < blocks; p.first += kAppendBlocksPerLaunch) {
    const int64_t left = blocks - p.first;
    const unsigned n = (unsigned)(left < kAppendBlocksPerLaunch ? left : kAppendBlocksPerLaunch);
    if (many)
      kv_append_kernel<INT8, BF16, 4><<<n, kAppendThreads, 0, st>>>(p);
    else
      kv_append_kernel<INT8, BF16, 1><<<n, kAppendThreads, 0, st>>>(p);
    const cwac_status s = launch_status();
    if (s != CWAC_OK) return s;
  }
  return CWAC_OK;
}

bool page_shift(int32_t page, int *shift) {
  for (int s = 4; s <= 10; ++s)
    if (page == 1 << s) {
      *shift = s;
      return true;
    }
  return false;
}

bool overlap(const void *a, int64_t na, const void *b, int64_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

}  // namespace
}  // namespace cwac

using namespace cwac;

extern "C" cwac_status llm_kv_assign_pages(const int32_t *old_lens, const int32_t *new_lens, int32_t batch, int32_t page,
                                           const int32_t *free_pages, int32_t free_capacity, const int32_t *n_free,
                                           int32_t *table, int64_t ldt, int32_t table_cols, int64_t *slots,
                                           int64_t slot_capacity, int32_t *token_start, int32_t *seq_lens, int32_t *n_left,
                                           void *stream) {
  AssignParams p{};
  if (!old_lens || !new_lens || !n_free || !table || !token_start || !seq_lens || !n_left || (!free_pages && free_capacity != 0) ||
      (!slots && slot_capacity != 0))
    return CWAC_E_NULL;
  if (batch < 1 || batch > kMaxBatch || !page_shift(page, &p.shift) || free_capacity < 0 || table_cols < 1 || ldt < table_cols ||
      slot_capacity < 0 || (int64_t)table_cols * page > 0x7fffffff)
    return CWAC_E_SHAPE;
  for (const void *q : {(const void *)old_lens, (const void *)new_lens, (const void *)free_pages, (const void *)n_free, (const void *)table,
                        (const void *)token_start, (const void *)seq_lens, (const void *)n_left})
    if (!aligned(q, 4)) return CWAC_E_ALIGN;
  if (!aligned(slots, 8)) return CWAC_E_ALIGN;
  // what is written is not what other workgroups may still read
  const struct {
    const void *p;
    int64_t n;
  } in[] = {{old_lens, 4 * (int64_t)batch}, {new_lens, 4 * (int64_t)batch}, {free_pages, 4 * (int64_t)free_capacity}, {n_free, 4}},
    outs[] = {{table, 4 * (ldt * (batch - 1) + table_cols)}, {slots, 8 * slot_capacity}, {token_start, 4 * ((int64_t)batch + 1)},
              {seq_lens, 4 * (int64_t)batch}, {n_left, 4}};
  for (const auto &o : outs)
    for (const auto &i : in)
      if (overlap(o.p, o.n, i.p, i.n)) return CWAC_E_MODE;
  p.old_lens = old_lens, p.new_lens = new_lens, p.free_pages = free_pages, p.n_free = n_free;
  p.table = table, p.token_start = token_start, p.seq_lens = seq_lens, p.n_left = n_left, p.slots = slots;
  p.ldt = ldt, p.capacity = slot_capacity, p.batch = batch, p.free_capacity = free_capacity, p.cols = table_cols;
  int64_t blocks = ceil_div(slot_capacity, kThreads);
  if (blocks < ceil_div(batch, 64)) blocks = ceil_div(batch, 64);
  if (blocks > 256) blocks = 256;
  static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void *>(&kv_assign_kernel),
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, 12 * kMaxBatch);
  if (attr != hipSuccess) return CWAC_E_LAUNCH;
  kv_assign_kernel<<<(unsigned)blocks, kThreads, 12 * batch, as_stream(stream)>>>(p);
  return launch_status();
}

extern "C" cwac_status llm_kv_append(const void *k, int64_t ldk, const void *v, int64_t ldv, int32_t type, const int64_t *slots,
                                     int64_t tokens, int32_t kv_heads, int32_t head_dim, void *k_cache, void *v_cache,
                                     int32_t cache_type, float *k_scales, float *v_scales, int32_t n_pages, int32_t page,
                                     void *stream) {
  AppendParams p{};
  if (type != CWAC_OUT_FP16 && type != CWAC_OUT_BF16) return CWAC_E_MODE;
  const bool int8 = cache_type == CWAC_OUT_INT8;
  if (!int8 && cache_type != type) return CWAC_E_MODE;
  if (tokens < 0 || tokens > 0x7fffffff || kv_heads < 1 || kv_heads > 1024 || (head_dim != 64 && head_dim != 128 && head_dim != 256) || n_pages < 1 ||
      !page_shift(page, &p.shift) || ldk < (int64_t)kv_heads * head_dim || ldv < (int64_t)kv_heads * head_dim)
    return CWAC_E_SHAPE;
  if (tokens == 0) return CWAC_OK;
  if (!k || !v || !slots || !k_cache || !v_cache || (int8 && (!k_scales || !v_scales))) return CWAC_E_NULL;
  if (!aligned(k, 16) || !aligned(v, 16) || ldk % 8 != 0 || ldv % 8 != 0 || !aligned(slots, 8) || !aligned(k_cache, 16) ||
      !aligned(v_cache, 16) || (int8 && (!aligned(k_scales, 4) || !aligned(v_scales, 4))))
    return CWAC_E_ALIGN;
  p.k = static_cast<const char *>(k), p.v = static_cast<const char *>(v), p.ldk = 2 * ldk, p.ldv = 2 * ldv;
  p.slots = slots, p.k_cache = static_cast<char *>(k_cache), p.v_cache = static_cast<char *>(v_cache);
  p.k_scales = k_scales, p.v_scales = v_scales, p.tokens = tokens, p.n_slots = (int64_t)n_pages << p.shift;
  p.heads = kv_heads, p.log_pieces = head_dim == 64 ? 3 : (head_dim == 128 ? 4 : 5);
  p.pieces = (uint32_t)kv_heads << p.log_pieces, p.units = 2 * p.pieces;
  hipStream_t st = as_stream(stream);
  if (type == CWAC_OUT_BF16) return int8 ? launch_append<true, true>(p, st) : launch_append<false, true>(p, st);
  return int8 ? launch_append<true, false>(p, st) : launch_append<false, false>(p, st);
}
