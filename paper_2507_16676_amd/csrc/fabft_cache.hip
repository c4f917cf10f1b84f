// The 4-bit key/value cache on gfx950: append, read, attention with the
// checksum of Algorithm 3, the keys' accumulated softmax weights, eviction.
//
// Values are e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and negatives) times a
// scale: K in blocks of 32 channels with a power of two, which the conversion
// instruction multiplies in, V with one scale s per row, which multiplies the
// softmax weight instead: p' = bf16(p s), o = sum p' code, c = sum p' (sum of
// codes). Both the codes and their sums are exact in bf16, so o and c differ by the
// rounding of their fp32 sums alone, as in the bf16 forward. The sums are taken
// when a row is appended: a V code or sum that changes in memory afterwards fails
// the check of the rows that see it.
#include "fabft_cache.h"

#include <algorithm>
#include <climits>
#include <type_traits>

// v_mul_legacy_f32: the product, 0 if a factor is 0, whatever the other one is
extern "C" __device__ __attribute__((const)) float mul_zero(float, float) __asm("llvm.amdgcn.fmul.legacy");

namespace fabft {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

constexpr float kInf = __builtin_inff();
// Max drift (exp2 domain) before a rescale, as in the forward: e is up to 2^8, p' = bf16(e s) up to
// 2^8 s, and o and c, sums over n keys, are below 2^10 n S with S the largest sum of |v| over a row (c
// holds hi, up to 16 above the sum of the codes): finite for n S < 2^118. A smaller e (2^-38 of it
// for every length) would take as much from the other end, where s is 2^-100 and p' 2^-126 at e = 2^-26.
constexpr float kLazy = 8.0f;

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  f32x2 f = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}
// The eight codes of x as four bf16 pairs (low half: the even code), times the power
// of two `scale` (infinity: NaN; checked with a probe on gfx950).
__device__ __forceinline__ u32x4 decode8(uint32_t x, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3));
  return r;
}
// a.lo*b.lo + a.hi*b.hi + c on bf16 pairs
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float c) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, a), __builtin_bit_cast(bf16x2, b), c,
                                         false);
}
// 2^(e - 127) from byte i of x; 255: infinity
__device__ __forceinline__ float scale_of_byte(uint32_t x, int i) {
  return __uint_as_float(((x >> (8 * i)) & 0xffu) << 23);
}
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(
      __builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}
template <int CTRL>
__device__ __forceinline__ uint32_t dppu(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kXor3 = 0x1B, kXor7 = 0x141, kXor15 = 0x140;

// over lanes i and i ^ 32
__device__ __forceinline__ float sum_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_xor32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float wave_sum(float x) {
  x += dpp<kXor1>(x);
  x += dpp<kXor2>(x);
  x += dpp<kXor7>(x);
  x += dpp<kXor15>(x);
  x += __shfl_xor(x, 16);
  return sum_xor32(x);
}
__device__ __forceinline__ float wave_max(float x) {
  x = __builtin_fmaxf(x, dpp<kXor1>(x));
  x = __builtin_fmaxf(x, dpp<kXor2>(x));
  x = __builtin_fmaxf(x, dpp<kXor7>(x));
  x = __builtin_fmaxf(x, dpp<kXor15>(x));
  x = __builtin_fmaxf(x, __shfl_xor(x, 16));
  return max_xor32(x);
}
// the test on the bits, which relaxed NaN rules cannot fold away
__device__ __forceinline__ bool nonfinite_bits(float x) {
  uint32_t b = __float_as_uint(x);
  asm volatile("" : "+v"(b));
  return (b & 0x7f800000u) == 0x7f800000u;
}

// What is read or written once and is large beside the 256 MB memory-side cache goes past it.
constexpr long long kStreamBytes = 96 << 20;

// A launch has at most 2^32 - 1 threads along a dimension of its grid.
bool grid_ok(long long groups, int threads) { return groups <= (long long)(UINT32_MAX / threads); }

// A load; STREAM: of what nothing reads again soon, past the caches' other content.
template <bool STREAM, class T>
__device__ __forceinline__ T load_from(const void* a) {
  const T* p = reinterpret_cast<const T*>(a);
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  else return *p;
}
// by value: a conditional expression of two array elements would keep the array in memory
__device__ __forceinline__ float pick(bool c, float a, float b) { return c ? a : b; }
__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// ---- a row's codes

// sum over aligned groups of N (8, 16 or 32) lanes
template <int N>
__device__ __forceinline__ float span_sum(float x) {
  x += dpp<kXor1>(x);
  x += dpp<kXor2>(x);
  x += dpp<kXor7>(x);
  if constexpr (N >= 16) x += dpp<kXor15>(x);
  if constexpr (N >= 32) x += __shfl_xor(x, 16);
  return x;
}
template <int N>
__device__ __forceinline__ uint32_t span_max(uint32_t x) {
  x = max(x, dppu<kXor1>(x));
  x = max(x, dppu<kXor2>(x));
  if constexpr (N >= 8) x = max(x, dppu<kXor7>(x));
  if constexpr (N >= 16) x = max(x, dppu<kXor15>(x));
  if constexpr (N >= 32) x = max(x, (uint32_t)__shfl_xor((int)x, 16));
  return x;
}
__device__ __forceinline__ uint32_t max_abs8(u32x4 x) {   // of eight bf16, as bits
  u16x2 m = __builtin_bit_cast(u16x2, x[0] & 0x7fff7fffu);
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    const uint32_t y = x[i] & 0x7fff7fffu;
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, y));
  }
  return max((uint32_t)m[0], (uint32_t)m[1]);
}

// Lanes of a row of D channels, eight each; 96 channels take 12 of 16 lanes.
template <int D>
struct RowLanes {
  static constexpr int N = D == 96 ? 16 : D / 8;
  static constexpr int ROWS = 256 / N;   // rows of a workgroup
};

// ---- append: one row of K and of V per RowLanes<D>::N lanes. Moves 4d bytes in and
// about d + 14 out per row: bound by memory with many rows, by latency with few.
template <int D>
__device__ __forceinline__ void append_row(uint8_t* tile, int key, int lane, bool live, u32x4 k, u32x4 v) {
  constexpr int N = RowLanes<D>::N;
  constexpr CacheTile T(D);
  // K: 2^e, the smallest with max < 7 * 2^e: m 2^x with m < 1.75 gives x - 2, else x - 1
  const uint32_t ka = span_max<4>(max_abs8(k));
  const bool kbad = ka >= 0x7f80u;
  // (at most 125: 4 * 2^126 is no number)
  const int e = kbad ? 255 : clampi((int)(ka >> 7) - 2 + ((ka & 127) >= 96 ? 1 : 0), 27, 252);
  const float ks = __uint_as_float((uint32_t)(kbad ? 127 : e) << 23);
  uint32_t kc = 0;
  {
    // x / 2^e to the nearest code, ties to the even one. (By value: a bit cast of a vector's
    // element takes the vector's first one.)
    const uint32_t k0 = k[0], k1 = k[1], k2 = k[2], k3 = k[3];
    kc = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(kc, __builtin_bit_cast(bf16x2, k0), ks, 0);
    kc = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(kc, __builtin_bit_cast(bf16x2, k1), ks, 1);
    kc = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(kc, __builtin_bit_cast(bf16x2, k2), ks, 2);
    kc = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(kc, __builtin_bit_cast(bf16x2, k3), ks, 3);
    if (kbad) kc = 0;
  }

  // V: s, the smallest number of six significant bits >= max / 6. max has eight bits, so a
  // quotient that is no such number is 2^-10 or more away from one: taken 2^-20 too small, a
  // quotient that is one does not move up to the next, and no other one changes
  const uint32_t va = span_max<N>(max_abs8(v));
  const bool vbad = va >= 0x7f80u;
  float s = __builtin_fmaxf(__uint_as_float(va << 16) * 0x1.55554p-3f, 0x1p-100f);
  s = __uint_as_float((__float_as_uint(s) + 0x3ffffu) & ~0x3ffffu);
  s = __builtin_fminf(s, 0x1.5p+125f);   // (6 s is a bf16 number)
  if (vbad) s = 1.0f;
  const float rs = __builtin_amdgcn_rcpf(s);
  uint32_t vc = 0;
  float sum = 0.f, wsum = 0.f;
  {
    // x / s in fp16: x and c s (c a border between codes) have at most 9 bits, so a
    // quotient is a border itself or at least 2^-9 of it away, and x * (1 / s), off by
    // 2^-22, rounds to the border or to its right side
    uint32_t hp[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f16x2 t = {(_Float16)(__uint_as_float(v[j] << 16) * rs),
                       (_Float16)(__uint_as_float(v[j] & 0xffff0000u) * rs)};
      hp[j] = __builtin_bit_cast(uint32_t, t);
    }
    vc = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(vc, __builtin_bit_cast(f16x2, hp[0]), 1.0f, 0);
    vc = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(vc, __builtin_bit_cast(f16x2, hp[1]), 1.0f, 1);
    vc = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(vc, __builtin_bit_cast(f16x2, hp[2]), 1.0f, 2);
    vc = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(vc, __builtin_bit_cast(f16x2, hp[3]), 1.0f, 3);
    if (vbad) vc = 0;
    const u32x4 x = decode8(vc, 1.0f);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      sum = dot2(x[j], 0x3f803f80u, sum);      // (1, 1)
      wsum = dot2(x[j], 0xbf803f80u, wsum);    // (1, -1)
    }
    sum = span_sum<N>(sum);     // multiples of 1/2 up to 1536: exact
    wsum = span_sum<N>(wsum);
  }
  if (!live) return;
  *reinterpret_cast<uint32_t*>(tile + key * T.row() + 4 * lane) = kc;
  *reinterpret_cast<uint32_t*>(tile + T.vcode() + key * T.row() + 4 * lane) = vc;
  if ((lane & 3) == 0) tile[T.kscale_at(key, lane / 4)] = (uint8_t)e;
  // lane 0: the scale, lanes 1 to 4: hi and lo of the sum and of the weighted sum
  if (lane < 5) {
    const float x = lane < 3 ? sum : wsum;
    const float hi = 16.0f * __builtin_floorf(x * 0.0625f);
    const float y = lane == 0 ? s : (lane & 1) ? hi : x - hi;
    const uint16_t u = lane == 0 && vbad ? (uint16_t)0x7fc0 : (uint16_t)(__float_as_uint(y) >> 16);
    *reinterpret_cast<uint16_t*>(tile + T.vscale() + lane * 2 * kCacheTile + 2 * key) = u;
  }
}

// ITER passes over ROWS rows. Many rows: a workgroup takes 64 neighbours of one head, all
// their loads first, so that it alone writes most lines of the scales and sums (their rows of
// 2 and 4 bytes; lines that several XCDs write in parts cost more) and has more on its way.
// (4 x 32 heads, 4,096 rows of 128: 80 us with 16 rows a workgroup and a division for s and
// 1 / s each, 65 now: 5.3 TB/s, the rate of a large copy.)
template <int D, int ITER, bool STREAM>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheRows p) {
  constexpr int N = RowLanes<D>::N, ROWS = RowLanes<D>::ROWS;
  constexpr CacheTile T(D);
  const int lane = threadIdx.x % N, sub = threadIdx.x / N;
  const bool live = lane < D / 8;
  long long bh;
  int i0;
  if constexpr (ITER > 1) {
    const int chunks = (p.n + ITER * ROWS - 1) / (ITER * ROWS);
    bh = blockIdx.x / chunks;
    i0 = (int)(blockIdx.x - bh * chunks) * ITER * ROWS + sub;
  } else {
    const long long row = (long long)blockIdx.x * ROWS + sub;
    bh = row / p.n;
    i0 = (int)(row - bh * p.n);
  }
  if (bh >= (long long)p.B * p.H) return;   // whole groups of N lanes leave together
  const int b = (int)(bh / p.H), h = (int)(bh - (long long)b * p.H);
  const int start = p.start[b], slots = p.tiles * kCacheTile;   // (at most 2^30)
  const int n = p.counts ? min(p.n, p.counts[b]) : p.n;
  uint8_t* base = p.cache + (size_t)bh * p.tiles * T.bytes();
  u32x4 k[ITER], v[ITER];
#pragma unroll
  for (int it = 0; it < ITER; ++it) {
    const int i = i0 + it * ROWS;
    k[it] = v[it] = u32x4{0, 0, 0, 0};
    if (live && i < n) {
      k[it] = load_from<STREAM, u32x4>(p.k + b * p.kb + h * p.kh + i * p.kn + 8 * lane);
      v[it] = load_from<STREAM, u32x4>(p.v + b * p.vb + h * p.vh + i * p.vn + 8 * lane);
    }
  }
#pragma unroll
  for (int it = 0; it < ITER; ++it) {
    const int i = i0 + it * ROWS;
    const uint32_t slot = (uint32_t)start + (uint32_t)i;   // (one before 0 is past the end)
    if (i < n && slot < (uint32_t)slots)
      append_row<D>(base + (size_t)(slot / kCacheTile) * T.bytes(), (int)(slot % kCacheTile), lane, live,
                    k[it], v[it]);
  }
}

// ---- read: the values of a row, zeros for rows that are not in the cache
template <int D, bool STREAM>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheRows p) {
  constexpr int N = RowLanes<D>::N;
  constexpr CacheTile T(D);
  const int lane = threadIdx.x % N;
  const long long row =
      ((long long)blockIdx.y * gridDim.x + blockIdx.x) * RowLanes<D>::ROWS + threadIdx.x / N;
  const long long bh = row / p.n;
  const int i = (int)(row - bh * p.n);
  if (bh >= (long long)p.B * p.H || lane >= D / 8) return;
  const int b = (int)(bh / p.H);
  const long long slot = (long long)p.start[b] + i;
  u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
  if (!(p.counts && i >= p.counts[b]) && slot >= 0 && slot < (long long)p.tiles * kCacheTile) {
    const uint8_t* tile = p.cache + (bh * p.tiles + slot / kCacheTile) * T.bytes();
    const int key = (int)(slot % kCacheTile);
    const uint32_t kc = *reinterpret_cast<const uint32_t*>(tile + key * T.row() + 4 * lane);
    const uint32_t vc = *reinterpret_cast<const uint32_t*>(tile + T.vcode() + key * T.row() + 4 * lane);
    const uint32_t e = tile[T.kscale_at(key, lane / 4)];
    const uint32_t s = *reinterpret_cast<const uint16_t*>(tile + T.vscale() + 2 * key);
    k = decode8(kc, scale_of_byte(e, 0));
    const u32x4 x = decode8(vc, 1.0f);
    const float sf = __uint_as_float(s << 16);
#pragma unroll
    for (int j = 0; j < 4; ++j)   // exact: 6 bits times 2
      v[j] = pack_bf16x2(__uint_as_float(x[j] << 16) * sf, __uint_as_float(x[j] & 0xffff0000u) * sf);
  }
  u32x4* kp = reinterpret_cast<u32x4*>(p.k + row * D + 8 * lane);
  u32x4* vp = reinterpret_cast<u32x4*>(p.v + row * D + 8 * lane);
  if constexpr (STREAM) {
    __builtin_nontemporal_store(k, kp);
    __builtin_nontemporal_store(v, vp);
  } else {
    *kp = k;
    *vp = v;
  }
}

// ---- attention

// What one sequence's query rows see. Row r of a key/value head is row i = r % Lq of one
// of its query heads; rows i >= cnt are padding and see nothing.
struct Seen {
  int len, cnt, off;   // causal: row i sees keys <= off + i
  // lengths and counts: those of the sequence as loaded (without counts anything)
  __device__ __forceinline__ Seen(const CacheParams& p, int lengths, int counts) {
    // (in scalar registers, and all that follows from them)
    len = clampi(__builtin_amdgcn_readfirstlane(lengths), 0, p.tiles * kCacheTile);
    cnt = p.counts ? clampi(__builtin_amdgcn_readfirstlane(counts), 0, p.Lq) : p.Lq;
    off = len - cnt;
  }
  // the last key that row r sees, -1: none
  __device__ __forceinline__ int last(const CacheParams& p, int r) const {
    const int i = r % p.Lq;
    return r >= p.R || i >= cnt ? -1 : p.causal ? max(-1, off + i) : len - 1;
  }
  // number of keys that hold all that rows r0 .. r0 + n - 1 see
  __device__ __forceinline__ int keys(const CacheParams& p, int r0, int n) const {
    const int a = r0 % p.Lq, z = min(p.R - r0, n) - 1 + a;
    if (cnt <= 0 || (z < p.Lq && a >= cnt)) return 0;
    if (!p.causal) return len;
    const int i = z < p.Lq ? min(z, cnt - 1) : cnt - 1;
    return max(0, off + i + 1);
  }
};

// The end of a row, by one wave: O = o / l, pred = c / l, the check against the sum of O
// (as in the forward: flagged when NOT |r| <= tau_rel * M + tau_abs, M = sum_j |O_j| + |pred|).
// Lane j holds columns CPL * j .. of o.
template <int D>
struct RowEnd {
  static constexpr int CPL = D == 256 ? 4 : 2;
  static constexpr int LANES = D / CPL;
  __device__ static __forceinline__ void run(const CacheParams& p, size_t row, int lane, int last,
                                             const float (&o)[CPL], float m, float l, float c,
                                             float cw) {
    float inv = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l;   // (l NaN: NaN)
    // keys, but l = 0: every score overflowed to -inf, and no weight is a number
    uint32_t none = last >= 0 && (__float_as_uint(l) << 1) == 0 ? 0x7fc00000u : 0u;
    asm volatile("" : "+v"(none));   // (as in nonfinite_bits)
    inv = __uint_as_float(__float_as_uint(inv) | none);
    float act = 0.f, absum = 0.f, actw = 0.f, x[CPL];
#pragma unroll
    for (int j = 0; j < CPL; ++j) {
      x[j] = lane < LANES ? o[j] * inv : 0.f;
      act += x[j];
      absum += __builtin_fabsf(x[j]);
      actw += (j & 1) ? -x[j] : x[j];
    }
    if (lane < LANES) {
      uint32_t* to = reinterpret_cast<uint32_t*>(p.o + row * D) + lane * (CPL / 2);
#pragma unroll
      for (int j = 0; j < CPL; j += 2) to[j / 2] = pack_bf16x2(x[j], x[j + 1]);
    }
    act = wave_sum(act);
    absum = wave_sum(absum);
    const float pred = c * inv, r = pred - act;
    bool bad = nonfinite_bits(r) || nonfinite_bits(absum);
    uint32_t f = __builtin_fabsf(r) <= p.tau_rel * (absum + __builtin_fabsf(pred)) + p.tau_abs ? 0 : 1;
    if (p.wcheck) {
      const float pw = cw * inv, rw = pw - wave_sum(actw);
      bad = bad || nonfinite_bits(rw);
      if (!(__builtin_fabsf(rw) <= p.tau_rel * (absum + __builtin_fabsf(pw)) + p.tau_abs)) f |= 4;
    }
    if (bad) f |= 3;
    if (lane == 0) {
      p.resid[row] = r;
      p.flags[row] = (uint8_t)f;
      if (p.stats) {
        // a row without keys, or with a flag, adds nothing to the weights
        const bool adds = f == 0 && l > 0.f;
        f32x4 st = {adds ? m : kInf, adds ? inv : 0.f, __int_as_float(adds ? last : -1), 0.f};
        *reinterpret_cast<f32x4*>(p.stats + 4 * row) = st;
      }
    }
  }
};

template <int D>
struct Lane {   // a lane's offsets in a tile
  int m, g, koff, ksoff, csoff;
  __device__ __forceinline__ Lane(int lane, bool wcheck) {
    constexpr CacheTile T(D);
    m = lane & 15;
    g = lane >> 4;
    koff = (16 * (m >> 2) + (m & 3)) * T.row() + g * (D / 8);
    // first 32-channel block of the lane's D / 4 channels
    const int blk = D == 64 ? g / 2 : D == 96 ? (3 * g) / 4 : D == 128 ? g : 2 * g;
    ksoff = T.kscale() + (m * T.blocks() + blk) * 4;
    // rows 0 and 1 (with the weighted check 2 and 3) of the check's operand; the
    // other rows hold copies, whose products nothing reads
    csoff = T.vsum() + (m & (wcheck ? 3 : 1)) * 2 * kCacheTile + 32 * g;
  }
};

// K of one 64-key tile in registers, as it lies in memory.
template <int D>
struct KRegs {
  static constexpr int KW = D / 32;   // 32-bit words per lane and 16-key block
  uint32_t k[4][KW];
  uint32_t ks[D == 256 || D == 96 ? 2 : 1];
  template <bool STREAM>
  __device__ __forceinline__ void load(const uint8_t* tile, const Lane<D>& ln) {
    constexpr CacheTile T(D);
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      const uint8_t* a = tile + ln.koff + kb * 4 * T.row();
      if constexpr (KW == 2) {
        const u32x2 x = load_from<STREAM, u32x2>(a);
        k[kb][0] = x[0], k[kb][1] = x[1];
      } else if constexpr (KW == 3) {
#pragma unroll
        for (int j = 0; j < 3; ++j) k[kb][j] = load_from<STREAM, uint32_t>(a + 4 * j);
      } else {
#pragma unroll
        for (int j = 0; j < KW; j += 4) {
          const u32x4 x = load_from<STREAM, u32x4>(a + 4 * j);
          k[kb][j] = x[0], k[kb][j + 1] = x[1], k[kb][j + 2] = x[2], k[kb][j + 3] = x[3];
        }
      }
    }
    ks[0] = *reinterpret_cast<const uint32_t*>(tile + ln.ksoff);
    if constexpr (D == 256) ks[1] = *reinterpret_cast<const uint32_t*>(tile + ln.ksoff + 4);
    // at d = 96 the lane's 24 channels lie in at most two blocks, the last of them (3g + 2) / 4
    if constexpr (D == 96)
      ks[1] = *reinterpret_cast<const uint32_t*>(
          tile + T.kscale() + (ln.m * T.blocks() + (3 * ln.g + 2) / 4) * 4);
  }
  // the MFMA operand of the lane's channels 8t .. 8t + 7 in 16-key block kb
  __device__ __forceinline__ u32x4 operand(int kb, int t, int g) const {
    float s;
    if constexpr (D == 96) {
      const bool second = t == 2 || (t == 1 && g == 1);   // (3g + t) / 4 is the second block
      s = scale_of_byte(second ? ks[1] : ks[0], kb);
    } else {
      s = scale_of_byte(ks[D == 256 ? t / 4 : 0], kb);
    }
    return decode8(k[kb][t], s);
  }
};

// How a workgroup's rows lie on the 16 columns of an MFMA result. RP = 32: two operands of
// 16 rows; 16: one; fewer: the RP rows repeat over the columns, so that column n has row
// n % RP, and a lane takes the softmax of VPL = RP of its 16 keys only, the column's share,
// instead of all for columns that nobody reads; the weights then meet through LDS.
// (One row, d = 128: 360 -> 225 vector instructions per tile.)
template <int RP>
struct Rows {
  static constexpr int N = RP == 32 ? 2 : 1;          // operands
  static constexpr int VPL = RP < 16 ? RP : 16;       // keys per lane and tile
  static constexpr int COLS = RP < 16 ? RP : 16;      // columns with different rows
};

// V of one tile: the codes as they lie in memory, the scales of the lane's VPL keys, the sums
// of 16 keys.
template <int D, int VPL>
struct VRegs {
  static constexpr int VC = D / 32;   // 16-byte chunks per lane
  static constexpr int SW = VPL == 1 ? 1 : VPL / 2;
  u32x4 v[VC];
  uint32_t s[SW];
  u32x4 cs[2];
  template <bool STREAM>
  __device__ __forceinline__ void load_codes(const uint8_t* tile, int lane) {
    constexpr CacheTile T(D);
#pragma unroll
    for (int j = 0; j < VC; ++j)
      v[j] = load_from<STREAM, u32x4>(tile + T.vcode() + 1024 * j + 16 * lane);
  }
  // key0: the first of the lane's keys
  __device__ __forceinline__ void load_scales(const uint8_t* tile, int key0, const Lane<D>& ln) {
    constexpr CacheTile T(D);
    const uint8_t* a = tile + T.vscale() + 2 * key0;
    if constexpr (VPL == 1) {
      s[0] = *reinterpret_cast<const uint16_t*>(a);
    } else if constexpr (VPL == 4) {
      const u32x2 x = *reinterpret_cast<const u32x2*>(a);
      s[0] = x[0], s[1] = x[1];
    } else {
#pragma unroll
      for (int j = 0; j < SW; j += 4) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(a + 4 * j);
        s[j] = x[0], s[j + 1] = x[1], s[j + 2] = x[2], s[j + 3] = x[3];
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) cs[j] = *reinterpret_cast<const u32x4*>(tile + ln.csoff + 16 * j);
  }
  __device__ __forceinline__ float scale(int j) const {
    return __uint_as_float((j & 1) ? s[j / 2] & 0xffff0000u : s[j / 2] << 16);
  }
};

// LDS address of 16-byte chunk q of V's codes: 16 bytes of room every 256, so that
// the 16 rows of a transposed read lie in different banks
template <int D>
__device__ __forceinline__ int v_chunk(int q) {
  return 16 * (D == 96 ? q : q + (q >> 4));
}

// Of the 16 scores of a lane (keys 16g + j) those of its column's share.
template <int VPL>
__device__ __forceinline__ void take_share(const f32x4 (&s)[4], int n, float (&x)[VPL]) {
  if constexpr (VPL == 16) {
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = s[j / 4][j & 3];
  } else {
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = pick(n & 8, s[2 + j / 4][j & 3], s[j / 4][j & 3]);
    if constexpr (VPL == 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = y[j];
    } else {
      float z[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) z[j] = pick(n & 4, y[j + 4], y[j]);
      if constexpr (VPL == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = z[j];
      } else {
        x[0] = pick(n & 1, pick(n & 2, z[3], z[1]), pick(n & 2, z[2], z[0]));
      }
    }
  }
}

// sum / max over the lanes that have the same row: columns n, n + COLS, .. of all four groups
template <int COLS>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int o = COLS; o < 32; o <<= 1) x += __shfl_xor(x, o);
  return sum_xor32(x);
}
template <int COLS>
__device__ __forceinline__ float row_max(float x) {
#pragma unroll
  for (int o = COLS; o < 32; o <<= 1) x = __builtin_fmaxf(x, __shfl_xor(x, o));
  return max_xor32(x);
}

constexpr int kAttnWaves = 4;

// The splits of a row tile that sees `tiles` tiles: each wave has a tile.
__device__ __forceinline__ int used_splits(int tiles, int nsplit) {
  return tiles <= kCacheFewTiles ? 1 : min(nsplit, (tiles + kAttnWaves - 1) / kAttnWaves);
}

// The sequence that has n longer ones (of equal ones the first comes first), of up to 64; by a
// whole wave.
__device__ __forceinline__ int nth_longest(const CacheParams& p, int n, int lane) {
  const int len = lane < p.B ? clampi(p.lengths[lane], 0, p.tiles * kCacheTile) : -1;
  int rank = 0;
  for (int i = 0; i < p.B; ++i) {
    const int x = __builtin_amdgcn_readlane(len, i);
    rank += x > len || (x == len && i < lane);
  }
  return __builtin_ctzll(__ballot(lane < p.B && rank == n));
}

// Two floats at once (one by one 4 heads x 256 rows of 256 over 8,192 keys, 8 splits, took 30.8
// us instead of 28.6).
__device__ __forceinline__ void put2(float* a, float x, float y) {
  const uint64_t u = __float_as_uint(x) | (uint64_t)__float_as_uint(y) << 32;
  __hip_atomic_store(reinterpret_cast<uint64_t*>(a), u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Called by the first wave of each of the n workgroups of a row tile when its records are out;
// true for one of them, when all are. Each workgroup has a word, which it sets to the
// launch's nonce (new for every launch that the host makes: nothing has to clear the words
// before) and then looks at all of them: the last one to set its word sees them all set. Of
// several that do, the one that takes the nonce out of the first word is meant (all of them
// merging 16 splits of 32 heads took 10 us longer). It clears the others too, for a captured
// launch that runs again with its nonce. (A single count of arrivals would have to start at
// a known value; exchanged into a word with the nonce it takes a round per workgroup: 64
// splits +70 us.)
__device__ __forceinline__ bool last_to_arrive(unsigned long long* words, unsigned long long nonce,
                                               int split, int n, int lane) {
  if (lane == 0) __hip_atomic_store(words + split, nonce, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // set before any other is read
  bool set = true;
  if (lane < n)
    set = __hip_atomic_load(words + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == nonce;
  if (!__all(set)) return false;
  int mine = 0;
  if (lane == 0)
    mine = __hip_atomic_exchange(words, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == nonce;
  if (!__builtin_amdgcn_readfirstlane(mine)) return false;
  if (lane < n) __hip_atomic_store(words + lane, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}

// Four columns of a row over the splits, U of them at a time; w: the splits' weights.
template <int U>
__device__ __forceinline__ f32x4 merge_columns(const float* a, size_t step, int ns, const float* w) {
  f32x4 o = {0, 0, 0, 0};
  for (int s0 = 0; s0 < ns; s0 += U) {
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = *reinterpret_cast<const f32x4*>(a + min(s0 + u, ns - 1) * step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float f = s0 + u < ns ? w[s0 + u] : 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = s0 + u < ns ? __builtin_fmaf(f, x[u][j], o[j]) : o[j];
    }
  }
  return o;
}

// The splits' records of the workgroup's rows: m = max_s m_s, x = sum_s x_s 2^(m_s - m) for x in
// {l, o, c, c_w} (c merges like one more column of o, Eq. 10), then the rows' ends. One
// workgroup reads all records from beyond its L2, so what counts is how many loads it has in
// flight: a thread takes four columns of a row over up to 32 splits at once.
constexpr int kMergeRows = 8;   // of the row tiles that merge so
template <int D>
__device__ __forceinline__ void merge_splits(const CacheParams& p, const Seen& seen, size_t row0, int r0,
                                             int rows_most, int ns, float* ex, float* st_w) {
  constexpr int RS = D + 4, C4 = D / 4, CPL = RowEnd<D>::CPL, W = kAttnWaves, K = kMergeRows / W;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int nr = min(rows_most, p.R - r0);
  const float* rec = p.ws + (row0 + r0) * p.nsplit * RS;
  f32x4 h[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int i = wave + W * k;
    h[k] = f32x4{-kInf, 0.f, 0.f, 0.f};
    if (i < nr && lane < ns)
      h[k] = *reinterpret_cast<const f32x4*>(rec + ((size_t)i * p.nsplit + lane) * RS);
  }
  float m[K], l[K], c[K], cw[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    m[k] = wave_max(h[k][0]);
    const float w = h[k][0] == -kInf ? (nonfinite_bits(h[k][1]) ? 1.f : 0.f)
                                     : __builtin_amdgcn_exp2f(h[k][0] - m[k]);
    l[k] = wave_sum(w * h[k][1]);
    c[k] = wave_sum(w * h[k][2]);
    cw[k] = wave_sum(w * h[k][3]);
    st_w[(wave + W * k) * 64 + lane] = w;
  }
  __syncthreads();
  for (int e = tid; e < nr * C4; e += 64 * W) {
    const int i = e / C4;
    const float* a = rec + (size_t)i * p.nsplit * RS + 4 + 4 * (e - i * C4);
    *reinterpret_cast<f32x4*>(ex + i * RS + 4 * (e - i * C4)) =
        ns <= 8 ? merge_columns<8>(a, RS, ns, st_w + i * 64) : merge_columns<32>(a, RS, ns, st_w + i * 64);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int i = wave + W * k;
    if (i < nr) {
      float y[CPL];
#pragma unroll
      for (int j = 0; j < CPL; ++j) y[j] = lane < RowEnd<D>::LANES ? ex[i * RS + CPL * lane + j] : 0.f;
      RowEnd<D>::run(p, row0 + r0 + i, lane, seen.last(p, r0 + i), y, m[k], l[k], c[k], cw[k]);
    }
  }
}

// One workgroup: up to RP query rows of one key/value head over one split of the keys. Each wave
// takes whole tiles of 64 keys, straight from memory into registers (K is in the layout
// of the MFMA operand; V turns through a wave's own piece of LDS with the transposing 4-bit
// read), and keeps the rows' m, l, c and o; the waves' states meet at the end. S^T = K Q^T and
// O^T = V^T P^T, as in the forward: a lane holds values of one query row (column
// n = lane % 16), keys 16g .. 16g + 15 (g = lane / 16). The tiles go round the waves of all
// splits, so that a wave's first tile depends on nothing that has to be loaded first.
// (STREAM: launch_attn.)
template <int D, int RP, bool STREAM>
__global__ __launch_bounds__(64 * kAttnWaves, D == 256 && RP == 32 ? 1 : 2) void cache_attn_kernel(CacheParams p) {
  constexpr CacheTile T(D);
  using R = Rows<RP>;
  constexpr int KT = D / 32, CB = D / 16, NT = R::N, VPL = R::VPL;
  constexpr int VLDS = D == 96 ? 32 * D : 32 * D + 2 * D;   // bytes of a wave's V (v_chunk)
  constexpr int PLDS = RP < 16 ? 128 * RP : 0;              // of its weights
  constexpr int RS = D + 4;                                 // floats of a row in the exchange
  constexpr int XLDS = R::COLS * RS * 4;
  __shared__ __align__(16) uint8_t lds[kAttnWaves * (VLDS + PLDS > XLDS ? VLDS + PLDS : XLDS)];
  __shared__ f32x4 st[kAttnWaves][16];
  __shared__ float st_w[kMergeRows * 64];
  __shared__ int last_one;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int id = blockIdx.x;
  const int inner = p.n_rt * p.nsplit, heads = p.B * p.H;
  int bh = id / inner, in = id - bh * inner;
  if ((heads & 7) == 0) {   // one head's workgroups on one XCD: they share its tiles in the L2
    const int j = id >> 3;
    bh = (j / inner) * 8 + (id & 7);
    in = j % inner;
  }
  const int rt = in / p.nsplit, split = in - rt * p.nsplit;
  const int r0 = rt * RP;
  int b = bh / p.H;
  if (p.by_length) {   // the b-th longest sequence
    b = nth_longest(p, b, lane);
    bh = b * p.H + bh % p.H;
  }
  const Lane<D> ln(lane, p.wcheck != 0);
  const int key0 = 16 * ln.g + (RP < 16 ? ln.m / RP * VPL : 0);   // the first of the lane's keys
  const size_t row0 = (size_t)bh * p.R;
  const uint8_t* base = p.cache + (size_t)bh * p.tiles * T.bytes();

  // the lengths load first, so that nothing else has to arrive before they are used, and the
  // first tile before they are known (every slot of the cache is memory)
  const int len_b = p.lengths[b], cnt_b = p.counts ? p.counts[b] : 0;
  int t = split * kAttnWaves + wave;
  KRegs<D> kr;
  VRegs<D, VPL> vr;
  {
    const uint8_t* tp = base + (size_t)min(t, p.tiles - 1) * T.bytes();
    vr.template load_codes<STREAM>(tp, lane);
    kr.template load<STREAM>(tp, ln);
    vr.load_scales(tp, key0, ln);
  }
  u32x4 q[NT][KT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    // (columns without a row take another one's, and padding rows whatever they hold:
    // a column's results depend on its own q alone)
    const int r = min(r0 + 16 * n + ln.m % R::COLS, p.R - 1);
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
      q[n][kt] = *reinterpret_cast<const u32x4*>(p.q + (row0 + r) * D + ln.g * (D / 4) + 8 * kt);
  }
  const Seen seen(p, len_b, cnt_b);
  const int keys = seen.keys(p, r0, RP);
  const int tiles = (keys + kCacheTile - 1) / kCacheTile;
  const int ns = used_splits(tiles, p.nsplit);
  if (split >= ns) return;
  int last[NT];
  int all = INT_MAX;   // keys below it need no mask: every row that sees any sees them
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    last[n] = seen.last(p, r0 + 16 * n + ln.m % R::COLS);
    all = min(all, last[n] < 0 ? INT_MAX : last[n] + 1);
  }
#pragma unroll
  for (int o = 1; o < R::COLS; o <<= 1) all = min(all, __shfl_xor(all, o));
  all = __builtin_amdgcn_readfirstlane(all);

  float m2[NT], l[NT];
  f32x4 o[NT][CB], ck[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m2[n] = -kInf;
    l[n] = 0.f;
    ck[n] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < CB; ++c) o[n][c] = f32x4{0, 0, 0, 0};
  }
  uint8_t* vl = lds + wave * (VLDS + PLDS);
  uint8_t* pl = vl + VLDS;

  // One tile; with MORE each part of the wave's next one loads into the registers of this one
  // as soon as they are free.
  const int stride = ns * kAttnWaves;
  auto step = [&](auto MORE) __attribute__((always_inline)) {
    const uint8_t* tp = base + (size_t)(t + stride) * T.bytes();
#pragma unroll
    for (int j = 0; j < VRegs<D, VPL>::VC; ++j)
      *reinterpret_cast<u32x4*>(vl + v_chunk<D>(64 * j + lane)) = vr.v[j];
    if constexpr (MORE) vr.template load_codes<STREAM>(tp, lane);
    f32x4 s[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) s[n][kb] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        const u32x4 a = kr.operand(kb, kt, ln.g);
#pragma unroll
        for (int n = 0; n < NT; ++n) s[n][kb] = mfma16(a, q[n][kt], s[n][kb]);
      }
    }
    if constexpr (MORE) kr.template load<STREAM>(tp, ln);
    float x[NT][VPL], mx[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) take_share<VPL>(s[n], ln.m, x[n]);
    if ((t + 1) * kCacheTile > all) {
      asm volatile("");   // a branch: most tiles pass it by, and selects would cost as much as the max
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int lim = last[n] - t * kCacheTile - key0;   // the row sees the lane's keys j <= lim
#pragma unroll
        for (int j = 0; j < VPL; ++j) x[n][j] = j <= lim ? x[n][j] : -kInf;
      }
      // sums of slots that were never written may be anything, NaN among it
      const int n = seen.len - t * kCacheTile - 16 * ln.g;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        vr.cs[j / 4][j & 3] &= (2 * j < n ? 0xffffu : 0u) | (2 * j + 1 < n ? 0xffff0000u : 0u);
    }
    bool far = false;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      mx[n] = x[n][0];
#pragma unroll
      for (int j = 1; j < VPL; ++j) mx[n] = __builtin_fmaxf(mx[n], x[n][j]);
      far = far || mx[n] * p.sl2 > m2[n] + kLazy;
    }
    if (__any(far)) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float mt = row_max<R::COLS>(mx[n]) * p.sl2;
        const float mn = mt > m2[n] + kLazy ? mt : m2[n];
        const float alpha = mn == m2[n] ? 1.0f : __builtin_amdgcn_exp2f(m2[n] - mn);
        l[n] *= alpha;
        ck[n] *= alpha;
#pragma unroll
        for (int c = 0; c < CB; ++c) o[n][c] *= alpha;
        m2[n] = mn;
      }
    }
    u32x4 pp[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float nm = m2[n] == -kInf ? 0.f : -m2[n];
#pragma unroll
      for (int j = 0; j < VPL; ++j) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][j], p.sl2, nm));
        l[n] += e;
        // 0 where e is 0, whatever the scale: that of a key that is not seen may be anything
        x[n][j] = mul_zero(e, vr.scale(j));
      }
      if constexpr (RP >= 16) {
#pragma unroll
        for (int j = 0; j < 8; ++j) pp[n][j / 4][j & 3] = pack_bf16x2(x[n][2 * j], x[n][2 * j + 1]);
      } else {
        // 16 weights of a row and group in 32 bytes; every column reads its row's
        uint8_t* a = pl + ((ln.m % RP) * 4 + ln.g) * 32;
        uint8_t* w = a + (ln.m / RP) * VPL * 2;
        if constexpr (VPL == 1) {
          *reinterpret_cast<uint16_t*>(w) = (uint16_t)pack_bf16x2(x[n][0], 0.f);
        } else if constexpr (VPL == 4) {
          *reinterpret_cast<u32x2*>(w) =
              u32x2{pack_bf16x2(x[n][0], x[n][1]), pack_bf16x2(x[n][2], x[n][3])};
        } else {
          *reinterpret_cast<u32x4*>(w) =
              u32x4{pack_bf16x2(x[n][0], x[n][1]), pack_bf16x2(x[n][2], x[n][3]),
                    pack_bf16x2(x[n][4], x[n][5]), pack_bf16x2(x[n][6], x[n][7])};
        }
        pp[n][0] = *reinterpret_cast<const u32x4*>(a);
        pp[n][1] = *reinterpret_cast<const u32x4*>(a + 16);
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      ck[n] = mfma16(vr.cs[0], pp[n][0], ck[n]);
      ck[n] = mfma16(vr.cs[1], pp[n][1], ck[n]);
    }
    if constexpr (MORE) vr.load_scales(tp, key0, ln);
#pragma unroll
    for (int c = 0; c < CB; ++c) {
      // lane i of a group reads columns 16c .. of key 16g + i and gets column 16c + i
      // of keys 16g .. 16g + 15
      const int a = v_chunk<D>((16 * ln.g + ln.m) * (D / 32) + c / 2) + 8 * (c & 1);
      const i32x2 y = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2*)(vl + a));
      const u32x4 a0 = decode8((uint32_t)y[0], 1.0f), a1 = decode8((uint32_t)y[1], 1.0f);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        o[n][c] = mfma16(a0, pp[n][0], o[n][c]);
        o[n][c] = mfma16(a1, pp[n][1], o[n][c]);
      }
    }
  };
  for (; t + stride < tiles; t += stride) step(std::true_type{});
  if (t < tiles) step(std::false_type{});

  // the waves' states: m = max_w m_w, x = sum_w x_w 2^(m_w - m), 16 rows at a time
  float* ex = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    l[n] = row_sum<R::COLS>(l[n]);
    __syncthreads();   // the LDS is free
    if (ln.m < R::COLS) {
      // hi and lo of c, and of c_w
      if (ln.g == 0) st[wave][ln.m] = f32x4{m2[n], l[n], ck[n][0] + ck[n][1], ck[n][2] + ck[n][3]};
      if (last[n] >= 0) {
#pragma unroll
        for (int c = 0; c < CB; ++c)
          *reinterpret_cast<f32x4*>(ex + (wave * R::COLS + ln.m) * RS + 16 * c + 4 * ln.g) = o[n][c];
      }
    }
    __syncthreads();
    constexpr int CPL = RowEnd<D>::CPL;
    for (int i = wave; i < R::COLS; i += kAttnWaves) {
      const int r = r0 + 16 * n + i;
      if (r >= p.R) break;   // wave-uniform, as all below
      const int lr = seen.last(p, r);
      // a row that sees no key: m = -inf and zeros, whatever its q made of the keys that the
      // tile's other rows see (m = +inf would be NaN where splits are merged)
      float mm = -kInf, x[CPL], ls = 0.f, cs = 0.f, cw = 0.f;
#pragma unroll
      for (int j = 0; j < CPL; ++j) x[j] = 0.f;
      if (lr >= 0) {
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) mm = __builtin_fmaxf(mm, st[w][i][0]);
#pragma unroll
        for (int w = 0; w < kAttnWaves; ++w) {
          const f32x4 sw = st[w][i];
          // a wave without a tile, or whose tiles the row does not see, has l = 0
          const float f = sw[0] == -kInf ? (nonfinite_bits(sw[1]) ? 1.f : 0.f)
                                         : __builtin_amdgcn_exp2f(sw[0] - mm);
          ls = __builtin_fmaf(f, sw[1], ls);
          cs = __builtin_fmaf(f, sw[2], cs);
          cw = __builtin_fmaf(f, sw[3], cw);
          if (lane < RowEnd<D>::LANES) {
#pragma unroll
            for (int j = 0; j < CPL; ++j)
              x[j] = __builtin_fmaf(f, ex[(w * R::COLS + i) * RS + CPL * lane + j], x[j]);
          }
        }
      }
      if (ns == 1) {
        RowEnd<D>::run(p, row0 + r, lane, lr, x, mm, ls, cs, cw);
      } else {
        // (to the memory that all XCDs see: their L2s are not coherent with each other)
        float* rec = p.ws + ((row0 + r) * p.nsplit + split) * RS;
        if (lane < 2) put2(rec + 2 * lane, lane ? cs : mm, lane ? cw : ls);
        if (lane < RowEnd<D>::LANES) {
#pragma unroll
          for (int j = 0; j < CPL; j += 2) put2(rec + 4 + CPL * lane + j, x[j], x[j + 1]);
        }
      }
    }
  }
  if (RP > kMergeRows || ns == 1 || !p.tickets) return;
  // the last of the row tile's workgroups to come here merges the splits
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's part of the records is out
  __syncthreads();
  if (wave == 0) {
    const bool is_last = last_to_arrive(p.tickets + ((size_t)bh * p.n_rt + rt) * p.nsplit, p.nonce, split,
                                        ns, lane);
    if (lane == 0) last_one = is_last;
  }
  __syncthreads();
  if (!last_one) return;
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");   // no older copy of a record is read
  merge_splits<D>(p, seen, row0, r0, RP, ns, ex, st_w);
}

// The same merge as a launch of its own, one wave per row, for records that are too much for
// one workgroup per row tile (launch_attn says when).
template <int D>
__global__ __launch_bounds__(256) void cache_merge_kernel(CacheParams p, int row_tile) {
  constexpr int RS = D + 4, CPL = RowEnd<D>::CPL;
  __shared__ float st_w[4][64];
  __shared__ __align__(16) float ex[4][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nrb = (p.R + 3) / 4;
  const int bh = blockIdx.x / nrb, b = bh / p.H;
  const int r = (blockIdx.x - bh * nrb) * 4 + wave;
  if (r >= p.R) return;   // (the waves do not meet)
  const Seen seen(p, p.lengths[b], p.counts ? p.counts[b] : 0);
  const int tiles = (seen.keys(p, r / row_tile * row_tile, row_tile) + kCacheTile - 1) / kCacheTile;
  const int ns = used_splits(tiles, p.nsplit);
  if (ns == 1) return;   // the row is done
  const size_t row = (size_t)bh * p.R + r;
  const float* rec = p.ws + row * p.nsplit * RS;
  f32x4 h = {-kInf, 0.f, 0.f, 0.f};
  if (lane < ns) h = *reinterpret_cast<const f32x4*>(rec + (size_t)lane * RS);
  const float m = wave_max(h[0]);
  const float w = h[0] == -kInf ? (nonfinite_bits(h[1]) ? 1.f : 0.f) : __builtin_amdgcn_exp2f(h[0] - m);
  const float l = wave_sum(w * h[1]), c = wave_sum(w * h[2]), cw = wave_sum(w * h[3]);
  st_w[wave][lane] = w;
  if (lane < D / 4)
    *reinterpret_cast<f32x4*>(&ex[wave][4 * lane]) = merge_columns<32>(rec + 4 + 4 * lane, RS, ns, st_w[wave]);
  float y[CPL];
#pragma unroll
  for (int j = 0; j < CPL; ++j) y[j] = lane < RowEnd<D>::LANES ? ex[wave][CPL * lane + j] : 0.f;
  RowEnd<D>::run(p, row, lane, seen.last(p, r), y, m, l, c, cw);
}

// ---- the keys' weights: weight_k <- decay * weight_k + sum over the head's rows of
// 2^(s - m) / l, with the m and l of the finished rows. A second product K Q^T (the scores of
// the attention, bit for bit); every key belongs to one wave, so the sums have one order.
// K turns into operands once per tile, the rows go by 16 at a time. More than 16 rows lie in
// LDS, 128 of them at once, for the four waves (each with its tile); loaded by every wave
// from the L2, one operand ahead, 128 rows took twice as long. What bounds it then is the
// exponentials.
constexpr int kWeightRows = 128;   // of q in LDS

template <int D, bool MANY>
__global__ __launch_bounds__(256, 2) void cache_weight_kernel(CacheParams p, int chunks) {
  constexpr CacheTile T(D);
  constexpr int KT = D / 32;
  constexpr int QS = 2 * D + 16;   // bytes of a row in LDS (the rows in different banks)
  __shared__ __align__(16) uint8_t lq[MANY ? kWeightRows * QS : 16];
  __shared__ f32x4 lst[MANY ? kWeightRows : 1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bh = blockIdx.x / chunks, chunk = blockIdx.x - bh * chunks;
  const int b = bh / p.H;
  const Lane<D> ln(lane, false);
  const size_t row0 = (size_t)bh * p.R;
  const uint8_t* base = p.cache + (size_t)bh * p.tiles * T.bytes();
  const int len_b = p.lengths[b], cnt_b = p.counts ? p.counts[b] : 0;
  int t = chunk * 4 + wave;
  KRegs<D> r;
  r.template load<false>(base + (size_t)min(t, p.tiles - 1) * T.bytes(), ln);
  // rows c0 .. of q and their m, 1 / l: to LDS, by all
  auto stage = [&](int c0) __attribute__((always_inline)) {
    const int n = min(kWeightRows, p.R - c0);
    for (int e = tid; e < n * (D / 8); e += 256) {
      const int i = e / (D / 8), c = e - i * (D / 8);
      *reinterpret_cast<u32x4*>(lq + i * QS + 16 * c) =
          *reinterpret_cast<const u32x4*>(p.q + (row0 + c0 + i) * D + 8 * c);
    }
    if (tid < n) lst[tid] = *reinterpret_cast<const f32x4*>(p.stats + 4 * (row0 + c0 + tid));
  };
  u32x4 q1[KT];
  f32x4 st1;
  if constexpr (MANY) {
    stage(0);
    __syncthreads();
  } else {
    const size_t row = row0 + min(ln.m, p.R - 1);
    st1 = *reinterpret_cast<const f32x4*>(p.stats + 4 * row);
    if (ln.m >= p.R) st1[1] = 0.f;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
      q1[kt] = *reinterpret_cast<const u32x4*>(p.q + row * D + ln.g * (D / 4) + 8 * kt);
  }
  const Seen seen(p, len_b, cnt_b);
  const int tiles = (seen.len + kCacheTile - 1) / kCacheTile;
  // (the waves of a workgroup go round together, with or without a tile: they meet at the LDS)
  for (; t - wave < tiles; t += chunks * 4) {
    const bool work = t < tiles;
    if (!MANY && !work) break;
    float* wp = p.weight + ((size_t)bh * p.tiles + t) * kCacheTile + lane;
    const bool in = t * kCacheTile + lane < seen.len;
    const float old = in && p.decay != 0.f ? *wp : 0.f;
    u32x4 a[4][KT];
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) a[kb][kt] = r.operand(kb, kt, ln.g);
    const int tn = t + chunks * 4;
    if (tn < tiles) r.template load<false>(base + (size_t)tn * T.bytes(), ln);
    // keys that some row that sees any does not see
    const bool edge = (t + 1) * kCacheTile > (p.causal ? seen.off + 1 : seen.len);
    float acc[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) acc[j] = 0.f;
    // rows that add nothing (1 / l = 0) have to, whatever their q and the keys hold, NaN too:
    // one operand by a product that is 0 then, several by the mask (st[2] is -1)
    auto rows16 = [&](const u32x4 (&q)[KT], const f32x4& st, bool mask) __attribute__((always_inline)) {
      f32x4 s[4];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) s[kb] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) s[kb] = mfma16(a[kb][kt], q[kt], s[kb]);
      if (mask) {
        asm volatile("");   // (a branch)
        const int lim = __float_as_int(st[2]) - t * kCacheTile - 16 * ln.g;
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j / 4][j & 3] = j <= lim ? s[j / 4][j & 3] : -kInf;
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j / 4][j & 3], p.sl2, -st[0]));
        if constexpr (MANY) acc[j] = __builtin_fmaf(e, st[1], acc[j]);
        else acc[j] = mul_zero(e, st[1]);
      }
    };
    if constexpr (!MANY) {
      rows16(q1, st1, edge);
    } else {
      for (int c0 = 0; c0 < p.R; c0 += kWeightRows) {
        if (p.R > kWeightRows) {
          __syncthreads();
          stage(c0);
          __syncthreads();
        }
        if (!work) continue;
        const int n = min(kWeightRows, p.R - c0);
        for (int r0 = 0; r0 < n; r0 += 16) {
          const int i = min(r0 + ln.m, n - 1);
          f32x4 st = lst[i];
          if (r0 + ln.m >= n) st = f32x4{kInf, 0.f, __int_as_float(-1), 0.f};
          u32x4 q[KT];
#pragma unroll
          for (int kt = 0; kt < KT; ++kt)
            q[kt] = *reinterpret_cast<const u32x4*>(lq + i * QS + ln.g * (D / 2) + 16 * kt);
          rows16(q, st, edge || __any(!(st[1] > 0.f)));
        }
      }
      if (!work) continue;
    }
    // sum over the 16 rows (lanes n) with half the values left after each step: lane n
    // ends with key 16g + n
    float y[8], z[4], u[2];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool hi = ln.m & 8;
      const float keep = pick(hi, acc[j + 8], acc[j]), give = pick(hi, acc[j], acc[j + 8]);
      y[j] = keep + dpp<kXor15>(give);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool hi = ln.m & 4;
      const float keep = pick(hi, y[j + 4], y[j]), give = pick(hi, y[j], y[j + 4]);
      z[j] = keep + dpp<kXor7>(give);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bool hi = ln.m & 2;
      const float keep = pick(hi, z[j + 2], z[j]), give = pick(hi, z[j], z[j + 2]);
      u[j] = keep + dpp<kXor3>(give);
    }
    const bool hi = ln.m & 1;
    const float keep = pick(hi, u[1], u[0]), give = pick(hi, u[0], u[1]);
    const float sum = keep + dpp<kXor1>(give);
    if (in) *wp = p.decay != 0.f ? __builtin_fmaf(p.decay, old, sum) : sum;
  }
}

template <int D>
int launch_attn(const CacheParams& p0, hipStream_t s) {
  const int rt = cache_row_tile(p0.R);
  const long long g = (long long)p0.B * p0.H * p0.n_rt * p0.nsplit;
  const long long heads = (long long)p0.B * p0.H, mg = heads * ((p0.R + 3) / 4);
  // the weights: about four workgroups per CU, each wave one tile or more
  const int most = (p0.tiles + 3) / 4;
  long long ch = (1024 + heads - 1) / heads;
  if (ch > most) ch = most;
  (void)hipGetLastError();
  const dim3 grid((unsigned)g), block(64 * kAttnWaves);
  // One CU takes 60 GB/s or so from beyond its L2: with 135 KB of records a row tile (32 rows of
  // 128, 8 splits) the call took 66 us with the merge in the last workgroup and 60 with it as a
  // launch of its own, with 67 KB (4 rows, 32 splits) 16.9 and 17.2. Of 16 rows and more always:
  // 16 of 64, 16 splits, 16.1 and 14.2, 128 row tiles of 16, 4 splits, 27.2 and 25.4 (192 in two
  // splits 53 and 55), 64 row tiles of 32, 4 splits, 35.1 and 28.7.
  const bool apart =
      p0.nsplit > 1 && (rt > kMergeRows || (long long)std::min(rt, p0.R) * p0.nsplit * (D + 4) * 4 > 100000);
  if (!grid_ok(g, 64 * kAttnWaves) || (apart && !grid_ok(mg, 256)) || (p0.weight && !grid_ok(heads * ch, 256)))
    return kCacheGrid;
  CacheParams p = p0;
  // More workgroups than fit at once: the longest sequences first, so that none of them starts
  // when the others end.
  p.by_length = p.n_rt > 1 && p.B > 1 && p.B <= 64 && g > 512;
  if (apart) p.tickets = nullptr;
  // A stream where every tile is read once: 579 MB 108 us, 93 as a stream (6.1 TB/s), 114 MB 28.6
  // and 26.4. Where what an earlier call left in the memory-side cache is read again, it costs
  // (three caches in turn, 70 MB each: 23.4 and 25.3).
  const bool stream =
      p.n_rt == 1 && (long long)p.B * p.H * p.tiles * CacheTile(D).bytes() > kStreamBytes;
  auto launch = [&](auto RP) {
    if (RP <= 16 && stream)
      hipLaunchKernelGGL((cache_attn_kernel<D, RP, RP <= 16>), grid, block, 0, s, p);
    else
      hipLaunchKernelGGL((cache_attn_kernel<D, RP, false>), grid, block, 0, s, p);
  };
  if (rt == 1) launch(std::integral_constant<int, 1>{});
  else if (rt == 4) launch(std::integral_constant<int, 4>{});
  else if (rt == 8) launch(std::integral_constant<int, 8>{});
  else if (rt == 16) launch(std::integral_constant<int, 16>{});
  else launch(std::integral_constant<int, 32>{});
  if (apart) hipLaunchKernelGGL((cache_merge_kernel<D>), dim3((unsigned)mg), dim3(256), 0, s, p, rt);
  if (p.weight) {
    const dim3 wg((unsigned)(heads * ch));
    if (p.R > 16) hipLaunchKernelGGL((cache_weight_kernel<D, true>), wg, dim3(256), 0, s, p, (int)ch);
    else hipLaunchKernelGGL((cache_weight_kernel<D, false>), wg, dim3(256), 0, s, p, (int)ch);
  }
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

// ---- eviction

// Weights in ascending order as unsigned numbers; NaN above all, -0 as 0.
__device__ __forceinline__ uint32_t order_of(float w) {
  uint32_t u = __float_as_uint(w);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  if (u == 0x80000000u) u = 0;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

constexpr int kEvictThreads = 1024;
constexpr int kEvictKeys = 32;   // candidates in a thread's registers

// An array in LDS that one wave scans, each lane C neighbours: a word of room every 32, so that
// the lanes read different banks.
__device__ __forceinline__ constexpr int skew(int i) { return i + i / 32; }

// The bin (from the top, of N) in which the running count of a histogram reaches `need` >= 1,
// and the count above it, by one wave.
template <int N>
__device__ __forceinline__ void find_bin(const int* hist, int need, int lane, int* bin, int* above) {
  constexpr int C = N / 64;
  int x[C], s = 0;
#pragma unroll
  for (int j = 0; j < C; ++j) s += x[j] = hist[skew(N - 1 - C * lane - j)];
  int before = s;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(before, o);
    if (lane >= o) before += y;
  }
  before -= s;
  if (before < need && need <= before + s) {   // one lane
    int at = N - 1 - C * lane, n = before;
#pragma unroll
    for (int j = 0; j < C - 1; ++j) {
      const bool on = before + x[j] < need;   // (then for all before it too)
      before += x[j];
      if (on) n = before, --at;
    }
    *bin = at;
    *above = n;
  }
}

// One workgroup per head: the slots it keeps, in slot order. The last min(recent, len)
// slots stay; of the others those with the largest weights, found as a threshold by three
// passes over 11, 11 and 10 bits of the weight (a histogram in LDS of the candidates that
// share the bits found so far; 11 bits hold two of the mantissa, without which most weights
// of a head would meet in a few bins); equal weights at the threshold go by slot. Up to
// 32 candidates a thread are read once and stay in registers (with a load for each pass and
// key, one after the other, 32,768 candidates took 71 us).
template <int THREADS>
__global__ __launch_bounds__(THREADS) void cache_select_kernel(CacheEvict p) {
  constexpr int K = kEvictKeys, W = THREADS / 64, CHUNK = K * THREADS;
  __shared__ int hists[3][skew(2048)];
  __shared__ int cnt[2][skew(K * W) + 1];   // per row of 64 candidates: above the threshold, equal
  __shared__ int sh_bin, sh_above;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int bh = blockIdx.x, b = bh / p.H;
  const int slots = p.tiles * kCacheTile;
  const float* w = p.weight + (size_t)bh * slots;
  uint32_t u[K];
  auto load = [&](int c0) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int i = c0 + k * THREADS;
      u[k] = 0;
      if (i + THREADS <= slots) u[k] = __float_as_uint((w + i)[tid]);   // (the same for all)
      else if (i + tid < slots) u[k] = __float_as_uint((w + i)[tid]);
    }
  };
  auto order = [&](int c0, int old) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (c0 + k * THREADS < old) u[k] = order_of(__uint_as_float(u[k]));
    }
  };
  const int len_b = p.lengths[b];
  load(0);   // before the length is known: every slot has a weight
  for (int j = tid; j < 3 * skew(2048); j += THREADS) hists[0][j] = 0;
  const int len = clampi(__builtin_amdgcn_readfirstlane(len_b), 0, slots);
  const int kept = min(len, p.keep);
  int* index = p.index + (size_t)bh * p.keep;
  if (tid == 0 && bh == b * p.H) p.new_lengths[b] = kept;
  for (int j = kept + tid; j < p.keep; j += THREADS) index[j] = -1;
  if (len <= p.keep) {
    for (int j = tid; j < len; j += THREADS) index[j] = j;
    return;
  }
  const int old = len - min(p.recent, p.keep);   // candidates: slots [0, old)
  const int want = kept - (len - old);           // of them to keep, < old
  for (int j = tid; j < len - old; j += THREADS) index[want + j] = old + j;
  if (want <= 0) return;
  order(0, old);
  uint32_t prefix = 0;
  int need = want;   // how many of the candidates with the prefix to keep
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    int* hist = hists[pass];
    if (pass == 0) __syncthreads();
    for (int c0 = 0; c0 < old; c0 += CHUNK) {
      if (old > CHUNK) {
        load(c0);
        order(c0, old);
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int i = c0 + k * THREADS;
        if (i >= old) break;
        if (i + tid < old && (pass == 0 || (u[k] >> (shift + bits)) == (prefix >> (shift + bits))))
          atomicAdd(&hist[skew((u[k] >> shift) & ((1 << bits) - 1))], 1);
      }
    }
    __syncthreads();
    if (wave == 0) {
      if (pass < 2) find_bin<2048>(hist, need, lane, &sh_bin, &sh_above);
      else find_bin<1024>(hist, need, lane, &sh_bin, &sh_above);
    }
    __syncthreads();
    prefix |= (uint32_t)sh_bin << shift;
    need -= sh_above;
  }
  // prefix is the threshold: all above it, and the first `need` equal to it
  const uint64_t below = (1ull << lane) - 1;
  int ng0 = 0, ne0 = 0;   // of the chunks before
  for (int c0 = 0; c0 < old; c0 += CHUNK) {
    if (old > CHUNK) {
      load(c0);
      order(c0, old);
    }
    __syncthreads();
    for (int j = tid; j < skew(K * W); j += THREADS) cnt[0][j] = cnt[1][j] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int i = c0 + k * THREADS;
      if (i >= old) break;
      const bool in = i + tid < old;
      const uint64_t mg = __ballot(in && u[k] > prefix), me = __ballot(in && u[k] == prefix);
      if (lane == 0) {
        cnt[0][skew(k * W + wave)] = __popcll(mg);
        cnt[1][skew(k * W + wave)] = __popcll(me);
      }
    }
    __syncthreads();
    // running counts of the K * W rows: wave 0 the first kind, wave 1 the second
    if (wave < 2) {
      constexpr int C = K * W / 64;
      int s = 0, x[C];
#pragma unroll
      for (int j = 0; j < C; ++j) s += x[j] = cnt[wave][skew(C * lane + j)];
      int before = s;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(before, o);
        if (lane >= o) before += y;
      }
      if (lane == 63) cnt[wave][skew(K * W)] = before;
      before -= s;
#pragma unroll
      for (int j = 0; j < C; ++j) {
        cnt[wave][skew(C * lane + j)] = before;
        before += x[j];
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int i = c0 + k * THREADS;
      if (i >= old) break;
      const bool in = i + tid < old, gt = in && u[k] > prefix, eq = in && u[k] == prefix;
      const uint64_t mg = __ballot(gt), me = __ballot(eq);
      const int ng = ng0 + cnt[0][skew(k * W + wave)] + __popcll(mg & below);
      const int ne = ne0 + cnt[1][skew(k * W + wave)] + __popcll(me & below);
      if (gt || (eq && ne < need)) index[ng + min(ne, need)] = i + tid;
    }
    ng0 += cnt[0][skew(K * W)];
    ne0 += cnt[1][skew(K * W)];
  }
}

// The kept rows move to their new slots. In place (into == cache) one workgroup per head
// and half (K, V) takes the rows in order, a batch at a time: a row only moves down, so
// once a batch is in registers its slots may be written, and no later batch needs them.
// Into another cache every batch has its own workgroup.
// Half 0 moves K's codes and scales and the weights, half 1 V's codes, scales and sums.
template <int D>
__global__ __launch_bounds__(kEvictThreads) void cache_move_kernel(CacheEvict p, int batches) {
  constexpr CacheTile T(D);
  constexpr int CH = D / 32;            // 16-byte chunks of a row's codes
  constexpr int BATCH = 1024;           // rows
  constexpr int NC = BATCH * CH / kEvictThreads;
  const int tid = threadIdx.x;
  const int part = blockIdx.x & 1;
  const int chunk = (blockIdx.x >> 1) % batches;
  const int bh = (blockIdx.x >> 1) / batches;
  const int len_b = p.lengths[bh / p.H];
  const int* index = p.index + (size_t)bh * p.keep;   // -1 behind the kept ones
  const uint8_t* src = p.cache + (size_t)bh * p.tiles * T.bytes();
  uint8_t* dst = p.into + (size_t)bh * p.into_tiles * T.bytes();
  const float* w = p.weight + (size_t)bh * p.tiles * kCacheTile;
  float* nw = p.into_weight + (size_t)bh * p.into_tiles * kCacheTile;
  const int codes = part ? T.vcode() : 0;
  for (int j0 = chunk * BATCH; j0 < p.keep; j0 += batches * BATCH) {
    u32x4 c[NC];
    int from[NC];
#pragma unroll
    for (int k = 0; k < NC; ++k) from[k] = index[min(j0 + (k * kEvictThreads + tid) / CH, p.keep - 1)];
    // the small parts: one row per thread
    const int j = j0 + tid, i = index[min(j, p.keep - 1)];
    const bool mine = j < p.keep && i >= 0;
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int e = k * kEvictThreads + tid, f = from[k];
      if (f >= 0)
        c[k] = *reinterpret_cast<const u32x4*>(src + (size_t)(f / kCacheTile) * T.bytes() + codes +
                                               (f % kCacheTile) * T.row() + 16 * (e % CH));
    }
    uint8_t ks[T.blocks()];
    uint16_t vs[5];
    float wt = 0.f;
    if (mine) {
      const uint8_t* tile = src + (size_t)(i / kCacheTile) * T.bytes();
      if (part == 0) {
#pragma unroll
        for (int k = 0; k < T.blocks(); ++k) ks[k] = tile[T.kscale_at(i % kCacheTile, k)];
        wt = w[i];
      } else {
#pragma unroll
        for (int k = 0; k < 5; ++k)
          vs[k] = *reinterpret_cast<const uint16_t*>(tile + T.vscale() + 2 * kCacheTile * k +
                                                     2 * (i % kCacheTile));
      }
    }
    // every value of the batch has arrived before any slot of it is written
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NC; ++k) {
      const int e = k * kEvictThreads + tid, jj = j0 + e / CH;
      if (jj < p.keep && from[k] >= 0)
        *reinterpret_cast<u32x4*>(dst + (size_t)(jj / kCacheTile) * T.bytes() + codes +
                                  (jj % kCacheTile) * T.row() + 16 * (e % CH)) = c[k];
    }
    if (mine) {
      uint8_t* tile = dst + (size_t)(j / kCacheTile) * T.bytes();
      if (part == 0) {
#pragma unroll
        for (int k = 0; k < T.blocks(); ++k) tile[T.kscale_at(j % kCacheTile, k)] = ks[k];
        nw[j] = wt;
      } else {
#pragma unroll
        for (int k = 0; k < 5; ++k)
          *reinterpret_cast<uint16_t*>(tile + T.vscale() + 2 * kCacheTile * k +
                                       2 * (j % kCacheTile)) = vs[k];
      }
    }
  }
  const int kept = min(clampi(len_b, 0, p.tiles * kCacheTile), p.keep);
  // the slots behind them have no weight. In place the same workgroup has read all it
  // needs of them by now
  if (part == 0)
    for (int j = kept + chunk * kEvictThreads + tid; j < p.into_tiles * kCacheTile;
         j += batches * kEvictThreads)
      nw[j] = 0.f;
}

template <int D>
int launch_evict(const CacheEvict& p, hipStream_t s) {
  const long long heads = (long long)p.B * p.H;
  const int batches = p.into == p.cache ? 1 : (p.keep + 1023) / 1024;
  if (!grid_ok(heads * batches * 2, kEvictThreads)) return kCacheGrid;
  (void)hipGetLastError();
  // four waves meet sooner than sixteen, as long as they hold the candidates
  if (p.tiles * kCacheTile <= 256 * kEvictKeys)
    hipLaunchKernelGGL((cache_select_kernel<256>), dim3((unsigned)heads), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((cache_select_kernel<1024>), dim3((unsigned)heads), dim3(1024), 0, s, p);
  hipLaunchKernelGGL((cache_move_kernel<D>), dim3((unsigned)(heads * batches * 2)),
                     dim3(kEvictThreads), 0, s, p, batches);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <int D>
int launch_append(const CacheRows& p, hipStream_t s) {
  constexpr int ROWS = RowLanes<D>::ROWS, ITER = 64 / ROWS;
  const long long heads = (long long)p.B * p.H;
  const bool many = p.n >= 64;   // (n: at most 2^30)
  const long long g = many ? heads * ((p.n + 63) / 64) : (heads * p.n + ROWS - 1) / ROWS;
  if (!grid_ok(g, 256)) return kCacheGrid;
  (void)hipGetLastError();
  const dim3 grid((unsigned)g), block(256);
  if (many && heads * p.n * 4 * D > kStreamBytes)
    hipLaunchKernelGGL((cache_append_kernel<D, ITER, true>), grid, block, 0, s, p);
  else if (many)
    hipLaunchKernelGGL((cache_append_kernel<D, ITER, false>), grid, block, 0, s, p);
  else
    hipLaunchKernelGGL((cache_append_kernel<D, 1, false>), grid, block, 0, s, p);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <int D>
int launch_read(const CacheRows& p, hipStream_t s) {
  const long long rows = (long long)p.B * p.H * p.n;
  const long long g = (rows + RowLanes<D>::ROWS - 1) / RowLanes<D>::ROWS;
  // (137 GB of values are more workgroups than one dimension holds)
  const long long gx = std::min(g, 1LL << 23), gy = (g + gx - 1) / gx;
  if (gy > 65535) return kCacheGrid;
  (void)hipGetLastError();
  const dim3 grid((unsigned)gx, (unsigned)gy), block(256);
  // (4 x 32 heads x 4,096 rows of 128, 268 MB of values: 58 -> 49 us)
  if (rows * 4 * D > kStreamBytes) hipLaunchKernelGGL((cache_read_kernel<D, true>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((cache_read_kernel<D, false>), grid, block, 0, s, p);
  return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace

int launch_cache_append(const CacheRows& p, int d, hipStream_t s) {
  return d == 64 ? launch_append<64>(p, s) : d == 96 ? launch_append<96>(p, s)
       : d == 128 ? launch_append<128>(p, s) : launch_append<256>(p, s);
}
int launch_cache_read(const CacheRows& p, int d, hipStream_t s) {
  return d == 64 ? launch_read<64>(p, s) : d == 96 ? launch_read<96>(p, s)
       : d == 128 ? launch_read<128>(p, s) : launch_read<256>(p, s);
}
int launch_cache_attn(const CacheParams& p, int d, hipStream_t s) {
  return d == 64 ? launch_attn<64>(p, s) : d == 96 ? launch_attn<96>(p, s)
       : d == 128 ? launch_attn<128>(p, s) : launch_attn<256>(p, s);
}
int launch_cache_evict(const CacheEvict& p, int d, hipStream_t s) {
  return d == 64 ? launch_evict<64>(p, s) : d == 96 ? launch_evict<96>(p, s)
       : d == 128 ? launch_evict<128>(p, s) : launch_evict<256>(p, s);
}

}  // namespace fabft
