// What the kernels of the attention over the cache share (attention_cached.hip, attention_cached_few.hip).
#pragma once
#include "cache.h"

namespace aqt {

struct CachedGeom {
  int64_t T, ld;            // new rows per stream, columns of a row
  int heads, group;         // query heads, and how many of them share a key / value head
  int row_tiles, splits;
  int64_t left, right;      // negative: no limit
  float scale_log2e;
};
// Wavefronts per SIMD that the kernel's registers are shared out to, with five spilled at most (packed heads of 128: no slower so) (dt: blocks of 16 head columns, r: rows).
constexpr int few_waves(int dt, bool packed, int r) { return dt == 8 ? (packed && r < 4 ? 3 : 2) : r > 1 && !packed ? 3 : 4; }
constexpr int kFewRows = 4;   // rows per key / value head and stream up to which attention_cached_few.hip takes the call
// part: the splits' rows, [rows][columns], then maxima and sums [rows] each, one after the other (nullptr: straight to ctx)
aqt_status launch_attention_cached_few(const float *qkv, const CacheGeom &g, const CachedGeom &a, const int32_t *count, float *ctx,
                                       uint32_t *absmax, float *part, hipStream_t st);

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr float kLowest = -3.402823466e38f;
constexpr float kDigits = 8355584.0f;     // 0x7F7F00: balanced digits of at most 0x7F7F7F, a rounding of the quotient allowed for
typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));

// Four integers of 24 bits, the digits of one weight each to a dword: d[0] the highest.
__device__ __forceinline__ void digits4(const int (&n)[4], int &d0, int &d1, int &d2) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = (static_cast<uint32_t>(n[i]) + 0x00808080u) ^ 0x00808080u;
  const uint32_t ab = __builtin_amdgcn_perm(u[1], u[0], 0x05010400u), cd = __builtin_amdgcn_perm(u[3], u[2], 0x05010400u);   // a0 b0 a1 b1
  const uint32_t at = __builtin_amdgcn_perm(u[1], u[0], 0x0C0C0602u), ct = __builtin_amdgcn_perm(u[3], u[2], 0x0C0C0602u);   // a2 b2
  d2 = static_cast<int>(__builtin_amdgcn_perm(cd, ab, 0x05040100u));
  d1 = static_cast<int>(__builtin_amdgcn_perm(cd, ab, 0x07060302u));
  d0 = static_cast<int>(__builtin_amdgcn_perm(ct, at, 0x05040100u));
}

// Whether a lane's 16 KS columns x of a row (from column 16 lg and 64 + 16 lg on, zeros behind dh) say that the row, whose largest column
// is `top`, loses by integers relative to that: eight of them (twelve of 32; half of 9 to 15; all others of 8 and less) lie under 1 / 64 of it.
// One in 25 of normally distributed columns does: it takes a row of 64 such columns once in three million (with six of them once in
// ten thousand: one call in two of 8192 rows over a long history then waited for a row that it had taken, 62 us for 50).
template <int KS>
__device__ __forceinline__ bool lane_is_wide(const float (&x)[KS][16], float top, int lg, int dh) {
  const float below = top * 0.015625f;
  int small = 0;
#pragma unroll
  for (int k = 0; k < KS; ++k) {
    small -= min(max(64 * k + 16 * lg + 16 - dh, 0), 16);
#pragma unroll
    for (int i = 0; i < 16; ++i) small += fabsf(x[k][i]) < below ? 1 : 0;
  }
  const int enough = KS == 2 ? 12 : dh <= 8 ? max(dh - 1, 1) : min((dh + 1) / 2, 8);
  return small >= enough && top < __builtin_inff();
}
// What a row's integers x `to` leave of it, in units of 2^-23 of theirs and again as digits (nothing of rows that are not wide: their
// scores are the same with and without).
__device__ __forceinline__ void rest_digits(const float (&x)[16], float to, bool wide, v4i (&d)[3]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    int n[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = x[4 * w + i];
      n[i] = wide ? static_cast<int>(rintf(fmaf(v, to, -rintf(v * to)) * 8388608.0f)) : 0;
    }
    int d0, d1, d2;
    digits4(n, d0, d1, d2);
    d[0][w] = d0;
    d[1][w] = d1;
    d[2][w] = d2;
  }
}
constexpr float kRestUnit = 1.0f / 8388608.0f;

// A weight of 0 .. 1 as an integer w of 23 bits: 0x808080 + w, as a float of the binade 2^23 .. 2^24, whose steps are ones; the
// sum rounds to nearest.  Its bytes are the balanced digits (the highest lacks the sign bit that the exponent's place took; the others
// are off by 128, i.e. by their highest bit).
__device__ __forceinline__ uint32_t weight_bits(float weight, float to) { return __float_as_uint(fmaf(weight, to, 8421504.0f)); }

// Four of them, a dword of each digit.
__device__ __forceinline__ void weight_digits4(const uint32_t (&u)[4], int &d0, int &d1, int &d2) {
  const uint32_t ab = __builtin_amdgcn_perm(u[1], u[0], 0x05010400u), cd = __builtin_amdgcn_perm(u[3], u[2], 0x05010400u);   // a0 b0 a1 b1
  const uint32_t at = __builtin_amdgcn_perm(u[1], u[0], 0x0C0C0602u), ct = __builtin_amdgcn_perm(u[3], u[2], 0x0C0C0602u);   // a2 b2
  d2 = static_cast<int>(__builtin_amdgcn_perm(cd, ab, 0x05040100u) ^ 0x80808080u);
  d1 = static_cast<int>(__builtin_amdgcn_perm(cd, ab, 0x07060302u) ^ 0x80808080u);
  d0 = static_cast<int>(__builtin_amdgcn_perm(ct, at, 0x05040100u));
}

__device__ __forceinline__ v4i mfma_i8(v4i a, v4i b, v4i c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }

// The three digits' sums as one number, 256^2 a + 256 b + c.
__device__ __forceinline__ float joined(int a, int b, int c) {
  return fmaf(static_cast<float>(a), 65536.0f, static_cast<float>(b * 256 + c));
}

__device__ __forceinline__ float max_of_groups(float v) {   // over the four lanes of a row
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}

// The rows, of 16, that have it in one of their four lanes.
__device__ __forceinline__ uint32_t rows_with(bool has) {
  uint64_t b = __ballot(has);
  b |= b >> 32;
  return static_cast<uint32_t>(b | b >> 16) & 0xFFFFu;
}

// Of a number that is not negative; a NaN stays one.
__device__ __forceinline__ float at_least_tiny(float v) { return __uint_as_float(max(__float_as_uint(v), 0x0D800000u)); }   // 2^-100

// The largest of a wavefront's 64 words.  (The steps fuse with the moves between lanes, as they do not for float32.)
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  auto step = [&](int w) { v = max(v, static_cast<uint32_t>(w)); };
  step(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x111, 0xF, 0xF, true));   // row_shr:1, 2, 4, 8: a row's last lane has its largest
  step(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x112, 0xF, 0xF, true));
  step(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x114, 0xF, 0xF, true));
  step(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x118, 0xF, 0xF, true));
  step(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x142, 0xA, 0xF, false));  // row_bcast:15 into rows 1 and 3, row_bcast:31 into 2 and 3
  step(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x143, 0xC, 0xF, false));
  return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), 63));
}
// Of floats: as they are where none is negative, otherwise as words in their order.
__device__ __forceinline__ float wave_max_positive(float v) { return __uint_as_float(wave_max(__float_as_uint(v))); }
__device__ __forceinline__ float wave_max_signed(float v) {
  const uint32_t u = __float_as_uint(v);
  const uint32_t w = wave_max(u ^ (static_cast<uint32_t>(static_cast<int>(u) >> 31) | 0x80000000u));
  return __uint_as_float(w ^ (w >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}

// Four columns of a row of ctx.
__device__ __forceinline__ uint32_t put_ctx(float *to, int col, int dh, v4f v) {
  uint32_t amax = 0u;
  const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (col + e < dh) {
      to[col + e] = x[e];
      amax = max(amax, __float_as_uint(x[e]) & 0x7FFFFFFFu);
    }
  return amax;
}
__device__ __forceinline__ void put_absmax(uint32_t *absmax, uint32_t amax) {   // the word only grows: a stale read can only cost an atomic
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) amax = max(amax, static_cast<uint32_t>(__shfl_xor(static_cast<int>(amax), off, 64)));
  if ((threadIdx.x & 63u) == 0 && amax > *reinterpret_cast<volatile uint32_t *>(absmax)) atomicMax(absmax, amax);
}

// What a workgroup leaves where several share the tiles: [rows][columns], then the rows' maxima and sums.
template <int ROWS, int COLS>
struct Partial {
  static constexpr int kMax = ROWS * COLS, kSum = kMax + ROWS, kFloats = (kSum + ROWS + 3) / 4 * 4;
};

}  // namespace
}  // namespace aqt
