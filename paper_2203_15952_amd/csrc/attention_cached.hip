// Attention of every stream's new frames over its quantized cache (cache.h), for each query head and new frame t:
//   score_j = (q . codes_j) s_j / sqrt(dh),   p = softmax over the frames j that the window admits and the cache holds,
//   ctx = sum_j p_j s'_j codes'_j          (s, s' the scales of the frame's key and value).
// The codes never become floats: both products run on the int8 matrix cores (v_mfma_i32_16x16x64_i8, exact 32-bit sums), and it
// is the float operand that is carried whole, as an integer of 24 bits relative to its row's largest, in three balanced
// base-256 digits, i.e. three int8 operands.  (A code turned into bf16 costs a vector instruction or two for every code of
// the cache; the digits of a query are made once, those of a probability once for all columns of the values.)  An integer
// rounded at 2^-24 of the largest is as good as a float32 sum over the row.
//
// A workgroup owns 16 rows (frame, query head) that share a key / value head, and its wavefronts take the tiles of 64 frames
// in turn, each with its own running maximum and sum, joined through LDS at the end; where that leaves the chip empty, several
// workgroups (splits) share the tiles and a second launch joins what they leave behind.  Both products are formed transposed,
// so that a lane's registers belong to one row:
//   S^T (64 frames x 16 rows) = K q^T     A operand: key rows as they lie in the cache; B operand: the digits of the rows
//   a lane (row lr = lane % 16, g = lane / 16) then holds the scores of the frames 16 t + 4 g + r of its row
//   O^T (dh x 16 rows) += V^T P^T         B operand: the digits of the lane's own probabilities, where they stand; A operand:
//                                         value rows, whose frames the cache keeps in that order
#include "cache.h"

namespace aqt {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kRows = 16;                 // rows of a workgroup
constexpr float kLowest = -3.402823466e38f;
constexpr float kDigits = 8355584.0f;     // 0x7F7F00: balanced digits of at most 0x7F7F7F, a rounding of the quotient allowed for
typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));

struct CachedGeom {
  int64_t T, ld;            // new rows per stream, columns of a row
  int heads, group;         // query heads, and how many of them share a key / value head
  int row_tiles, splits;
  int64_t left, right;      // negative: no limit
  float scale_log2e;
};

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

__device__ __forceinline__ v4i mfma_i8(v4i a, v4i b, v4i c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }

// The three digits' sums as one number, 256^2 a + 256 b + c.
__device__ __forceinline__ float joined(int a, int b, int c) {
  return fmaf(static_cast<float>(a), 65536.0f, static_cast<float>(b * 256 + c));
}

__device__ __forceinline__ float max_of_groups(float v) {   // over the four lanes of a row
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}

// What a workgroup leaves: the rows' running maxima and sums, and their sums of values.
template <int COLS>
struct Partial {
  static constexpr int kMax = 0, kSum = kRows, kOut = 2 * kRows, kFloats = kOut + kRows * COLS;
};

// The rows of a workgroup or of its joined parts leave as ctx; thread (row = tid / 16, columns 4 (tid % 16) + 64 k).
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

// DT: blocks of 16 head columns that a workgroup holds (2, 4 or 8)
template <int DT, bool PACKED>
__global__ __launch_bounds__(kThreads, 2) void attention_cached_kernel(const float *__restrict__ qkv, CacheGeom g, CachedGeom a,
                                                                       const int32_t *__restrict__ count, float *__restrict__ ctx,
                                                                       uint32_t *__restrict__ absmax, float *__restrict__ part) {
  constexpr int KS = DT == 8 ? 2 : 1;        // steps of 64 head columns
  constexpr int COLS = 16 * DT, LD = COLS + 4;
  __shared__ __attribute__((aligned(16))) float so[kWaves][kRows][LD];
  __shared__ float sm[kWaves][kRows], sl[kWaves][kRows];
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int64_t id = blockIdx.x;
  const int split = static_cast<int>(id % a.splits);
  id /= a.splits;
  const int rt = static_cast<int>(id % a.row_tiles);
  id /= a.row_tiles;
  const int h = static_cast<int>(id % g.kv_heads);
  const int64_t b = id / g.kv_heads;
  const StreamFrames f = stream_frames(g, count, a.T, b);
  const int n = static_cast<int>(f.end - f.length);
  const int t_first = rt * kRows / a.group;
  if (t_first >= n) return;                  // frames that the stream did not bring: their rows stay as they are
  const int t_last = min((rt * kRows + kRows - 1) / a.group, n - 1);

  // the frames that the workgroup's rows see, and this lane's row; counted from the first tile
  auto from = [&](int t) { const int64_t x = f.length + t - a.left; return a.left < 0 || x < f.oldest ? f.oldest : x; };
  auto upto = [&](int t) { const int64_t x = f.length + t + a.right; return a.right < 0 || x > f.end - 1 ? f.end - 1 : x; };
  const int64_t first = from(t_first), last = upto(t_last), tile0 = first >> 6, base = tile0 * 64;
  const int tiles = last < first ? 0 : static_cast<int>((last >> 6) - tile0) + 1;
  const int row = rt * kRows + lr, t_own = min(row / a.group, n - 1);   // rows behind the last repeat it and are not stored
  const int lo = static_cast<int>(from(t_own) - base), hi = static_cast<int>(upto(t_own) - base);
  const int all_lo = static_cast<int>(from(t_last) - base), all_hi = static_cast<int>(upto(t_first) - base);

  // the row's digits: 16 columns per lane and step
  v4i q[KS][3];
  float row_scale;
  {
    const float *const src = qkv + (b * a.T + t_own) * a.ld + (static_cast<int64_t>(h) * a.group + row % a.group) * g.dh;
    float x[KS][16];
    uint32_t m = 0u;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = 64 * k + 16 * lg + i;
        x[k][i] = src[min(c, g.dh - 1)];
        x[k][i] = c < g.dh ? x[k][i] : 0.0f;
        m = max(m, __float_as_uint(x[k][i]) & 0x7FFFFFFFu);
      }
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16, 64)));
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32, 64)));
    const float top = __uint_as_float(m);    // a NaN or an infinity makes the row's scores NaN
    const float to = kDigits / fmaxf(top, 0x1p-100f);
    row_scale = (m > 0x7F800000u ? top : fmaxf(top, 0x1p-100f)) * (1.0f / kDigits) * a.scale_log2e * (PACKED ? 0.0625f : 1.0f);
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        int nn[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) nn[i] = static_cast<int>(rintf(x[k][4 * w + i] * to));
        int d0, d1, d2;
        digits4(nn, d0, d1, d2);
        q[k][0][w] = d0;
        q[k][1][w] = d1;
        q[k][2][w] = d2;
      }
  }

  const uint8_t *const head = g.data + (b * g.kv_heads + h) * g.tiles * static_cast<int64_t>(g.tile_bytes);
  const int step = a.splits * kWaves, slot_step = step % g.tiles;
  float m = kLowest, l = 0.0f;
  v4f o[DT];                                 // element r of block d: column 16 d + 4 lg + r of this lane's row
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  int i = split * kWaves + wave;
  int slot = tile_slot(tile0 + i, g.tiles);
  for (; i < tiles; i += step) {
    const uint8_t *const tile = head + static_cast<int64_t>(slot) * g.tile_bytes;
    slot += slot_step;
    slot = slot >= g.tiles ? slot - g.tiles : slot;
    const float *const scales = reinterpret_cast<const float *>(tile + cache_scales(g));
    // scores
    float s[16];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      v4i c[3];
#pragma unroll
      for (int d = 0; d < 3; ++d) c[d] = v4i{0, 0, 0, 0};
      const uint8_t *const key = tile + (16 * t + lr) * g.key_row;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        v4i w;
        if (PACKED) {   // sixteen columns in eight bytes; a lane beyond the row meets digits of zero
          const int at = 32 * k + 8 * lg;
          const v2i x = *reinterpret_cast<const v2i *>(key + (at < g.key_row ? at : 0));
          w = v4i{static_cast<int>(static_cast<uint32_t>(x.x) << 4 & 0xF0F0F0F0u), static_cast<int>(static_cast<uint32_t>(x.y) << 4 & 0xF0F0F0F0u),
                  static_cast<int>(static_cast<uint32_t>(x.x) & 0xF0F0F0F0u), static_cast<int>(static_cast<uint32_t>(x.y) & 0xF0F0F0F0u)};
        } else {
          const int at = 64 * k + 16 * lg;
          w = *reinterpret_cast<const v4i *>(key + (at < g.key_row ? at : 0));
        }
#pragma unroll
        for (int d = 0; d < 3; ++d) c[d] = mfma_i8(w, q[k][d], c[d]);
      }
      const v4f ks = *reinterpret_cast<const v4f *>(scales + 16 * t + 4 * lg);
      const float kse[4] = {ks.x, ks.y, ks.z, ks.w};
#pragma unroll
      for (int r = 0; r < 4; ++r) s[4 * t + r] = joined(c[0][r], c[1][r], c[2][r]) * (row_scale * kse[r]);
    }
    // window: what it hides, and what is no frame of the stream's, may hold anything
    const int j0 = 64 * i;
    uint32_t seen = 0xFFFFu;
    if (j0 < all_lo || j0 + 63 > all_hi) {
      seen = 0u;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int j = j0 + 16 * (e >> 2) + 4 * lg + (e & 3);
        seen |= (j >= lo && j <= hi ? 1u : 0u) << e;
      }
    }
    float mx = kLowest;
#pragma unroll
    for (int e = 0; e < 16; ++e) mx = fmaxf(mx, seen >> e & 1u ? s[e] : kLowest);
    mx = max_of_groups(mx);
    const float mnew = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - mnew);
    m = mnew;
    l *= alpha;
    // probabilities, times the values' scales, and their digits
    float top = 0.0f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const v4f vs = *reinterpret_cast<const v4f *>(scales + 64 + 16 * t + 4 * lg);
      const float vse[4] = {vs.x, vs.y, vs.z, vs.w};
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int e = 4 * t + r;
        const bool see = seen >> e & 1u;
        const float p = see ? __builtin_amdgcn_exp2f(s[e] - m) : 0.0f;
        l += p;
        s[e] = see ? p * vse[r] : 0.0f;
        top = fmaxf(top, s[e]);
      }
    }
    top = fmaxf(max_of_groups(top), 0x1p-100f);
    const float to = kDigits / top;
    v4i p[3];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      int nn[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) nn[r] = static_cast<int>(rintf(s[4 * t + r] * to));
      int d0, d1, d2;
      digits4(nn, d0, d1, d2);
      p[0][t] = d0;
      p[1][t] = d1;
      p[2][t] = d2;
    }
    const float unit = top * (1.0f / kDigits) * (PACKED ? 0.0625f : 1.0f);
    const uint8_t *const values = tile + cache_values(g) + 16 * lg;
    auto add = [&](v4f &to_o, v4i w) {
      v4i c[3];
#pragma unroll
      for (int d = 0; d < 3; ++d) c[d] = mfma_i8(w, p[d], v4i{0, 0, 0, 0});
#pragma unroll
      for (int r = 0; r < 4; ++r) to_o[r] = fmaf(joined(c[0][r], c[1][r], c[2][r]), unit, to_o[r] * alpha);
    };
#pragma unroll
    for (int d = 0; d < DT; d += PACKED ? 2 : 1) {
      const int at = 16 * (PACKED ? d / 2 : d) + lr;
      const v4i x = *reinterpret_cast<const v4i *>(values + (at < g.value_rows ? at : lr) * 64);   // columns beyond the head are not stored
      if (PACKED) {
        v4i lo4, hi4;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo4[e] = static_cast<int>(static_cast<uint32_t>(x[e]) << 4 & 0xF0F0F0F0u);
          hi4[e] = static_cast<int>(static_cast<uint32_t>(x[e]) & 0xF0F0F0F0u);
        }
        add(o[d], lo4);
        add(o[d + 1], hi4);
      } else {
        add(o[d], x);
      }
    }
  }

  // the wavefronts' parts of the rows
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (lg == 0) {
    sm[wave][lr] = m;
    sl[wave][lr] = l;
  }
#pragma unroll
  for (int d = 0; d < DT; ++d) *reinterpret_cast<v4f *>(&so[wave][lr][16 * d + 4 * lg]) = o[d];
  __syncthreads();
  const int orow = tid >> 4;
  float top = kLowest, sum = 0.0f, weight[kWaves];
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm[w][orow]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    weight[w] = __builtin_amdgcn_exp2f(sm[w][orow] - top);
    sum = fmaf(sl[w][orow], weight[w], sum);
  }
  const int out_row = rt * kRows + orow, t = out_row / a.group;
  const bool store = t < n;
  float *const to = ctx + ((b * a.T + t) * a.heads + h * a.group + out_row % a.group) * g.dh;
  float *const left = part ? part + static_cast<int64_t>(blockIdx.x) * Partial<COLS>::kFloats : nullptr;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;   // nothing seen: zeros
  uint32_t amax = 0u;
#pragma unroll
  for (int c = 4 * (tid & 15); c < COLS; c += 64) {
    v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const v4f x = *reinterpret_cast<const v4f *>(&so[w][orow][c]);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(x[e], weight[w], v[e]);
    }
    if (left) {
      *reinterpret_cast<v4f *>(left + Partial<COLS>::kOut + orow * COLS + c) = v;
    } else if (store) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= inv;
      amax = max(amax, put_ctx(to, c, g.dh, v));
    }
  }
  if (left) {
    if ((tid & 15) == 0) {
      left[Partial<COLS>::kMax + orow] = top;
      left[Partial<COLS>::kSum + orow] = sum;
    }
  } else if (absmax) {
    put_absmax(absmax, amax);
  }
}

// The splits' parts of 16 rows, in their order.
template <int COLS>
__global__ __launch_bounds__(kThreads) void attention_cached_join_kernel(const float *__restrict__ part, CacheGeom g, CachedGeom a,
                                                                         const int32_t *__restrict__ count, float *__restrict__ ctx,
                                                                         uint32_t *__restrict__ absmax) {
  constexpr int F = Partial<COLS>::kFloats;
  const int tid = static_cast<int>(threadIdx.x), orow = tid >> 4;
  int64_t id = blockIdx.x;
  const float *const from = part + id * a.splits * F;
  const int rt = static_cast<int>(id % a.row_tiles);
  id /= a.row_tiles;
  const int h = static_cast<int>(id % g.kv_heads);
  const int64_t b = id / g.kv_heads;
  const StreamFrames f = stream_frames(g, count, a.T, b);
  const int n = static_cast<int>(f.end - f.length);
  if (rt * kRows / a.group >= n) return;   // its parts were not written
  const int out_row = rt * kRows + orow, t = out_row / a.group;
  float top = kLowest, sum = 0.0f;
  for (int s = 0; s < a.splits; ++s) top = fmaxf(top, from[static_cast<int64_t>(s) * F + Partial<COLS>::kMax + orow]);
  constexpr int N = (COLS + 63) / 64;
  v4f v[N];
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  const int c0 = 4 * (tid & 15);
#pragma unroll 4
  for (int s = 0; s < a.splits; ++s) {
    const float *const p = from + static_cast<int64_t>(s) * F;
    const float w = __builtin_amdgcn_exp2f(p[Partial<COLS>::kMax + orow] - top);
    sum = fmaf(p[Partial<COLS>::kSum + orow], w, sum);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int c = c0 + 64 * k < COLS ? c0 + 64 * k : 0;
      const v4f x = *reinterpret_cast<const v4f *>(p + Partial<COLS>::kOut + orow * COLS + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[k][e] = fmaf(x[e], w, v[k][e]);
    }
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint32_t amax = 0u;
  if (t < n) {
    float *const to = ctx + ((b * a.T + t) * a.heads + h * a.group + out_row % a.group) * g.dh;
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[k][e] *= inv;
      if (c0 + 64 * k < COLS) amax = max(amax, put_ctx(to, c0 + 64 * k, g.dh, v[k]));
    }
  }
  if (absmax) put_absmax(absmax, amax);
}

__global__ void zero_word_kernel(uint32_t *p) {
  if (threadIdx.x == 0) *p = 0u;
}

int cols_of(int dh) { return dh <= 32 ? 32 : dh <= 64 ? 64 : 128; }

// Workgroups that share the tiles of 16 rows.  Two thousand wavefronts keep every SIMD busy with two; a split takes at least one
// tile per wavefront.  `window`: the longest run of frames that a row tile sees.
int splits_of(const CacheGeom &g, int64_t row_tiles, int64_t window) {
  const int64_t groups = g.streams * g.kv_heads * row_tiles, tiles = cdiv(window, 64) + 1;
  const int64_t want = cdiv(1024, groups), most = cdiv(tiles, kWaves);
  const int64_t s = want < most ? want : most;
  return static_cast<int>(s < 1 ? 1 : s);
}

}  // namespace

bool cached_attention_ok(const aqt_cache &c, int64_t T, int heads) {
  if (T > (int64_t(1) << 24)) return false;
  const int64_t row_tiles = cdiv(T * (heads / c.kv_heads), kRows);
  return row_tiles * kRows <= (int64_t(1) << 30) && row_tiles * c.kv_heads <= (int64_t(1) << 30) / c.streams;
}

size_t cached_attention_ws_bytes(const aqt_cache &c, int64_t T, int heads) {
  const CacheGeom g = cache_geom(c);
  const int64_t row_tiles = cdiv(T * (heads / c.kv_heads), kRows);
  const int splits = splits_of(g, row_tiles, c.capacity);
  const size_t floats = 2 * kRows + static_cast<size_t>(kRows) * cols_of(c.dh);
  return splits == 1 ? 256 : align_up(static_cast<size_t>(splits) * g.streams * g.kv_heads * row_tiles * floats * sizeof(float), 256);
}

aqt_status launch_attention_cached(const float *qkv, int64_t T, int heads, const aqt_cache &c, const int32_t *count, int left, int right,
                                   float *ctx, uint32_t *absmax, void *ws, hipStream_t st) {
  const CacheGeom g = cache_geom(c);
  CachedGeom a;
  a.T = T;
  a.heads = heads;
  a.group = heads / c.kv_heads;
  a.ld = (static_cast<int64_t>(heads) + 2 * static_cast<int64_t>(c.kv_heads)) * c.dh;
  a.row_tiles = static_cast<int>(cdiv(T * a.group, kRows));
  a.left = left;
  a.right = right;
  a.scale_log2e = static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(c.dh)));
  // 16 rows span at most that many frames, and a window on either side of them
  const int64_t span = cdiv(kRows, a.group) + 1, window = left < 0 ? c.capacity : span + left + (right < 0 ? T : right);
  a.splits = splits_of(g, a.row_tiles, window < c.capacity ? window : c.capacity);
  if (absmax) {
    zero_word_kernel<<<1, 64, 0, st>>>(absmax);
    AQT_HIP(hipGetLastError());
  }
  const int64_t groups = g.streams * g.kv_heads * a.row_tiles;
  float *const part = a.splits > 1 ? static_cast<float *>(ws) : nullptr;
  auto kern = g.packed ? (c.dh <= 32   ? attention_cached_kernel<2, true>
                          : c.dh <= 64 ? attention_cached_kernel<4, true>
                                       : attention_cached_kernel<8, true>)
                       : (c.dh <= 32   ? attention_cached_kernel<2, false>
                          : c.dh <= 64 ? attention_cached_kernel<4, false>
                                       : attention_cached_kernel<8, false>);
  kern<<<static_cast<unsigned>(groups * a.splits), kThreads, 0, st>>>(qkv, g, a, count, ctx, absmax, part);
  AQT_HIP(hipGetLastError());
  if (!part) return AQT_OK;
  auto join = c.dh <= 32 ? attention_cached_join_kernel<32> : c.dh <= 64 ? attention_cached_join_kernel<64> : attention_cached_join_kernel<128>;
  join<<<static_cast<unsigned>(groups), kThreads, 0, st>>>(part, g, a, count, ctx, absmax);
  AQT_HIP(hipGetLastError());
  return AQT_OK;
}

}  // namespace aqt
