// Attention of every stream's new frames over its quantized cache (cache.h), for each query head and new frame t:
//   score_j = (q . codes_j) s_j / sqrt(dh),   p = softmax over the frames j that the window admits and the cache holds,
//   ctx = sum_j p_j s'_j codes'_j          (s, s' the scales of the frame's key and value).
// The codes never become floats: both products run on the int8 matrix cores (v_mfma_i32_16x16x64_i8, exact 32-bit sums), and it
// is the float operand that becomes an integer of 24 bits, in three balanced base-256 digits, i.e. three int8 operands.  (A code
// turned into bf16 costs a vector instruction or two for every code of the cache; the digits of a query are made once, those of a
// weight once for all columns of the values.)
// What is rounded, and to what: a query's columns to 2^-24 of the row's largest column, as good as a float32 sum where that is like
// the others.  Where a column stands out of its row it may meet keys of zero, and would leave the others the bits that it has not
// taken (r times their size, r = 64, 1000, 10^6: errors of the result of 2e-6, 4e-5, 4e-2): the integers of such rows (lane_is_wide)
// are followed by 23 bits more, whose products a branch that all other tiles step over adds to the scores.  A frame's weight p_j s'_j
// is rounded to 2^-24 .. 2^-22 of the largest of its tile: relative to sum_j p_j max|v_j| a float32 sum's error or less, but not
// column by column: where the frame with the weight has a value of zero in a column, and a large one in another, the other frames'
// values in that column keep the bits that are left.  (Codes are off by 2^-8 and more of a value's largest column anyway.)
//
// A workgroup owns 16 rows (frame, query head) that share a key / value head, and its wavefronts take the tiles of 64 frames
// in turn, each with its own running maximum and sum, joined through LDS at the end; where that leaves the chip empty, several
// workgroups (splits) share the tiles and a second launch joins what they leave behind.  Where row tiles are many, every wavefront has
// one to itself.  Both products are formed transposed,
// so that a lane's registers belong to one row:
//   S^T (64 frames x 16 rows) = K q^T     A operand: key rows as they lie in the cache; B operand: the digits of the rows
//   a lane (row lr = lane % 16, g = lane / 16) then holds the scores of the frames 16 t + 4 g + r of its row
//   O^T (dh x 16 rows) += V^T P^T         B operand: the digits of the lane's own probabilities, where they stand; A operand:
//                                         value rows, whose frames the cache keeps in that order
#include "attention_cached.h"

namespace aqt {
namespace {

constexpr int kRows = 16;                 // rows of a workgroup
// Wavefronts per SIMD that the kernel's registers are shared out to, without spills (dt: blocks of 16 head columns).
constexpr int many_waves(int dt, bool packed) { return dt == 8 ? 2 : dt == 2 || packed ? 4 : 3; }
// A row tile to a wavefront: fewer bytes of LDS, and three registers spilled for packed heads of 128 (8192 row tiles of 128 int4 columns over 3 tiles: 95 us with two wavefronts, 90 so).
constexpr int own_waves(int dt, bool packed) { return dt == 8 && packed ? 3 : many_waves(dt, packed); }

// The workgroup's place: (stream and head, row tile, split).  The row tiles of a split read the same codes; workgroup ids eight apart run
// on one XCD, so that with a multiple of eight of them the row tiles of a split are given to one XCD's L2.
struct Place {
  int bh, rt, split;
};
template <bool OWN>
__device__ __forceinline__ Place place_of(const CachedGeom &a, int64_t heads, int wave) {
  const int id = OWN ? static_cast<int>(blockIdx.x) * kWaves + wave : static_cast<int>(blockIdx.x);
  if constexpr (OWN) return Place{id / a.row_tiles, id % a.row_tiles, 0};
  const int64_t lanes = heads * a.splits;   // of row tiles
  int lane, rt;
  if (lanes % 8 == 0) {
    lane = id / (8 * a.row_tiles) * 8 + id % 8;
    rt = id / 8 % a.row_tiles;
  } else {
    lane = id / a.row_tiles;
    rt = id % a.row_tiles;
  }
  return Place{lane / a.splits, rt, lane % a.splits};
}

// DT: blocks of 16 head columns that a workgroup holds (2, 4 or 8); OWN: every wavefront has a row tile to itself (splits is 1 then)
template <int DT, bool PACKED, bool OWN>
__global__ __launch_bounds__(kThreads, OWN ? own_waves(DT, PACKED) : many_waves(DT, PACKED)) void attention_cached_kernel(const float *__restrict__ qkv, CacheGeom g, CachedGeom a,
                                                                       const int32_t *__restrict__ count, float *__restrict__ ctx,
                                                                       uint32_t *__restrict__ absmax, float *__restrict__ part) {
  constexpr int KS = DT == 8 ? 2 : 1;        // steps of 64 head columns
  constexpr int COLS = 16 * DT, LD = COLS + 4;
  constexpr int KEYS = PACKED ? 2 : 4, VALUES = PACKED ? DT / 2 : DT;
  using P = Partial<kRows, COLS>;
  __shared__ __attribute__((aligned(16))) float so[kWaves][kRows][LD];
  __shared__ __attribute__((aligned(16))) float scales[kWaves][128];
  __shared__ __attribute__((aligned(16))) int rest[kWaves][KS][3][64][4];   // of rows whose integers do not hold them
  __shared__ float sm[kWaves][kRows], sl[kWaves][kRows];
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Place pl = place_of<OWN>(a, g.streams * g.kv_heads, wave);
  if (OWN && pl.bh >= g.streams * g.kv_heads) return;
  const int h = pl.bh % g.kv_heads;
  const int64_t b = pl.bh / g.kv_heads;
  const StreamFrames f = stream_frames(g, count, a.T, b);
  const int n = static_cast<int>(f.end - f.length);
  const int row0 = pl.rt * kRows, t_first = row0 / a.group;
  if (t_first >= n) return;                  // frames that the stream did not bring: their rows stay as they are
  const int t_last = min((row0 + kRows - 1) / a.group, n - 1);

  // the frames that the workgroup's rows see, and this lane's rows; counted from the first tile
  auto from = [&](int t) { const int64_t x = f.length + t - a.left; return a.left < 0 || x < f.oldest ? f.oldest : x; };
  auto upto = [&](int t) { const int64_t x = f.length + t + a.right; return a.right < 0 || x > f.end - 1 ? f.end - 1 : x; };
  const int64_t first = from(t_first), last = upto(t_last), tile0 = first >> 6, base = tile0 * 64;
  const int tiles = last < first ? 0 : static_cast<int>((last >> 6) - tile0) + 1;
  const int first_seen = static_cast<int>(first - base), last_seen = static_cast<int>(last - base);
  const int all_lo = static_cast<int>(from(t_last) - base), all_hi = static_cast<int>(upto(t_first) - base);

  // the rows: 16 columns per lane and step, requested in front of the first tile, so that their digits are formed under its trip from memory
  const int row = row0 + lr, t_own = min(row / a.group, n - 1);   // rows behind the last repeat it and are not stored
  const int lo = static_cast<int>(from(t_own) - base), hi = static_cast<int>(upto(t_own) - base);
  float x[KS][16];
  {
    const float *const src = qkv + (b * a.T + t_own) * a.ld + (static_cast<int64_t>(h) * a.group + row % a.group) * g.dh;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[k][i] = src[min(64 * k + 16 * lg + i, g.dh - 1)];
  }

  // A tile's codes and scales are requested where the tile before has given up their registers: the keys' trip from memory passes
  // under the rest of that tile, the values' under this one's scores (8 streams of 128 rows: 60 us with both at the head of a tile, 57 so).
  typedef int key_piece __attribute__((ext_vector_type(KEYS)));
  key_piece keys[4][KS];
  v4i values[VALUES];
  float ks_next, vs_next;
  auto key_of = [&](const uint8_t *tile, int t, int k) {   // sixteen columns to a lane; one beyond the row meets digits of zero
    const int at = (64 * k + 16 * lg) * KEYS / 4;
    return *reinterpret_cast<const key_piece *>(tile + (16 * t + lr) * g.key_row + (at < g.key_row ? at : 0));
  };
  auto load_keys = [&](const uint8_t *tile) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int k = 0; k < KS; ++k) keys[t][k] = key_of(tile, t, k);
    ks_next = reinterpret_cast<const float *>(tile + cache_scales(g))[lane];
    vs_next = reinterpret_cast<const float *>(tile + cache_scales(g))[64 + lane];
  };
  auto load_values = [&](const uint8_t *tile) {
#pragma unroll
    for (int d = 0; d < VALUES; ++d) {
      const int at = 16 * d + lr;      // columns beyond the head are not stored
      values[d] = *reinterpret_cast<const v4i *>(tile + cache_values(g) + (at < g.value_rows ? at : lr) * 64 + 16 * lg);
    }
  };

  const uint8_t *const head = g.data + (b * g.kv_heads + h) * g.tiles * static_cast<int64_t>(g.tile_bytes);
  const int step = OWN ? 1 : a.splits * kWaves, slot_step = step % g.tiles;
  float m = kLowest, l = 0.0f;
  v4f o[DT];                                 // element r of block d: column 16 d + 4 lg + r of this lane's row
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  int i = OWN ? 0 : pl.split * kWaves + wave;
  int slot = tile_slot(tile0 + i, g.tiles);
  if (i < tiles) {
    const uint8_t *const tile = head + static_cast<int64_t>(slot) * g.tile_bytes;
    load_keys(tile);
    load_values(tile);
  }
  // their digits
  v4i q[KS][3];
  float row_scale;
  bool wide;
  {
    uint32_t m = 0u;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[k][i] = 64 * k + 16 * lg + i < g.dh ? x[k][i] : 0.0f;
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
    const uint32_t wide_rows = rows_with(lane_is_wide<KS>(x, top, lg, g.dh));
    wide = wide_rows != 0u;
    if (wide) {
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        v4i d[3];
        rest_digits(x[k], to, wide_rows >> lr & 1u, d);
#pragma unroll
        for (int e = 0; e < 3; ++e) *reinterpret_cast<v4i *>(rest[wave][k][e][lane]) = d[e];
      }
      wave_lds_order();
    }
  }
  auto codes = [&](key_piece x) {
    if constexpr (PACKED) {
      const uint32_t lo8 = static_cast<uint32_t>(x[0]), hi8 = static_cast<uint32_t>(x[1]);
      return v4i{static_cast<int>(lo8 << 4 & 0xF0F0F0F0u), static_cast<int>(hi8 << 4 & 0xF0F0F0F0u), static_cast<int>(lo8 & 0xF0F0F0F0u),
                 static_cast<int>(hi8 & 0xF0F0F0F0u)};
    } else {
      return x;
    }
  };

  for (; i < tiles; i += step) {
    const uint8_t *const tile = head + static_cast<int64_t>(slot) * g.tile_bytes;
    if (i + step < tiles) {   // otherwise this tile's once more: never another's memory
      slot += slot_step;
      slot = slot >= g.tiles ? slot - g.tiles : slot;
    }
    const uint8_t *const next = head + static_cast<int64_t>(slot) * g.tile_bytes;
    const int j0 = 64 * i;
    const bool whole = j0 >= all_lo && j0 + 63 <= all_hi;
    // the frames' scales go round through LDS: a lane's frames are 16 t + 4 lg + r
    float *const sc = scales[wave];
    const float vs = j0 + lane >= first_seen && j0 + lane <= last_seen ? vs_next : 0.0f;   // others may hold anything
    sc[lane] = ks_next;
    sc[64 + lane] = vs;
    const float vs_top = wave_max_positive(vs);
    wave_lds_order();
    v4i p[3];
    float unit;
    {
      // scores
      float s[16];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        v4i c[3];
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const v4i w = codes(keys[t][k]);
#pragma unroll
          for (int d = 0; d < 3; ++d) c[d] = mfma_i8(w, q[k][d], k == 0 ? v4i{0, 0, 0, 0} : c[d]);
        }
        const v4f ks = *reinterpret_cast<const v4f *>(&sc[16 * t + 4 * lg]);
#pragma unroll
        for (int r = 0; r < 4; ++r) s[4 * t + r] = joined(c[0][r], c[1][r], c[2][r]) * (ks[r] * row_scale);   // (the sum, up to 2^37, by the small factor)
      }
      load_keys(next);
      if (wide) {   // the digits behind those (few rows have any, so that the tile's keys are read again)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int d = 0; d < 3; ++d) {
            v4i c = {0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < KS; ++k) c = mfma_i8(codes(key_of(tile, t, k)), *reinterpret_cast<const v4i *>(rest[wave][k][d][lane]), c);
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[r] = fmaf(sum[r], 256.0f, static_cast<float>(c[r]));
          }
          const v4f ks = *reinterpret_cast<const v4f *>(&sc[16 * t + 4 * lg]);
#pragma unroll
          for (int r = 0; r < 4; ++r) s[4 * t + r] = fmaf(sum[r], ks[r] * row_scale * kRestUnit, s[4 * t + r]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (!whole) {   // what the window hides, and what is no frame of the stream's, may hold anything
        asm volatile("");   // a branch: as selections they would be taken in every tile
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = j0 + 16 * (e >> 2) + 4 * lg + (e & 3);
          s[e] = j >= lo && j <= hi ? s[e] : -__builtin_inff();
        }
      }
      float mx = kLowest;
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
      mx = max_of_groups(mx);
      if (__any(mx > m)) {
        const float mnew = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - mnew);
        m = mnew;
        l *= alpha;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[d][r] *= alpha;
      }
      // Probabilities, and weights: probabilities times the values' scales.  The weights' digits are relative to the largest probability
      // times the largest scale, a bound of the largest weight; where a row's weights all lie under a quarter of it (most of the
      // probability meets a small value, or the large value is not the row's to see), to the row's largest weight itself, which takes
      // moves between lanes.  So the largest of a row and tile is an integer of 2^21 at least.  (32 streams, 512 new
      // frames and no others, 8 heads of 64, int8: 68.5 us without the look at the weights, 72 so; other forms and sizes: equal.)
      float most = 0.0f;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const v4f vs4 = *reinterpret_cast<const v4f *>(&sc[64 + 16 * t + 4 * lg]);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float e = __builtin_amdgcn_exp2f(s[4 * t + r] - m);
          l += e;
          s[4 * t + r] = e * vs4[r];
          most = fmaxf(most, s[4 * t + r]);
        }
      }
      float top = __builtin_amdgcn_exp2f(mx - m) * vs_top;
      const uint32_t near = rows_with(most >= 0.25f * top);
      if (near != 0xFFFFu) {   // ... and where a scale is NaN: what a row does not see is nothing to it
        uint32_t own = 0u;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = j0 + 16 * (e >> 2) + 4 * lg + (e & 3);
          s[e] = j >= lo && j <= hi ? s[e] : 0.0f;
          own = max(own, __float_as_uint(s[e]) & 0x7FFFFFFFu);
        }
        own = max(own, static_cast<uint32_t>(__shfl_xor(static_cast<int>(own), 16, 64)));
        own = max(own, static_cast<uint32_t>(__shfl_xor(static_cast<int>(own), 32, 64)));
        top = near >> lr & 1u ? top : __uint_as_float(own);   // a row's own affair, whatever the others do
      }
      top = at_least_tiny(top);
      const float to = kDigits * __builtin_amdgcn_rcpf(top);
      unit = top * (1.0f / kDigits) * (PACKED ? 0.0625f : 1.0f);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        uint32_t w[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) w[r] = weight_bits(s[4 * t + r], to);
        int d0, d1, d2;
        weight_digits4(w, d0, d1, d2);
        p[0][t] = d0;
        p[1][t] = d1;
        p[2][t] = d2;
      }
    }
    wave_lds_order();   // the scales are read before the next tile's are written
    auto add = [&](int d, v4i w) {
      v4i c[3];
#pragma unroll
      for (int e = 0; e < 3; ++e) c[e] = mfma_i8(w, p[e], v4i{0, 0, 0, 0});
#pragma unroll
      for (int r = 0; r < 4; ++r) o[d][r] = fmaf(joined(c[0][r], c[1][r], c[2][r]), unit, o[d][r]);
    };
#pragma unroll
    for (int d = 0; d < VALUES; ++d) {
      if constexpr (PACKED) {
        v4i lo4, hi4;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          lo4[e] = static_cast<int>(static_cast<uint32_t>(values[d][e]) << 4 & 0xF0F0F0F0u);
          hi4[e] = static_cast<int>(static_cast<uint32_t>(values[d][e]) & 0xF0F0F0F0u);
        }
        add(2 * d, lo4);
        add(2 * d + 1, hi4);
      } else {
        add(d, values[d]);
      }
    }
    load_values(next);
  }

  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  uint32_t amax = 0u;
  if constexpr (OWN) {
    const int t = row / a.group;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // nothing seen: zeros
    float *const to = ctx + ((b * a.T + t) * a.heads + h * a.group + row % a.group) * g.dh;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
#pragma unroll
      for (int r = 0; r < 4; ++r) o[d][r] *= inv;
      if (t < n) amax = max(amax, put_ctx(to, 16 * d + 4 * lg, g.dh, o[d]));
    }
    if (absmax) put_absmax(absmax, amax);
    return;
  }
  // the wavefronts' parts of the rows
  if (lg == 0) {
    sm[wave][lr] = m;
    sl[wave][lr] = l;
  }
#pragma unroll
  for (int d = 0; d < DT; ++d) *reinterpret_cast<v4f *>(&so[wave][lr][16 * d + 4 * lg]) = o[d];
  __syncthreads();
  float *const left = part ? part + ((static_cast<int64_t>(pl.bh) * a.row_tiles + pl.rt) * a.splits + pl.split) * P::kFloats : nullptr;
  const int orow = tid >> 4;
  float top = kLowest, sum = 0.0f, weight[kWaves];
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm[w][orow]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    weight[w] = __builtin_amdgcn_exp2f(sm[w][orow] - top);
    sum = fmaf(sl[w][orow], weight[w], sum);
  }
  const int out_row = row0 + orow, t = out_row / a.group;
  float *const to = ctx + ((b * a.T + t) * a.heads + h * a.group + out_row % a.group) * g.dh;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;   // nothing seen: zeros
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
      *reinterpret_cast<v4f *>(left + orow * COLS + c) = v;
    } else if (t < n) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= inv;
      amax = max(amax, put_ctx(to, c, g.dh, v));
    }
  }
  if (left) {
    if ((tid & 15) == 0) {
      left[P::kMax + orow] = top;
      left[P::kSum + orow] = sum;
    }
  } else if (absmax) {
    put_absmax(absmax, amax);
  }
}

// The splits' parts of a workgroup's rows.  Threads in as many slices as there are for the rows' columns, four columns each; a
// slice takes every so many-th split, and the slices are joined in their order.
template <int ROWS, int COLS>
__global__ __launch_bounds__(kThreads) void attention_cached_join_kernel(const float *__restrict__ part, CacheGeom g, CachedGeom a,
                                                                         const int32_t *__restrict__ count, float *__restrict__ ctx,
                                                                         uint32_t *__restrict__ absmax) {
  using P = Partial<ROWS, COLS>;
  constexpr int QUADS = ROWS * COLS / 4, PER = QUADS > kThreads ? QUADS / kThreads : 1, SLICES = QUADS > kThreads ? 1 : kThreads / QUADS;
  constexpr int N = SLICES == 1 ? 1 : SLICES;
  __shared__ __attribute__((aligned(16))) float so[N][N == 1 ? 4 : ROWS * COLS];
  __shared__ float sm[N][ROWS], sl[N][ROWS];
  const int tid = static_cast<int>(threadIdx.x), slice = SLICES == 1 ? 0 : tid / QUADS;
  const int id = static_cast<int>(blockIdx.x), rt = id % a.row_tiles, bh = id / a.row_tiles, h = bh % g.kv_heads;
  const float *const from = part + static_cast<int64_t>(id) * a.splits * P::kFloats;
  const int64_t b = bh / g.kv_heads;
  const StreamFrames f = stream_frames(g, count, a.T, b);
  const int n = static_cast<int>(f.end - f.length);
  uint32_t amax = 0u;                     // (parts of frames that the stream did not bring were not written, and are not stored)
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int quad = SLICES == 1 ? k * kThreads + tid : tid % QUADS, row = quad / (COLS / 4), c = 4 * (quad % (COLS / 4));
    float top = kLowest, sum = 0.0f;
    v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = slice; s0 < a.splits; s0 += 4 * SLICES) {   // four parts' loads in flight
      float m[4], l[4];
      v4f x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int s = s0 + u * SLICES;
        const float *const p = from + static_cast<int64_t>(s < a.splits ? s : slice) * P::kFloats;
        m[u] = s < a.splits ? p[P::kMax + row] : kLowest;
        l[u] = s < a.splits ? p[P::kSum + row] : 0.0f;
        x[u] = *reinterpret_cast<const v4f *>(p + row * COLS + c);
      }
      const float next = fmaxf(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), top), alpha = __builtin_amdgcn_exp2f(top - next);
      top = next;
      sum *= alpha;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= alpha;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float w = s0 + u * SLICES < a.splits ? __builtin_amdgcn_exp2f(m[u] - top) : 0.0f;
        sum = fmaf(l[u], w, sum);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = s0 + u * SLICES < a.splits ? fmaf(x[u][e], w, v[e]) : v[e];
      }
    }
    if (SLICES > 1) {
      *reinterpret_cast<v4f *>(&so[slice][row * COLS + c]) = v;
      if (c == 0) {
        sm[slice][row] = top;
        sl[slice][row] = sum;
      }
      __syncthreads();
      if (slice == 0) {
#pragma unroll
        for (int s = 0; s < SLICES; ++s) top = fmaxf(top, sm[s][row]);
        sum = 0.0f;
        v = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < SLICES; ++s) {
          const float w = __builtin_amdgcn_exp2f(sm[s][row] - top);
          sum = fmaf(sl[s][row], w, sum);
          const v4f x = *reinterpret_cast<const v4f *>(&so[s][row * COLS + c]);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = fmaf(x[e], w, v[e]);
        }
      }
    }
    const int out_row = rt * ROWS + row, t = out_row / a.group;
    if (slice == 0 && t < n) {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] *= inv;
      amax = max(amax, put_ctx(ctx + ((b * a.T + t) * a.heads + h * a.group + out_row % a.group) * g.dh, c, g.dh, v));
    }
  }
  if (absmax) put_absmax(absmax, amax);
}

__global__ void zero_word_kernel(uint32_t *p) {
  if (threadIdx.x == 0) *p = 0u;
}

int cols_of(int dh) { return dh <= 32 ? 32 : dh <= 64 ? 64 : 128; }

constexpr int64_t kSplitTiles = 24;

// How a call is cut up: rows of a workgroup (all that share a key / value head, where they are few), row tiles, and the workgroups
// (splits) that share the tiles of a row tile: a tile for every wavefront at most.
struct CachedCut {
  int rows, row_tiles, splits;
  bool own;
  int64_t groups;
};
// window: the longest run of frames that a row tile sees
CachedCut cut_of(const CacheGeom &g, int64_t rows, int64_t window) {
  CachedCut c;
  const int dt = cols_of(g.dh) / 16;
  c.rows = rows <= kFewRows ? (rows == 1 ? 1 : rows == 2 ? 2 : 4) : kRows;
  c.row_tiles = static_cast<int>(cdiv(rows, c.rows));
  c.groups = g.streams * g.kv_heads * c.row_tiles;
  // As many workgroups as the chip holds at a time, a wavefront of each on every SIMD: what comes behind them would form its rows' digits
  // and request its first tile while the others work (32 streams, four rows of 128 columns: 109 us with 512 or 1024
  // workgroups, 116 with 2048; 8 streams of 128 rows: 57 us with 512, 62 with 1024, 76 with 2048).
  const int64_t want = 256 * (c.rows <= kFewRows ? few_waves(dt, g.packed, c.rows) : many_waves(dt, g.packed)) / c.groups;
  // A split has its price, the second launch: under kSplitTiles it takes longer than the tiles that it saves (32 streams of 16 frames with a
  // window of 5 tiles: 11.0 us in two splits, 9.0 in one), and a wavefront gets two tiles at least.
  const int64_t tiles = cdiv(window, 64) + 1, most = tiles < kSplitTiles ? 1 : tiles / (2 * kWaves), s = want < most ? want : most;
  c.splits = static_cast<int>(s < 1 ? 1 : s);
  // Where the row tiles are two wavefronts to a SIMD by themselves, nothing is shared: digits are formed once instead of four times and no
  // parts are joined (2048 row tiles of 64 int8 columns over 3 tiles: 29 us shared, 18 so; over 50: 119, 110).  At half as many a
  // wavefront stands alone on its SIMD for the whole of a long window (1024 over 8 tiles: 21 and 18; over 20: 30 and 31; over 50: 53 and 63).
  c.own = c.rows == kRows && (c.groups >= 2048 || (c.groups >= 1024 && tiles <= 10));
  return c;
}

size_t part_floats(const CachedCut &c, int dh) {
  const size_t rows = static_cast<size_t>(c.rows), one = (rows * cols_of(dh) + 2 * rows + 3) / 4 * 4;   // Partial<rows, columns>
  return c.splits == 1 ? 0 : one * c.groups * c.splits;
}

template <int ROWS>
void launch_join(const float *part, const CacheGeom &g, const CachedGeom &a, const int32_t *count, float *ctx, uint32_t *absmax,
                 unsigned groups, hipStream_t st) {
  auto join = g.dh <= 32   ? attention_cached_join_kernel<ROWS, 32>
              : g.dh <= 64 ? attention_cached_join_kernel<ROWS, 64>
                           : attention_cached_join_kernel<ROWS, 128>;
  join<<<groups, kThreads, 0, st>>>(part, g, a, count, ctx, absmax);
}

template <bool OWN>
auto many_kernel(int dh, bool packed) {
  return packed ? (dh <= 32   ? attention_cached_kernel<2, true, OWN>
                   : dh <= 64 ? attention_cached_kernel<4, true, OWN>
                              : attention_cached_kernel<8, true, OWN>)
                : (dh <= 32   ? attention_cached_kernel<2, false, OWN>
                   : dh <= 64 ? attention_cached_kernel<4, false, OWN>
                              : attention_cached_kernel<8, false, OWN>);
}

}  // namespace

bool cached_attention_ok(const aqt_cache &c, int64_t T, int heads) {
  if (T > (int64_t(1) << 24)) return false;
  const int64_t rows = T * (heads / c.kv_heads), row_tiles = cdiv(rows, rows <= kFewRows ? rows : kRows);
  return row_tiles * kRows <= (int64_t(1) << 30) && row_tiles * c.kv_heads <= kMostBlocks / c.streams;
}

size_t cached_attention_ws_bytes(const aqt_cache &c, int64_t T, int heads) {
  const size_t bytes = part_floats(cut_of(cache_geom(c), T * (heads / c.kv_heads), c.capacity), c.dh) * sizeof(float);
  return bytes < 256 ? 256 : align_up(bytes, 256);
}

aqt_status launch_attention_cached(const float *qkv, int64_t T, int heads, const aqt_cache &c, const int32_t *count, int left, int right,
                                   float *ctx, uint32_t *absmax, void *ws, hipStream_t st) {
  const CacheGeom g = cache_geom(c);
  CachedGeom a;
  a.T = T;
  a.heads = heads;
  a.group = heads / c.kv_heads;
  a.ld = (static_cast<int64_t>(heads) + 2 * static_cast<int64_t>(c.kv_heads)) * c.dh;
  a.left = left;
  a.right = right;
  a.scale_log2e = static_cast<float>(1.4426950408889634 / sqrt(static_cast<double>(c.dh)));
  // a tile's rows span at most that many frames, and a window on either side of them
  const int64_t span = cdiv(kRows, a.group) + 1, window = left < 0 ? c.capacity : span + left + (right < 0 ? T : right);
  const CachedCut cut = cut_of(g, T * a.group, window < c.capacity ? window : c.capacity);
  a.row_tiles = cut.row_tiles;
  a.splits = cut.splits;
  if (absmax) {
    zero_word_kernel<<<1, 64, 0, st>>>(absmax);
    AQT_HIP(hipGetLastError());
  }
  float *const part = cut.splits > 1 ? static_cast<float *>(ws) : nullptr;
  const unsigned blocks = static_cast<unsigned>(cut.own ? cdiv(cut.groups, kWaves) : cut.groups * cut.splits);
  if (cut.rows <= kFewRows) {
    AQT_TRY(launch_attention_cached_few(qkv, g, a, count, ctx, absmax, part, st));
  } else {
    const auto kern = cut.own ? many_kernel<true>(c.dh, g.packed) : many_kernel<false>(c.dh, g.packed);
    kern<<<blocks, kThreads, 0, st>>>(qkv, g, a, count, ctx, absmax, part);
    AQT_HIP(hipGetLastError());
  }
  if (!part) return AQT_OK;
  auto join = cut.rows == 1 ? launch_join<1> : cut.rows == 2 ? launch_join<2> : cut.rows == 4 ? launch_join<4> : launch_join<kRows>;
  join(part, g, a, count, ctx, absmax, static_cast<unsigned>(cut.groups), st);
  AQT_HIP(hipGetLastError());
  return AQT_OK;
}

}  // namespace aqt
