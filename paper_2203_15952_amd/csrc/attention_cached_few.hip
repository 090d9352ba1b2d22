// Attention over the quantized cache where at most four rows (new frame, query head) share a key / value head: single frames, with
// or without grouped heads.  The digits and products of attention_cached.hip; there a lane holds sixteen scores of one of
// sixteen rows, which for one row is sixteen times the vector work that there is (16 streams, one frame over 4000 to 16000 frames,
// int8: 32 us, 27 here; 32 streams, four rows, heads of 128, int4: 109 us, 104 here; reading the codes takes 23 and 88).  Here a lane
// holds one frame's score for each row, and one column of the result:
//   S (rows x 64 frames) = q K^T   A operand: the rows, repeated in each group of four; B operand: 16 frames at a time.  All four groups
//                                  of lanes then hold the scores of all 16; group g keeps those of the g-th 16
//   O (rows x dh) = P V            A operand: the probabilities' digits, through LDS (a byte per digit); B operand: value rows.  Again
//                                  every group holds all of 16 columns, and group g keeps the g-th 16
// The weights' digits are relative to exp2(largest score - running maximum) times the tile's largest value scale, a bound of the
// tile's largest weight that takes one maximum over the wavefront per row and tile; where a row's weights all lie under a quarter
// of it, to the row's largest weight itself.
#include "attention_cached.h"

namespace aqt {
namespace {

__device__ __forceinline__ float of_lane(float v, int lane) {
  return __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(__float_as_uint(v)), lane)));
}
// The group's own of four.
__device__ __forceinline__ int of_group(int a, int b, int c, int d, bool odd, bool upper) {
  const int x = odd ? b : a, y = odd ? d : c;
  return upper ? y : x;
}

// DT: blocks of 16 head columns (2, 4 or 8); R: rows (1, 2 or 4)
template <int DT, bool PACKED, int R>
__global__ __launch_bounds__(kThreads, few_waves(DT, PACKED, R)) void attention_cached_few_kernel(const float *__restrict__ qkv, CacheGeom g, CachedGeom a,
                                                                           const int32_t *__restrict__ count, float *__restrict__ ctx,
                                                                           uint32_t *__restrict__ absmax, float *__restrict__ part) {
  constexpr int KS = DT == 8 ? 2 : 1, COLS = 16 * DT, HALVES = DT == 8 ? 2 : 1, BLOCKS = DT < 4 ? DT : 4;   // HALVES of 64 columns
  using P = Partial<R, COLS>;
  __shared__ __attribute__((aligned(16))) uint8_t digits[kWaves][3][R][64];
  __shared__ __attribute__((aligned(16))) int rest[kWaves][KS][3][64][4];   // of rows whose integers do not hold them
  __shared__ float so[kWaves][R][COLS], sm[kWaves][R], sl[kWaves][R];
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, lr = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool odd = lg & 1, upper = lg >> 1;
  const int split = static_cast<int>(blockIdx.x) % a.splits, bh = static_cast<int>(blockIdx.x) / a.splits;
  const int h = bh % g.kv_heads;
  const int64_t b = bh / g.kv_heads;
  const StreamFrames f = stream_frames(g, count, a.T, b);
  const int n = static_cast<int>(f.end - f.length);
  if (n == 0) return;
  const int rows = min(static_cast<int>(a.T) * a.group, R);

  // the frames that the rows see, counted from the first tile
  auto from = [&](int t) { const int64_t x = f.length + t - a.left; return a.left < 0 || x < f.oldest ? f.oldest : x; };
  auto upto = [&](int t) { const int64_t x = f.length + t + a.right; return a.right < 0 || x > f.end - 1 ? f.end - 1 : x; };
  auto frame_of = [&](int row) { return min(min(row, rows - 1) / a.group, n - 1); };   // rows behind the last repeat it
  const int64_t first = from(0), last = upto(n - 1), tile0 = first >> 6, base = tile0 * 64;
  const int tiles = last < first ? 0 : static_cast<int>((last >> 6) - tile0) + 1;
  int lo[R], hi[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    lo[r] = static_cast<int>(from(frame_of(r)) - base);
    hi[r] = static_cast<int>(upto(frame_of(r)) - base);
  }

  // The rows (requested in front of the first tile, so that their digits are formed under its trip from memory)
  float x[KS][16];
  {
    const int own = min(lr & 3, R - 1), t = frame_of(own);
    const float *const src = qkv + (b * a.T + t) * a.ld + (static_cast<int64_t>(h) * a.group + min(own, rows - 1) % a.group) * g.dh;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[k][i] = src[min(64 * k + 16 * lg + i, g.dh - 1)];
  }

  const uint8_t *const head = g.data + (b * g.kv_heads + h) * g.tiles * static_cast<int64_t>(g.tile_bytes);
  const int step = a.splits * kWaves, slot_step = step % g.tiles;
  float m[R], l[R], o[HALVES][R];            // o: column 64 half + lane
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = kLowest;
    l[r] = 0.0f;
#pragma unroll
    for (int k = 0; k < HALVES; ++k) o[k][r] = 0.0f;
  }
  uint8_t *const put = &digits[wave][0][0][frame_slot(lane)];
  const uint8_t *const take = &digits[wave][0][min(lr & 3, R - 1)][16 * lg];
  // A tile's keys, values and scales are requested where the tile before has given up their registers: the keys' trip from memory
  // passes under the rest of that tile, the values' under this one's scores.
  constexpr int KEYS = PACKED ? 2 : 4, VALUES = PACKED ? DT / 2 : DT;
  typedef int key_piece __attribute__((ext_vector_type(KEYS)));
  key_piece keys[4][KS];
  v4i values[VALUES];
  float ks, vs_next;
  auto key_of = [&](const uint8_t *tile, int t, int k) {   // sixteen columns to a lane; one beyond the row meets digits of zero
    const int at = (64 * k + 16 * lg) * KEYS / 4;
    return *reinterpret_cast<const key_piece *>(tile + (16 * t + lr) * g.key_row + (at < g.key_row ? at : 0));
  };
  auto load_keys = [&](const uint8_t *tile) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int k = 0; k < KS; ++k) keys[t][k] = key_of(tile, t, k);
    ks = reinterpret_cast<const float *>(tile + cache_scales(g))[lane];
  };
  auto load_values = [&](const uint8_t *tile) {
#pragma unroll
    for (int d = 0; d < VALUES; ++d) {
      const int at = 16 * d + lr;      // columns beyond the head are not stored
      values[d] = *reinterpret_cast<const v4i *>(tile + cache_values(g) + (at < g.value_rows ? at : lr) * 64 + 16 * lg);
    }
    vs_next = reinterpret_cast<const float *>(tile + cache_scales(g))[64 + lane];
  };
  int i = split * kWaves + wave;
  int slot = tile_slot(tile0 + i, g.tiles);
  if (i < tiles) {
    const uint8_t *const tile = head + static_cast<int64_t>(slot) * g.tile_bytes;
    load_keys(tile);
    load_values(tile);
  }
  // the rows' digits: row lr % 4 of R, 16 columns per lane and step
  v4i q[KS][3];
  float row_scale[R];
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
    const float unit = (m > 0x7F800000u ? top : fmaxf(top, 0x1p-100f)) * (1.0f / kDigits) * a.scale_log2e * (PACKED ? 0.0625f : 1.0f);
#pragma unroll
    for (int r = 0; r < R; ++r) row_scale[r] = of_lane(unit, r);
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
    float vs = vs_next;
    const float ks_now = ks;
    v4i c[4][3];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const v4i w = codes(keys[t][k]);
#pragma unroll
        for (int d = 0; d < 3; ++d) c[t][d] = mfma_i8(q[k][d], w, k == 0 ? v4i{0, 0, 0, 0} : c[t][d]);
      }
    load_keys(next);
    // the lane's frame: window (what it hides, and what is no frame of the stream's, may hold anything)
    const int j0 = 64 * i, j = j0 + lane;
    bool whole = true;
#pragma unroll
    for (int r = 0; r < R; ++r) whole = whole && j0 >= lo[r] && j0 + 63 <= hi[r];
    float s[R];
    bool see[R], any = false;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      int d[3];
#pragma unroll
      for (int e = 0; e < 3; ++e) d[e] = of_group(c[0][e][r], c[1][e][r], c[2][e][r], c[3][e][r], odd, upper);
      see[r] = whole || (j >= lo[r] && j <= hi[r]);
      any = any || see[r];
      s[r] = joined(d[0], d[1], d[2]) * (row_scale[r] * ks_now);
    }
    if (wide) {   // the digits behind those (few rows have any, so that the tile's keys are read again)
      float sum[R];
#pragma unroll
      for (int r = 0; r < R; ++r) sum[r] = 0.0f;
#pragma unroll
      for (int d = 0; d < 3; ++d) {
        v4i e[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int k = 0; k < KS; ++k)
            e[t] = mfma_i8(*reinterpret_cast<const v4i *>(rest[wave][k][d][lane]), codes(key_of(tile, t, k)), k == 0 ? v4i{0, 0, 0, 0} : e[t]);
#pragma unroll
        for (int r = 0; r < R; ++r) sum[r] = fmaf(sum[r], 256.0f, static_cast<float>(of_group(e[0][r], e[1][r], e[2][r], e[3][r], odd, upper)));
      }
#pragma unroll
      for (int r = 0; r < R; ++r) s[r] = fmaf(sum[r], row_scale[r] * ks_now * kRestUnit, s[r]);
    }
    vs = any ? vs : 0.0f;
    const float vs_top = wave_max_positive(vs);
    float alpha[R], unit[R], weight[R], top[R];
    bool near[R], all_near = true;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float mx = wave_max_signed(see[r] ? s[r] : kLowest), mnew = fmaxf(m[r], mx);
      alpha[r] = __builtin_amdgcn_exp2f(m[r] - mnew);
      m[r] = mnew;
      const float p = see[r] ? __builtin_amdgcn_exp2f(s[r] - mnew) : 0.0f;
      l[r] = fmaf(l[r], alpha[r], p);
      weight[r] = p * vs;
      top[r] = __builtin_amdgcn_exp2f(mx - mnew) * vs_top;
      near[r] = __any(weight[r] >= 0.25f * top[r]);
      all_near = all_near && near[r];
    }
    if (!all_near) {   // ... and where a scale is NaN: what a row does not see is nothing to it
#pragma unroll
      for (int r = 0; r < R; ++r) {
        weight[r] = see[r] ? weight[r] : 0.0f;
        if (!near[r]) top[r] = wave_max_positive(fabsf(weight[r]));
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      top[r] = at_least_tiny(top[r]);
      unit[r] = top[r] * (1.0f / kDigits) * (PACKED ? 0.0625f : 1.0f);
      const uint32_t u = weight_bits(weight[r], kDigits * __builtin_amdgcn_rcpf(top[r])) ^ 0x00008080u;
      put[(2 * R + r) * 64] = static_cast<uint8_t>(u);
      put[(R + r) * 64] = static_cast<uint8_t>(u >> 8);
      put[r * 64] = static_cast<uint8_t>(u >> 16);
    }
    wave_lds_order();
    v4i p[3];
#pragma unroll
    for (int d = 0; d < 3; ++d) p[d] = *reinterpret_cast<const v4i *>(take + d * R * 64);
    wave_lds_order();   // read before the next tile's are written
#pragma unroll
    for (int k = 0; k < HALVES; ++k) {
      v4i e[4][3];
      auto product = [&](v4i (&to)[3], v4i w) {
#pragma unroll
        for (int d = 0; d < 3; ++d) to[d] = mfma_i8(p[d], w, v4i{0, 0, 0, 0});
      };
#pragma unroll
      for (int d = 0; d < BLOCKS; d += PACKED ? 2 : 1) {
        const v4i x = values[PACKED ? (4 * k + d) / 2 : 4 * k + d];
        if (PACKED) {
          v4i lo4, hi4;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            lo4[w] = static_cast<int>(static_cast<uint32_t>(x[w]) << 4 & 0xF0F0F0F0u);
            hi4[w] = static_cast<int>(static_cast<uint32_t>(x[w]) & 0xF0F0F0F0u);
          }
          product(e[d], lo4);
          product(e[d + 1], hi4);
        } else {
          product(e[d], x);
        }
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        int d[3];
#pragma unroll
        for (int w = 0; w < 3; ++w)
          d[w] = BLOCKS == 4 ? of_group(e[0][w][r], e[1][w][r], e[2 % BLOCKS][w][r], e[3 % BLOCKS][w][r], odd, upper) : odd ? e[1][w][r] : e[0][w][r];
        o[k][r] = fmaf(joined(d[0], d[1], d[2]), unit[r], o[k][r] * alpha[r]);
      }
    }
    load_values(next);
  }

  // the wavefronts' parts of the rows
#pragma unroll
  for (int r = 0; r < R; ++r) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) l[r] += __shfl_xor(l[r], off, 64);
    if (lane == 0) {
      sm[wave][r] = m[r];
      sl[wave][r] = l[r];
    }
#pragma unroll
    for (int k = 0; k < HALVES; ++k)
      if (lane < COLS) so[wave][r][64 * k + lane] = o[k][r];
  }
  __syncthreads();
  uint32_t amax = 0u;
  float *const left = part ? part + static_cast<int64_t>(blockIdx.x) * P::kFloats : nullptr;
  for (int x = tid; x < R * COLS; x += kThreads) {
    const int r = x / COLS, c = x % COLS, t = r / a.group;
    float top = kLowest, sum = 0.0f, v = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm[w][r]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float weight = __builtin_amdgcn_exp2f(sm[w][r] - top);
      sum = fmaf(sl[w][r], weight, sum);
      v = fmaf(so[w][r][c], weight, v);
    }
    if (left) {
      left[x] = v;
      if (c == 0) {
        left[P::kMax + r] = top;
        left[P::kSum + r] = sum;
      }
    } else if (t < n && r < rows && c < g.dh) {
      v *= sum == 0.0f ? 0.0f : 1.0f / sum;   // nothing seen: zeros
      ctx[((b * a.T + t) * a.heads + h * a.group + r % a.group) * g.dh + c] = v;
      amax = max(amax, __float_as_uint(v) & 0x7FFFFFFFu);
    }
  }
  if (!left && absmax) put_absmax(absmax, amax);
}

template <int DT, bool PACKED>
aqt_status launch_rows(const float *qkv, const CacheGeom &g, const CachedGeom &a, const int32_t *count, float *ctx, uint32_t *absmax,
                       float *part, hipStream_t st) {
  const int64_t rows = a.T * a.group;
  const unsigned blocks = static_cast<unsigned>(g.streams * g.kv_heads * a.splits);
  auto kern = rows == 1   ? attention_cached_few_kernel<DT, PACKED, 1>
              : rows == 2 ? attention_cached_few_kernel<DT, PACKED, 2>
                          : attention_cached_few_kernel<DT, PACKED, 4>;
  kern<<<blocks, kThreads, 0, st>>>(qkv, g, a, count, ctx, absmax, part);
  AQT_HIP(hipGetLastError());
  return AQT_OK;
}

}  // namespace

aqt_status launch_attention_cached_few(const float *qkv, const CacheGeom &g, const CachedGeom &a, const int32_t *count, float *ctx,
                                       uint32_t *absmax, float *part, hipStream_t st) {
  auto launch = g.packed ? (g.dh <= 32 ? launch_rows<2, true> : g.dh <= 64 ? launch_rows<4, true> : launch_rows<8, true>)
                         : (g.dh <= 32 ? launch_rows<2, false> : g.dh <= 64 ? launch_rows<4, false> : launch_rows<8, false>);
  return launch(qkv, g, a, count, ctx, absmax, part, st);
}

}  // namespace aqt
