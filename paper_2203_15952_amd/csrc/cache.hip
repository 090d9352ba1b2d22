// Keys and values of a stream's new frames into its quantized cache, and back out of it (the layout is cache.h's).
//
// Writing, per frame and key / value head, separately for keys and values (Fig. 2 of arxiv 2203.15952, reduced over the head):
//   scale = max|x| / qmax,   code = floor(x / scale + 0.5)   (0 where the scale is 0),   every operation one float32 rounding.
// Reading: code * scale.  Memory bounds both: a frame's float32 row in one and its codes in the other direction.
//
// A group of L lanes takes four consecutive frames (aligned, so that they share a tile) of one head, a lane the same eight
// columns of the four: a frame's maximum is L lanes' shuffles, a key row leaves (and comes) as dwords of four columns, and a
// value row, whose four frames are neighbours, as dwords of four frames after a 4 x 4 transposition of bytes in registers.  Where a
// call brings only some of the four frames the others' bytes are not touched.
#include "cache.h"
#include "lanes.h"
#include "quant_code.h"

namespace aqt {
namespace {

constexpr int kThreads = 256;
typedef float v4f __attribute__((ext_vector_type(4)));

// Four dwords of four bytes each, transposed: out[i] byte f = in[f] byte i.
__device__ __forceinline__ void transpose_bytes(uint32_t (&w)[4]) {
  const uint32_t ab0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), ab1 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const uint32_t cd0 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), cd1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  w[0] = __builtin_amdgcn_perm(cd0, ab0, 0x05040100u);
  w[1] = __builtin_amdgcn_perm(cd0, ab0, 0x07060302u);
  w[2] = __builtin_amdgcn_perm(cd1, ab1, 0x05040100u);
  w[3] = __builtin_amdgcn_perm(cd1, ab1, 0x07060302u);
}

// Four codes, the first in the lowest byte.  r is 1 / s to 2^-23 of it: then x r is within 2^-16 of x / s (up to 127), whose own rounding
// and that of the sum with 1 / 2 are 2^-18 each, and where it lies no nearer than 2^-14 to the middle between two whole numbers its
// nearest one is the floor that defines the code; otherwise (one quad in two thousand) the four are divided.  x r + 1.5 2^23 rounds to that whole number, in its lowest bits.  No value exceeds its group's maximum, so no
// code is clamped.  r is 0 where s is no ordinary number.
__device__ __forceinline__ uint32_t codes4(const float (&x)[4], float s, float r, float fq) {
  constexpr float kWhole = 12582912.0f;
  uint32_t n[4];
  float off[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float w = fmaf(x[e], r, kWhole);
    n[e] = __float_as_uint(w);
    off[e] = fabsf(fmaf(x[e], r, kWhole - w));
  }
  if (r == 0.0f || !(fmaxf(fmaxf(off[0], off[1]), fmaxf(off[2], off[3])) < 0.5f - 0x1p-14f))
    return quant4_divided(x[0], x[1], x[2], x[3], Quantizer{s, fq, 0.0f, false});
  const uint32_t lo = __builtin_amdgcn_perm(n[1], n[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(n[3], n[2], 0x0C0C0400u);
  return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}

// What a group of lanes works on: four frames from `frame` (a multiple of four, possibly negative) of head h.
struct Quad {
  int64_t frame;
  int h;
  bool values;
};
// A stream's work, counted in items: runs of `run` quads (a power of two, aligned: 16 make a tile), the run's quads the fastest, then
// keys or values and head, then runs.  So a workgroup writes the tiles it touches whole: frames of one head that eight
// workgroups on eight L2s share cost every line eight partial writes (4096 frames of 16 streams
// with runs of one quad: written in 130 us, 69 so; read back in 93, 57).
__device__ __forceinline__ Quad quad_of(const CacheGeom &g, int item, int log2_run, int64_t from) {
  const int per = 2 * g.kv_heads, group = item >> log2_run, r = group / per, w = group - r * per;
  const bool values = w >= g.kv_heads;
  const int64_t quad = ((((from >> 2) >> log2_run) + r) << log2_run) + (item & ((1 << log2_run) - 1));
  return Quad{quad * 4, values ? w - g.kv_heads : w, values};
}

// A lane's eight columns, two times four: so that the group's float32 pieces are neighbours, or, two to a byte, those that share
// one (a key row's are 8 apart, a value row's 16).
template <int L>
struct Columns {
  int lo, hi;
  __device__ __forceinline__ Columns(int j, bool packed, bool values) {
    lo = !packed ? 4 * j : values ? 32 * (j >> 2) + 4 * (j & 3) : 16 * (j >> 1) + 4 * (j & 1);
    hi = lo + (!packed ? 4 * L : values ? 16 : 8);
  }
};

__device__ __forceinline__ uint8_t *tile_of(const CacheGeom &g, int64_t b, const Quad &q) {
  const int64_t at = (b * g.kv_heads + q.h) * g.tiles + tile_slot(q.frame >> 6, g.tiles);
  return g.data + at * g.tile_bytes;
}

// A float32 row is not read again: without a place in the caches it leaves them to the codes and to what else is under way
// (4096 frames of 16 streams, written and read back in turn: 92 and 64 us, 69 and 57 so).
template <bool VEC>
__device__ __forceinline__ void load4(float (&x)[4], const float *row, int col, int dh) {
  if (VEC) {
    if (col < dh) {
      const v4f v = __builtin_nontemporal_load(reinterpret_cast<const v4f *>(row + col));
      x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
      x[0] = x[1] = x[2] = x[3] = 0.0f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = col + i < dh ? row[col + i] : 0.0f;
  }
}
template <bool VEC>
__device__ __forceinline__ void store4(const float (&x)[4], float *row, int col, int dh) {
  if (VEC) {
    if (col < dh) *reinterpret_cast<v4f *>(row + col) = v4f{x[0], x[1], x[2], x[3]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (col + i < dh) row[col + i] = x[i];
  }
}

template <int L, bool VEC>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(const float *__restrict__ qkv, CacheGeom g, int64_t T, int heads,
                                                                const int32_t *__restrict__ count, int log2_run, int blocks_per_stream,
                                                                int32_t *__restrict__ dev_status) {
  const int tid = static_cast<int>(threadIdx.x), j = tid % L;
  const int b = static_cast<int>(blockIdx.x) / blocks_per_stream, block = static_cast<int>(blockIdx.x) - b * blocks_per_stream;
  const StreamFrames f = stream_frames(g, count, T, b);
  const int64_t from = f.length > f.oldest ? f.length : f.oldest;   // later frames of this call take the place of those before
  const Quad q = quad_of(g, block * (kThreads / L) + tid / L, log2_run, from);
  const int64_t ld = (static_cast<int64_t>(heads) + 2 * static_cast<int64_t>(g.kv_heads)) * g.dh;
  const int64_t at = (heads + (q.values ? g.kv_heads : 0) + static_cast<int64_t>(q.h)) * g.dh;
  const Columns<L> c(j, g.packed, q.values);
  float x[4][2][4];
  bool mine[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t p = q.frame + i;
    mine[i] = p >= from && p < f.end;   // (from == f.end: a stream without new frames)
    const int64_t t = mine[i] ? p - f.length : 0;   // always a row of the call
    const float *const row = qkv + (b * T + t) * ld + at;
    load4<VEC>(x[i][0], row, mine[i] ? c.lo : g.dh, g.dh);
    load4<VEC>(x[i][1], row, mine[i] ? c.hi : g.dh, g.dh);
  }
  uint8_t *const tile = tile_of(g, b, q);
  const int key = static_cast<int>(q.frame & 63);
  // A lane divides for one of the four frames and hands on.
  uint32_t top[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    top[i] = 0u;
    if (!__any(mine[i])) continue;   // single frames: three of the four
    uint32_t m = 0u;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = max(m, __float_as_uint(x[i][h][e]) & 0x7FFFFFFFu);
    top[i] = group_max<L>(m);
  }
  const bool odd = j & 1, upper = j & 2, own = upper ? (odd ? mine[3] : mine[2]) : odd ? mine[1] : mine[0];
  const uint32_t own_top = upper ? (odd ? top[3] : top[2]) : odd ? top[1] : top[0];
  // (Inf or NaN in the head: a scale of NaN, which makes NaN of all that is read from it, whatever the codes are)
  const float fq = static_cast<float>(g.qmax), own_s = own_top < 0x7F800000u ? __uint_as_float(own_top) / fq : __builtin_nanf("");
  const float own_r = own_s > 0x1p-60f && own_s < 0x1p60f ? __builtin_amdgcn_rcpf(own_s) : 0.0f;
  if (j < 4 && own) {
    reinterpret_cast<float *>(tile + cache_scales(g))[(q.values ? 64 : 0) + key + j] = own_s;
    if (dev_status && own_top >= 0x7F800000u) *dev_status = AQT_ERR_NONFINITE;
  }
  const float s[4] = {of_four<0>(own_s), of_four<1>(own_s), of_four<2>(own_s), of_four<3>(own_s)};
  const float r[4] = {of_four<0>(own_r), of_four<1>(own_r), of_four<2>(own_r), of_four<3>(own_r)};
  uint32_t code[2][4];   // [half][frame]
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    code[0][i] = code[1][i] = 0u;
    if (!__any(mine[i])) continue;
#pragma unroll
    for (int h = 0; h < 2; ++h) code[h][i] = codes4(x[i][h], s[i], r[i], fq);
  }
  if (!q.values) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!mine[i]) continue;
      uint8_t *const row = tile + (key + i) * g.key_row;
      if (g.packed) {
        if (c.lo < 2 * g.key_row)
          *reinterpret_cast<uint32_t *>(row + 8 * (j >> 1) + 4 * (j & 1)) = (code[0][i] & 0x0F0F0F0Fu) | (code[1][i] & 0x0F0F0F0Fu) << 4;
      } else {
        if (c.lo < g.key_row) *reinterpret_cast<uint32_t *>(row + c.lo) = code[0][i];
        if (c.hi < g.key_row) *reinterpret_cast<uint32_t *>(row + c.hi) = code[1][i];
      }
    }
    return;
  }
  transpose_bytes(code[0]);
  transpose_bytes(code[1]);
  uint8_t *const values = tile + cache_values(g) + frame_slot(key);
  const bool whole = mine[0] && mine[1] && mine[2] && mine[3];
  auto put = [&](int row, uint32_t w) {
    if (row >= g.value_rows) return;
    uint8_t *const at4 = values + row * 64;
    if (whole) {
      *reinterpret_cast<uint32_t *>(at4) = w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (mine[i]) at4[i] = static_cast<uint8_t>(w >> (8 * i));
    }
  };
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (g.packed) {
      put(16 * (j >> 2) + 4 * (j & 3) + e, (code[0][e] & 0x0F0F0F0Fu) | (code[1][e] & 0x0F0F0F0Fu) << 4);
    } else {
      put(c.lo + e, code[0][e]);
      put(c.hi + e, code[1][e]);
    }
  }
}

// Four signed codes from a dword: bytes, or the low or high nibbles of bytes.
__device__ __forceinline__ void codes_of(float (&x)[4], uint32_t w, bool packed, bool high) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t byte = w >> (8 * e) & 0xFFu;
    const int v = packed ? static_cast<int>((high ? byte >> 4 : byte) << 28) >> 28 : static_cast<int>(byte << 24) >> 24;
    x[e] = static_cast<float>(v);
  }
}

template <int L, bool VEC>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(CacheGeom g, int64_t pending, const int32_t *__restrict__ count,
                                                              const int64_t *__restrict__ first, int64_t n, int log2_run,
                                                              int blocks_per_stream, float *__restrict__ keys, float *__restrict__ values) {
  const int tid = static_cast<int>(threadIdx.x), j = tid % L;
  const int b = static_cast<int>(blockIdx.x) / blocks_per_stream, block = static_cast<int>(blockIdx.x) - b * blocks_per_stream;
  const StreamFrames f = stream_frames(g, count, pending, b);
  const int64_t far = int64_t(1) << 61;
  int64_t from = first ? first[b] : f.end - n;
  from = from < -far ? -far : from > far ? far : from;
  const Quad q = quad_of(g, block * (kThreads / L) + tid / L, log2_run, from);
  if (q.frame >= from + n || q.frame + 3 < from) return;
  float *const to = q.values ? values : keys;
  if (!to) return;
  const Columns<L> c(j, g.packed, q.values);
  bool held[4];
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    held[i] = q.frame + i >= f.oldest && q.frame + i < f.end;   // oldest is not negative
    any = any || held[i];
  }
  uint32_t code[2][4] = {};   // [half][frame], packed: both halves in code[0]
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (any) {   // the tile is the cache's own whichever of its frames are held
    const uint8_t *const tile = tile_of(g, b, q);
    const int key = static_cast<int>(q.frame & 63);
    const v4f scales = *reinterpret_cast<const v4f *>(tile + cache_scales(g) + 4 * ((q.values ? 64 : 0) + key));
    s[0] = scales.x; s[1] = scales.y; s[2] = scales.z; s[3] = scales.w;
    if (!q.values) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint8_t *const row = tile + (key + i) * g.key_row;
        if (g.packed) {
          if (c.lo < 2 * g.key_row) code[0][i] = *reinterpret_cast<const uint32_t *>(row + 8 * (j >> 1) + 4 * (j & 1));
        } else {
          if (c.lo < g.key_row) code[0][i] = *reinterpret_cast<const uint32_t *>(row + c.lo);
          if (c.hi < g.key_row) code[1][i] = *reinterpret_cast<const uint32_t *>(row + c.hi);
        }
      }
    } else {
      const uint8_t *const at = tile + cache_values(g) + frame_slot(key);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int lo = g.packed ? 16 * (j >> 2) + 4 * (j & 3) + e : c.lo + e;
        if (lo < g.value_rows) code[0][e] = *reinterpret_cast<const uint32_t *>(at + lo * 64);
        if (!g.packed && c.hi + e < g.value_rows) code[1][e] = *reinterpret_cast<const uint32_t *>(at + (c.hi + e) * 64);
      }
      transpose_bytes(code[0]);
      transpose_bytes(code[1]);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t r = q.frame + i - from;
    if (r < 0 || r >= n) continue;
    float *const row = to + ((b * n + r) * g.kv_heads + q.h) * g.dh;
    float x[2][4];
    codes_of(x[0], code[0][i], g.packed, false);
    codes_of(x[1], g.packed ? code[0][i] : code[1][i], g.packed, true);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[h][e] = held[i] ? x[h][e] * s[i] : 0.0f;
    store4<VEC>(x[0], row, c.lo, g.dh);
    store4<VEC>(x[1], row, c.hi, g.dh);
  }
}

__global__ void cache_advance_kernel(int64_t *__restrict__ length, int64_t streams, int64_t T, const int32_t *__restrict__ count) {
  const int64_t b = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (b >= streams) return;
  const int64_t n = count ? count[b] : T, L = length[b];
  length[b] = (L < 0 ? 0 : L) + (n < 0 ? 0 : n > T ? T : n);
}

// How a call over `n` consecutive frames of every stream is cut up.
struct Cut {
  int log2_run;
  int64_t items, blocks;   // of a stream
};
int lanes_of(int dh) { return dh <= 32 ? 4 : dh <= 64 ? 8 : 16; }
Cut cut_of(const CacheGeom &g, int64_t n) {
  const int64_t quads = (n + 2) / 4 + 1;   // that n frames can touch
  Cut c{0, 0, 0};
  while (c.log2_run < 4 && (int64_t(1) << c.log2_run) < quads) ++c.log2_run;
  const int64_t runs = ((quads - 2) >> c.log2_run) + 2;   // and as many runs of them, wherever the first begins
  c.items = ((quads == 1 ? 1 : runs) << c.log2_run) * 2 * g.kv_heads;
  c.blocks = cdiv(c.items, kThreads / lanes_of(g.dh));
  return c;
}
// Items of a stream count in 32 bits, and so do the threads of the launch.
bool grid_ok(const CacheGeom &g, int64_t n) {
  if (n > (int64_t(1) << 40)) return false;
  const Cut c = cut_of(g, n);
  return c.items <= INT32_MAX - kThreads && c.blocks <= kMostBlocks / g.streams;
}

}  // namespace

bool cache_shape_ok(const aqt_cache &c) {
  const int64_t tiles = c.capacity / 64;
  return c.streams >= 1 && c.capacity >= 64 && c.capacity % 64 == 0 && tiles <= (1 << 24) && c.kv_heads >= 1 && c.kv_heads <= 4096 &&
         c.dh >= 1 && c.dh <= 128 && bits_ok(c.bits) && c.streams <= (int64_t(1) << 24) &&
         c.streams * c.kv_heads <= (int64_t(1) << 46) / tiles;   // a tile takes 17 KB at most: bytes count in 64 bits
}

CacheGeom cache_geom(const aqt_cache &c) {
  CacheGeom g;
  const int d16 = static_cast<int>(align_up(c.dh, 16));
  g.streams = c.streams;
  g.tiles = static_cast<int>(c.capacity / 64);
  g.kv_heads = c.kv_heads;
  g.dh = c.dh;
  g.qmax = qmax_of(c.bits);
  g.packed = packed4(c.bits);
  g.key_row = g.packed ? d16 / 2 : d16;
  g.value_rows = g.packed ? 16 * static_cast<int>(cdiv(c.dh, 32)) : d16;
  g.tile_bytes = 64 * (g.key_row + g.value_rows + 8);
  g.data = static_cast<uint8_t *>(c.data);
  g.length = c.length;
  return g;
}

aqt_status launch_cache_append(const float *qkv, int64_t T, int heads, const aqt_cache &c, const int32_t *count, hipStream_t st,
                               int32_t *dev_status) {
  const CacheGeom g = cache_geom(c);
  const int64_t most = T < c.capacity ? T : c.capacity;
  if (!grid_ok(g, most)) return AQT_ERR_UNSUPPORTED;
  const size_t streams = static_cast<size_t>(g.streams);
  if (!apart({{g.data, cache_bytes(g)}, {dev_status, sizeof(int32_t)}},
             {{qkv, cache_rows_bytes(g, T, heads)}, {g.length, streams * sizeof(int64_t)}, {count, streams * sizeof(int32_t)}}))
    return AQT_ERR_INVALID_ARG;
  const Cut cut = cut_of(g, most);
  const bool vec = reinterpret_cast<uintptr_t>(qkv) % 16 == 0 && c.dh % 4 == 0;
  auto kern = c.dh <= 32   ? (vec ? cache_append_kernel<4, true> : cache_append_kernel<4, false>)
              : c.dh <= 64 ? (vec ? cache_append_kernel<8, true> : cache_append_kernel<8, false>)
                           : (vec ? cache_append_kernel<16, true> : cache_append_kernel<16, false>);
  kern<<<static_cast<unsigned>(cut.blocks * c.streams), kThreads, 0, st>>>(qkv, g, T, heads, count, cut.log2_run, static_cast<int>(cut.blocks),
                                                                          dev_status);
  AQT_HIP(hipGetLastError());
  return AQT_OK;
}

aqt_status launch_cache_read(const aqt_cache &c, int64_t pending, const int32_t *count, const int64_t *first, int64_t n, float *keys,
                             float *values, hipStream_t st) {
  const CacheGeom g = cache_geom(c);
  if (!grid_ok(g, n)) return AQT_ERR_UNSUPPORTED;
  const size_t streams = static_cast<size_t>(g.streams), bytes = streams * n * g.kv_heads * g.dh * sizeof(float);
  if (!apart({{keys, bytes}, {values, bytes}}, {{g.data, cache_bytes(g)}, {g.length, streams * sizeof(int64_t)},
                                                {count, streams * sizeof(int32_t)}, {first, streams * sizeof(int64_t)}}))
    return AQT_ERR_INVALID_ARG;
  const Cut cut = cut_of(g, n);
  const bool vec = reinterpret_cast<uintptr_t>(keys) % 16 == 0 && reinterpret_cast<uintptr_t>(values) % 16 == 0 && c.dh % 4 == 0;
  auto kern = c.dh <= 32   ? (vec ? cache_read_kernel<4, true> : cache_read_kernel<4, false>)
              : c.dh <= 64 ? (vec ? cache_read_kernel<8, true> : cache_read_kernel<8, false>)
                           : (vec ? cache_read_kernel<16, true> : cache_read_kernel<16, false>);
  kern<<<static_cast<unsigned>(cut.blocks * c.streams), kThreads, 0, st>>>(g, pending, count, first, n, cut.log2_run,
                                                                          static_cast<int>(cut.blocks), keys, values);
  AQT_HIP(hipGetLastError());
  return AQT_OK;
}

aqt_status launch_cache_advance(int64_t *length, int64_t streams, int64_t T, const int32_t *count, hipStream_t st) {
  cache_advance_kernel<<<static_cast<unsigned>(cdiv(streams, kThreads)), kThreads, 0, st>>>(length, streams, T, count);
  AQT_HIP(hipGetLastError());
  return AQT_OK;
}

}  // namespace aqt
