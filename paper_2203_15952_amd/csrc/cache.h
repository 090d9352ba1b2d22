// Where a quantized cache keeps what (cache.hip writes and reads it back, attention_cached.hip attends over it).
//
// For every stream and key / value head the cache is a ring of tiles of 64 frames: frame p lives in tile (p / 64) mod tiles, so
// a tile of 64 consecutive frames is one piece of memory and a frame overwrites the one `capacity` frames before it.  A tile is
//   keys    [64 frames][key row]     codes as the A operand of v_mfma_i32_16x16x64_i8 reads them: 16 columns per lane
//   values  [value rows][64 frames]  transposed, so that the product over frames reads 16 frames of a column per lane
//   key scales [64], value scales [64] float32
// The 64 frames of a value row stand in the order in which a lane holds the probabilities: frame 16 t + 4 g + r (the lanes of
// group g own it, as accumulator register r of the t-th key block) at byte 16 g + 4 t + r.  Four frames 4 i .. 4 i + 3 are
// neighbours in both orders.
// Codes of 5 to 8 bits take a byte.  Up to 4 bits they are two to a byte: of a key row's 16 columns 16 c .. the low nibbles
// hold the first eight, the high nibbles the others; a value row holds column 32 u + c low and 32 u + 16 + c high.
#pragma once
#include "aqt_internal.h"

namespace aqt {

struct CacheGeom {
  int64_t streams;
  int tiles;                     // per stream and head
  int kv_heads, dh, qmax;
  int packed;
  int key_row, value_rows;       // bytes of a key row; rows of values (16 or, packed, 32 columns make 16 rows)
  int tile_bytes;
  uint8_t *data;
  const int64_t *length;         // frames of every stream in front of the call's
};

// Bytes from a tile's start, where its keys are.
__host__ __device__ inline int cache_values(const CacheGeom &g) { return 64 * g.key_row; }
__host__ __device__ inline int cache_scales(const CacheGeom &g) { return 64 * (g.key_row + g.value_rows); }   // keys', then values'
__host__ __device__ inline int frame_slot(int frame) { return (frame & 3) | ((frame >> 2) & 0x0C) | ((frame << 2) & 0x30); }

// frame / 64 mod tiles
__host__ __device__ inline int tile_slot(int64_t tile, int tiles) {
  return (tile >> 32) == 0 ? static_cast<int>(static_cast<uint32_t>(tile) % static_cast<uint32_t>(tiles)) : static_cast<int>(tile % tiles);
}

// The frames of one stream: `length` in front of the call, `count` new ones; a stream cannot have fewer than none, nor more new
// ones than the call brings.
struct StreamFrames {
  int64_t length, end;   // frames before the call, and with its own
  int64_t oldest;        // the first frame that the cache holds after the call
};
__host__ __device__ inline StreamFrames stream_frames(const CacheGeom &g, const int32_t *count, int64_t T, int64_t b) {
  const int64_t top = int64_t(1) << 61;
  int64_t L = g.length[b], n = count ? count[b] : T;
  L = L < 0 ? 0 : L > top ? top : L;
  n = n < 0 ? 0 : n > T ? T : n;
  const int64_t end = L + n, cap = static_cast<int64_t>(g.tiles) * 64;
  return StreamFrames{L, end, end > cap ? end - cap : 0};
}

constexpr int64_t kMostBlocks = (int64_t(1) << 24) - 1;   // of 256 threads: a launch's threads count in 32 bits

inline size_t cache_bytes(const CacheGeom &g) { return static_cast<size_t>(g.streams) * g.kv_heads * g.tiles * g.tile_bytes; }
// Of the rows of a call, as many as an address space holds at most.
inline size_t cache_rows_bytes(const CacheGeom &g, int64_t T, int heads) {
  const size_t row = (static_cast<size_t>(heads) + 2 * static_cast<size_t>(g.kv_heads)) * g.dh * sizeof(float) * static_cast<size_t>(g.streams);
  const size_t most = size_t(1) << 60;   // (row: at most 2^24 streams of 2^30 bytes)
  return static_cast<size_t>(T) > most / row ? most : row * static_cast<size_t>(T);
}

bool cache_shape_ok(const aqt_cache &c);
CacheGeom cache_geom(const aqt_cache &c);
aqt_status launch_cache_append(const float *qkv, int64_t T, int heads, const aqt_cache &c, const int32_t *count, hipStream_t st,
                               int32_t *dev_status);
aqt_status launch_cache_read(const aqt_cache &c, int64_t pending, const int32_t *count, const int64_t *first, int64_t n, float *keys,
                             float *values, hipStream_t st);
aqt_status launch_cache_advance(int64_t *length, int64_t streams, int64_t T, const int32_t *count, hipStream_t st);
bool cached_attention_ok(const aqt_cache &c, int64_t T, int heads);
size_t cached_attention_ws_bytes(const aqt_cache &c, int64_t T, int heads);
aqt_status launch_attention_cached(const float *qkv, int64_t T, int heads, const aqt_cache &c, const int32_t *count, int left, int right,
                                   float *ctx, uint32_t *absmax, void *ws, hipStream_t st);

}  // namespace aqt
