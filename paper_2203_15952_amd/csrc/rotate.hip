// Queries and keys of projected rows normalised per head and rotated by their frame's position, in one pass, and its gradient.
// A row holds `heads` queries, `kv_heads` keys and `kv_heads` values of dh columns.  For every query and key head x:
//   n = x / sqrt(mean(x^2) + eps) * gamma          (norm; gamma shared by the heads, one for queries, one for keys)
//   (a, b) -> (a cos - b sin, a sin + b cos)       for the pairs (a, b) of the first `rot` columns, angle = 2 pi frame turns[i]
// and backward, with u the upstream gradient rotated back by the same angles and x^ = x / sqrt(mean(x^2) + eps):
//   dgamma = sum over rows and heads of u x^;   g = u gamma;   dx = (g - x^ mean(g x^)) / sqrt(mean(x^2) + eps).
// The normaliser is formed again from x (it is in registers), so the forward keeps nothing.
//
// Memory bounds both directions: a row is read once and written once.  A group of LANES lanes owns one head at a time and a
// lane the same columns of every head, so the gains' gradients and the cosines stay in registers while the group walks the
// heads of its row; the wavefronts walk the rows side by side.  A lane's columns are whole pairs, so rotating takes no exchange: for
// halves (i, i + rot / 2) the 16-byte pieces at j and rot / 8 + j, for neighbours (2 i, 2 i + 1) two adjacent pieces.  Heads
// that are not whole pieces, or not aligned, or whose rotated halves are not, meet their pairs' other halves in LDS (`Apart`).
//
// The angle is exact where it matters: frame * turns in float64, reduced there to an eighth of a turn around the nearest
// quarter, and only that remainder goes on in float32 (a position of a million frames costs no accuracy; in float32 its
// angle would be off by 0.06).
#include "lanes.h"

namespace aqt {
namespace {

constexpr int kThreads = 256;
constexpr int kBlocks = 16384;      // one row to a wavefront up to there (128 x 512 rows of 1024 columns, forward: 113 us with 2048, 97)
constexpr int kFoldBlocks = 1024;   // where every workgroup leaves column sums behind: what fits the chip (gradient 144 us, 152 with 4096)
constexpr int kFwdHeads = 2, kBwdHeads = 1;   // heads of a lane whose loads are in flight together (two backward: 44 -> 52 us, fewer wavefronts fit)
// Terms of a lane that are added up in float32 before they go to float64 sums: so the error of a gain's gradient does not grow with the
// rows (65536 rows of 8 heads: 1e-7 of it, a million: 3.6e-7 with float32 throughout).  Float64 in registers from the first term takes
// them from the wavefronts (12800 rows of 1536, halves of 30 columns, both directions: 77 us, 90 so); handing over every 4 terms instead
// of 8 costs where a lane has no more than that (12800 rows of 1536, whole heads rotated, both directions: 75 us, 77 so).
constexpr int kInFloat = 8;
constexpr int kMaxPairs = 64;                 // of the widest head
typedef float v4f __attribute__((ext_vector_type(4)));

struct RotateGeom {
  int64_t T, M, ld;         // frames per utterance, rows, columns of a row
  int heads, kv_heads, dh;
  int rot;                  // columns that are rotated
  int norm, in_place;       // in place: values are where they belong already
  int per_row;              // groups of lanes that share a row: a power of two
  int64_t stride;           // rows that all wavefronts take at a time
  int64_t stride_b, stride_t;   // ... in utterances and frames
  float eps;
  const double *turns;
  const int64_t *first;     // nullable: frame number of every utterance's first row
  const float *gamma[2];    // queries, keys; nullable
};

struct __attribute__((aligned(8))) Angle {
  float c, s;
};

// cos and sin of 2 pi x.  x = (quarter + r) / 4 with |r| <= 1/2; the next terms of the Taylor series at pi / 4 are 2e-9 (sine,
// behind x^9) and 1.2e-10 (cosine, behind x^10).
__device__ __forceinline__ Angle angle_of(double turn) {
  const double q = rint(4.0 * turn);
  const float r = static_cast<float>(4.0 * turn - q) * 1.57079632679489662f;
  const int quarter = static_cast<int>(q - 4.0 * rint(0.25 * q)) & 3;   // -2 .. 2, mod 4
  const float z = r * r;
  float s = fmaf(z, 2.7557319224e-6f, -1.9841269841e-4f);
  s = fmaf(z, s, 8.3333333333e-3f);
  s = fmaf(z, s, -1.6666666667e-1f);
  s = fmaf(r * z, s, r);
  float c = fmaf(z, -2.7557319224e-7f, 2.4801587302e-5f);
  c = fmaf(z, c, -1.3888888889e-3f);
  c = fmaf(z, c, 4.1666666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.0f);
  const float cc = quarter & 1 ? s : c, ss = quarter & 1 ? c : s;
  return Angle{quarter == 1 || quarter == 2 ? -cc : cc, quarter >= 2 ? -ss : ss};
}

// Eight columns of a head in two 16-byte pieces: lane j of the group.
template <int L, bool HALVES>
struct Pieces {
  static constexpr int LANES = L, N = 8, ANGLES = 4, PAIRS = 4 * L, SCRATCH = 4;   // PAIRS: of a head, at most
  int at[2];       // the pieces' first columns
  bool has[2];
  int pair;        // the first of this lane's four pairs
  int pairs;       // ... and how many of them are rotated
  __device__ __forceinline__ Pieces(int j, int dh, int rot) {
    const int half = rot >> 3;   // pieces in half of the rotated columns
    pair = 4 * j;
    pairs = (rot >> 1) - pair;
    if (HALVES) {
      at[0] = j < half ? 4 * j : 8 * j;            // behind the rotated ones: pieces 2 half + 2 (j - half)
      at[1] = j < half ? 4 * (j + half) : at[0] + 4;
    } else {
      at[0] = 8 * j;
      at[1] = 8 * j + 4;
    }
    has[0] = at[0] < dh;
    has[1] = at[1] < dh;
  }
  __device__ __forceinline__ int column(int i) const { return at[i >> 2] + (i & 3); }
  __device__ __forceinline__ bool own(int i) const { return has[i >> 2]; }
  __device__ __forceinline__ int pair_of(int i) const { return pair + i; }
  __device__ __forceinline__ void load(float (&x)[N], const float *p, bool on) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
      if (on && has[h]) v = *reinterpret_cast<const v4f *>(p + at[h]);
      x[4 * h] = v.x; x[4 * h + 1] = v.y; x[4 * h + 2] = v.z; x[4 * h + 3] = v.w;
    }
  }
  __device__ __forceinline__ void load_gains(float (&x)[N], const float *p) const {   // 128 of them, whatever the head
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const v4f v = *reinterpret_cast<const v4f *>(p + (has[h] ? at[h] : 0));
      x[4 * h] = v.x; x[4 * h + 1] = v.y; x[4 * h + 2] = v.z; x[4 * h + 3] = v.w;
    }
  }
  __device__ __forceinline__ void store(const float (&x)[N], float *p) const {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (has[h]) *reinterpret_cast<v4f *>(p + at[h]) = v4f{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
  }
  __device__ __forceinline__ void turn(float (&x)[N], const Angle (&t)[ANGLES], bool back, float *) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int ia = HALVES ? i : 2 * i, ib = HALVES ? i + 4 : 2 * i + 1;
      const float a = x[ia], b = x[ib], s = back ? -t[i].s : t[i].s;
      x[ia] = i < pairs ? a * t[i].c - b * s : a;
      x[ib] = i < pairs ? a * s + b * t[i].c : b;
    }
  }
};

// Eight columns of a head whose pairs another lane may hold the other half of: any width, alignment and number of rotated columns.
// VEC: two 16-byte pieces, on 16-byte boundaries, where only the rotated halves are no whole pieces; otherwise every L-th column,
// so that the lanes of a load are neighbours.
template <int L, bool HALVES, bool VEC>
struct Apart {
  static_assert(HALVES || !VEC, "neighbours on 16-byte boundaries: Pieces");
  static constexpr int LANES = L, N = 8, ANGLES = 8, PAIRS = 4 * L, SCRATCH = HALVES ? 512 : 4;
  int j, dh, rot;
  __device__ __forceinline__ Apart(int j_, int dh_, int rot_) : j(j_), dh(dh_), rot(rot_) {}
  __device__ __forceinline__ int column(int i) const { return VEC ? 4 * j + (i & 3) + (i >> 2) * 4 * L : j + L * i; }
  __device__ __forceinline__ bool own(int i) const { return column(i) < dh; }
  __device__ __forceinline__ int pair_of(int i) const {
    const int c = column(i);
    return c >= rot ? 0 : HALVES ? (c < (rot >> 1) ? c : c - (rot >> 1)) : c >> 1;
  }
  __device__ __forceinline__ void load(float (&x)[N], const float *p, bool on) const {
    if constexpr (VEC) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (on && own(4 * h)) v = *reinterpret_cast<const v4f *>(p + column(4 * h));
        x[4 * h] = v.x; x[4 * h + 1] = v.y; x[4 * h + 2] = v.z; x[4 * h + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = on && own(i) ? p[column(i)] : 0.0f;
    }
  }
  __device__ __forceinline__ void load_gains(float (&x)[N], const float *p) const {   // 128 of them, whatever the head
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = p[column(i)];
  }
  __device__ __forceinline__ void store(const float (&x)[N], float *p) const {
    if constexpr (VEC) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (own(4 * h)) *reinterpret_cast<v4f *>(p + column(4 * h)) = v4f{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (own(i)) p[column(i)] = x[i];
    }
  }
  // head: the group's 8 L words of LDS, through which the halves meet
  __device__ __forceinline__ void turn(float (&x)[N], const Angle (&t)[ANGLES], bool back, float *head) const {
    const int half = rot >> 1;
    float y[N];
    if constexpr (HALVES) {
#pragma unroll
      for (int i = 0; i < N; ++i) head[column(i)] = x[i];
      wave_lds_order();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = column(i);
        y[i] = head[c >= rot ? c : c < half ? c + half : c - half];
      }
      wave_lds_order();   // read before the next head's are written
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] = of_neighbour(x[i]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = column(i);
      const bool second = HALVES ? c >= half : c & 1;
      const float s = second == back ? -t[i].s : t[i].s;
      x[i] = c >= rot ? x[i] : x[i] * t[i].c + y[i] * s;
    }
  }
};

// 1 / rms of a head from a lane's columns v.  Heads whose squares float32 does not hold (their mean and eps under 2^-100, of which
// the instruction takes what lies under 2^-126 for zeros, or infinite) are scaled by a power of two first, v with them: by h h, and 1 / rms
// is h h times the result.  A branch that the wavefront steps over where none of its heads is such.
template <int L, int N>
__device__ __forceinline__ float inverse_rms(float (&v)[N], float inv, float eps, bool value, float &h) {
  auto mean = [&] {
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) ss = fmaf(v[i], v[i], ss);
    return group_sum<L>(ss) * inv;
  };
  const float own = mean() + eps;   // (all lanes)
  float m = value ? 1.0f : own;     // a value beside keys stays as it is
  h = 1.0f;
  if (__any(!(m >= 0x1p-100f && m < __builtin_inff()))) {
    h = m >= 0x1p-100f && m < __builtin_inff() ? 1.0f : m < 0x1p-100f ? 0x1p48f : 0x1p-48f;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] *= h * h;
    m = mean() + eps * (h * h) * (h * h);
  }
  return __builtin_amdgcn_rsqf(m);
}

// BWD: y is the upstream gradient, out the gradient with respect to x; GAINS: part [workgroups][2][dh] column sums (a kernel of its own,
// for the registers of their sums: 32 x 400 rows of 1536 columns without them 33 us, and 36 in a kernel for both).
template <class F, bool BWD, bool GAINS = BWD>
__global__ __launch_bounds__(kThreads, GAINS ? 4 : BWD ? 1 : 5) void rotate_kernel(const float *x, const float *y, RotateGeom g, float *out, float *part) {
  constexpr int L = F::LANES, N = F::N, GROUPS = 64 / L, U = BWD ? kBwdHeads : kFwdHeads, PAIRS = F::PAIRS;
  const int tid = static_cast<int>(threadIdx.x), lane = tid & 63, group = lane / L, j = lane % L;
  const F f(j, g.dh, g.rot);
  const int sub = group % g.per_row, row_of = group / g.per_row, rows_at_once = GROUPS / g.per_row;
  const int turned = g.heads + g.kv_heads, all = turned + (g.in_place ? 0 : g.kv_heads);

  // In LDS: gains and turns (in registers they cost the kernel half of its wavefronts), and the angles of a row, which the lanes
  // that share it form once between them.
  __shared__ __attribute__((aligned(16))) float gains[2][128];
  __shared__ double turns[kMaxPairs];
  __shared__ Angle angles[kThreads / 64][64 * 4];
  __shared__ __attribute__((aligned(16))) float heads[kThreads / 64][F::SCRATCH];
  if (tid < 2 * 128) {
    const int w = tid >> 7, c = tid & 127;
    gains[w][c] = g.gamma[w] && c < g.dh ? g.gamma[w][c] : 1.0f;
  }
  if (tid < kMaxPairs) turns[tid] = tid < g.rot / 2 ? g.turns[tid] : 0.0;
  const int row_lanes = L * g.per_row, place = sub * L + j;
  Angle *const row_angles = angles[tid >> 6] + row_of * PAIRS;
  float *const head = F::SCRATCH > 4 ? heads[tid >> 6] + group * 8 * L : nullptr;
  float dgain[2][N];   // GAINS
#pragma unroll
  for (int w = 0; w < 2; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) dgain[w][i] = 0.0f;
  __shared__ double sums[kThreads / 64][2][GAINS ? 128 : 1];
  if (GAINS)
    for (int i = tid; i < kThreads / 64 * 2 * 128; i += kThreads) (&sums[0][0][0])[i] = 0.0;
  __syncthreads();
  // What the lanes have added up, over the groups of the wavefront, to its sums in float64.
  auto hand_over = [&](auto in_between) {
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float s = dgain[w][i];
#pragma unroll
        for (int off = L; off < 64; off <<= 1) s += __shfl_xor(s, off, 64);
        if (group == 0 && f.own(i)) sums[tid >> 6][w][f.column(i)] += static_cast<double>(s);
        dgain[w][i] = 0.0f;
        if (in_between()) __builtin_amdgcn_sched_barrier(0);   // one after the other: side by side they take registers from the rows
      }
  };
  int in_float = 0;
  const int steps = (g.heads + g.per_row - 1) / g.per_row;

  // All wavefronts walk the rows side by side: what is in flight at a time is one piece of memory
  // (32 x 400 rows of 1536 columns, forward, with a run of rows to each instead: 32 us, 26.5 so).
  const int64_t wave = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + (tid >> 6);
  const int64_t begin = wave * rows_at_once, own = begin + row_of;
  const float inv = 1.0f / static_cast<float>(g.dh);
  int64_t b, t;
  if (g.M >> 30 == 0) {   // (a divide of 64 bits takes longer than the rest of a short call)
    const uint32_t q = static_cast<uint32_t>(own) / static_cast<uint32_t>(g.T);
    b = q;
    t = static_cast<uint32_t>(own) - q * static_cast<uint32_t>(g.T);
  } else {
    b = own / g.T;
    t = own - b * g.T;
  }
  for (int64_t m0 = begin; m0 < g.M; m0 += g.stride) {
    if (GAINS) {
      if (in_float >= kInFloat) {
        in_float = 0;
        hand_over([] { return true; });
      }
      in_float += steps;
    }
    const int64_t m = m0 + row_of;
    const bool row_ok = m < g.M;
    const double frame = row_ok ? static_cast<double>((g.first ? g.first[b] : 0) + t) : 0.0;
    const float *const xr = x + m * g.ld, *const yr = BWD ? y + m * g.ld : nullptr;
    float *const outr = out + m * g.ld;
    Angle a[F::ANGLES];
    for (int h0 = 0; h0 < all; h0 += U * g.per_row) {   // the same number of steps for every lane of the wavefront
      // U heads at a time, all of their loads in front of what is computed
      float v[U][N], w[U][N];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int h = h0 + k * g.per_row + sub;
        const bool on = row_ok && h < all;
        const int64_t at = static_cast<int64_t>(h) * g.dh;
        if (BWD) f.load(w[k], yr + at, on);
        if (!BWD || g.norm) f.load(v[k], xr + at, on && (!BWD || h < turned));
      }
      if (h0 == 0) {
#pragma unroll 1
        for (int at = place; at < PAIRS; at += row_lanes) row_angles[at] = angle_of(frame * turns[at]);
        wave_lds_order();
#pragma unroll
        for (int i = 0; i < F::ANGLES; ++i) a[i] = row_angles[f.pair_of(i)];
        wave_lds_order();   // read before the next row's are written
      }
#pragma unroll
      for (int k = 0; k < U; ++k) {
        if (h0 + k * g.per_row >= all) break;
        const int h = h0 + k * g.per_row + sub;
        const bool on = row_ok && h < all, value = h >= turned, query = h < g.heads;
        float u[N];
        if (h0 + k * g.per_row >= turned) {   // nothing but values
#pragma unroll
          for (int i = 0; i < N; ++i) u[i] = BWD ? w[k][i] : v[k][i];
        } else if (!BWD) {
          if (g.norm) {
            float gain[N], half_scale;
            f.load_gains(gain, gains[query ? 0 : 1]);
            const float r = inverse_rms<L>(v[k], inv, g.eps, value, half_scale);
#pragma unroll
            for (int i = 0; i < N; ++i) u[i] = v[k][i] * r * gain[i];
          } else {
#pragma unroll
            for (int i = 0; i < N; ++i) u[i] = v[k][i];
          }
          f.turn(u, a, false, head);
#pragma unroll
          for (int i = 0; i < N; ++i) u[i] = value ? v[k][i] : u[i];
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) u[i] = w[k][i];
          f.turn(u, a, true, head);
          if (g.norm) {
            float gain[N], half_scale;
            f.load_gains(gain, gains[query ? 0 : 1]);
            const float r = inverse_rms<L>(v[k], inv, g.eps, value, half_scale);
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
              v[k][i] *= r;
              const float mine = on && !value ? u[i] * v[k][i] : 0.0f;
              if (GAINS) {
                dgain[0][i] += query ? mine : 0.0f;
                dgain[1][i] += query ? 0.0f : mine;
              }
              u[i] *= gain[i];
              dot = fmaf(u[i], v[k][i], dot);
            }
            dot = group_sum<L>(dot) * inv;
#pragma unroll
            for (int i = 0; i < N; ++i) u[i] -= v[k][i] * dot;
            if (__any(half_scale != 1.0f)) {   // one half in front of r, one behind: the product in between stays a number
#pragma unroll
              for (int i = 0; i < N; ++i) u[i] = u[i] * half_scale * r * half_scale;
            } else {
#pragma unroll
              for (int i = 0; i < N; ++i) u[i] *= r;
            }
          }
#pragma unroll
          for (int i = 0; i < N; ++i) u[i] = value ? w[k][i] : u[i];
        }
        if (on) f.store(u, outr + static_cast<int64_t>(h) * g.dh);
      }
    }
    b += g.stride_b;
    t += g.stride_t;
    if (t >= g.T) {
      t -= g.T;
      ++b;
    }
  }
  if constexpr (GAINS) {
    hand_over([] { return false; });
    __syncthreads();
    if (tid < 2 * g.dh) {
      const int w = tid >= g.dh, c = w ? tid - g.dh : tid;
      double s = 0.0;
      for (int k = 0; k < kThreads / 64; ++k) s += sums[k][w][c];
      part[static_cast<int64_t>(blockIdx.x) * 2 * g.dh + tid] = static_cast<float>(s);
    }
  }
}

// dgamma[c] = sum over workgroups, in a fixed order, in float64: sixteen columns to a workgroup, 64 threads to a column, each
// with eight loads in flight.
constexpr int kFoldThreads = 1024, kFoldSlices = kFoldThreads / 16;
__global__ __launch_bounds__(kFoldThreads) void rotate_fold_kernel(const float *__restrict__ part, int parts, int dh, float *__restrict__ dgq,
                                                                   float *__restrict__ dgk) {
  __shared__ double sums[kFoldSlices][16];
  const int c = static_cast<int>(blockIdx.x) * 16 + static_cast<int>(threadIdx.x & 15u), slice = static_cast<int>(threadIdx.x >> 4);
  const int cc = c < 2 * dh ? c : 2 * dh - 1;
  double s = 0.0;
  for (int p = slice; p < parts; p += 8 * kFoldSlices) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = part[static_cast<int64_t>(min(p + u * kFoldSlices, parts - 1)) * 2 * dh + cc];
#pragma unroll
    for (int u = 0; u < 8; ++u) s += p + u * kFoldSlices < parts ? static_cast<double>(v[u]) : 0.0;
  }
  sums[slice][threadIdx.x & 15u] = s;
  __syncthreads();
  for (int half = kFoldSlices / 2; half > 0; half >>= 1) {
    if (slice < half) sums[slice][threadIdx.x & 15u] += sums[slice + half][threadIdx.x & 15u];
    __syncthreads();
  }
  if (slice == 0 && c < 2 * dh) {
    float *const to = c < dh ? dgq : dgk;
    if (to) to[c < dh ? c : c - dh] = static_cast<float>(sums[0][threadIdx.x & 15u]);
  }
}

__global__ void rotation_turns_kernel(int pairs, double log2_base, double *__restrict__ turns) {
  const int i = static_cast<int>(threadIdx.x);
  if (i < pairs) turns[i] = exp2(-log2_base * static_cast<double>(i) / static_cast<double>(pairs)) * 0.15915494309189533577;
}

unsigned rotate_blocks(int64_t M, int rows_at_once, int most) {
  const int64_t want = cdiv(cdiv(M, rows_at_once), kThreads / 64);
  return static_cast<unsigned>(want < most ? want : most);
}

template <class F, bool BWD>
aqt_status launch_as(const float *x, const float *y, RotateGeom g, float *out, float *part, hipStream_t st, unsigned *blocks) {
  g.per_row = 1;   // by all heads, in place too: the same lanes add up the same terms
  while (g.per_row < 64 / F::LANES && g.per_row < g.heads + 2 * g.kv_heads) g.per_row *= 2;
  const int rows_at_once = 64 / F::LANES / g.per_row;
  *blocks = rotate_blocks(g.M, rows_at_once, part ? kFoldBlocks : kBlocks);
  g.stride = static_cast<int64_t>(*blocks) * (kThreads / 64) * rows_at_once;
  g.stride_b = g.stride / g.T;
  g.stride_t = g.stride % g.T;
  // The gradient without gains' has registers for seven wavefronts to a SIMD, but memory is better served by the streams of five, whose
  // workgroups this much LDS leaves room for (128 x 512 rows of 1024 columns: 137 us with seven, 130 so; smaller calls equal).
  constexpr size_t kRoom = 20480;
  auto kern = part ? rotate_kernel<F, BWD, BWD> : rotate_kernel<F, BWD, false>;   // (forward: the same)
  kern<<<*blocks, kThreads, BWD && !part ? kRoom : 0, st>>>(x, y, g, out, part);
  AQT_HIP(hipGetLastError());
  return AQT_OK;
}

template <bool HALVES, bool BWD>
aqt_status launch_paired(const float *x, const float *y, const RotateGeom &g, float *out, float *part, bool aligned, hipStream_t st,
                         unsigned *blocks) {
  // Whole 16-byte pieces; in halves a lane has both of a pair only where either half is whole pieces too (25628 rows of 1536, heads of 64
  // with 24 rotated columns: 61 us; with 18, whose pairs meet in LDS, 62, and 112 with single columns).
  const bool pieces = aligned && g.dh % 4 == 0;
  if (pieces && (!HALVES || g.rot % 8 == 0)) {
    if (g.dh <= 32) return launch_as<Pieces<4, HALVES>, BWD>(x, y, g, out, part, st, blocks);
    if (g.dh <= 64) return launch_as<Pieces<8, HALVES>, BWD>(x, y, g, out, part, st, blocks);
    return launch_as<Pieces<16, HALVES>, BWD>(x, y, g, out, part, st, blocks);
  }
  if constexpr (HALVES) {
    if (pieces) {
      if (g.dh <= 32) return launch_as<Apart<4, true, true>, BWD>(x, y, g, out, part, st, blocks);
      if (g.dh <= 64) return launch_as<Apart<8, true, true>, BWD>(x, y, g, out, part, st, blocks);
      return launch_as<Apart<16, true, true>, BWD>(x, y, g, out, part, st, blocks);
    }
  }
  if (g.dh <= 32) return launch_as<Apart<4, HALVES, false>, BWD>(x, y, g, out, part, st, blocks);
  if (g.dh <= 64) return launch_as<Apart<8, HALVES, false>, BWD>(x, y, g, out, part, st, blocks);
  return launch_as<Apart<16, HALVES, false>, BWD>(x, y, g, out, part, st, blocks);
}

RotateGeom rotate_geom(int64_t B, int64_t T, const aqt_qk_norm_rotate &s, const int64_t *first, bool in_place) {
  RotateGeom g;
  g.T = T; g.M = B * T;
  g.ld = (static_cast<int64_t>(s.heads) + 2 * static_cast<int64_t>(s.kv_heads)) * s.dh;
  g.heads = s.heads; g.kv_heads = s.kv_heads; g.dh = s.dh; g.rot = s.rot;
  g.norm = s.norm; g.in_place = in_place; g.per_row = 1; g.stride = g.stride_b = g.stride_t = 0;
  g.eps = s.eps; g.turns = s.turns; g.first = first;
  g.gamma[0] = s.gamma_q; g.gamma[1] = s.gamma_k;
  return g;
}

bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

size_t rotate_bwd_ws_bytes(int dh) { return align_up(static_cast<size_t>(kFoldBlocks) * 2 * dh * sizeof(float), 256); }

aqt_status launch_rotation_turns(int rot, double base, double *turns, hipStream_t st) {
  rotation_turns_kernel<<<1, 64, 0, st>>>(rot / 2, log2(base), turns);
  AQT_HIP(hipGetLastError());
  return AQT_OK;
}

aqt_status launch_rotate_fwd(const float *qkv, int64_t B, int64_t T, const aqt_qk_norm_rotate &s, const int64_t *first, float *out,
                             hipStream_t st) {
  const RotateGeom g = rotate_geom(B, T, s, first, out == qkv);
  const bool al = aligned16(qkv) && aligned16(out);
  unsigned blocks;
  return s.pairing == AQT_ROTATE_HALVES ? launch_paired<true, false>(qkv, nullptr, g, out, nullptr, al, st, &blocks)
                                        : launch_paired<false, false>(qkv, nullptr, g, out, nullptr, al, st, &blocks);
}

aqt_status launch_rotate_bwd(const float *qkv, const float *dout, int64_t B, int64_t T, const aqt_qk_norm_rotate &s, const int64_t *first,
                             float *dqkv, float *dgamma_q, float *dgamma_k, void *ws, hipStream_t st) {
  const RotateGeom g = rotate_geom(B, T, s, first, dqkv == dout);
  const bool al = aligned16(dout) && aligned16(dqkv) && aligned16(qkv);
  float *const part = dgamma_q || dgamma_k ? static_cast<float *>(ws) : nullptr;
  unsigned blocks;
  AQT_TRY((s.pairing == AQT_ROTATE_HALVES ? launch_paired<true, true>(qkv, dout, g, dqkv, part, al, st, &blocks)
                                          : launch_paired<false, true>(qkv, dout, g, dqkv, part, al, st, &blocks)));
  if (!part) return AQT_OK;
  rotate_fold_kernel<<<static_cast<unsigned>(cdiv(2 * s.dh, 16)), kFoldThreads, 0, st>>>(part, static_cast<int>(blocks), s.dh, dgamma_q, dgamma_k);
  AQT_HIP(hipGetLastError());
  return AQT_OK;
}

}  // namespace aqt
