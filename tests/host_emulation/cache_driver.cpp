// Driver of the host emulation of the kernels around positions and the quantized cache: the test splices cache.h, the kernels of
// cache.hip (namespace cache_), attention_cached.hip (attend), attention_cached_few.hip (few) and rotate.hip (turn) in front of this file.  Buffers are heap blocks of exactly the
// sizes the kernels may touch, the cache starts out as NaNs in every reading, and results are compared with plain float64 loops.
namespace aqt {
static int bad = 0;
static uint32_t seed = 7u;
static float uniform() { seed = seed * 1664525u + 1013904223u; return (float)(seed >> 8) / 8388608.0f - 1.0f; }
static void complain(const char *what) { printf("  MISMATCH %s\n", what); bad = 1; }

struct Ref {   // what the streams' caches stand for: value, by stream, frame, head, column
  std::vector<std::vector<std::vector<double>>> k, v;   // [stream][frame][kv_heads * dh]
};
static void quantized(const float *x, int dh, int qmax, std::vector<double> &to, int at) {
  float m = 0;
  for (int i = 0; i < dh; ++i) m = std::max(m, fabsf(x[i]));
  const float s = m / (float)qmax;
  for (int i = 0; i < dh; ++i) {
    const float t = s == 0.0f ? 0.0f : x[i] / s;
    to[at + i] = (double)(std::min(std::max(floorf(t + 0.5f), (float)-qmax), (float)qmax) * s);
  }
}

template <int L, bool VEC> static void append(unsigned grid, const float *qkv, const CacheGeom &g, int64_t T, int heads, const int32_t *count, int run_, int per, int32_t *st) {
  run(grid, 256, 0, [&] { cache_::cache_append_kernel<L, VEC>(qkv, g, T, heads, count, run_, per, st); });
}
template <int L, bool VEC> static void read_(unsigned grid, const CacheGeom &g, int64_t pend, const int32_t *count, const int64_t *first, int64_t n, int run_, int per, float *k, float *v) {
  run(grid, 256, 0, [&] { cache_::cache_read_kernel<L, VEC>(g, pend, count, first, n, run_, per, k, v); });
}

template <int DT, bool PACKED> static void attention_as(const CacheGeom &g, int rows, bool own, const float *qkv, const CachedGeom &a, const int32_t *count, float *ctx, uint32_t *am, float *part) {
  if (own) attend::attention_cached_kernel<DT, PACKED, true>(qkv, g, a, count, ctx, am, part);
  else if (rows == 16) attend::attention_cached_kernel<DT, PACKED, false>(qkv, g, a, count, ctx, am, part);
  else if (rows == 1) few::attention_cached_few_kernel<DT, PACKED, 1>(qkv, g, a, count, ctx, am, part);
  else if (rows == 2) few::attention_cached_few_kernel<DT, PACKED, 2>(qkv, g, a, count, ctx, am, part);
  else few::attention_cached_few_kernel<DT, PACKED, 4>(qkv, g, a, count, ctx, am, part);
}
static void attention(const CacheGeom &g, int rows, bool own, int cols, const float *qkv, const CachedGeom &a, const int32_t *count, float *ctx, uint32_t *am, float *part) {
  if (g.packed) (cols == 32 ? attention_as<2, true> : cols == 64 ? attention_as<4, true> : attention_as<8, true>)(g, rows, own, qkv, a, count, ctx, am, part);
  else (cols == 32 ? attention_as<2, false> : cols == 64 ? attention_as<4, false> : attention_as<8, false>)(g, rows, own, qkv, a, count, ctx, am, part);
}
template <int ROWS> static void join_as(int cols, const float *part, const CacheGeom &g, const CachedGeom &a, const int32_t *count, float *ctx, uint32_t *am) {
  if (cols == 32) attend::attention_cached_join_kernel<ROWS, 32>(part, g, a, count, ctx, am);
  else if (cols == 64) attend::attention_cached_join_kernel<ROWS, 64>(part, g, a, count, ctx, am);
  else attend::attention_cached_join_kernel<ROWS, 128>(part, g, a, count, ctx, am);
}
static void join(int rows, int cols, const float *part, const CacheGeom &g, const CachedGeom &a, const int32_t *count, float *ctx, uint32_t *am) {
  (rows == 1 ? join_as<1> : rows == 2 ? join_as<2> : rows == 4 ? join_as<4> : join_as<16>)(cols, part, g, a, count, ctx, am);
}
static void one(int streams, int64_t capacity, int heads, int kv, int dh, int bits, std::vector<int> steps, std::vector<std::pair<int, int>> windows, bool ragged) {
  printf("case %d streams, capacity %ld, heads %d / %d, dh %d, bits %d\n", streams, (long)capacity, heads, kv, dh, bits); fflush(stdout);
  const int cols = (heads + 2 * kv) * dh, qmax = (1 << (bits - 1)) - 1, group = heads / kv;
  aqt_cache c{};
  c.streams = streams; c.capacity = capacity; c.kv_heads = kv; c.dh = dh; c.bits = bits;
  CacheGeom g = cache_geom(c);
  const size_t bytes = (size_t)streams * kv * g.tiles * g.tile_bytes;
  g.data = (uint8_t *)aligned_alloc(64, (bytes + 63) / 64 * 64);   // tiles are whole 64-byte pieces
  memset(g.data, 0xFF, bytes);
  int64_t *length = (int64_t *)malloc(8 * streams);
  for (int b = 0; b < streams; ++b) length[b] = 0;
  g.length = length;
  Ref ref;
  ref.k.resize(streams); ref.v.resize(streams);
  int32_t status = 0;
  for (int T : steps) {
    const size_t n = (size_t)streams * T * cols;
    float *qkv = (float *)malloc(n * 4);
    for (size_t i = 0; i < n; ++i) qkv[i] = 2.0f * uniform();
    for (int i = 0; i < dh; ++i) qkv[(heads + kv - 1) * dh + i] = 0.0f;   // a key of zeros
    int32_t *count = nullptr;
    if (ragged || length[0] == 0) {   // streams of different lengths in any case
      count = (int32_t *)malloc(4 * streams);
      for (int b = 0; b < streams; ++b) count[b] = (3 * b + T / 2) % (T + 1);
      count[0] = T + 5;   // as many as there are
      if (streams > 2) count[2] = -1;
    }
    const int64_t most = std::min<int64_t>(T, capacity);
    const int L = cache_::lanes_of(dh), per = (int)cache_::cut_of(g, most).blocks;
    const bool vec = dh % 4 == 0;
    auto ap = L == 4 ? (vec ? append<4, true> : append<4, false>) : L == 8 ? (vec ? append<8, true> : append<8, false>) : (vec ? append<16, true> : append<16, false>);
    ap((unsigned)(per * streams), qkv, g, T, heads, count, cache_::cut_of(g, most).log2_run, per, &status);
    std::vector<int> cnt(streams);
    for (int b = 0; b < streams; ++b) {
      cnt[b] = count ? std::min(std::max(count[b], 0), T) : T;
      for (int t = 0; t < cnt[b]; ++t) {
        std::vector<double> k(kv * dh), v(kv * dh);
        for (int h = 0; h < kv; ++h) {
          quantized(qkv + (size_t)(b * T + t) * cols + (heads + h) * dh, dh, qmax, k, h * dh);
          quantized(qkv + (size_t)(b * T + t) * cols + (heads + kv + h) * dh, dh, qmax, v, h * dh);
        }
        ref.k[b].push_back(k); ref.v[b].push_back(v);
      }
    }
    // read back: more frames than there are on either side
    const int64_t nr = T + 9;
    int64_t *first = (int64_t *)malloc(8 * streams);
    for (int b = 0; b < streams; ++b) first[b] = length[b] - 3;
    float *rk = (float *)malloc(streams * nr * kv * dh * 4), *rv = (float *)malloc(streams * nr * kv * dh * 4);
    memset(rk, 0xFF, streams * nr * kv * dh * 4); memset(rv, 0xFF, streams * nr * kv * dh * 4);
    const int rper = (int)cache_::cut_of(g, nr).blocks;
    auto rd = L == 4 ? (vec ? read_<4, true> : read_<4, false>) : L == 8 ? (vec ? read_<8, true> : read_<8, false>) : (vec ? read_<16, true> : read_<16, false>);
    rd((unsigned)(rper * streams), g, T, count, first, nr, cache_::cut_of(g, nr).log2_run, rper, rk, rv);
    for (int b = 0; b < streams; ++b) for (int64_t i = 0; i < nr; ++i) {
      const int64_t p = first[b] + i, end = (int64_t)ref.k[b].size();
      for (int e = 0; e < kv * dh; ++e) {
        const bool held = p >= 0 && p < end && p >= end - capacity;
        const size_t at = (size_t)(b * nr + i) * kv * dh + e;
        if (rk[at] != (held ? (float)ref.k[b][p][e] : 0.0f)) { complain("keys read back"); i = nr; b = streams; break; }
        if (rv[at] != (held ? (float)ref.v[b][p][e] : 0.0f)) { complain("values read back"); i = nr; b = streams; break; }
      }
    }
    free(first); free(rk); free(rv);
    // attention of the new frames
    for (auto [left, right] : windows) {
      if (T > 32 && left != windows[0].first) continue;
      CachedGeom a{};
      a.T = T; a.ld = cols; a.heads = heads; a.group = group;
      a.left = left; a.right = right; a.scale_log2e = (float)(1.4426950408889634 / sqrt((double)dh));
      // in tiles of 16 rows, and where they are few, each in its own place; by itself, and joined from three parts; a tile to a wavefront
      for (int form = 0; form < 5; ++form) {
        const int few_rows = T * group <= kFewRows ? (T * group == 1 ? 1 : T * group == 2 ? 2 : 4) : 0, rows = form & 2 ? few_rows : 16;
        const bool own = form == 4;
        if (rows == 0 || (T > 32 && form == 0)) continue;
        a.splits = form & 1 ? 3 : 1;
        a.row_tiles = (T * group + rows - 1) / rows;
        const int groups = streams * kv * a.row_tiles, COLS = attend::cols_of(dh), splits = a.splits;
        float *ctx = (float *)malloc((size_t)streams * T * heads * dh * 4);
        const size_t pf = (size_t)groups * splits * ((rows * COLS + 2 * rows + 3) / 4 * 4);
        float *part = splits > 1 ? (float *)aligned_alloc(16, (pf * 4 + 15) / 16 * 16) : nullptr;
        for (size_t i = 0; i < (size_t)streams * T * heads * dh; ++i) ctx[i] = 77.0f;
        uint32_t am = 0;
        const unsigned grid = (unsigned)(own ? (groups + 3) / 4 : groups * splits);
        run(grid, 256, 0, [&] { attention(g, rows, own, COLS, qkv, a, count, ctx, &am, part); });
        if (part) run((unsigned)groups, 256, 0, [&] { join(rows, COLS, part, g, a, count, ctx, &am); });
        double worst = 0, largest = 0;
        for (int b = 0; b < streams; ++b) for (int t = 0; t < T; ++t) for (int h = 0; h < heads; ++h) {
          const float *got = ctx + ((size_t)(b * T + t) * heads + h) * dh;
          if (t >= cnt[b]) { for (int e = 0; e < dh; ++e) if (got[e] != 77.0f) { complain("a row that the stream did not bring"); break; } continue; }
          const int64_t end = (int64_t)ref.k[b].size(), f = length[b] + t;
          int64_t lo = std::max<int64_t>(0, end - capacity), hi = end - 1;
          if (left >= 0) lo = std::max(lo, f - left);
          if (right >= 0) hi = std::min(hi, f + right);
          // an error is measured against what the weights make of the largest value of every frame: they are integers relative
          // to the largest of them, whatever a column's own values are
          std::vector<double> ref_o(dh, 0.0), sc;
          double top = -1e300, sum = 0, mag = 1e-30;
          for (int64_t j = lo; j <= hi; ++j) {
            double d = 0;
            for (int e = 0; e < dh; ++e) d += ref.k[b][j][(h / group) * dh + e] * qkv[(size_t)(b * T + t) * cols + h * dh + e];
            sc.push_back(d / sqrt((double)dh)); top = std::max(top, sc.back());
          }
          for (int64_t j = lo; j <= hi; ++j) sum += exp(sc[j - lo] - top);
          for (int64_t j = lo; j <= hi; ++j) {
            const double w = exp(sc[j - lo] - top) / sum;
            double most = 0;
            for (int e = 0; e < dh; ++e) { const double x = ref.v[b][j][(h / group) * dh + e]; ref_o[e] += w * x; most = std::max(most, fabs(x)); }
            mag += w * most;
          }
          for (int e = 0; e < dh; ++e) { at_least(worst, fabs(got[e] - ref_o[e]) / mag); at_least(largest, (double)fabsf(got[e])); }
        }
        printf("  T %d window %d %d splits %d rows %d own %d: worst error / sum of magnitudes %.3g\n", T, left, right, splits, rows, own, worst);
        if (!(worst < 4e-6)) complain("attention");
        if (__float_as_uint((float)largest) != am) complain("absmax");
        free(ctx); free(part);
      }
    }
    for (int b = 0; b < streams; ++b) length[b] += cnt[b];
    free(qkv); free(count);
  }
  if (status) complain("status");
  free(g.data); free(length);
}

template <class F, bool BWD> static void turn_kernel(const float *x, const float *y, turn::RotateGeom g, float *out, float *part, int blocks) {
  g.per_row = 1;
  while (g.per_row < 64 / F::LANES && g.per_row < g.heads + 2 * g.kv_heads) g.per_row *= 2;
  const int rows = 64 / F::LANES / g.per_row;
  g.stride = 4 * blocks * rows;
  g.stride_b = g.stride / g.T;
  g.stride_t = g.stride % g.T;
  run((unsigned)blocks, 256, 0, [&] { turn::rotate_kernel<F, BWD>(x, y, g, out, part); });
}
// form 2: whole pieces with both of every pair; 1: whole pieces; 0: single columns
template <bool HALVES, bool BWD> static void turn_paired(const float *x, const float *y, const turn::RotateGeom &g, float *out, float *part, int form, int blocks) {
  if (form == 2) { if (g.dh <= 32) turn_kernel<turn::Pieces<4, HALVES>, BWD>(x, y, g, out, part, blocks); else if (g.dh <= 64) turn_kernel<turn::Pieces<8, HALVES>, BWD>(x, y, g, out, part, blocks); else turn_kernel<turn::Pieces<16, HALVES>, BWD>(x, y, g, out, part, blocks); }
  else if (form == 1) {
    if constexpr (HALVES) { if (g.dh <= 32) turn_kernel<turn::Apart<4, true, true>, BWD>(x, y, g, out, part, blocks); else if (g.dh <= 64) turn_kernel<turn::Apart<8, true, true>, BWD>(x, y, g, out, part, blocks); else turn_kernel<turn::Apart<16, true, true>, BWD>(x, y, g, out, part, blocks); }
  }
  else { if (g.dh <= 32) turn_kernel<turn::Apart<4, HALVES, false>, BWD>(x, y, g, out, part, blocks); else if (g.dh <= 64) turn_kernel<turn::Apart<8, HALVES, false>, BWD>(x, y, g, out, part, blocks); else turn_kernel<turn::Apart<16, HALVES, false>, BWD>(x, y, g, out, part, blocks); }
}
static void rotate_case(int64_t B, int64_t T, int heads, int kv, int dh, int rot, bool halves, bool norm, bool gains, bool first, bool in_place) {
  printf("rotate B %ld T %ld heads %d / %d dh %d rot %d halves %d norm %d gains %d\n", (long)B, (long)T, heads, kv, dh, rot, halves, norm, gains); fflush(stdout);
  const int cols = (heads + 2 * kv) * dh, np = rot / 2;
  const size_t n = (size_t)B * T * cols;
  auto floats = [](size_t k) { return (float *)malloc(k * 4); };
  float *x = floats(n), *dy = floats(n), *out = floats(n), *dx = floats(n), *gq = floats(dh), *gk = floats(dh), *dgq = floats(dh), *dgk = floats(dh);
  for (size_t i = 0; i < n; ++i) { x[i] = uniform(); dy[i] = uniform(); out[i] = dx[i] = NAN; }
  for (int i = 0; i < dh; ++i) { gq[i] = 1.0f + 0.3f * uniform(); gk[i] = 1.0f + 0.3f * uniform(); dgq[i] = dgk[i] = NAN; }
  double *turns = (double *)malloc(8 * (np ? np : 1));
  for (int i = 0; i < np; ++i) turns[i] = pow(10000.0, -(double)i / np) / (2 * M_PI);
  int64_t *f0 = (int64_t *)malloc(8 * B);
  for (int64_t b = 0; b < B; ++b) f0[b] = 100000 * b + 17;
  turn::RotateGeom g{};
  g.T = T; g.M = B * T; g.ld = cols; g.heads = heads; g.kv_heads = kv; g.dh = dh; g.rot = rot; g.norm = norm; g.in_place = 0; g.eps = 1e-6f;
  g.turns = np ? turns : nullptr; g.first = first ? f0 : nullptr; g.gamma[0] = gains ? gq : nullptr; g.gamma[1] = gains ? gk : nullptr;
  const int most = dh % 4 ? 0 : !halves || rot % 8 == 0 ? 2 : 1;
  for (int pieces = most; pieces >= 0; --pieces) for (int blocks : {1, 3}) {
    if ((blocks == 1 && dh != 36) || (pieces == 1 && !halves)) continue;
    float *part = floats((size_t)blocks * 2 * dh);
    if (halves) { turn_paired<true, false>(x, nullptr, g, out, nullptr, pieces, blocks); turn_paired<true, true>(norm ? x : nullptr, dy, g, dx, part, pieces, blocks); }
    else { turn_paired<false, false>(x, nullptr, g, out, nullptr, pieces, blocks); turn_paired<false, true>(norm ? x : nullptr, dy, g, dx, part, pieces, blocks); }
    if (in_place) {
      float *io = floats(n);
      memcpy(io, x, n * 4);
      turn::RotateGeom gi = g;
      gi.in_place = 1;
      if (halves) turn_paired<true, false>(io, nullptr, gi, io, nullptr, pieces, blocks); else turn_paired<false, false>(io, nullptr, gi, io, nullptr, pieces, blocks);
      if (memcmp(io, out, n * 4)) complain("in place");
      free(io);
    }
    run((unsigned)((2 * dh + 15) / 16), turn::kFoldThreads, 0, [&] { turn::rotate_fold_kernel(part, blocks, dh, dgq, dgk); });
    double worst = 0, worst_dx = 0, worst_g = 0;
    std::vector<double> rq(dh, 0.0), rk(dh, 0.0), mq(dh, 1e-30), mk(dh, 1e-30);
    for (int64_t m = 0; m < B * T; ++m) for (int h = 0; h < heads + 2 * kv; ++h) {
      const float *xr = x + m * cols + h * dh, *dr = dy + m * cols + h * dh, *o = out + m * cols + h * dh, *d = dx + m * cols + h * dh;
      if (h >= heads + kv) { if (memcmp(o, xr, dh * 4) || memcmp(d, dr, dh * 4)) complain("values"); continue; }
      double ss = 0;
      for (int i = 0; i < dh; ++i) ss += (double)xr[i] * xr[i];
      const double r = norm ? 1.0 / sqrt(ss / dh + (double)g.eps) : 1.0;
      std::vector<double> u(dh), w(dh), ga(dh);
      for (int i = 0; i < dh; ++i) { ga[i] = norm && gains ? (h < heads ? gq : gk)[i] : 1.0; u[i] = xr[i] * r * ga[i]; w[i] = dr[i]; }
      for (int p = 0; p < np; ++p) {
        const int a = halves ? p : 2 * p, b = halves ? p + np : 2 * p + 1;
        const double f = (double)((first ? f0[m / T] : 0) + m % T), an = 2 * M_PI * (f * turns[p] - rint(f * turns[p])), cc = cos(an), s = sin(an);
        const double ua = u[a], ub = u[b], wa = w[a], wb = w[b];
        u[a] = ua * cc - ub * s; u[b] = ua * s + ub * cc; w[a] = wa * cc + wb * s; w[b] = wb * cc - wa * s;
      }
      double dot = 0;
      for (int i = 0; i < dh; ++i) { dot += w[i] * ga[i] * xr[i] * r; (h < heads ? rq : rk)[i] += w[i] * xr[i] * r; (h < heads ? mq : mk)[i] += fabs(w[i] * xr[i] * r); }
      for (int i = 0; i < dh; ++i) {
        at_least(worst, fabs(o[i] - u[i]));
        const double e = norm ? (w[i] * ga[i] - xr[i] * r * dot / dh) * r : w[i];
        at_least(worst_dx, fabs(d[i] - e) / r);
      }
    }
    if (norm) for (int i = 0; i < dh; ++i) { at_least(worst_g, fabs(dgq[i] - rq[i]) / mq[i]); at_least(worst_g, fabs(dgk[i] - rk[i]) / mk[i]); }
    printf("  pieces %d blocks %d: out %.3g dx %.3g gains %.3g\n", pieces, blocks, worst, worst_dx, worst_g);
    if (!(worst < 4e-6) || !(worst_dx < 4e-6) || !(worst_g < 4e-6)) complain("rotation");
    free(part);
  }
  free(x); free(dy); free(out); free(dx); free(gq); free(gk); free(dgq); free(dgk); free(turns); free(f0);
}
}  // namespace aqt
int main(int argc, char **) {
  using namespace aqt;
  if (argc > 1) {
    rotate_case(2, 5, 8, 8, 64, 64, true, true, true, true, true);
    rotate_case(3, 1, 4, 2, 36, 36, false, true, true, true, true);
    rotate_case(1, 7, 2, 1, 36, 36, true, true, true, false, false);
    rotate_case(2, 3, 3, 3, 7, 6, true, true, false, true, true);
    rotate_case(1, 2, 2, 2, 1, 0, false, true, true, false, false);
    rotate_case(2, 9, 4, 1, 128, 32, true, true, true, true, true);
    rotate_case(1, 3, 1, 1, 20, 10, false, false, false, true, true);
    rotate_case(1, 40, 2, 1, 8, 8, false, true, true, true, false);
    rotate_case(1, 2, 2, 2, 101, 100, true, true, true, true, false);
  } else {
    one(2, 64, 1, 1, 64, 8, {5, 62, 1, 70}, {{-1, 0}, {7, 3}}, true);
    one(1, 128, 2, 1, 36, 4, {17, 115, 2}, {{-1, -1}, {0, 0}}, false);
    one(1, 64, 6, 1, 128, 4, {3, 1}, {{2, 0}, {-1, 2}}, false);
    one(2, 64, 1, 1, 5, 6, {4, 66, 3}, {{-1, 0}}, true);
    one(1, 128, 1, 1, 80, 3, {60, 90}, {{30, 1}}, false);
    one(1, 64, 2, 1, 128, 8, {9, 1}, {{-1, 0}}, false);
    one(2, 64, 20, 1, 16, 2, {3, 1}, {{-1, 0}, {1, 1}}, true);
  }
  printf(bad ? "MISMATCH\n" : "ok\n");
  return bad;
}
