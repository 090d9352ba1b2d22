// Driver of the host emulation of the attention over the quantized cache for values, keys and queries of very different sizes: one
// stream, one key / value head, every form of the kernels, against float64 loops.  It follows cache_driver.cpp's helpers (quantized,
// append, attention, join) in the same file, which the test puts in front.
namespace aqt {
constexpr double kU = 0x1p-24;

struct Rows {   // of one stream: `frames` rows of group queries, one key, one value; the last T are the call's own
  int frames, T, group, dh, bits;
  std::vector<float> x;
  int cols() const { return (group + 2) * dh; }
  float *query(int j, int h) { return &x[(size_t)j * cols() + h * dh]; }
  float *key(int j) { return &x[(size_t)j * cols() + group * dh]; }
  float *value(int j) { return &x[(size_t)j * cols() + (group + 1) * dh]; }
};
static Rows make_rows(int frames, int T, int group, int dh, int bits) {
  Rows r{frames, T, group, dh, bits, {}};
  r.x.resize((size_t)frames * r.cols());
  for (float &v : r.x) v = 2.0f * uniform();
  return r;
}

struct Cached {   // the rows in their cache
  CacheGeom g;
  int64_t length;
  std::vector<std::vector<double>> k, v;   // code * scale
};
static void fill(Cached &c, Rows &r) {
  aqt_cache shape{};
  shape.streams = 1; shape.capacity = (r.frames + 63) / 64 * 64; shape.kv_heads = 1; shape.dh = r.dh; shape.bits = r.bits;
  c.g = cache_geom(shape);
  const size_t bytes = (size_t)c.g.tiles * c.g.tile_bytes;
  c.g.data = (uint8_t *)aligned_alloc(64, (bytes + 63) / 64 * 64);
  memset(c.g.data, 0xFF, bytes);
  c.length = 0;
  c.g.length = &c.length;
  const int L = cache_::lanes_of(r.dh), per = (int)cache_::cut_of(c.g, r.frames).blocks;
  const bool vec = r.dh % 4 == 0;
  auto ap = L == 4 ? (vec ? append<4, true> : append<4, false>) : L == 8 ? (vec ? append<8, true> : append<8, false>) : (vec ? append<16, true> : append<16, false>);
  ap((unsigned)per, r.x.data(), c.g, r.frames, r.group, nullptr, cache_::cut_of(c.g, r.frames).log2_run, per, nullptr);
  c.length = r.frames - r.T;
  for (int j = 0; j < r.frames; ++j) {
    std::vector<double> k(r.dh), v(r.dh);
    quantized(r.key(j), r.dh, c.g.qmax, k, 0);
    quantized(r.value(j), r.dh, c.g.qmax, v, 0);
    c.k.push_back(k); c.v.push_back(v);
  }
}

// ctx of the T * group rows, in one of the five forms: 0 / 1 tiles of 16 rows, by themselves / from three splits; 2 / 3 few rows; 4 a
// wavefront to every tile.  Empty where the form does not take so many rows.
static std::vector<float> attend_form(Cached &c, Rows &r, int64_t left, int64_t right, int form) {
  const int n = r.T * r.group, few_rows = n <= kFewRows ? (n == 1 ? 1 : n == 2 ? 2 : 4) : 0, rows = form & 2 ? few_rows : 16;
  if (rows == 0) return {};
  CachedGeom a{};
  a.T = r.T; a.ld = r.cols(); a.heads = r.group; a.group = r.group; a.left = left; a.right = right;
  a.scale_log2e = (float)(1.4426950408889634 / sqrt((double)r.dh));
  a.splits = form & 1 ? 3 : 1;
  a.row_tiles = (n + rows - 1) / rows;
  const int COLS = attend::cols_of(r.dh);
  const size_t pf = (size_t)a.row_tiles * a.splits * ((rows * COLS + 2 * rows + 3) / 4 * 4);
  float *part = a.splits > 1 ? (float *)aligned_alloc(16, (pf * 4 + 15) / 16 * 16) : nullptr;
  float *ctx = (float *)malloc((size_t)n * r.dh * 4);
  const float *qkv = r.x.data() + (size_t)(r.frames - r.T) * r.cols();
  const unsigned grid = (unsigned)(form == 4 ? (a.row_tiles + 3) / 4 : a.row_tiles * a.splits);
  run(grid, 256, 0, [&] { attention(c.g, rows, form == 4, COLS, qkv, a, nullptr, ctx, nullptr, part); });
  if (part) run((unsigned)a.row_tiles, 256, 0, [&] { join(rows, COLS, part, c.g, a, nullptr, ctx, nullptr); });
  std::vector<float> out(ctx, ctx + (size_t)n * r.dh);
  free(ctx); free(part);
  return out;
}

// One row in float64, and its tolerance relative to the sum of weights times the frames' largest values.  A score: the query's digits
// are off by half a unit of its largest column over 2^23, and eight roundings.  A weight: an integer of which the largest of a tile is
// 2^21 at least, so half a unit is 4 U of it, for each of 64 frames; four roundings for every tile, the sum of weights sixteen.
struct Want { std::vector<double> o; double mag, tol; };
// wide: a row of which a column stands out far.  Then the query's digits go on for 23 bits, and what is left is the rounding of their sums:
// 2^-24 of the magnitudes of the products.
static Want want_of(const Cached &c, Rows &r, int t, int h, int64_t left, int64_t right, bool wide = false) {
  const int64_t f = r.frames - r.T + t, lo = left < 0 ? 0 : std::max<int64_t>(0, f - left), hi = right < 0 ? r.frames - 1 : std::min<int64_t>(r.frames - 1, f + right);
  const float *q = r.query((int)f, h);
  double qmax = 0, top = -1e300, reach = 0, terms = 0, largest = 0, spread = 0, sum = 0;
  for (int e = 0; e < r.dh; ++e) qmax = std::max(qmax, (double)fabsf(q[e]));
  std::vector<double> s;
  for (int64_t j = lo; j <= hi; ++j) {
    double d = 0, m = 0, a = 0;
    for (int e = 0; e < r.dh; ++e) { d += c.k[j][e] * q[e]; m += fabs(c.k[j][e]); a += fabs(c.k[j][e] * q[e]); }
    terms = std::max(terms, a / sqrt((double)r.dh));
    s.push_back(d / sqrt((double)r.dh));
    top = std::max(top, s.back()); largest = std::max(largest, fabs(s.back())); reach = std::max(reach, qmax * m / sqrt((double)r.dh));
  }
  for (double x : s) { spread = std::max(spread, top - x); sum += exp(x - top); }
  Want w{std::vector<double>(r.dh, 0.0), 1e-30, 0};
  for (int64_t j = lo; j <= hi; ++j) {
    const double p = exp(s[j - lo] - top) / sum;
    double most = 0;
    for (int e = 0; e < r.dh; ++e) { w.o[e] += p * c.v[j][e]; most = std::max(most, fabs(c.v[j][e])); }
    w.mag += p * most;
  }
  // (frames whose score lies more than 110 below the largest weigh nothing, and their roundings neither)
  const double e = kU * (wide ? terms + reach * 0x1p-23 : reach) + 8 * kU * largest + kU * (std::min(spread, 110.0) + 8);
  w.tol = 2 * e + (256 + 20 * ((double)(hi - lo + 1) / 64 + 2) + 30) * kU;
  return w;
}

static void compare(Rows &r, int64_t left, int64_t right, const char *what, bool wide = false) {
  printf("%s: %d frames, %d new, group %d, dh %d, bits %d\n", what, r.frames, r.T, r.group, r.dh, r.bits); fflush(stdout);
  Cached c;
  fill(c, r);
  for (int form = 0; form < 5; ++form) {
    const std::vector<float> got = attend_form(c, r, left, right, form);
    if (got.empty()) continue;
    double worst = 0, part = 0;
    for (int t = 0; t < r.T; ++t) for (int h = 0; h < r.group; ++h) {
      const Want w = want_of(c, r, t, h, left, right, wide);
      for (int e = 0; e < r.dh; ++e) {
        const double d = fabs(got[((size_t)t * r.group + h) * r.dh + e] - w.o[e]) / w.mag;
        at_least(worst, d); at_least(part, d / w.tol);
      }
    }
    printf("  form %d: worst error %.3g, %.3g of its tolerance\n", form, worst, part);
    if (!(part <= 1.0)) complain(what);
  }
  free(c.g.data);
}

// The first frame draws `lift` more than the others and has values of `size`: most of the weight, and next to no value.
static void sink(int T, int group, int dh, int bits, double lift, float size) {
  Rows r = make_rows(200, T, group, dh, bits);
  for (int j = 0; j < r.frames; ++j) {
    for (int h = 0; h < group; ++h) r.query(j, h)[0] = 3.0f;
    r.key(j)[0] = 0.0f;
  }
  for (int e = 0; e < dh; ++e) { r.key(0)[e] = 0.0f; r.value(0)[e] *= size; }
  r.key(0)[0] = (float)(lift * sqrt((double)dh) / 3.0);
  char what[64];
  snprintf(what, sizeof what, "sink + %g, value x %g", lift, size);
  compare(r, -1, 0, what);
}
// The call's last frame, which the rows in front of it do not see, and one that nobody listens to have values `size` times the others'.
static void large_elsewhere(int T, int group, int dh, int bits, float size) {
  Rows r = make_rows(130, T, group, dh, bits);
  for (int j = 0; j < r.frames; ++j) {
    for (int h = 0; h < group; ++h) r.query(j, h)[0] = 4.0f;
    r.key(j)[0] = 0.0f;
  }
  r.key(r.frames - 9)[0] = -30.0f * sqrtf((float)dh);   // score -120: a weight of nothing
  for (int e = 0; e < dh; ++e) { r.value(r.frames - 1)[e] *= size; r.value(r.frames - 9)[e] *= size; }
  char what[64];
  snprintf(what, sizeof what, "values x %g where no weight is", size);
  compare(r, -1, 0, what);
}
static void drawn_sizes(int T, int group, int dh, int bits) {
  Rows r = make_rows(200, T, group, dh, bits);
  for (int j = 0; j < r.frames; ++j) {
    const float size = exp2f(-10.0f + 10.0f * uniform());
    for (int e = 0; e < dh; ++e) r.value(j)[e] *= size;
    for (int h = 0; h < group; ++h) for (int e = 0; e < dh; ++e) r.query(j, h)[e] *= 3.0f;
  }
  compare(r, -1, 0, "values of 2^-20 to 1");
}
static void weights() {
  for (float size : {0.1f, 0.01f, 0.0f}) sink(1, 1, 64, 8, 10, size);
  sink(1, 2, 64, 8, 14, 0.01f);
  sink(4, 1, 64, 8, 20, 0.0f);
  sink(2, 4, 128, 4, 20, 0.0f);
  sink(3, 1, 36, 4, 20, 0.0f);
  sink(17, 1, 20, 8, 20, 0.0f);
  for (float size : {1e3f, 1e7f}) { large_elsewhere(4, 1, 64, 8, size); large_elsewhere(12, 1, 64, 8, size); }
  large_elsewhere(2, 2, 128, 4, 1e5f);
  large_elsewhere(2, 10, 32, 4, 1e5f);
  drawn_sizes(2, 1, 64, 8);
  drawn_sizes(5, 2, 64, 4);
}
// A number that is none in the key or the value of a frame: NaN in all rows that see it and read back, nothing in the others.
static void one_nonfinite(int T, int group, int dh, int bits, int at, int64_t left, int64_t right, float what, bool key) {
  printf("%f in the %s of frame %d: %d new, group %d, dh %d, bits %d\n", what, key ? "key" : "value", at, T, group, dh, bits); fflush(stdout);
  Rows r = make_rows(130, T, group, dh, bits);
  for (int h = 0; h < group; ++h) r.query(r.frames - T, h)[dh / 2] = -1.0f;   // (an infinite key against a query of either sign)
  float *const row = key ? r.key(at) : r.value(at);
  row[dh / 2] = what;
  Cached c;
  fill(c, r);
  for (int form = 0; form < 5; ++form) {
    const std::vector<float> got = attend_form(c, r, left, right, form);
    if (got.empty()) continue;
    for (int t = 0; t < T; ++t) for (int h = 0; h < group; ++h) {
      const int64_t f = r.frames - T + t;
      const bool seen = (left < 0 || at >= f - left) && (right < 0 || at <= f + right);
      const Want w = want_of(c, r, t, h, left, right);
      for (int e = 0; e < dh; ++e) {
        const float x = got[((size_t)t * group + h) * dh + e];
        if (seen ? !std::isnan(x) : !(fabs((double)x - w.o[e]) <= w.tol * w.mag)) {
          printf("  form %d row %d head %d column %d: %g, seen %d\n", form, t, h, e, x, seen);
          complain("a number that is none");
          t = T; h = group;
          break;
        }
      }
    }
  }
  const int L = cache_::lanes_of(dh), per = (int)cache_::cut_of(c.g, r.frames).blocks, run_ = cache_::cut_of(c.g, r.frames).log2_run;
  const bool vec = dh % 4 == 0;
  std::vector<float> keys((size_t)r.frames * dh, 7.0f), values((size_t)r.frames * dh, 7.0f);
  auto rd = L == 4 ? (vec ? read_<4, true> : read_<4, false>) : L == 8 ? (vec ? read_<8, true> : read_<8, false>) : (vec ? read_<16, true> : read_<16, false>);
  rd((unsigned)per, c.g, T, nullptr, nullptr, r.frames, run_, per, keys.data(), values.data());
  for (int j = 0; j < r.frames; ++j) for (int e = 0; e < dh; ++e) {
    const size_t i = (size_t)j * dh + e;
    if (std::isnan(keys[i]) != (key && j == at) || std::isnan(values[i]) != (!key && j == at)) { complain("read back"); j = r.frames; break; }
  }
  free(c.g.data);
}
static void nonfinite() {
  for (float what : {NAN, INFINITY, -INFINITY}) for (bool key : {false, true}) {
    one_nonfinite(4, 1, 64, 8, 127, -1, 0, what, key);    // seen by the last three of four
    one_nonfinite(12, 1, 36, 4, 125, -1, 0, what, key);   // ... by five of twelve
    one_nonfinite(9, 3, 128, 8, 61, 64, 1, what, key);    // ... by the first five of nine, in another tile than theirs
  }
  one_nonfinite(1, 2, 20, 8, 3, -1, 0, NAN, false);
  one_nonfinite(2, 1, 64, 4, 129, -1, 0, NAN, false);
  one_nonfinite(20, 1, 128, 4, 129, 40, 0, NAN, false);
}
// Small queries against large keys, and the other way round: scores of ordinary size.
static void scores_of(int T, int group, int dh, int bits, float q, float k) {
  Rows r = make_rows(130, T, group, dh, bits);
  for (int j = 0; j < r.frames; ++j) for (int e = 0; e < dh; ++e) {
    for (int h = 0; h < group; ++h) r.query(j, h)[e] *= q;
    r.key(j)[e] *= k;
  }
  char what[64];
  snprintf(what, sizeof what, "queries x %g, keys x %g", q, k);
  compare(r, -1, 0, what);
}
static void scores() {
  for (auto [q, k] : {std::pair<float, float>{1e-30f, 1e30f}, {1e-28f, 1e27f}, {1e30f, 1e-30f}, {3e-30f, 1e36f / 4e6f}}) {
    scores_of(2, 1, 64, 8, q, k);
    scores_of(9, 2, 128, 4, q, k);
    scores_of(20, 1, 128, 8, q, k);
  }
}
// `many` query columns `ratio` times the others, where the keys are zero.
static void outlier_query(int T, int group, int dh, int bits, float ratio, int many = 1) {
  Rows r = make_rows(130, T, group, dh, bits);
  for (int j = 0; j < r.frames; ++j) for (int i = 0; i < many; ++i) {
    for (int h = 0; h < group; ++h) r.query(j, h)[3 + i] = 2.0f * ratio;
    r.key(j)[3 + i] = 0.0f;
  }
  char what[64];
  snprintf(what, sizeof what, "a query column x %g", ratio);
  compare(r, -1, 0, what, ratio >= 300.0f);
}
// Rows whose column stands out beside others: the others' bits are the same as without.
static void neighbours_of_outliers() {
  printf("neighbours of a row with an outlier\n");
  for (int T : {2, 4, 20}) {
    const uint32_t start = seed;
    std::vector<float> got[2][5];
    for (int with = 0; with < 2; ++with) {
      seed = start;
      Rows r = make_rows(130, T, 1, 64, 8);
      if (with) r.query(129, 0)[7] = 1e5f;
      Cached c;
      fill(c, r);
      for (int form = 0; form < 5; ++form) got[with][form] = attend_form(c, r, -1, 0, form);
      free(c.g.data);
    }
    for (int form = 0; form < 5; ++form)
      if (!got[0][form].empty() && memcmp(got[0][form].data(), got[1][form].data(), (size_t)(T - 1) * 64 * 4)) complain("a neighbour of an outlier");
  }
}
static void queries() {
  for (float ratio : {8.0f, 64.0f, 300.0f, 1000.0f, 1e6f, 1e12f}) {
    outlier_query(1, 2, 64, 8, ratio);
    outlier_query(9, 2, 128, 4, ratio);
  }
  outlier_query(4, 1, 128, 8, 1000.0f, 5);
  outlier_query(3, 1, 100, 8, 1e4f, 8);
  outlier_query(17, 1, 80, 8, 1e4f, 1);
  outlier_query(2, 1, 36, 4, 1e5f, 2);
  outlier_query(5, 3, 20, 4, 1e4f, 1);
  outlier_query(1, 1, 8, 8, 1e3f, 1);
  outlier_query(20, 1, 5, 8, 1e3f, 1);
  outlier_query(2, 1, 9, 8, 1e3f, 3);
  outlier_query(6, 1, 12, 4, 1e4f, 4);
  neighbours_of_outliers();
}
// Gains' gradients over many rows of a lane: the first of each a term of 1, the others 2^-25 and a little less, which a float32 sum
// would lose one by one.  Of a term 16 steps; eight terms of a lane, its groups' sums, the workgroup's word and the result.
static void gains_of_many_rows(int64_t T, int dh, bool vec) {
  const int heads = 1, kv = 1, cols = 3 * dh, L = dh <= 32 ? 4 : dh <= 64 ? 8 : 16;
  const int per_row = std::min(64 / L, 4), stride = 4 * (64 / L / per_row);   // rows that the one workgroup takes at a time
  printf("gains of %ld rows, dh %d, %ld to a lane\n", (long)T, dh, (long)(T / stride)); fflush(stdout);
  std::vector<float> x((size_t)T * cols, 1.0f), dy((size_t)T * cols), dx((size_t)T * cols), part(2 * dh), dgq(dh), dgk(dh);
  double want = 0;
  for (int64_t m = 0; m < T; ++m) {
    const float t = m < stride ? 1.0f : 0.9f * 0x1p-25f;
    for (int c = 0; c < cols; ++c) dy[(size_t)m * cols + c] = t;
    want += t / sqrt(1.0 + 1e-6);
  }
  turn::RotateGeom g{};
  g.T = T; g.M = T; g.ld = cols; g.heads = heads; g.kv_heads = kv; g.dh = dh; g.norm = 1; g.eps = 1e-6f;
  turn_paired<false, true>(x.data(), dy.data(), g, dx.data(), part.data(), vec ? 2 : 0, 1);
  run((unsigned)((2 * dh + 15) / 16), turn::kFoldThreads, 0, [&] { turn::rotate_fold_kernel(part.data(), 1, dh, dgq.data(), dgk.data()); });
  double worst = 0;
  for (int c = 0; c < dh; ++c) { at_least(worst, fabs(dgq[c] - want) / want); at_least(worst, fabs(dgk[c] - want) / want); }
  printf("  worst error %.3g\n", worst);
  if (!(worst <= (16 + 8 + 4 + 1 + 1) * kU)) complain("gains of many rows");
}
static void gains() {
  gains_of_many_rows(16 * 250 + 3, 8, true);
  gains_of_many_rows(8 * 250, 7, false);
  gains_of_many_rows(8 * 200, 36, true);
  gains_of_many_rows(4 * 200, 101, false);
}
// Heads of any size without an epsilon, one head of each size in a row: columns whose squares float32 does not hold.  Rounding steps of
// 2^-24 as in the tests of ordinary heads: 18 forward, 48 for the gradient, each of the magnitudes of its pair.
static void rotate_sizes(int dh, int rot, bool halves, bool vec, std::vector<float> sizes, float eps) {
  const int heads = (int)sizes.size(), kv = 1, cols = (heads + 2) * dh, np = rot / 2;
  const int64_t T = 5;
  printf("heads of all sizes, dh %d, rot %d, halves %d, eps %g\n", dh, rot, halves, eps); fflush(stdout);
  std::vector<float> x((size_t)T * cols), dy(x.size()), out(x.size()), dx(x.size()), part(2 * dh), gq(dh), dgq(dh), dgk(dh);
  for (int64_t m = 0; m < T; ++m) for (int h = 0; h < heads + 2; ++h) for (int i = 0; i < dh; ++i) {
    const float s = h < heads ? sizes[h] : 1.0f;
    x[m * cols + h * dh + i] = s * uniform();
    dy[m * cols + h * dh + i] = s * uniform();   // a gradient of the head's own size: that of x is about 1
  }
  for (float &v : gq) v = 1.0f + 0.3f * uniform();
  std::vector<double> turns(np ? np : 1);
  for (int i = 0; i < np; ++i) turns[i] = pow(10000.0, -(double)i / np) / (2 * M_PI);
  turn::RotateGeom g{};
  g.T = T; g.M = T; g.ld = cols; g.heads = heads; g.kv_heads = kv; g.dh = dh; g.rot = rot; g.norm = 1; g.eps = eps; g.turns = turns.data(); g.gamma[0] = gq.data();
  const int form = vec ? (!halves || rot % 8 == 0 ? 2 : 1) : 0;
  if (halves) { turn_paired<true, false>(x.data(), nullptr, g, out.data(), nullptr, form, 1); turn_paired<true, true>(x.data(), dy.data(), g, dx.data(), part.data(), form, 1); }
  else { turn_paired<false, false>(x.data(), nullptr, g, out.data(), nullptr, form, 1); turn_paired<false, true>(x.data(), dy.data(), g, dx.data(), part.data(), form, 1); }
  double worst = 0, worst_dx = 0;
  for (int64_t m = 0; m < T; ++m) for (int h = 0; h < heads; ++h) {
    const float *xr = &x[m * cols + h * dh], *dr = &dy[m * cols + h * dh], *o = &out[m * cols + h * dh], *d = &dx[m * cols + h * dh];
    double ss = 0;
    for (int i = 0; i < dh; ++i) ss += (double)xr[i] * xr[i];
    const double r = 1.0 / sqrt(ss / dh + (double)eps);
    std::vector<double> u(dh), um(dh), w(dh), wm(dh);
    for (int i = 0; i < dh; ++i) { u[i] = xr[i] * r * gq[i]; um[i] = fabs(u[i]); w[i] = dr[i]; wm[i] = fabs(w[i]); }
    for (int p = 0; p < np; ++p) {
      const int a = halves ? p : 2 * p, b = halves ? p + np : 2 * p + 1;
      const double an = 2 * M_PI * m * turns[p], cc = cos(an), s = sin(an), ua = u[a], ub = u[b], wa = w[a], wb = w[b];
      u[a] = ua * cc - ub * s; u[b] = ua * s + ub * cc; w[a] = wa * cc + wb * s; w[b] = wb * cc - wa * s;
      um[a] = um[b] = um[a] + um[b]; wm[a] = wm[b] = wm[a] + wm[b];
    }
    // A gradient of 3e38: |a cos| + |b sin| reaches 3e38 sqrt(2) = 4.2e38, and times a gain of 1.3 5.5e38, where float32 ends at
    // 3.4e38: the rotated gradient itself is no number, and neither is what is made of it.
    bool beyond = false;
    for (int i = 0; i < dh; ++i) beyond = beyond || wm[i] * fabs(gq[i]) > 3.4e38;
    double dot = 0, dotm = 0;
    for (int i = 0; i < dh; ++i) { dot += w[i] * gq[i] * xr[i] * r; dotm += wm[i] * fabs(gq[i] * xr[i] * r); }
    for (int i = 0; i < dh; ++i) {
      at_least(worst, fabs(o[i] - u[i]) / (18 * kU * um[i] + 1e-30));
      // (gradients next to the smallest numbers have these as steps)
      if (!beyond) at_least(worst_dx, fabs(d[i] - (w[i] * gq[i] - xr[i] * r * dot / dh) * r) / (48 * kU * r * (wm[i] * fabs(gq[i]) + fabs(xr[i] * r) * dotm / dh) + 0x1p-149 * r * dh + 1e-30));
    }
  }
  printf("  worst of their tolerances: out %.3g dx %.3g\n", worst, worst_dx);
  if (!(worst <= 1.0) || !(worst_dx <= 1.0)) complain("heads of all sizes");
}
static void sizes() {
  const std::vector<float> all = {1.0f, 1e-20f, 3e-38f, 1e20f, 1e-10f, 3e38f, 1e-30f, 1e15f};
  rotate_sizes(64, 64, true, true, all, 0.0f);
  rotate_sizes(36, 36, false, true, all, 0.0f);
  rotate_sizes(20, 20, true, true, all, 0.0f);
  rotate_sizes(100, 100, true, true, all, 0.0f);
  rotate_sizes(101, 100, true, false, all, 0.0f);
  rotate_sizes(128, 64, true, true, all, 1e-35f);
  rotate_sizes(8, 4, false, false, {1e20f, 1.0f, 1e19f}, 1e-6f);
}
}  // namespace aqt
int main(int argc, char **argv) {
  using namespace aqt;
  const std::string what = argc > 1 ? argv[1] : "";
  if (what == "weights") weights();
  else if (what == "nonfinite") nonfinite();
  else if (what == "scores") scores();
  else if (what == "queries") queries();
  else if (what == "gains") gains();
  else if (what == "sizes") sizes();
  else complain("no such test");
  printf(bad ? "MISMATCH\n" : "ok\n");
  return bad;
}
