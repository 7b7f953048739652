// Attention over the paged cache on the CPU (tests/cpu_hip) beside plain loops in
// float64, for values at which the way to a result shows: no numbers in one part of
// the keys, scores far apart.  Prints "ok".
#include <hip/hip_runtime.h>

static long g_products;  // terms of matrix products, the instruction's for the most part
#define fmaf(a, b, c) (g_products++, (fmaf)(a, b, c))
#define main paged_cpu_main
#include "paged_cpu.cpp"
#undef main

struct Problem {
  int hd, page, Hkv, G, window, sinks, shared, max_new;
  std::vector<int> T, len;  // new tokens of each sequence, tokens before them
  int pad;                  // rows of no token behind them
};

// A batch whose numbers are set one by one.  The first `shared` tokens of all
// sequences are those of the first.
struct Attention {
  Problem p;
  int B, most, n, Hq;
  std::vector<int> starts;
  std::vector<float> q, kv[2];  // [n, Hq, hd]; [B, most page, Hkv, hd]
  static constexpr float scale = 0.125f;
  double absolute = 1e-37;  // what a result may be off by whatever it is
  Attention(const Problem& p, int seed) : p(p), B((int)p.T.size()), most(0), Hq(p.Hkv * p.G), starts{0} {
    for (int b = 0; b < B; b++) {
      starts.push_back(starts[b] + p.T[b]);
      most = std::max(most, (p.len[b] + p.T[b] + p.page - 1) / p.page);
    }
    n = starts[B] + p.pad;
    std::mt19937 rng(seed);
    std::normal_distribution<float> normal;
    q.resize((size_t)n * Hq * p.hd);
    for (auto& x : kv) x.resize((size_t)B * most * p.page * p.Hkv * p.hd);
    for (auto* x : {&q, &kv[0], &kv[1]})
      for (auto& e : *x) e = normal(rng);
  }
  float& query(int row, int h, int d) { return q[((size_t)row * Hq + h) * p.hd + d]; }
  float& token(int i, int b, int t, int h, int d) { return kv[i][((((size_t)(t < p.shared ? 0 : b) * most * p.page) + t) * p.Hkv + h) * p.hd + d]; }
  float& key(int b, int t, int h, int d) { return token(0, b, t, h, d); }
  float& value(int b, int t, int h, int d) { return token(1, b, t, h, d); }

  std::vector<uint16_t> run() {
    const int hd = p.hd, lead = p.shared / p.page, n_pages = lead + B * (most - lead), tokens = most * p.page;
    check(p.shared % p.page == 0, "whole pages", p.shared);
    std::vector<int> pages(B * most);
    for (int b = 0; b < B; b++)
      for (int i = 0; i < most; i++) pages[b * most + i] = i < lead ? i : lead + b * (most - lead) + i - lead;
    std::vector<uint16_t> pool[2], wq(q.size());
    for (auto& x : pool) x.assign((size_t)n_pages * p.Hkv * p.page * hd, 0x7fc1);
    for (int i = 0; i < 2; i++)
      for (int b = 0; b < B; b++)
        for (int t = 0; t < p.len[b] + p.T[b]; t++)
          for (int h = 0; h < p.Hkv; h++)
            for (int d = 0; d < hd; d++)
              pool[i][(((size_t)pages[b * most + t / p.page] * p.Hkv + h) * p.page + t % p.page / 32 * 32) * hd + (i ? at_value(t % 32, d) : at_key(t % 32, d, hd))] =
                  f32_to_bf16(token(i, b, t, h, d));
    for (size_t i = 0; i < q.size(); i++) wq[i] = f32_to_bf16(q[i]);
    uint16_t* out = (uint16_t*)guarded(q.size() * 2);
    std::fill(out, out + q.size(), (uint16_t)0x1234);
    const int64_t bytes = paged_workspace_bytes(n, B, Hq, p.Hkv, hd, p.max_new, tokens, p.shared);
    char* ws = guarded(bytes);
    memset(ws, 0xff, bytes);
    const Ragged r{copy(pages), copy(starts), copy(p.len), B, n, most, p.page, n_pages};
    const PagedAttnArgs a{copy(wq), copy(pool[0]), copy(pool[1]), Hq * hd, Hq, p.Hkv, hd, p.max_new, p.window, p.sinks, p.shared, scale, out, ws, r};
    launch_attention_paged(a, nullptr);
    for (auto& l : g_loads) check(l.empty(), "a load outlives its kernel", 0);
    return std::vector<uint16_t>(out, out + q.size());
  }

  // Against softmax(scale q.k) v: probabilities rounded to bf16 (2^-8 of each) as the
  // result is, scores in float32 (2^-24 (hd + 8) of the sum of their terms' sizes).
  // A probability below 2^-126 of the largest is zero.
  void compare(const char* what, int id) {
    g_late = id % 2;
    const std::vector<uint16_t> got = run();
    auto bf16 = [](float x) { return (double)bf16_to_f32(f32_to_bf16(x)); };
    for (int b = 0; b < B; b++)
      for (int t = 0; t < std::min(p.T[b], p.max_new); t++)
        for (int h = 0; h < Hq; h++) {
          const int row = starts[b] + t, pos = p.len[b] + t, kvh = h / p.G;
          std::vector<int> seen;
          std::vector<double> s;
          double top = -INFINITY, size = 0, sum = 0;
          for (int j = 0; j <= pos; j++) {
            if (p.window && j <= pos - p.window && j >= p.sinks) continue;
            double x = 0, terms = 0;
            for (int d = 0; d < p.hd; d++) {
              const double y = scale * bf16(query(row, h, d)) * bf16(key(b, j, kvh, d));
              x += y;
              terms += fabs(y);
            }
            seen.push_back(j);
            s.push_back(x);
            if (x > top) top = x;
            if (std::isfinite(terms)) size = std::max(size, terms);
          }
          for (double& x : s) {
            x = top == -INFINITY && x == x ? 0 : exp(x - top);
            if (x < 0x1p-126) x = 0;
            sum += x;
          }
          for (int d = 0; d < p.hd; d++) {
            double w = 0, dev = 0;
            for (size_t i = 0; i < seen.size() && sum != 0; i++) {
              const double x = s[i] / sum * bf16(value(b, seen[i], kvh, d));
              w += x;
              dev += fabs(x);
            }
            dev += fabs(w);
            const double g = bf16_to_f32(got[((size_t)row * Hq + h) * p.hd + d]);
            const double tol = (0x1p-8 + 0x1p-22 + 0x1p-24 * (p.hd + 8) * size) * dev * (1 + 0x1p-6) + 0x1p-8 * fabs(w) + absolute;
            if (g != g ? w == w : std::isfinite(w) ? !(fabs(g - w) <= tol) : g != w) {
              printf("%s %d, row %d head %d dim %d: %g, not %g\n", what, id, row, h, d, g, w);
              exit(1);
            }
          }
        }
    for (size_t i = (size_t)starts[B] * Hq * p.hd; i < got.size(); i++) check(got[i] == 0x1234, "a row of no token", (int)i);
  }
};

// Keys of two sizes along the first dim: scores of -160 for tokens before `half` and of
// 160 from there on, so that the former's probabilities are zero.
static void far_apart(Attention& a, int half) {
  for (auto* x : {&a.q, &a.kv[0]}) std::fill(x->begin(), x->end(), 0.f);
  for (int row = 0; row < a.n; row++)
    for (int h = 0; h < a.Hq; h++) a.query(row, h, 0) = 1;
  for (int b = 0; b < a.B; b++)
    for (int t = 0; t < a.p.len[b] + a.p.T[b]; t++)
      for (int h = 0; h < a.p.Hkv; h++) a.key(b, t, h, 0) = t < half ? -1280 : 1280;
}

// A visible value that is no number is one in the result, whichever part of the keys it is
// in and however little that part weighs.
static void no_numbers_in_a_part() {
  const std::vector<Problem> problems = {
      {128, 64, 1, 1, 0, 0, 0, 1, {1}, {1100}, 0},             // three parts of few columns
      {128, 64, 1, 1, 0, 0, 0, 70, {70}, {1100}, 0},           // of many
      {64, 64, 1, 2, 0, 0, 1024, 1, {1, 1}, {1100, 1040}, 1},  // four of a prefix, few columns, and the sequences' own
      {64, 64, 1, 8, 0, 0, 1024, 20, {20, 17}, {1024, 1040}, 0},  // many
  };
  int id = 0;
  for (const Problem& p : problems)
    for (float odd : {(float)NAN, (float)INFINITY, (float)-INFINITY})
      for (int at : {3, 600, 1030}) {
        Attention a(p, id);
        far_apart(a, 512);
        a.value(0, at, 0, 5) = odd;
        a.compare("no number in a part", id++);
      }
}

// A query whose scores are all -infinity gets zeros, whatever the values are.
static void no_weight_at_all() {
  const std::vector<Problem> problems = {
      {64, 32, 1, 1, 0, 0, 0, 1, {1}, {40}, 0},             // one part of few columns
      {64, 32, 1, 2, 0, 0, 0, 1, {1}, {1100}, 0},           // two
      {64, 32, 1, 4, 0, 0, 0, 1000, {20}, {70}, 0},         // one of many
      {64, 32, 1, 4, 0, 0, 0, 20, {20}, {1100}, 0},         // three
      {64, 32, 1, 1, 0, 0, 64, 2, {1, 2}, {70, 70}, 0},     // a prefix, few columns
      {64, 32, 1, 8, 0, 0, 64, 20, {20, 18}, {70, 70}, 0},  // many
  };
  int id = 0;
  for (const Problem& p : problems)
    for (float odd : {(float)NAN, (float)INFINITY}) {
      Attention a(p, id);
      for (int row = 0; row < a.n; row++)
        for (int h = 0; h < a.Hq; h++) a.query(row, h, 0) = 1;
      for (int b = 0; b < a.B; b++)
        for (int t = 0; t < p.len[b] + p.T[b]; t++) a.key(b, t, 0, 0) = -INFINITY;
      a.value(0, 3, 0, 5) = a.value(0, p.len[0], 0, 6) = odd;
      a.compare("no weight at all", id++);
    }
}

// Values near bf16's largest: their mean is a number, their sum is none.
static void large_values() {
  const std::vector<Problem> problems = {
      {64, 32, 1, 1, 0, 0, 0, 1, {1}, {40}, 0},             // one part of few columns
      {128, 32, 1, 2, 0, 0, 0, 1, {1}, {1500}, 0},          // three
      {64, 32, 1, 4, 0, 0, 0, 1000, {20}, {170}, 0},        // one of many
      {64, 32, 1, 4, 60, 3, 0, 1000, {20}, {170}, 0},       // behind a window
      {128, 32, 1, 4, 0, 0, 0, 20, {20}, {1100}, 0},        // three
      {64, 32, 1, 1, 0, 0, 640, 2, {1, 2}, {700, 650}, 0},  // a prefix, few columns
      {64, 32, 1, 8, 0, 0, 640, 20, {20, 18}, {700, 650}, 1},  // many
  };
  int id = 0;
  for (const Problem& p : problems)
    for (int rising : {0, 1}) {
      Attention a(p, id);
      // scores around zero, or 7 (in powers of two) larger with every 30 keys
      for (int row = 0; row < a.n && rising; row++)
        for (int h = 0; h < a.Hq; h++) a.query(row, h, 0) = 1;
      for (int b = 0; b < a.B; b++)
        for (int t = 0; t < p.len[b] + p.T[b]; t++) {
          if (rising) a.key(b, t, 0, 0) = 8 * 0.23f * 0.693f * (t % 1024);
          for (int d = 0; d < p.hd; d++) a.value(b, t, 0, d) = (d % 2 ? -1 : 1) * (3.3e38f - 1e37f * (t % 7));
        }
      a.compare("large values", id++);
    }
}

// A chunk beside single tokens, so that partial results lie row by row, and single tokens
// beside sequences without rows, so that they lie sequence by sequence.
static void places_of_parts() {
  const std::vector<Problem> problems = {
      {128, 64, 2, 2, 0, 0, 0, 8, {1, 8, 1, 0, 1, 2}, {1100, 700, 3, 9, 600, 1030}, 2},
      {64, 64, 1, 4, 0, 0, 64, 8, {1, 8, 1, 0, 1, 2}, {1100, 700, 66, 70, 600, 1300}, 2},
      {64, 64, 2, 4, 700, 5, 0, 8, {1, 8, 1, 0, 1, 2}, {1100, 700, 66, 70, 600, 1300}, 0},
      {128, 64, 2, 2, 0, 0, 0, 1, {1, 0, 0, 1}, {1100, 9, 4, 600}, 0},
      {128, 64, 1, 8, 0, 0, 0, 60, {1, 60, 1}, {1100, 400, 600}, 3},
  };
  int id = 0;
  for (const Problem& p : problems) Attention(p, id).compare("places of parts", id), id++;
}

// What rows of no token hold costs nothing: they are in the prefix's columns, whose results
// nobody takes.
static void rows_of_no_token() {
  for (int G : {1, 8}) {  // few columns of a prefix, many
    long products[2];
    for (int odd = 0; odd < 2; odd++) {
      Attention a({64, 64, 1, G, 0, 0, 640, 40, {3, 40}, {640, 700}, 30}, G);
      for (int row = a.starts[2]; row < a.n; row++)
        for (int h = 0; h < G; h++) a.query(row, h, 7) = odd ? row % 2 ? NAN : INFINITY : 1;
      g_products = 0;
      a.run();
      products[odd] = g_products;
      a.compare("rows of no token", G);
    }
    check(products[0] == products[1], "more products for rows of no token", G);
  }
}

// NaN and infinities in a shared prefix, among keys and values that a window hides from
// some of the columns of a wave and not from others (and from all of some waves): in
// both forms, whole and behind the sinks.
static void no_numbers_in_a_prefix() {
  int id = 0;
  for (int G : {2, 12})
    for (int hd : {64, 128})
      for (int sinks : {0, 3})
        for (int at : {1, 95, 100, 105, 119, 150}) {
          // 48 columns, or 288, whose windows begin at 92 to 111, 120 and behind the prefix
          Attention a({hd, 64, 1, G, 101, sinks, 192, 12, {12, 1, 9, 1}, {200, 220, 192, 300}, 1}, id);
          const float odd[] = {NAN, INFINITY, -INFINITY};
          a.value(0, at, 0, 5) = odd[id % 3];
          if (id % 2) a.key(0, at, 0, 7) = odd[(id + 1) % 3];
          a.compare("no numbers in a prefix", id++);
        }
}

// Appended keys and values and rotated queries, signs and all, against float64: float32
// arithmetic (2^-23 of the products' sizes), one rounding to bf16 (2^-8).
template <class T>
static void rotation_signs(int hd, int rot, int layout, int skew, int id) {
  const int Hkv = 2, Hq = 4, n = 9, old = 27, page = 32, ld = (Hkv + Hq) * hd + 8;
  std::mt19937 rng(id);
  std::normal_distribution<float> normal;
  std::vector<T> rows((size_t)n * ld + 1), vrows((size_t)n * Hkv * hd);
  auto number = [](T x) { return sizeof(T) == 2 ? (double)bf16_to_f32(x) : (double)x; };
  auto make = [&](float x) { return sizeof(T) == 2 ? (T)f32_to_bf16(x) : (T)x; };
  for (auto* x : {&rows, &vrows})
    for (auto& e : *x) e = make(normal(rng));
  std::vector<float> table((size_t)64 * rot);
  for (auto& e : table) e = normal(rng);
  uint16_t *kc = (uint16_t*)guarded(2 * Hkv * page * hd * 2), *vc = (uint16_t*)guarded(2 * Hkv * page * hd * 2), *qo = (uint16_t*)guarded(n * Hq * hd * 2);
  const T *in = copy(rows) + skew, *vin = copy(vrows);
  const std::vector<int> pages = {1, 0}, starts = {0, n}, lens = {old};
  const Ragged r{copy(pages), copy(starts), copy(lens), 1, n, 2, page, 2};
  const AppendArgs a{in, vin, in + Hkv * hd, ld, Hkv * hd, ld, Hq * hd, sizeof(T) == 2 ? LMGC_DTYPE_BF16 : LMGC_DTYPE_F32, Hq, Hkv, hd, rot, layout,
                     kc, vc, qo, copy(table), 64, r};
  launch_paged_append(a, nullptr);
  for (int t = 0; t < n; t++)
    for (int h = 0; h < Hkv + Hq; h++)
      for (int d = 0; d < hd; d++) {
        const T* x = in + (size_t)t * ld + h * hd;
        const int pos = old + t, half = rot / 2;
        double y = number(x[d]), size = 0;
        if (d < rot) {
          const bool split = layout == LMGC_ROPE_HALF, second = split ? d >= half : d & 1;
          const int i = split ? d % half : d / 2, other = split ? (second ? d - half : d + half) : d ^ 1;
          const double c = table[((size_t)pos * half + i) * 2], s = table[((size_t)pos * half + i) * 2 + 1];
          const double u = y * c, v = number(x[other]) * s * (second ? 1 : -1);
          y = u + v;
          size = fabs(u) + fabs(v);
        }
        const size_t at = (((size_t)pages[pos / page] * Hkv + h) * page) * hd;
        const double got = bf16_to_f32(h < Hkv ? kc[at + at_key(pos % page, d, hd)] : qo[((size_t)t * Hq + h - Hkv) * hd + d]);
        check(fabs(got - y) <= 0x1p-23 * size + 0x1p-8 * fabs(y) * (1 + 0x1p-8), h < Hkv ? "a key's number" : "a query's number", id);
        if (h < Hkv) check(vc[at + at_value(pos % page, d)] == f32_to_bf16((float)number(vin[((size_t)t * Hkv + h) * hd + d])), "a value's number", id);
      }
}

static void rotations() {
  int id = 0;
  for (int layout : {LMGC_ROPE_HALF, LMGC_ROPE_INTERLEAVED})
    for (int hd : {64, 128})
      for (int rot : {hd, 32, 6})
        for (int skew : {0, 1}) {
          rotation_signs<uint16_t>(hd, rot, layout, skew, id++);
          rotation_signs<float>(hd, rot, layout, skew, id++);
        }
}

// Long walks of the form for many: as a max_new of many columns has it, in one part, with
// more than the 32 steps whose pages are looked up at once; twice where a value that some
// queries do not see is no number.
static void long_walks() {
  int id = 0;
  for (int hd : {64, 128})
    for (int window : {0, 2500})
      for (bool odd : {false, true}) {
        Attention a({hd, 64, 1, 1, window, window ? 70 : 0, 0, 1 << 20, {70, 1}, {2700, 2300}, 0}, id);
        if (odd) a.value(0, 2740, 0, 3) = a.value(0, 230, 0, 4) = NAN;
        a.compare("a long walk", id++);
      }
}

// Values of bf16's smallest normal exponents keep their digits through every join.
static void small_values() {
  const std::vector<Problem> problems = {
      {64, 32, 1, 1, 0, 0, 0, 1, {1}, {40}, 0},                // one part of few columns
      {128, 32, 1, 2, 0, 0, 0, 1, {1}, {1500}, 0},             // three
      {128, 32, 1, 4, 0, 0, 0, 20, {20}, {1100}, 0},           // three of many
      {64, 32, 1, 1, 0, 0, 640, 2, {1, 2}, {700, 650}, 0},     // a prefix, few columns
      {64, 32, 1, 8, 0, 0, 640, 20, {20, 18}, {700, 650}, 1},  // many
  };
  int id = 0;
  for (const Problem& p : problems) {
    Attention a(p, id);
    for (float& e : a.kv[1]) e = (1 + fminf(fabsf(e), 2)) * 0x1p-126f;
    a.absolute = 0;
    a.compare("small values", id++);
  }
}

int main() {
  small_values();
  long_walks();
  rotations();
  no_numbers_in_a_prefix();
  rows_of_no_token();
  places_of_parts();
  large_values();
  no_weight_at_all();
  no_numbers_in_a_part();
  printf("ok\n");
}
