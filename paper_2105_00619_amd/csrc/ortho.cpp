// Host side of the orthogonalised updates: the plan of a list of matrices (optorch_ortho_*).
//
// A Newton-Schulz step X <- (a + b A + c A^2) X with A = X X^T changes the singular values of X alone, so that the steps can be
// made on A: with P = a + b A + c A^2,  A <- P A P  and  Q <- P Q,  and in the end X <- Q X.  Only A = X X^T at the start and
// Q X at the end touch the long side of X; all other products are m x m and symmetric, so that half of their tiles are made.
//
// But a rounding of A (about 2^-23 of its largest value) grows by a^2 a step in the directions of small singular values,
// where P passes it on to the result.  Largest errors over m = 2 .. 512 with one or m / 16 singular values of 1 and the
// others 0.5 .. 1e-4, five steps (emulated; the steps on X in fp32: 0.6e-6 to 8e-5, the more the smaller the others):
//   X made anew after every step: as the steps on X;  after two: up to 7e-6 more;  three: 8e-5;  four: 2.3e-4;  five: 1.8e-3.
// A result stored in bf16 is rounded by 1.7e-3 and takes three steps on A, any other two.  (For n = 4 m that is 38 and 47 m^3 of
// products, 65 with steps on X.)
//
// The operands are pairs of fp16 planes (hi + lo, 22 bits and a sign), times a power of two for each kind of matrix, since
// the bounds of all of them are known (host: from the polynomials): three products of 16-bit matrix cores for one, with an
// error of 2^-24 a value.  One plane alone would do for a bf16 result of well-conditioned matrices, but is 1e-2 off where a
// few singular values are large: in small directions an error of the first iterate is multiplied by 485.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <functional>
#include <new>
#include <string>

#include "matrix.h"

using namespace oseq;

int oseq_mat_err(int code, const std::string& m);  // matrix.cpp

struct optorch_ortho {
  OrthoPlanHost p;
  char* ws = nullptr;
};

namespace {

// the power of two that brings values of at most `bound` into fp16's range with room to spare; small bounds gain nothing
// beyond 2^12 (the low plane of a value of 2^-12 then still has all its bits)
float plane_scale(double bound) { return (float)std::exp2(std::min(12.0, std::floor(std::log2(16384.0 / std::max(bound, 1e-3))))); }

// Steps on A between two iterates at most, and how far they may let an error of A grow (the product of their a^2): with larger
// coefficients a restart comes sooner
struct Restart { int steps; double growth; };
constexpr Restart RESTART[OUT_COUNT] = {{2, 150.}, {ORTHO_RESTART, 2e3}};

// The launches and their scales.  Returns false where the steps let a singular value grow too far.
bool plan_steps(OrthoPlanHost& p, std::vector<OrthoLaunch>& launches, Restart restart, int steps, const float* co) {
  constexpr int GRID = 4096;
  std::vector<double> l(GRID + 1), q(GRID + 1);
  for (int i = 0; i <= GRID; ++i) l[i] = (double)i / GRID;  // squares of singular values; sampled, the bounds have a margin
  double xmax = 1.0;
  int src = 0;
  auto top = [&](auto f) { double t = 0; for (int i = 0; i <= GRID; ++i) t = std::max(t, std::fabs(f(i))); return t * 1.01; };
  p.first_scale = plane_scale(1.0);
  float sx = p.first_scale;
  for (int s = 0; s < steps;) {
    int e = s;
    for (double growth = 1; e < steps && e < s + restart.steps; ++e) {
      growth *= (double)co[3 * e] * co[3 * e];
      if (e > s && growth > restart.growth) break;
    }
    const double amax = top([&](int i) { return l[i]; });
    float sa = plane_scale(amax), sq = 1.f;
    OrthoLaunch g = {};
    g.kind = OL_GRAM; g.src = src; g.ops = 1;
    g.op[0] = OrthoOp{0, 0, OB_A, -1, sa / (sx * sx), 0.f, 0.f};
    launches.push_back(g);
    int qbuf = OB_Q0;
    std::fill(q.begin(), q.end(), 1.0);
    for (int k = s; k < e; ++k) {
      const double a = co[3 * k], b = co[3 * k + 1], c = co[3 * k + 2];
      auto poly = [&](int i) { return a + l[i] * (b + l[i] * c); };
      const double pmax = std::max(top(poly), 1e-3);
      const float sp = plane_scale(pmax);
      const int pbuf = k == s ? OB_Q0 : OB_P;
      OrthoLaunch lp = {};
      lp.kind = OL_CHAIN; lp.ops = 1;
      lp.op[0] = OrthoOp{OB_A, OB_A, pbuf, OB_A, (float)(sp * c / (sa * sa)), (float)(sp * b / sa), (float)(sp * a)};
      launches.push_back(lp);
      for (int i = 0; i <= GRID; ++i) q[i] *= poly(i);
      const float sq_new = plane_scale(top([&](int i) { return q[i]; }));
      OrthoLaunch ln = {};
      ln.kind = OL_CHAIN;
      if (k + 1 < e) {
        const float sc = plane_scale(top([&](int i) { return l[i] * poly(i); }));
        for (int i = 0; i <= GRID; ++i) { const double t = poly(i); l[i] *= t * t; }
        const float sa_new = plane_scale(top([&](int i) { return l[i]; }));
        ln.op[ln.ops++] = OrthoOp{pbuf, OB_A, OB_C, -1, sc / (sp * sa), 0.f, 0.f};
        if (k > s) {
          ln.op[ln.ops++] = OrthoOp{OB_P, qbuf, qbuf ^ OB_Q0 ^ OB_Q1, -1, sq_new / (sp * sq), 0.f, 0.f};
          qbuf ^= OB_Q0 ^ OB_Q1;
          sq = sq_new;
        } else {
          sq = sp;
        }
        launches.push_back(ln);
        OrthoLaunch la = {};
        la.kind = OL_CHAIN; la.ops = 1;
        la.op[0] = OrthoOp{OB_C, pbuf, OB_A, -1, sa_new / (sc * sp), 0.f, 0.f};
        launches.push_back(la);
        sa = sa_new;
      } else {
        for (int i = 0; i <= GRID; ++i) { const double t = poly(i); l[i] *= t * t; }
        if (k > s) {
          ln.op[ln.ops++] = OrthoOp{OB_P, qbuf, qbuf ^ OB_Q0 ^ OB_Q1, -1, sq_new / (sp * sq), 0.f, 0.f};
          qbuf ^= OB_Q0 ^ OB_Q1;
          sq = sq_new;
          launches.push_back(ln);
        } else {
          sq = sp;
        }
      }
      xmax = std::sqrt(top([&](int i) { return l[i]; }));
      if (!(xmax <= 64.0)) return false;
    }
    OrthoLaunch x = {};
    x.kind = OL_APPLY; x.src = src; x.ops = 1; x.last = e == steps;
    const float sx_new = plane_scale(xmax);
    x.op[0] = OrthoOp{qbuf, 0, 0, -1, x.last ? 1.f / (sq * sx) : sx_new / (sq * sx), 0.f, 0.f};
    launches.push_back(x);
    sx = sx_new;
    src ^= 1;
    s = e;
    // (the next segment's squares lie anywhere up to the bound, not only where the grid has them now)
    const double m = top([&](int i) { return l[i]; });
    for (int i = 0; i <= GRID; ++i) l[i] = m * i / GRID;
  }
  return true;
}

int up32(int n) { return (n + 31) & ~31; }
int cdiv(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// ---- which block makes what ----------------------------------------------------------------------------------------------
// What a launch is estimated to take, in us, from the time of a tile step (64 places of two operands), of a block's
// beginning and end, and of what it writes and reads besides (a CU's share of 4.5 TB/s; alone on its CU a block does not
// reach it).  Two blocks of 128 x 128 or three of 64 x 64 run on a CU: their products take turns, their ends overlap with
// them.  Measured on products of 2048 and 4096 rows and on ResNet-152's, whose last products take 380 us as 256 x 256 tiles
// and 310 as 128 x 128.
double step_us(int w) { return w == 128 ? 2.0 : w == 64 ? 0.65 : 0.25; }
double block_us(int w) { return w == 128 ? 8.0 : w == 64 ? 6.0 : 5.0; }
int blocks_of_cu(int w) { return w == 128 ? 1 : w == 64 ? 2 : 3; }
constexpr double CU_BYTES_US = 17600., CU_BYTES_US_ALONE = 11000.;
constexpr int CUS = 256, XCDS = 8;

// How the tiles of one matrix are cut: the first `whole` in one block each, the others' sums in `parts` of `per` steps
struct Cut { int64_t count, whole; int steps, parts, per; };

int64_t triangle(int64_t t) { return t * (t + 1) / 2; }

// Sums of more than `most` steps are cut; with `tail` only those of the tiles that do not fill a round of all places (the
// shortest sums), which come last.
std::vector<Cut> cuts_of(const OrthoPlanHost& p, bool lower, bool along_n, int w, int most, bool tail) {
  std::vector<Cut> cuts;
  std::vector<int> order;
  int64_t all = 0;
  for (size_t i = 0; i < p.mats.size(); ++i) {
    const OrthoMat& m = p.mats[i];
    const int tm = cdiv(m.m, 2 * w), K = along_n ? m.n : m.m;
    Cut c = {};
    c.count = lower ? triangle(tm) : (int64_t)tm * cdiv(m.n, 2 * w);
    c.steps = cdiv(K, 32);
    c.per = cdiv(c.steps, cdiv(c.steps, most));
    c.parts = cdiv(c.steps, c.per);
    cuts.push_back(c);
    order.push_back((int)i);
    all += c.count;
  }
  const int places = CUS * blocks_of_cu(w);
  int64_t whole = tail ? all / places * places : 0;
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return cuts[a].steps > cuts[b].steps; });
  for (int i : order) {
    Cut& c = cuts[i];
    c.whole = c.parts == 1 ? c.count : std::min(whole, c.count);
    whole -= std::min(whole, c.count);
  }
  return cuts;
}

// blocks are taken by the place on a CU that is free first, the longest ones first; bytes: of memory for each value of a tile
double launch_us(const std::vector<Cut>& list, int w, int bytes) {
  const int per = blocks_of_cu(w), edge = 2 * w;
  std::vector<std::pair<double, int64_t>> blocks;
  double join = 0;
  int64_t all = 0;
  for (const Cut& c : list) {
    const int64_t n = (c.count - c.whole) * c.parts;
    all += c.whole + n;
    if (c.parts > 1) join += (double)n * edge * edge * 8 / 3e6;  // written and read again
  }
  const double share = all > CUS ? (double)std::min<int64_t>(per, cdiv(all, CUS)) : 1.;  // blocks that run on a CU together
  auto add = [&](int steps, int value_bytes, int64_t n) {
    const double mem = (double)edge * edge * value_bytes / (w == 128 ? CU_BYTES_US_ALONE : CU_BYTES_US);
    if (n) blocks.push_back({steps * step_us(w) * (share > 1 ? 0.9 * share : 1.) + block_us(w) + mem * share, n});
  };
  for (const Cut& c : list) {
    add(c.steps, bytes, c.whole);
    add(c.per, c.parts > 1 ? 4 : bytes, (c.count - c.whole) * c.parts);
  }
  std::sort(blocks.begin(), blocks.end(), [](auto& a, auto& b) { return a.first > b.first; });
  const int places = CUS * per;
  std::vector<double> at(places, 0.);  // a heap, the earliest on top
  for (auto& b : blocks) {
    if (b.second > 16 * places) {  // (many alike: a whole round for every place, as often as it goes)
      const int64_t rounds = b.second / places - 1;
      for (double& c : at) c += rounds * b.first;
      b.second -= rounds * places;
    }
    for (int64_t i = 0; i < b.second; ++i) {
      std::pop_heap(at.begin(), at.end(), std::greater<>());
      at.back() += b.first;
      std::push_heap(at.begin(), at.end(), std::greater<>());
    }
  }
  return *std::max_element(at.begin(), at.end()) + (join > 0 ? join + 5.0 : 0.0);
}

// The blocks of a product: its tiles (all of rows x cols, or the lower triangle), cut as `cuts` says. Tiles are taken in
// squares of four by four, so that neighbours share operands, and neighbours go to one XCD: each has its own L2.
void add_list(OrthoPlanHost& p, OrthoList& l, bool lower, int w, const std::vector<Cut>& cuts, bool along_n) {
  l.w = w;
  l.work0 = p.works.size();
  l.join0 = p.joins.size();
  struct Unit { std::vector<OrthoWork> works; double cost = 0; int steps = 0; };
  std::vector<Unit> units;
  for (size_t i = 0; i < p.mats.size(); ++i) {
    const OrthoMat& m = p.mats[i];
    const Cut& cut = cuts[i];
    const int e = 2 * w, tm = cdiv(m.m, e), tn = lower ? tm : cdiv(m.n, e), K = along_n ? m.n : m.m;
    // an eighth of the uncut tiles, of the others' parts
    const size_t unit_whole = std::max(1, cdiv(cut.whole, XCDS)), unit_parts = std::max(1, cdiv((cut.count - cut.whole) * cut.parts, XCDS));
    int64_t tile = 0;
    Unit u;
    auto flush = [&]() { if (!u.works.empty()) units.push_back(std::move(u)); u = Unit(); };
    for (int a4 = 0; a4 < tm; a4 += 4)
      for (int b4 = 0; b4 < (lower ? a4 + 1 : tn); b4 += 4)
        for (int a = a4; a < std::min(tm, a4 + 4); ++a)
          for (int b = b4; b < std::min(lower ? a + 1 : tn, b4 + 4); ++b, ++tile) {
            if (tile == cut.whole) flush();
            const int parts = tile < cut.whole ? 1 : cut.parts, per = parts > 1 ? cut.per : cut.steps;
            if (parts > 1) p.joins.push_back(OrthoJoin{(int)i, a, b, l.slots, parts});
            for (int s = 0; s < parts; ++s) {
              u.works.push_back(OrthoWork{(int)i, a, b, s * per * 32, std::min(K, (s + 1) * per * 32), parts > 1 ? l.slots + s : -1});
              u.steps = per;
              u.cost += per * step_us(w) + block_us(w);
              if (u.works.size() >= (tile < cut.whole ? unit_whole : unit_parts)) flush();
            }
            if (parts > 1) l.slots += parts;
          }
    flush();
  }
  l.joins = (int)(p.joins.size() - l.join0);
  // the longest sums first, each unit to the XCD with the least to do
  std::stable_sort(units.begin(), units.end(), [](const Unit& a, const Unit& b) { return a.steps > b.steps; });
  std::vector<OrthoWork> bin[XCDS];
  double load[XCDS] = {};
  for (const Unit& u : units) {
    const int x = (int)(std::min_element(load, load + XCDS) - load);
    bin[x].insert(bin[x].end(), u.works.begin(), u.works.end());
    load[x] += u.cost;
  }
  size_t most_in = 0;
  for (const auto& b : bin) most_in = std::max(most_in, b.size());
  // block i runs on XCD i % 8
  for (size_t i = 0; i < most_in; ++i)
    for (const auto& b : bin) p.works.push_back(i < b.size() ? b[i] : OrthoWork{-1, 0, 0, 0, 0, -1});
  l.n = (int)(p.works.size() - l.work0);
}

void plan_list(OrthoPlanHost& p, OrthoList& l, bool lower, bool along_n, bool cut, int bytes) {
  int best_w = 32;
  double best = 1e300;
  std::vector<Cut> cuts;
  for (int w : {128, 64, 32})
    for (int most : {1 << 20, 256, 128, 96, 64, 48, 32, 24, 16, 8}) {
      if (most < (1 << 20) && !cut) continue;
      for (bool tail : {false, true}) {
        std::vector<Cut> c = cuts_of(p, lower, along_n, w, most, tail);
        const double us = launch_us(c, w, bytes);
        if (us < best) { best = us; best_w = w; cuts = std::move(c); }
      }
    }
  add_list(p, l, lower, best_w, cuts, along_n);
}

}  // namespace

static int ortho_create(const optorch_matrix_t* matrices, int32_t n, const optorch_ortho_config_t* cfg, optorch_ortho_t** out) {
  if (out) *out = nullptr;
  if (!matrices || !cfg || !out || n < 1) return oseq_mat_err(OPTORCH_E_INVALID, "null argument or empty list of matrices");
  const int steps = cfg->steps <= 0 ? 5 : cfg->steps;
  if (steps > 16) return oseq_mat_err(OPTORCH_E_INVALID, "at most 16 steps");
  std::vector<float> co(3 * steps);
  for (int i = 0; i < 3 * steps; ++i) {
    const float usual[3] = {3.4445f, -4.7750f, 2.0315f};
    co[i] = cfg->coefficients ? cfg->coefficients[i] : usual[i % 3];
    if (!std::isfinite(co[i])) return oseq_mat_err(OPTORCH_E_INVALID, "coefficients must be finite");
  }
  if (cfg->eps != cfg->eps || std::isinf(cfg->eps)) return oseq_mat_err(OPTORCH_E_INVALID, "eps must be finite");
  std::vector<std::pair<int64_t, int>> where;
  for (int i = 0; i < n; ++i) {
    const optorch_matrix_t& m = matrices[i];
    const std::string name = "matrix " + std::to_string(i);
    if (m.rows < 1 || m.cols < 1 || m.rows > (1 << 20) || m.cols > (1 << 20)) return oseq_mat_err(OPTORCH_E_INVALID, name + ": rows and cols must be 1 .. 2^20");
    if (std::min(m.rows, m.cols) > 32768) return oseq_mat_err(OPTORCH_E_INVALID, name + ": the shorter side must be at most 32768");
    if (m.offset < 0 || m.offset > ((int64_t)1 << 48) || m.ld < m.cols || m.ld > (1 << 24)) return oseq_mat_err(OPTORCH_E_INVALID, name + ": bad offset or leading dimension");
    where.push_back({m.offset, i});
  }
  // Matrices side by side in shared rows (equal ld) are fine as long as no element belongs to two.
  std::sort(where.begin(), where.end());
  auto end = [&](const optorch_matrix_t& m) { return m.offset + (m.rows - 1) * m.ld + m.cols; };
  int64_t span = 0;
  for (size_t i = 0; i < where.size(); ++i) {
    const optorch_matrix_t& a = matrices[where[i].second];
    span = std::max(span, end(a));
    for (size_t j = i + 1; j < where.size() && where[j].first < end(a); ++j) {
      const optorch_matrix_t& b = matrices[where[j].second];
      bool apart = false;
      if (a.ld == b.ld) {
        const int64_t d = (b.offset - a.offset) % a.ld;  // b's first column, counted from a's
        apart = d >= a.cols && d + b.cols <= a.ld;
      }
      if (!apart) return oseq_mat_err(OPTORCH_E_INVALID, "matrices " + std::to_string(where[i].second) + " and " + std::to_string(where[j].second) + " overlap");
    }
  }
  optorch_ortho_t* h = new optorch_ortho();
  struct Drop { optorch_ortho_t* h; ~Drop() { delete h; } } drop{h};  // unless it is handed out below
  OrthoPlanHost& p = h->p;
  p.eps = cfg->eps > 0 ? cfg->eps : 1e-7f;
  p.span = span;
  size_t iterates = 0;  // that are made on the way
  for (int k = 0; k < OUT_COUNT; ++k) {
    if (!plan_steps(p, p.launches[k], RESTART[k], steps, co.data()))
      return oseq_mat_err(OPTORCH_E_INVALID, "the coefficients let a singular value grow beyond 64");
    size_t n = 0;
    for (const OrthoLaunch& l : p.launches[k]) n += l.kind == OL_APPLY && !l.last;
    iterates = std::max(iterates, n);
  }
  for (int i = 0; i < n; ++i) {
    const optorch_matrix_t& s = matrices[i];
    OrthoMat m = {};
    m.offset = s.offset; m.ld = s.ld; m.rows = s.rows; m.cols = s.cols;
    m.tall = s.rows > s.cols;
    m.m = up32(std::min(s.rows, s.cols)); m.n = up32(std::max(s.rows, s.cols));
    m.chunk0 = (int)p.chunks.size();
    const int64_t groups = (int64_t)m.m * (m.n / 8);
    if (groups > 0x7fff0000) return oseq_mat_err(OPTORCH_E_INVALID, "matrix " + std::to_string(i) + " has too many elements");
    if (m.tall) {
      for (int r = 0; r < m.n; r += 64)
        for (int c = 0; c < m.m; c += 128) p.chunks.push_back(OrthoChunk{i, c, r});
    } else {
      for (int64_t g = 0; g < groups; g += ORTHO_GROUPS) p.chunks.push_back(OrthoChunk{i, (int32_t)g, 0});
    }
    m.chunks = (int)p.chunks.size() - m.chunk0;
    p.most_m = std::max(p.most_m, m.m);
    p.mats.push_back(m);
  }
  // bytes of memory for each value of a tile: a symmetric result is written twice; Q X: planes, the caller's values,
  // weights read and written with their copy
  plan_list(p, p.gram, true, true, true, 8);
  plan_list(p, p.chain, true, false, true, 8);
  plan_list(p, p.apply, false, false, false, 8);
  plan_list(p, p.last[0], false, false, false, 6);
  plan_list(p, p.last[1], false, false, false, 14);
  uint64_t o = 0;
  auto take = [&](uint64_t bytes) { const uint64_t at = o; o = up256(o + bytes); return at; };
  p.off_mats = take(p.mats.size() * sizeof(OrthoMat));
  p.off_chunks = take(p.chunks.size() * sizeof(OrthoChunk));
  p.off_works = take(p.works.size() * sizeof(OrthoWork));
  p.off_joins = take(p.joins.size() * sizeof(OrthoJoin));
  p.off_partial = take(p.chunks.size() * 8);
  p.off_scale = take(p.mats.size() * 8);
  p.off_bad = take(p.mats.size() * 4 + 4);
  p.off_slots = take(std::max((uint64_t)p.gram.slots * p.gram.w * p.gram.w, 2 * (uint64_t)p.chain.slots * p.chain.w * p.chain.w) * 16);
  // A single iterate on the way is made where the first one lies if a block has all rows of its columns: it has read them
  // before it writes.
  const bool in_place = iterates == 0 || (iterates == 1 && p.most_m <= 2 * p.apply.w);
  for (OrthoMat& m : p.mats) {
    m.x[0] = take((uint64_t)m.m * m.n * 4);
    m.x[1] = in_place ? m.x[0] : take((uint64_t)m.m * m.n * 4);
    m.chain = take((uint64_t)OB_COUNT * m.m * m.m * 4);
  }
  p.bytes = o;
  drop.h = nullptr;
  *out = h;
  return OPTORCH_OK;
}

template <class F> static int ortho_guarded(F&& f) {
  try { return f(); } catch (...) { return oseq_mat_err(OPTORCH_E_INVALID, "out of host memory"); }
}

extern "C" int optorch_ortho_create(const optorch_matrix_t* matrices, int32_t n, const optorch_ortho_config_t* cfg, optorch_ortho_t** out) {
  return ortho_guarded([&] { return ortho_create(matrices, n, cfg, out); });
}

extern "C" int optorch_ortho_query(const optorch_ortho_t* h, uint64_t* workspace_bytes, int64_t* span) {
  if (!h) return oseq_mat_err(OPTORCH_E_INVALID, "null handle");
  if (workspace_bytes) *workspace_bytes = h->p.bytes;
  if (span) *span = h->p.span;
  return OPTORCH_OK;
}

extern "C" int optorch_ortho_bind(optorch_ortho_t* h, void* workspace_dev, uint64_t workspace_bytes) {
  return ortho_guarded([&]() -> int {
    if (!h) return oseq_mat_err(OPTORCH_E_INVALID, "null handle");
    if (!workspace_dev || (uintptr_t)workspace_dev % 256) return oseq_mat_err(OPTORCH_E_INVALID, "workspace must be 256-byte aligned device memory");
    if (workspace_bytes < h->p.bytes) return oseq_mat_err(OPTORCH_E_BUDGET, "workspace too small: " + std::to_string(h->p.bytes) + " bytes are needed");
    const OrthoPlanHost& p = h->p;
    std::vector<char> t(p.off_partial);  // the tables come first
    auto put = [&](uint64_t off, const void* src, size_t bytes) { if (bytes) std::memcpy(t.data() + off, src, bytes); };
    put(p.off_mats, p.mats.data(), p.mats.size() * sizeof(OrthoMat));
    put(p.off_chunks, p.chunks.data(), p.chunks.size() * sizeof(OrthoChunk));
    put(p.off_works, p.works.data(), p.works.size() * sizeof(OrthoWork));
    put(p.off_joins, p.joins.data(), p.joins.size() * sizeof(OrthoJoin));
    h->ws = nullptr;
    const hipError_t e = hipMemcpy(workspace_dev, t.data(), t.size(), hipMemcpyHostToDevice);
    if (e != hipSuccess) return oseq_mat_err(OPTORCH_E_HIP, std::string("hipMemcpy: ") + hipGetErrorString(e));
    h->ws = (char*)workspace_dev;
    return OPTORCH_OK;
  });
}

static bool known(int32_t precision) { return precision == OPTORCH_FP32 || precision == OPTORCH_BF16 || precision == OPTORCH_FP16; }
static bool misaligned(const void* p, int32_t precision) { return (uintptr_t)p % (precision == OPTORCH_FP32 ? 4 : 2) != 0; }

// Flat vectors of one list: whether an element of one matrix shares a byte with an element of another vector's
struct Flat { const char* name; const void* p; int32_t precision; };
static bool overlap(const OrthoPlanHost& p, const Flat& a, const Flat& b) {
  auto bytes = [](const Flat& f) { return f.precision == OPTORCH_FP32 ? 4 : 2; };
  auto place = [&](const Flat& f, const OrthoMat& m) {
    return place_in((const char*)f.p + m.offset * bytes(f), m.rows, m.cols, m.ld, bytes(f));
  };
  const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
  if (pa + (uintptr_t)(p.span * bytes(a)) <= pb || pb + (uintptr_t)(p.span * bytes(b)) <= pa) return false;
  for (const OrthoMat& m : p.mats)
    for (const OrthoMat& o : p.mats)
      if (oseq::overlap(place(a, m), place(b, o))) return true;
  return false;
}
// the same for a check without a device, where no plan is bound (not part of the API)
namespace oseq {
bool ortho_vectors_overlap(const optorch_ortho_t* h, const void* a, int32_t a_precision, const void* b, int32_t b_precision);
bool ortho_vectors_overlap(const optorch_ortho_t* h, const void* a, int32_t a_precision, const void* b, int32_t b_precision) {
  return ::overlap(h->p, Flat{"a", a, a_precision}, Flat{"b", b, b_precision});
}
// how the products of a plan are cut: 1000 * values of a tile's edge + 1 if some sums are cut; list 0: X X^T, 1: m x m, 2:
// Q X on the way, 3: to the caller's vectors, 4: to weights
int ortho_shape(const optorch_ortho_t* h, int list);
int ortho_shape(const optorch_ortho_t* h, int list) {
  const OrthoList& l = list == 0 ? h->p.gram : list == 1 ? h->p.chain : list == 2 ? h->p.apply : h->p.last[list - 3];
  return 2000 * l.w + (l.joins ? 1 : 0);
}
}  // namespace oseq
static int overlap_error(const Flat& a, const Flat& b) {
  return oseq_mat_err(OPTORCH_E_INVALID, std::string(a.name) + " and " + b.name + " overlap");
}

static int ortho_launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return oseq_mat_err(OPTORCH_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
  return OPTORCH_OK;
}

extern "C" int optorch_orthogonalize(optorch_ortho_t* h, int32_t g_precision, const void* g, int32_t o_precision, void* o, void* hip_stream) {
  return ortho_guarded([&]() -> int {
    if (!h) return oseq_mat_err(OPTORCH_E_INVALID, "null handle");
    if (!h->ws) return oseq_mat_err(OPTORCH_E_ORDER, "orthogonalize before bind");
    if (!known(g_precision) || !known(o_precision)) return oseq_mat_err(OPTORCH_E_INVALID, "unknown precision");
    if (!g || !o || misaligned(g, g_precision) || misaligned(o, o_precision)) return oseq_mat_err(OPTORCH_E_INVALID, "null or misaligned vector");
    const Flat fg{"g", g, g_precision}, fo{"o", o, o_precision};
    if (!(g == o && g_precision == o_precision) && overlap(h->p, fg, fo)) return overlap_error(fg, fo);
    OrthoRun r = {};
    r.g_precision = g_precision; r.g = g; r.o_precision = o_precision; r.o = o;
    launch_ortho((hipStream_t)hip_stream, h->p, h->ws, r);
    return ortho_launched("orthogonalize");
  });
}

extern "C" int optorch_muon_update(optorch_ortho_t* h, const optorch_muon_t* a, void* hip_stream) {
  return ortho_guarded([&]() -> int {
    if (!h || !a) return oseq_mat_err(OPTORCH_E_INVALID, "null argument");
    if (!h->ws) return oseq_mat_err(OPTORCH_E_ORDER, "muon_update before bind");
    if (!known(a->g_precision)) return oseq_mat_err(OPTORCH_E_INVALID, "unknown precision");
    if (a->w16 && a->w16_precision != OPTORCH_BF16 && a->w16_precision != OPTORCH_FP16) return oseq_mat_err(OPTORCH_E_INVALID, "w16 must be bf16 or fp16");
    if (!a->g || !a->w || !a->v || misaligned(a->g, a->g_precision) || misaligned(a->w, OPTORCH_FP32) || misaligned(a->v, OPTORCH_FP32) ||
        misaligned(a->w16, OPTORCH_BF16) || misaligned(a->skipped, OPTORCH_FP32))
      return oseq_mat_err(OPTORCH_E_INVALID, "null or misaligned vector");
    if (a->scale_mode < OPTORCH_SCALE_NONE || a->scale_mode > OPTORCH_SCALE_RMS) return oseq_mat_err(OPTORCH_E_INVALID, "unknown scale mode");
    if (!std::isfinite(a->lr) || !std::isfinite(a->momentum) || !std::isfinite(a->weight_decay) || !std::isfinite(a->grad_scale))
      return oseq_mat_err(OPTORCH_E_INVALID, "lr, momentum, weight_decay and grad_scale must be finite");
    const Flat f[4] = {{"g", a->g, a->g_precision}, {"w", a->w, OPTORCH_FP32}, {"v", a->v, OPTORCH_FP32},
                       {"w16", a->w16, a->w16_precision}};
    for (int i = 0; i < 4; ++i)
      for (int j = i + 1; j < (a->w16 ? 4 : 3); ++j)
        if (overlap(h->p, f[i], f[j])) return overlap_error(f[i], f[j]);
    OrthoRun r = {};
    r.g_precision = a->g_precision; r.g = a->g; r.muon = true; r.m = *a;
    launch_ortho((hipStream_t)hip_stream, h->p, h->ws, r);
    return ortho_launched("muon_update");
  });
}

extern "C" void optorch_ortho_destroy(optorch_ortho_t* h) { delete h; }
