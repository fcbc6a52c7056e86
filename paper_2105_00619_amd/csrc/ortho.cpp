// Host side of the orthogonalised updates: the plan of a list of matrices (optorch_ortho_*).
//
// A Newton-Schulz step X <- (a + b A + c A^2) X with A = X X^T changes the singular values of X alone, so that the steps can be
// made on A: with P = a + b A + c A^2,  A <- P A P  and  Q <- P Q,  and in the end X <- Q X.  Only A = X X^T at the start and
// Q X at the end touch the long side of X; all other products are m x m and symmetric, so that half of their tiles are made.  For
// m = n that costs what the steps on X cost (20 m^3 for five steps), for n = 4 m 38 m^3 instead of 65.  But an error of A grows by
// a^2 a step in the directions of small singular values, and rounding errors of A are not small against those: after five
// steps on A the result is off by up to 3e-4.  So after three steps X is made and A from it again: 1e-6 to 2e-5, what the
// steps on X give in fp32.
//
// The operands are pairs of fp16 planes (hi + lo, 22 bits and a sign), times a power of two for each kind of matrix, since
// the bounds of all of them are known (host: from the polynomials): three products of 16-bit matrix cores for one, with an error
// of 2^-24 a value.  One plane alone would do for a bf16 result of well-conditioned matrices, but is 1e-2 off where a few singular
// values are large: in small directions an error of the first iterate is multiplied by 485.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
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

constexpr int RESTART = 3;  // steps on A between two iterates

// The launches and their scales.  Returns false where the steps let a singular value grow too far.
bool plan_steps(OrthoPlanHost& p, int steps, const float* co) {
  constexpr int GRID = 4096;
  std::vector<double> l(GRID + 1), q(GRID + 1);
  for (int i = 0; i <= GRID; ++i) l[i] = (double)i / GRID;  // squares of singular values; sampled, the bounds have a margin
  double xmax = 1.0;
  int src = 0;
  auto top = [&](auto f) { double t = 0; for (int i = 0; i <= GRID; ++i) t = std::max(t, std::fabs(f(i))); return t * 1.01; };
  p.first_scale = plane_scale(1.0);
  float sx = p.first_scale;
  for (int s = 0; s < steps;) {
    const int e = std::min(steps, s + RESTART);
    const double amax = top([&](int i) { return l[i]; });
    float sa = plane_scale(amax), sq = 1.f;
    OrthoLaunch g = {};
    g.kind = OL_GRAM; g.src = src; g.ops = 1;
    g.op[0] = OrthoOp{0, 0, OB_A, -1, sa / (sx * sx), 0.f, 0.f};
    p.launches.push_back(g);
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
      p.launches.push_back(lp);
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
        p.launches.push_back(ln);
        OrthoLaunch la = {};
        la.kind = OL_CHAIN; la.ops = 1;
        la.op[0] = OrthoOp{OB_C, pbuf, OB_A, -1, sa_new / (sc * sp), 0.f, 0.f};
        p.launches.push_back(la);
        sa = sa_new;
      } else {
        for (int i = 0; i <= GRID; ++i) { const double t = poly(i); l[i] *= t * t; }
        if (k > s) {
          ln.op[ln.ops++] = OrthoOp{OB_P, qbuf, qbuf ^ OB_Q0 ^ OB_Q1, -1, sq_new / (sp * sq), 0.f, 0.f};
          qbuf ^= OB_Q0 ^ OB_Q1;
          sq = sq_new;
          p.launches.push_back(ln);
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
    p.launches.push_back(x);
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
int64_t tiles_of(int64_t m, int64_t n, int w) { return (int64_t)cdiv(m, 2 * w) * cdiv(n, 2 * w); }

// the largest tiles that give the CUs work
template <class F> int tile_for(F&& count) {
  for (int w : {128, 64})
    if (count(w) >= 256) return w;
  return 32;
}

void plan_works(OrthoPlanHost& p) {
  auto tri = [](int64_t t) { return t * (t + 1) / 2; };
  auto chain_tiles = [&](int w) { int64_t n = 0; for (const OrthoMat& m : p.mats) n += tri(cdiv(m.mp, 2 * w)); return n; };
  p.w_chain = tile_for(chain_tiles);
  p.w_apply = tile_for([&](int w) { int64_t n = 0; for (const OrthoMat& m : p.mats) n += tiles_of(m.rp, m.cp, w); return n; });
  p.w_gram = tile_for(chain_tiles);
  // longest sums first
  std::vector<int> order(p.mats.size());
  for (size_t i = 0; i < order.size(); ++i) order[i] = (int)i;
  auto list = [&](OrthoList& l, auto&& add) {
    l.off = p.works.size();
    for (int i : order) add(i, p.mats[i]);
    l.n = (int)(p.works.size() - l.off);
  };
  auto by = [&](auto key) { std::stable_sort(order.begin(), order.end(), [&](int i, int j) { return key(p.mats[i]) > key(p.mats[j]); }); };
  by([](const OrthoMat& m) { return m.mp; });
  list(p.chain, [&](int i, const OrthoMat& m) {
    const int t = cdiv(m.mp, 2 * p.w_chain);
    for (int a = 0; a < t; ++a)
      for (int b = 0; b <= a; ++b) p.works.push_back(OrthoWork{i, a, b, 0, m.mp, -1});
  });
  for (int tall = 0; tall < 2; ++tall)
    list(p.apply[tall], [&](int i, const OrthoMat& m) {
      if (m.tall != tall) return;
      const int tm = cdiv(m.rp, 2 * p.w_apply), tn = cdiv(m.cp, 2 * p.w_apply);
      // (bands of eight rows of tiles: neighbours share operands)
      for (int band = 0; band < tm; band += 8)
        for (int b = 0; b < tn; ++b)
          for (int a = band; a < std::min(tm, band + 8); ++a) p.works.push_back(OrthoWork{i, a, b, 0, m.mp, -1});
    });
  // X X^T: the long sums are cut where there are few tiles
  by([](const OrthoMat& m) { return std::max(m.rp, m.cp); });
  int64_t steps = 0;
  for (const OrthoMat& m : p.mats) steps += tri(cdiv(m.mp, 2 * p.w_gram)) * cdiv(std::max(m.rp, m.cp), 64);
  const int64_t share = std::max<int64_t>(4, (steps + 511) / 512);  // 64-deep steps a block should have
  for (int tall = 0; tall < 2; ++tall)
    list(p.gram[tall], [&](int i, const OrthoMat& m) {
      if (m.tall != tall) return;
      const int K = std::max(m.rp, m.cp), ks = cdiv(K, 64), t = cdiv(m.mp, 2 * p.w_gram);
      int parts = (int)std::min<int64_t>(32, std::max<int64_t>(1, (ks + share / 2) / share));
      const int per = cdiv(ks, parts) * 64;
      parts = cdiv(K, per);
      for (int a = 0; a < t; ++a)
        for (int b = 0; b <= a; ++b) {
          if (parts > 1) p.joins.push_back(OrthoJoin{i, a, b, p.slots, parts});
          for (int s = 0; s < parts; ++s)
            p.works.push_back(OrthoWork{i, a, b, s * per, std::min(K, (s + 1) * per), parts > 1 ? p.slots + s : -1});
          if (parts > 1) p.slots += parts;
        }
    });
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
  if (!plan_steps(p, steps, co.data()))
    return oseq_mat_err(OPTORCH_E_INVALID, "the coefficients let a singular value grow beyond 64");
  for (int i = 0; i < n; ++i) {
    const optorch_matrix_t& s = matrices[i];
    OrthoMat m = {};
    m.offset = s.offset; m.ld = s.ld; m.rows = s.rows; m.cols = s.cols;
    m.rp = up32(s.rows); m.cp = up32(s.cols); m.mp = std::min(m.rp, m.cp);
    m.tall = m.rp > m.cp;
    m.chunk0 = (int)p.chunks.size();
    const int64_t groups = (int64_t)m.rp * (m.cp / 8);
    if (groups > 0x7fff0000) return oseq_mat_err(OPTORCH_E_INVALID, "matrix " + std::to_string(i) + " has too many elements");
    for (int64_t g = 0; g < groups; g += ORTHO_GROUPS) p.chunks.push_back(OrthoChunk{i, (int32_t)g});
    m.chunks = (int)p.chunks.size() - m.chunk0;
    p.mats.push_back(m);
  }
  plan_works(p);
  uint64_t o = 0;
  auto take = [&](uint64_t bytes) { const uint64_t at = o; o = up256(o + bytes); return at; };
  p.off_mats = take(p.mats.size() * sizeof(OrthoMat));
  p.off_chunks = take(p.chunks.size() * sizeof(OrthoChunk));
  p.off_works = take(p.works.size() * sizeof(OrthoWork));
  p.off_joins = take(p.joins.size() * sizeof(OrthoJoin));
  p.off_partial = take(p.chunks.size() * 8);
  p.off_scale = take(p.mats.size() * 8);
  p.off_bad = take(p.mats.size() * 4 + 4);
  p.off_slots = take((uint64_t)p.slots * (2 * p.w_gram) * (2 * p.w_gram) * 4);
  const bool two = steps > RESTART;
  for (OrthoMat& m : p.mats) {
    m.x[0] = take((uint64_t)m.rp * m.cp * 4);
    m.x[1] = two ? take((uint64_t)m.rp * m.cp * 4) : m.x[0];
    m.chain = take((uint64_t)OB_COUNT * m.mp * m.mp * 4);
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
    OrthoRun r = {};
    r.g_precision = a->g_precision; r.g = a->g; r.muon = true; r.m = *a;
    launch_ortho((hipStream_t)hip_stream, h->p, h->ws, r);
    return ortho_launched("muon_update");
  });
}

extern "C" void optorch_ortho_destroy(optorch_ortho_t* h) { delete h; }
