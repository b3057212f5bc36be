// Host runtime of the orthogonalised updates (include/edit_outer.h,
// "orthogonalised updates").
//
// A handle owns, for one unit layout, a workspace for every matrix and the
// tables its launches run over: chunks of the unit for the streaming passes,
// tiles of all matrices for the products.  A call enqueues source -> load ->
// steps x (gram, square, update; after a symmetric product the join of what was
// cut) on the caller's stream, or one launch for
// small matrices.
#include <algorithm>
#include <cmath>
#include <memory>
#include <string>
#include <vector>

#include "edit_group_internal.h"
#include "edit_ortho_internal.h"

using namespace edit;

namespace {

#define ORTHO_TRY(expr)               \
  do {                                \
    const edit_status_t st_ = (expr); \
    if (st_ != EDIT_OK) return st_;   \
  } while (0)

edit_status_t ofail(edit_status_t s, const std::string& msg) { return set_error(s, msg.c_str()); }

edit_status_t ofail_hip(hipError_t e, const char* what) {
  return ofail(EDIT_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

int64_t oceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t oround_up(int64_t a, int64_t b) { return oceil_div(a, b) * b; }

constexpr double kDefaultCoef[3] = {3.4445, -4.7750, 2.0315};
constexpr int64_t kMaxSide = int64_t(1) << 24;
constexpr int64_t kMaxMatrix = int64_t(1) << 29;
constexpr int kGapChunks = 4096;                  // blocks for a run of elements of no matrix, at most
// Sides of the products' tiles.  A CU runs two 128 x 128 tiles side by side at
// about the time of one, and 64 x 64 tiles take up to 1.4 times the time per
// operation but fill the GPU with a quarter of the work.  us at 128 and 64, n
// matrices of 1024 x 1024 (FAST): symmetric products of 40 tiles (of 128 x
// 128) 19 and 8, 160: 22 and 18, 240: 23 and 24, 280: 33 and 25, 400: 34 and
// 33, 480: 35 and 39 (with the XCDs' shares as spread_tiles() deals them, of
// which some are a quarter larger than others where a matrix's tiles do not
// divide by eight); update product of 64 tiles 14 and 8, 192: 18 and 15, 256:
// 19 and 20, 512: 29 and 35.
//
// FAST's update product of much work takes 256 x 256 tiles, which load half as
// much per operation, but a CU runs one at a time, so that the last round of
// them has to be nearly full.  us at 128 and 256: 192 tiles (of 256 x 256) of
// r = 1024 43 and 45, 256: 53 and 51, 384: 77 and 89, 512: 111 and 103; r =
// 2048, 256: 80 and 71, 384: 116 and 130, 512: 163 and 145; r = 4096, 256: 138
// and 120.  Whole calls: one 4096 x 11008 matrix (688 tiles) 3830 and 3670, a
// 1B layer's local step (784, the last round nearly empty) 2533 and 2563.
// FULL's is bound by its operations, and has no registers for them.
constexpr int kLargeSide = kOrthoLargeSide, kSmallSide = 64, kHugeSide = 256;
// 64 x 64 tiles take four slabs in LDS instead of two where the blocks that
// then fit, two a CU, are all there are.  Whole calls, us with two and four: one
// 1024 x 1024 matrix, FULL (256 tiles) 238 and 208; a layer of hidden size 256
// (88 and 208) 106.5 and 99.2.  With more tiles: 208 and 234 where that matrix's
// gram product has 544; a 350M layer (952) 501 and 523.
int few_tiles(int num_cu) { return 2 * num_cu; }
int symmetric_side(int64_t large_tiles, int num_cu) { return 2 * large_tiles <= 3 * num_cu ? kSmallSide : kLargeSide; }
int update_side(int64_t large_tiles, int64_t huge_tiles, int num_cu, bool full) {
  if (large_tiles < num_cu) return kSmallSide;
  const int64_t idle = oround_up(huge_tiles, num_cu) - huge_tiles;  // CUs of the last round
  const bool padded = 10 * 4 * huge_tiles > 11 * large_tiles;  // more work for it than it saves
  return !full && !padded && 8 * idle <= huge_tiles ? kHugeSide : kLargeSide;
}
// Side, in tiles, of the groups that tiles are taken in.  Products of a 1B
// layer and of a 4096 x 11008 matrix, us with groups of 1, 2, 4 and 8: update
// (FAST) 294, 259, 255, 260 and 465, 410, 373, 375; gram 164, 149, 148, 149
// and 286, 265, 265, 263.
constexpr int32_t kGroup = 4;

struct Tables {
  std::vector<OrthoMat> mats;
  std::vector<OrthoChunk> chunks;
  int matrix_chunks = 0;  // the first ones belong to matrices
  std::vector<OrthoTile> load, gram, gram_join, square, square_join, update;
  int pieces = 0;  // of one product at most
  int gram_side = kLargeSide, update_side = kLargeSide;
  bool small = false;  // one block takes each matrix whole
};

}  // namespace

struct edit_ortho {
  int64_t numel = 0;
  bool bf16 = false, full = false;
  int device = 0;
  std::vector<OrthoCoef> coef;
  char* arena = nullptr;
  OrthoMat* mats = nullptr;
  OrthoChunk* chunks = nullptr;
  int matrix_chunks = 0, all_chunks = 0;
  OrthoTile* load = nullptr;
  int load_tiles = 0;
  OrthoTiles gram{}, gram_join{}, square{}, square_join{}, update{};
  float* pieces = nullptr;
  int gram_side = 0, update_side = 0;
  bool small = false;
  int matrices = 0, widest = 0;  // widest: the largest r
  float* u = nullptr;
};

namespace {

// Singular values start within [0, 1] (the Frobenius norm is 1); their images
// and the polynomial have to stay within what the fp16 scales leave room for.
edit_status_t check_coefficients(const std::vector<OrthoCoef>& coef) {
  double top = 1.0;
  for (size_t k = 0; k < coef.size(); ++k) {
    const OrthoCoef& q = coef[k];
    const std::string where = "coefficients of step " + std::to_string(k);
    if (!std::isfinite(q.a) || !std::isfinite(q.b) || !std::isfinite(q.c))
      return ofail(EDIT_EINVAL, where + " must be finite");
    constexpr int kGrid = 4096;
    double next = 0.0, poly = 0.0;
    for (int i = 0; i <= kGrid; ++i) {
      const double s = top * i / kGrid, x = s * s, p = q.a + q.b * x + q.c * x * x;
      poly = std::max(poly, std::fabs(p));
      next = std::max(next, std::fabs(s * p));
    }
    if (!(poly <= kMaxPoly)) return ofail(EDIT_EINVAL, where + ": |a + b x + c x^2| exceeds 15");
    if (!(next <= kMaxSigma)) return ofail(EDIT_EINVAL, where + " take a singular value beyond 4");
    top = next;
  }
  return EDIT_OK;
}

edit_status_t check_layout(const edit_ortho_config_t* cfg) {
  if (cfg->numel < 0) return ofail(EDIT_EINVAL, "numel must be >= 0");
  if (cfg->num_matrices < 0) return ofail(EDIT_EINVAL, "num_matrices must be >= 0");
  if (cfg->num_matrices > 0 && !cfg->matrices) return ofail(EDIT_EINVAL, "matrices must not be NULL");
  if (cfg->dtype != EDIT_F32 && cfg->dtype != EDIT_BF16)
    return ofail(EDIT_EINVAL, "dtype must be EDIT_F32 or EDIT_BF16");
  if (cfg->precision != EDIT_ORTHO_FAST && cfg->precision != EDIT_ORTHO_FULL)
    return ofail(EDIT_EINVAL, "precision must be EDIT_ORTHO_FAST or EDIT_ORTHO_FULL");
  if (cfg->steps < 1 || cfg->steps > EDIT_ORTHO_MAX_STEPS)
    return ofail(EDIT_EINVAL, "steps must be in 1.." + std::to_string(EDIT_ORTHO_MAX_STEPS));
  std::vector<std::pair<int64_t, int64_t>> used;
  for (int i = 0; i < cfg->num_matrices; ++i) {
    const edit_ortho_matrix_t& m = cfg->matrices[i];
    const std::string where = "matrix " + std::to_string(i);
    if (m.rows < 0 || m.cols < 0) return ofail(EDIT_EINVAL, where + ": rows and cols must be >= 0");
    if (m.rows > kMaxSide || m.cols > kMaxSide) return ofail(EDIT_EINVAL, where + ": rows and cols must be at most 2^24");
    const int64_t n = static_cast<int64_t>(m.rows) * m.cols;
    // Padding the short side to a multiple of 64 at most doubles it from 32 on,
    // and 64 sides of 2^24 are 2^30: at four bytes, offsets stay below 2^32.
    if (n > kMaxMatrix) return ofail(EDIT_EINVAL, where + " is too large");
    if (m.offset < 0 || m.offset > cfg->numel || n > cfg->numel - m.offset)
      return ofail(EDIT_EINVAL, where + " reaches beyond the unit");
    if (!std::isfinite(m.scale)) return ofail(EDIT_EINVAL, where + ": scale must be finite");
    if (n) used.push_back({m.offset, m.offset + n});
  }
  std::sort(used.begin(), used.end());
  for (size_t i = 1; i < used.size(); ++i)
    if (used[i].first < used[i - 1].second) return ofail(EDIT_EINVAL, "matrices must not overlap");
  return EDIT_OK;
}

// [begin, end) in about `most` chunks at most, cut at whole vectors: one a thread
// at least (four: 272 us for 264 of a 1024 x 1024 matrix's outer step).
void add_chunks(std::vector<OrthoChunk>& out, int64_t begin, int64_t end, int mat, int most, int* count) {
  constexpr int64_t kUnit = 2048;
  const int64_t size = std::max(kUnit, oround_up(oceil_div(end - begin, most), kUnit));
  int slot = 0;
  for (int64_t at = begin; at < end;) {
    const int64_t to = std::min(end, at / kUnit * kUnit + size);
    out.push_back({at, to, mat, slot++});
    at = to;
  }
  if (count) *count = slot;
}

Tables make_tables(const edit_ortho_config_t* cfg, int num_cu) {
  Tables t;
  std::vector<std::pair<int64_t, int64_t>> used;
  std::vector<std::vector<OrthoTile>> gram, square, update;
  for (int i = 0; i < cfg->num_matrices; ++i) {
    const edit_ortho_matrix_t& in = cfg->matrices[i];
    if (in.rows == 0 || in.cols == 0) continue;
    const int k = static_cast<int>(t.mats.size());
    OrthoMat m = {};
    m.offset = in.offset;
    m.scale = in.scale;
    m.rows = in.rows, m.cols = in.cols;
    m.r = std::min(in.rows, in.cols), m.c = std::max(in.rows, in.cols);
    m.ldr = static_cast<int32_t>(oround_up(m.r, kOrthoPad));
    m.tall = in.rows > in.cols;
    const int64_t end = in.offset + static_cast<int64_t>(in.rows) * in.cols;
    used.push_back({in.offset, end});
    add_chunks(t.chunks, in.offset, end, k, kOrthoMaxChunks, &m.chunks);
    for (int32_t a = 0; a < oceil_div(in.rows, kOrthoLoadTile); ++a)
      for (int32_t b = 0; b < oceil_div(in.cols, kOrthoLoadTile); ++b) t.load.push_back({k, a, b, 0, 0, 0});
    t.mats.push_back(m);
  }
  const bool full = cfg->precision == EDIT_ORTHO_FULL;
  int64_t symmetric = 0, whole = 0, huge = 0;  // tiles at the large side; at the huge one
  for (const OrthoMat& m : t.mats) {
    const int64_t tr = oceil_div(m.r, kLargeSide), tc = oceil_div(m.c, kLargeSide);
    symmetric += tr * (tr + 1) / 2;
    whole += tr * tc;
    huge += oceil_div(m.r, kHugeSide) * oceil_div(m.c, kHugeSide);
  }
  t.small = !t.mats.empty() && std::all_of(t.mats.begin(), t.mats.end(),
                                           [](const OrthoMat& m) { return ortho_is_small(m.r, m.c); });
  t.gram_side = symmetric_side(symmetric, num_cu);
  t.update_side = update_side(whole, huge, num_cu, full);
  const int slab = ortho_slab(full);
  for (size_t k = 0; k < t.mats.size(); ++k) {
    OrthoMat& m = t.mats[k];
    const int32_t id = static_cast<int32_t>(k);
    // in groups of kGroup x kGroup tiles, which share operands while they run
    const int32_t ts = static_cast<int32_t>(oceil_div(m.r, t.gram_side));
    const int32_t slabs_r = m.ldr / slab, slabs_c = static_cast<int32_t>(oround_up(m.c, kOrthoPad)) / slab;
    gram.emplace_back();
    square.emplace_back();
    for (int32_t p = 0; p < ts; p += kGroup)
      for (int32_t q = 0; q <= p; q += kGroup)
        for (int32_t a = p; a < std::min(ts, p + kGroup); ++a)
          for (int32_t b = q; b <= std::min(a, q + kGroup - 1); ++b) {
            square.back().push_back({id, a, b, -1, 0, slabs_r});
            gram.back().push_back({id, a, b, -1, 0, slabs_c});
          }
    const int32_t tr = static_cast<int32_t>(oceil_div(m.r, t.update_side));
    const int32_t tc = static_cast<int32_t>(oceil_div(m.c, t.update_side));
    update.emplace_back();
    for (int32_t q = 0; q < tc; q += kGroup)
      for (int32_t p = 0; p < tr; p += kGroup)
        for (int32_t b = q; b < std::min(tc, q + kGroup); ++b)
          for (int32_t a = p; a < std::min(tr, p + kGroup); ++a) update.back().push_back({id, a, b, m.x_tiles++, 0, slabs_r});
  }
  t.matrix_chunks = static_cast<int>(t.chunks.size());
  std::sort(used.begin(), used.end());
  int64_t at = 0;
  used.push_back({cfg->numel, cfg->numel});
  for (const auto& [lo, hi] : used) {
    if (lo > at) add_chunks(t.chunks, at, lo, -1, kGapChunks, nullptr);
    at = hi;
  }
  std::vector<int> order(t.mats.size());
  for (size_t i = 0; i < order.size(); ++i) order[i] = static_cast<int>(i);
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return t.mats[a].c > t.mats[b].c; });
  t.pieces = cut_tiles(gram, order, t.gram_side, num_cu, &t.gram, &t.gram_join);
  std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return t.mats[a].r > t.mats[b].r; });
  t.pieces = std::max(t.pieces, cut_tiles(square, order, t.gram_side, num_cu, &t.square, &t.square_join));
  t.update = spread_tiles(update, order);
  return t;
}

// Hands out 256-byte aligned pieces of the arena; with no arena it counts.
struct Carver {
  char* base;
  size_t at = 0;
  template <typename T>
  T* take(size_t count) {
    const size_t here = at;
    at += (count * sizeof(T) + 255) & ~size_t(255);
    return base ? reinterpret_cast<T*>(base + here) : nullptr;
  }
};

size_t lay_out(edit_ortho* h, Tables& t, char* base, int num_cu) {
  auto tiles = [&](const OrthoTile* at, const std::vector<OrthoTile>& list) {
    return OrthoTiles{at, static_cast<int32_t>(list.size()), static_cast<int>(list.size()) <= few_tiles(num_cu)};
  };
  Carver c{base};
  for (OrthoMat& m : t.mats) {
    const size_t xt = static_cast<size_t>(oround_up(m.c, kOrthoPad)) * m.ldr, a = static_cast<size_t>(m.r) * m.ldr;
    if (h->full) {
      m.t[0][0] = c.take<_Float16>(2 * xt), m.t[1][0] = c.take<_Float16>(2 * xt);
      m.g[0] = c.take<_Float16>(2 * a), m.q[0] = c.take<_Float16>(2 * a);
    } else {  // X's low half is read and written in place
      m.t[0][0] = c.take<_Float16>(xt), m.t[1][0] = c.take<_Float16>(xt);
      m.t[0][1] = m.t[1][1] = c.take<_Float16>(xt);
      m.g[0] = c.take<_Float16>(a), m.q[0] = c.take<_Float16>(a);
    }
    m.norm_part = c.take<double>(m.chunks);
    m.x_part = c.take<double>(m.x_tiles);
    m.shift = c.take<double>(1);
  }
  h->u = c.take<float>(static_cast<size_t>(h->numel));
  h->mats = c.take<OrthoMat>(t.mats.size());
  h->chunks = c.take<OrthoChunk>(t.chunks.size());
  h->load = c.take<OrthoTile>(t.load.size());
  OrthoTile* gram = c.take<OrthoTile>(t.gram.size());
  OrthoTile* update = c.take<OrthoTile>(t.update.size());
  OrthoTile* gram_join = c.take<OrthoTile>(t.gram_join.size());
  OrthoTile* square = c.take<OrthoTile>(t.square.size());
  OrthoTile* square_join = c.take<OrthoTile>(t.square_join.size());
  h->pieces = c.take<float>(static_cast<size_t>(t.pieces) * t.gram_side * t.gram_side);
  h->gram_join = tiles(gram_join, t.gram_join);
  h->square = tiles(square, t.square);
  h->square_join = tiles(square_join, t.square_join);
  h->gram = tiles(gram, t.gram);
  h->update = tiles(update, t.update);
  h->gram_side = t.gram_side, h->update_side = t.update_side;
  h->small = t.small;
  h->matrices = static_cast<int>(t.mats.size());
  for (const OrthoMat& m : t.mats) h->widest = std::max(h->widest, m.r);
  h->matrix_chunks = t.matrix_chunks;
  h->all_chunks = static_cast<int>(t.chunks.size());
  h->load_tiles = static_cast<int>(t.load.size());
  return c.at;
}

template <typename T>
hipError_t upload(const T* to, const std::vector<T>& from) {
  if (from.empty()) return hipSuccess;
  return hipMemcpy(const_cast<T*>(to), from.data(), from.size() * sizeof(T), hipMemcpyHostToDevice);
}

edit_status_t check_ortho_device(const edit_ortho* h) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return ofail_hip(e, "hipGetDevice");
  if (dev != h->device)
    return ofail(EDIT_EINVAL, "call made with device " + std::to_string(dev) +
                                  " current; the handle belongs to device " + std::to_string(h->device));
  return EDIT_OK;
}

edit_status_t check_buffer(const void* p, const char* name) {
  if (!p) return ofail(EDIT_EINVAL, std::string(name) + " must not be NULL");
  if (reinterpret_cast<uintptr_t>(p) & 15u) return ofail(EDIT_EINVAL, std::string(name) + " must be 16-byte aligned");
  return EDIT_OK;
}

bool buffers_overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + static_cast<uintptr_t>(b_bytes) && y < x + static_cast<uintptr_t>(a_bytes);
}

edit_status_t enqueue(edit_ortho* h, OrthoCall call, hipStream_t s) {
  call.u = h->u;
  const int steps = static_cast<int>(h->coef.size());
  hipError_t e = hipSuccess;
  if (h->small) {
    if (call.source == kSourceOuter) e = launch_ortho_source(call, h->mats, h->chunks, h->all_chunks, s);
    if (e == hipSuccess) e = launch_ortho_small(h->full, call, h->mats, h->matrices, h->widest, h->coef.data(), steps, s);
    return e == hipSuccess ? EDIT_OK : ofail_hip(e, "small matrices launch");
  }
  e = launch_ortho_source(call, h->mats, h->chunks,
                                     call.source == kSourceOuter ? h->all_chunks : h->matrix_chunks, s);
  if (e != hipSuccess) return ofail_hip(e, "source pass launch");
  if (h->matrix_chunks == 0) return EDIT_OK;
  if ((e = launch_ortho_load(h->full, call, h->mats, h->load, h->load_tiles, s)) != hipSuccess)
    return ofail_hip(e, "load pass launch");
  for (int k = 0; k < steps; ++k) {
    auto product = [&](OrthoProduct p, int side, const OrthoTiles& tiles) {
      if (e == hipSuccess)
        e = launch_ortho_product(p, h->full, side, h->mats, tiles, h->coef[k], k, steps, call, h->pieces, s);
    };
    product(kProductGram, h->gram_side, h->gram);
    product(kProductGramJoin, h->gram_side, h->gram_join);
    product(kProductSquare, h->gram_side, h->square);
    product(kProductSquareJoin, h->gram_side, h->square_join);
    product(kProductUpdate, h->update_side, h->update);
    if (e != hipSuccess) return ofail_hip(e, "product launch");
  }
  return EDIT_OK;
}

}  // namespace

namespace edit {

edit_status_t check_ortho_unit(const edit_ortho* h, int64_t numel, int device) {
  if (h->numel != numel)
    return ofail(EDIT_EINVAL, "the ortho handle is for units of " + std::to_string(h->numel) + " elements, the unit has " +
                                  std::to_string(numel));
  if (h->device != device)
    return ofail(EDIT_EINVAL, "the ortho handle belongs to device " + std::to_string(h->device));
  return EDIT_OK;
}

edit_status_t enqueue_ortho_outer(edit_ortho* h, bool bf16, float* theta, float* momentum, void* const* replicas,
                                  int workers, const UnitRecord* rec, double lr, double rho, hipStream_t stream) {
  OrthoCall c = {};
  c.source = kSourceOuter;
  c.bf16 = bf16;
  c.momentum = momentum;
  c.theta = theta;
  c.reps = replicas;
  c.rec = rec;
  c.workers = h->numel == 0 ? 0 : workers;
  c.mu = rho;
  c.lr = lr;
  return enqueue(h, c, stream);
}

}  // namespace edit

extern "C" {

edit_status_t edit_ortho_init(const edit_ortho_config_t* cfg, edit_ortho_t* out) {
  set_error(EDIT_OK, "");
  if (!cfg || !out) return ofail(EDIT_EINVAL, "cfg and out must not be NULL");
  *out = nullptr;
  try {
    ORTHO_TRY(check_layout(cfg));
    std::vector<OrthoCoef> coef(cfg->steps);
    for (int k = 0; k < cfg->steps; ++k) {
      const double* q = cfg->coefficients ? cfg->coefficients + 3 * k : kDefaultCoef;
      coef[k] = {q[0], q[1], q[2]};
    }
    ORTHO_TRY(check_coefficients(coef));
    int dev = 0, num_cu = 0;
    ORTHO_TRY(current_gfx950(&dev, &num_cu));
    auto h = std::make_unique<edit_ortho>();
    h->numel = cfg->numel;
    h->bf16 = cfg->dtype == EDIT_BF16;
    h->full = cfg->precision == EDIT_ORTHO_FULL;
    h->device = dev;
    h->coef = coef;
    Tables t = make_tables(cfg, num_cu);
    // a launch takes less than 2^32 threads; no kernel has more than 512 a block
    for (const size_t blocks : {t.mats.size(), t.chunks.size(), t.load.size(), t.gram.size(), t.square.size(), t.update.size(),
                                4 * t.gram_join.size(), 4 * t.square_join.size()})
      if (blocks >= (size_t(1) << 32) / 512) return ofail(EDIT_EINVAL, "too many matrices, gaps or tiles for one launch");
    const size_t total = std::max<size_t>(lay_out(h.get(), t, nullptr, num_cu), 256);
    hipError_t e = hipMalloc(reinterpret_cast<void**>(&h->arena), total);
    if (e != hipSuccess) return ofail(EDIT_ENOMEM, std::string("hipMalloc of the workspace: ") + hipGetErrorString(e));
    e = hipMemset(h->arena, 0, total);  // what pads the matrices stays zero
    lay_out(h.get(), t, h->arena, num_cu);
    if (e == hipSuccess) e = upload(h->mats, t.mats);
    if (e == hipSuccess) e = upload(h->chunks, t.chunks);
    if (e == hipSuccess) e = upload(h->load, t.load);
    if (e == hipSuccess) e = upload(h->gram.tile, t.gram);
    if (e == hipSuccess) e = upload(h->update.tile, t.update);
    if (e == hipSuccess) e = upload(h->gram_join.tile, t.gram_join);
    if (e == hipSuccess) e = upload(h->square.tile, t.square);
    if (e == hipSuccess) e = upload(h->square_join.tile, t.square_join);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) {
      (void)hipFree(h->arena);
      return ofail_hip(e, "edit_ortho_init");
    }
    *out = h.release();
    return EDIT_OK;
  } catch (const std::exception&) {  // the tables' host memory
    return ofail(EDIT_ENOMEM, "host allocation failed");
  }
}

edit_status_t edit_ortho_apply(edit_ortho_t h, const void* x, void* out, void* stream) {
  if (!h) return ofail(EDIT_EINVAL, "NULL handle");
  ORTHO_TRY(check_ortho_device(h));
  if (h->matrix_chunks == 0) return EDIT_OK;
  ORTHO_TRY(check_buffer(x, "x"));
  ORTHO_TRY(check_buffer(out, "out"));
  const int64_t bytes = h->numel * (h->bf16 ? 2 : 4);
  if (x != out && buffers_overlap(x, bytes, out, bytes))
    return ofail(EDIT_EINVAL, "x and out must be the same buffer or not overlap");
  OrthoCall c = {};
  c.source = kSourcePlain;
  c.bf16 = h->bf16;
  c.x = x;
  c.out = out;
  return enqueue(h, c, reinterpret_cast<hipStream_t>(stream));
}

edit_status_t edit_ortho_local_step(edit_ortho_t h, void* param, const void* grad, float* momentum, double lr, double mu,
                                    double weight_decay, int32_t nesterov, void* stream) {
  if (!h) return ofail(EDIT_EINVAL, "NULL handle");
  if (!(mu >= 0.0 && mu < 1.0)) return ofail(EDIT_EINVAL, "mu must be in [0, 1)");
  if (!(lr >= 0.0) || !std::isfinite(lr)) return ofail(EDIT_EINVAL, "lr must be finite and >= 0");
  if (!(weight_decay >= 0.0) || !std::isfinite(weight_decay))
    return ofail(EDIT_EINVAL, "weight_decay must be finite and >= 0");
  ORTHO_TRY(check_ortho_device(h));
  if (h->matrix_chunks == 0) return EDIT_OK;
  ORTHO_TRY(check_buffer(param, "param"));
  ORTHO_TRY(check_buffer(grad, "grad"));
  ORTHO_TRY(check_buffer(momentum, "momentum"));
  const int64_t bytes = h->numel * (h->bf16 ? 2 : 4);
  if (buffers_overlap(param, bytes, grad, bytes) || buffers_overlap(param, bytes, momentum, 4 * h->numel) ||
      buffers_overlap(grad, bytes, momentum, 4 * h->numel))
    return ofail(EDIT_EINVAL, "param, grad and momentum must not overlap");
  OrthoCall c = {};
  c.source = kSourceLocal;
  c.bf16 = h->bf16;
  c.x = grad;
  c.out = param;
  c.momentum = momentum;
  c.nesterov = nesterov != 0;
  c.mu = mu;
  c.keep = 1.0 - lr * weight_decay;
  c.lr = lr;
  return enqueue(h, c, reinterpret_cast<hipStream_t>(stream));
}

void edit_ortho_destroy(edit_ortho_t h) {
  if (!h) return;
  int prev = -1;
  if (hipGetDevice(&prev) == hipSuccess && prev != h->device) (void)hipSetDevice(h->device);
  if (h->arena) {
    (void)hipDeviceSynchronize();
    (void)hipFree(h->arena);
  }
  if (prev >= 0 && prev != h->device) (void)hipSetDevice(prev);
  delete h;
}

}  // extern "C"
