// Host runtime of libedit_outer.so: the C ABI declared in include/edit_outer.h.
//
// A handle owns, per sync unit: the device record (EMA state + decision),
// the per-block Gram partials, a completion event and (when profiling) four
// timing events.  A step validates its arguments, enqueues Gram pass ->
// decision -> update pass on the caller's stream and returns.  A round does
// that for batches of consecutive units; with EDIT_ONE_PASS it enqueues one
// fused pass per unit and one record launch at the end.  The host-state round adds a staging ring
// and two copy streams.  There is no host synchronisation on the step path
// and, apart from the host-state round's copies, no host-device traffic.
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <new>
#include <string>
#include <vector>

#include "disjoint_ranges.h"
#include "edit_outer_internal.h"
#include "edit_group_internal.h"
#include "edit_ortho_internal.h"

#define EDIT_TRY(expr)                    \
  do {                                    \
    const edit_status_t st_ = (expr);     \
    if (st_ != EDIT_OK) return st_;       \
  } while (0)

using namespace edit;

namespace {

thread_local std::string g_last_error;

edit_status_t fail(edit_status_t s, const std::string& msg) {
  // The runtime keeps a call's error until somebody asks for it; a later launch
  // that asks for its own (here or in the caller's program) would take it for that.
  if (s == EDIT_EHIP || s == EDIT_ENOMEM) (void)hipGetLastError();
  g_last_error = msg;
  return s;
}

edit_status_t fail_hip(hipError_t e, const char* what) {
  return fail(EDIT_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

struct Unit {
  int64_t n = 0;
  int rows = 1;         // Gram-pass blocks = partial rows (one-pass mode: fused blocks)
  int blocks2 = 1;      // update-pass blocks
  int slice = 1;        // one-pass mode: rows per slice of the fold launch (1: none)
  double* partials = nullptr;
  double* sums = nullptr;  // one-pass mode: slice sums of a sliced unit
  UnitRecord* rec = nullptr;
  hipEvent_t done = nullptr;
  hipEvent_t prof[4] = {nullptr, nullptr, nullptr, nullptr};
  bool pending = false;   // a completion to wait for has been recorded
  int done_slot = -1;     // -1: `done` (a single step); else the round-event slot
  uint64_t done_gen = 0;  // generation of that slot's record the unit belongs to
  bool profiled = false;  // prof[] hold the last step's timestamps
  bool has_state = false; // stepped or state_set at least once
};

}  // namespace

namespace {

// Staging of theta and momentum for rounds whose master copies live in host
// memory: a ring of device slots, one stream per copy direction, and per
// slot the events that order copy-in -> compute -> copy-out -> reuse.
constexpr int kOffloadSlots = 3;

struct Offload {
  int64_t cap = 0;           // elements per slot (theta and b each)
  float* buf = nullptr;      // [kOffloadSlots][2][cap] fp32
  hipStream_t h2d = nullptr, d2h = nullptr;
  hipEvent_t in_done[kOffloadSlots] = {};
  hipEvent_t comp_done[kOffloadSlots] = {};
  hipEvent_t out_done[kOffloadSlots] = {};
  hipEvent_t start = nullptr;  // the caller's stream at the start of a round
  bool used[kOffloadSlots] = {};
  bool ready = false;
};

}  // namespace

// Device scratch of edit_outer_step_layer_noalloc: the per-block Gram partials
// of one step, in a fixed array that each GPU holds for the life of the
// process (no allocation per call).  Host code never names the array itself
// (on the host `scratch` is only a stand-in for the symbol): its device
// address comes from hipGetSymbolAddress, taken once per device at the first
// edit_outer_init on that device, with that device current.
constexpr size_t kNoAllocScratchBytes = size_t(1) << 20;  // EDIT_NOALLOC_SCRATCH_BYTES
static_assert(kNoAllocScratchBytes == EDIT_NOALLOC_SCRATCH_BYTES, "header and library disagree");
static __device__ __align__(256) double scratch[kNoAllocScratchBytes / sizeof(double)];

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mutex;
void* g_scratch_ptr[kMaxDevices] = {};  // device address of `scratch` on each device

// The device address of the scratch array on `device` (current), looked up
// on first use.
edit_status_t noalloc_scratch(int device, void** out) {
  if (device < 0 || device >= kMaxDevices)
    return fail(EDIT_EINVAL, "device index " + std::to_string(device) + " beyond the scratch table");
  std::lock_guard<std::mutex> lock(g_scratch_mutex);
  if (!g_scratch_ptr[device]) {
    void* ptr = nullptr;
    const hipError_t e = hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch));
    if (e != hipSuccess || !ptr) return fail_hip(e, "hipGetSymbolAddress(scratch)");
    g_scratch_ptr[device] = ptr;
  }
  *out = g_scratch_ptr[device];
  return EDIT_OK;
}

}  // namespace

struct edit_outer {
  edit_outer_config_t cfg{};
  std::vector<int64_t> numel;
  int device = 0;
  int num_cu = 0;
  int pass2_lds = 0;       // dynamic LDS per update-pass block (occupancy cap)
  int fused_lds = 0;       // the same for the one-pass kernel
  int32_t profile_every = 0;  // record kernel events on units l with l % every == 0
  char* arena = nullptr;   // one device allocation for every unit's scratch
  void* noalloc = nullptr; // this device's fixed scratch array (step_layer_noalloc)
  bool one_pass = false;
  Offload off;
  std::vector<Unit> units;
  // Completion of a round: one event recorded after its last kernel, shared
  // by its units (an event record costs a few microseconds of stream time,
  // one per unit would cost ~1% of a 1B round).  A ring of slots; before a
  // slot is recorded again the host waits for its previous record, so every
  // generation up to round_complete[slot] is known to have finished.
  static constexpr int kRoundEvents = 4;
  hipEvent_t round_ev[kRoundEvents] = {};
  uint64_t round_gen[kRoundEvents] = {};       // generation of the slot's latest record
  uint64_t round_complete[kRoundEvents] = {};  // generations <= this have finished
  uint64_t next_gen = 1;
  int next_slot = 0;
};

namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Rows per slice of a one-pass unit's fold launch (1: one block sums them
// all).  Up to 1 MiB of partials one block takes less time than the extra
// launch saves (28.3M elements: 0.7 MB at K = 2 281 us a round of two without
// and 286 with it, 2.0 MB at K = 8 1,003 and 981 a round of four).
int32_t fold_slice(int32_t rows, int K) {
  const int64_t doubles = static_cast<int64_t>(rows) * (K + 1);
  return doubles > 131072 ? static_cast<int32_t>(ceil_div(rows, kFoldSlices)) : 1;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

edit_status_t check_device(const edit_outer* h) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail_hip(e, "hipGetDevice");
  if (dev != h->device)
    return fail(EDIT_EINVAL, "call made with device " + std::to_string(dev) +
                                 " current; the handle belongs to device " +
                                 std::to_string(h->device));
  return EDIT_OK;
}

void destroy_offload(edit_outer* h) {
  Offload& o = h->off;
  if (o.h2d) (void)hipStreamSynchronize(o.h2d);
  if (o.d2h) (void)hipStreamSynchronize(o.d2h);
  for (int s = 0; s < kOffloadSlots; ++s) {
    if (o.in_done[s]) (void)hipEventDestroy(o.in_done[s]);
    if (o.comp_done[s]) (void)hipEventDestroy(o.comp_done[s]);
    if (o.out_done[s]) (void)hipEventDestroy(o.out_done[s]);
  }
  if (o.start) (void)hipEventDestroy(o.start);
  if (o.h2d) (void)hipStreamDestroy(o.h2d);
  if (o.d2h) (void)hipStreamDestroy(o.d2h);
  if (o.buf) (void)hipFree(o.buf);
  o = Offload{};
}

void destroy_units(edit_outer* h) {
  destroy_offload(h);
  for (hipEvent_t& ev : h->round_ev)
    if (ev) {
      (void)hipEventDestroy(ev);
      ev = nullptr;
    }
  for (Unit& u : h->units) {
    if (u.done) (void)hipEventDestroy(u.done);
    for (hipEvent_t& ev : u.prof)
      if (ev) (void)hipEventDestroy(ev);
  }
  h->units.clear();
  if (h->arena) (void)hipFree(h->arena);
  h->arena = nullptr;
}

}  // namespace

namespace edit {

edit_status_t set_error(edit_status_t s, const char* msg) { return fail(s, msg); }

edit_status_t validate_config(const edit_outer_config_t* cfg) {
  const int K = cfg->num_workers;
  if (K < 1 || K > EDIT_MAX_K)
    return fail(EDIT_EINVAL, "num_workers must be in 1.." + std::to_string(EDIT_MAX_K));
  if (cfg->num_layers < 1) return fail(EDIT_EINVAL, "num_layers must be >= 1");
  if (!cfg->layer_numel) return fail(EDIT_EINVAL, "layer_numel must not be NULL");
  if (cfg->replica_dtype != EDIT_F32 && cfg->replica_dtype != EDIT_BF16)
    return fail(EDIT_EINVAL, "replica_dtype must be EDIT_F32 or EDIT_BF16");
  if (cfg->flags & ~(EDIT_AE | EDIT_WA | EDIT_GC | EDIT_ONE_PASS))
    return fail(EDIT_EINVAL, "unknown flag bits");
  if ((cfg->flags & EDIT_ONE_PASS) && (cfg->flags & (EDIT_AE | EDIT_WA | EDIT_GC)))
    return fail(EDIT_EINVAL, "flag EDIT_ONE_PASS needs EDIT_AE, EDIT_WA and EDIT_GC clear");
  if (!(cfg->ema_alpha > 0.0 && cfg->ema_alpha <= 1.0))
    return fail(EDIT_EINVAL, "ema_alpha must be in (0, 1]");
  if (!(cfg->clip_eps > 0.0)) return fail(EDIT_EINVAL, "clip_eps must be > 0");
  if (!(cfg->clip_threshold >= 0.0)) return fail(EDIT_EINVAL, "clip_threshold must be >= 0");
  if (!std::isfinite(cfg->outer_lr) || !std::isfinite(cfg->momentum) ||
      !std::isfinite(cfg->z_threshold))
    return fail(EDIT_EINVAL, "outer_lr, momentum and z_threshold must be finite");
  if (cfg->ema_warmup_rounds < 0) return fail(EDIT_EINVAL, "ema_warmup_rounds must be >= 0");
  if (cfg->flags & EDIT_AE) {
    const int64_t w_min = edit_outer_min_warmup(cfg->ema_alpha, cfg->z_threshold);
    if (w_min < 0)
      return fail(EDIT_EINVAL, "z_threshold must be > 0 with EDIT_AE: no EMA warm-up lets a worker "
                               "with a steady norm pass the z-test");
    if (cfg->ema_warmup_rounds < w_min) {
      char msg[200];
      std::snprintf(msg, sizeof msg,
                    "ema_warmup_rounds must be >= %lld for ema_alpha = %g and z_threshold = %g: a "
                    "shorter warm-up flags every worker with a steady norm for good",
                    static_cast<long long>(w_min), cfg->ema_alpha, cfg->z_threshold);
      return fail(EDIT_EINVAL, msg);
    }
  }
  for (int l = 0; l < cfg->num_layers; ++l)
    if (cfg->layer_numel[l] < 0)
      return fail(EDIT_EINVAL, "layer_numel[" + std::to_string(l) + "] is negative");
  return EDIT_OK;
}

edit_status_t current_gfx950(int* device, int* num_cu) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail_hip(e, "hipGetDevice");
  hipDeviceProp_t prop;
  e = hipGetDeviceProperties(&prop, dev);
  if (e != hipSuccess) return fail_hip(e, "hipGetDeviceProperties");
  if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0)
    return fail(EDIT_ENODEV, std::string("device arch is ") + prop.gcnArchName +
                                 "; this library is built for gfx950 only");
  *device = dev;
  *num_cu = prop.multiProcessorCount;
  return EDIT_OK;
}

}  // namespace edit

extern "C" {

// The z-test of Eq. 1 against the EMA state after k updates by a norm that
// stays G every round, from the zero state: mu_k = G(1 - (1-alpha)^k) lags
// G, so a clean worker passes only once k is large enough.  The recurrence
// is homogeneous in G, so G = 1 stands for every G > 0.
int64_t edit_outer_min_warmup(double alpha, double delta) {
  if (!(alpha > 0.0 && alpha <= 1.0) || !std::isfinite(delta)) return -1;
  constexpr int64_t kSearch = 1 << 20;  // z falls like (1-alpha)^(k/2): far beyond any alpha in use
  const double G = 1.0;
  double mu = 0.0, sigma = 0.0;
  for (int64_t k = 0; k <= kSearch; ++k) {
    if (!((G - mu) > delta * sigma)) return k;
    const double m = alpha * G + (1.0 - alpha) * mu;
    const double dev = G - m;
    sigma = std::sqrt((1.0 - alpha) * sigma * sigma + alpha * dev * dev);
    mu = m;
  }
  return -1;
}

const char* edit_outer_strerror(edit_status_t s) {
  switch (s) {
    case EDIT_OK: return "ok";
    case EDIT_EINVAL: return "invalid argument";
    case EDIT_ENOMEM: return "out of memory";
    case EDIT_EHIP: return "HIP runtime error";
    case EDIT_ESTATE: return "invalid state";
    case EDIT_ENODEV: return "no gfx950 device";
  }
  return "unknown status";
}

const char* edit_outer_last_error(void) { return g_last_error.c_str(); }

edit_status_t edit_outer_init(const edit_outer_config_t* cfg, edit_outer_t* out) {
  g_last_error.clear();
  if (!cfg || !out) return fail(EDIT_EINVAL, "cfg and out must not be NULL");
  *out = nullptr;
  const int K = cfg->num_workers;
  EDIT_TRY(validate_config(cfg));
  int dev = 0, num_cu = 0;
  EDIT_TRY(current_gfx950(&dev, &num_cu));
  void* noalloc = nullptr;
  EDIT_TRY(noalloc_scratch(dev, &noalloc));
  hipError_t e = hipSuccess;

  edit_outer* h = new (std::nothrow) edit_outer;
  if (!h) return fail(EDIT_ENOMEM, "host allocation failed");
  h->cfg = *cfg;
  h->numel.assign(cfg->layer_numel, cfg->layer_numel + cfg->num_layers);
  h->cfg.layer_numel = h->numel.data();
  h->device = dev;
  h->num_cu = num_cu;
  {
    int lds_per_cu = 0;
    e = hipDeviceGetAttribute(&lds_per_cu, hipDeviceAttributeMaxSharedMemoryPerMultiprocessor, dev);
    if (e != hipSuccess) {
      delete h;
      return fail_hip(e, "hipDeviceGetAttribute(LDS per CU)");
    }
    h->pass2_lds = update_pass_lds(K, cfg->replica_dtype == EDIT_BF16, lds_per_cu);
    h->fused_lds = one_pass_lds(K, cfg->replica_dtype == EDIT_BF16, lds_per_cu);
  }
  h->noalloc = noalloc;
  const bool bf16 = cfg->replica_dtype == EDIT_BF16;
  h->one_pass = (cfg->flags & EDIT_ONE_PASS) != 0;

  // Lay out every unit's record and partials in one allocation.
  const int ve = bf16 ? 8 : 4;
  const size_t rec_bytes = (sizeof(UnitRecord) + 255) & ~size_t(255);
  size_t total = 0;
  h->units.resize(cfg->num_layers);
  std::vector<size_t> offs(cfg->num_layers), sums_offs(cfg->num_layers);
  for (int l = 0; l < cfg->num_layers; ++l) {
    Unit& u = h->units[l];
    u.n = h->numel[l];
    const int64_t nvec = u.n / ve;
    // one partial row per CU (fewer for small units), whatever launch the
    // unit shares, so that a round and step_layer reduce in the same order
    u.rows = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(h->num_cu, ceil_div(nvec, kRowVectors))));
    // the update pass (and the one-pass kernel): a fixed number of vectors per thread,
    // so the block count grows with the unit
    if (ceil_div(nvec, kUpdateThreads) > INT32_MAX) {
      delete h;
      return fail(EDIT_EINVAL, "layer_numel[" + std::to_string(l) + "] is too large");
    }
    u.blocks2 = static_cast<int>(std::max<int64_t>(1, ceil_div(nvec, kUpdateThreads)));
    if (h->one_pass)
      u.rows = static_cast<int>(std::max<int64_t>(
          1, ceil_div(nvec, int64_t(kFusedThreads) * fused_vectors_per_thread(K, bf16))));
    offs[l] = total;
    const size_t per_row = h->one_pass ? size_t(K + 1) : size_t(num_pairs(K));
    const size_t part_bytes = (per_row * u.rows * sizeof(double) + 255) & ~size_t(255);
    total += rec_bytes + part_bytes;
    if (h->one_pass) u.slice = fold_slice(u.rows, K);
    if (u.slice > 1) {
      sums_offs[l] = total;
      total += (per_row * kFoldSlices * sizeof(double) + 255) & ~size_t(255);
    }
  }
  e = hipMalloc(reinterpret_cast<void**>(&h->arena), total);
  if (e != hipSuccess) {
    delete h;
    return fail(EDIT_ENOMEM, std::string("hipMalloc of scratch: ") + hipGetErrorString(e));
  }
  e = hipMemset(h->arena, 0, total);  // EMA state mu = sigma = 0, round 0
  for (int l = 0; l < cfg->num_layers && e == hipSuccess; ++l) {
    Unit& u = h->units[l];
    u.rec = reinterpret_cast<UnitRecord*>(h->arena + offs[l]);
    u.partials = reinterpret_cast<double*>(h->arena + offs[l] + rec_bytes);
    if (u.slice > 1) u.sums = reinterpret_cast<double*>(h->arena + sums_offs[l]);
    e = hipEventCreateWithFlags(&u.done, hipEventDisableTiming);
  }
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    destroy_units(h);
    delete h;
    return fail_hip(e, "init");
  }
  *out = h;
  return EDIT_OK;
}

}  // extern "C"

namespace {

// Argument checks shared by the step entry points.  `momentum` may be NULL
// only when `need_momentum` is false (the Gram pass does not touch it).
// `extra`, when not NULL, is one more buffer of `extra_bytes` (a Gram vector)
// that must not overlap the others.
edit_status_t check_step(const edit_outer* h, int32_t layer, const float* theta,
                         const float* momentum, void* const* replicas,
                         bool need_momentum = true, const void* extra = nullptr,
                         int64_t extra_bytes = 0) {
  if (layer < 0 || layer >= h->cfg.num_layers)
    return fail(EDIT_EINVAL, "layer " + std::to_string(layer) + " out of range");
  const Unit& u = h->units[layer];
  const int K = h->cfg.num_workers;
  const int64_t n = u.n;
  if (n == 0) return EDIT_OK;
  if (!replicas) return fail(EDIT_EINVAL, "replicas must not be NULL");
  if (!theta || (need_momentum && !momentum))
    return fail(EDIT_EINVAL, "theta and momentum must not be NULL");
  if (!aligned16(theta) || (momentum && !aligned16(momentum)))
    return fail(EDIT_EINVAL, "theta and momentum must be 16-byte aligned");
  // Every buffer's byte range, for the alias check.
  struct Range {
    uintptr_t lo, hi;
  };
  Range r[EDIT_MAX_K + 3];
  int nr = 0;
  r[nr++] = {reinterpret_cast<uintptr_t>(theta), reinterpret_cast<uintptr_t>(theta) + 4 * n};
  if (momentum)
    r[nr++] = {reinterpret_cast<uintptr_t>(momentum), reinterpret_cast<uintptr_t>(momentum) + 4 * n};
  if (extra)
    r[nr++] = {reinterpret_cast<uintptr_t>(extra), reinterpret_cast<uintptr_t>(extra) + extra_bytes};
  const int64_t rb = h->cfg.replica_dtype == EDIT_BF16 ? 2 : 4;
  for (int j = 0; j < K; ++j) {
    if (!replicas[j]) return fail(EDIT_EINVAL, "replica pointer " + std::to_string(j) + " is NULL");
    if (!aligned16(replicas[j]))
      return fail(EDIT_EINVAL, "replica " + std::to_string(j) + " is not 16-byte aligned");
    const uintptr_t p = reinterpret_cast<uintptr_t>(replicas[j]);
    r[nr++] = {p, p + rb * n};
  }
  for (int a = 0; a < nr; ++a)
    for (int b = a + 1; b < nr; ++b)
      if (r[a].lo < r[b].hi && r[b].lo < r[a].hi)
        return fail(EDIT_EINVAL, extra ? "theta, momentum, the replicas and gram must not overlap"
                                       : "theta, momentum and the replicas must not overlap");
  return EDIT_OK;
}

// A Gram vector argument: non-NULL and 8-byte aligned.
edit_status_t check_gram(const void* gram) {
  if (!gram) return fail(EDIT_EINVAL, "gram must not be NULL");
  if (reinterpret_cast<uintptr_t>(gram) & 7u) return fail(EDIT_EINVAL, "gram must be 8-byte aligned");
  return EDIT_OK;
}

DecideParams decide_params(const edit_outer* h) {
  DecideParams prm;
  prm.alpha = h->cfg.ema_alpha;
  prm.delta = h->cfg.z_threshold;
  prm.phi = h->cfg.clip_threshold;
  prm.eps = h->cfg.clip_eps;
  prm.warmup = h->cfg.ema_warmup_rounds;
  prm.flags = h->cfg.flags;
  return prm;
}

// A round's batch ends before its Gram pass would read more than this: past
// it another unit in the batch saves nothing (rounds of six 1B units, 1.03 GB
// each: 3,394 us at one unit per batch and at four, 3,411 at six).
constexpr int64_t kBatchBytes = int64_t(4) << 30;
// From 9 to 16 workers a unit that reads more than this takes a batch of its
// own.  That Gram pass reads all of its input through the cache, and the
// update pass finds the end of it there; a larger batch loses that for all
// its units but the last.  Rounds of four units, us at one and at four per
// batch: bf16 of 128 MB each 359 and 336 (K = 16), 338 and 323 (K = 12); of
// 256 MB 633 and 633, 613 and 610, K = 9 706 and 717; of 448 MB 1,073 and
// 1,082, 1,016 and 1,040, K = 9 1,202 and 1,219.  fp32 at K = 16 of 448 MB 962
// and 960, of 1 GB 2,169 and 2,186.  Above K = 16 the decision costs more than
// that: K = 24 bf16 of 448 MB 1,225 and 1,208, K = 32 of 1 GB 2,992 and 2,943.
constexpr int64_t kAloneBytesBf16 = int64_t(240) << 20;
constexpr int64_t kAloneBytesF32 = int64_t(768) << 20;
// The end of a step's Gram input that is read through the cache (VALU pass),
// for the update pass to find in the 256 MB Infinity Cache, which also takes
// that pass's stores.  Six 1B bf16 units: 3,412 us with none, 3,405 at 120
// MB, 3,394 at 200 MB; six 350M fp32 units: 1,431, 1,417 and 1,428; 9 of
// 1.05M elements (K = 4 fp32): 132, 131 and 129.
constexpr int64_t kCachedBytes = int64_t(160) << 20;

static void* const kNoReplicas[EDIT_MAX_K] = {};

// Enqueue helpers; each returns EDIT_OK or the failure (message already set).
struct Enqueue {
  edit_outer* h;
  hipStream_t s;
  DecideParams prm;
  int K;
  bool bf16;

  bool profiled(int32_t layer) const {
    return h->profile_every > 0 && layer % h->profile_every == 0;
  }
  edit_status_t event(Unit& u, int32_t layer, int k) {
    if (!profiled(layer)) return EDIT_OK;
    hipError_t e = hipSuccess;
    // timing only: no system-scope fence (it would add stream time)
    if (!u.prof[k] && (e = hipEventCreateWithFlags(&u.prof[k], hipEventDisableSystemFence)) != hipSuccess)
      return fail_hip(e, "hipEventCreate");
    if ((e = hipEventRecord(u.prof[k], s)) != hipSuccess) return fail_hip(e, "hipEventRecord");
    return EDIT_OK;
  }
  // bytes of theta and the replicas per element, which the Gram pass reads
  int64_t element_bytes() const { return 4 + (bf16 ? 2 : 4) * static_cast<int64_t>(K); }
  // What a unit takes of a batch's kBatchBytes.
  int64_t batch_bytes(int32_t layer) const {
    const int64_t b = h->units[layer].n * element_bytes();
    const bool alone = K > 8 && K <= 16 && b > (bf16 ? kAloneBytesBf16 : kAloneBytesF32);
    return alone ? std::max(b, kBatchBytes) : b;
  }
  UnitDesc desc(int32_t layer, const float* theta, float* momentum, void* const* replicas) const {
    const Unit& u = h->units[layer];
    UnitDesc d;
    d.theta = const_cast<float*>(theta);  // the Gram pass only reads it
    d.mom = momentum;
    d.reps = u.n == 0 ? kNoReplicas : replicas;
    d.n = u.n;
    d.cut = u.n;
    d.partials = u.partials;
    d.rec = u.rec;
    d.rows = u.rows;
    d.update_blocks = u.blocks2;
    return d;
  }
  // The units' last kCachedBytes of Gram input go through the cache, where the
  // update pass that follows finds them.
  void cache_end(UnitDesc* d, int count) const {
    int64_t left = kCachedBytes / element_bytes();
    for (int i = count - 1; i >= 0; --i) {
      const int64_t cached = std::min(left, d[i].n);
      d[i].cut = d[i].n - cached;
      left -= cached;
    }
  }
  edit_status_t gram(const UnitDesc* d, int count) {
    hipError_t e = launch_gram(K, bf16, d, count, h->num_cu, s);
    return e == hipSuccess ? EDIT_OK : fail_hip(e, "Gram pass launch");
  }
  edit_status_t decide(const UnitDesc* d, int count) {
    hipError_t e = launch_decide(K, d, count, prm, s);
    return e == hipSuccess ? EDIT_OK : fail_hip(e, "decide launch");
  }
  edit_status_t update(const UnitDesc* d, int count) {
    hipError_t e = launch_update(K, bf16, d, count, h->pass2_lds, h->cfg.outer_lr, h->cfg.momentum, s);
    return e == hipSuccess ? EDIT_OK : fail_hip(e, "update pass launch");
  }
  // the whole step of a batch: units of one partial row by a block each, any
  // other batch in three launches
  edit_status_t step(const UnitDesc* d, int count) {
    if (std::all_of(d, d + count, [](const UnitDesc& u) { return u.rows == 1; })) {
      hipError_t e = launch_small_step(K, bf16, d, count, prm, h->cfg.outer_lr, h->cfg.momentum, s);
      return e == hipSuccess ? EDIT_OK : fail_hip(e, "small step launch");
    }
    EDIT_TRY(gram(d, count));
    EDIT_TRY(decide(d, count));
    return update(d, count);
  }
  // the step of one unit, timed when `layer` is
  edit_status_t step_unit(int32_t layer, UnitDesc d) {
    cache_end(&d, 1);
    if (!profiled(layer)) return step(&d, 1);
    Unit& u = h->units[layer];
    EDIT_TRY(event(u, layer, 0));
    EDIT_TRY(gram(&d, 1));
    EDIT_TRY(decide(&d, 1));
    EDIT_TRY(event(u, layer, 1));
    EDIT_TRY(event(u, layer, 2));
    EDIT_TRY(update(&d, 1));
    return event(u, layer, 3);
  }
  edit_status_t gram_out(int32_t layer, double* gram) {
    Unit& u = h->units[layer];
    hipError_t e = launch_gram_reduce(K, u.partials, u.rows, gram, s);
    return e == hipSuccess ? EDIT_OK : fail_hip(e, "gram reduce launch");
  }
  edit_status_t decide_from(int32_t layer, const double* gram) {
    Unit& u = h->units[layer];
    hipError_t e = launch_decide_gram(K, gram, u.rec, prm, s);
    return e == hipSuccess ? EDIT_OK : fail_hip(e, "decide launch");
  }
  // one-pass mode: the fused pass of `layer`, and the record reductions of
  // the units stepped
  edit_status_t fused(int32_t layer, float* theta, float* momentum, void* const* replicas) {
    Unit& u = h->units[layer];
    void* const* mreps = u.n == 0 ? kNoReplicas : replicas;
    hipError_t e = launch_fused_mean(K, bf16, u.rows, h->fused_lds, theta, momentum, mreps, u.partials, u.n,
                                     h->cfg.outer_lr, h->cfg.momentum, s);
    return e == hipSuccess ? EDIT_OK : fail_hip(e, "one-pass launch");
  }
  edit_status_t records(const int32_t* layers, int32_t count) {
    for (int32_t at = 0; at < count; at += kMaxFinishUnits) {
      const int units = std::min<int32_t>(count - at, kMaxFinishUnits);
      FinishDesc d[kMaxFinishUnits];
      int sliced = 0, rest = units;  // sliced units from the front, others from the back
      for (int i = 0; i < units; ++i) {
        const Unit& u = h->units[layers[at + i]];
        d[u.slice > 1 ? sliced++ : --rest] = {u.partials, u.sums, u.rec, u.rows, u.slice};
      }
      hipError_t e = launch_fused_finish(K, d, units, sliced, s);
      if (e != hipSuccess) return fail_hip(e, "record launch");
    }
    return EDIT_OK;
  }
  edit_status_t finish(int32_t layer) {
    Unit& u = h->units[layer];
    hipError_t e = hipEventRecord(u.done, s);
    if (e != hipSuccess) return fail_hip(e, "hipEventRecord");
    u.pending = true;
    u.done_slot = -1;
    u.profiled = profiled(layer);
    u.has_state = true;
    return EDIT_OK;
  }
  // The end of a round: one event for all of its units.
  edit_status_t finish_round(const int32_t* layers, int32_t count) {
    const int slot = h->next_slot;
    h->next_slot = (slot + 1) % edit_outer::kRoundEvents;
    hipError_t e = hipSuccess;
    if (!h->round_ev[slot] && (e = hipEventCreateWithFlags(&h->round_ev[slot], hipEventDisableTiming)) != hipSuccess)
      return fail_hip(e, "hipEventCreate");
    if (h->round_gen[slot] > h->round_complete[slot]) {  // its previous round may still run
      if ((e = hipEventSynchronize(h->round_ev[slot])) != hipSuccess) return fail_hip(e, "hipEventSynchronize");
      h->round_complete[slot] = h->round_gen[slot];
    }
    if ((e = hipEventRecord(h->round_ev[slot], s)) != hipSuccess) return fail_hip(e, "hipEventRecord");
    const uint64_t gen = h->next_gen++;
    h->round_gen[slot] = gen;
    for (int32_t i = 0; i < count; ++i) {
      Unit& u = h->units[layers[i]];
      u.pending = true;
      u.done_slot = slot;
      u.done_gen = gen;
      u.profiled = profiled(layers[i]);
      u.has_state = true;
    }
    return EDIT_OK;
  }
};

// Wait until the last enqueued step of `u` has finished.
edit_status_t wait_unit(edit_outer* h, Unit& u) {
  if (!u.pending) return EDIT_OK;
  hipError_t e = hipSuccess;
  if (u.done_slot < 0) {
    e = hipEventSynchronize(u.done);
  } else {
    const int slot = u.done_slot;
    if (h->round_complete[slot] >= u.done_gen) return EDIT_OK;
    // not recorded again since (that would have completed this generation)
    e = hipEventSynchronize(h->round_ev[slot]);
    if (e == hipSuccess) h->round_complete[slot] = h->round_gen[slot];
  }
  return e == hipSuccess ? EDIT_OK : fail_hip(e, "hipEventSynchronize");
}


}  // namespace

extern "C" {

edit_status_t edit_outer_step_layer(edit_outer_t h, int32_t layer, float* theta, float* momentum,
                                    void* const* replicas, void* stream) {
  if (!h) return fail(EDIT_EINVAL, "NULL handle");
  EDIT_TRY(check_step(h, layer, theta, momentum, replicas));
  EDIT_TRY(check_device(h));
  Enqueue q{h, reinterpret_cast<hipStream_t>(stream), decide_params(h), h->cfg.num_workers,
            h->cfg.replica_dtype == EDIT_BF16};
  if (h->one_pass) {
    EDIT_TRY(q.event(h->units[layer], layer, 0));
    EDIT_TRY(q.fused(layer, theta, momentum, replicas));
    EDIT_TRY(q.event(h->units[layer], layer, 1));
    EDIT_TRY(q.event(h->units[layer], layer, 2));
    EDIT_TRY(q.records(&layer, 1));
    EDIT_TRY(q.event(h->units[layer], layer, 3));
    return q.finish(layer);
  }
  EDIT_TRY(q.step_unit(layer, q.desc(layer, theta, momentum, replicas)));
  return q.finish(layer);
}

edit_status_t edit_outer_step_layer_noalloc(edit_outer_t h, int32_t layer, float* theta, float* momentum,
                                            void* const* replicas, void* stream) {
  if (!h) return fail(EDIT_EINVAL, "NULL handle");
  if (h->one_pass) return fail(EDIT_EINVAL, "edit_outer_step_layer_noalloc is not available with EDIT_ONE_PASS");
  EDIT_TRY(check_step(h, layer, theta, momentum, replicas));
  const int K = h->cfg.num_workers;
  Unit& u = h->units[layer];
  const size_t need = static_cast<size_t>(num_pairs(K)) * static_cast<size_t>(u.rows) * sizeof(double);
  if (need > kNoAllocScratchBytes)
    return fail(EDIT_EINVAL, "unit " + std::to_string(layer) + " needs " + std::to_string(need) +
                                 " bytes of partial sums; the fixed scratch holds " +
                                 std::to_string(kNoAllocScratchBytes));
  EDIT_TRY(check_device(h));
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool bf16 = h->cfg.replica_dtype == EDIT_BF16;
  Enqueue q{h, s, decide_params(h), K, bf16};
  UnitDesc d = q.desc(layer, theta, momentum, replicas);
  d.partials = static_cast<double*>(h->noalloc);  // the device address, never `scratch` itself
  q.cache_end(&d, 1);
  EDIT_TRY(q.step(&d, 1));
  hipError_t e = hipSuccess;
  if ((e = hipEventRecord(u.done, s)) != hipSuccess) return fail_hip(e, "hipEventRecord");
  u.pending = true;
  u.done_slot = -1;
  u.profiled = false;
  u.has_state = true;
  return EDIT_OK;
}

edit_status_t edit_outer_gram_layer(edit_outer_t h, int32_t layer, const float* theta,
                                    void* const* replicas, double* gram, void* stream) {
  if (!h) return fail(EDIT_EINVAL, "NULL handle");
  if (h->one_pass) return fail(EDIT_EINVAL, "the Gram entry points are not available with EDIT_ONE_PASS");
  EDIT_TRY(check_gram(gram));
  const int K = h->cfg.num_workers;
  EDIT_TRY(check_step(h, layer, theta, nullptr, replicas, false, gram,
                      static_cast<int64_t>(num_pairs(K)) * 8));
  EDIT_TRY(check_device(h));
  Enqueue q{h, reinterpret_cast<hipStream_t>(stream), decide_params(h), K,
            h->cfg.replica_dtype == EDIT_BF16};
  const UnitDesc d = q.desc(layer, theta, nullptr, replicas);
  EDIT_TRY(q.gram(&d, 1));
  return q.gram_out(layer, gram);
}

edit_status_t edit_outer_apply_layer(edit_outer_t h, int32_t layer, const double* gram,
                                     float* theta, float* momentum, void* const* replicas,
                                     void* stream) {
  if (!h) return fail(EDIT_EINVAL, "NULL handle");
  if (h->one_pass) return fail(EDIT_EINVAL, "the Gram entry points are not available with EDIT_ONE_PASS");
  EDIT_TRY(check_gram(gram));
  const int K = h->cfg.num_workers;
  EDIT_TRY(check_step(h, layer, theta, momentum, replicas, true, gram,
                      static_cast<int64_t>(num_pairs(K)) * 8));
  EDIT_TRY(check_device(h));
  Enqueue q{h, reinterpret_cast<hipStream_t>(stream), decide_params(h), K,
            h->cfg.replica_dtype == EDIT_BF16};
  Unit& u = h->units[layer];
  const UnitDesc d = q.desc(layer, theta, momentum, replicas);
  EDIT_TRY(q.event(u, layer, 0));
  EDIT_TRY(q.decide_from(layer, gram));
  EDIT_TRY(q.event(u, layer, 1));
  EDIT_TRY(q.event(u, layer, 2));
  EDIT_TRY(q.update(&d, 1));
  EDIT_TRY(q.event(u, layer, 3));
  return q.finish(layer);
}

edit_status_t edit_outer_step_layer_ortho(edit_outer_t h, int32_t layer, edit_ortho_t ortho, float* theta,
                                          float* momentum, void* const* replicas, void* stream) {
  if (!h || !ortho) return fail(EDIT_EINVAL, "NULL handle");
  if (h->one_pass) return fail(EDIT_EINVAL, "edit_outer_step_layer_ortho is not available with EDIT_ONE_PASS");
  EDIT_TRY(check_step(h, layer, theta, momentum, replicas));
  EDIT_TRY(check_device(h));
  Unit& u = h->units[layer];
  EDIT_TRY(check_ortho_unit(ortho, u.n, h->device));
  const int K = h->cfg.num_workers;
  const bool bf16 = h->cfg.replica_dtype == EDIT_BF16;
  Enqueue q{h, reinterpret_cast<hipStream_t>(stream), decide_params(h), K, bf16};
  UnitDesc d = q.desc(layer, theta, momentum, replicas);
  q.cache_end(&d, 1);
  EDIT_TRY(q.event(u, layer, 0));
  EDIT_TRY(q.gram(&d, 1));
  EDIT_TRY(q.decide(&d, 1));
  EDIT_TRY(q.event(u, layer, 1));
  EDIT_TRY(q.event(u, layer, 2));
  EDIT_TRY(enqueue_ortho_outer(ortho, bf16, theta, momentum, replicas, K, u.rec, h->cfg.outer_lr, h->cfg.momentum,
                               q.s));
  EDIT_TRY(q.event(u, layer, 3));
  return q.finish(layer);
}

edit_status_t edit_outer_step_round(edit_outer_t h, int32_t count, const int32_t* layers,
                                    float* const* theta, float* const* momentum,
                                    void* const* replicas, void* stream) {
  if (!h) return fail(EDIT_EINVAL, "NULL handle");
  if (count < 1) return fail(EDIT_EINVAL, "count must be >= 1");
  if (!layers || !theta || !momentum || !replicas)
    return fail(EDIT_EINVAL, "layers, theta, momentum and replicas must not be NULL");
  const int K = h->cfg.num_workers;
  std::vector<char> seen(h->cfg.num_layers, 0);
  for (int32_t i = 0; i < count; ++i) {
    EDIT_TRY(check_step(h, layers[i], theta[i], momentum[i], replicas + static_cast<size_t>(i) * K));
    if (seen[layers[i]]++)
      return fail(EDIT_EINVAL, "layer " + std::to_string(layers[i]) + " appears twice in a round");
  }
  EDIT_TRY(check_device(h));
  Enqueue q{h, reinterpret_cast<hipStream_t>(stream), decide_params(h), K,
            h->cfg.replica_dtype == EDIT_BF16};
  if (h->one_pass) {
    // No later kernel of the round needs a unit's record, so the fused passes
    // run back to back and one launch then reduces every stepped unit's norms.
    for (int32_t i = 0; i < count; ++i) {
      const int32_t l = layers[i];
      EDIT_TRY(q.event(h->units[l], l, 0));
      EDIT_TRY(q.fused(l, theta[i], momentum[i], replicas + static_cast<size_t>(i) * K));
      EDIT_TRY(q.event(h->units[l], l, 1));
      EDIT_TRY(q.event(h->units[l], l, 2));
      EDIT_TRY(q.event(h->units[l], l, 3));
    }
    EDIT_TRY(q.records(layers, count));
    return q.finish_round(layers, count);
  }
  // Consecutive units go in batches of three launches: Gram pass, decisions,
  // update pass.  A launch's start and drain and the decision are then paid
  // once per batch, and the next batch's Gram pass does not come between a
  // batch's two passes.  Measured per round, one unit per batch against one
  // batch: nine 2.9M units (K = 4 fp32) 374 and 329 us, six 4.2M (K = 8
  // bf16) 364 and 293, six 12.8M fp32 (K = 8) 1,513 and 1,428.  Units of one
  // Gram block take no part in that: they are stepped whole, a block each,
  // in launches of their own.  In a batch with a large unit they would wait
  // for its passes (a 51.4M unit and two gains at K = 16: 1,100 us against
  // 1,050).  Units that wait for their launch share no buffer: a unit that
  // shares one with a waiting unit (a tied parameter listed twice) first sends
  // off all that wait, so that the units of a launch are independent and
  // shared buffers see the steps in the round's order.
  const int most = batch_units(K);
  UnitDesc batch[kMaxBatchUnits], small[kMaxBatchUnits];
  int in = 0, nsmall = 0;
  int64_t bytes = 0;  // what the batch's units take of kBatchBytes
  // at most 2 * 16 units of 18 buffers up to K = 16, 2 * 8 of 34 above
  DisjointRanges<kMaxBatchUnits * (EDIT_MAX_K + 4)> waiting;
  ByteRange r[EDIT_MAX_K + 2];
  auto ranges = [&](const UnitDesc& d) {  // the unit's buffers in r; their number
    if (d.n == 0) return 0;
    auto range = [&](const void* p, int64_t each) {
      const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
      return ByteRange{lo, lo + static_cast<uintptr_t>(d.n * each)};
    };
    r[0] = range(d.theta, 4);
    r[1] = range(d.mom, 4);
    for (int j = 0; j < K; ++j) r[2 + j] = range(d.reps[j], q.bf16 ? 2 : 4);
    return K + 2;
  };
  auto flush = [&]() -> edit_status_t {
    if (in == 0) return EDIT_OK;
    q.cache_end(batch, in);
    const int units = in;
    in = 0;
    bytes = 0;
    waiting.clear();
    for (int i = 0; i < nsmall; ++i) {
      const int nr = ranges(small[i]);
      waiting.add(r, nr);
    }
    return q.step(batch, units);
  };
  auto flush_small = [&]() -> edit_status_t {
    if (nsmall == 0) return EDIT_OK;
    const int units = nsmall;
    nsmall = 0;
    waiting.clear();
    for (int i = 0; i < in; ++i) {
      const int nr = ranges(batch[i]);
      waiting.add(r, nr);
    }
    return q.step(small, units);
  };
  for (int32_t i = 0; i < count; ++i) {
    const int32_t l = layers[i];
    const UnitDesc d = q.desc(l, theta[i], momentum[i], replicas + static_cast<size_t>(i) * K);
    const bool alone = q.profiled(l);
    const bool whole = !alone && d.rows == 1;
    const int64_t b = q.batch_bytes(l);
    if (alone || (!whole && (in == most || (in > 0 && bytes + b > kBatchBytes)))) EDIT_TRY(flush());
    if (whole && nsmall == most) EDIT_TRY(flush_small());
    int nr = ranges(d);
    if (waiting.meets(r, nr)) {
      EDIT_TRY(flush());
      EDIT_TRY(flush_small());
      nr = ranges(d);  // the flushes used r
    }
    if (alone) {
      EDIT_TRY(q.step_unit(l, d));
      continue;
    }
    waiting.add(r, nr);
    if (whole) {
      small[nsmall++] = d;
    } else {
      batch[in++] = d;
      bytes += b;
    }
  }
  EDIT_TRY(flush());
  EDIT_TRY(flush_small());
  return q.finish_round(layers, count);
}

}  // extern "C"

namespace {

// Page-locked host memory (hipHostMalloc, or torch's pin_memory), which the
// copy engines can read and write asynchronously.
bool is_pinned_host(const void* p) {
  hipPointerAttribute_t attr;
  const hipError_t e = hipPointerGetAttributes(&attr, p);
  if (e != hipSuccess) {
    (void)hipGetLastError();  // an unregistered pointer is an answer, not a failure
    return false;
  }
  return attr.type == hipMemoryTypeHost;
}

edit_status_t offload_setup(edit_outer* h) {
  Offload& o = h->off;
  if (o.ready) return EDIT_OK;
  int64_t cap = 64;
  for (const Unit& u : h->units) cap = std::max(cap, u.n);
  cap = ceil_div(cap, 64) * 64;  // each half of a slot stays 256-byte aligned
  hipError_t e = hipMalloc(reinterpret_cast<void**>(&o.buf),
                           sizeof(float) * 2 * kOffloadSlots * static_cast<size_t>(cap));
  if (e != hipSuccess) {
    o.buf = nullptr;
    return fail(EDIT_ENOMEM, std::string("hipMalloc of the staging ring: ") + hipGetErrorString(e));
  }
  o.cap = cap;
  if ((e = hipStreamCreateWithFlags(&o.h2d, hipStreamNonBlocking)) != hipSuccess ||
      (e = hipStreamCreateWithFlags(&o.d2h, hipStreamNonBlocking)) != hipSuccess ||
      (e = hipEventCreateWithFlags(&o.start, hipEventDisableTiming)) != hipSuccess) {
    destroy_offload(h);
    return fail_hip(e, "offload streams");
  }
  for (int s = 0; s < kOffloadSlots; ++s)
    if ((e = hipEventCreateWithFlags(&o.in_done[s], hipEventDisableTiming)) != hipSuccess ||
        (e = hipEventCreateWithFlags(&o.comp_done[s], hipEventDisableTiming)) != hipSuccess ||
        (e = hipEventCreateWithFlags(&o.out_done[s], hipEventDisableTiming)) != hipSuccess) {
      destroy_offload(h);
      return fail_hip(e, "offload events");
    }
  o.ready = true;
  return EDIT_OK;
}

}  // namespace

extern "C" {

edit_status_t edit_outer_step_round_host(edit_outer_t h, int32_t count, const int32_t* layers,
                                         float* const* theta_host, float* const* momentum_host,
                                         void* const* replicas, void* stream) {
  if (!h) return fail(EDIT_EINVAL, "NULL handle");
  if (count < 1) return fail(EDIT_EINVAL, "count must be >= 1");
  if (!layers || !theta_host || !momentum_host || !replicas)
    return fail(EDIT_EINVAL, "layers, theta_host, momentum_host and replicas must not be NULL");
  EDIT_TRY(check_device(h));
  EDIT_TRY(offload_setup(h));
  Offload& o = h->off;
  const int K = h->cfg.num_workers;
  std::vector<char> seen(h->cfg.num_layers, 0);
  for (int32_t i = 0; i < count; ++i) {
    const int32_t l = layers[i];
    // the replicas are checked against a staging slot standing in for theta/b
    EDIT_TRY(check_step(h, l, o.buf, o.buf + o.cap, replicas + static_cast<size_t>(i) * K));
    if (seen[l]++) return fail(EDIT_EINVAL, "layer " + std::to_string(l) + " appears twice in a round");
    const int64_t n = h->units[l].n;
    if (n == 0) continue;
    const float* th = theta_host[i];
    const float* mo = momentum_host[i];
    if (!th || !mo) return fail(EDIT_EINVAL, "theta_host and momentum_host must not be NULL");
    if (!is_pinned_host(th) || !is_pinned_host(mo))
      return fail(EDIT_EINVAL, "theta_host and momentum_host of layer " + std::to_string(l) +
                                   " must be pinned host memory (hipHostMalloc)");
    const uintptr_t a = reinterpret_cast<uintptr_t>(th), b = reinterpret_cast<uintptr_t>(mo);
    if (a < b + 4 * n && b < a + 4 * n)
      return fail(EDIT_EINVAL, "theta_host and momentum_host overlap");
  }
  hipStream_t cs = reinterpret_cast<hipStream_t>(stream);
  Enqueue q{h, cs, decide_params(h), K, h->cfg.replica_dtype == EDIT_BF16};
  hipError_t e = hipEventRecord(o.start, cs);
  if (e == hipSuccess) e = hipStreamWaitEvent(o.h2d, o.start, 0);
  if (e != hipSuccess) return fail_hip(e, "round start");
  bool used_now[kOffloadSlots] = {};
  for (int32_t i = 0; i < count; ++i) {
    const int32_t l = layers[i];
    Unit& u = h->units[l];
    const int s = i % kOffloadSlots;
    float* dth = o.buf + static_cast<size_t>(s) * 2 * o.cap;
    float* db = dth + o.cap;
    void* const* reps = replicas + static_cast<size_t>(i) * K;
    const size_t bytes = sizeof(float) * static_cast<size_t>(u.n);
    // copy in, once the slot's previous unit has been copied out
    if (o.used[s] && (e = hipStreamWaitEvent(o.h2d, o.out_done[s], 0)) != hipSuccess)
      return fail_hip(e, "hipStreamWaitEvent");
    if (u.n > 0 &&
        ((e = hipMemcpyAsync(dth, theta_host[i], bytes, hipMemcpyHostToDevice, o.h2d)) != hipSuccess ||
         (e = hipMemcpyAsync(db, momentum_host[i], bytes, hipMemcpyHostToDevice, o.h2d)) != hipSuccess))
      return fail_hip(e, "copy to device");
    if ((e = hipEventRecord(o.in_done[s], o.h2d)) != hipSuccess ||
        (e = hipStreamWaitEvent(cs, o.in_done[s], 0)) != hipSuccess)
      return fail_hip(e, "copy-in event");
    // the step itself, on the caller's stream, from the staging slot
    if (h->one_pass) {
      EDIT_TRY(q.event(u, l, 0));
      EDIT_TRY(q.fused(l, dth, db, reps));
      EDIT_TRY(q.event(u, l, 1));
      EDIT_TRY(q.event(u, l, 2));
      EDIT_TRY(q.records(&l, 1));
      EDIT_TRY(q.event(u, l, 3));
    } else {
      EDIT_TRY(q.step_unit(l, q.desc(l, dth, db, reps)));
    }
    // copy out once the step is done
    if ((e = hipEventRecord(o.comp_done[s], cs)) != hipSuccess ||
        (e = hipStreamWaitEvent(o.d2h, o.comp_done[s], 0)) != hipSuccess)
      return fail_hip(e, "compute event");
    if (u.n > 0 &&
        ((e = hipMemcpyAsync(theta_host[i], dth, bytes, hipMemcpyDeviceToHost, o.d2h)) != hipSuccess ||
         (e = hipMemcpyAsync(momentum_host[i], db, bytes, hipMemcpyDeviceToHost, o.d2h)) != hipSuccess))
      return fail_hip(e, "copy to host");
    if ((e = hipEventRecord(o.out_done[s], o.d2h)) != hipSuccess) return fail_hip(e, "copy-out event");
    o.used[s] = true;
    used_now[s] = true;
  }
  // the caller's stream covers the copies back: synchronising it makes the
  // host arrays current
  for (int s = 0; s < kOffloadSlots; ++s)
    if (used_now[s] && (e = hipStreamWaitEvent(cs, o.out_done[s], 0)) != hipSuccess)
      return fail_hip(e, "round end");
  return q.finish_round(layers, count);
}

edit_status_t edit_outer_state_get(edit_outer_t h, int32_t layer, edit_layer_state_t* out) {
  if (!h || !out) return fail(EDIT_EINVAL, "NULL argument");
  if (layer < 0 || layer >= h->cfg.num_layers)
    return fail(EDIT_EINVAL, "layer " + std::to_string(layer) + " out of range");
  Unit& u = h->units[layer];
  if (!u.has_state) return fail(EDIT_ESTATE, "unit has neither stepped nor had its state set");
  edit_status_t st = check_device(h);
  if (st != EDIT_OK) return st;
  EDIT_TRY(wait_unit(h, u));
  hipError_t e = hipSuccess;
  UnitRecord rec;
  if ((e = hipMemcpy(&rec, u.rec, sizeof rec, hipMemcpyDeviceToHost)) != hipSuccess)
    return fail_hip(e, "hipMemcpy D2H");
  std::memset(out, 0, sizeof *out);
  const int K = h->cfg.num_workers;
  out->round = rec.round;
  out->num_workers = K;
  out->rolled_back = rec.rollback;
  out->z_tested = rec.z_tested;
  for (int j = 0; j < K; ++j) {
    out->ema_mean[j] = rec.mu[j];
    out->ema_std[j] = rec.sigma[j];
    out->norm[j] = rec.norm[j];
    out->weight[j] = rec.weight[j];
    out->anomalous[j] = rec.anomalous[j];
  }
  out->synced_norm = rec.synced_norm;
  out->clip_coef = rec.clip_coef;
  return EDIT_OK;
}

edit_status_t edit_outer_state_set(edit_outer_t h, int32_t layer, const edit_layer_state_t* in) {
  if (!h || !in) return fail(EDIT_EINVAL, "NULL argument");
  if (layer < 0 || layer >= h->cfg.num_layers)
    return fail(EDIT_EINVAL, "layer " + std::to_string(layer) + " out of range");
  if (in->round < 0) return fail(EDIT_EINVAL, "round must be >= 0");
  const int K = h->cfg.num_workers;
  for (int j = 0; j < K; ++j)
    if (!std::isfinite(in->ema_mean[j]) || !(in->ema_std[j] >= 0.0) || !std::isfinite(in->ema_std[j]))
      return fail(EDIT_EINVAL, "EMA state must be finite with ema_std >= 0");
  Unit& u = h->units[layer];
  edit_status_t st = check_device(h);
  if (st != EDIT_OK) return st;
  EDIT_TRY(wait_unit(h, u));
  hipError_t e = hipSuccess;
  UnitRecord rec;
  if ((e = hipMemcpy(&rec, u.rec, sizeof rec, hipMemcpyDeviceToHost)) != hipSuccess)
    return fail_hip(e, "hipMemcpy D2H");
  for (int j = 0; j < K; ++j) {
    rec.mu[j] = in->ema_mean[j];
    rec.sigma[j] = in->ema_std[j];
  }
  rec.round = in->round;
  rec.stepped = 1;
  if ((e = hipMemcpy(u.rec, &rec, sizeof rec, hipMemcpyHostToDevice)) != hipSuccess)
    return fail_hip(e, "hipMemcpy H2D");
  u.has_state = true;
  return EDIT_OK;
}

void edit_outer_destroy(edit_outer_t h) {
  if (!h) return;
  int prev = -1;
  if (hipGetDevice(&prev) == hipSuccess && prev != h->device) (void)hipSetDevice(h->device);
  for (Unit& u : h->units) (void)wait_unit(h, u);
  destroy_units(h);
  if (prev >= 0 && prev != h->device) (void)hipSetDevice(prev);
  delete h;
}

edit_status_t edit_outer_set_profiling(edit_outer_t h, int32_t every) {
  if (!h) return fail(EDIT_EINVAL, "NULL handle");
  if (every < 0) return fail(EDIT_EINVAL, "every must be >= 0");
  h->profile_every = every;
  return EDIT_OK;
}

edit_status_t edit_outer_kernel_times(edit_outer_t h, int32_t layer, float ms[2]) {
  if (!h || !ms) return fail(EDIT_EINVAL, "NULL argument");
  if (layer < 0 || layer >= h->cfg.num_layers)
    return fail(EDIT_EINVAL, "layer " + std::to_string(layer) + " out of range");
  Unit& u = h->units[layer];
  if (!u.profiled) return fail(EDIT_ESTATE, "the unit's last step was not profiled");
  hipError_t e = hipEventSynchronize(u.prof[3]);
  if (e != hipSuccess) return fail_hip(e, "hipEventSynchronize");
  if ((e = hipEventElapsedTime(&ms[0], u.prof[0], u.prof[1])) != hipSuccess ||
      (e = hipEventElapsedTime(&ms[1], u.prof[2], u.prof[3])) != hipSuccess)
    return fail_hip(e, "hipEventElapsedTime");
  return EDIT_OK;
}

edit_status_t edit_outer_update_probe(edit_outer_t h, int32_t layer, float* theta, float* momentum,
                                      void* const* replicas, void* stream) {
  if (!h) return fail(EDIT_EINVAL, "NULL handle");
  EDIT_TRY(check_step(h, layer, theta, momentum, replicas));
  EDIT_TRY(check_device(h));
  const Unit& u = h->units[layer];
  if (u.n == 0) return EDIT_OK;
  const hipError_t e =
      launch_pattern_probe(h->cfg.num_workers, h->cfg.replica_dtype == EDIT_BF16, u.blocks2, h->pass2_lds, theta,
                           momentum, replicas, u.n, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? EDIT_OK : fail_hip(e, "update probe launch");
}

edit_status_t edit_outer_copy_probe(void* dst, const void* src, int64_t nbytes, void* stream) {
  if (nbytes < 0 || (nbytes & 15)) return fail(EDIT_EINVAL, "nbytes must be a non-negative multiple of 16");
  if (nbytes == 0) return EDIT_OK;
  if (!dst || !src || !aligned16(dst) || !aligned16(src))
    return fail(EDIT_EINVAL, "dst and src must be non-NULL and 16-byte aligned");
  const uintptr_t d = reinterpret_cast<uintptr_t>(dst), s = reinterpret_cast<uintptr_t>(src);
  if (d < s + nbytes && s < d + nbytes) return fail(EDIT_EINVAL, "dst and src overlap");
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return fail_hip(e, "hipGetDevice");
  // One 16-byte vector per thread, a flat grid, as in the update pass (a
  // persistent grid-stride copy measured 4.6 TB/s against 6.2 here); the
  // grid-stride loop only takes over past the largest grid.
  const int64_t nvec = nbytes / 16;
  const int blocks = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(INT32_MAX, ceil_div(nvec, kCopyThreads))));
  e = launch_copy(dst, src, nbytes, blocks, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail_hip(e, "copy launch");
  return EDIT_OK;
}

}  // extern "C"
