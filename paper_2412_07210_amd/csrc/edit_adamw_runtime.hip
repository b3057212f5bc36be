// Host runtime of the AdamW step (include/edit_outer.h, "AdamW over many
// tensors"): checks, the tables of tensors that launches take as kernel
// arguments, and the launches.  A call enqueues norm pass (with a clip) ->
// decision -> update passes on the caller's stream.
#include <algorithm>
#include <cmath>
#include <memory>
#include <string>
#include <vector>

#include "edit_adamw_internal.h"
#include "edit_group_internal.h"
#include "written_ranges.h"

using namespace edit;

namespace {

#define ADAM_TRY(expr)                \
  do {                                \
    const edit_status_t st_ = (expr); \
    if (st_ != EDIT_OK) return st_;   \
  } while (0)

edit_status_t afail(edit_status_t s, const std::string& msg) { return set_error(s, msg.c_str()); }

edit_status_t afail_hip(hipError_t e, const char* what) {
  return afail(EDIT_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}

// No exception leaves the library: what the lists and messages of a call throw.
template <typename F>
edit_status_t guarded(const F& f) {
  try {
    return f();
  } catch (const std::exception&) {
    return afail(EDIT_ENOMEM, "host allocation failed");
  }
}

constexpr int64_t kMaxNumel = int64_t(1) << 33;
constexpr int64_t kMaxStep = int64_t(1) << 62;
constexpr int64_t kMaxBlocks = (int64_t(1) << 32) / kAdamThreads - 1;  // of a launch: fewer than 2^32 threads
static_assert(kMaxNumel / (kAdamThreads * 4) <= kMaxBlocks, "a tensor fits a launch");

int64_t chunks_of(int64_t numel, int64_t chunk) { return (numel + chunk - 1) / chunk; }

constexpr int kKinds = 6;  // parameters, gradients, m, v and their scales; of a conversion the fp32 m and v first

}  // namespace

struct edit_adamw {
  std::vector<int64_t> numel;
  std::vector<double> decay;
  AdamKind kind{};
  AdamHyper hyper{};
  double weight_decay = 0.0;
  int device = 0, num_cu = 0;
  int64_t blocks = 0;  // of the update pass over all tensors
  char* arena = nullptr;
  AdamState state{};
  double* partials = nullptr;  // a norm launch's follow the one's before
  WrittenRanges<kKinds> ranges;  // of the call being checked
};

namespace {

edit_status_t check_adamw_config(const edit_adamw_config_t* cfg) {
  if (cfg->num_tensors < 0) return afail(EDIT_EINVAL, "num_tensors must be >= 0");
  if (cfg->num_tensors > 0 && !cfg->numel) return afail(EDIT_EINVAL, "numel must not be NULL");
  for (const auto& [value, name] : {std::pair<int32_t, const char*>{cfg->dtype, "dtype"}, {cfg->grad_dtype, "grad_dtype"}})
    if (value != EDIT_F32 && value != EDIT_BF16)
      return afail(EDIT_EINVAL, std::string(name) + " must be EDIT_F32 or EDIT_BF16");
  if (cfg->held != EDIT_ADAMW_F32 && cfg->held != EDIT_ADAMW_E4M3)
    return afail(EDIT_EINVAL, "held must be EDIT_ADAMW_F32 or EDIT_ADAMW_E4M3");
  if (cfg->flags & ~EDIT_ADAMW_STOCHASTIC) return afail(EDIT_EINVAL, "unknown flag bits");
  if ((cfg->flags & EDIT_ADAMW_STOCHASTIC) && cfg->dtype != EDIT_BF16)
    return afail(EDIT_EINVAL, "EDIT_ADAMW_STOCHASTIC needs bf16 parameters");
  if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0)) return afail(EDIT_EINVAL, "beta1 must be in [0, 1)");
  if (!(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return afail(EDIT_EINVAL, "beta2 must be in [0, 1)");
  if (!(cfg->eps >= 1e-12) || !(cfg->eps <= 1e30)) return afail(EDIT_EINVAL, "eps must be in [1e-12, 1e30]");
  if (!(cfg->weight_decay >= 0.0) || !std::isfinite(cfg->weight_decay))
    return afail(EDIT_EINVAL, "weight_decay must be finite and >= 0");
  for (int k = 0; k < cfg->num_tensors; ++k) {
    const std::string at = "[" + std::to_string(k) + "]";
    if (cfg->numel[k] < 0) return afail(EDIT_EINVAL, "numel" + at + " is negative");
    if (cfg->numel[k] > kMaxNumel) return afail(EDIT_EINVAL, "numel" + at + " must be at most 2^33");
    if (cfg->decay && (!(cfg->decay[k] >= 0.0) || !std::isfinite(cfg->decay[k])))
      return afail(EDIT_EINVAL, "decay" + at + " must be finite and >= 0");
  }
  return EDIT_OK;
}

edit_status_t check_adamw_device(const edit_adamw* h) {
  int dev = -1;
  const hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return afail_hip(e, "hipGetDevice");
  if (dev != h->device)
    return afail(EDIT_EINVAL, "call made with device " + std::to_string(dev) +
                                  " current; the handle belongs to device " + std::to_string(h->device));
  return EDIT_OK;
}

// Notes the buffer of tensor k for the check of overlaps.
edit_status_t note(edit_adamw* h, int kind, const void* p, int64_t bytes, uintptr_t align, const char* name, int k) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  if (!p || (lo & (align - 1))) {
    const std::string what = std::string(name) + "[" + std::to_string(k) + "]";
    if (!p) return afail(EDIT_EINVAL, what + " must not be NULL");
    return afail(EDIT_EINVAL, what + " must be " + std::to_string(align) + "-byte aligned");
  }
  h->ranges.add(kind, lo, lo + static_cast<uintptr_t>(bytes));
  return EDIT_OK;
}

// `writes`: a bit for each kind of buffer that the call writes.
edit_status_t check_overlaps(edit_adamw* h, unsigned writes) {
  switch (h->ranges.find(writes)) {
    case kOverlapWritten:
      return afail(EDIT_EINVAL, "what is written must not overlap: parameters and states, or one of them twice");
    case kOverlapRead:
      return afail(EDIT_EINVAL, "what is read must not overlap what is written");
    default:
      return EDIT_OK;
  }
}

edit_status_t check_states(edit_adamw* h, const edit_adamw_tensors_t* t, int k) {
  const int64_t n = h->numel[k], bytes = h->kind.held ? n : 4 * n, scales = 4 * chunks_of(n, EDIT_ADAMW_BLOCK);
  ADAM_TRY(note(h, 2, t->exp_avg[k], bytes, 16, "exp_avg", k));
  ADAM_TRY(note(h, 3, t->exp_avg_sq[k], bytes, 16, "exp_avg_sq", k));
  if (h->kind.held) {
    ADAM_TRY(note(h, 4, t->exp_avg_scale[k], scales, 4, "exp_avg_scale", k));
    ADAM_TRY(note(h, 5, t->exp_avg_sq_scale[k], scales, 4, "exp_avg_sq_scale", k));
  }
  return EDIT_OK;
}

edit_status_t check_state_arrays(const edit_adamw* h, const edit_adamw_tensors_t* t) {
  if (!t->exp_avg || !t->exp_avg_sq) return afail(EDIT_EINVAL, "exp_avg and exp_avg_sq must not be NULL");
  if (h->kind.held && (!t->exp_avg_scale || !t->exp_avg_sq_scale))
    return afail(EDIT_EINVAL, "exp_avg_scale and exp_avg_sq_scale must not be NULL");
  return EDIT_OK;
}

// The gradients from tensor *k on that a table has room for.
void fill_norm_table(const edit_adamw* h, const void* const* grad, int chunk, int* k, AdamNormTable* t) {
  int used = 0;
  int64_t chunks = 0;
  for (; *k < static_cast<int>(h->numel.size()) && used < kAdamNormTensors; ++*k) {
    if (!grad[*k] || h->numel[*k] == 0) continue;
    const int64_t more = chunks_of(h->numel[*k], chunk);
    if (chunks + more > INT32_MAX / 2) break;
    t->first[used] = static_cast<int32_t>(chunks);
    t->numel[used] = h->numel[*k];
    t->grad[used++] = grad[*k];
    chunks += more;
  }
  std::fill(t->first + used, t->first + kAdamNormTensors, INT32_MAX);
  t->chunks = static_cast<int32_t>(chunks);
  t->keep = t->chunks;
}

// S of the gradients: to *out, or with no `out` as parts in the workspace, named in *call.
edit_status_t enqueue_sum(edit_adamw* h, const void* const* grad, double* out, AdamCall* call, hipStream_t s) {
  const int tensors = static_cast<int>(h->numel.size()), chunk = adamw_norm_chunk(h->kind.grad_bf16);
  int64_t left = 0, waves = 0;  // chunks of this launch and those behind it; ones of a wave
  int present = 0;
  for (int k = 0; k < tensors; ++k)
    if (grad[k] && h->numel[k]) {
      left += chunks_of(h->numel[k], chunk);
      waves += chunks_of(h->numel[k], adamw_norm_chunk(h->kind.grad_bf16, 64));
      ++present;
    }
  hipError_t e = hipSuccess;
  int k = 0, count = 0;
  if (present <= kAdamNormTensors && waves <= kAdamSmallChunks) {
    AdamNormTable t;
    fill_norm_table(h, grad, adamw_norm_chunk(h->kind.grad_bf16, 64), &k, &t);
    e = launch_adamw_small(h->kind.grad_bf16, t, out ? out : h->partials, s);
    count = 1;
  } else {
    // the update pass reads the gradients next, the last ones first
    const int64_t keep = out ? 0 : kAdamNormKeep / (chunk * (h->kind.grad_bf16 ? 2 : 4));
    while (e == hipSuccess && k < tensors) {
      AdamNormTable t;
      fill_norm_table(h, grad, chunk, &k, &t);
      if (t.chunks == 0) continue;
      t.keep = static_cast<int32_t>(std::min<int64_t>(std::max<int64_t>(left - keep, 0), t.chunks));
      left -= t.chunks;
      const int blocks = std::min(t.chunks, kAdamNormBlocksPerCu * h->num_cu);
      e = launch_adamw_norm(h->kind.grad_bf16, blocks, t, h->partials + count, s);
      count += blocks;
    }
    if (e == hipSuccess && out) e = launch_adamw_sum(h->partials, count, out, s);
  }
  if (e != hipSuccess) return afail_hip(e, "norm pass launch");
  if (call) call->sums = h->partials, call->count = count;
  return EDIT_OK;
}

// Calls launch(blocks, table, before) for every table of tensors, the last ones
// first; fill(k, &tensor): whether tensor k takes part; chunk: elements of a block;
// before: blocks of the tensors before the table's, were all to take part.
template <typename Fill, typename Launch>
edit_status_t for_tables(const edit_adamw* h, int chunk, const Fill& fill, const Launch& launch) {
  int64_t before = 0;
  for (int64_t n : h->numel) before += chunks_of(n, chunk);
  for (int end = static_cast<int>(h->numel.size()), begin = end; end > 0; end = begin) {
    int64_t blocks = 0;
    for (; begin > 0 && end - begin < kAdamTensors; --begin) {
      const int64_t more = chunks_of(h->numel[begin - 1], chunk);
      if (blocks + more > kMaxBlocks) break;
      blocks += more;
    }
    before -= blocks;
    AdamTable t;
    t.base = begin;
    blocks = 0;
    // a tensor that takes no part keeps its place, so that base + place is its index
    for (int k = begin; k < end; ++k) {
      AdamTensor& to = t.tensor[k - begin];
      t.first[k - begin] = static_cast<int32_t>(blocks);
      t.decay[k - begin] = h->decay[k];
      to = {};
      if (h->numel[k] && fill(k, &to)) {
        to.numel = h->numel[k];
        blocks += chunks_of(h->numel[k], chunk);
      }
    }
    if (blocks == 0) continue;
    std::fill(t.first + (end - begin), t.first + 64, INT32_MAX);
    const hipError_t e = launch(static_cast<int>(blocks), t, before);
    if (e != hipSuccess) return afail_hip(e, "update pass launch");
  }
  return EDIT_OK;
}

void fill_states(const edit_adamw* h, const edit_adamw_tensors_t* t, int k, AdamTensor* to) {
  to->m = t->exp_avg[k];
  to->v = t->exp_avg_sq[k];
  if (h->kind.held) {
    to->m_scale = t->exp_avg_scale[k];
    to->v_scale = t->exp_avg_sq_scale[k];
  }
}

edit_status_t convert(edit_adamw* h, bool pack, const edit_adamw_tensors_t* t, const float* const* m, const float* const* v,
                      uint64_t seed, hipStream_t s) {
  if (!h) return afail(EDIT_EINVAL, "NULL handle");
  if (!h->kind.held) return afail(EDIT_EINVAL, "the handle holds its states in fp32");
  if (!t || (!h->numel.empty() && (!m || !v))) return afail(EDIT_EINVAL, "tensors, exp_avg and exp_avg_sq must not be NULL");
  ADAM_TRY(check_adamw_device(h));
  if (h->numel.empty()) return EDIT_OK;
  ADAM_TRY(check_state_arrays(h, t));
  h->ranges.clear();
  for (int k = 0; k < static_cast<int>(h->numel.size()); ++k) {
    const int64_t n = h->numel[k];
    if (n == 0) continue;
    ADAM_TRY(note(h, 0, m[k], 4 * n, 16, "fp32 exp_avg", k));
    ADAM_TRY(note(h, 1, v[k], 4 * n, 16, "fp32 exp_avg_sq", k));
    ADAM_TRY(check_states(h, t, k));
  }
  ADAM_TRY(check_overlaps(h, pack ? 0x3cu : 0x03u));
  return for_tables(
      h, adamw_convert_chunk(pack),
      [&](int k, AdamTensor* to) {
        fill_states(h, t, k, to);
        to->param = const_cast<float*>(m[k]);
        to->grad = v[k];
        return true;
      },
      [&](int blocks, const AdamTable& table, int64_t) { return launch_adamw_convert(pack, blocks, table, adamw_key(seed, 0), s); });
}

edit_status_t sum_squares(edit_adamw* h, const void* const* grad, double* sumsq, hipStream_t s) {
  if (!h) return afail(EDIT_EINVAL, "NULL handle");
  if (!h->numel.empty() && !grad) return afail(EDIT_EINVAL, "grad must not be NULL");
  ADAM_TRY(check_adamw_device(h));
  h->ranges.clear();
  ADAM_TRY(note(h, 0, sumsq, 8, 8, "sumsq", 0));
  const int64_t size = h->kind.grad_bf16 ? 2 : 4;
  for (size_t k = 0; k < h->numel.size(); ++k)
    if (h->numel[k] && grad[k]) ADAM_TRY(note(h, 1, grad[k], size * h->numel[k], size, "grad", static_cast<int>(k)));
  ADAM_TRY(check_overlaps(h, 1u));
  return enqueue_sum(h, grad, sumsq, nullptr, s);
}

edit_status_t step(edit_adamw* h, const edit_adamw_tensors_t* t, const edit_adamw_call_t* call, hipStream_t s) {
  if (!h) return afail(EDIT_EINVAL, "NULL handle");
  if (!t || !call) return afail(EDIT_EINVAL, "tensors and call must not be NULL");
  if (!call->lr_device && (!(call->lr >= 0.0) || !std::isfinite(call->lr)))
    return afail(EDIT_EINVAL, "lr must be finite and >= 0");
  if (reinterpret_cast<uintptr_t>(call->lr_device) & 7u) return afail(EDIT_EINVAL, "lr_device must be 8-byte aligned");
  if (reinterpret_cast<uintptr_t>(call->sumsq) & 7u) return afail(EDIT_EINVAL, "sumsq must be 8-byte aligned");
  if (!(call->max_norm >= 0.0) || !std::isfinite(call->max_norm))
    return afail(EDIT_EINVAL, "max_norm must be finite and > 0, or 0 for no clip");
  ADAM_TRY(check_adamw_device(h));
  const int tensors = static_cast<int>(h->numel.size());
  h->ranges.clear();
  if (tensors > 0) {
    if (!t->param || !t->grad) return afail(EDIT_EINVAL, "param and grad must not be NULL");
    ADAM_TRY(check_state_arrays(h, t));
  }
  const int64_t pb = h->kind.param_bf16 ? 2 : 4, gb = h->kind.grad_bf16 ? 2 : 4;
  bool all = true;  // tensors take part
  for (int k = 0; k < tensors; ++k) {
    const int64_t n = h->numel[k];
    all = all && (n == 0 || t->grad[k]);
    if (n == 0 || !t->grad[k]) continue;
    ADAM_TRY(note(h, 0, t->param[k], pb * n, pb, "param", k));
    ADAM_TRY(note(h, 1, t->grad[k], gb * n, gb, "grad", k));
    ADAM_TRY(check_states(h, t, k));
  }
  constexpr unsigned writes = 0x3du;
  ADAM_TRY(check_overlaps(h, writes));
  for (const double* p : {call->lr_device, call->sumsq}) {
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    if (p && h->ranges.written_at(writes, lo, lo + sizeof *p))
      return afail(EDIT_EINVAL, "lr_device and sumsq must not overlap what is written");
  }

  AdamCall c = {};
  c.lr = call->lr;
  c.lr_device = call->lr_device;
  c.weight_decay = h->weight_decay;
  c.max_norm = call->max_norm > 0.0 ? call->max_norm : INFINITY;
  c.seed = call->seed;
  if (call->sumsq)
    c.sums = call->sumsq, c.count = 1;
  else if (call->max_norm > 0.0)
    ADAM_TRY(enqueue_sum(h, t->grad, nullptr, &c, s));
  // where every block has a t of its own, and every one counts it on
  const bool fused = all && h->blocks > 0 && h->blocks == h->state.slots;
  if (!fused) {
    const hipError_t e = launch_adamw_decide(c, h->hyper, h->state, s);
    if (e != hipSuccess) return afail_hip(e, "decision launch");
  }
  return for_tables(
      h, adamw_chunk(h->kind.param_bf16, h->kind.grad_bf16, h->kind.held),
      [&](int k, AdamTensor* to) {
        if (!t->grad[k]) return false;
        to->param = t->param[k];
        to->grad = t->grad[k];
        fill_states(h, t, k, to);
        return true;
      },
      [&](int blocks, const AdamTable& table, int64_t before) {
        return launch_adamw_step(h->kind, blocks, table, h->hyper, h->state, fused ? &c : nullptr, static_cast<int>(before), s);
      });
}

}  // namespace

extern "C" {

edit_status_t edit_adamw_init(const edit_adamw_config_t* cfg, edit_adamw_t* out) {
  set_error(EDIT_OK, "");
  if (!cfg || !out) return afail(EDIT_EINVAL, "cfg and out must not be NULL");
  *out = nullptr;
  try {
    ADAM_TRY(check_adamw_config(cfg));
    int dev = 0, num_cu = 0;
    ADAM_TRY(current_gfx950(&dev, &num_cu));
    auto h = std::make_unique<edit_adamw>();
    const size_t tensors = static_cast<size_t>(cfg->num_tensors);
    h->numel.assign(cfg->numel, cfg->numel + tensors);
    h->decay.assign(tensors, 1.0);
    if (cfg->decay) h->decay.assign(cfg->decay, cfg->decay + tensors);
    h->kind.param_bf16 = cfg->dtype == EDIT_BF16;
    h->kind.grad_bf16 = cfg->grad_dtype == EDIT_BF16;
    h->kind.held = cfg->held == EDIT_ADAMW_E4M3;
    h->kind.stochastic = cfg->flags & EDIT_ADAMW_STOCHASTIC;
    h->hyper = {cfg->beta1, cfg->beta2, cfg->eps};
    h->weight_decay = cfg->weight_decay;
    h->device = dev;
    h->num_cu = num_cu;
    h->ranges.reserve(tensors + 1);
    // launches of the norm pass: full tables, and ones that end at their count of chunks
    int64_t chunks = 0;
    for (int64_t n : h->numel) chunks += chunks_of(n, adamw_norm_chunk(false));
    const size_t launches = tensors / kAdamNormTensors + 2 + static_cast<size_t>(2 * (chunks / (INT32_MAX / 2)));
    const size_t partials = launches * kAdamNormBlocksPerCu * num_cu * sizeof(double);
    const int chunk = adamw_chunk(h->kind.param_bf16, h->kind.grad_bf16, h->kind.held);
    for (int64_t n : h->numel) h->blocks += chunks_of(n, chunk);
    h->state.slots = h->blocks > 0 && h->blocks <= kAdamFusedBlocks ? static_cast<int32_t>(h->blocks) : 1;
    const size_t kept = 256 + (h->state.slots * sizeof(int64_t) + 255) / 256 * 256;  // the record and t, zero at first
    hipError_t e = hipMalloc(reinterpret_cast<void**>(&h->arena), kept + partials);
    if (e != hipSuccess) return afail(EDIT_ENOMEM, std::string("hipMalloc of the workspace: ") + hipGetErrorString(e));
    e = hipMemset(h->arena, 0, kept);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    if (e != hipSuccess) {
      (void)hipFree(h->arena);
      return afail_hip(e, "edit_adamw_init");
    }
    h->state.rec = reinterpret_cast<AdamRecord*>(h->arena);
    h->state.steps = reinterpret_cast<int64_t*>(h->arena + 256);
    h->partials = reinterpret_cast<double*>(h->arena + kept);
    *out = h.release();
    return EDIT_OK;
  } catch (const std::exception&) {  // the lists' host memory
    return afail(EDIT_ENOMEM, "host allocation failed");
  }
}

edit_status_t edit_adamw_sumsq(edit_adamw_t h, const void* const* grad, double* sumsq, void* stream) {
  return guarded([&] { return sum_squares(h, grad, sumsq, reinterpret_cast<hipStream_t>(stream)); });
}

edit_status_t edit_adamw_step(edit_adamw_t h, const edit_adamw_tensors_t* t, const edit_adamw_call_t* call, void* stream) {
  return guarded([&] { return step(h, t, call, reinterpret_cast<hipStream_t>(stream)); });
}
edit_status_t edit_adamw_pack(edit_adamw_t h, const float* const* exp_avg, const float* const* exp_avg_sq,
                              const edit_adamw_tensors_t* tensors, uint64_t seed, void* stream) {
  return guarded([&] { return convert(h, true, tensors, exp_avg, exp_avg_sq, seed, reinterpret_cast<hipStream_t>(stream)); });
}

edit_status_t edit_adamw_unpack(edit_adamw_t h, const edit_adamw_tensors_t* tensors, float* const* exp_avg,
                                float* const* exp_avg_sq, void* stream) {
  return guarded([&] { return convert(h, false, tensors, exp_avg, exp_avg_sq, 0, reinterpret_cast<hipStream_t>(stream)); });
}

edit_status_t edit_adamw_state_get(edit_adamw_t h, edit_adamw_state_t* out) {
  if (!h || !out) return afail(EDIT_EINVAL, "h and out must not be NULL");
  ADAM_TRY(check_adamw_device(h));
  hipError_t e = hipDeviceSynchronize();
  AdamRecord r;
  int64_t step = 0;
  if (e == hipSuccess) e = hipMemcpy(&r, h->state.rec, sizeof r, hipMemcpyDeviceToHost);
  if (e == hipSuccess) e = hipMemcpy(&step, h->state.steps, sizeof step, hipMemcpyDeviceToHost);
  if (e != hipSuccess) return afail_hip(e, "edit_adamw_state_get");
  *out = {step, r.skipped, r.norm, r.clip};
  return EDIT_OK;
}

edit_status_t edit_adamw_state_set(edit_adamw_t h, int64_t step) {
  if (!h) return afail(EDIT_EINVAL, "NULL handle");
  if (step < 0 || step > kMaxStep) return afail(EDIT_EINVAL, "step must be in [0, 2^62]");
  ADAM_TRY(check_adamw_device(h));
  return guarded([&] {
    const std::vector<int64_t> steps(h->state.slots, step);
    hipError_t e = hipDeviceSynchronize();
    if (e == hipSuccess) e = hipMemcpy(h->state.steps, steps.data(), steps.size() * sizeof step, hipMemcpyHostToDevice);
    if (e == hipSuccess) e = hipDeviceSynchronize();
    return e == hipSuccess ? EDIT_OK : afail_hip(e, "edit_adamw_state_set");
  });
}

void edit_adamw_destroy(edit_adamw_t h) {
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
