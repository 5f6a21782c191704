// C ABI of the AdamW step.  Argument checks are made on the host before any HIP call.
#include "checks.h"

namespace {

pb_status check_adamw(const pb_adamw_config* c) {
  if (!c) return fail(PB_ERR_INVALID_ARG, "cfg is NULL");
  if (!std::isfinite(c->lr)) return fail(PB_ERR_INVALID_ARG, "lr is not finite");
  if (!(c->beta1 >= 0.f && c->beta1 < 1.f) || !(c->beta2 >= 0.f && c->beta2 < 1.f))
    return fail(PB_ERR_INVALID_ARG, "beta1=%g, beta2=%g: each must be in [0, 1)",
                (double)c->beta1, (double)c->beta2);
  if (!(c->eps > 0.f) || !std::isfinite(c->eps))
    return fail(PB_ERR_INVALID_ARG, "eps=%g must be positive and finite", (double)c->eps);
  if (!std::isfinite(c->grad_scale)) return fail(PB_ERR_INVALID_ARG, "grad_scale is not finite");
  if (c->step < 1) return fail(PB_ERR_INVALID_ARG, "step=%d must be >= 1", c->step);
  if (c->bias_correction != 0 && c->bias_correction != 1)
    return fail(PB_ERR_INVALID_ARG, "bias_correction must be 0 or 1");
  if (c->state != PB_ADAMW_F32 && c->state != PB_ADAMW_E4M3)
    return fail(PB_ERR_INVALID_ARG, "state=%d", c->state);
  return PB_OK;
}

struct Piece {
  uintptr_t at;
  size_t bytes;
  int tensor;
  bool out;
};
constexpr int kArrays = 7;

// Whether an array that is written meets another: neighbours in the order of their
// addresses tell, each with the furthest end before it.
pb_status check_pieces(Piece* p, int n) {
  std::sort(p, p + n, [](const Piece& a, const Piece& b) { return a.at < b.at; });
  uintptr_t end = 0, out_end = 0;  // of all before, and of those that are written
  int last = 0;
  for (int i = 0; i < n; ++i) {
    if (p[i].at < out_end || (p[i].out && p[i].at < end))
      return fail(PB_ERR_INVALID_ARG, "an array of tensor %d that is written overlaps one of tensor %d",
                  p[last].tensor, p[i].tensor);
    if (p[i].at + p[i].bytes >= end) end = p[i].at + p[i].bytes, last = i;
    if (p[i].out) out_end = std::max(out_end, p[i].at + p[i].bytes);
  }
  return PB_OK;
}

}  // namespace

extern "C" {

pb_status pblock_adamw_step(const pb_adamw_config* cfg, int n_tensors,
                            const pb_adamw_tensor* tensors, pb_dtype copy_dtype,
                            hipStream_t stream) {
  const pb_status st = check_adamw(cfg);
  if (st != PB_OK) return st;
  if (!known(copy_dtype)) return fail(PB_ERR_INVALID_ARG, "copy_dtype=%d", (int)copy_dtype);
  if (n_tensors < 1 || n_tensors > PB_ADAMW_MAX_TENSORS)
    return fail(PB_ERR_INVALID_ARG, "n_tensors=%d must be in 1..%d", n_tensors,
                PB_ADAMW_MAX_TENSORS);
  if (!tensors) return fail(PB_ERR_INVALID_ARG, "tensors is NULL");
  static_assert(PB_ADAMW_BLOCK == pb::kAdamBlock, "elements of a scale");
  const bool e4m3 = cfg->state == PB_ADAMW_E4M3;
  Piece pieces[kArrays * PB_ADAMW_MAX_TENSORS];
  int n_pieces = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const pb_adamw_tensor& x = tensors[i];
    if (!(x.weight_decay >= 0.f) || !std::isfinite(x.weight_decay))
      return fail(PB_ERR_INVALID_ARG, "tensor %d: weight_decay=%g", i, (double)x.weight_decay);
    if (x.numel > (size_t)(kMaxBlocks - 1) * pb::kAdamChunk)
      return fail(PB_ERR_UNSUPPORTED, "tensor %d: %zu elements, over 2^34 - 2^10", i, x.numel);
    if (x.numel == 0) continue;
    const size_t s = e4m3 ? 1 : 4, scales = 4 * ((x.numel + PB_ADAMW_BLOCK - 1) / PB_ADAMW_BLOCK);
    const struct {
      const char* name;
      const void* p;
      size_t align, bytes;
      bool need;
    } a[kArrays] = {
        {"param", x.param, 4, 4 * x.numel, true},
        {"grad", x.grad, 4, 4 * x.numel, true},
        {"exp_avg", x.exp_avg, s, s * x.numel, true},
        {"exp_avg_sq", x.exp_avg_sq, s, s * x.numel, true},
        {"avg_scale", e4m3 ? x.avg_scale : nullptr, 4, scales, e4m3},
        {"sq_scale", e4m3 ? x.sq_scale : nullptr, 4, scales, e4m3},
        {"param_copy", x.param_copy, size_of(copy_dtype), size_of(copy_dtype) * x.numel, false}};
    for (int k = 0; k < kArrays; ++k) {
      if (!a[k].p) {
        if (a[k].need) return fail(PB_ERR_INVALID_ARG, "tensor %d: %s is NULL", i, a[k].name);
        continue;
      }
      if ((uintptr_t)a[k].p % a[k].align)
        return fail(PB_ERR_INVALID_ARG, "tensor %d: %s is not aligned to its element", i, a[k].name);
      pieces[n_pieces++] = Piece{(uintptr_t)a[k].p, a[k].bytes, i, k != 1};
    }
  }
  const pb_status apart = check_pieces(pieces, n_pieces);
  if (apart != PB_OK) return apart;
  if (n_pieces == 0) return nothing_to_do();

  pb::AdamScalars c{};
  c.lr = cfg->lr, c.eps = cfg->eps, c.grad_scale = cfg->grad_scale;
  c.beta1 = cfg->beta1, c.rest1 = 1.0f - cfg->beta1;
  c.beta2 = cfg->beta2, c.rest2 = 1.0f - cfg->beta2;
  c.c1 = cfg->bias_correction ? (float)(1.0 / (1.0 - pow((double)cfg->beta1, cfg->step))) : 1.f;
  c.c2 = cfg->bias_correction ? (float)(1.0 / (1.0 - pow((double)cfg->beta2, cfg->step))) : 1.f;
  c.eps_in_range = cfg->eps >= 0x1p-90f && cfg->eps <= 0x1p40f;
  pb::AdamTable t{};
  long long chunks = 0;
  auto launch = [&] {
    if (t.n > 0) pb::launch_adamw(t, c, e4m3, dt_of(copy_dtype), stream);
    t.n = 0, chunks = 0;
  };
  for (int i = 0; i < n_tensors; ++i) {
    const pb_adamw_tensor& x = tensors[i];
    if (x.numel == 0) continue;
    const long long more = ((long long)x.numel + pb::kAdamChunk - 1) / pb::kAdamChunk;
    if (t.n == pb::kAdamMax || chunks + more >= kMaxBlocks) launch();
    const int k = t.n++;
    t.w[k] = x.param, t.g[k] = x.grad, t.m[k] = x.exp_avg, t.v[k] = x.exp_avg_sq;
    t.m_scale[k] = x.avg_scale, t.v_scale[k] = x.sq_scale, t.copy[k] = x.param_copy;
    t.numel[k] = (long long)x.numel;
    t.seed[k] = x.seed;
    t.decay[k] = (float)(1.0 - (double)cfg->lr * (double)x.weight_decay);
    t.chunk0[k] = (int)chunks;
    t.chunk0[k + 1] = (int)(chunks += more);
  }
  launch();
  return finish_launches();
}

}  // extern "C"
