// C ABI of attention with terms in its scores.  Argument checks are made on the host
// before any HIP call.
#include "checks.h"

#include "score_attn.h"

namespace {

constexpr size_t kMaxLd = (size_t)1 << 24;
constexpr long long kMaxRows = 1LL << 26, kMaxHeads = 1LL << 21, kMaxEntries = 1LL << 26;
static_assert(2 * (kMaxRows / 16 + kMaxHeads) < kMaxBlocks, "workgroups of a launch");
static_assert(kMaxEntries * 64 <= kMaxBlocks * 256, "threads of the table's sums");

pb_status check_config(const pb_score_attn_config* c) {
  if (!c) return fail(PB_ERR_INVALID_ARG, "cfg is NULL");
  if (!known(c->dtype)) return fail(PB_ERR_INVALID_ARG, "unknown dtype %d", (int)c->dtype);
  if (!known(c->products)) return fail(PB_ERR_INVALID_ARG, "unknown products %d", (int)c->products);
  if (c->batch < 1 || c->seq_q < 1 || c->seq_k < 1 || c->heads < 1 || c->kv_heads < 1)
    return fail(PB_ERR_INVALID_ARG, "batch=%d, seq_q=%d, seq_k=%d, heads=%d, kv_heads=%d: each "
                "must be >= 1", c->batch, c->seq_q, c->seq_k, c->heads, c->kv_heads);
  if (c->seq_q > c->seq_k)
    return fail(PB_ERR_INVALID_ARG, "seq_q=%d > seq_k=%d", c->seq_q, c->seq_k);
  if (c->heads % c->kv_heads)
    return fail(PB_ERR_INVALID_ARG, "heads=%d is no multiple of kv_heads=%d", c->heads, c->kv_heads);
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128)
    return fail(PB_ERR_UNSUPPORTED, "head_dim=%d must be 64, 96 or 128", c->head_dim);
  if (c->causal != 0 && c->causal != 1) return fail(PB_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (c->window < 1) return fail(PB_ERR_INVALID_ARG, "window=%d must be >= 1", c->window);
  if (!(c->scale > 0.f) || !std::isfinite(c->scale))
    return fail(PB_ERR_INVALID_ARG, "scale must be finite and > 0");
  // (the coefficients of tanh hold powers of scale / cap up to the ninth)
  if (c->cap != 0.f && !(c->cap >= c->scale / 4096.f && c->cap <= 0x1p100f &&
                         c->cap <= c->scale * 0x1p120f))
    return fail(PB_ERR_INVALID_ARG, "cap must be 0, or in scale / 2^12 .. scale 2^120, and at most "
                "2^100");
  if (c->buckets != 0) {
    const int side = c->causal ? c->buckets : c->buckets / 2;
    if (c->buckets > PB_SCORE_MAX_BUCKETS || side < 2 || (!c->causal && c->buckets % 2))
      return fail(PB_ERR_INVALID_ARG, "buckets=%d must be 2..%d, or even from 4 on when not causal",
                  c->buckets, PB_SCORE_MAX_BUCKETS);
    if (c->max_distance <= side / 2 || c->max_distance > (1 << 20))
      return fail(PB_ERR_INVALID_ARG, "max_distance=%d must be in %d..2^20", c->max_distance,
                  side / 2 + 1);
  }
  // A launch has workgroups for 16 rows at least of each head's queries and keys: fewer
  // than kMaxBlocks, also where a head has one row.
  if ((long long)c->batch * c->seq_q > kMaxRows / c->heads ||
      (long long)c->batch * c->seq_k > kMaxRows / c->kv_heads)
    return fail(PB_ERR_UNSUPPORTED, "over 2^26 rows of queries' or of keys' heads");
  if ((long long)c->batch * c->heads > kMaxHeads)
    return fail(PB_ERR_UNSUPPORTED, "batch*heads is over 2^21");
  // The table's gradient is summed by a wave an entry.
  if ((long long)c->buckets * c->heads >= kMaxEntries)
    return fail(PB_ERR_UNSUPPORTED, "a table of 2^26 entries or more");
  return PB_OK;
}

// The first distance of each bucket of a side: of one distance each below E = side / 2,
// then the least d with d >= E (max_distance / E)^(k / (side - E)).  A power that is a
// whole number comes out of pow() next to it; none other is as near (to 1e-11 of its
// value) for the sizes that are allowed.
void borders_of(const pb_score_attn_config* c, int* first) {
  const int side = c->causal ? c->buckets : c->buckets / 2, e = side / 2;
  for (int i = 0; i < side; ++i) {
    if (i <= e) {
      first[i] = i;
      continue;
    }
    const double x = e * pow((double)c->max_distance / e, (double)(i - e) / (side - e));
    const double r = nearbyint(x);
    first[i] = (int)(fabs(x - r) < 1e-11 * x ? r : ceil(x));
  }
}

// A tensor's rows (in bytes), by name.
struct Named {
  const char* name;
  Span s;
  bool out;
};
Span rows_of(const pb_score_attn_config* c, const void* p, size_t ld, bool kv) {
  const size_t e = size_of(c->dtype);
  return Span{p, ld * e, (size_t)(kv ? c->kv_heads : c->heads) * c->head_dim * e,
              (int64_t)c->batch * (kv ? c->seq_k : c->seq_q)};
}
Span dense(const void* p, size_t bytes) { return Span{p, bytes, bytes, 1}; }
pb_status check_tensor(const pb_score_attn_config* c, const char* name, const void* p, size_t ld,
                       bool kv) {
  const pb_status st = check_ptr(p, 16, name);
  if (st != PB_OK) return st;
  const size_t width = (size_t)(kv ? c->kv_heads : c->heads) * c->head_dim;
  if (ld < width) return fail(PB_ERR_INVALID_ARG, "%s: ld=%zu < heads*head_dim=%zu", name, ld, width);
  if (ld * size_of(c->dtype) % 16)
    return fail(PB_ERR_INVALID_ARG, "%s: ld=%zu is no multiple of 16 bytes", name, ld);
  if (ld >= kMaxLd) return fail(PB_ERR_UNSUPPORTED, "%s: ld=%zu is 2^24 or more", name, ld);
  return PB_OK;
}
template <size_t N>
pb_status check_named(const Named (&x)[N]) {
  for (size_t i = 0; i < N; ++i)
    for (size_t j = 0; j < i; ++j)
      if ((x[i].out || x[j].out) && overlap(x[i].s, x[j].s, 1))
        return fail(PB_ERR_INVALID_ARG, "%s and %s overlap", x[j].name, x[i].name);
  return PB_OK;
}

pb_status check_terms(const pb_score_attn_config* c, const pb_score_terms* t) {
  if (t->docs && t->n_docs < 0) return fail(PB_ERR_INVALID_ARG, "n_docs=%d", t->n_docs);
  PB_CHECK(check_opt(t->docs, 4, "docs"));
  PB_CHECK(check_opt(t->prefix, 4, "prefix"));
  PB_CHECK(check_opt(t->slopes, 4, "slopes"));
  PB_CHECK(check_opt(t->table, 4, "table"));
  if (t->slopes && t->table) return fail(PB_ERR_INVALID_ARG, "slopes and a table");
  if ((t->table != nullptr) != (c->buckets != 0))
    return fail(PB_ERR_INVALID_ARG, "buckets=%d %s a table", c->buckets,
                t->table ? "with" : "without");
  return PB_OK;
}

size_t docs_bytes(const pb_score_terms* t) { return t->docs ? 4 * ((size_t)t->n_docs + 1) : 0; }
size_t prefix_bytes(const pb_score_attn_config* c, const pb_score_terms* t) {
  return 4 * (size_t)(t->docs ? t->n_docs : c->batch);
}

const pb_score_terms kNoTerms{};
constexpr int kMaxPack = 8;  // heads of a block of rows

pb::ScoreArgs args_of(const pb_score_attn_config* c, const pb_score_terms* t) {
  pb::ScoreArgs a{};
  a.batch = c->batch, a.seq_q = c->seq_q, a.seq_k = c->seq_k;
  a.heads = c->heads, a.kv_heads = c->kv_heads, a.group = c->heads / c->kv_heads;
  a.causal = c->causal, a.window = c->window;
  a.scale = c->scale, a.cap = c->cap;
  a.wide = c->products == PB_F32;
  a.dscale = c->seq_k == 1 || (c->window == 1 && !t->prefix) ? 0.f : c->scale;
  a.docs = t->docs, a.prefix = t->prefix, a.n_docs = t->n_docs;
  a.slopes = t->slopes, a.table = t->table;
  a.buckets = c->buckets, a.side = c->causal ? c->buckets : c->buckets / 2;
  if (c->buckets) {
    borders_of(c, a.first);
    unsigned char* map = reinterpret_cast<unsigned char*>(a.map);
    for (int d = 0, k = 0; d < pb::kScoreMap; ++d) {
      while (k + 1 < a.side && a.first[k + 1] <= d) ++k;
      map[d] = (unsigned char)k;
    }
  }
  a.pack = 1;
  // (with a table a power of two: lanes of the table's gradient have one head each)
  for (int n = 2; n <= kMaxPack; ++n)
    if (a.group % n == 0 && (!c->buckets || (n & (n - 1)) == 0)) a.pack = n;
  return a;
}
// What a call's plans depend on beside the config: the workspace's sizes are for any
// terms.
size_t fwd_bytes(const pb_score_attn_config* c) {
  if (c->dtype != PB_BF16) return 0;
  size_t most = 0;
  for (int prefix = 0; prefix < 2; ++prefix) {
    pb::ScoreArgs a = args_of(c, &kNoTerms);
    static const int some = 0;
    a.prefix = prefix ? &some : nullptr;
    most = std::max(most, pb::score_fwd_part_bytes(c->head_dim, a, pb::score_fwd_plan(c->head_dim, a)));
  }
  return align256(most);
}

// min: without room for partial results.
size_t bwd_bytes(const pb_score_attn_config* c, bool min) {
  if (c->dtype != PB_BF16) return align256(4 * pb::score_bias_part_floats_f32(args_of(c, &kNoTerms)));
  size_t most = 0;
  for (int prefix = 0; prefix < 2; ++prefix) {
    pb::ScoreArgs a = args_of(c, &kNoTerms);
    static const int some = 0;
    a.prefix = prefix ? &some : nullptr;
    const pb::ScoreBwdPlan p = min ? pb::score_bwd_whole(a) : pb::score_bwd_plan(c->head_dim, a);
    most = std::max(most, pb::score_bwd_bytes(c->head_dim, a, p));
  }
  return align256(most);
}

}  // namespace

extern "C" {

pb_status pblock_score_attn_borders(const pb_score_attn_config* cfg, int* first) {
  PB_CHECK(check_config(cfg));
  if (!first) return fail(PB_ERR_INVALID_ARG, "first is NULL");
  if (cfg->buckets == 0) return fail(PB_ERR_INVALID_ARG, "buckets=0");
  borders_of(cfg, first);
  return nothing_to_do();
}

size_t pblock_score_attn_workspace_bytes(const pb_score_attn_config* cfg, int mode) {
  if (check_config(cfg) != PB_OK) return 0;
  switch (mode) {
    case PB_ATTN_WS_FORWARD: return fwd_bytes(cfg);
    case PB_ATTN_WS_BACKWARD_MIN: return bwd_bytes(cfg, true);
    case PB_ATTN_WS_BACKWARD: return bwd_bytes(cfg, false);
    default: return 0;
  }
}

pb_status pblock_score_attn_forward(const pb_score_attn_config* cfg, const pb_score_terms* terms,
                                    const void* q, size_t ld_q, const void* k, const void* v,
                                    size_t ld_kv, void* o, size_t ld_o, float* lse, void* ws,
                                    size_t ws_bytes, hipStream_t stream) {
  PB_CHECK(check_config(cfg));
  const pb_score_terms* t = terms ? terms : &kNoTerms;
  PB_CHECK(check_terms(cfg, t));
  PB_CHECK(check_tensor(cfg, "q", q, ld_q, false));
  PB_CHECK(check_tensor(cfg, "k", k, ld_kv, true));
  PB_CHECK(check_tensor(cfg, "v", v, ld_kv, true));
  PB_CHECK(check_tensor(cfg, "o", o, ld_o, false));
  PB_CHECK(check_ptr(lse, 4, "lse"));
  if (ws && (uintptr_t)ws % 256) return fail(PB_ERR_INVALID_ARG, "ws is not 256-byte aligned");
  const size_t rows = (size_t)cfg->batch * cfg->heads * cfg->seq_q;
  const Named all[] = {{"q", rows_of(cfg, q, ld_q, false), false},
                       {"k", rows_of(cfg, k, ld_kv, true), false},
                       {"v", rows_of(cfg, v, ld_kv, true), false},
                       {"docs", dense(t->docs, docs_bytes(t)), false},
                       {"prefix", dense(t->prefix, prefix_bytes(cfg, t)), false},
                       {"slopes", dense(t->slopes, 4 * (size_t)cfg->heads), false},
                       {"table", dense(t->table, 4 * (size_t)cfg->buckets * cfg->heads), false},
                       {"o", rows_of(cfg, o, ld_o, false), true},
                       {"lse", dense(lse, 4 * rows), true},
                       {"ws", dense(ws, ws ? ws_bytes : 0), true}};
  PB_CHECK(check_named(all));
  pb::ScoreArgs a = args_of(cfg, t);
  a.q = q, a.k = k, a.v = v, a.ld_q = (int)ld_q, a.ld_kv = (int)ld_kv;
  a.o = o, a.ld_o = (int)ld_o, a.lse = lse;
  if (cfg->dtype == PB_BF16) {
    pb::ScorePlan p = pb::score_fwd_plan(cfg->head_dim, a);
    if (!ws || ws_bytes < pb::score_fwd_part_bytes(cfg->head_dim, a, p)) p = {1};
    pb::launch_score_forward_bf16(cfg->head_dim, a, p, ws, stream);
  } else {
    pb::launch_score_forward_f32(cfg->head_dim, a, stream);
  }
  return finish_launches();
}

pb_status pblock_score_attn_backward(const pb_score_attn_config* cfg, const pb_score_terms* terms,
                                     const void* q, size_t ld_q, const void* k, const void* v,
                                     size_t ld_kv, const void* o, size_t ld_o, const void* d_o,
                                     size_t ld_do, const float* lse, void* dq, size_t ld_dq,
                                     void* dk, void* dv, size_t ld_dkv, float* dtable, void* ws,
                                     size_t ws_bytes, hipStream_t stream) {
  PB_CHECK(check_config(cfg));
  const pb_score_terms* t = terms ? terms : &kNoTerms;
  PB_CHECK(check_terms(cfg, t));
  PB_CHECK(check_tensor(cfg, "q", q, ld_q, false));
  PB_CHECK(check_tensor(cfg, "k", k, ld_kv, true));
  PB_CHECK(check_tensor(cfg, "v", v, ld_kv, true));
  PB_CHECK(check_tensor(cfg, "o", o, ld_o, false));
  PB_CHECK(check_tensor(cfg, "d_o", d_o, ld_do, false));
  PB_CHECK(check_ptr(lse, 4, "lse"));
  PB_CHECK(check_tensor(cfg, "dq", dq, ld_dq, false));
  PB_CHECK(check_tensor(cfg, "dk", dk, ld_dkv, true));
  PB_CHECK(check_tensor(cfg, "dv", dv, ld_dkv, true));
  PB_CHECK(check_opt(dtable, 4, "dtable"));
  if (dtable && !t->table) return fail(PB_ERR_INVALID_ARG, "dtable without a table");
  PB_CHECK(check_ws(ws, ws_bytes,
                    pblock_score_attn_workspace_bytes(cfg, PB_ATTN_WS_BACKWARD_MIN)));
  const size_t rows = (size_t)cfg->batch * cfg->heads * cfg->seq_q;
  const size_t table = 4 * (size_t)cfg->buckets * cfg->heads;
  const Named all[] = {{"q", rows_of(cfg, q, ld_q, false), false},
                       {"k", rows_of(cfg, k, ld_kv, true), false},
                       {"v", rows_of(cfg, v, ld_kv, true), false},
                       {"o", rows_of(cfg, o, ld_o, false), false},
                       {"d_o", rows_of(cfg, d_o, ld_do, false), false},
                       {"lse", dense(lse, 4 * rows), false},
                       {"docs", dense(t->docs, docs_bytes(t)), false},
                       {"prefix", dense(t->prefix, prefix_bytes(cfg, t)), false},
                       {"slopes", dense(t->slopes, 4 * (size_t)cfg->heads), false},
                       {"table", dense(t->table, table), false},
                       {"dq", rows_of(cfg, dq, ld_dq, false), true},
                       {"dk", rows_of(cfg, dk, ld_dkv, true), true},
                       {"dv", rows_of(cfg, dv, ld_dkv, true), true},
                       {"dtable", dense(dtable, table), true},
                       {"ws", dense(ws, ws ? ws_bytes : 0), true}};
  PB_CHECK(check_named(all));
  pb::ScoreArgs a = args_of(cfg, t);
  a.q = q, a.k = k, a.v = v, a.ld_q = (int)ld_q, a.ld_kv = (int)ld_kv;
  a.o = const_cast<void*>(o), a.ld_o = (int)ld_o, a.lse = const_cast<float*>(lse);
  a.d_o = d_o, a.ld_do = (int)ld_do;
  a.dq = dq, a.ld_dq = (int)ld_dq, a.dk = dk, a.dv = dv, a.ld_dkv = (int)ld_dkv;
  a.dtable = dtable, a.bias_part = (float*)ws;
  if (cfg->dtype == PB_BF16) {
    pb::ScoreBwdPlan p = pb::score_bwd_plan(cfg->head_dim, a);
    if (ws_bytes < pb::score_bwd_bytes(cfg->head_dim, a, p)) p = pb::score_bwd_whole(a);
    pb::launch_score_backward_bf16(cfg->head_dim, a, p, ws, stream);
  } else {
    pb::launch_score_backward_f32(cfg->head_dim, a, stream);
  }
  return finish_launches();
}

}  // extern "C"
