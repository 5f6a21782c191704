// C ABI of the operators around the block: rotary positions, the root-mean-square
// norm, the Muon step and its orthogonalisation.  Argument checks are made on the
// host before any HIP call.
#include "abi.h"

#include <math.h>

#include <cmath>

#include <algorithm>

#include "kernels.h"

using pb::align256;
using pb::fail;
using pb::finish_launches;

namespace {

constexpr long long kMaxInt = 2147483647LL;
// Workgroups of 256 threads in a launch of fewer than 2^32 threads.
constexpr long long kMaxBlocks = 1LL << 24;

bool known(pb_dtype dt) { return dt == PB_BF16 || dt == PB_F32; }
size_t size_of(pb_dtype dt) { return dt == PB_BF16 ? 2 : 4; }
pb::Dt dt_of(pb_dtype dt) { return dt == PB_BF16 ? pb::Dt::BF16 : pb::Dt::F32; }

pb_status check_ptr(const void* p, size_t align, const char* name) {
  if (!p) return fail(PB_ERR_INVALID_ARG, "%s is NULL", name);
  if ((uintptr_t)p % align)
    return fail(PB_ERR_INVALID_ARG, "%s is not %zu-byte aligned", name, align);
  return PB_OK;
}
pb_status check_opt(const void* p, size_t align, const char* name) {
  return p ? check_ptr(p, align, name) : PB_OK;
}
pb_status check_ws(const void* ws, size_t bytes, size_t need) {
  if (!need) return PB_OK;
  if (!ws || (uintptr_t)ws % 256)
    return fail(PB_ERR_INVALID_ARG, "ws is NULL or not 256-byte aligned");
  if (bytes < need) return fail(PB_ERR_WORKSPACE, "ws_bytes=%zu < %zu needed", bytes, need);
  return PB_OK;
}

// Rows of `width` elements of `e` bytes, ld elements apart.
struct Span {
  const void* p;
  size_t ld, width;
  int64_t rows;
};
// Whether two such share memory.  Tensors apart as a whole, or of one leading dimension
// (whose rows may interleave), are told at once; else the rows of one are looked up among
// the other's, a few ns each.
bool overlap(const Span& a, const Span& b, size_t e) {
  if (!a.rows || !b.rows || !a.p || !b.p) return false;
  const Span &lo = (uintptr_t)a.p <= (uintptr_t)b.p ? a : b, &hi = &lo == &a ? b : a;
  const size_t off = ((uintptr_t)hi.p - (uintptr_t)lo.p) / e;  // elements from lo to hi
  if (off >= (size_t)(lo.rows - 1) * lo.ld + lo.width) return false;
  if (lo.rows > 1 && off % lo.ld < lo.width) return true;
  if (lo.ld == hi.ld || lo.rows == 1 || hi.rows == 1) {
    const size_t ld = lo.rows > 1 ? lo.ld : hi.ld, at = off % ld;
    return at < lo.width || ld - at < hi.width;
  }
  const Span &few = lo.rows < hi.rows ? lo : hi, &many = &few == &lo ? hi : lo;
  const int64_t first = &few == &hi ? (int64_t)off : -(int64_t)off;  // of few, from many's
  const int64_t ld = (int64_t)few.ld, width = (int64_t)few.width, ld2 = (int64_t)many.ld;
  const int64_t end = (many.rows - 1) * ld2 + (int64_t)many.width;
  for (int64_t r = first < 0 ? -first / ld : 0; r < few.rows && first + r * ld < end; ++r) {
    const int64_t at = first + r * ld;
    if (at + width <= 0) continue;
    // many's last row that begins before this one ends
    const int64_t k = std::min((at + width - 1) / ld2, many.rows - 1);
    if (k * ld2 + (int64_t)many.width > at) return true;
  }
  return false;
}
// A workspace (or other dense range) and the rows of an element of e bytes.
bool overlap(const void* ws, size_t bytes, const Span& x, size_t e) {
  return overlap(Span{ws, bytes, bytes, 1}, Span{x.p, x.ld * e, x.width * e, x.rows}, 1);
}

// A dense range of a call's memory.  An output may be an input where both are rows of
// the same size that the call reads before it writes them.
struct Range {
  const char* name;
  const void* p;
  size_t bytes;
  bool out, same;
};
template <size_t N>
pb_status check_apart(const Range (&r)[N]) {
  for (size_t i = 0; i < N; ++i)
    for (size_t j = 0; j < i; ++j) {
      const Range &a = r[i], &b = r[j];
      if (!a.p || !b.p || !(a.out || b.out)) continue;
      if (a.p == b.p && a.same && b.same && !(a.out && b.out)) continue;
      const uintptr_t pa = (uintptr_t)a.p, pb = (uintptr_t)b.p;
      if (pa < pb + b.bytes && pb < pa + a.bytes)
        return fail(PB_ERR_INVALID_ARG, "%s and %s overlap", a.name, b.name);
    }
  return PB_OK;
}

// A call without any element: as finish_launches(), but no HIP call is made.
pb_status nothing_to_do() {
  pb::clear_error();
  return PB_OK;
}

#define PB_CHECK(expr)                      \
  do {                                      \
    const pb_status st_ = (expr);           \
    if (st_ != PB_OK) return st_;           \
  } while (0)

// ------------------------------------------------------- rotary positions
pb_status check_rope(const pb_rope_config* c) {
  if (!c) return fail(PB_ERR_INVALID_ARG, "cfg is NULL");
  if (!known(c->dtype)) return fail(PB_ERR_INVALID_ARG, "unknown dtype %d", (int)c->dtype);
  if (c->head_dim < 2 || c->head_dim % 2)
    return fail(PB_ERR_INVALID_ARG, "head_dim=%d must be even and >= 2", c->head_dim);
  if (c->head_dim > pb::kRopeMaxDim)
    return fail(PB_ERR_UNSUPPORTED, "head_dim=%d > %d", c->head_dim, pb::kRopeMaxDim);
  if (c->rot_dim < 2 || c->rot_dim % 2 || c->rot_dim > c->head_dim)
    return fail(PB_ERR_INVALID_ARG, "rot_dim=%d must be even, in 2..head_dim=%d", c->rot_dim,
                c->head_dim);
  if (c->interleaved != 0 && c->interleaved != 1)
    return fail(PB_ERR_INVALID_ARG, "interleaved must be 0 or 1");
  if (!(c->base > 0.0) || !std::isfinite(c->base))
    return fail(PB_ERR_INVALID_ARG, "base must be finite and > 0");
  if (!((float)c->magnitude > 0.f) || !std::isfinite((float)c->magnitude))
    return fail(PB_ERR_INVALID_ARG, "magnitude must be finite and > 0 in fp32");
  if (c->scaling < PB_ROPE_PLAIN || c->scaling > PB_ROPE_BY_PARTS)
    return fail(PB_ERR_INVALID_ARG, "scaling=%d", c->scaling);
  if (c->scaling != PB_ROPE_PLAIN && (!(c->factor > 0.0) || !std::isfinite(c->factor)))
    return fail(PB_ERR_INVALID_ARG, "factor must be finite and > 0");
  if (c->scaling == PB_ROPE_BY_PARTS) {
    if (!(c->orig_len > 0.0) || !std::isfinite(c->orig_len))
      return fail(PB_ERR_INVALID_ARG, "orig_len must be finite and > 0");
    if (!(c->low_turns >= 0.0) || !(c->high_turns > c->low_turns) || !std::isfinite(c->high_turns))
      return fail(PB_ERR_INVALID_ARG, "need 0 <= low_turns < high_turns, finite");
  }
  return PB_OK;
}

pb_status rope(const pb_rope_config* c, int n, const pb_rope_tensor* x, int64_t tokens,
               int64_t seq, const int64_t* positions, bool backward, hipStream_t stream) {
  PB_CHECK(check_rope(c));
  if (n < 1 || n > PB_ROPE_MAX_TENSORS)
    return fail(PB_ERR_INVALID_ARG, "n_tensors=%d must be in 1..%d", n, PB_ROPE_MAX_TENSORS);
  if (!x) return fail(PB_ERR_INVALID_ARG, "tensors is NULL");
  if (tokens < 0) return fail(PB_ERR_INVALID_ARG, "tokens=%lld", (long long)tokens);
  if (tokens >= kMaxBlocks)
    return fail(PB_ERR_UNSUPPORTED, "tokens=%lld >= 2^24", (long long)tokens);
  if (!positions && tokens > 0 && seq < 1) return fail(PB_ERR_INVALID_ARG, "seq must be >= 1");
  PB_CHECK(check_opt(positions, 8, "positions"));
  static_assert(PB_ROPE_MAX_TENSORS == pb::kRopeMaxTensors, "tensor limit");
  static_assert(sizeof(int64_t) == sizeof(long long), "positions");
  pb::RopeArgs a{};
  const size_t e = size_of(c->dtype);
  for (int i = 0; i < n; ++i) {
    if (x[i].heads < 1) return fail(PB_ERR_INVALID_ARG, "tensor %d: heads=%d", i, x[i].heads);
    if (x[i].heads > 8192)
      return fail(PB_ERR_UNSUPPORTED, "tensor %d: heads=%d > 8192", i, x[i].heads);
    const size_t width = (size_t)x[i].heads * c->head_dim;
    if (x[i].ld_in < width || x[i].ld_out < width)
      return fail(PB_ERR_INVALID_ARG, "tensor %d: ld_in=%zu, ld_out=%zu < heads*head_dim=%zu", i,
                  x[i].ld_in, x[i].ld_out, width);
    if (std::max(x[i].ld_in, x[i].ld_out) > ((size_t)1 << 31))
      return fail(PB_ERR_UNSUPPORTED, "tensor %d: ld over 2^31 elements", i);
    if (tokens > 0) {
      if (!x[i].in || (uintptr_t)x[i].in % e)
        return fail(PB_ERR_INVALID_ARG, "tensor %d: in is NULL or misaligned", i);
      if (!x[i].out || (uintptr_t)x[i].out % e)
        return fail(PB_ERR_INVALID_ARG, "tensor %d: out is NULL or misaligned", i);
    }
    if (x[i].in == x[i].out && x[i].ld_in != x[i].ld_out)
      return fail(PB_ERR_INVALID_ARG, "tensor %d: in place needs ld_out = ld_in", i);
    a.in[i] = x[i].in;
    a.out[i] = x[i].out;
    a.ld_in[i] = (long long)x[i].ld_in;
    a.ld_out[i] = (long long)x[i].ld_out;
    a.heads[i] = x[i].heads;
    a.copy_rest[i] = x[i].in != x[i].out;
  }
  for (int i = 0; i < n; ++i) {
    const Span out{x[i].out, x[i].ld_out, (size_t)x[i].heads * c->head_dim, tokens};
    if (overlap(positions, (size_t)tokens * 8, out, e))
      return fail(PB_ERR_INVALID_ARG, "out of tensor %d overlaps positions", i);
    for (int j = 0; j < n; ++j) {
      const Span in{x[j].in, x[j].ld_in, (size_t)x[j].heads * c->head_dim, tokens};
      const Span out2{x[j].out, x[j].ld_out, (size_t)x[j].heads * c->head_dim, tokens};
      if (i != j && overlap(out, out2, e))
        return fail(PB_ERR_INVALID_ARG, "tensors %d and %d overlap in out", i, j);
      if (!(i == j && x[i].in == x[i].out) && overlap(out, in, e))
        return fail(PB_ERR_INVALID_ARG, "out of tensor %d overlaps in of tensor %d", i, j);
    }
  }
  a.n = n;
  a.head_dim = c->head_dim;
  a.rot_dim = c->rot_dim;
  a.backward = backward;
  a.magnitude = (float)c->magnitude;
  a.tokens = tokens;
  a.seq = positions ? 1 : std::min<int64_t>(seq, kMaxInt);
  a.pos = (const long long*)positions;
  const double two_pi = 6.283185307179586476925286766559;
  for (int i = 0; i < c->rot_dim / 2; ++i) {
    double f = pow(c->base, -2.0 * i / c->rot_dim);
    if (c->scaling == PB_ROPE_LINEAR) f /= c->factor;
    if (c->scaling == PB_ROPE_BY_PARTS) {
      const double g = std::min(1.0, std::max(0.0, (c->orig_len * f / two_pi - c->low_turns) /
                                                       (c->high_turns - c->low_turns)));
      f *= g + (1.0 - g) / c->factor;
    }
    if (!std::isfinite(f))
      return fail(PB_ERR_INVALID_ARG, "the frequency of pair %d is not finite", i);
    a.turns[i] = f / two_pi;
  }
  if (tokens == 0) return nothing_to_do();
  pb::launch_rope(dt_of(c->dtype), a, c->interleaved != 0, stream);
  return finish_launches();
}

// ------------------------------------------------- root-mean-square norm
pb_status check_rms(const pb_rmsnorm_config* c) {
  if (!c) return fail(PB_ERR_INVALID_ARG, "cfg is NULL");
  if (!known(c->dtype)) return fail(PB_ERR_INVALID_ARG, "unknown dtype %d", (int)c->dtype);
  if (c->rows < 0 || c->cols < 1)
    return fail(PB_ERR_INVALID_ARG, "rows=%lld must be >= 0, cols=%d >= 1", (long long)c->rows,
                c->cols);
  if (c->rows > kMaxInt) return fail(PB_ERR_UNSUPPORTED, "rows=%lld > 2^31 - 1", (long long)c->rows);
  if (c->cols > 32768)
    return fail(PB_ERR_UNSUPPORTED, "cols=%d > 32768 (a row is kept in registers)", c->cols);
  if (c->group != 0 && c->group != 32 && c->group != 64 && c->group != 128)
    return fail(PB_ERR_INVALID_ARG, "group=%d must be 0, 32, 64 or 128", c->group);
  if (!(c->eps >= 0.f) || !std::isfinite(c->eps))
    return fail(PB_ERR_INVALID_ARG, "eps must be finite and >= 0");
  return PB_OK;
}

// ------------------------------------------------------------- Muon step
static_assert(PB_MUON_MAX_TENSORS == pb::kNsMaxTensors, "tensor limit");

// Workspace: partial sums, norms, each matrix's planes, the products' K-slices.
struct NsLayout {
  size_t partial, norm, part;  // offsets
  size_t total;
};

int pad(int v) { return (v + pb::kNsPad - 1) / pb::kNsPad * pb::kNsPad; }

pb_status ns_sizes(int i, int rows, int cols) {
  if (rows < 0 || cols < 0)
    return fail(PB_ERR_INVALID_ARG, "tensor %d: rows=%d, cols=%d", i, rows, cols);
  if (std::min(rows, cols) > 65536 || std::max(rows, cols) > (1 << 20))
    return fail(PB_ERR_UNSUPPORTED, "tensor %d: %d x %d is over 65536 x 2^20", i, rows, cols);
  return PB_OK;
}

// Fills the sizes of t.mat[i] (an empty matrix is left out); false: too many tiles.
bool ns_add(pb::NsTable& t, int rows, int cols) {
  pb::NsMat& x = t.mat[t.count];
  x.rows = rows;
  x.cols = cols;
  x.m = pad(std::min(rows, cols));
  x.n = pad(std::max(rows, cols));
  // rows an odd number of 64 values apart: rows a power of two apart lie in few of the
  // L2's channels (five steps of 2048 x 2048 in fp32 849 us, so 816; 2048 x 8192 in one
  // plane 827 and 792; 256 x 1024 the same)
  x.ldm = x.m | pb::kNsPad;
  x.ldn = x.n | pb::kNsPad;
  const long long tiles =
      t.tile0[t.count] + (long long)(pad(rows) / pb::kNsPad) * (pad(cols) / pb::kNsPad);
  t.tile0[++t.count] = (int)std::min(tiles, kMaxBlocks);
  return tiles < kMaxBlocks;
}

// Plans the products, and places the planes of every matrix from base on (nullptr: sizes
// alone).  lend: the symmetric matrix that is dead before X is replaced lies in the X that
// replaces it (for matrices held in bf16, whose workspace is then 6 values an element of a
// square matrix instead of 8; fp32 calls keep it apart).
NsLayout ns_layout(pb::NsTable& t, bool f32_products, bool lend, char* base, pb::NsChains* c) {
  NsLayout L{};
  if (t.count == 0) return L;
  pb::ns_plan(t, f32_products, c);
  L.norm = align256((size_t)t.tile0[t.count] * sizeof(double));
  size_t o = L.norm + align256((size_t)t.count * sizeof(double));
  for (int i = 0, chain = 0; i < t.count; ++i) {
    pb::NsMat& x = t.mat[i];
    while (i >= c->end[chain]) ++chain;
    const int planes = c->planes[chain];
    const size_t big = align256((size_t)planes * x.m * x.ldn * 2);
    const size_t small = align256((size_t)planes * x.m * x.ldm * 2);
    x.x[0] = (_Float16*)(base + o);
    x.x[1] = (_Float16*)(base + o + big);
    o += 2 * big;
    const int n = pb::ns_symmetric(c->p[chain]), lent = lend ? pb::ns_lent(c->p[chain]) : -1;
    for (int k = 0; k < n; ++k) {
      x.s[k] = k == lent ? nullptr : (_Float16*)(base + o);
      if (k != lent) o += small;
    }
  }
  L.part = o;
  L.total = o + align256(c->partial_floats * sizeof(float));
  return L;
}

pb_status check_count(int n, const void* tensors) {
  if (n < 1 || n > PB_MUON_MAX_TENSORS)
    return fail(PB_ERR_INVALID_ARG, "n_tensors=%d must be in 1..%d", n, PB_MUON_MAX_TENSORS);
  if (!tensors) return fail(PB_ERR_INVALID_ARG, "tensors is NULL");
  return PB_OK;
}

// The table of a call's matrices without their pointers into the workspace.
template <typename X>
pb_status ns_table(int n, const X* x, pb::NsTable& t) {
  PB_CHECK(check_count(n, x));
  for (int i = 0; i < n; ++i) {
    PB_CHECK(ns_sizes(i, x[i].rows, x[i].cols));
    if (x[i].rows == 0 || x[i].cols == 0) continue;
    if (!ns_add(t, x[i].rows, x[i].cols))
      return fail(PB_ERR_UNSUPPORTED, "too many elements in one call");
  }
  return PB_OK;
}

pb_status check_steps(int steps, float eps) {
  if (steps < 1 || steps > 16) return fail(PB_ERR_INVALID_ARG, "steps=%d must be in 1..16", steps);
  if (!(eps > 0.f) || !std::isfinite(eps))
    return fail(PB_ERR_INVALID_ARG, "eps=%g must be positive and finite", (double)eps);
  return PB_OK;
}

pb_status ns_launch(pb::NsTable& t, const pb::NsScalars& sc, pb::NsMode mode,
                    bool f32_products, pb::Dt copy_dt, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (t.count == 0) return nothing_to_do();
  pb::NsChains c;
  const NsLayout L = ns_layout(t, f32_products, mode == pb::NsMode::Bf16, (char*)ws, &c);
  PB_CHECK(check_ws(ws, ws_bytes, L.total));
  for (int i = 0; i < t.count; ++i) {
    const pb::NsMat& x = t.mat[i];
    const size_t e = mode == pb::NsMode::Bf16 ? 2 : 4, e_copy = copy_dt == pb::Dt::BF16 ? 2 : 4;
    auto span = [&](const void* p, long long ld) {
      return Span{p, (size_t)ld, (size_t)x.cols, x.rows};
    };
    if (overlap(ws, L.total, span(x.src, x.ld_src), e) ||
        overlap(ws, L.total, span(x.out, x.ld_out), e) ||
        overlap(ws, L.total, span(x.w, x.ld_src), 4) ||
        overlap(ws, L.total, span(x.mom, x.ld_src), 4) ||
        overlap(ws, L.total, span(x.copy, x.ld_src), e_copy))
      return fail(PB_ERR_INVALID_ARG, "ws overlaps a tensor");
  }
  char* w = (char*)ws;
  pb::launch_newton_schulz(t, sc, mode, copy_dt, c, (double*)(w + L.partial),
                           (double*)(w + L.norm), (float*)(w + L.part), stream);
  return finish_launches();
}

// The bytes that the table's call needs.
size_t ns_bytes(pb::NsTable& t, bool f32_products, bool lend) {
  pb::NsChains c;
  return ns_layout(t, f32_products, lend, nullptr, &c).total;
}

}  // namespace

extern "C" {

pb_status pblock_rope_forward(const pb_rope_config* cfg, int n_tensors,
                              const pb_rope_tensor* tensors, int64_t tokens, int64_t seq,
                              const int64_t* positions, hipStream_t stream) {
  return rope(cfg, n_tensors, tensors, tokens, seq, positions, false, stream);
}

pb_status pblock_rope_backward(const pb_rope_config* cfg, int n_tensors,
                               const pb_rope_tensor* tensors, int64_t tokens, int64_t seq,
                               const int64_t* positions, hipStream_t stream) {
  return rope(cfg, n_tensors, tensors, tokens, seq, positions, true, stream);
}

pb_status pblock_rmsnorm_forward(const pb_rmsnorm_config* cfg, const void* x, const void* resid,
                                 const void* gamma, void* sum, void* y, uint8_t* q8, float* scales,
                                 float* rstd, hipStream_t stream) {
  PB_CHECK(check_rms(cfg));
  const size_t e = size_of(cfg->dtype);
  if (cfg->rows > 0) {
    PB_CHECK(check_ptr(x, e, "x"));
    PB_CHECK(check_opt(resid, e, "resid"));
    PB_CHECK(check_opt(sum, e, "sum"));
    PB_CHECK(check_opt(y, e, "y"));
    PB_CHECK(check_opt(scales, 4, "scales"));
    PB_CHECK(check_opt(rstd, 4, "rstd"));
    if (!y && !q8) return fail(PB_ERR_INVALID_ARG, "y and q8 are both NULL");
    if (!q8 != !scales) return fail(PB_ERR_INVALID_ARG, "q8 and scales come together");
    if (sum && !resid) return fail(PB_ERR_INVALID_ARG, "sum without resid");
  }
  PB_CHECK(check_ptr(gamma, e, "gamma"));
  if (cfg->rows == 0) return nothing_to_do();
  const size_t n = (size_t)cfg->rows * cfg->cols, rows = (size_t)cfg->rows * 4;
  const int groups = cfg->group ? (cfg->cols + cfg->group - 1) / cfg->group : 1;
  const Range ranges[] = {
      {"x", x, n * e, false, true},     {"resid", resid, n * e, false, true},
      {"sum", sum, n * e, true, true},  {"y", y, n * e, true, true},
      {"q8", q8, n, true, false},       {"scales", scales, rows * groups, true, false},
      {"rstd", rstd, rows, true, false}, {"gamma", gamma, cfg->cols * e, false, false}};
  PB_CHECK(check_apart(ranges));
  pb::RmsForward a{};
  a.x = x;
  a.resid = resid;
  a.gamma = gamma;
  a.sum = sum;
  a.y = y;
  a.q8 = q8;
  a.scales = scales;
  a.rstd = rstd;
  a.rows = cfg->rows;
  a.cols = cfg->cols;
  a.group = cfg->group;
  a.eps = cfg->eps;
  pb::launch_rms_forward(dt_of(cfg->dtype), a, stream);
  return finish_launches();
}

size_t pblock_rmsnorm_workspace_bytes(const pb_rmsnorm_config* cfg) {
  if (check_rms(cfg) != PB_OK) return 0;
  return align256((size_t)pb::rms_backward_parts(cfg->rows, cfg->cols) *
                  pb::rms_part_ld(cfg->cols) * sizeof(float));
}

pb_status pblock_rmsnorm_backward(const pb_rmsnorm_config* cfg, const void* s, const void* gamma,
                                  const float* rstd, const void* dy, const void* dsum, void* dx,
                                  float* dgamma, void* ws, size_t ws_bytes, hipStream_t stream) {
  PB_CHECK(check_rms(cfg));
  const size_t e = size_of(cfg->dtype);
  if (cfg->rows > 0) {
    PB_CHECK(check_ptr(s, e, "s"));
    PB_CHECK(check_ptr(rstd, 4, "rstd"));
    PB_CHECK(check_ptr(dy, e, "dy"));
    PB_CHECK(check_opt(dsum, e, "dsum"));
    PB_CHECK(check_ptr(dx, e, "dx"));
  }
  PB_CHECK(check_ptr(gamma, e, "gamma"));
  PB_CHECK(check_ptr(dgamma, 4, "dgamma"));
  const size_t need = pblock_rmsnorm_workspace_bytes(cfg);
  PB_CHECK(check_ws(ws, ws_bytes, need));
  const size_t n = (size_t)cfg->rows * cfg->cols;
  const Range ranges[] = {{"s", s, n * e, false, true},
                          {"dy", dy, n * e, false, true},
                          {"dsum", dsum, n * e, false, true},
                          {"dx", dx, n * e, true, true},
                          {"gamma", gamma, cfg->cols * e, false, false},
                          {"rstd", rstd, (size_t)cfg->rows * 4, false, false},
                          {"dgamma", dgamma, (size_t)cfg->cols * 4, true, false},
                          {"ws", ws, need, true, false}};
  PB_CHECK(check_apart(ranges));
  pb::RmsBackward a{};
  a.s = s;
  a.gamma = gamma;
  a.dy = dy;
  a.dsum = dsum;
  a.rstd = rstd;
  a.dx = dx;
  a.dgamma = dgamma;
  a.part = (float*)ws;
  a.rows = cfg->rows;
  a.cols = cfg->cols;
  pb::launch_rms_backward(dt_of(cfg->dtype), a, stream);
  return finish_launches();
}

size_t pblock_muon_workspace_bytes(const pb_muon_config* cfg, int n_tensors,
                                   const pb_muon_tensor* tensors) {
  pb::NsTable t{};
  if (!cfg || !known(cfg->products) || ns_table(n_tensors, tensors, t) != PB_OK) return 0;
  return ns_bytes(t, cfg->products == PB_F32, false);
}

pb_status pblock_muon_step(const pb_muon_config* cfg, int n_tensors, const pb_muon_tensor* tensors,
                           pb_dtype copy_dtype, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!cfg) return fail(PB_ERR_INVALID_ARG, "cfg is NULL");
  if (!std::isfinite(cfg->lr)) return fail(PB_ERR_INVALID_ARG, "lr is not finite");
  if (!(cfg->momentum >= 0.f && cfg->momentum < 1.f))
    return fail(PB_ERR_INVALID_ARG, "momentum=%g must be in [0, 1)", (double)cfg->momentum);
  if (!std::isfinite(cfg->grad_scale)) return fail(PB_ERR_INVALID_ARG, "grad_scale is not finite");
  PB_CHECK(check_steps(cfg->steps, cfg->eps));
  if (cfg->nesterov != 0 && cfg->nesterov != 1)
    return fail(PB_ERR_INVALID_ARG, "nesterov must be 0 or 1");
  if (!known(cfg->products)) return fail(PB_ERR_INVALID_ARG, "products=%d", (int)cfg->products);
  if (!known(copy_dtype)) return fail(PB_ERR_INVALID_ARG, "copy_dtype=%d", (int)copy_dtype);
  pb::NsTable t{};
  PB_CHECK(ns_table(n_tensors, tensors, t));
  int k = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const pb_muon_tensor& x = tensors[i];
    if (!(x.weight_decay >= 0.f) || !std::isfinite(x.weight_decay))
      return fail(PB_ERR_INVALID_ARG, "tensor %d: weight_decay=%g", i, (double)x.weight_decay);
    if (!std::isfinite(x.scale))
      return fail(PB_ERR_INVALID_ARG, "tensor %d: scale=%g", i, (double)x.scale);
    if (x.rows == 0 || x.cols == 0) continue;
    if (x.ld < (size_t)x.cols || x.ld > ((size_t)1 << 31))
      return fail(PB_ERR_INVALID_ARG, "tensor %d: ld=%zu outside cols=%d .. 2^31", i, x.ld, x.cols);
    const char* names[3] = {"param", "grad", "momentum"};
    const void* ptrs[3] = {x.param, x.grad, x.momentum};
    for (int j = 0; j < 3; ++j)
      if (!ptrs[j] || (uintptr_t)ptrs[j] % 4)
        return fail(PB_ERR_INVALID_ARG, "tensor %d: %s is NULL or not 4-byte aligned", i, names[j]);
    if (x.param_copy && (uintptr_t)x.param_copy % size_of(copy_dtype))
      return fail(PB_ERR_INVALID_ARG, "tensor %d: param_copy is misaligned", i);
    pb::NsMat& m = t.mat[k++];
    m.src = x.grad;
    m.mom = x.momentum;
    m.w = x.param;
    m.copy = x.param_copy;
    m.ld_src = m.ld_out = (long long)x.ld;
    m.decay = x.weight_decay;
    m.scale = x.scale;
  }
  const size_t e_copy = size_of(copy_dtype);
  for (int i = 0; i < t.count; ++i)
    for (int j = 0; j < t.count; ++j) {
      const pb::NsMat &x = t.mat[i], &y = t.mat[j];
      auto span = [](const pb::NsMat& v, const void* p) {
        return Span{p, (size_t)v.ld_src, (size_t)v.cols, v.rows};
      };
      if (i < j && (overlap(span(x, x.w), span(y, y.w), 4) ||
                    overlap(span(x, x.mom), span(y, y.mom), 4) ||
                    overlap(span(x, x.copy), span(y, y.copy), e_copy)))
        return fail(PB_ERR_INVALID_ARG, "two tensors overlap in param, momentum or copy");
      if (overlap(span(x, x.w), span(y, y.mom), 4) || overlap(span(x, x.w), span(y, y.src), 4) ||
          overlap(span(x, x.mom), span(y, y.src), 4))
        return fail(PB_ERR_INVALID_ARG, "param, grad and momentum overlap");
      auto bytes = [](Span v, size_t e) { return Span{v.p, v.ld * e, v.width * e, v.rows}; };
      for (const void* p : {(const void*)y.w, (const void*)y.mom, y.src})
        if (overlap(bytes(span(x, x.copy), e_copy), bytes(span(y, p), 4), 1))
          return fail(PB_ERR_INVALID_ARG, "param_copy overlaps a param, grad or momentum");
    }
  pb::NsScalars sc{};
  sc.lr = cfg->lr;
  sc.momentum = cfg->momentum;
  sc.grad_scale = cfg->grad_scale;
  sc.eps = cfg->eps;
  sc.nesterov = cfg->nesterov;
  sc.steps = cfg->steps;
  return ns_launch(t, sc, pb::NsMode::Muon, cfg->products == PB_F32, dt_of(copy_dtype), ws,
                   ws_bytes, stream);
}

size_t pblock_orthogonalize_workspace_bytes(int n_tensors, const pb_ortho_tensor* tensors,
                                            pb_dtype dtype) {
  pb::NsTable t{};
  if (!known(dtype) || ns_table(n_tensors, tensors, t) != PB_OK) return 0;
  return ns_bytes(t, true, dtype == PB_BF16);
}

pb_status pblock_orthogonalize(int n_tensors, const pb_ortho_tensor* tensors, pb_dtype dtype,
                               int steps, float eps, void* ws, size_t ws_bytes,
                               hipStream_t stream) {
  if (!known(dtype)) return fail(PB_ERR_INVALID_ARG, "unknown dtype %d", (int)dtype);
  PB_CHECK(check_steps(steps, eps));
  pb::NsTable t{};
  PB_CHECK(ns_table(n_tensors, tensors, t));
  const size_t e = size_of(dtype);
  int k = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const pb_ortho_tensor& x = tensors[i];
    if (x.rows == 0 || x.cols == 0) continue;
    if (!x.in || (uintptr_t)x.in % e)
      return fail(PB_ERR_INVALID_ARG, "tensor %d: in is NULL or misaligned", i);
    if (!x.out || (uintptr_t)x.out % e)
      return fail(PB_ERR_INVALID_ARG, "tensor %d: out is NULL or misaligned", i);
    for (size_t ld : {x.ld_in, x.ld_out})
      if (ld < (size_t)x.cols || ld > ((size_t)1 << 31))
        return fail(PB_ERR_INVALID_ARG, "tensor %d: ld=%zu outside cols=%d .. 2^31", i, ld, x.cols);
    if (x.in == x.out && x.ld_in != x.ld_out)
      return fail(PB_ERR_INVALID_ARG, "tensor %d: in place needs ld_out = ld_in", i);
    pb::NsMat& m = t.mat[k++];
    m.src = x.in;
    m.out = x.out;
    m.ld_src = (long long)x.ld_in;
    m.ld_out = (long long)x.ld_out;
  }
  for (int i = 0; i < t.count; ++i)
    for (int j = 0; j < t.count; ++j) {
      const pb::NsMat &x = t.mat[i], &y = t.mat[j];
      const Span out{x.out, (size_t)x.ld_out, (size_t)x.cols, x.rows};
      if (i != j && overlap(out, Span{y.out, (size_t)y.ld_out, (size_t)y.cols, y.rows}, e))
        return fail(PB_ERR_INVALID_ARG, "two tensors overlap in out");
      if (!(i == j && x.src == x.out) &&
          overlap(out, Span{y.src, (size_t)y.ld_src, (size_t)y.cols, y.rows}, e))
        return fail(PB_ERR_INVALID_ARG, "an out overlaps an in");
    }
  pb::NsScalars sc{};
  sc.eps = eps;
  sc.steps = steps;
  return ns_launch(t, sc, dtype == PB_F32 ? pb::NsMode::F32 : pb::NsMode::Bf16,
                   true, dt_of(dtype), ws, ws_bytes, stream);
}

}  // extern "C"
