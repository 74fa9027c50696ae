// Host side of include/sketchssm_mixer.h: argument checks before any launch,
// and the kernels' argument blocks.
#include "../../../include/sketchssm_mixer.h"

#include "../host.h"
#include "../mixer.h"

using skssm::aligned;
using skssm::fail;
using skssm::launched;
using skssm::overlap;

namespace {

constexpr int64_t kMaxTokens = (int64_t)1 << 30;

int elem(int dtype) { return dtype == SKSSM_F32 ? 4 : dtype == SKSSM_BF16 ? 2 : 1; }

// A row stride in elements of e bytes: at least the row, whole 16-byte pieces.
int check_stride(const char* what, const char* name, int64_t ld, int64_t row, int e) {
  if (ld < row) return fail(SKSSM_EINVAL, "%s: %s stride %lld is less than its row of %lld", what, name, (long long)ld, (long long)row);
  if ((ld * e) & 15) return fail(SKSSM_EALIGN, "%s: %s stride %lld is not a multiple of 16 bytes", what, name, (long long)ld);
  return SKSSM_OK;
}

// Bytes from the first to past the last element of `rows` rows.
size_t span(int64_t rows, int64_t ld, int64_t row, int e) { return rows > 0 ? (size_t)(((rows - 1) * ld + row) * e) : 0; }

// Arrays by address and bytes (NULL or 0 bytes: none); whether one of the first overlaps one of the second.
struct Range { const void* p; size_t n; };
template <size_t N, size_t M> bool any_overlap(const Range (&a)[N], const Range (&b)[M]) {
  for (const Range& x : a)
    for (const Range& y : b)
      if (x.n && y.n && overlap(x.p, x.n, y.p, y.n)) return true;
  return false;
}

int check_packed(const char* what, int batch, int64_t tokens, const int32_t* offsets) {
  if (batch < 1) return fail(SKSSM_EINVAL, "%s: batch must be >= 1", what);
  if (tokens < 0 || tokens > kMaxTokens)
    return fail(tokens < 0 ? SKSSM_EINVAL : SKSSM_EUNSUPPORTED, "%s: %lld tokens: 0 to 2^30", what, (long long)tokens);
  if (!offsets && tokens % batch) return fail(SKSSM_EINVAL, "%s: %lld tokens are not %d equal sequences (offsets is NULL)", what, (long long)tokens, batch);
  if (reinterpret_cast<uintptr_t>(offsets) & 3u) return fail(SKSSM_EALIGN, "%s: offsets not aligned", what);
  return SKSSM_OK;
}

skssm::Sequences sequences(int batch, int64_t tokens, const int32_t* offsets) {
  skssm::Sequences q;
  q.offsets = offsets;
  q.batch = batch;
  q.tokens = (int)tokens;
  q.each = (int)(tokens / batch);
  return q;
}

int check_groups(const char* what, const skssm_config* cfg, int groups) {
  int rc = skssm::check_shape(cfg, false, true);
  if (rc) return rc;
  if (cfg->kind != SKSSM_MAMBA2) return fail(SKSSM_EUNSUPPORTED, "%s: kind %d (SKSSM_MAMBA2 only)", what, cfg->kind);
  if (groups < 1 || cfg->heads % groups) return fail(SKSSM_EINVAL, "%s: %d groups do not divide %d heads", what, groups, cfg->heads);
  return SKSSM_OK;
}

}  // namespace

extern "C" {

int sketchssm_conv(const skssm_conv_config* cfg, int32_t batch, int64_t tokens, const int32_t* offsets, const void* x,
                   int64_t ldx, const float* taps, const float* bias, const void* state_in, void* state_out, void* y,
                   int64_t ldy, void* stream) {
  const char* what = "sketchssm_conv";
  if (!cfg) return fail(SKSSM_EINVAL, "%s: cfg is NULL", what);
  if (cfg->io_dtype != SKSSM_F32 && cfg->io_dtype != SKSSM_BF16) return fail(SKSSM_EINVAL, "%s: unknown io_dtype %d", what, cfg->io_dtype);
  const int e = elem(cfg->io_dtype), C = cfg->channels, w = cfg->width;
  if (C < 1) return fail(SKSSM_EINVAL, "%s: channels must be >= 1", what);
  if ((int64_t)C * e % 16) return fail(SKSSM_EUNSUPPORTED, "%s: %d channels are not a multiple of 16 bytes", what, C);
  if (C > kMaxTokens) return fail(SKSSM_EUNSUPPORTED, "%s: %d channels: at most 2^30", what, C);
  if (w < 2 || w > 4) return fail(SKSSM_EUNSUPPORTED, "%s: width %d outside 2..4", what, w);
  if (cfg->silu != 0 && cfg->silu != 1) return fail(SKSSM_EINVAL, "%s: silu must be 0 or 1", what);
  int rc = check_packed(what, batch, tokens, offsets);
  if (rc) return rc;
  if ((rc = check_stride(what, "x", ldx, C, e)) || (rc = check_stride(what, "y", ldy, C, e))) return rc;
  if (!taps || (tokens > 0 && (!x || !y))) return fail(SKSSM_EINVAL, "%s: x, taps and y are required", what);
  if (!aligned(x) || !aligned(y) || !aligned(taps) || !aligned(bias) || !aligned(state_in) || !aligned(state_out))
    return fail(SKSSM_EALIGN, "%s: a pointer is not 16-byte aligned", what);
  const size_t nx = span(tokens, ldx, C, e), ny = span(tokens, ldy, C, e), ns = (size_t)batch * (w - 1) * C * e;
  if (overlap(y, ny, x, nx) || overlap(y, ny, state_in, ns) || overlap(y, ny, state_out, ns) || overlap(state_out, ns, x, nx))
    return fail(SKSSM_EINVAL, "%s: an output overlaps x or a state", what);
  const Range outs[] = {{y, ny}, {state_out, ns}};
  const Range parameters[] = {{taps, (size_t)C * w * 4}, {bias, (size_t)C * 4}, {offsets, ((size_t)batch + 1) * 4}};
  if (any_overlap(outs, parameters)) return fail(SKSSM_EINVAL, "%s: an output overlaps taps, bias or offsets", what);
  if (state_in != state_out && overlap(state_in, ns, state_out, ns))
    return fail(SKSSM_EINVAL, "%s: the states overlap without being the same", what);
  skssm::ConvArgs a{};
  a.seq = sequences(batch, tokens, offsets);
  a.C = C;
  a.x = x;
  a.ldx = (size_t)ldx;
  a.taps = taps;
  a.bias = bias;
  a.state_in = state_in;
  a.state_out = state_out;
  a.y = y;
  a.ldy = (size_t)ldy;
  return launched(skssm::run_conv(a, w, cfg->io_dtype, cfg->silu, state_out && state_in == state_out, stream), what);
}

int sketchssm_conv_token(const skssm_config* cfg, int32_t groups, int32_t width, const void* x, int64_t ldx,
                         const float* taps, const float* bias, void* state, const void* dt, int64_t lddt,
                         const float* dt_bias, const float* A, const skssm_ring* ring, int32_t n_buffered, void* q,
                         void* stream) {
  const char* what = "sketchssm_conv_token";
  int rc = check_groups(what, cfg, groups);
  if (rc) return rc;
  if (width < 2 || width > 4) return fail(SKSSM_EUNSUPPORTED, "%s: width %d outside 2..4", what, width);
  const int e = elem(cfg->io_dtype);
  const int64_t B = cfg->batch, H = cfg->heads, C = H * cfg->dv + 2 * (int64_t)groups * cfg->dk;
  if (C > kMaxTokens) return fail(SKSSM_EUNSUPPORTED, "%s: %lld channels: at most 2^30", what, (long long)C);
  if (n_buffered < 0 || n_buffered >= cfg->window)
    return fail(SKSSM_ESTATE, "%s: n_buffered %d outside 0..%d", what, n_buffered, cfg->window - 1);
  if (!x || !taps || !state || !dt || !A || !q) return fail(SKSSM_EINVAL, "%s: x, taps, state, dt, A and q are required", what);
  if ((rc = skssm::check_ring(cfg, ring, false, false))) return rc;
  if (!aligned(x) || !aligned(taps) || !aligned(bias) || !aligned(state) || !aligned(q))
    return fail(SKSSM_EALIGN, "%s: a pointer is not 16-byte aligned", what);
  if ((reinterpret_cast<uintptr_t>(dt) % e) || (reinterpret_cast<uintptr_t>(A) & 3u) || (reinterpret_cast<uintptr_t>(dt_bias) & 3u))
    return fail(SKSSM_EALIGN, "%s: dt, dt_bias or A not aligned", what);
  if ((rc = check_stride(what, "x", ldx, C, e))) return rc;
  if (lddt < H) return fail(SKSSM_EINVAL, "%s: dt stride %lld is less than %lld heads", what, (long long)lddt, (long long)H);
  const size_t items = (size_t)B * H, W = (size_t)cfg->window;
  const Range out[6] = {{ring->k, items * W * cfg->dk * e}, {ring->v, items * W * cfg->dv * e},
      {ring->beta, items * W * 4}, {ring->log_decay, items * W * 4}, {q, items * cfg->dk * e}, {state, (size_t)B * (width - 1) * C * e}};
  for (const auto& o : out)
    if (overlap(o.p, o.n, x, span(B, ldx, C, e)) || overlap(o.p, o.n, dt, span(B, lddt, H, e)))
      return fail(SKSSM_EINVAL, "%s: x or dt overlaps what is written", what);
  const Range parameters[] = {{taps, (size_t)C * width * 4}, {bias, (size_t)C * 4}, {dt_bias, (size_t)H * 4}, {A, (size_t)H * 4}};
  if (any_overlap(out, parameters)) return fail(SKSSM_EINVAL, "%s: taps, bias, dt_bias or A overlaps what is written", what);
  for (int i = 0; i < 6; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return fail(SKSSM_EINVAL, "%s: the arrays that are written overlap", what);
  skssm::ConvTokenArgs a{};
  a.B = cfg->batch;
  a.H = cfg->heads;
  a.G = groups;
  a.W = cfg->window;
  a.n = n_buffered;
  a.K = cfg->dk;
  a.V = cfg->dv;
  a.x = x;
  a.ldx = (size_t)ldx;
  a.taps = taps;
  a.bias = bias;
  a.state = state;
  a.dt = dt;
  a.lddt = (size_t)lddt;
  a.dt_bias = dt_bias;
  a.A = A;
  a.rk = const_cast<void*>(ring->k);
  a.rv = const_cast<void*>(ring->v);
  a.rbeta = const_cast<float*>(ring->beta);
  a.rla = const_cast<float*>(ring->log_decay);
  a.q = q;
  return launched(skssm::run_conv_token(a, width, cfg->io_dtype, stream), what);
}

size_t sketchssm_scan_workspace(const skssm_config* cfg, int32_t groups, int64_t tokens) {
  if (check_groups("sketchssm_scan_workspace", cfg, groups) || tokens < 0 || tokens > kMaxTokens) return 0;
  return skssm::scan_workspace(cfg->batch, (int)tokens, cfg->heads, groups, cfg->dk, cfg->dv);
}

int sketchssm_scan(const skssm_config* cfg, int32_t groups, int64_t tokens, const int32_t* offsets, const void* x,
                   int64_t ldx, const void* b, int64_t ldb, const void* c, int64_t ldc, const void* dt, int64_t lddt,
                   const float* dt_bias, const float* A, const float* D, const float* S_in, float* S_out, void* y,
                   int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
  const char* what = "sketchssm_scan";
  int rc = check_groups(what, cfg, groups);
  if (rc) return rc;
  if ((rc = check_packed(what, cfg->batch, tokens, offsets))) return rc;
  const int e = elem(cfg->io_dtype);
  const int64_t HV = (int64_t)cfg->heads * cfg->dv, GK = (int64_t)groups * cfg->dk, H = cfg->heads;
  if (!A || !S_out || (tokens > 0 && (!x || !b || !c || !dt || !y)))
    return fail(SKSSM_EINVAL, "%s: x, b, c, dt, A, S_out and y are required", what);
  if (!aligned(x) || !aligned(b) || !aligned(c) || !aligned(y) || !aligned(S_in) || !aligned(S_out) || !aligned(workspace))
    return fail(SKSSM_EALIGN, "%s: a pointer is not 16-byte aligned", what);
  if ((reinterpret_cast<uintptr_t>(dt) % e) || (reinterpret_cast<uintptr_t>(A) & 3u) || (reinterpret_cast<uintptr_t>(D) & 3u) ||
      (reinterpret_cast<uintptr_t>(dt_bias) & 3u))
    return fail(SKSSM_EALIGN, "%s: dt, dt_bias, A or D not aligned", what);
  if ((rc = check_stride(what, "x", ldx, HV, e)) || (rc = check_stride(what, "b", ldb, GK, e)) ||
      (rc = check_stride(what, "c", ldc, GK, e)) || (rc = check_stride(what, "y", ldy, HV, e)))
    return rc;
  for (const int64_t ld : {ldx, ldb, ldc, ldy})  // 32 rows are reached by 32-bit offsets
    if (ld >= (int64_t)1 << 24) return fail(SKSSM_EUNSUPPORTED, "%s: a row stride of %lld: less than 2^24", what, (long long)ld);
  if (lddt < H) return fail(SKSSM_EINVAL, "%s: dt stride %lld is less than %lld heads", what, (long long)lddt, (long long)H);
  const size_t need = skssm::scan_workspace(cfg->batch, (int)tokens, cfg->heads, groups, cfg->dk, cfg->dv);
  if (need && (!workspace || workspace_bytes < need))
    return fail(SKSSM_EINVAL, "%s: workspace of %zu bytes, %zu needed", what, workspace ? workspace_bytes : (size_t)0, need);
  const size_t states = (size_t)cfg->batch * HV * cfg->dk * 4;
  const Range in[] = {{x, span(tokens, ldx, HV, e)}, {b, span(tokens, ldb, GK, e)}, {c, span(tokens, ldc, GK, e)}, {dt, span(tokens, lddt, H, e)},
      {offsets, ((size_t)cfg->batch + 1) * 4}, {dt_bias, (size_t)H * 4}, {A, (size_t)H * 4}, {D, (size_t)H * 4}};
  const Range out[] = {{y, span(tokens, ldy, HV, e)}, {S_out, states}, {workspace, need}};
  if (any_overlap(out, in)) return fail(SKSSM_EINVAL, "%s: an output overlaps an input", what);
  for (const Range& o : out)
    if (o.p != S_out && overlap(o.p, o.n, S_in, states)) return fail(SKSSM_EINVAL, "%s: an output overlaps S_in", what);
  if (overlap(y, out[0].n, S_out, states) || overlap(workspace, need, S_out, states) || overlap(workspace, need, y, out[0].n))
    return fail(SKSSM_EINVAL, "%s: the outputs overlap", what);
  if (S_in != S_out && overlap(S_in, states, S_out, states))
    return fail(SKSSM_EINVAL, "%s: S_in and S_out overlap without being the same", what);
  skssm::ScanArgs a{};
  a.seq = sequences(cfg->batch, tokens, offsets);
  a.H = cfg->heads;
  a.G = groups;
  a.x = x;
  a.ldx = (size_t)ldx;
  a.b = b;
  a.ldb = (size_t)ldb;
  a.c = c;
  a.ldc = (size_t)ldc;
  a.dt = dt;
  a.lddt = (size_t)lddt;
  a.dt_bias = dt_bias;
  a.A = A;
  a.D = D;
  a.S_in = S_in;
  a.S_out = S_out;
  a.y = y;
  a.ldy = (size_t)ldy;
  a.work = need ? static_cast<float*>(workspace) : nullptr;
  return launched(skssm::run_scan(a, cfg->dk, cfg->dv, cfg->io_dtype, stream), what);
}

int sketchssm_norm(const skssm_norm_args* args, void* stream) {
  const char* what = "sketchssm_norm";
  if (!args) return fail(SKSSM_EINVAL, "%s: args is NULL", what);
  const skssm_norm_args& p = *args;
  if (p.io_dtype != SKSSM_F32 && p.io_dtype != SKSSM_BF16) return fail(SKSSM_EINVAL, "%s: unknown io_dtype %d", what, p.io_dtype);
  if (p.x_dtype != SKSSM_F32 && p.x_dtype != p.io_dtype) return fail(SKSSM_EINVAL, "%s: x_dtype %d is neither F32 nor the io dtype", what, p.x_dtype);
  if (p.out_dtype != p.io_dtype && p.out_dtype != SKSSM_E4M3)
    return fail(SKSSM_EINVAL, "%s: out_dtype %d is neither the io dtype nor E4M3", what, p.out_dtype);
  if (p.rows < 0 || p.columns < 1 || p.group < 1) return fail(SKSSM_EINVAL, "%s: rows, columns and group", what);
  if (p.columns % p.group) return fail(SKSSM_EINVAL, "%s: groups of %d do not divide %d columns", what, p.group, p.columns);
  const bool fp8 = p.out_dtype == SKSSM_E4M3;
  if (p.columns % 8 || p.group % 8) return fail(SKSSM_EUNSUPPORTED, "%s: columns %d and group %d must be multiples of 8", what, p.columns, p.group);
  if (p.group > 32768) return fail(SKSSM_EUNSUPPORTED, "%s: group of %d columns: at most 32768", what, p.group);
  if (fp8 && p.group != p.columns && p.group % 128)
    return fail(SKSSM_EUNSUPPORTED, "%s: a group of %d columns cuts blocks of 128", what, p.group);
  if (p.rows > kMaxTokens) return fail(SKSSM_EUNSUPPORTED, "%s: %lld rows: at most 2^30", what, (long long)p.rows);
  if (!(p.eps >= 0.f)) return fail(SKSSM_EINVAL, "%s: eps must be >= 0", what);
  if (p.residual && p.gate) return fail(SKSSM_EINVAL, "%s: residual and gate exclude each other", what);
  if (p.residual_out && !p.residual) return fail(SKSSM_EINVAL, "%s: residual_out without residual", what);
  if ((p.skip != nullptr) != (p.D != nullptr) || (p.skip && !p.gate)) return fail(SKSSM_EINVAL, "%s: skip goes with D and a gate", what);
  const int ei = elem(p.io_dtype), ex = elem(p.x_dtype), eo = elem(p.out_dtype);
  const int64_t n = p.columns, M = p.rows;
  int rc;
  if ((rc = check_stride(what, "x", p.ldx, n, ex))) return rc;
  if (p.residual && (rc = check_stride(what, "residual", p.ld_residual, n, ei))) return rc;
  if (p.residual_out && (rc = check_stride(what, "residual_out", p.ld_residual_out, n, ei))) return rc;
  if (p.gate && (rc = check_stride(what, "gate", p.ld_gate, n, ei))) return rc;
  int64_t skip_row = 0;
  if (p.skip) {
    if (p.skip_width < 8 || p.skip_width % 8 || n % p.skip_width) return fail(SKSSM_EINVAL, "%s: skip_width %d", what, p.skip_width);
    const int64_t heads = n / p.skip_width;
    if ((rc = check_stride(what, "skip head", p.skip_head, p.skip_width, ei))) return rc;
    skip_row = (heads - 1) * p.skip_head + p.skip_width;
    if ((rc = check_stride(what, "skip", p.ld_skip, skip_row, ei))) return rc;
  }
  if (p.ld_out < n) return fail(SKSSM_EINVAL, "%s: out stride %lld is less than its row", what, (long long)p.ld_out);
  if ((p.ld_out * eo) % (fp8 ? 8 : 16)) return fail(SKSSM_EALIGN, "%s: out stride %lld", what, (long long)p.ld_out);
  const int64_t blocks = (n + 127) / 128;
  if (fp8 && p.ld_scales < M) return fail(SKSSM_EINVAL, "%s: scales stride %lld is less than %lld rows", what, (long long)p.ld_scales, (long long)M);
  if (!p.weight || (M > 0 && (!p.x || !p.out || (fp8 && !p.scales)))) return fail(SKSSM_EINVAL, "%s: x, weight, out (and scales) are required", what);
  if (!aligned(p.x) || !aligned(p.residual) || !aligned(p.residual_out) || !aligned(p.gate) || !aligned(p.skip) || !aligned(p.weight) ||
      !aligned(p.out) || !aligned(p.scales))
    return fail(SKSSM_EALIGN, "%s: a pointer is not 16-byte aligned", what);
  if (reinterpret_cast<uintptr_t>(p.D) & 3u) return fail(SKSSM_EALIGN, "%s: D not aligned", what);
  const struct { const void* p; size_t n; int64_t ld; int dtype; } in[4] = {{p.x, span(M, p.ldx, n, ex), p.ldx, p.x_dtype},
      {p.residual, span(M, p.ld_residual, n, ei), p.ld_residual, p.io_dtype}, {p.gate, span(M, p.ld_gate, n, ei), 0, -1},
      {p.skip, span(M, p.ld_skip, skip_row, ei), 0, -1}};
  const size_t no = span(M, p.ld_out, n, eo), ns = fp8 ? span(blocks, p.ld_scales, M, 4) : 0, nr = span(M, p.ld_residual_out, n, ei);
  for (const auto& x : in) {
    if (overlap(p.out, no, x.p, x.n) || overlap(fp8 ? p.scales : nullptr, ns, x.p, x.n))
      return fail(SKSSM_EINVAL, "%s: an output overlaps an input", what);
    // a lane reads the elements of residual_out's row that it writes, if they lie alike
    const bool same = x.p == p.residual_out && x.ld == p.ld_residual_out && x.dtype == p.io_dtype;
    if (!same && overlap(p.residual_out, nr, x.p, x.n)) return fail(SKSSM_EINVAL, "%s: residual_out overlaps an input", what);
  }
  const Range outs[] = {{p.out, no}, {fp8 ? p.scales : nullptr, ns}, {p.residual_out, nr}};
  const Range parameters[] = {{p.weight, (size_t)n * 4}, {p.D, p.D ? (size_t)(n / p.skip_width) * 4 : 0}};
  if (any_overlap(outs, parameters)) return fail(SKSSM_EINVAL, "%s: an output overlaps weight or D", what);
  if (overlap(p.out, no, p.residual_out, nr) || (fp8 && (overlap(p.out, no, p.scales, ns) || overlap(p.residual_out, nr, p.scales, ns))))
    return fail(SKSSM_EINVAL, "%s: the outputs overlap", what);
  if (M == 0) return fail(SKSSM_OK, "%s", "");  // nothing to do: no launch, no error
  skssm::NormArgs a{};
  a.rows = (int)M;
  a.columns = p.columns;
  a.group = p.group;
  a.skip_width = p.skip_width;
  a.eps = p.eps;
  a.x = p.x;
  a.ldx = (size_t)p.ldx;
  a.residual = p.residual;
  a.ld_residual = (size_t)p.ld_residual;
  a.residual_out = p.residual_out;
  a.ld_residual_out = (size_t)p.ld_residual_out;
  a.gate = p.gate;
  a.ld_gate = (size_t)p.ld_gate;
  a.skip = p.skip;
  a.ld_skip = (size_t)p.ld_skip;
  a.skip_head = (size_t)p.skip_head;
  a.D = p.D;
  a.weight = p.weight;
  a.out = p.out;
  a.ld_out = (size_t)p.ld_out;
  a.scales = p.scales;
  a.ld_scales = (size_t)p.ld_scales;
  return launched(skssm::run_norm(a, p.x_dtype, p.io_dtype, p.out_dtype, stream), what);
}

size_t sketchssm_matmul_fp8_workspace(int64_t M, int32_t N, int32_t K) {
  if (M < 1 || M > kMaxTokens || N < 1 || N > kMaxTokens || K < 1) return 0;
  return skssm::matmul_fp8_workspace((int)M, N, K);
}

int sketchssm_matmul_fp8(int64_t M, int32_t N, int32_t K, const void* a, int64_t lda, const float* a_scale,
                         int64_t ld_ascale, const void* w, int64_t ldw, const float* w_scale, int32_t out_dtype, void* y,
                         int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
  const char* what = "sketchssm_matmul_fp8";
  if (M < 0 || N < 1 || K < 1) return fail(SKSSM_EINVAL, "%s: sizes %lld x %d x %d", what, (long long)M, N, K);
  if (K % 16) return fail(SKSSM_EUNSUPPORTED, "%s: K = %d is not a multiple of 16", what, K);
  if (M > kMaxTokens || N > kMaxTokens) return fail(SKSSM_EUNSUPPORTED, "%s: M = %lld, N = %d: at most 2^30", what, (long long)M, N);
  if (out_dtype != SKSSM_F32 && out_dtype != SKSSM_BF16) return fail(SKSSM_EINVAL, "%s: unknown out_dtype %d", what, out_dtype);
  int rc;
  if ((rc = check_stride(what, "a", lda, K, 1)) || (rc = check_stride(what, "w", ldw, K, 1))) return rc;
  // a tile's rows are stepped through in 32 bits
  if (lda >= 1 << 24 || ldw >= 1 << 24) return fail(SKSSM_EUNSUPPORTED, "%s: row strides must be less than 2^24", what);
  if (ld_ascale < M) return fail(SKSSM_EINVAL, "%s: a_scale stride %lld is less than %lld rows", what, (long long)ld_ascale, (long long)M);
  if (ldy < N) return fail(SKSSM_EINVAL, "%s: y stride %lld is less than %d columns", what, (long long)ldy, N);
  if (!w || !w_scale || (M > 0 && (!a || !a_scale || !y))) return fail(SKSSM_EINVAL, "%s: a, w, their scales and y are required", what);
  if (!aligned(a) || !aligned(w) || !aligned(a_scale) || !aligned(w_scale) || !aligned(y) || !aligned(workspace))
    return fail(SKSSM_EALIGN, "%s: a pointer is not 16-byte aligned", what);
  const size_t need = sketchssm_matmul_fp8_workspace(M, N, K);
  if (need && (!workspace || workspace_bytes < need))
    return fail(SKSSM_EINVAL, "%s: workspace of %zu bytes, %zu needed", what, workspace ? workspace_bytes : (size_t)0, need);
  const int64_t kb = ((int64_t)K + 127) / 128, nb = ((int64_t)N + 127) / 128;
  const size_t ny = span(M, ldy, N, elem(out_dtype));
  const Range in[] = {{a, span(M, lda, K, 1)}, {w, span(N, ldw, K, 1)}, {a_scale, span(kb, ld_ascale, M, 4)}, {w_scale, (size_t)(nb * kb * 4)}};
  const Range out[] = {{y, ny}, {workspace, need}};
  if (any_overlap(out, in)) return fail(SKSSM_EINVAL, "%s: y or workspace overlaps an input", what);
  if (overlap(y, ny, workspace, need)) return fail(SKSSM_EINVAL, "%s: y overlaps workspace", what);
  if (M == 0) return fail(SKSSM_OK, "%s", "");  // nothing to do: no launch, no error
  skssm::MatmulArgs p{};
  p.M = (int)M;
  p.N = N;
  p.K = K;
  p.a = static_cast<const uint8_t*>(a);
  p.lda = (size_t)lda;
  p.sa = a_scale;
  p.ldsa = (size_t)ld_ascale;
  p.w = static_cast<const uint8_t*>(w);
  p.ldw = (size_t)ldw;
  p.sw = w_scale;
  p.y = y;
  p.ldy = (size_t)ldy;
  p.part = need ? static_cast<float*>(workspace) : nullptr;
  return launched(skssm::run_matmul_fp8(p, out_dtype, stream), what);
}

}  // extern "C"
