// Host side of include/sketchssm_attention.h: argument checks before any launch,
// and the kernels' argument blocks.
#include "../../../include/sketchssm_attention.h"

#include "../attention.h"
#include "../checks.h"

using namespace skssm;

namespace {

constexpr int64_t kMaxStride = (int64_t)1 << 30;  // rows and strides together stay far inside 63 bits

bool four_bytes(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

int check_io(const char* what, int io) {
  if (io != SKSSM_F32 && io != SKSSM_BF16) return fail(SKSSM_EINVAL, "%s: unknown io_dtype %d", what, io);
  return SKSSM_OK;
}

int check_cache(const char* what, const skssm_cache* c) {
  if (!c) return fail(SKSSM_EINVAL, "%s: cache is NULL", what);
  if (c->dim != 64 && c->dim != 96 && c->dim != 128 && c->dim != 192 && c->dim != 256)
    return fail(SKSSM_EUNSUPPORTED, "%s: heads of %d channels: 64, 96, 128, 192 or 256", what, c->dim);
  if (c->page < 16 || c->page > 1024 || (c->page & (c->page - 1)))
    return fail(SKSSM_EUNSUPPORTED, "%s: pages of %d tokens: a power of two from 16 to 1024", what, c->page);
  if (c->pages < 1 || c->kv_heads < 1) return fail(SKSSM_EINVAL, "%s: %d pages of %d heads", what, c->pages, c->kv_heads);
  if (c->kv_heads > 1 << 16) return fail(SKSSM_EUNSUPPORTED, "%s: %d key heads: at most 65536", what, c->kv_heads);
  if ((int64_t)c->pages * c->kv_heads > (int64_t)1 << 40) return fail(SKSSM_EUNSUPPORTED, "%s: %d pages of %d heads: too many", what, c->pages, c->kv_heads);
  return SKSSM_OK;
}

size_t cache_bytes(const skssm_cache* c) { return (size_t)c->pages * c->kv_heads * (c->page / 16) * (17 * c->dim); }

int check_tokens(const char* what, const skssm_cache* c, const skssm_new_tokens* s) {
  if (!s) return fail(SKSSM_EINVAL, "%s: seq is NULL", what);
  int rc = check_packed(what, s->batch, s->tokens, s->offsets);
  if (rc) return rc;
  if (s->columns < 1 || s->ld_table < s->columns || s->ld_table > kMaxStride)
    return fail(SKSSM_EINVAL, "%s: table of %d columns, rows %lld apart", what, s->columns, (long long)s->ld_table);
  if ((int64_t)s->columns * c->page > kMaxTokens) return fail(SKSSM_EUNSUPPORTED, "%s: %d pages of %d tokens a sequence: at most 2^30 tokens", what, s->columns, c->page);
  if (!s->lengths || !s->table || !c->data) return fail(SKSSM_EINVAL, "%s: the cache's data, lengths and table are required", what);
  if (!four_bytes(s->lengths) || !four_bytes(s->table)) return fail(SKSSM_EALIGN, "%s: lengths or table not aligned", what);
  if (!aligned(c->data)) return fail(SKSSM_EALIGN, "%s: a pointer is not 16-byte aligned", what);
  return SKSSM_OK;
}

int check_rotation(const char* what, const skssm_rotation* r, int dim) {
  if (r->places < 1) return fail(SKSSM_EINVAL, "%s: angles of %d places", what, r->places);
  if (r->rotated < 2 || r->rotated % 2 || r->rotated > dim) return fail(SKSSM_EINVAL, "%s: %d rotated channels of %d: an even number", what, r->rotated, dim);
  if (r->interleaved != 0 && r->interleaved != 1) return fail(SKSSM_EINVAL, "%s: interleaved must be 0 or 1", what);
  if (!aligned(r->angles)) return fail(SKSSM_EALIGN, "%s: a pointer is not 16-byte aligned", what);
  if (!four_bytes(r->positions)) return fail(SKSSM_EALIGN, "%s: positions not aligned", what);
  return SKSSM_OK;
}

// An array [tokens][heads][dim]: its strides, pointer, and bytes from first to last.
int check_heads(const char* what, const char* name, const void* p, int64_t tokens, int64_t heads, int64_t dim, int64_t ld, int64_t head, int e,
                size_t* bytes) {
  if (heads < 1) return fail(SKSSM_EINVAL, "%s: %lld heads of %s", what, (long long)heads, name);
  if (ld > kMaxStride || head > kMaxStride || heads * dim > kMaxStride || heads * head > kMaxStride * 64)
    return fail(SKSSM_EUNSUPPORTED, "%s: strides of %s: at most 2^30", what, name);
  if (head < dim || (head * e) & 15) return fail(head < dim ? SKSSM_EINVAL : SKSSM_EALIGN, "%s: %s head stride %lld for %lld channels", what, name, (long long)head, (long long)dim);
  const int64_t row = (heads - 1) * head + dim;
  int rc = check_stride(what, name, ld, row, e);
  if (rc) return rc;
  if (tokens > 0 && !p) return fail(SKSSM_EINVAL, "%s: %s is required", what, name);
  if (!aligned(p)) return fail(SKSSM_EALIGN, "%s: a pointer is not 16-byte aligned", what);
  *bytes = span(tokens, ld, row, e);
  return SKSSM_OK;
}

// Whether arrays of T rows share a byte: rows of a and b bytes, lda and ldb bytes apart.  Rows that lie the same distance
// apart may lie between one another (the parts of a projection's output).
bool rows_overlap(const void* p, int64_t a, int64_t lda, const void* q, int64_t b, int64_t ldb, int64_t T) {
  if (T < 1 || !overlap(p, (size_t)((T - 1) * lda + a), q, (size_t)((T - 1) * ldb + b))) return false;
  if (lda != ldb || T == 1) return true;
  int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(q) - reinterpret_cast<uintptr_t>(p)) % lda;
  if (d < 0) d += lda;
  return d < a || d + b > lda;
}

Cache cache_of(const skssm_cache* c) {
  Cache o;
  o.data = static_cast<uint8_t*>(c->data);
  o.pages = c->pages;
  o.heads = c->kv_heads;
  o.shift = __builtin_ctz((unsigned)c->page >> 4);
  return o;
}

NewTokens tokens_of(const skssm_new_tokens* s) {
  NewTokens o;
  o.seq = sequences(s->batch, s->tokens, s->offsets);
  o.lengths = s->lengths;
  o.table = s->table;
  o.ld_table = (size_t)s->ld_table;
  o.columns = s->columns;
  return o;
}

Rotation rotation_of(const skssm_rotation* r) {
  Rotation o{};
  if (r && r->angles) o = {r->angles, r->positions, r->places, r->rotated, r->interleaved};
  return o;
}

size_t table_bytes(const skssm_new_tokens* s) { return span(s->batch, s->ld_table, s->columns, 4); }

}  // namespace

extern "C" {

size_t sketchssm_cache_bytes(const skssm_cache* cache) {
  return check_cache("sketchssm_cache_bytes", cache) ? 0 : cache_bytes(cache);
}

int sketchssm_rotary(int32_t io_dtype, int64_t tokens, int32_t heads, int32_t dim, const skssm_rotation* rotation, const void* x, int64_t ldx,
                     int64_t x_head, void* y, int64_t ldy, int64_t y_head, void* stream) {
  const char* what = "sketchssm_rotary";
  int rc;
  if ((rc = check_io(what, io_dtype)) || (rc = check_packed(what, 1, tokens, nullptr))) return rc;
  if (!rotation || !rotation->angles) return fail(SKSSM_EINVAL, "%s: the angles are required", what);
  if (dim < 8 || dim % 8 || dim > 512) return fail(SKSSM_EUNSUPPORTED, "%s: heads of %d channels: a multiple of 8 up to 512", what, dim);
  if ((rc = check_rotation(what, rotation, dim))) return rc;
  const int e = elem(io_dtype);
  size_t nx, ny;
  if ((rc = check_heads(what, "x", x, tokens, heads, dim, ldx, x_head, e, &nx)) || (rc = check_heads(what, "y", y, tokens, heads, dim, ldy, y_head, e, &ny)))
    return rc;
  const Range out[] = {{y, ny}};
  const Range in[] = {{rotation->angles, (size_t)rotation->places * rotation->rotated * 4}, {rotation->positions, (size_t)tokens * 4}};
  const bool same = x == y && ldx == ldy && x_head == y_head;
  const int64_t xr = ((heads - 1) * x_head + dim) * e, yr = ((heads - 1) * y_head + dim) * e;
  if (any_overlap(out, in) || (!same && rows_overlap(x, xr, ldx * e, y, yr, ldy * e, tokens))) return fail(SKSSM_EINVAL, "%s: y overlaps an input", what);
  if (tokens == 0) return fail(SKSSM_OK, "%s", "");  // nothing to do: no launch, no error
  CacheAppendArgs a{};
  a.tok.seq = sequences(1, tokens, nullptr);
  a.rot = rotation_of(rotation);
  a.H = heads;
  a.D = dim;
  a.q = x;
  a.ldq = (size_t)ldx;
  a.q_head = (size_t)x_head;
  a.y = y;
  a.ldy = (size_t)ldy;
  a.y_head = (size_t)y_head;
  return launched(run_append(a, io_dtype, stream), what);
}

int sketchssm_cache_append(const skssm_cache* cache, const skssm_new_tokens* seq, const skssm_rotation* rotation, const skssm_append_args* args,
                           void* stream) {
  const char* what = "sketchssm_cache_append";
  int rc;
  if ((rc = check_cache(what, cache)) || (rc = check_tokens(what, cache, seq))) return rc;
  if (!args) return fail(SKSSM_EINVAL, "%s: args is NULL", what);
  const skssm_append_args& p = *args;
  if ((rc = check_io(what, p.io_dtype))) return rc;
  const bool turns = rotation && rotation->angles;
  if (turns && (rc = check_rotation(what, rotation, cache->dim))) return rc;
  if (p.q && !turns) return fail(SKSSM_EINVAL, "%s: q without angles", what);
  if (p.q && !p.q_out) return fail(SKSSM_EINVAL, "%s: q_out is required with q", what);
  const int e = elem(p.io_dtype);
  const int64_t T = seq->tokens, D = cache->dim;
  size_t nk, nv, nq = 0, ny = 0;
  if ((rc = check_heads(what, "k", p.k, T, cache->kv_heads, D, p.ldk, p.k_head, e, &nk)) ||
      (rc = check_heads(what, "v", p.v, T, cache->kv_heads, D, p.ldv, p.v_head, e, &nv)))
    return rc;
  if (p.q && ((rc = check_heads(what, "q", p.q, T, p.heads, D, p.ldq, p.q_head, e, &nq)) ||
              (rc = check_heads(what, "q_out", p.q_out, T, p.heads, D, p.ld_qout, p.qout_head, e, &ny))))
    return rc;
  const Range out[] = {{cache->data, cache_bytes(cache)}, {p.q_out, ny}};
  const Range in[] = {{seq->offsets, ((size_t)seq->batch + 1) * 4}, {seq->lengths, (size_t)seq->batch * 4},
                      {seq->table, table_bytes(seq)}, {turns ? rotation->angles : nullptr, turns ? (size_t)rotation->places * rotation->rotated * 4 : 0},
                      {turns ? rotation->positions : nullptr, (size_t)T * 4}};
  const bool same = p.q == p.q_out && p.ldq == p.ld_qout && p.q_head == p.qout_head;
  const Range held[] = {out[0]};
  const Range rows[] = {{p.k, nk}, {p.v, nv}, {p.q, nq}};
  const int64_t kv = (int64_t)cache->kv_heads - 1, yr = ny ? ((p.heads - 1) * p.qout_head + D) * e : 0, yl = p.ld_qout * e;
  if (any_overlap(out, in) || any_overlap(held, rows) || (ny && rows_overlap(p.q_out, yr, yl, p.k, (kv * p.k_head + D) * e, p.ldk * e, T)) ||
      (ny && rows_overlap(p.q_out, yr, yl, p.v, (kv * p.v_head + D) * e, p.ldv * e, T)) ||
      (ny && !same && rows_overlap(p.q_out, yr, yl, p.q, ((p.heads - 1) * p.q_head + D) * e, p.ldq * e, T)))
    return fail(SKSSM_EINVAL, "%s: an output overlaps an input", what);
  if (ny && overlap(p.q_out, ny, cache->data, out[0].n)) return fail(SKSSM_EINVAL, "%s: the outputs overlap", what);
  if (T == 0) return fail(SKSSM_OK, "%s", "");  // nothing to do: no launch, no error
  CacheAppendArgs a{};
  a.tok = tokens_of(seq);
  a.cache = cache_of(cache);
  a.rot = rotation_of(rotation);
  a.H = p.q ? p.heads : 0;
  a.D = (int)D;
  a.q = p.q;
  a.ldq = (size_t)p.ldq;
  a.q_head = (size_t)p.q_head;
  a.y = p.q_out;
  a.ldy = (size_t)p.ld_qout;
  a.y_head = (size_t)p.qout_head;
  a.k = p.k;
  a.ldk = (size_t)p.ldk;
  a.k_head = (size_t)p.k_head;
  a.v = p.v;
  a.ldv = (size_t)p.ldv;
  a.v_head = (size_t)p.v_head;
  return launched(run_append(a, p.io_dtype, stream), what);
}

int sketchssm_cache_read(const skssm_cache* cache, const skssm_new_tokens* seq, int32_t io_dtype, void* k, void* v, void* stream) {
  const char* what = "sketchssm_cache_read";
  int rc;
  if ((rc = check_cache(what, cache)) || (rc = check_tokens(what, cache, seq)) || (rc = check_io(what, io_dtype))) return rc;
  if (!aligned(k) || !aligned(v)) return fail(SKSSM_EALIGN, "%s: a pointer is not 16-byte aligned", what);
  const size_t n = (size_t)seq->tokens * cache->kv_heads * cache->dim * elem(io_dtype);
  const Range out[] = {{k, k ? n : 0}, {v, v ? n : 0}};
  const Range in[] = {{cache->data, cache_bytes(cache)}, {seq->offsets, ((size_t)seq->batch + 1) * 4}, {seq->lengths, (size_t)seq->batch * 4},
                      {seq->table, table_bytes(seq)}};
  if (any_overlap(out, in)) return fail(SKSSM_EINVAL, "%s: an output overlaps an input", what);
  if (out[0].n && out[1].n && overlap(k, n, v, n)) return fail(SKSSM_EINVAL, "%s: the outputs overlap", what);
  if (seq->tokens == 0 || (!k && !v)) return fail(SKSSM_OK, "%s", "");  // nothing to do: no launch, no error
  ReadArgs a{};
  a.tok = tokens_of(seq);
  a.cache = cache_of(cache);
  a.D = cache->dim;
  a.k = k;
  a.v = v;
  return launched(run_cache_read(a, io_dtype, stream), what);
}

size_t sketchssm_attention_workspace(const skssm_cache* cache, int32_t heads, int32_t batch, int64_t tokens, int32_t columns) {
  if (check_cache("sketchssm_attention_workspace", cache) || heads < 1 || heads % cache->kv_heads || batch < 1 || tokens < 1 ||
      tokens > kMaxTokens || (tokens + 1) * heads > (int64_t)1 << 30 || columns < 1 || (int64_t)columns * cache->page > kMaxTokens)
    return 0;
  return attention_workspace(batch, (int)tokens, heads, cache->kv_heads, cache->dim, columns, cache->page);
}

int sketchssm_attention(const skssm_cache* cache, const skssm_new_tokens* seq, const skssm_attention_args* args, void* stream) {
  const char* what = "sketchssm_attention";
  int rc;
  if ((rc = check_cache(what, cache)) || (rc = check_tokens(what, cache, seq))) return rc;
  if (!args) return fail(SKSSM_EINVAL, "%s: args is NULL", what);
  const skssm_attention_args& p = *args;
  if ((rc = check_io(what, p.io_dtype))) return rc;
  if (p.out_dtype != p.io_dtype && p.out_dtype != SKSSM_E4M3)
    return fail(SKSSM_EINVAL, "%s: out_dtype %d is neither the io dtype nor E4M3", what, p.out_dtype);
  const bool fp8 = p.out_dtype == SKSSM_E4M3;
  if ((seq->tokens + 1) * (int64_t)p.heads > (int64_t)1 << 30) return fail(SKSSM_EUNSUPPORTED, "%s: %lld tokens of %d heads: at most 2^30 rows", what, (long long)seq->tokens, p.heads);
  if (p.heads < 1 || p.heads % cache->kv_heads) return fail(SKSSM_EINVAL, "%s: %d key heads do not divide %d heads", what, cache->kv_heads, p.heads);
  if (!(p.scale >= 0x1p-96f && p.scale <= 0x1p96f)) return fail(SKSSM_EINVAL, "%s: scale %g outside 2^-96..2^96", what, (double)p.scale);
  const int64_t T = seq->tokens, D = cache->dim, H = p.heads;
  if (fp8 && D % 128 && (D != 64 || (H / cache->kv_heads) % 2))
    return fail(SKSSM_EUNSUPPORTED, "%s: E4M3 with %lld channels and %lld heads a key head: blocks of 128 columns lie in one key head's", what, (long long)D,
                (long long)(H / cache->kv_heads));
  const int e = elem(p.io_dtype), eo = elem(p.out_dtype);
  size_t nq;
  if ((rc = check_heads(what, "q", p.q, T, H, D, p.ldq, p.q_head, e, &nq)) || (rc = check_stride(what, "out", p.ld_out, H * D, eo))) return rc;
  if (p.ld_out > kMaxStride) return fail(SKSSM_EUNSUPPORTED, "%s: strides of out: at most 2^30", what);
  if (fp8 && (p.ld_scales < T || p.ld_scales > kMaxStride)) return fail(SKSSM_EINVAL, "%s: scales stride %lld for %lld rows", what, (long long)p.ld_scales, (long long)T);
  if (T > 0 && (!p.out || (fp8 && !p.scales))) return fail(SKSSM_EINVAL, "%s: out (and scales) are required", what);
  if (!aligned(p.out) || !aligned(p.workspace) || !four_bytes(p.scales)) return fail(SKSSM_EALIGN, "%s: out, scales or workspace not aligned", what);
  const size_t need = sketchssm_attention_workspace(cache, p.heads, seq->batch, T, seq->columns);
  if (need && (!p.workspace || p.workspace_bytes < need))
    return fail(SKSSM_EINVAL, "%s: workspace of %zu bytes, %zu needed", what, p.workspace ? p.workspace_bytes : (size_t)0, need);
  const size_t no = span(T, p.ld_out, H * D, eo), ns = fp8 ? span(H * D / 128, p.ld_scales, T, 4) : 0;
  const Range out[] = {{p.out, no}, {p.scales, ns}, {p.workspace, need}};
  const Range beside[] = {out[1], out[2]};  // out itself may lie between q's rows
  const Range queries[] = {{p.q, nq}};
  const Range in[] = {{cache->data, cache_bytes(cache)}, {seq->offsets, ((size_t)seq->batch + 1) * 4}, {seq->lengths, (size_t)seq->batch * 4},
                      {seq->table, table_bytes(seq)}};
  if (any_overlap(out, in) || any_overlap(beside, queries) ||
      rows_overlap(p.out, H * D * eo, p.ld_out * eo, p.q, ((H - 1) * p.q_head + D) * e, p.ldq * e, T))
    return fail(SKSSM_EINVAL, "%s: an output overlaps an input", what);
  if ((ns && overlap(p.out, no, p.scales, ns)) || (need && (overlap(p.out, no, p.workspace, need) || (ns && overlap(p.scales, ns, p.workspace, need)))))
    return fail(SKSSM_EINVAL, "%s: the outputs overlap", what);
  if (T == 0) return fail(SKSSM_OK, "%s", "");  // nothing to do: no launch, no error
  AttentionArgs a{};
  a.tok = tokens_of(seq);
  a.cache = cache_of(cache);
  a.H = p.heads;
  a.group = p.heads / cache->kv_heads;
  while ((int64_t)1 << a.bits < a.group) ++a.bits;
  a.magic = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << a.bits) - a.group)) / a.group + 1);
  a.scale = p.scale;
  a.q = p.q;
  a.ldq = (size_t)p.ldq;
  a.q_head = (size_t)p.q_head;
  a.out = p.out;
  a.ld_out = (size_t)p.ld_out;
  a.scales = p.scales;
  a.ld_scales = (size_t)p.ld_scales;
  a.work = need ? static_cast<float*>(p.workspace) : nullptr;
  return launched(run_attention(a, (int)D, p.io_dtype, fp8, stream), what);
}

}  // extern "C"
