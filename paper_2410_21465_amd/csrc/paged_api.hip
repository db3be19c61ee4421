// C ABI of rotary positions and the paged cache (see include/shadowkv.h): argument checks, and what the kernels are handed.
// Nothing here touches the GPU before the arguments have been accepted.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "api.hpp"
#include "kernels.hpp"

using namespace skv;

namespace {

constexpr double kLog2e = 1.4426950408889634074;
constexpr int64_t kMaxSeqTokens = (int64_t)1 << 30;      // of a sequence in the cache
constexpr int64_t kMaxLaunchTokens = (int64_t)1 << 27;   // of a launch with up to 16 threads a token: 2^31 threads

int elem_bytes(int dtype) { return dtype == SHADOWKV_KV_FP8_E5M2 ? 1 : 2; }
bool known_dtype(int dtype) { return dtype == SHADOWKV_KV_BF16 || dtype == SHADOWKV_KV_FP8_E5M2; }
bool known_head_dim(int d) { return d == 64 || d == 96 || d == 128; }

// Strides of dimensions of these sizes, innermost rows of `row` elements: multiples of 16 bytes, and not negative, in all within what can
// be addressed; of an array that is written no two rows may overlap.
int check_strides(const char* name, const int64_t* stride, const int64_t* size, int n, int64_t row, int eb, bool written) {
  int64_t st[3], sz[3];
  int k = 0;
  double span = 0.0;
  for (int i = 0; i < n; ++i) {
    if (size[i] <= 1) continue;
    span += (double)stride[i] * (double)(size[i] - 1);
    if (stride[i] < 0 || stride[i] > ((int64_t)1 << 48) || stride[i] * eb % 16)
      return fail_inval("%s: strides must be multiples of 16 bytes and not negative", name);
    st[k] = stride[i]; sz[k] = size[i]; ++k;
  }
  if (span * eb > 281474976710656.0) return fail_inval("%s: the strides span more than 2^48 bytes", name);
  if (!written) return SHADOWKV_OK;
  for (int i = 1; i < k; ++i)
    for (int j = i; j > 0 && st[j] < st[j - 1]; --j) { std::swap(st[j], st[j - 1]); std::swap(sz[j], sz[j - 1]); }
  int64_t extent = row;
  for (int i = 0; i < k; ++i) {
    if (st[i] < extent) return fail_inval("%s is written and overlaps itself", name);
    extent += st[i] * (sz[i] - 1);
  }
  return SHADOWKV_OK;
}

int check_heads(const char* name, const shadowkv_heads* h, int d, bool written) {
  if (!h) return fail_inval("%s is NULL", name);
  if (h->n_seqs < 0 || h->n_tokens < 0 || h->n_heads < 1 || h->n_heads > 65535) return fail_inval("%s: sizes out of range", name);
  if ((int64_t)h->n_seqs * h->n_tokens > 0x7fffffff) return fail_inval("%s: more than 2^31 - 1 tokens", name);
  if (!known_dtype(h->dtype)) return fail_inval("%s: dtype must be SHADOWKV_KV_BF16 or SHADOWKV_KV_FP8_E5M2", name);
  if (h->n_seqs == 0 || h->n_tokens == 0) return SHADOWKV_OK;
  if (!h->data) return fail_inval("%s: data is NULL", name);
  if (!aligned16(h->data)) return fail_inval("%s: data must be 16-byte aligned", name);
  const int64_t st[3] = {h->seq_stride, h->token_stride, h->head_stride}, sz[3] = {h->n_seqs, h->n_tokens, h->n_heads};
  return check_strides(name, st, sz, 3, d, elem_bytes(h->dtype), written);
}

HeadsArg heads_arg(const shadowkv_heads* h) {
  const int eb = elem_bytes(h->dtype);
  return {static_cast<uint8_t*>(h->data), h->seq_stride * eb, h->token_stride * eb, h->head_stride * eb, eb};
}

// (of equal sizes; the stride of a dimension of one says nothing)
bool same_array(const shadowkv_heads* a, const shadowkv_heads* b) {
  return a->data == b->data && a->dtype == b->dtype && (a->n_seqs <= 1 || a->seq_stride == b->seq_stride) &&
         (a->n_tokens <= 1 || a->token_stride == b->token_stride) && (a->n_heads <= 1 || a->head_stride == b->head_stride);
}

// The bytes of an array of heads, as nested loops over its rows with the widest stride outside.
struct Rows {
  const char* p;
  int64_t st[3], sz[3], row, last;   // last: where the last row begins, from p
  Rows(const shadowkv_heads* h, int d) : p(static_cast<const char*>(h->data)) {
    const int eb = elem_bytes(h->dtype);
    const int64_t s[3] = {h->seq_stride, h->token_stride, h->head_stride}, n[3] = {h->n_seqs, h->n_tokens, h->n_heads};
    row = (int64_t)d * eb;
    last = 0;
    for (int i = 0; i < 3; ++i) { st[i] = n[i] > 1 ? s[i] * eb : 0; sz[i] = n[i]; last += st[i] * (n[i] - 1); }
    for (int i = 1; i < 3; ++i)
      for (int j = i; j > 0 && st[j] > st[j - 1]; --j) { std::swap(st[j], st[j - 1]); std::swap(sz[j], sz[j - 1]); }
  }
  bool holds(const char* at) const {   // whether a row that this finds holds the byte
    int64_t off = at - p;
    if (off < 0 || off >= last + row) return false;
    for (int i = 0; i < 3; ++i)
      if (st[i] > 0) off -= std::min(off / st[i], sz[i] - 1) * st[i];
    return off < row;
  }
  bool holds_ends(const Rows& o) const { return holds(o.p) || holds(o.p + o.row - 1) || holds(o.p + o.last) || holds(o.p + o.last + o.row - 1); }
};
// Whether the first or the last row of one array lies in the other, so that arrays are refused that begin or end inside each other and
// those that only interleave are not.
bool share_memory(const shadowkv_heads* a, const shadowkv_heads* b, int d) {
  const Rows x(a, d), y(b, d);
  return x.p < y.p + y.last + y.row && y.p < x.p + x.last + x.row && (x.holds_ends(y) || y.holds_ends(x));
}
int check_apart(const char* read, const shadowkv_heads* a, const char* written, const shadowkv_heads* b, int d) {
  if (a->n_seqs == 0 || a->n_tokens == 0 || same_array(a, b) || !share_memory(a, b, d)) return SHADOWKV_OK;
  return fail_inval("%s and %s share memory and are laid out differently", read, written);
}

int rope_table(const shadowkv_rope* r, double* w) {   // radians per position
  const int rot = r->rot_dim ? r->rot_dim : r->head_dim, n = rot / 2;
  const double f = r->factor, two_pi = 6.283185307179586476925;
  const double theta = r->scaling == SHADOWKV_ROPE_NTK ? r->theta * std::pow(f, rot / (rot - 2.0)) : r->theta;
  double first = 0.0, last = 0.0;
  if (r->scaling == SHADOWKV_ROPE_YARN) {
    auto index = [&](double turns) { return rot * std::log(r->original_len / (turns * two_pi)) / (2.0 * std::log(r->theta)); };
    first = std::max(std::floor(index(r->high)), 0.0);
    last = std::min(std::ceil(index(r->low)), rot - 1.0);
  }
  for (int i = 0; i < n; ++i) {
    const double plain = std::pow(theta, -2.0 * i / rot);
    double keep = 1.0;
    if (r->scaling == SHADOWKV_ROPE_LINEAR) keep = 0.0;
    if (r->scaling == SHADOWKV_ROPE_BANDS) keep = (r->original_len * plain / two_pi - r->low) / (r->high - r->low);
    if (r->scaling == SHADOWKV_ROPE_YARN) keep = 1.0 - (i - first) / std::max(last - first, 1e-3);
    keep = std::min(1.0, std::max(0.0, keep));
    w[i] = (r->scaling == SHADOWKV_ROPE_PLAIN || r->scaling == SHADOWKV_ROPE_NTK) ? plain : plain * keep + plain / f * (1.0 - keep);
  }
  return n;
}

// w: the frequencies, unless the caller's own replace them
int check_rope(const shadowkv_rope* r, double (&w)[kMaxHalfDim]) {
  if (!r) return fail_inval("rope is NULL");
  if (!known_head_dim(r->head_dim)) return fail_inval("head_dim must be 64, 96 or 128");
  const int rot = r->rot_dim ? r->rot_dim : r->head_dim;
  if (rot < 8 || rot > r->head_dim || rot % 8) return fail_inval("rot_dim must be a multiple of 8 in [8, head_dim]");
  if (r->layout != SHADOWKV_ROPE_HALF && r->layout != SHADOWKV_ROPE_INTERLEAVED)
    return fail_inval("layout must be SHADOWKV_ROPE_HALF or SHADOWKV_ROPE_INTERLEAVED");
  if (r->scaling < SHADOWKV_ROPE_PLAIN || r->scaling > SHADOWKV_ROPE_YARN) return fail_inval("unknown frequency scaling");
  if (r->reserved) return fail_inval("reserved must be 0");
  if (!std::isfinite((float)r->magnitude) || r->magnitude < 0.0) return fail_inval("magnitude must be finite (in fp32) and >= 0");
  if (r->inv_freq) {
    if (r->scaling != SHADOWKV_ROPE_PLAIN) return fail_inval("inv_freq replaces the frequencies: scaling must be SHADOWKV_ROPE_PLAIN");
    return SHADOWKV_OK;
  }
  if (!(r->theta > 0.0) || !std::isfinite(r->theta)) return fail_inval("theta must be finite and > 0");
  if (r->scaling != SHADOWKV_ROPE_PLAIN && (!(r->factor > 0.0) || !std::isfinite(r->factor))) return fail_inval("factor must be finite and > 0");
  if (r->scaling == SHADOWKV_ROPE_BANDS || r->scaling == SHADOWKV_ROPE_YARN) {
    if (r->original_len < 1) return fail_inval("original_len must be >= 1");
    if (!std::isfinite(r->low) || !std::isfinite(r->high) || !(r->low < r->high)) return fail_inval("low and high must be finite, low < high");
  }
  if (r->scaling == SHADOWKV_ROPE_YARN && (!(r->low > 0.0) || !(r->theta > 1.0))) return fail_inval("YARN needs low > 0 and theta > 1");
  const int n = rope_table(r, w);
  for (int i = 0; i < n; ++i)
    if (!std::isfinite(w[i])) return fail_inval("the frequencies are not finite");
  return SHADOWKV_OK;
}

RopeArgs rope_args(const shadowkv_rope* r, const double (&w)[kMaxHalfDim], bool transposed) {
  RopeArgs a{};
  a.d = r->head_dim;
  a.rot = r->rot_dim ? r->rot_dim : r->head_dim;
  a.interleaved = r->layout == SHADOWKV_ROPE_INTERLEAVED;
  const double by_itself = r->scaling == SHADOWKV_ROPE_YARN && r->factor > 1.0 ? 0.1 * std::log(r->factor) + 1.0 : 1.0;
  a.mag = (float)(r->magnitude != 0.0 ? r->magnitude : by_itself);
  a.sign = transposed ? -1.f : 1.f;
  a.inv_freq = r->inv_freq;
  if (!r->inv_freq)
    for (int i = 0; i < a.rot / 2; ++i) a.rev[i] = w[i] / 6.283185307179586476925;
  return a;
}

int check_cache(const shadowkv_paged_cache* c, bool pointers, bool written) {
  if (!c) return fail_inval("cache is NULL");
  if (c->batch < 1 || c->pages_per_seq < 1 || c->n_pages < 1) return fail_inval("batch, pages_per_seq and n_pages must be >= 1");
  if (c->n_kv_heads < 1 || c->n_kv_heads > 65535) return fail_inval("n_kv_heads must be in [1, 65535]");
  if (!known_head_dim(c->head_dim)) return fail_inval("head_dim must be 64, 96 or 128");
  if (c->page_size < 1 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)))
    return fail_inval("page_size must be a power of two in [1, 65536]");
  if ((int64_t)c->pages_per_seq * c->page_size > kMaxSeqTokens) return fail_inval("more than 2^30 tokens a sequence");
  if (!known_dtype(c->kv_dtype)) return fail_inval("kv_dtype must be SHADOWKV_KV_BF16 or SHADOWKV_KV_FP8_E5M2");
  if (c->reserved) return fail_inval("reserved must be 0");
  if (c->table_stride < c->pages_per_seq && c->batch > 1) return fail_inval("table_stride is less than pages_per_seq");
  if (!pointers) return SHADOWKV_OK;
  if (!c->k || !c->v || !c->page_table) return fail_inval("k, v and page_table must not be NULL");
  if (!aligned16(c->k) || !aligned16(c->v)) return fail_inval("k and v must be 16-byte aligned");
  const int eb = elem_bytes(c->kv_dtype);
  const int64_t sz[3] = {c->n_pages, c->n_kv_heads, c->page_size};
  const int64_t ks[3] = {c->k_page_stride, c->k_head_stride, c->k_token_stride}, vs[3] = {c->v_page_stride, c->v_head_stride, c->v_token_stride};
  // (pages of a dense array lie inside each other's strides, so overlap is not looked for; a row has to have room)
  for (const int64_t* st : {ks, vs})
    if ((double)(c->n_pages - 1) * st[0] * eb + (double)(c->page_size - 1) * st[2] * eb >= 68719476736.0)
      return fail_inval("the pages of a head span more than 64 GiB");
  int rc = check_strides("k pages", ks, sz, 3, c->head_dim, eb, false);
  if (rc == SHADOWKV_OK) rc = check_strides("v pages", vs, sz, 3, c->head_dim, eb, false);
  if (rc != SHADOWKV_OK || !written) return rc;
  for (int i = 0; i < 3; ++i)
    if (sz[i] > 1 && (ks[i] < c->head_dim || vs[i] < c->head_dim)) return fail_inval("pages are written and rows of theirs overlap");
  return SHADOWKV_OK;
}

PagesArg pages_arg(void* p, int64_t page, int64_t head, int64_t tok, int eb) { return {static_cast<uint8_t*>(p), page * eb, head * eb, tok * eb}; }
PageTableArg table_arg(const shadowkv_paged_cache* c) {
  int shift = 0;
  while ((1 << shift) < c->page_size) ++shift;
  return {c->page_table, c->table_stride, c->pages_per_seq, c->n_pages, shift};
}

int check_runs(const shadowkv_paged_cache* c, const shadowkv_heads* rows, const int32_t* seq_starts, const int32_t* kv_lens) {
  if (!kv_lens) return fail_inval("kv_lens is NULL");
  if (!seq_starts && rows->n_tokens % c->batch) return fail_inval("seq_starts is NULL and batch does not divide the tokens");
  return SHADOWKV_OK;
}

struct PagedAttnLayout {
  int G, tb, block_rows, n_wg;
  size_t desc, part_acc, part_ml, total;
};
int paged_attn_layout(const shadowkv_paged_cache* c, int hq, int n_tokens, PagedAttnLayout* L) {
  if (hq < 1 || hq % c->n_kv_heads) return fail_inval("the query heads must be a multiple of n_kv_heads");
  L->G = hq / c->n_kv_heads;
  if (L->G > 64) return fail_inval("group size above 64 is not supported");
  if (n_tokens < 0) return fail_inval("n_tokens must be >= 0");
  if (n_tokens > kMaxSeqTokens) return fail_inval("more than 2^30 tokens");   // (block counts are 32 bits wide)
  L->block_rows = paged_attn_block_rows(L->G, ((long)n_tokens + c->batch - 1) / c->batch * L->G);
  L->tb = L->block_rows / L->G;
  L->n_wg = paged_attn_workgroups();
  const size_t rows = (size_t)2 * L->n_wg * L->block_rows;
  size_t off = 0;
  L->desc = off; off += up((size_t)L->n_wg * sizeof(int4));
  L->part_acc = off; off += up(rows * c->head_dim * sizeof(float));
  L->part_ml = off; off += up(rows * sizeof(float2));
  L->total = off;
  return SHADOWKV_OK;
}

int check_pool(const shadowkv_page_pool* p, bool pointers) {
  if (!p) return fail_inval("pool is NULL");
  if (p->batch < 1 || p->batch > kMaxPoolRows) return fail_inval("batch must be in [1, %d]", kMaxPoolRows);
  if (p->pages_per_seq < 1) return fail_inval("pages_per_seq must be >= 1");
  if (p->n_pages < 1 || p->n_pages > (1 << 28)) return fail_inval("n_pages must be in [1, 2^28]");
  if (p->page_size < 1 || p->page_size > 65536 || (p->page_size & (p->page_size - 1)))
    return fail_inval("page_size must be a power of two in [1, 65536]");
  if ((int64_t)p->pages_per_seq * p->page_size > kMaxSeqTokens) return fail_inval("more than 2^30 tokens a sequence");
  if (p->batch > 1 && (p->table_stride < p->pages_per_seq || p->table_stride > ((int64_t)1 << 40)))
    return fail_inval("table_stride must be in [pages_per_seq, 2^40]");
  if (!pointers) return SHADOWKV_OK;
  if (!p->page_table || !p->kv_lens || !p->page_refs) return fail_inval("page_table, kv_lens and page_refs must not be NULL");
  return SHADOWKV_OK;
}

int check_moves(const shadowkv_page_moves* m) {
  if (!m) return fail_inval("moves is NULL");
  if (m->reserved) return fail_inval("reserved must be 0");
  if (m->capacity < 0) return fail_inval("capacity must be >= 0");
  return SHADOWKV_OK;
}

PoolArg pool_arg(const shadowkv_page_pool* p) {
  int shift = 0;
  while ((1 << shift) < p->page_size) ++shift;
  return {p->page_table, p->table_stride, p->kv_lens, p->page_refs, p->batch, p->pages_per_seq, p->n_pages, shift, aligned16(p->page_refs)};
}
MovesArg moves_arg(const shadowkv_page_moves* m) { return {m->src, m->dst, m->rows, m->count, m->capacity}; }

bool overlap(const Bytes* of, int n) {
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < i; ++j)
      if (meet(of[i], of[j])) return true;
  return false;
}

size_t pages_workspace(const shadowkv_page_pool* p) { return kAlign + up((size_t)p->n_pages * sizeof(int32_t)); }

// a cache whose pages alone matter
int check_pages(const shadowkv_paged_cache* c, bool written) {
  if (!c) return fail_inval("a cache is NULL");
  shadowkv_paged_cache bare = *c;
  bare.batch = bare.pages_per_seq = 1;
  bare.page_table = static_cast<const int32_t*>(c->k);
  return check_cache(&bare, true, written);
}
bool same_geometry(const shadowkv_paged_cache* a, const shadowkv_paged_cache* b) {
  return a->k_page_stride == b->k_page_stride && a->k_head_stride == b->k_head_stride && a->k_token_stride == b->k_token_stride &&
         a->v_page_stride == b->v_page_stride && a->v_head_stride == b->v_head_stride && a->v_token_stride == b->v_token_stride &&
         a->n_pages == b->n_pages && a->n_kv_heads == b->n_kv_heads && a->head_dim == b->head_dim && a->page_size == b->page_size &&
         a->kv_dtype == b->kv_dtype;
}

}  // namespace

extern "C" {

size_t shadowkv_pages_workspace_bytes(const shadowkv_page_pool* pool) { return check_pool(pool, false) == SHADOWKV_OK ? pages_workspace(pool) : 0; }

int shadowkv_pages_update(const shadowkv_page_pool* pool, const int32_t* parents, const int32_t* keep_lens, const int32_t* n_new, int32_t n_new_all,
                          const shadowkv_page_moves* moves, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_pool(pool, true);
  if (rc == SHADOWKV_OK) rc = check_moves(moves);
  if (rc != SHADOWKV_OK) return rc;
  if (!moves->src || !moves->dst || !moves->rows || !moves->count) return fail_inval("src, dst, rows and count of moves must not be NULL");
  if (moves->capacity < pool->batch) return fail_inval("moves has room for %d, batch is %d", moves->capacity, pool->batch);
  if (n_new_all < 0) return fail_inval("n_new_all must be >= 0");
  rc = check_workspace(workspace, workspace_bytes, pages_workspace(pool));
  if (rc != SHADOWKV_OK) return rc;
  const size_t b = (size_t)pool->batch * sizeof(int32_t);
  const Bytes ins[3] = {{parents, b}, {keep_lens, b}, {n_new, b}};
  const Bytes outs[8] = {{pool->page_table, ((size_t)(pool->batch - 1) * pool->table_stride + pool->pages_per_seq) * sizeof(int32_t)}, {pool->kv_lens, b},
                         {pool->page_refs, (size_t)pool->n_pages * sizeof(int32_t)}, {workspace, pages_workspace(pool)}, {moves->src, b}, {moves->dst, b},
                         {moves->rows, b}, {moves->count, sizeof(int32_t)}};
  for (const Bytes& o : outs)
    for (const Bytes& i : ins)
      if (meet(o, i)) return fail_inval("parents, keep_lens or n_new share memory with what is written");
  if (overlap(outs, 8)) return fail_inval("the pool, moves and the workspace share memory");
  const hipError_t e = launch_pages_update(pool_arg(pool), parents, keep_lens, n_new, n_new_all, moves_arg(moves),
                                           reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + kAlign), static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SHADOWKV_OK : fail_hip("pages update", e);
}

int shadowkv_pages_compact(const shadowkv_page_pool* pool, int32_t max_moves, const shadowkv_page_moves* moves, int32_t* n_used, void* workspace,
                           size_t workspace_bytes, void* stream) {
  int rc = check_pool(pool, true);
  if (rc == SHADOWKV_OK) rc = check_moves(moves);
  if (rc != SHADOWKV_OK) return rc;
  if (!moves->count || (moves->capacity > 0 && (!moves->src || !moves->dst))) return fail_inval("src, dst and count of moves must not be NULL");
  if (max_moves < 0) return fail_inval("max_moves must be >= 0");
  rc = check_workspace(workspace, workspace_bytes, pages_workspace(pool));
  if (rc != SHADOWKV_OK) return rc;
  const size_t b = (size_t)pool->batch * sizeof(int32_t), c = (size_t)moves->capacity * sizeof(int32_t);
  const Bytes outs[9] = {{pool->page_table, ((size_t)(pool->batch - 1) * pool->table_stride + pool->pages_per_seq) * sizeof(int32_t)}, {pool->kv_lens, b},
                         {pool->page_refs, (size_t)pool->n_pages * sizeof(int32_t)}, {workspace, pages_workspace(pool)}, {moves->src, c}, {moves->dst, c},
                         {moves->rows, c}, {moves->count, sizeof(int32_t)}, {n_used, sizeof(int32_t)}};
  if (overlap(outs, 9)) return fail_inval("the pool, moves, n_used and the workspace share memory");
  int32_t* ws = static_cast<int32_t*>(workspace);
  const hipError_t e = launch_pages_compact(pool_arg(pool), max_moves, moves_arg(moves), n_used, ws + kAlign / sizeof(int32_t), ws,
                                            static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SHADOWKV_OK : fail_hip("pages compact", e);
}

int shadowkv_pages_copy(const shadowkv_paged_cache* const* from, const shadowkv_paged_cache* const* to, int32_t n_layers,
                        const shadowkv_page_moves* moves, void* stream) {
  int rc = check_moves(moves);
  if (rc != SHADOWKV_OK) return rc;
  if (n_layers < 0 || n_layers > 4096) return fail_inval("n_layers must be in [0, 4096]");
  if (n_layers && (!from || !to)) return fail_inval("from and to must not be NULL");
  if (moves->capacity > 0 && (!moves->src || !moves->dst)) return fail_inval("src and dst of moves must not be NULL");
  for (int l = 0; l < n_layers; ++l) {
    rc = check_pages(from[l], false);
    if (rc == SHADOWKV_OK) rc = check_pages(to[l], true);
    if (rc != SHADOWKV_OK) return rc;
    if (from[l]->n_kv_heads != to[l]->n_kv_heads || from[l]->head_dim != to[l]->head_dim || from[l]->page_size != to[l]->page_size ||
        from[l]->kv_dtype != to[l]->kv_dtype)
      return fail_inval("layer %d: the caches differ in heads, page size or type", l);
  }
  if (moves->capacity == 0) return SHADOWKV_OK;
  for (int l = 0; l < n_layers;) {
    const shadowkv_paged_cache *f = from[l], *t = to[l];
    const int eb = elem_bytes(f->kv_dtype);
    PagesCopyArgs a{};
    for (; l < n_layers && a.n_layers < kMaxCopyLayers && same_geometry(from[l], f) && same_geometry(to[l], t); ++l, ++a.n_layers) {
      a.from_k[a.n_layers] = static_cast<const uint8_t*>(from[l]->k);
      a.from_v[a.n_layers] = static_cast<const uint8_t*>(from[l]->v);
      a.to_k[a.n_layers] = static_cast<uint8_t*>(to[l]->k);
      a.to_v[a.n_layers] = static_cast<uint8_t*>(to[l]->v);
    }
    const int64_t st[4][3] = {{f->k_page_stride, f->k_head_stride, f->k_token_stride}, {f->v_page_stride, f->v_head_stride, f->v_token_stride},
                              {t->k_page_stride, t->k_head_stride, t->k_token_stride}, {t->v_page_stride, t->v_head_stride, t->v_token_stride}};
    for (int i = 0; i < 3; ++i) { a.fk[i] = st[0][i] * eb; a.fv[i] = st[1][i] * eb; a.tk[i] = st[2][i] * eb; a.tv[i] = st[3][i] * eb; }
    a.hkv = f->n_kv_heads;
    a.row_bytes = f->head_dim * eb;
    a.page_size = f->page_size;
    a.from_pages = f->n_pages;
    a.to_pages = t->n_pages;
    a.m = moves_arg(moves);
    const hipError_t e = launch_pages_copy(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail_hip("pages copy", e);
  }
  return SHADOWKV_OK;
}

int shadowkv_rope_frequencies(const shadowkv_rope* rope, double* out) {
  double w[kMaxHalfDim];
  const int rc = check_rope(rope, w);
  if (rc != SHADOWKV_OK) return rc;
  if (!out) return fail_inval("out is NULL");
  if (rope->inv_freq) return fail_inval("the frequencies are in inv_freq, on the device");
  std::copy_n(w, (rope->rot_dim ? rope->rot_dim : rope->head_dim) / 2, out);
  return SHADOWKV_OK;
}

int shadowkv_rotate(const shadowkv_rope* rope, const shadowkv_heads* x, const shadowkv_heads* out, const int32_t* positions,
                    const int32_t* pos_offset, int32_t transposed, void* stream) {
  double w[kMaxHalfDim];
  int rc = check_rope(rope, w);
  if (rc == SHADOWKV_OK) rc = check_heads("x", x, rope->head_dim, false);
  if (rc == SHADOWKV_OK) rc = check_heads("out", out, rope->head_dim, true);
  if (rc != SHADOWKV_OK) return rc;
  if (x->n_seqs != out->n_seqs || x->n_tokens != out->n_tokens || x->n_heads != out->n_heads) return fail_inval("x and out differ in size");
  if (positions && pos_offset) return fail_inval("positions and pos_offset exclude each other");
  if ((int64_t)x->n_seqs * x->n_tokens > kMaxLaunchTokens) return fail_inval("more than 2^27 tokens");
  rc = check_apart("x", x, "out", out, rope->head_dim);
  if (rc != SHADOWKV_OK) return rc;
  if (x->n_seqs == 0 || x->n_tokens == 0) return SHADOWKV_OK;
  const hipError_t e = launch_rotate(rope_args(rope, w, transposed != 0), heads_arg(x), heads_arg(out), positions, pos_offset, x->n_seqs, x->n_tokens,
                                     x->n_heads, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SHADOWKV_OK : fail_hip("rotate", e);
}

int shadowkv_paged_append(const shadowkv_paged_cache* cache, const shadowkv_rope* rope, const shadowkv_heads* k, const shadowkv_heads* v,
                          const shadowkv_heads* q, const shadowkv_heads* q_out, const int32_t* seq_starts, const int32_t* kv_lens,
                          const int32_t* pos_offset, void* stream) {
  int rc = check_cache(cache, true, true);
  if (rc != SHADOWKV_OK) return rc;
  const int d = cache->head_dim;
  double w[kMaxHalfDim];
  if (rope) {
    rc = check_rope(rope, w);
    if (rc != SHADOWKV_OK) return rc;
    if (rope->head_dim != d) return fail_inval("rope and cache differ in head_dim");
  }
  if ((q == nullptr) != (q_out == nullptr)) return fail_inval("q and q_out go together");
  if (q && !rope) return fail_inval("q is given without rope");
  rc = check_heads("k", k, d, false);
  if (rc == SHADOWKV_OK) rc = check_heads("v", v, d, false);
  if (rc == SHADOWKV_OK && q) rc = check_heads("q", q, d, false);
  if (rc == SHADOWKV_OK && q) rc = check_heads("q_out", q_out, d, true);
  if (rc != SHADOWKV_OK) return rc;
  if (k->n_seqs != 1 || v->n_seqs != 1 || (q && (q->n_seqs != 1 || q_out->n_seqs != 1))) return fail_inval("k, v, q and q_out are one run of tokens: n_seqs must be 1");
  if (k->n_heads != cache->n_kv_heads || v->n_heads != cache->n_kv_heads) return fail_inval("k and v must have n_kv_heads heads");
  if (k->n_tokens != v->n_tokens || (q && (q->n_tokens != k->n_tokens || q_out->n_tokens != k->n_tokens || q->n_heads != q_out->n_heads)))
    return fail_inval("k, v, q and q_out differ in size");
  if (k->dtype != v->dtype || (k->dtype != SHADOWKV_KV_BF16 && k->dtype != cache->kv_dtype)) return fail_inval("k and v must both be bf16, or both the cache's type");
  if (q && (q->dtype != SHADOWKV_KV_BF16 || q_out->dtype != SHADOWKV_KV_BF16)) return fail_inval("q and q_out must be bf16");
  rc = check_runs(cache, k, seq_starts, kv_lens);
  if (rc != SHADOWKV_OK) return rc;
  if (k->n_tokens > kMaxLaunchTokens) return fail_inval("more than 2^27 tokens");
  if (q) rc = check_apart("q", q, "q_out", q_out, d);
  if (rc != SHADOWKV_OK) return rc;
  if (k->n_tokens == 0) return SHADOWKV_OK;
  const int eb = elem_bytes(cache->kv_dtype);
  RopeArgs ra{};
  if (rope) ra = rope_args(rope, w, false);
  const hipError_t e = launch_paged_append(
      rope ? &ra : nullptr, pages_arg(cache->k, cache->k_page_stride, cache->k_head_stride, cache->k_token_stride, eb),
      pages_arg(cache->v, cache->v_page_stride, cache->v_head_stride, cache->v_token_stride, eb), table_arg(cache), eb, heads_arg(k), heads_arg(v),
      q ? heads_arg(q) : HeadsArg{}, q ? heads_arg(q_out) : HeadsArg{}, d, cache->n_kv_heads, q ? q->n_heads : 0,
      RunsArg{seq_starts, kv_lens, cache->batch, k->n_tokens}, pos_offset, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SHADOWKV_OK : fail_hip("paged append", e);
}

size_t shadowkv_paged_attention_workspace_bytes(const shadowkv_paged_cache* cache, int32_t n_q_heads, int32_t n_tokens) {
  PagedAttnLayout L;
  if (check_cache(cache, false, false) != SHADOWKV_OK || paged_attn_layout(cache, n_q_heads, n_tokens, &L) != SHADOWKV_OK) return 0;
  return L.total;
}

int shadowkv_paged_attention(const shadowkv_paged_cache* cache, const shadowkv_heads* q, const shadowkv_heads* out, float* lse,
                             const int32_t* seq_starts, const int32_t* kv_lens, int32_t causal, double softmax_scale, void* workspace,
                             size_t workspace_bytes, void* stream) {
  int rc = check_cache(cache, true, false);
  if (rc != SHADOWKV_OK) return rc;
  const int d = cache->head_dim;
  rc = check_heads("q", q, d, false);
  if (rc == SHADOWKV_OK) rc = check_heads("out", out, d, true);
  if (rc != SHADOWKV_OK) return rc;
  if (q->n_seqs != 1 || out->n_seqs != 1) return fail_inval("q and out are one run of tokens: n_seqs must be 1");
  if (q->n_tokens != out->n_tokens || q->n_heads != out->n_heads) return fail_inval("q and out differ in size");
  if (q->dtype != SHADOWKV_KV_BF16 || out->dtype != SHADOWKV_KV_BF16) return fail_inval("q and out must be bf16");
  const float scale_log2 = (float)((softmax_scale != 0.0 ? softmax_scale : 1.0 / std::sqrt((double)d)) * kLog2e);
  // (below: no scale at all, and a hidden logit of minus infinity times zero would be NaN)
  if (!(scale_log2 >= FLT_MIN) || !std::isfinite(scale_log2)) return fail_inval("softmax_scale must be 0, or positive and a normal number in fp32 when multiplied by log2(e)");
  rc = check_runs(cache, q, seq_starts, kv_lens);
  if (rc != SHADOWKV_OK) return rc;
  PagedAttnLayout L;
  rc = paged_attn_layout(cache, q->n_heads, q->n_tokens, &L);
  if (rc == SHADOWKV_OK) rc = check_apart("q", q, "out", out, d);
  if (rc == SHADOWKV_OK) rc = check_workspace(workspace, workspace_bytes, L.total);
  if (rc != SHADOWKV_OK) return rc;
  if (q->n_tokens == 0) return SHADOWKV_OK;
  const int eb = elem_bytes(cache->kv_dtype);
  char* ws = static_cast<char*>(workspace);
  PagedAttnArgs a{};
  a.q = heads_arg(q);
  a.out = heads_arg(out);
  a.lse = lse;
  a.kp = pages_arg(cache->k, cache->k_page_stride, cache->k_head_stride, cache->k_token_stride, eb);
  a.vp = pages_arg(cache->v, cache->v_page_stride, cache->v_head_stride, cache->v_token_stride, eb);
  a.pt = table_arg(cache);
  a.runs = RunsArg{seq_starts, kv_lens, cache->batch, q->n_tokens};
  a.hq = q->n_heads; a.hkv = cache->n_kv_heads; a.G = L.G; a.d = d; a.kv_bytes = eb; a.causal = causal != 0;
  a.scale_log2 = scale_log2;
  a.tb = L.tb;
  a.n_wg = L.n_wg;
  // 64 / 128 / 256 / 512 keys, us: a token over 4K keys 19.6 / 18.3 / 19.4 / 22.4, eight sequences of 1K (14/2 heads of 64, 3 tokens) 19.1 / 16.7 /
  // 17.7 / 21.4; with blocks of 128 rows 17 tokens over 600 keys of four sequences 25.9 / 22.5 / 26.2 / 32.0, 64 over 4K 35.0 / 35.0 / 32.6 / 35.8, 512 over
  // 512 32.0 / 33.9 / 31.7 / 37.6; no difference from 256 tokens over 4K keys on
  a.min_share = 128;
  a.desc = reinterpret_cast<int4*>(ws + L.desc);
  a.part_acc = reinterpret_cast<float*>(ws + L.part_acc);
  a.part_ml = reinterpret_cast<float2*>(ws + L.part_ml);
  const hipError_t e = launch_paged_attention(a, L.block_rows, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SHADOWKV_OK : fail_hip("paged attention", e);
}

}  // extern "C"
