// C ABI of a search's choice and of the dense state that follows it (see include/shadowkv.h): argument checks, and what the kernels are
// handed.  Nothing here touches the GPU before the arguments have been accepted.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "api.hpp"
#include "kernels.hpp"

using namespace skv;

namespace {

constexpr int64_t kMost = (int64_t)1 << 48;              // bytes that an array may span

int logit_bytes(int dtype) { return dtype == SHADOWKV_LOGITS_FP32 ? 4 : 2; }

int check_logits(const shadowkv_logits* x, int n_out, bool pointers) {
  if (!x) return fail_inval("logits is NULL");
  if (x->dtype != SHADOWKV_LOGITS_BF16 && x->dtype != SHADOWKV_LOGITS_FP16 && x->dtype != SHADOWKV_LOGITS_FP32)
    return fail_inval("logits: dtype must be SHADOWKV_LOGITS_BF16, SHADOWKV_LOGITS_FP16 or SHADOWKV_LOGITS_FP32");
  if (x->n_groups < 0 || x->n_beams < 1 || x->n_beams > 64) return fail_inval("n_groups must be >= 0 and n_beams in [1, 64]");
  if ((int64_t)x->n_groups * x->n_beams > (1 << 20)) return fail_inval("more than 2^20 rows");
  if (x->vocab < 1 || x->vocab > (1 << 30)) return fail_inval("vocab must be in [1, 2^30]");
  if (n_out < 1 || n_out > 64) return fail_inval("n_out must be in [1, 64]");
  if (!pointers || x->n_groups == 0) return SHADOWKV_OK;
  if (!x->data) return fail_inval("logits: data is NULL");
  const int eb = logit_bytes(x->dtype);
  if (reinterpret_cast<uintptr_t>(x->data) % eb) return fail_inval("logits: data must be aligned to its element");
  if ((x->n_groups > 1 && (x->group_stride < 0 || x->group_stride > kMost)) || (x->n_beams > 1 && (x->beam_stride < 0 || x->beam_stride > kMost)))
    return fail_inval("logits: strides must be in [0, 2^48]");
  if (((double)(x->n_groups - 1) * (double)(x->n_groups > 1 ? x->group_stride : 0) + (double)(x->n_beams - 1) * (double)(x->n_beams > 1 ? x->beam_stride : 0)) * eb > (double)kMost)
    return fail_inval("logits: the strides span more than 2^48 bytes");
  return SHADOWKV_OK;
}

struct BeamLayout {
  int part_len, n_parts, n_blocks;
  size_t peaks, offers, total;
};
BeamLayout beam_layout(const shadowkv_logits* x, int n_out) {
  BeamLayout L;
  const int64_t rows = (int64_t)x->n_groups * x->n_beams;
  L.part_len = beam_part_len(rows, x->vocab);
  L.n_parts = (int)(((int64_t)x->vocab + L.part_len - 1) / L.part_len);
  L.n_blocks = beam_blocks(x->vocab);
  L.peaks = up((size_t)rows * L.n_parts * sizeof(BeamPart));
  L.offers = L.peaks + up((size_t)rows * L.n_blocks * sizeof(uint32_t));
  L.total = std::max(L.offers + up((size_t)rows * n_out * sizeof(BeamOffer)), kAlign);
  return L;
}

// The bytes of an array of rows, as nested loops over its pieces with the wider stride outside.
struct Pieces {
  const char* p;
  int64_t st[2], sz[2], inner, last;                     // last: where the last piece begins, from p
  Pieces(const shadowkv_rows& a, int n_rows) : p(static_cast<const char*>(a.data)), inner(a.inner) {
    st[0] = n_rows > 1 ? a.row_stride : 0; sz[0] = n_rows;
    st[1] = a.n_outer > 1 ? a.outer_stride : 0; sz[1] = a.n_outer;
    if (st[1] > st[0]) { std::swap(st[0], st[1]); std::swap(sz[0], sz[1]); }
    last = st[0] * (sz[0] - 1) + st[1] * (sz[1] - 1);
  }
  bool holds(const char* at) const {                     // whether a piece that this finds holds the byte
    int64_t off = at - p;
    if (off < 0 || off >= last + inner) return false;
    for (int i = 0; i < 2; ++i)
      if (st[i] > 0) off -= std::min(off / st[i], sz[i] - 1) * st[i];
    return off < inner;
  }
  bool holds_ends(const Pieces& o) const { return holds(o.p) || holds(o.p + o.inner - 1) || holds(o.p + o.last) || holds(o.p + o.last + o.inner - 1); }
};

}  // namespace

extern "C" {

size_t shadowkv_beam_select_workspace_bytes(const shadowkv_logits* logits, int32_t n_out) {
  return check_logits(logits, n_out, false) == SHADOWKV_OK ? beam_layout(logits, n_out).total : 0;
}

int shadowkv_beam_select(const shadowkv_logits* logits, const float* scores, const uint8_t* finished, const int32_t* lengths, double length_penalty,
                         double logit_scale, int32_t end_token, int32_t n_out, float* out_scores, int32_t* out_parents, int32_t* out_tokens,
                         uint8_t* out_finished, int32_t* out_lengths, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_logits(logits, n_out, true);
  if (rc != SHADOWKV_OK) return rc;
  if (!(std::fabs(length_penalty) <= 16.0)) return fail_inval("length_penalty must be in [-16, 16]");
  const double scale = logit_scale != 0.0 ? logit_scale : 1.0;
  if (!(scale >= FLT_MIN) || !(scale <= FLT_MAX)) return fail_inval("logit_scale must be 0, or positive and a normal number in fp32");
  if (end_token < -1 || end_token >= logits->vocab) return fail_inval("end_token must be in [-1, vocab)");
  if ((length_penalty != 0.0 || out_lengths) && !lengths) return fail_inval("length_penalty and out_lengths need lengths");
  if (logits->n_groups == 0) return SHADOWKV_OK;
  if (!scores || !out_scores || !out_parents || !out_tokens) return fail_inval("scores, out_scores, out_parents and out_tokens must not be NULL");
  const size_t in = (size_t)logits->n_groups * logits->n_beams, out = (size_t)logits->n_groups * n_out;
  const int eb = logit_bytes(logits->dtype);
  const size_t span = ((logits->n_groups > 1 ? (size_t)(logits->n_groups - 1) * logits->group_stride : 0) +
                       (logits->n_beams > 1 ? (size_t)(logits->n_beams - 1) * logits->beam_stride : 0) + logits->vocab) * eb;
  const Bytes ins[4] = {{scores, in * 4}, {finished, in}, {lengths, in * 4}, {logits->data, span}};
  const Bytes outs[6] = {{out_scores, out * 4}, {out_finished, out}, {out_lengths, out * 4}, {out_parents, out * 4}, {out_tokens, out * 4},
                         {workspace, workspace_bytes}};
  for (int i = 0; i < 6; ++i) {
    for (int j = 0; j < 4; ++j)
      if (meet(outs[i], ins[j]) && !(i == j && i < 3 && n_out == logits->n_beams && outs[i].p == ins[j].p))
        return fail_inval("an output or the workspace shares memory with an input");
    for (int j = 0; j < i; ++j)
      if (meet(outs[i], outs[j])) return fail_inval("outputs share memory with each other or the workspace");
  }
  const BeamLayout L = beam_layout(logits, n_out);
  rc = check_workspace(workspace, workspace_bytes, L.total);
  if (rc != SHADOWKV_OK) return rc;
  BeamArgs a{};
  a.logits = static_cast<const uint8_t*>(logits->data);
  a.group_stride = logits->group_stride * eb;
  a.beam_stride = logits->beam_stride * eb;
  a.groups = logits->n_groups; a.beams = logits->n_beams; a.vocab = logits->vocab; a.dtype = logits->dtype; a.n = n_out;
  a.part_len = L.part_len; a.n_parts = L.n_parts;
  a.scale = scale; a.penalty = length_penalty;
  a.range = beam_range(scale);
  a.scores = scores; a.finished = finished; a.lengths = lengths;
  a.end_token = end_token;
  a.out_scores = out_scores; a.out_parents = out_parents; a.out_tokens = out_tokens; a.out_finished = out_finished; a.out_lengths = out_lengths;
  a.parts = static_cast<BeamPart*>(workspace);
  a.n_blocks = L.n_blocks;
  a.peaks = reinterpret_cast<uint32_t*>(static_cast<char*>(workspace) + L.peaks);
  a.offers = reinterpret_cast<BeamOffer*>(static_cast<char*>(workspace) + L.offers);
  const hipError_t e = launch_beam_select(a, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? SHADOWKV_OK : fail_hip("beam select", e);
}

int shadowkv_reorder_rows(const shadowkv_rows* arrays, int32_t n_arrays, const int32_t* parents, int32_t n_rows, void* stream) {
  if (n_arrays < 0 || n_arrays > 4096) return fail_inval("n_arrays must be in [0, 4096]");
  if (n_rows < 0 || n_rows > kMaxReorderRows) return fail_inval("n_rows must be in [0, %d]", kMaxReorderRows);
  if (n_arrays && !arrays) return fail_inval("arrays is NULL");
  if (n_arrays && n_rows && !parents) return fail_inval("parents is NULL");
  for (int k = 0; k < n_arrays; ++k) {
    const shadowkv_rows& a = arrays[k];
    if (a.reserved) return fail_inval("reserved must be 0");
    if (a.n_outer < 0 || a.inner < 0 || a.inner > kMost) return fail_inval("array %d: sizes out of range", k);
    if (n_rows == 0 || a.n_outer == 0 || a.inner == 0) continue;
    if (!a.data) return fail_inval("array %d: data is NULL", k);
    if ((n_rows > 1 && (a.row_stride < 0 || a.row_stride > kMost)) || (a.n_outer > 1 && (a.outer_stride < 0 || a.outer_stride > kMost)))
      return fail_inval("array %d: strides must be in [0, 2^48]", k);
    const Pieces p(a, n_rows);
    if ((double)p.st[0] * (double)(p.sz[0] - 1) + (double)p.st[1] * (double)(p.sz[1] - 1) + (double)p.inner > (double)kMost)
      return fail_inval("array %d: the strides span more than 2^48 bytes", k);
    const int64_t low = p.st[1] * (p.sz[1] - 1) + p.inner;   // of all that the narrower stride runs over
    if ((p.sz[1] > 1 && p.st[1] < p.inner) || (p.sz[0] > 1 && p.st[0] < low)) return fail_inval("array %d is written and overlaps itself", k);
    const char* par = reinterpret_cast<const char*>(parents);
    const size_t par_bytes = (size_t)n_rows * sizeof(int32_t);
    if (meet({p.p, (size_t)(p.last + p.inner)}, {par, par_bytes}) && (p.holds(par) || p.holds(par + par_bytes - 1))) return fail_inval("array %d shares memory with parents", k);
    for (int j = 0; j < k; ++j) {
      const shadowkv_rows& b = arrays[j];
      if (b.n_outer == 0 || b.inner == 0) continue;
      const Pieces q(b, n_rows);
      if (p.p < q.p + q.last + q.inner && q.p < p.p + p.last + p.inner && (p.holds_ends(q) || q.holds_ends(p)))
        return fail_inval("arrays %d and %d share memory", j, k);
    }
  }
  for (int k = 0; k < n_arrays;) {
    ReorderArgs g{};
    g.n_rows = n_rows;
    g.parents = parents;
    for (; k < n_arrays && g.n_arrays < kMaxReorderArrays; ++k) {
      const shadowkv_rows& a = arrays[k];
      if (n_rows == 0 || a.n_outer == 0 || a.inner == 0) continue;
      ReorderArray& r = g.a[g.n_arrays++];
      r.p = static_cast<uint8_t*>(a.data);
      r.row = n_rows > 1 ? a.row_stride : 0;
      r.outer = a.n_outer > 1 ? a.outer_stride : 0;
      r.n_outer = a.n_outer;
      const uint64_t bits = reinterpret_cast<uintptr_t>(a.data) | (uint64_t)r.row | (uint64_t)r.outer | (uint64_t)a.inner;
      r.unit = bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 1;
      r.units = a.inner / r.unit;
    }
    if (g.n_arrays == 0) break;
    g.n_wide = (int)(std::stable_partition(g.a, g.a + g.n_arrays, [](const ReorderArray& r) { return r.unit == 16; }) - g.a);
    const hipError_t e = launch_reorder_rows(g, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail_hip("reorder rows", e);
  }
  return SHADOWKV_OK;
}

}  // extern "C"
