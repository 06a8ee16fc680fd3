// C entries of the operators between a layer's QKV projection and its output projection: checks of arguments, workspace
// layout, launches.  Nothing is enqueued before every check has passed.
#include "../../include/mslt.h"
#include "common.h"
#include "host.h"

#include <cmath>

using namespace mslt;

static FormHeads heads_of(const mslt_heads* h) { return h ? FormHeads{h->data, h->batch_stride, h->row_stride, h->head_stride} : FormHeads{}; }

// Whether [batch, rows, heads, width] with these strides is addressable; unit: elements every stride has to be a multiple
// of (1: any); out: no element may be reached twice.
static const char* bad_heads(const mslt_heads* h, int batch, int rows, int heads, int width, int esize, bool vectors, bool out) {
  if (!h || !h->data) return "is null";
  long long dim[3] = {batch, rows, heads}, st[3] = {h->batch_stride, h->row_stride, h->head_stride};
  const long long unit = vectors ? 16 / esize : 1;
  if (reinterpret_cast<uintptr_t>(h->data) % (vectors ? 16 : esize)) return "is not aligned";
  for (int i = 0; i < 3; ++i) {
    if (st[i] < 0 || st[i] > (1ll << 40)) return "has a stride outside 0..2^40";
    if (dim[i] > 1 && st[i] % unit) return "has a stride that is no multiple of 16 bytes";
  }
  if (!out) return nullptr;
  // from the closest dimension outwards, each has to step over what the ones inside it cover
  long long extent = width;
  bool done[3] = {dim[0] == 1, dim[1] == 1, dim[2] == 1};
  for (;;) {
    int best = -1;
    for (int i = 0; i < 3; ++i)
      if (!done[i] && (best < 0 || st[i] < st[best])) best = i;
    if (best < 0) return nullptr;
    if (st[best] < extent) return "overlaps itself";
    extent = st[best] * (dim[best] - 1) + extent;
    done[best] = true;
  }
}
#define HEADS_OK(h, rows, heads, vectors, out)                                                              \
  do {                                                                                                      \
    const char* why__ = bad_heads(h, batch, rows, heads, width, precision ? 2 : 4, vectors, out);            \
    if (why__) return fail(MSLT_ERR_ARG, "%s: %s %s", who, #h, why__);                                       \
  } while (0)

// ---- rotary positions, norm of each head --------------------------------------------------------------------------
static int rotary_sizes(const char* who, int precision, int batch, int seq, int q_heads, int k_heads, int width) {
  if (precision != 0 && precision != 1) return fail(MSLT_ERR_ARG, "%s: precision must be 0 or 1", who);
  if (batch < 1 || seq < 1 || q_heads < 1 || k_heads < 0 || width < 1 || width > 256 || q_heads > 16384 || k_heads > 16384 ||
      (long long)batch * seq > (1ll << 30))
    return fail(MSLT_ERR_ARG, "%s: size outside batch, seq, q_heads >= 1, batch * seq <= 2^30, width 1..256, 16384 heads", who);
  return MSLT_OK;
}
// Frequencies in turns per position, as fractions of 2^64.
static int rotary_form(const char* who, const mslt_rotary_form* f, int width, RotaryArgs& a) {
  if (!f) return fail(MSLT_ERR_ARG, "%s: form is null", who);
  const int r = f->rotary_width;
  if (r < 0 || r > width || r % 2) return fail(MSLT_ERR_ARG, "%s: rotary_width %d is odd or outside 0..%d", who, r, width);
  if (f->scaling < 0 || f->scaling > 2) return fail(MSLT_ERR_ARG, "%s: scaling must be 0, 1 or 2", who);
  if (!(f->theta > 1.0) || !std::isfinite(f->theta) || !std::isfinite(f->magnitude))
    return fail(MSLT_ERR_ARG, "%s: theta must be above 1, magnitude finite", who);
  if (f->scaling && (!(f->factor > 0.0) || !std::isfinite(f->factor))) return fail(MSLT_ERR_ARG, "%s: factor must be above 0", who);
  if (f->scaling == 2 && (!(f->original_length > 0.0) || !std::isfinite(f->original_length) || !std::isfinite(f->low_turns) ||
                          !std::isfinite(f->high_turns) || !(f->low_turns < f->high_turns)))
    return fail(MSLT_ERR_ARG, "%s: scaling 2 needs original_length > 0 and low_turns < high_turns", who);
  a.pairs = r / 2;
  a.interleaved = f->interleaved != 0;
  a.magnitude = f->magnitude;
  // theta^(-2i/r) as products of one ratio: r/2 factors, each rounding 2^-64 of the value
  const long double turns = 0.159154943091895335768883763372514362L;      // 1 / 2pi
  const long double ratio = r ? powl((long double)f->theta, -2.0L / r) : 1.0L;
  long double freq = 1.0L;
  for (int i = 0; i < a.pairs; ++i, freq *= ratio) {
    long double x = freq;
    if (f->scaling == 1) x = freq / f->factor;
    if (f->scaling == 2) {
      long double t = ((long double)f->original_length * freq * turns - f->low_turns) / ((long double)f->high_turns - f->low_turns);
      t = t < 0.0L ? 0.0L : t > 1.0L ? 1.0L : t;
      x = freq * (t + (1.0L - t) / f->factor);
    }
    x *= turns;
    if (x >= 1.0L) x -= floorl(x);          // whole turns per position turn nothing
    const long double units = x * 18446744073709551616.0L + 0.5L;
    a.freq[i] = units >= 18446744073709551616.0L ? 0ull : (unsigned long long)units;
  }
  return MSLT_OK;
}
static int run_rotary(void* stream, int precision, const RotaryArgs& a, bool backward) {
  HIP_TRY(rotary_run(precision, a, backward, reinterpret_cast<hipStream_t>(stream)));
  return MSLT_OK;
}

extern "C" int mslt_rotary(void* hip_stream, int precision, int batch, int seq, int q_heads, int k_heads, int width, const mslt_heads* q,
                           const mslt_heads* k, const int32_t* positions, const mslt_rotary_form* form, int inverse,
                           const mslt_heads* q_out, const mslt_heads* k_out) {
  const char* who = "rotary";
  if (!k) k_heads = 0;
  int rc = rotary_sizes(who, precision, batch, seq, q_heads, k_heads, width);
  if (rc) return rc;
  if (k && k_heads < 1) return fail(MSLT_ERR_ARG, "%s: k without heads", who);
  HEADS_OK(q, seq, q_heads, false, false);
  HEADS_OK(q_out, seq, q_heads, false, true);
  if (k) {
    HEADS_OK(k, seq, k_heads, false, false);
    HEADS_OK(k_out, seq, k_heads, false, true);
  }
  RotaryArgs a;
  if ((rc = rotary_form(who, form, width, a))) return rc;
  a.q = heads_of(q), a.k = heads_of(k), a.oq = heads_of(q_out), a.ok = heads_of(k ? k_out : nullptr);
  a.positions = positions;
  a.B = batch, a.S = seq, a.hq = q_heads, a.hk = k_heads, a.w = width, a.inverse = inverse != 0;
  return run_rotary(hip_stream, precision, a, false);
}

static int norm_args(const char* who, int precision, int batch, int seq, int q_heads, int k_heads, int width, const mslt_heads* q,
                     const mslt_heads* k, const float* gain_q, const float* gain_k, int gain_per_head, float eps,
                     const int32_t* positions, const mslt_rotary_form* form, RotaryArgs& a) {
  int rc = rotary_sizes(who, precision, batch, seq, q_heads, k_heads, width);
  if (rc) return rc;
  if (k_heads < 1) return fail(MSLT_ERR_ARG, "%s: k without heads", who);
  HEADS_OK(q, seq, q_heads, false, false);
  HEADS_OK(k, seq, k_heads, false, false);
  if (!gain_q || !gain_k) return fail(MSLT_ERR_ARG, "%s: a gain is null", who);
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(MSLT_ERR_ARG, "%s: eps must be 0 or above", who);
  if ((rc = rotary_form(who, form, width, a))) return rc;
  a.q = heads_of(q), a.k = heads_of(k);
  a.gain_q = gain_q, a.gain_k = gain_k, a.per_head = gain_per_head != 0, a.eps = eps;
  a.positions = positions;
  a.B = batch, a.S = seq, a.hq = q_heads, a.hk = k_heads, a.w = width;
  return MSLT_OK;
}

extern "C" int mslt_head_norm_rotary(void* hip_stream, int precision, int batch, int seq, int q_heads, int k_heads, int width,
                                     const mslt_heads* q, const mslt_heads* k, const float* gain_q, const float* gain_k,
                                     int gain_per_head, float eps, const int32_t* positions, const mslt_rotary_form* form,
                                     const mslt_heads* q_out, const mslt_heads* k_out) {
  const char* who = "head_norm_rotary";
  RotaryArgs a;
  int rc = norm_args(who, precision, batch, seq, q_heads, k_heads, width, q, k, gain_q, gain_k, gain_per_head, eps, positions, form, a);
  if (rc) return rc;
  HEADS_OK(q_out, seq, q_heads, false, true);
  HEADS_OK(k_out, seq, k_heads, false, true);
  a.oq = heads_of(q_out), a.ok = heads_of(k_out);
  return run_rotary(hip_stream, precision, a, false);
}

extern "C" int mslt_head_norm_workspace(int batch, int seq, int q_heads, int k_heads, int width, size_t* bytes) {
  if (!bytes) return fail(MSLT_ERR_ARG, "head_norm_workspace: bytes is null");
  int rc = rotary_sizes("head_norm_workspace", 0, batch, seq, q_heads, k_heads, width);
  if (rc) return rc;
  *bytes = rotary_partial_floats((long long)batch * seq, q_heads + k_heads, width) * sizeof(float);
  return MSLT_OK;
}

extern "C" int mslt_head_norm_rotary_backward(void* hip_stream, int precision, int batch, int seq, int q_heads, int k_heads, int width,
                                              const mslt_heads* q, const mslt_heads* k, const float* gain_q, const float* gain_k,
                                              int gain_per_head, float eps, const int32_t* positions, const mslt_rotary_form* form,
                                              const mslt_heads* grad_q, const mslt_heads* grad_k, const mslt_heads* dq,
                                              const mslt_heads* dk, float* dgain_q, float* dgain_k, void* workspace,
                                              size_t workspace_bytes) {
  const char* who = "head_norm_rotary_backward";
  RotaryArgs a;
  int rc = norm_args(who, precision, batch, seq, q_heads, k_heads, width, q, k, gain_q, gain_k, gain_per_head, eps, positions, form, a);
  if (rc) return rc;
  HEADS_OK(grad_q, seq, q_heads, false, false);
  HEADS_OK(grad_k, seq, k_heads, false, false);
  HEADS_OK(dq, seq, q_heads, false, true);
  HEADS_OK(dk, seq, k_heads, false, true);
  if (!dgain_q || !dgain_k) return fail(MSLT_ERR_ARG, "%s: a gain's gradient is null", who);
  size_t need = 0;
  if ((rc = mslt_head_norm_workspace(batch, seq, q_heads, k_heads, width, &need))) return rc;
  if (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 16)
    return fail(MSLT_ERR_ARG, "%s: needs a workspace of %zu bytes, 16-byte aligned", who, need);
  a.gq = heads_of(grad_q), a.gk = heads_of(grad_k), a.oq = heads_of(dq), a.ok = heads_of(dk);
  a.dgain_q = dgain_q, a.dgain_k = dgain_k, a.partial = static_cast<float*>(workspace);
  return run_rotary(hip_stream, precision, a, true);
}

// ---- attention ------------------------------------------------------------------------------------------------------
static int attention_sizes(const char* who, int precision, int batch, int queries, int keys, int heads, int kv_heads, int width) {
  if (precision != 0 && precision != 1) return fail(MSLT_ERR_ARG, "%s: precision must be 0 or 1", who);
  if (batch < 1 || queries < 1 || keys < queries || heads < 1 || kv_heads < 1 || heads % kv_heads || width < 1)
    return fail(MSLT_ERR_ARG, "%s: needs 1 <= queries <= keys and heads a multiple of kv_heads", who);
  if (heads / kv_heads > 64) return fail(MSLT_ERR_ARG, "%s: more than 64 heads to a kv head", who);
  if (width > 128 || width % (precision ? 8 : 4)) return fail(MSLT_ERR_ARG, "%s: width must be a multiple of 16 bytes, at most 128", who);
  // positions as fp32, and a grid of fewer than 2^32 threads: two to a row of a head, four to a key of a kv head
  const long long all = (long long)batch * heads;
  if (keys > (1 << 24) || all > (1 << 20) || all * queries > (1ll << 30) || all / heads * kv_heads * keys > (1ll << 29))
    return fail(MSLT_ERR_ARG, "%s: more than 2^24 keys, 2^20 heads, 2^30 queries of all heads or 2^29 keys of all kv heads", who);
  return MSLT_OK;
}
namespace {
struct Workspace {
  size_t ranges, part, part_ml, delta, total;
};
Workspace attention_layout(int precision, int batch, int queries, int keys, int heads, int kv_heads, int width, bool backward, int* splits, int* row_splits) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  Workspace w{};
  const size_t rows = (size_t)batch * heads * queries;
  size_t at = up((size_t)batch * ((keys + 63) / 64) * sizeof(int2));
  *splits = backward ? 1 : form_splits(batch, queries, keys, heads, kv_heads, width);
  if (*splits > 1) {
    w.part = at;
    at += up(rows * *splits * width * sizeof(float));
    w.part_ml = at;
    at += up(rows * *splits * sizeof(float2));
  }
  *row_splits = backward ? form_row_splits(batch, queries, keys, heads, kv_heads, width) : 1;
  if (*row_splits > 1) {
    w.part = at;
    at += up((size_t)2 * *row_splits * batch * kv_heads * keys * width * sizeof(float));
  }
  if (backward) {
    w.delta = at;
    at += up(rows * sizeof(float));
  }
  w.total = at;
  return w;
}
}  // namespace

extern "C" int mslt_attention_workspace(int precision, int batch, int queries, int keys, int heads, int kv_heads, int width, int backward,
                                        size_t* bytes) {
  if (!bytes) return fail(MSLT_ERR_ARG, "attention_workspace: bytes is null");
  int rc = attention_sizes("attention_workspace", precision, batch, queries, keys, heads, kv_heads, width), splits = 1, row_splits = 1;
  if (rc) return rc;
  *bytes = attention_layout(precision, batch, queries, keys, heads, kv_heads, width, backward != 0, &splits, &row_splits).total;
  return MSLT_OK;
}

static int attention_args(const char* who, int precision, int batch, int queries, int keys, int heads, int kv_heads, int width,
                          const mslt_heads* q, const mslt_heads* k, const mslt_heads* v, const mslt_attention_form* f, bool backward,
                          void* workspace, size_t workspace_bytes, FormArgs& a) {
  int rc = attention_sizes(who, precision, batch, queries, keys, heads, kv_heads, width);
  if (rc) return rc;
  HEADS_OK(q, queries, heads, true, false);
  HEADS_OK(k, keys, kv_heads, true, false);
  HEADS_OK(v, keys, kv_heads, true, false);
  // a tile is addressed by 32-bit offsets from its first row
  if (keys > 1 && (k->row_stride > (1 << 22) || v->row_stride > (1 << 22)))
    return fail(MSLT_ERR_ARG, "%s: a row stride of k or v above 2^22 elements", who);
  if (!f) return fail(MSLT_ERR_ARG, "%s: form is null", who);
  // (the kernels divide by the scale, and take (scale / cap)^9 cap)
  if (!(f->scale >= 0x1p-20f && f->scale <= 0x1p20f)) return fail(MSLT_ERR_ARG, "%s: scale must be 2^-20 to 2^20", who);
  if (!(f->cap == 0.f || (f->cap >= f->scale * 0x1p-12f && f->cap <= f->scale * 0x1p24f)))
    return fail(MSLT_ERR_ARG, "%s: cap must be 0, or scale / cap 2^-24 to 2^12", who);
  if (f->prefix && !f->causal) return fail(MSLT_ERR_ARG, "%s: a prefix needs causal", who);
  const Workspace w = attention_layout(precision, batch, queries, keys, heads, kv_heads, width, backward, &a.splits, &a.row_splits);
  if (!workspace || workspace_bytes < w.total || reinterpret_cast<uintptr_t>(workspace) % 16)
    return fail(MSLT_ERR_ARG, "%s: needs a workspace of %zu bytes, 16-byte aligned", who, w.total);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  a.q = heads_of(q), a.k = heads_of(k), a.v = heads_of(v);
  a.docs = f->documents, a.prefix = f->prefix, a.slopes = f->slopes;
  a.ranges = reinterpret_cast<int2*>(ws);
  a.part = reinterpret_cast<float*>(ws + w.part);
  a.part_ml = reinterpret_cast<float2*>(ws + w.part_ml);
  a.delta = reinterpret_cast<float*>(ws + w.delta);
  a.B = batch, a.n = queries, a.S = keys, a.nh = heads, a.nkv = kv_heads, a.w = width;
  a.causal = f->causal != 0, a.scale = f->scale, a.cap = f->cap;
  return MSLT_OK;
}

extern "C" int mslt_attention(void* hip_stream, int precision, int batch, int queries, int keys, int heads, int kv_heads, int width,
                              const mslt_heads* q, const mslt_heads* k, const mslt_heads* v, const mslt_attention_form* form,
                              const mslt_heads* out, float* lse, void* workspace, size_t workspace_bytes) {
  const char* who = "attention";
  FormArgs a;
  int rc = attention_args(who, precision, batch, queries, keys, heads, kv_heads, width, q, k, v, form, false, workspace, workspace_bytes, a);
  if (rc) return rc;
  HEADS_OK(out, queries, heads, true, true);
  if (!lse) return fail(MSLT_ERR_ARG, "%s: lse is null", who);
  a.o = heads_of(out), a.lse = lse;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  HIP_TRY(form_ranges(a, st));
  HIP_TRY(precision ? form_fwd_bf16(a, st) : form_fwd_f32(a, st));
  return MSLT_OK;
}

extern "C" int mslt_attention_backward(void* hip_stream, int precision, int batch, int queries, int keys, int heads, int kv_heads,
                                       int width, const mslt_heads* q, const mslt_heads* k, const mslt_heads* v, const mslt_heads* out,
                                       const float* lse, const mslt_heads* grad_out, const mslt_attention_form* form,
                                       const mslt_heads* dq, const mslt_heads* dk, const mslt_heads* dv, void* workspace,
                                       size_t workspace_bytes) {
  const char* who = "attention_backward";
  FormArgs a;
  int rc = attention_args(who, precision, batch, queries, keys, heads, kv_heads, width, q, k, v, form, true, workspace, workspace_bytes, a);
  if (rc) return rc;
  HEADS_OK(out, queries, heads, true, false);
  HEADS_OK(grad_out, queries, heads, true, false);
  for (const mslt_heads* x : {q, grad_out}) {
    const int group = heads / kv_heads;
    if ((queries > 1 && x->row_stride > (1 << 22)) || (group > 1 && x->head_stride > (1ll << 28) / group))
      return fail(MSLT_ERR_ARG, "%s: q or grad_out: a row stride above 2^22 elements, or heads of a group 2^28 elements apart", who);
  }
  HEADS_OK(dq, queries, heads, true, true);
  HEADS_OK(dk, keys, kv_heads, true, true);
  HEADS_OK(dv, keys, kv_heads, true, true);
  if (!lse) return fail(MSLT_ERR_ARG, "%s: lse is null", who);
  a.o = heads_of(out), a.g = heads_of(grad_out), a.dq = heads_of(dq), a.dk = heads_of(dk), a.dv = heads_of(dv);
  a.lse = const_cast<float*>(lse);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  HIP_TRY(form_ranges(a, st));
  HIP_TRY(precision ? form_bwd_bf16(a, st) : form_bwd_f32(a, st));
  return MSLT_OK;
}
