// extern "C" entry points of the token operators (attention, coupling, dropout, head norms
// with rotation, the loss over a vocabulary, AdamW): argument validation and dispatch.  Nothing here allocates device memory.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <iterator>
#include <limits>
#include <string>
#include <vector>

#include "../../include/petra.h"
#include "ops.h"

namespace petra {
petra_status set_error(petra_status s, const std::string& msg);
}

namespace {

using petra::set_error;

// Errors leave through this: thrown inside an entry point, caught at its end.
struct Refused {
  petra_status status;
  std::string what;
};

void need(bool ok, petra_status s, const char* what) {
  if (!ok) throw Refused{s, what};
}

// Runs an entry point's body, which says whether it enqueued work; nothing it throws
// crosses the C boundary.
template <typename F>
petra_status entry(const char* name, F body) {
  try {
    const hipError_t e = body() ? hipGetLastError() : hipSuccess;
    if (e != hipSuccess) return set_error(PETRA_ERR_HIP, std::string(name) + ": " + hipGetErrorString(e));
    return PETRA_OK;
  } catch (const Refused& r) {
    return set_error(r.status, r.what);
  } catch (...) {
    return set_error(PETRA_ERR_STATE, std::string(name) + ": out of host memory");
  }
}

size_t size_of(int32_t dtype) { return dtype == PETRA_BF16 ? 2 : 4; }

void need_dtype(int32_t dtype) {
  need(dtype == PETRA_FP32 || dtype == PETRA_BF16, PETRA_ERR_DTYPE, "dtype must be fp32 or bf16");
}

// A tensor's pointer: present unless it has no elements, 16-byte aligned.
void need_ptr(const void* p, const char* name, bool empty = false) {
  if (empty) return;
  if (p == nullptr) throw Refused{PETRA_ERR_INVALID_ARG, std::string("null pointer: ") + name};
  if (reinterpret_cast<uintptr_t>(p) & 15u)
    throw Refused{PETRA_ERR_ALIGN, std::string("misaligned pointer: ") + name};
}

void need_int_ptr(const void* p, const char* name, uintptr_t align) {
  if (p != nullptr && (reinterpret_cast<uintptr_t>(p) & (align - 1)))
    throw Refused{PETRA_ERR_ALIGN, std::string("misaligned pointer: ") + name};
}

// A range of memory that a call reads or writes.
struct Span {
  const void* p;
  size_t bytes;
  const char* name;
};

bool overlap(const Span& a, const Span& b) {
  if (a.p == nullptr || b.p == nullptr || a.bytes == 0 || b.bytes == 0) return false;
  const char *x = static_cast<const char*>(a.p), *y = static_cast<const char*>(b.p);
  return x < y + b.bytes && y < x + a.bytes;
}

void need_apart(const Span& a, const Span& b, bool same_allowed = false) {
  if (same_allowed && a.p == b.p) return;
  if (overlap(a, b)) throw Refused{PETRA_ERR_ALIAS, std::string("buffers overlap: ") + a.name + " and " + b.name};
}

// Threshold of the generator's 16 bits, 0 for no dropout.
uint32_t need_dropout(float p, const uint64_t* rng, bool check_rng) {
  need(p >= 0.f && p < 1.f, PETRA_ERR_INVALID_ARG, "dropout probability outside [0, 1)");
  const long cut = std::lround(65536.0 * p);
  need(cut < 65536, PETRA_ERR_INVALID_ARG, "dropout probability keeps nothing");
  if (check_rng && cut > 0) need(rng != nullptr, PETRA_ERR_INVALID_ARG, "dropout without rng");
  need_int_ptr(rng, "rng", 8);
  return static_cast<uint32_t>(cut);
}

float inv_keep(uint32_t cut) { return static_cast<float>(65536.0 / (65536.0 - cut)); }

void need_workspace(const void* w, size_t have, size_t want) {
  if (want == 0) return;
  need(w != nullptr && have >= want, PETRA_ERR_WORKSPACE, "workspace missing or too small");
  need_ptr(w, "workspace");
}

// ---------------------------------------------------------------------------
// attention
// ---------------------------------------------------------------------------

// Strides of [batch][len][heads][dim], contiguous where all three are zero.
void strides(const int64_t in[3], int64_t out[3], int64_t len, int64_t heads, int64_t dim, size_t esz,
             const char* name) {
  const bool dense = in[0] == 0 && in[1] == 0 && in[2] == 0;
  out[0] = dense ? len * heads * dim : in[0];
  out[1] = dense ? heads * dim : in[1];
  out[2] = dense ? dim : in[2];
  for (int i = 0; i < 3; ++i) {
    if (out[i] < 0 || out[i] > (int64_t{1} << 46))
      throw Refused{PETRA_ERR_SHAPE, std::string("negative or too large stride: ") + name};
    if (out[i] * static_cast<int64_t>(esz) % 16 != 0)
      throw Refused{PETRA_ERR_ALIGN, std::string("stride not a multiple of 16 bytes: ") + name};
  }
}

// The bytes from a tensor's first element to its last lie within the address space, so that
// sums of its strides fit 64 bits.
void need_reach(const int64_t st[3], const int64_t n[3], int64_t dim, size_t esz, const char* name) {
  __int128 extent = dim;
  for (int i = 0; i < 3; ++i)
    if (n[i] > 0) extent += static_cast<__int128>(n[i] - 1) * st[i];
  if (extent * static_cast<__int128>(esz) >= __int128{1} << 47)
    throw Refused{PETRA_ERR_SHAPE, std::string("strides reach past the address space: ") + name};
}

// No two elements of a written tensor share memory: by growing stride, each dimension
// steps past what the smaller ones cover.
void need_distinct(const int64_t st[3], const int64_t n[3], int64_t dim, const char* name) {
  if (n[0] == 0 || n[1] == 0 || n[2] == 0) return;
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int a, int b) { return st[a] < st[b]; });
  int64_t extent = dim;
  for (int i : order) {
    if (n[i] <= 1) continue;
    if (st[i] < extent) throw Refused{PETRA_ERR_SHAPE, std::string("elements share memory: ") + name};
    extent += (n[i] - 1) * st[i];
  }
}

// The memory of a strided tensor: runs of `run` bytes, at n[i] positions step[i] bytes apart in
// each of `dims` dimensions, the largest step first.
struct Runs {
  const void* p = nullptr;
  const char* name = "";
  int64_t run = 0, step[3] = {}, n[3] = {};
  int dims = 0;

  Runs() = default;
  Runs(const Span& s) : p(s.p), name(s.name), run(static_cast<int64_t>(s.bytes)) {}
  Runs(const void* at, const int64_t st[3], const int64_t count[3], int64_t dim, size_t esz, const char* what)
      : p(at), name(what), run(dim * static_cast<int64_t>(esz)) {
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int x, int y) { return st[x] > st[y]; });
    for (int i : order) {
      if (count[i] <= 0) run = 0;
      if (count[i] <= 1 || st[i] == 0) continue;   // (positions that share their memory are one)
      step[dims] = st[i] * static_cast<int64_t>(esz);
      n[dims++] = count[i];
    }
    // dimensions without gaps are one, and a run where they reach the channels
    for (int i = dims - 2; i >= 0; --i)
      if (step[i] == n[i + 1] * step[i + 1]) {
        n[i] *= n[i + 1];
        step[i] = step[i + 1];
        for (int j = i + 1; j + 1 < dims; ++j) n[j] = n[j + 1], step[j] = step[j + 1];
        --dims;
      }
    if (dims > 0 && step[dims - 1] == run) run *= n[--dims];
  }
  // Bytes from the first to the last, of the dimensions from d on.
  int64_t extent(int d) const {
    int64_t e = run;
    for (; d < dims; ++d) e += (n[d] - 1) * step[d];
    return e;
  }
};

int64_t div_up(int64_t x, int64_t y) { return x > 0 ? (x + y - 1) / y : -(-x / y); }
int64_t div_down(int64_t x, int64_t y) { return -div_up(-x, y); }

// Whether a's dimensions from da on and b's from db on share a byte, b's first being `off` past a's.
// Slices of one tensor have their steps in common, so that only the difference of two positions
// matters and few are near enough; other pairs go by the positions of the larger step.  `budget`
// bounds the pairs looked at: two tensors woven into each other past it count as sharing.
bool meet(const Runs& a, int da, const Runs& b, int db, int64_t off, int& budget) {
  const int64_t ea = a.extent(da), eb = b.extent(db);
  if (off >= ea || -off >= eb) return false;
  const bool more_a = da < a.dims, more_b = db < b.dims;
  if (!more_a && !more_b) return true;
  if (--budget < 0) return true;
  const int64_t sa = more_a ? a.step[da] : 0, sb = more_b ? b.step[db] : 0, s = std::max(sa, sb);
  const bool in_a = sa == s, in_b = sb == s;
  // off + k s for k = (b's position, where it has this step) - (a's)
  const int64_t first = std::max(in_a ? 1 - a.n[da] : 0, div_up(1 - off - (in_b ? b.extent(db + 1) : eb), s));
  const int64_t last = std::min(in_b ? b.n[db] - 1 : 0, div_down((in_a ? a.extent(da + 1) : ea) - 1 - off, s));
  for (int64_t k = first; k <= last; ++k)
    if (meet(a, da + in_a, b, db + in_b, off + k * s, budget)) return true;
  return false;
}

void need_apart(const Runs& a, const Runs& b) {
  if (a.p == nullptr || b.p == nullptr || a.run == 0 || b.run == 0) return;
  int budget = 1 << 16;
  if (meet(a, 0, b, 0, static_cast<int64_t>(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p)), budget))
    throw Refused{PETRA_ERR_ALIAS, std::string("buffers overlap: ") + a.name + " and " + b.name};
}

struct Attn {
  petra::AttnArgs a{};
  petra::AttnPlan plan{};
  size_t esz;

  bool no_q() const { return a.batch == 0 || a.q_len == 0; }
  bool no_kv() const { return a.batch == 0 || a.kv_len == 0; }

  Attn(const petra_attn_desc* d, const uint64_t* rng, bool call, bool backward) {
    need(d != nullptr, PETRA_ERR_INVALID_ARG, "null description");
    need_dtype(d->dtype);
    esz = size_of(d->dtype);
    need(d->batch >= 0 && d->q_len >= 0 && d->kv_len >= 0, PETRA_ERR_SHAPE, "negative size");
    need(d->heads >= 1 && d->kv_heads >= 1 && d->heads % d->kv_heads == 0, PETRA_ERR_SHAPE,
         "heads must be a positive multiple of kv_heads");
    need(d->head_dim >= 8 && d->head_dim <= 128 && d->head_dim % 8 == 0, PETRA_ERR_SHAPE,
         "head_dim must be a multiple of 8, at most 128");
    need(d->scale > 0.f && std::isfinite(d->scale), PETRA_ERR_INVALID_ARG, "scale must be positive and finite");
    a.batch = d->batch;
    a.q_len = d->q_len;
    a.kv_len = d->kv_len;
    a.heads = d->heads;
    a.kv_heads = d->kv_heads;
    a.group = d->heads / d->kv_heads;
    a.dim = d->head_dim;
    a.causal = d->causal != 0;
    const int64_t most = int64_t{1} << 30;
    need(static_cast<int64_t>(a.q_len) * a.group <= most && a.kv_len <= most, PETRA_ERR_SHAPE, "sequence too long");
    need(static_cast<int64_t>(a.batch) * a.kv_heads <= 65535, PETRA_ERR_SHAPE, "batch * kv_heads above 65535");
    a.scale = d->scale;
    a.scale_log2 = d->scale * 1.44269504088896340736f;
    a.cut = need_dropout(d->dropout, rng, call);
    a.inv_keep = inv_keep(a.cut);
    a.rng = a.cut > 0 ? rng : nullptr;
    strides(d->q_stride, a.q_stride, a.q_len, a.heads, a.dim, esz, "q");
    strides(d->k_stride, a.k_stride, a.kv_len, a.kv_heads, a.dim, esz, "k");
    strides(d->v_stride, a.v_stride, a.kv_len, a.kv_heads, a.dim, esz, "v");
    strides(d->o_stride, a.o_stride, a.q_len, a.heads, a.dim, esz, "o");
    need(a.k_stride[1] < (1 << 22) && a.v_stride[1] < (1 << 22), PETRA_ERR_SHAPE,
         "token stride of k or v of 2^22 elements or more");
    const int64_t nq[3] = {a.batch, a.q_len, a.heads}, nk[3] = {a.batch, a.kv_len, a.kv_heads};
    need_reach(a.q_stride, nq, a.dim, esz, "q");
    need_reach(a.k_stride, nk, a.dim, esz, "k");
    need_reach(a.v_stride, nk, a.dim, esz, "v");
    need_reach(a.o_stride, nq, a.dim, esz, "o");
    // tiles of keys, and in the backward of queries, are addressed by 32-bit offsets from their first row
    need(a.kv_len <= 1 || (a.k_stride[1] >= a.dim && a.v_stride[1] >= a.dim), PETRA_ERR_SHAPE,
         "token stride of k or v below head_dim");
    need_distinct(a.o_stride, nq, a.dim, "o");
    if (backward) {
      for (const int64_t* st : {a.q_stride, a.o_stride})
        need((64 * st[1] + a.group * st[2]) * static_cast<int64_t>(esz) < (int64_t{1} << 31), PETRA_ERR_SHAPE,
             "heads that share a key head, or tokens of q or o, too far apart");
      need_distinct(a.q_stride, nq, a.dim, "dq");
      need_distinct(a.k_stride, nk, a.dim, "dk");
      need_distinct(a.v_stride, nk, a.dim, "dv");
    }
    plan = petra::attn_plan(a);
  }

  // The memory of q, k, v, o or what is laid out like it, and of lse.
  Runs tensor(const void* p, const int64_t st[3], bool kv, const char* name) const {
    const int64_t n[3] = {a.batch, kv ? a.kv_len : a.q_len, kv ? a.kv_heads : a.heads};
    return {p, st, n, a.dim, esz, name};
  }
  Runs stats(const float* p) const { return Span{p, static_cast<size_t>(a.batch) * a.heads * a.q_len * 4, "lse"}; }
};

}  // namespace

extern "C" {

petra_status petra_attn_query(const petra_attn_desc* desc, size_t* forward_bytes, size_t* backward_bytes) {
  return entry("petra_attn_query", [&]() -> bool {
    const Attn t(desc, nullptr, false, false);
    if (forward_bytes != nullptr) *forward_bytes = t.plan.fwd_bytes;
    if (backward_bytes != nullptr) *backward_bytes = t.plan.bwd_bytes;
    return false;
  });
}

petra_status petra_attn_forward(const petra_attn_desc* desc, const void* q, const void* k, const void* v,
                                const int32_t* q_lens, const int32_t* kv_lens, const uint64_t* rng, void* o,
                                float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  return entry("petra_attn_forward", [&]() -> bool {
    Attn t(desc, rng, true, false);
    need_ptr(q, "q", t.no_q());
    need_ptr(k, "k", t.no_kv());
    need_ptr(v, "v", t.no_kv());
    need_ptr(o, "o", t.no_q());
    need_ptr(lse, "lse", t.no_q());
    need_int_ptr(q_lens, "q_lens", 4);
    need_int_ptr(kv_lens, "kv_lens", 4);
    const Runs ro = t.tensor(o, t.a.o_stride, false, "o"), rl = t.stats(lse);
    for (const Runs& in : {t.tensor(q, t.a.q_stride, false, "q"), t.tensor(k, t.a.k_stride, true, "k"),
                           t.tensor(v, t.a.v_stride, true, "v")}) {
      need_apart(ro, in);
      need_apart(rl, in);
    }
    need_apart(ro, rl);
    need_workspace(workspace, workspace_bytes, t.plan.fwd_bytes);
    if (t.no_q()) return false;
    t.a.q = q;
    t.a.k = k;
    t.a.v = v;
    t.a.q_lens = q_lens;
    t.a.kv_lens = kv_lens;
    t.a.out = o;
    t.a.lse = lse;
    petra::attn_forward(t.a, t.plan, desc->dtype, workspace, static_cast<hipStream_t>(stream));
    return true;
  });
}

petra_status petra_attn_backward(const petra_attn_desc* desc, const void* q, const void* k, const void* v,
                                 const void* o, const float* lse, const void* d_o, const int32_t* q_lens,
                                 const int32_t* kv_lens, const uint64_t* rng, void* dq, void* dk, void* dv,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  return entry("petra_attn_backward", [&]() -> bool {
    Attn t(desc, rng, true, true);
    const bool nq = t.no_q(), nk = t.no_kv();
    need_ptr(q, "q", nq);
    need_ptr(k, "k", nk);
    need_ptr(v, "v", nk);
    need_ptr(o, "o", nq);
    need_ptr(lse, "lse", nq);
    need_ptr(d_o, "d_o", nq);
    need_ptr(dq, "dq", nq);
    need_ptr(dk, "dk", nk);
    need_ptr(dv, "dv", nk);
    need_int_ptr(q_lens, "q_lens", 4);
    need_int_ptr(kv_lens, "kv_lens", 4);
    const Runs in[6] = {t.tensor(q, t.a.q_stride, false, "q"), t.tensor(k, t.a.k_stride, true, "k"),
                        t.tensor(v, t.a.v_stride, true, "v"), t.tensor(o, t.a.o_stride, false, "o"),
                        t.tensor(d_o, t.a.o_stride, false, "d_o"), t.stats(lse)};
    const Runs out[3] = {t.tensor(dq, t.a.q_stride, false, "dq"), t.tensor(dk, t.a.k_stride, true, "dk"),
                         t.tensor(dv, t.a.v_stride, true, "dv")};
    for (int i = 0; i < 3; ++i) {
      for (const Runs& r : in) need_apart(out[i], r);
      for (int j = 0; j < i; ++j) need_apart(out[i], out[j]);
    }
    need_workspace(workspace, workspace_bytes, t.plan.bwd_bytes);
    if (t.a.batch == 0) return false;
    t.a.q = q;
    t.a.k = k;
    t.a.v = v;
    t.a.o = o;
    t.a.lse = const_cast<float*>(lse);
    t.a.d_o = d_o;
    t.a.q_lens = q_lens;
    t.a.kv_lens = kv_lens;
    t.a.dq = dq;
    t.a.dk = dk;
    t.a.dv = dv;
    petra::attn_backward(t.a, t.plan, desc->dtype, workspace, static_cast<hipStream_t>(stream));
    return true;
  });
}

}  // extern "C"

// ---------------------------------------------------------------------------
// coupling
// ---------------------------------------------------------------------------

namespace {

struct Coupling {
  petra::CoupleArgs a{};
  size_t bytes, param, gates;   // of an activation, a parameter vector, the gates

  Coupling(const petra_coupling_desc* d, const uint64_t* rng, bool with_f) {
    need(d != nullptr, PETRA_ERR_INVALID_ARG, "null description");
    need_dtype(d->dtype);
    need(d->rows >= 0 && d->rows_per_gate >= 0, PETRA_ERR_SHAPE, "negative size");
    need(d->width >= 8 && d->width <= 8192 && d->width % 8 == 0, PETRA_ERR_SHAPE,
         "width must be a multiple of 8, at most 8192");
    need(d->rows <= (int64_t{1} << 31) - 64, PETRA_ERR_SHAPE, "too many rows");
    need(d->norm == PETRA_NORM_RMS || d->norm == PETRA_NORM_LAYER, PETRA_ERR_INVALID_ARG, "unknown norm");
    need(d->eps > 0.f && std::isfinite(d->eps), PETRA_ERR_INVALID_ARG, "eps must be positive and finite");
    need(d->residual_scale != 0.f && std::isfinite(d->residual_scale), PETRA_ERR_INVALID_ARG,
         "residual_scale must be finite and not 0");
    a.rows = d->rows;
    a.width = d->width;
    a.rows_per_gate = d->rows_per_gate > 0 ? d->rows_per_gate : std::max<int64_t>(d->rows, 1);
    need(a.rows % a.rows_per_gate == 0, PETRA_ERR_SHAPE, "rows must be a multiple of rows_per_gate");
    a.gates = d->rows_per_gate > 0 ? a.rows / a.rows_per_gate : 1;
    a.layer = d->norm == PETRA_NORM_LAYER;
    a.eps = d->eps;
    a.scale = d->residual_scale;
    a.inv_scale = 1.f / d->residual_scale;
    a.inv_width = 1.f / static_cast<float>(d->width);
    a.cut = need_dropout(d->dropout, rng, with_f);
    a.inv_keep = inv_keep(a.cut);
    a.rng = with_f && a.cut > 0 ? rng : nullptr;
    bytes = static_cast<size_t>(a.rows) * a.width * size_of(d->dtype);
    param = static_cast<size_t>(a.width) * 4;
    gates = static_cast<size_t>(a.gates) * param;
    petra::couple_plan(a);
  }

  size_t part_bytes() const { return static_cast<size_t>(a.blocks) * param; }
};

void need_norm(const petra_norm_params* p, const char* name) {
  if (p == nullptr) throw Refused{PETRA_ERR_INVALID_ARG, std::string("null pointer: ") + name};
  need_ptr(p->gamma, name);
  need_ptr(p->beta, name, p->beta == nullptr);
}

}  // namespace

extern "C" {

petra_status petra_coupling_query(const petra_coupling_desc* desc, size_t* backward_bytes) {
  return entry("petra_coupling_query", [&]() -> bool {
    const Coupling t(desc, nullptr, false);
    if (backward_bytes != nullptr) *backward_bytes = 5 * t.part_bytes();
    return false;
  });
}

petra_status petra_coupling_forward(const petra_coupling_desc* desc, const void* x, const void* f,
                                    const float* gate, const petra_norm_params* post,
                                    const petra_norm_params* pre, const uint64_t* rng, void* y, void* u,
                                    void* stream) {
  return entry("petra_coupling_forward", [&]() -> bool {
    Coupling t(desc, rng, f != nullptr);
    const bool empty = t.a.rows == 0;
    need_ptr(x, "x", empty);
    if (f != nullptr) {
      need_ptr(f, "f");
      need_ptr(y, "y", empty);
      need_ptr(gate, "gate", empty);
      need_norm(post, "post");
      t.a.post_gamma = post->gamma;
      t.a.post_beta = post->beta;
    } else {
      need(empty || (y == nullptr && gate == nullptr && post == nullptr), PETRA_ERR_INVALID_ARG,
           "y, gate and post belong to f");
      need(empty || u != nullptr, PETRA_ERR_INVALID_ARG, "nothing to compute: neither f nor u");
    }
    if (u != nullptr) {
      need_ptr(u, "u");
      need_norm(pre, "pre");
      t.a.pre_gamma = pre->gamma;
      t.a.pre_beta = pre->beta;
    }
    const Span sx{x, t.bytes, "x"}, sf{f, t.bytes, "f"}, sy{y, t.bytes, "y"}, su{u, t.bytes, "u"},
        sg{gate, t.gates, "gate"};
    need_apart(sy, sx, true);
    need_apart(sy, sf);
    need_apart(sy, su);
    need_apart(su, sf, true);
    need_apart(su, sx);
    const Span params[5] = {sg,
                            {f != nullptr ? post->gamma : nullptr, t.param, "post.gamma"},
                            {f != nullptr ? post->beta : nullptr, t.param, "post.beta"},
                            {u != nullptr ? pre->gamma : nullptr, t.param, "pre.gamma"},
                            {u != nullptr ? pre->beta : nullptr, t.param, "pre.beta"}};
    for (const Span& p : params) {
      need_apart(sy, p);
      need_apart(su, p);
    }
    if (empty) return false;
    t.a.x = x;
    t.a.f = f;
    t.a.gate = gate;
    t.a.y = y;
    t.a.u = u;
    petra::couple_forward(t.a, desc->dtype, static_cast<hipStream_t>(stream));
    return true;
  });
}

petra_status petra_coupling_backward(const petra_coupling_desc* desc, const void* y, const void* f, const void* dy,
                                     const void* du, const float* gate, const petra_norm_params* post,
                                     const petra_norm_params* pre, const uint64_t* rng, void* x, void* dx, void* df,
                                     float* dgate, const petra_norm_params* dpost, const petra_norm_params* dpre,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  return entry("petra_coupling_backward", [&]() -> bool {
    // without rows the parameters' gradients are still written
    const bool with_f = post != nullptr, with_u = pre != nullptr;
    Coupling t(desc, rng, with_f);
    const bool empty = t.a.rows == 0;
    need_ptr(y, "y", empty);
    need_ptr(dy, "dy", empty);
    need_ptr(dx, "dx", empty);
    if (with_f) {
      need_ptr(f, "f", empty);
      need_ptr(df, "df", empty);
      need_ptr(x, "x", empty || x == nullptr);
      const bool no_gates = t.a.gates == 0;
      need_ptr(gate, "gate", no_gates);
      need_ptr(dgate, "dgate", no_gates);
      need_norm(post, "post");
      need_norm(dpost, "dpost");
      need((post->beta != nullptr) == (dpost->beta != nullptr), PETRA_ERR_INVALID_ARG, "post and dpost differ in beta");
    } else {
      need(f == nullptr && gate == nullptr && x == nullptr && df == nullptr && dgate == nullptr && dpost == nullptr,
           PETRA_ERR_INVALID_ARG, "f, gate, x, df, dgate and dpost belong to post");
    }
    if (with_u) {
      need_ptr(du, "du", empty);
      need_norm(pre, "pre");
      need_norm(dpre, "dpre");
      need((pre->beta != nullptr) == (dpre->beta != nullptr), PETRA_ERR_INVALID_ARG, "pre and dpre differ in beta");
    } else {
      need(du == nullptr && dpre == nullptr, PETRA_ERR_INVALID_ARG, "du and dpre belong to pre");
    }
    need(with_f || with_u, PETRA_ERR_INVALID_ARG, "nothing to compute: neither post nor pre");
    const Span in[4] = {{y, t.bytes, "y"}, {dy, t.bytes, "dy"}, {f, t.bytes, "f"}, {du, t.bytes, "du"}};
    const Span out[3] = {{x, t.bytes, "x"}, {dx, t.bytes, "dx"}, {df, t.bytes, "df"}};
    const Span small[5] = {{dgate, t.gates, "dgate"},
                           {with_f ? dpost->gamma : nullptr, t.param, "dpost.gamma"},
                           {with_f ? dpost->beta : nullptr, t.param, "dpost.beta"},
                           {with_u ? dpre->gamma : nullptr, t.param, "dpre.gamma"},
                           {with_u ? dpre->beta : nullptr, t.param, "dpre.beta"}};
    for (int i = 0; i < 3; ++i) {
      for (int j = 0; j < 4; ++j) need_apart(out[i], in[j], i == j || (i == 1 && j == 3));
      for (int j = 0; j < i; ++j) need_apart(out[i], out[j]);
      for (const Span& s : small) need_apart(out[i], s);
    }
    const Span params[5] = {{gate, t.gates, "gate"},
                            {with_f ? post->gamma : nullptr, t.param, "post.gamma"},
                            {with_f ? post->beta : nullptr, t.param, "post.beta"},
                            {with_u ? pre->gamma : nullptr, t.param, "pre.gamma"},
                            {with_u ? pre->beta : nullptr, t.param, "pre.beta"}};
    for (int i = 0; i < 5; ++i) {
      for (const Span& s : in) need_apart(small[i], s);
      for (const Span& s : params) need_apart(small[i], s);
      for (const Span& s : out) need_apart(params[i], s);
      for (int j = 0; j < i; ++j) need_apart(small[i], small[j]);
    }
    need_workspace(workspace, workspace_bytes, 5 * t.part_bytes());
    petra::CoupleArgs& a = t.a;
    a.y_in = y;
    a.dy = dy;
    a.dx = dx;
    float* const ws = static_cast<float*>(workspace);
    const size_t part = t.part_bytes() / 4;
    if (with_f) {
      a.f = empty ? y : f;
      a.has_f = 1;
      a.gate = gate;
      a.x_out = x;
      a.df = df;
      a.dgate = dgate;
      a.post_gamma = post->gamma;
      a.post_beta = post->beta;
      a.dpost_gamma = dpost->gamma;
      a.dpost_beta = dpost->beta;
      a.part_gate = ws;
      a.part_post_gamma = ws + part;
      a.part_post_beta = ws + 2 * part;
    }
    if (with_u) {
      a.du = du;
      a.has_u = 1;
      a.pre_gamma = pre->gamma;
      a.pre_beta = pre->beta;
      a.dpre_gamma = dpre->gamma;
      a.dpre_beta = dpre->beta;
      a.part_pre_gamma = ws + 3 * part;
      a.part_pre_beta = ws + 4 * part;
    }
    petra::couple_backward(a, desc->dtype, static_cast<hipStream_t>(stream));
    return true;
  });
}

petra_status petra_dropout(int64_t n, int32_t dtype, float p, float alpha, const void* x, const void* residual,
                           const uint64_t* rng, void* y, void* stream) {
  return entry("petra_dropout", [&]() -> bool {
    need_dtype(dtype);
    need(n >= 0 && n < (int64_t{1} << 46), PETRA_ERR_SHAPE, "negative or too large size");
    need(std::isfinite(alpha), PETRA_ERR_INVALID_ARG, "alpha must be finite");
    const uint32_t cut = need_dropout(p, rng, true);
    need_ptr(x, "x", n == 0);
    need_ptr(y, "y", n == 0);
    need_ptr(residual, "residual", n == 0 || residual == nullptr);
    const size_t bytes = static_cast<size_t>(n) * size_of(dtype);
    const Span sx{x, bytes, "x"}, sr{residual, bytes, "residual"}, sy{y, bytes, "y"};
    need_apart(sy, sx, true);
    need_apart(sy, sr, true);
    if (n == 0) return false;
    petra::dropout(x, residual, y, n, alpha * inv_keep(cut), cut, rng, dtype, static_cast<hipStream_t>(stream));
    return true;
  });
}

}  // extern "C"

// ---------------------------------------------------------------------------
// head norms and rotation
// ---------------------------------------------------------------------------

namespace {

static_assert(petra::HEADS_AXES == PETRA_HEAD_AXES && petra::HEADS_PAIRS == PETRA_HEAD_PAIRS, "the header's limits");

// The binary digits of 1 / 2 pi, from the one of 2^-1 on: by 2 pi = 8 (4 arctan 1/5 - arctan 1/239) in whole numbers.
constexpr uint64_t TURN[19] = {
    0x28be60db9391054a, 0x7f09d5f47d4d3770, 0x36d8a5664f10e410, 0x7f9458eaf7aef158,
    0x6dc91b8e909374b8, 0x01924bba82746487, 0x3f877ac72c4a69cf, 0xba208d7d4baed121,
    0x3a671c09ad17df90, 0x4e64758e60d4ce7d, 0x272117e2ef7e4a0e, 0xc7fe25fff7816603,
    0xfbcbc462d6829b47, 0xdb4d9fb3c9f2c26d, 0xd3d18fd9a797fa8b, 0x5d49eeb1faf97c5e,
    0xcf41ce7de294a4ba, 0x9afed7ec47e35742, 0x1580cc11bf1edaea};

// 128 digits of 1 / 2 pi that begin with the one of 2^-(at + 1); before the first they are zeros.
unsigned __int128 turn_digits(int at) {
  auto word = [](int i) { return i < 0 || i >= static_cast<int>(std::size(TURN)) ? uint64_t{0} : TURN[i]; };
  const int first = at >> 6, by = at & 63;   // (rounded down)
  const uint64_t a = word(first), b = word(first + 1), c = word(first + 2);
  const uint64_t hi = by == 0 ? a : a << by | b >> (64 - by), lo = by == 0 ? b : b << by | c >> (64 - by);
  return static_cast<unsigned __int128>(hi) << 64 | lo;
}

// The fraction of a turn that finite `radians` are, in 64 bits, to the nearest; a whole one wraps.  radians = m 2^e with a whole m
// below 2^53: digits of 1 / 2 pi before the e-th give whole turns, and those past the next 128 less than 2^-75 of one.  (The bits
// are taken apart here: library calls for it take longer than all else that a call does on the host.)
uint64_t turn_fraction(double radians) {
  uint64_t bits;
  std::memcpy(&bits, &radians, 8);
  const int e = static_cast<int>(bits >> 52 & 0x7ff);
  const uint64_t m = (bits & 0xfffffffffffffULL) | (e > 0 ? uint64_t{1} << 52 : 0);
  const unsigned __int128 f = turn_digits((e > 0 ? e : 1) - 1075) * m + (uint64_t{1} << 63);
  const auto u = static_cast<uint64_t>(f >> 64);
  return radians < 0. ? 0 - u : u;
}

struct Heads {
  petra::HeadsArgs a{};
  int64_t n[2][3];   // positions of the queries and of the keys
  size_t esz;
  bool empty;

  Heads(const petra_heads_desc* d, bool backward) {
    need(d != nullptr, PETRA_ERR_INVALID_ARG, "null description");
    need_dtype(d->dtype);
    esz = size_of(d->dtype);
    need(d->batch >= 0 && d->len >= 0, PETRA_ERR_SHAPE, "negative size");
    need(d->heads >= 1 && d->heads <= 65535 && d->kv_heads >= 0 && d->kv_heads <= 65535, PETRA_ERR_SHAPE,
         "heads must be 1 .. 65535, kv_heads 0 .. 65535");
    need(d->head_dim >= 8 && d->head_dim <= 128 && d->head_dim % 8 == 0, PETRA_ERR_SHAPE,
         "head_dim must be a multiple of 8, at most 128");
    need(d->norm == PETRA_NORM_RMS || d->norm == PETRA_NORM_LAYER, PETRA_ERR_INVALID_ARG, "unknown norm");
    need(d->eps > 0.f && std::isfinite(d->eps), PETRA_ERR_INVALID_ARG, "eps must be positive and finite");
    need(d->layout == PETRA_PAIRS_HALVES || d->layout == PETRA_PAIRS_NEIGHBOURS, PETRA_ERR_INVALID_ARG, "unknown layout of pairs");
    need(d->pairs >= 0 && d->pairs % 4 == 0 && 2 * d->pairs <= d->head_dim, PETRA_ERR_SHAPE,
         "pairs must be a multiple of 4, at most head_dim / 2");
    need(d->axes >= 1 && d->axes <= PETRA_HEAD_AXES, PETRA_ERR_SHAPE, "axes must be 1 .. 4");
    const int64_t tokens = static_cast<int64_t>(d->batch) * d->len;
    need(tokens < (int64_t{1} << 31), PETRA_ERR_SHAPE, "batch * len of 2^31 or more");
    a.tokens = tokens;
    a.len = static_cast<uint32_t>(d->len);
    a.dim = d->head_dim;
    a.pairs = d->pairs;
    a.axes = d->axes;
    a.halves = d->layout == PETRA_PAIRS_HALVES;
    a.layer = d->norm == PETRA_NORM_LAYER;
    a.eps = d->eps;
    a.inv_dim = 1.f / static_cast<float>(d->head_dim);
    empty = tokens == 0;
    for (int i = 0; i < d->pairs; ++i) {
      need(d->axis[i] >= 0 && d->axis[i] < d->axes, PETRA_ERR_INVALID_ARG, "a pair's axis is none of the axes");
      need(std::isfinite(d->freq[i]), PETRA_ERR_INVALID_ARG, "frequencies must be finite");
      a.axes4[i / 8] |= static_cast<uint32_t>(d->axis[i]) << (i % 8 * 4);
      a.freq[i] = turn_fraction(d->freq[i]);
    }
    for (int i = 0; i < 2; ++i) {
      petra::HeadsPart& p = a.part[i];
      p.heads = i == 0 ? d->heads : d->kv_heads;
      n[i][0] = d->batch, n[i][1] = d->len, n[i][2] = p.heads;
      const char *x = i == 0 ? "q" : "k", *y = i == 0 ? "yq" : "yk";
      strides(i == 0 ? d->q_stride : d->k_stride, p.x_stride, d->len, p.heads, a.dim, esz, x);
      strides(i == 0 ? d->yq_stride : d->yk_stride, p.y_stride, d->len, p.heads, a.dim, esz, y);
      need_reach(p.x_stride, n[i], a.dim, esz, x);
      need_reach(p.y_stride, n[i], a.dim, esz, y);
      if (backward) need_distinct(p.x_stride, n[i], a.dim, i == 0 ? "dq" : "dk");
      else need_distinct(p.y_stride, n[i], a.dim, y);
    }
    petra::heads_plan(a, backward);
  }

  bool none(int i) const { return empty || a.part[i].heads == 0; }
  Runs x(const void* p, int i, const char* name) const { return {none(i) ? nullptr : p, a.part[i].x_stride, n[i], a.dim, esz, name}; }
  Runs y(const void* p, int i, const char* name) const { return {none(i) ? nullptr : p, a.part[i].y_stride, n[i], a.dim, esz, name}; }
  bool same_strides(int i) const {
    for (int d = 0; d < 3; ++d)
      if (n[i][d] > 1 && a.part[i].x_stride[d] != a.part[i].y_stride[d]) return false;
    return true;
  }
  Span positions(const int32_t* p) const {
    return {empty ? nullptr : p, static_cast<size_t>(a.axes) * static_cast<size_t>(a.tokens) * 4, "positions"};
  }
  Span param(const float* p, const char* name) const { return {p, static_cast<size_t>(a.dim) * 4, name}; }
  // gamma and beta of both norms, or of their gradients
  int params(const petra_norm_params* q, const petra_norm_params* k, Span out[4], const char* const names[4]) const {
    int count = 0;
    for (int i = 0; i < 2; ++i) {
      const petra_norm_params* const p = i == 0 ? q : k;
      if (p == nullptr) continue;
      out[count++] = param(p->gamma, names[2 * i]);
      if (p->beta != nullptr) out[count++] = param(p->beta, names[2 * i + 1]);
    }
    return count;
  }
  size_t part_bytes(int i) const { return static_cast<size_t>(a.part[i].blocks) * a.dim * 4; }
  size_t backward_bytes() const { return 2 * (part_bytes(0) + part_bytes(1)); }
};

const char* const HEAD_PARAMS[4] = {"q_norm.gamma", "q_norm.beta", "k_norm.gamma", "k_norm.beta"};
const char* const HEAD_GRADS[4] = {"dq_norm.gamma", "dq_norm.beta", "dk_norm.gamma", "dk_norm.beta"};

}  // namespace

extern "C" {

petra_status petra_heads_query(const petra_heads_desc* desc, size_t* backward_bytes) {
  return entry("petra_heads_query", [&]() -> bool {
    const Heads t(desc, true);
    if (backward_bytes != nullptr) *backward_bytes = t.backward_bytes();
    return false;
  });
}

petra_status petra_heads_forward(const petra_heads_desc* desc, const void* q, const void* k,
                                 const petra_norm_params* q_norm, const petra_norm_params* k_norm,
                                 const int32_t* positions, void* yq, void* yk, void* stream) {
  return entry("petra_heads_forward", [&]() -> bool {
    Heads t(desc, false);
    const void* const in[2] = {q, k};
    void* const out[2] = {yq, yk};
    const petra_norm_params* const norm[2] = {q_norm, k_norm};
    const char* const names[6] = {"q", "k", "yq", "yk", "q_norm", "k_norm"};
    for (int i = 0; i < 2; ++i) {
      need_ptr(in[i], names[i], t.none(i));
      need_ptr(out[i], names[2 + i], t.none(i));
      if (norm[i] != nullptr) need_norm(norm[i], names[4 + i]);
    }
    need(desc->kv_heads > 0 || (k == nullptr && yk == nullptr && k_norm == nullptr), PETRA_ERR_INVALID_ARG,
         "k, yk and k_norm without key heads");
    need_int_ptr(positions, "positions", 4);
    Span small[5];
    int count = t.params(q_norm, k_norm, small, HEAD_PARAMS);
    small[count++] = t.positions(positions);
    for (int i = 0; i < 2; ++i) {
      const Runs y = t.y(out[i], i, names[2 + i]);
      for (int j = 0; j < 2; ++j)
        if (!(i == j && out[i] == in[j] && t.same_strides(i))) need_apart(y, t.x(in[j], j, names[j]));
      for (int j = 0; j < count; ++j) need_apart(y, small[j]);
    }
    need_apart(t.y(yq, 0, "yq"), t.y(yk, 1, "yk"));
    if (t.empty) return false;
    t.a.positions = positions;
    for (int i = 0; i < 2; ++i) {
      t.a.part[i].x = in[i];
      t.a.part[i].y = out[i];
      t.a.part[i].gamma = norm[i] != nullptr ? norm[i]->gamma : nullptr;
      t.a.part[i].beta = norm[i] != nullptr ? norm[i]->beta : nullptr;
    }
    petra::heads_forward(t.a, desc->dtype, static_cast<hipStream_t>(stream));
    return true;
  });
}

petra_status petra_heads_backward(const petra_heads_desc* desc, const void* q, const void* k,
                                  const petra_norm_params* q_norm, const petra_norm_params* k_norm,
                                  const int32_t* positions, const void* dyq, const void* dyk, void* dq, void* dk,
                                  const petra_norm_params* dq_norm, const petra_norm_params* dk_norm, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  return entry("petra_heads_backward", [&]() -> bool {
    Heads t(desc, true);
    const void *const x[2] = {q, k}, *const dy[2] = {dyq, dyk};
    void* const dx[2] = {dq, dk};
    const petra_norm_params *const norm[2] = {q_norm, k_norm}, *const dnorm[2] = {dq_norm, dk_norm};
    const char* const names[10] = {"q", "k", "dyq", "dyk", "dq", "dk", "q_norm", "k_norm", "dq_norm", "dk_norm"};
    need(desc->kv_heads > 0 || (k == nullptr && dyk == nullptr && dk == nullptr && k_norm == nullptr && dk_norm == nullptr),
         PETRA_ERR_INVALID_ARG, "k, dyk, dk, k_norm and dk_norm without key heads");
    for (int i = 0; i < 2; ++i) {
      need_ptr(x[i], names[i], t.none(i) || norm[i] == nullptr);
      need_ptr(dy[i], names[2 + i], t.none(i));
      need_ptr(dx[i], names[4 + i], t.none(i));
      if (norm[i] != nullptr) {
        need_norm(norm[i], names[6 + i]);
        need_norm(dnorm[i], names[8 + i]);
        need((norm[i]->beta != nullptr) == (dnorm[i]->beta != nullptr), PETRA_ERR_INVALID_ARG,
             "a norm and its gradient differ in beta");
      } else {
        need(dnorm[i] == nullptr, PETRA_ERR_INVALID_ARG, "a norm's gradient without the norm");
      }
    }
    need_int_ptr(positions, "positions", 4);
    Span in[5], out[4];
    int ins = t.params(q_norm, k_norm, in, HEAD_PARAMS);
    in[ins++] = t.positions(positions);
    const int outs = t.params(dq_norm, dk_norm, out, HEAD_GRADS);
    for (int i = 0; i < 2; ++i) {
      const Runs d = t.x(dx[i], i, names[4 + i]);
      for (int j = 0; j < 2; ++j) {
        if (norm[j] != nullptr && !(i == j && dx[i] == x[j])) need_apart(d, t.x(x[j], j, names[j]));
        if (!(i == j && dx[i] == dy[j] && t.same_strides(i))) need_apart(d, t.y(dy[j], j, names[2 + j]));
      }
      for (int j = 0; j < ins; ++j) need_apart(d, in[j]);
      for (int j = 0; j < outs; ++j) {
        need_apart(d, out[j]);
        if (norm[i] != nullptr) need_apart(t.x(x[i], i, names[i]), out[j]);
        need_apart(t.y(dy[i], i, names[2 + i]), out[j]);
      }
    }
    need_apart(t.x(dq, 0, "dq"), t.x(dk, 1, "dk"));
    for (int i = 0; i < outs; ++i) {
      for (int j = 0; j < ins; ++j) need_apart(out[i], in[j]);
      for (int j = 0; j < i; ++j) need_apart(out[i], out[j]);
    }
    const bool sums = q_norm != nullptr || k_norm != nullptr;
    need_workspace(workspace, workspace_bytes, sums ? t.backward_bytes() : 0);
    if (t.empty && !sums) return false;
    t.a.positions = positions;
    float* ws = static_cast<float*>(workspace);
    for (int i = 0; i < 2; ++i) {
      petra::HeadsPart& p = t.a.part[i];
      p.x = x[i];
      p.dy = dy[i];
      p.dx = dx[i];
      if (norm[i] != nullptr) {
        p.gamma = norm[i]->gamma;
        p.beta = norm[i]->beta;
        p.dgamma = dnorm[i]->gamma;
        p.dbeta = dnorm[i]->beta;
      }
      p.part_gamma = ws;
      p.part_beta = ws + t.part_bytes(i) / 4;
      ws += t.part_bytes(i) / 2;
    }
    petra::heads_backward(t.a, desc->dtype, static_cast<hipStream_t>(stream));
    return true;
  });
}

}  // extern "C"

// ---------------------------------------------------------------------------
// loss over a vocabulary
// ---------------------------------------------------------------------------

namespace {

struct Vocab {
  petra::VocabArgs a{};
  size_t x_bytes, w_bytes, row_bytes;
  int dtype;
  long piece_rows;

  explicit Vocab(const petra_vocab_desc* d) {
    need(d != nullptr, PETRA_ERR_INVALID_ARG, "null description");
    need_dtype(d->dtype);
    need(d->rows >= 0 && d->rows <= (int64_t{1} << 30) && d->piece_rows >= 0, PETRA_ERR_SHAPE, "negative size or too many rows");
    need(d->width >= 8 && d->width <= 65536 && d->width % 8 == 0, PETRA_ERR_SHAPE,
         "width must be a multiple of 8, at most 65536");
    need(d->vocab >= 1 && d->vocab <= (1 << 20), PETRA_ERR_SHAPE, "vocab must be 1 .. 2^20");
    // (2^127 and more pass fp32 with log2(e), and times a score of 0 are NaN)
    need(d->scale > 0.f && d->scale < 0x1p127f, PETRA_ERR_INVALID_ARG, "scale must be positive and below 2^127");
    a.rows = d->rows;
    a.width = d->width;
    a.vocab = d->vocab;
    a.vocab_padded = (d->vocab + 63) / 64 * 64;
    a.scale = d->scale;
    a.scale_log2 = d->scale * 1.44269504088896340736f;
    dtype = d->dtype;
    piece_rows = d->piece_rows;
    x_bytes = static_cast<size_t>(a.rows) * a.width * size_of(dtype);
    w_bytes = static_cast<size_t>(a.vocab) * a.width * size_of(dtype);
    row_bytes = static_cast<size_t>(a.rows) * 4;
  }

  petra::VocabPlan plan(bool gradients) const { return petra::vocab_plan(a, dtype, gradients, piece_rows); }
};

petra_status vocab_call(const char* name, const petra_vocab_desc* desc, const void* x, const void* w, const int32_t* targets,
                        const float* weight, float* loss, float* lse, void* dx, void* dw, bool gradients, void* workspace,
                        size_t workspace_bytes, void* stream) {
  return entry(name, [&]() -> bool {
    Vocab t(desc);
    const bool empty = t.a.rows == 0;
    need_ptr(x, "x", empty);
    need_ptr(w, "w");
    need_ptr(loss, "loss", empty);
    need_ptr(lse, "lse", empty);
    if (!empty && targets == nullptr) throw Refused{PETRA_ERR_INVALID_ARG, "null pointer: targets"};
    need_int_ptr(targets, "targets", 4);
    need_int_ptr(weight, "weight", 4);
    if (gradients) {
      need_ptr(dx, "dx", empty);
      need_ptr(dw, "dw");
    }
    const Span in[4] = {{x, t.x_bytes, "x"}, {w, t.w_bytes, "w"}, {targets, t.row_bytes, "targets"}, {weight, t.row_bytes, "weight"}};
    const Span out[4] = {{loss, t.row_bytes, "loss"}, {lse, t.row_bytes, "lse"}, {dx, t.x_bytes, "dx"}, {dw, t.w_bytes, "dw"}};
    for (int i = 0; i < (gradients ? 4 : 2); ++i) {
      for (const Span& s : in) need_apart(out[i], s);
      for (int j = 0; j < i; ++j) need_apart(out[i], out[j]);
    }
    const petra::VocabPlan plan = t.plan(gradients);
    need_workspace(workspace, workspace_bytes, plan.bytes);
    if (empty && !gradients) return false;
    t.a.x = x;
    t.a.w = w;
    t.a.targets = targets;
    t.a.weight = weight;
    t.a.loss = loss;
    t.a.lse = lse;
    t.a.dx = dx;
    t.a.dw = dw;
    petra::vocab_run(t.a, plan, t.dtype, gradients, workspace, static_cast<hipStream_t>(stream));
    return true;
  });
}

}  // namespace

extern "C" {

petra_status petra_vocab_query(const petra_vocab_desc* desc, size_t* loss_bytes, size_t* gradient_bytes) {
  return entry("petra_vocab_query", [&]() -> bool {
    const Vocab t(desc);
    if (loss_bytes != nullptr) *loss_bytes = t.plan(false).bytes;
    if (gradient_bytes != nullptr) *gradient_bytes = t.plan(true).bytes;
    return false;
  });
}

petra_status petra_vocab_loss(const petra_vocab_desc* desc, const void* x, const void* w, const int32_t* targets, float* loss,
                              float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  return vocab_call("petra_vocab_loss", desc, x, w, targets, nullptr, loss, lse, nullptr, nullptr, false, workspace,
                    workspace_bytes, stream);
}

petra_status petra_vocab_gradient(const petra_vocab_desc* desc, const void* x, const void* w, const int32_t* targets,
                                  const float* weight, float* loss, float* lse, void* dx, void* dw, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  return vocab_call("petra_vocab_gradient", desc, x, w, targets, weight, loss, lse, dx, dw, true, workspace, workspace_bytes,
                    stream);
}

}  // extern "C"

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------

namespace {

constexpr size_t ADAMW_WORKSPACE = 16;
constexpr int64_t ADAMW_CHUNKS = int64_t{1} << 24;   // a workgroup of 256 each: a grid has fewer than 2^32 lanes

struct AdamwTable {
  int64_t chunks = 0;
  size_t bytes = 0;
};

size_t adamw_bytes(int64_t count, int64_t chunks) {
  return (static_cast<size_t>(count) * sizeof(petra::AdamwEntry) + static_cast<size_t>(chunks) * 4 + 15) / 16 * 16;
}

void need_adamw(const petra_adamw_desc* d) {
  need(d != nullptr, PETRA_ERR_INVALID_ARG, "null description");
  need(d->beta1 >= 0. && d->beta1 < 1. && d->beta2 >= 0. && d->beta2 < 1., PETRA_ERR_INVALID_ARG, "betas outside [0, 1)");
  // (of less the reciprocal is infinite, and a state of 0 times it NaN)
  need(d->eps >= std::numeric_limits<float>::min() && std::isfinite(d->eps), PETRA_ERR_INVALID_ARG, "eps must be at least 2^-126 and finite");
  need_dtype(d->grad_dtype);
  need(d->state_dtype == PETRA_FP32 || d->state_dtype == PETRA_E4M3, PETRA_ERR_DTYPE, "states must be fp32 or e4m3");
}

AdamwTable adamw_table(const petra_adamw_desc* d, const petra_adamw_tensor* tensors, int64_t count) {
  need_adamw(d);
  need(count >= 0 && count <= (int64_t{1} << 20), PETRA_ERR_SHAPE, "negative or too large count");
  need(count == 0 || tensors != nullptr, PETRA_ERR_INVALID_ARG, "null pointer: tensors");
  AdamwTable t;
  for (int64_t i = 0; i < count; ++i) {
    need(tensors[i].n >= 0 && tensors[i].n <= (int64_t{1} << 42), PETRA_ERR_SHAPE, "negative or too large tensor");
    t.chunks += (tensors[i].n + petra::ADAMW_CHUNK - 1) / petra::ADAMW_CHUNK;
    need(t.chunks < ADAMW_CHUNKS, PETRA_ERR_SHAPE, "too many elements");
  }
  t.bytes = adamw_bytes(count, t.chunks);
  return t;
}

}  // namespace

extern "C" {

petra_status petra_adamw_query(const petra_adamw_desc* desc, const petra_adamw_tensor* tensors, int64_t count,
                               size_t* table_bytes, int64_t* chunks, size_t* workspace_bytes) {
  return entry("petra_adamw_query", [&]() -> bool {
    const AdamwTable t = adamw_table(desc, tensors, count);
    if (table_bytes != nullptr) *table_bytes = t.bytes;
    if (chunks != nullptr) *chunks = t.chunks;
    if (workspace_bytes != nullptr) *workspace_bytes = ADAMW_WORKSPACE;
    return false;
  });
}

petra_status petra_adamw_layout(const petra_adamw_desc* desc, const petra_adamw_tensor* tensors, int64_t count, void* table,
                                size_t table_bytes) {
  return entry("petra_adamw_layout", [&]() -> bool {
    const AdamwTable t = adamw_table(desc, tensors, count);
    need(t.bytes == 0 || (table != nullptr && table_bytes >= t.bytes), PETRA_ERR_WORKSPACE, "table missing or too small");
    const bool fp8 = desc->state_dtype == PETRA_E4M3;
    const size_t gsz = size_of(desc->grad_dtype);
    // each range of memory once: a step works on all tensors at the same time
    std::vector<Span> all;
    for (int64_t i = 0; i < count; ++i) {
      const petra_adamw_tensor& x = tensors[i];
      const bool empty = x.n == 0;
      need(std::isfinite(x.weight_decay), PETRA_ERR_INVALID_ARG, "weight_decay must be finite");
      need_ptr(x.theta, "theta", empty);
      need_ptr(x.grad, "grad", empty);
      need_ptr(x.m, "m", empty);
      need_ptr(x.v, "v", empty);
      need_ptr(x.copy, "copy", empty || x.copy == nullptr);
      for (float* const scale : {x.m_scale, x.v_scale}) {
        if (!fp8 || empty) continue;
        need(scale != nullptr, PETRA_ERR_INVALID_ARG, "null pointer: m_scale or v_scale");
        need_int_ptr(scale, "m_scale or v_scale", 4);
      }
      if (empty) continue;
      const size_t n = static_cast<size_t>(x.n), blocks = (n + 63) / 64, state = fp8 ? 64 * blocks : 4 * n;
      all.push_back({x.theta, 4 * n, "theta"});
      all.push_back({x.grad, gsz * n, "grad"});
      all.push_back({x.m, state, "m"});
      all.push_back({x.v, state, "v"});
      if (x.copy != nullptr) all.push_back({x.copy, 2 * n, "copy"});
      if (fp8) {
        all.push_back({x.m_scale, 4 * blocks, "m_scale"});
        all.push_back({x.v_scale, 4 * blocks, "v_scale"});
      }
    }
    std::sort(all.begin(), all.end(), [](const Span& a, const Span& b) {
      return reinterpret_cast<uintptr_t>(a.p) < reinterpret_cast<uintptr_t>(b.p);
    });
    for (size_t i = 1; i < all.size(); ++i) need_apart(all[i - 1], all[i]);
    auto* const entries = static_cast<petra::AdamwEntry*>(table);
    auto* const chunk_of = reinterpret_cast<int32_t*>(entries + count);
    int64_t chunk = 0, group = 0;
    for (int64_t i = 0; i < count; ++i) {
      const petra_adamw_tensor& x = tensors[i];
      const int64_t padded = (x.n + 63) / 64 * 64;
      entries[i] = {x.theta, x.grad, x.m, x.v, x.copy, x.m_scale, x.v_scale, x.n, padded, chunk, group, x.weight_decay, 0};
      group += padded / 4;
      for (int64_t c = 0; c < x.n; c += petra::ADAMW_CHUNK) chunk_of[chunk++] = static_cast<int32_t>(i);
    }
    return false;
  });
}

petra_status petra_adamw_step(const petra_adamw_desc* desc, const void* table, size_t table_bytes, int64_t count,
                              int64_t chunks, int64_t* steps, const float* lr, const float* grad_scale, const uint64_t* rng,
                              void* workspace, size_t workspace_bytes, void* stream) {
  return entry("petra_adamw_step", [&]() -> bool {
    need_adamw(desc);
    need(count >= 0 && count <= (int64_t{1} << 20) && chunks >= 0 && chunks < ADAMW_CHUNKS, PETRA_ERR_SHAPE,
         "negative or too large count");
    need(chunks == 0 || table != nullptr, PETRA_ERR_INVALID_ARG, "null pointer: table");
    need(table_bytes >= adamw_bytes(count, chunks), PETRA_ERR_WORKSPACE, "table too small for its tensors and chunks");
    need_ptr(table, "table", table == nullptr);
    if (steps == nullptr) throw Refused{PETRA_ERR_INVALID_ARG, "null pointer: steps"};
    if (lr == nullptr) throw Refused{PETRA_ERR_INVALID_ARG, "null pointer: lr"};
    need_int_ptr(steps, "steps", 8);
    need_int_ptr(lr, "lr", 4);
    need_int_ptr(grad_scale, "grad_scale", 4);
    need_int_ptr(rng, "rng", 8);
    const bool fp8 = desc->state_dtype == PETRA_E4M3;
    need(!fp8 || rng != nullptr, PETRA_ERR_INVALID_ARG, "states in 8 bits without rng");
    need_workspace(workspace, workspace_bytes, ADAMW_WORKSPACE);
    petra::AdamwArgs a{};
    a.entries = static_cast<const petra::AdamwEntry*>(table);
    a.chunk_of = reinterpret_cast<const int32_t*>(a.entries + count);
    a.chunks = chunks;
    a.steps = steps;
    a.lr = lr;
    a.grad_scale = grad_scale;
    a.rng = rng;
    a.hyper = static_cast<float*>(workspace);
    a.log_b1 = std::log(desc->beta1);
    a.log_b2 = std::log(desc->beta2);
    a.b1 = static_cast<float>(desc->beta1);
    a.c1 = static_cast<float>(1. - desc->beta1);
    a.b2 = static_cast<float>(desc->beta2);
    a.c2 = static_cast<float>(1. - desc->beta2);
    a.eps = desc->eps;
    a.zero_grads = desc->zero_grads != 0;
    petra::adamw_step(a, desc->grad_dtype == PETRA_BF16, fp8, static_cast<hipStream_t>(stream));
    return true;
  });
}

}  // extern "C"
