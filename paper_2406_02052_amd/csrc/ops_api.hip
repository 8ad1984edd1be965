// extern "C" entry points of the token operators (attention, coupling, dropout):
// argument validation and dispatch.  Nothing here allocates device memory.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

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
