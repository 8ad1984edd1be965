// The coupling of a reversible block over tokens, and dropout.
//
// Forward:  y = s x + g m n(f; post),  u = n(y as stored; pre)
// Backward: t = dy + (d n(y; pre))^T du          (t = dy without u)
//           x = (y - g m n(f; post)) / s,  dx = s t,  df = (d n(f; post))^T (g m t)
//           and the gradients of g, post and pre.
// n is a norm over a row's W channels, n(z) = z^ gamma (+ beta) with
// z^ = (z - mean) r or z r; its transposed derivative takes h to
// r (h gamma - z^ mean(h gamma z^) (- mean(h gamma))).  m is dropout's 0 or 1/keep.
//
// All of it is bound by memory: 2 reads and 2 writes an element forward, 4 and 3
// backward.  A row stays in registers from its load to its store (a team of lanes
// holds it, 8 elements a lane and step), so each tensor crosses memory once; the
// row's sums are taken in fp32, in registers and, where a team is a whole
// workgroup, through LDS.  The variance is the mean of squared differences from
// the mean, a second pass over registers.
#include "common.h"
#include "ops.h"
#include "philox.h"

namespace petra {

namespace {

// ---------------------------------------------------------------------------
// rows and teams
// ---------------------------------------------------------------------------

// A team of TEAM lanes holds a row in V chunks of 8 elements a lane: chunk v of
// lane l covers elements 8 (v TEAM + l) ..  Teams of up to 64 lanes share a wave;
// a team of 256 is a workgroup.
template <int TEAM>
struct TeamSum {
  // Sums of N values over the team, in every lane.
  template <int N>
  static __device__ __forceinline__ void sum(float (&x)[N], float* lds) {
    constexpr int W = TEAM < 64 ? TEAM : 64;
#pragma unroll
    for (int d = 1; d < W; d <<= 1)
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] += __shfl_xor(x[i], d, 64);
    if constexpr (TEAM > 64) {
      const int wave = threadIdx.x >> 6;
      __syncthreads();   // the last sum's readers are done
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) lds[wave * N + i] = x[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[i] = 0.f;
#pragma unroll
        for (int w = 0; w < TEAM / 64; ++w) x[i] += lds[w * N + i];
      }
    }
  }
};

// Normalises z in place to z^; returns 1 / deviation.  Lanes past the row hold
// zeros and are put back to zero.
template <int TEAM, int V>
__device__ __forceinline__ float unit(float (&z)[V][8], const bool (&in)[V], bool layer, float inv_w,
                                      float eps, float* lds) {
  if (layer) {
    float s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[0] += z[v][e];
    TeamSum<TEAM>::sum(s, lds);
    const float mean = s[0] * inv_w;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < 8; ++e) z[v][e] = in[v] ? z[v][e] - mean : 0.f;
  }
  float q[1] = {0.f};
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) q[0] = fmaf(z[v][e], z[v][e], q[0]);
  TeamSum<TEAM>::sum(q, lds);
  const float r = rsqrtf(q[0] * inv_w + eps);
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) z[v][e] *= r;
  return r;
}

template <typename T>
__device__ __forceinline__ void load_or_zero(const T* p, bool in, float* o) {
  if (in) {
    Vec8<T>::load(p, o);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.f;
  }
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------

template <typename T, int TEAM, int V, bool DROP>
__global__ __launch_bounds__(256) void couple_forward_kernel(CoupleArgs a) {
  __shared__ float lds[4];
  constexpr int TEAMS = 256 / TEAM;
  const int lane = threadIdx.x % TEAM;
  const long w = a.width;
  const long row = static_cast<long>(blockIdx.x) * TEAMS + threadIdx.x / TEAM;
  const bool live = row < a.rows;
  bool in[V];
  int col[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    col[v] = 8 * (v * TEAM + lane);
    in[v] = live && col[v] < w;
  }
  const bool layer = a.layer != 0;
  const T* x = static_cast<const T*>(a.x) + row * w;
  float y[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v) load_or_zero(x + col[v], in[v], y[v]);
  if (a.f != nullptr) {
    const T* f = static_cast<const T*>(a.f) + row * w;
    float n[V][8];
#pragma unroll
    for (int v = 0; v < V; ++v) load_or_zero(f + col[v], in[v], n[v]);
    unit<TEAM, V>(n, in, layer, a.inv_width, a.eps, lds);
    const float* gate = a.gate + (live ? row / a.rows_per_gate : 0) * w;
    Rng rng{};
    if (DROP) rng = load_rng(a.rng);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!in[v]) continue;
      float gm[8], gg[8], bb[8] = {};
      Vec8<float>::load(a.post_gamma + col[v], gm);
      if (a.post_beta != nullptr) Vec8<float>::load(a.post_beta + col[v], bb);
      Vec8<float>::load(gate + col[v], gg);
      uint32_t bits[4];
      if (DROP) philox(rng, static_cast<uint64_t>(row * w + col[v]) >> 3, bits);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float t = fmaf(n[v][e], gm[e], bb[e]);
        if (DROP) t = kept(bits, e, a.cut) ? t * a.inv_keep : 0.f;
        y[v][e] = quant(fmaf(gg[e], t, a.scale * y[v][e]), static_cast<const T*>(nullptr));
      }
      Vec8<T>::store(static_cast<T*>(a.y) + row * w + col[v], y[v]);
    }
  }
  if (a.u != nullptr) {
    unit<TEAM, V>(y, in, layer, a.inv_width, a.eps, lds);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if (!in[v]) continue;
      float gm[8], bb[8] = {};
      Vec8<float>::load(a.pre_gamma + col[v], gm);
      if (a.pre_beta != nullptr) Vec8<float>::load(a.pre_beta + col[v], bb);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[v][e] = fmaf(y[v][e], gm[e], bb[e]);
      Vec8<T>::store(static_cast<T*>(a.u) + row * w + col[v], y[v]);
    }
  }
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------

// Sums over rows for the parameters: dgate by gate, the others over all rows.  A
// workgroup takes a span of rows, each team every TEAMS-th row of it, and keeps
// the sums of its columns in registers; the teams' are then added in LDS in a
// fixed order and the workgroup's written to a row of partial sums.  A second
// kernel adds those rows, also in a fixed order: results do not depend on timing.
// Spans hold whole gates (their dgate is written at once) or a part of one gate; with
// a gate a row, a row's dgate is written with the row.
template <typename T, int TEAM, int V, bool DROP, bool PRE>
__global__ __launch_bounds__(256) void couple_backward_kernel(CoupleArgs a) {
  constexpr int TEAMS = 256 / TEAM;
  // partial sums of the teams, one parameter at a time
  __shared__ float lds[TEAM > 64 ? 16 : 256 * V * 8];
  const int lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  const long w = a.width;
  bool col_in[V];
  int col[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    col[v] = 8 * (v * TEAM + lane);
    col_in[v] = col[v] < w;
  }
  const bool layer = a.layer != 0;
  const bool has_f = a.has_f != 0;
  Rng rng{};
  if (DROP) rng = load_rng(a.rng);
  float gpost[V][8] = {}, bpost[V][8] = {}, gpre[V][8] = {}, bpre[V][8] = {};

  // this workgroup's rows, by gate
  long gate0, gate1, part = 0, first, last;
  const bool gate_a_row = a.rows_per_gate == 1;
  if (gate_a_row) {
    gate0 = 0;
    gate1 = 1;
  } else if (a.chunks_per_gate > 1) {
    gate0 = blockIdx.x / a.chunks_per_gate;
    gate1 = gate0 + 1;
    part = blockIdx.x % a.chunks_per_gate;
  } else {
    gate0 = static_cast<long>(blockIdx.x) * a.gates_per_block;
    gate1 = gate0 + a.gates_per_block < a.gates ? gate0 + a.gates_per_block : a.gates;
  }

  // adds the teams' sums of one parameter and writes them to `to`
  auto flush = [&](float (&x)[V][8], float* to) {
    if constexpr (TEAMS > 1) {
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v) Vec8<float>::store(lds + team * (TEAM * V * 8) + col[v], x[v]);
      __syncthreads();
      for (int c = threadIdx.x; c < w; c += 256) {
        float s = 0.f;
#pragma unroll
        for (int t = 0; t < TEAMS; ++t) s += lds[t * (TEAM * V * 8) + c];
        to[c] = s;
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (col_in[v]) Vec8<float>::store(to + col[v], x[v]);
    }
  };

  for (long g = gate0; g < gate1; ++g) {
    float dg[V][8] = {};
    first = g * a.rows_per_gate;
    last = first + a.rows_per_gate;
    if (gate_a_row) {
      first = static_cast<long>(blockIdx.x) * a.rows_per_chunk;
      last = first + a.rows_per_chunk < a.rows ? first + a.rows_per_chunk : a.rows;
    } else if (a.chunks_per_gate > 1) {
      first += part * a.rows_per_chunk;
      if (first + a.rows_per_chunk < last) last = first + a.rows_per_chunk;
    }
    // every team makes as many rounds: the sums over a team wait for its waves
    for (long base = first; base < last; base += TEAMS) {
      const long row = base + team;
      const bool live = row < last;
      bool in[V];
#pragma unroll
      for (int v = 0; v < V; ++v) in[v] = live && col_in[v];
      float y[V][8], t[V][8];
      const long at = row * w;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        load_or_zero(static_cast<const T*>(a.y_in) + at + col[v], in[v], y[v]);
        load_or_zero(static_cast<const T*>(a.dy) + at + col[v], in[v], t[v]);
      }
      if constexpr (PRE) {
        float yn[V][8], h[V][8], s[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
          load_or_zero(static_cast<const T*>(a.du) + at + col[v], in[v], h[v]);
#pragma unroll
          for (int e = 0; e < 8; ++e) yn[v][e] = y[v][e];
        }
        const float r = unit<TEAM, V>(yn, in, layer, a.inv_width, a.eps, lds);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float gm[8] = {};
          if (col_in[v]) Vec8<float>::load(a.pre_gamma + col[v], gm);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            gpre[v][e] = fmaf(h[v][e], yn[v][e], gpre[v][e]);
            bpre[v][e] += h[v][e];
            h[v][e] *= gm[e];
            s[0] = fmaf(h[v][e], yn[v][e], s[0]);
            s[1] += h[v][e];
          }
        }
        TeamSum<TEAM>::sum(s, lds);
        const float c0 = s[0] * a.inv_width, c1 = layer ? s[1] * a.inv_width : 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            t[v][e] = fmaf(r, h[v][e] - yn[v][e] * c0 - c1, t[v][e]);
      }
      if (has_f) {
        float n[V][8], h[V][8], s[2] = {0.f, 0.f};
#pragma unroll
        for (int v = 0; v < V; ++v) load_or_zero(static_cast<const T*>(a.f) + at + col[v], in[v], n[v]);
        const float r = unit<TEAM, V>(n, in, layer, a.inv_width, a.eps, lds);
        const float* gate = a.gate + (gate_a_row ? row : g) * w;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (gate_a_row)
#pragma unroll
            for (int e = 0; e < 8; ++e) dg[v][e] = 0.f;
          if (!in[v]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) h[v][e] = 0.f;
            continue;
          }
          float gm[8], gg[8], bb[8] = {};
          Vec8<float>::load(a.post_gamma + col[v], gm);
          if (a.post_beta != nullptr) Vec8<float>::load(a.post_beta + col[v], bb);
          Vec8<float>::load(gate + col[v], gg);
          uint32_t bits[4];
          if (DROP) philox(rng, static_cast<uint64_t>(at + col[v]) >> 3, bits);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float nm = fmaf(n[v][e], gm[e], bb[e]), d = gg[e] * t[v][e];
            if (DROP) {
              const bool k = kept(bits, e, a.cut);
              nm = k ? nm * a.inv_keep : 0.f;
              d = k ? d * a.inv_keep : 0.f;
            }
            dg[v][e] = fmaf(t[v][e], nm, dg[v][e]);
            gpost[v][e] = fmaf(d, n[v][e], gpost[v][e]);
            bpost[v][e] += d;
            h[v][e] = d * gm[e];
            s[0] = fmaf(h[v][e], n[v][e], s[0]);
            s[1] += h[v][e];
            y[v][e] = fmaf(-gg[e], nm, y[v][e]) * a.inv_scale;
          }
        }
        TeamSum<TEAM>::sum(s, lds);
        const float c0 = s[0] * a.inv_width, c1 = layer ? s[1] * a.inv_width : 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (!in[v]) continue;
#pragma unroll
          for (int e = 0; e < 8; ++e) h[v][e] = r * (h[v][e] - n[v][e] * c0 - c1);
          Vec8<T>::store(static_cast<T*>(a.df) + at + col[v], h[v]);
          if (a.x_out != nullptr) Vec8<T>::store(static_cast<T*>(a.x_out) + at + col[v], y[v]);
          if (gate_a_row) Vec8<float>::store(a.dgate + at + col[v], dg[v]);
        }
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (!in[v]) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) t[v][e] *= a.scale;
        Vec8<T>::store(static_cast<T*>(a.dx) + at + col[v], t[v]);
      }
    }
    if (has_f && !gate_a_row)
      flush(dg, a.chunks_per_gate > 1 ? a.part_gate + static_cast<long>(blockIdx.x) * w : a.dgate + g * w);
  }
  const long block = blockIdx.x;
  if (has_f) {
    flush(gpost, a.part_post_gamma + block * w);
    if (a.post_beta != nullptr) flush(bpost, a.part_post_beta + block * w);
  }
  if (PRE) {
    flush(gpre, a.part_pre_gamma + block * w);
    if (a.pre_beta != nullptr) flush(bpre, a.part_pre_beta + block * w);
  }
}

// Adds rows of partial sums: out[o][c] = sum over r of part[o * rows + r][c], in 16
// interleaved sums a column, then joined.
struct JoinSet {
  const float* part;
  float* out;
  long outs, rows;
};
struct JoinArgs {
  JoinSet set[5];
  long width;
};

__global__ __launch_bounds__(1024) void couple_join_kernel(JoinArgs a) {
  __shared__ float lds[16][64];
  const JoinSet s = a.set[blockIdx.z];
  const long c = static_cast<long>(blockIdx.x) * 64 + (threadIdx.x & 63);
  const int lane = threadIdx.x >> 6;
  for (long o = blockIdx.y; o < s.outs; o += gridDim.y) {
    float v = 0.f;
    if (c < a.width)
      for (long r = lane; r < s.rows; r += 16) v += s.part[(o * s.rows + r) * a.width + c];
    lds[lane][threadIdx.x & 63] = v;
    __syncthreads();
    if (lane == 0 && c < a.width) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) t += lds[i][threadIdx.x & 63];
      s.out[o * a.width + c] = t;
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------

// y = residual + alpha m x, 8 elements a thread (a group of the generator): 16 or 32
// bytes a load.  The last, partial group goes element by element.
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, const T* residual, T* y, long n,
                                                      float factor, uint32_t cut, const uint64_t* rng_at) {
  const Rng rng = load_rng(rng_at);
  const long groups = (n + 7) >> 3;
  for (long g = static_cast<long>(blockIdx.x) * 256 + threadIdx.x; g < groups; g += static_cast<long>(gridDim.x) * 256) {
    uint32_t bits[4];
    const long at = g << 3;
    float v[8], r[8] = {};
    if (at + 8 <= n) {
      Vec8<T>::load(x + at, v);
      if (residual != nullptr) Vec8<T>::load(residual + at, r);
      philox(rng, static_cast<uint64_t>(g), bits);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = kept(bits, e, cut) ? fmaf(factor, v[e], r[e]) : r[e];
      Vec8<T>::store(y + at, v);
    } else {
      philox(rng, static_cast<uint64_t>(g), bits);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < n) {
          const float q = residual != nullptr ? load1(residual + at + e) : 0.f;
          store1(y + at + e, kept(bits, e, cut) ? fmaf(factor, load1(x + at + e), q) : q);
        }
    }
  }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

template <typename T, int TEAM, int V>
void forward_launch(const CoupleArgs& a, hipStream_t s) {
  const unsigned blocks = static_cast<unsigned>((a.rows + 256 / TEAM - 1) / (256 / TEAM));
  if (a.rng != nullptr)
    couple_forward_kernel<T, TEAM, V, true><<<blocks, 256, 0, s>>>(a);
  else
    couple_forward_kernel<T, TEAM, V, false><<<blocks, 256, 0, s>>>(a);
}

template <typename T, int TEAM, int V>
void backward_launch(const CoupleArgs& a, hipStream_t s) {
  const unsigned n = static_cast<unsigned>(a.blocks);
  if (a.rng != nullptr) {
    if (a.has_u)
      couple_backward_kernel<T, TEAM, V, true, true><<<n, 256, 0, s>>>(a);
    else
      couple_backward_kernel<T, TEAM, V, true, false><<<n, 256, 0, s>>>(a);
  } else {
    if (a.has_u)
      couple_backward_kernel<T, TEAM, V, false, true><<<n, 256, 0, s>>>(a);
    else
      couple_backward_kernel<T, TEAM, V, false, false><<<n, 256, 0, s>>>(a);
  }
}

// Lanes a row by its width: 8 elements a lane up to 64 lanes, then more chunks a
// lane, then the whole workgroup.
#define PETRA_BY_WIDTH(LAUNCH, T)                      \
  if (a.width <= 64) LAUNCH<T, 8, 1>(a, s);            \
  else if (a.width <= 256) LAUNCH<T, 32, 1>(a, s);     \
  else if (a.width <= 512) LAUNCH<T, 64, 1>(a, s);     \
  else if (a.width <= 1024) LAUNCH<T, 64, 2>(a, s);    \
  else if (a.width <= 2048) LAUNCH<T, 256, 1>(a, s);   \
  else if (a.width <= 4096) LAUNCH<T, 256, 2>(a, s);   \
  else LAUNCH<T, 256, 4>(a, s);

}  // namespace

void couple_plan(CoupleArgs& a) {
  // rows that a workgroup works on at once
  const long teams = a.width <= 64 ? 32 : a.width <= 256 ? 8 : a.width <= 1024 ? 4 : 1;
  // about two workgroups a CU: partial sums are a row of the width for each of them
  long span = (a.rows + 511) / 512;
  span = span < 1 ? teams : (span + teams - 1) / teams * teams;
  a.gates_per_block = a.chunks_per_gate = 1;
  a.rows_per_chunk = span;
  if (a.rows_per_gate == 1) {
    a.blocks = (a.rows + span - 1) / span;
  } else if (a.rows_per_gate > span) {
    const long chunks = (a.rows_per_gate + span - 1) / span;
    const long per = (a.rows_per_gate + chunks - 1) / chunks;
    a.rows_per_chunk = (per + teams - 1) / teams * teams;
    a.chunks_per_gate = (a.rows_per_gate + a.rows_per_chunk - 1) / a.rows_per_chunk;
    a.blocks = a.gates * a.chunks_per_gate;
  } else {
    a.gates_per_block = span / a.rows_per_gate;
    a.blocks = (a.gates + a.gates_per_block - 1) / a.gates_per_block;
  }
}

void couple_forward(const CoupleArgs& a, int dtype, hipStream_t s) {
  if (dtype == 1) {
    PETRA_BY_WIDTH(forward_launch, bf16_t)
  } else {
    PETRA_BY_WIDTH(forward_launch, float)
  }
}

void couple_backward(const CoupleArgs& a, int dtype, hipStream_t s) {
  if (a.blocks == 0) {
  } else if (dtype == 1) {
    PETRA_BY_WIDTH(backward_launch, bf16_t)
  } else {
    PETRA_BY_WIDTH(backward_launch, float)
  }
  JoinArgs j{};
  int n = 0;
  long most = 1;
  j.width = a.width;
  auto add = [&](const float* part, float* out, long outs, long rows) {
    j.set[n++] = {part, out, outs, rows};
    if (outs > most) most = outs;
  };
  if (a.has_f) {
    // without rows the sums are zeros, that of the one gate too
    if (a.blocks == 0) add(nullptr, a.dgate, a.gates, 0);
    if (a.chunks_per_gate > 1) add(a.part_gate, a.dgate, a.gates, a.chunks_per_gate);
    add(a.part_post_gamma, a.dpost_gamma, 1, a.blocks);
    if (a.post_beta != nullptr) add(a.part_post_beta, a.dpost_beta, 1, a.blocks);
  }
  if (a.has_u) {
    add(a.part_pre_gamma, a.dpre_gamma, 1, a.blocks);
    if (a.pre_beta != nullptr) add(a.part_pre_beta, a.dpre_beta, 1, a.blocks);
  }
  if (n > 0)
    couple_join_kernel<<<dim3(static_cast<unsigned>((a.width + 63) / 64),
                              static_cast<unsigned>(most < 1024 ? most : 1024), n),
                         1024, 0, s>>>(j);
}

void dropout(const void* x, const void* residual, void* y, long n, float factor, uint32_t cut,
             const uint64_t* rng, int dtype, hipStream_t s) {
  const long groups = (n + 7) >> 3, want = (groups + 255) / 256;
  const unsigned blocks = static_cast<unsigned>(want < 16384 ? want : 16384);
  if (dtype == 1)
    dropout_kernel<bf16_t><<<blocks, 256, 0, s>>>(static_cast<const bf16_t*>(x), static_cast<const bf16_t*>(residual),
                                                  static_cast<bf16_t*>(y), n, factor, cut, rng);
  else
    dropout_kernel<float><<<blocks, 256, 0, s>>>(static_cast<const float*>(x), static_cast<const float*>(residual),
                                                 static_cast<float*>(y), n, factor, cut, rng);
}

}  // namespace petra
