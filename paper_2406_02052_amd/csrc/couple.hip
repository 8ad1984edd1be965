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
// backward.  A row stays in registers from its load to its store, 8 elements a lane
// of the team that holds it, so each tensor crosses memory once; the row's sums are
// taken in fp32, in registers and, where a team has several waves, through LDS.  The
// variance is the mean of squared differences from the mean, a second pass over
// registers.
#include "common.h"
#include "ops.h"
#include "philox.h"

namespace petra {

namespace {

// ---------------------------------------------------------------------------
// rows and teams
// ---------------------------------------------------------------------------

// A team of TEAM lanes holds a row, lane l its elements 8 l .. 8 l + 7.  A workgroup
// has THREADS / TEAM teams.
template <int TEAM>
struct Team {
  static constexpr int THREADS = TEAM > 256 ? TEAM : 256, TEAMS = THREADS / TEAM;
  static constexpr int WAVES = TEAM > 64 ? TEAM / 64 : 1;
  static constexpr int LDS = WAVES > 1 ? 4 * (THREADS / 64) : 1;   // floats: two sums, twice

  template <int DPP>
  static __device__ __forceinline__ float swapped(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), DPP, 0xF, 0xF, false));
  }

  // Sums of N (at most 2) values over the team, in every lane.  `turn` alternates: a wave that
  // writes one half of lds has seen every wave leave it, at the barrier for the other half.
  template <int N>
  static __device__ __forceinline__ void sum(float (&x)[N], float* lds, int& turn) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (TEAM < 16) {
        if constexpr (TEAM >= 2) x[i] += swapped<0xB1>(x[i]);    // [1,0,3,2]
        if constexpr (TEAM >= 4) x[i] += swapped<0x4E>(x[i]);    // [2,3,0,1]
        if constexpr (TEAM >= 8) x[i] += swapped<0x141>(x[i]);   // half mirror
      } else {
        x[i] = sum16(x[i]);
        if constexpr (TEAM >= 32) x[i] = sum_quarters(x[i]);
        if constexpr (TEAM >= 64) x[i] = sum_halves(x[i]);
      }
    }
    if constexpr (WAVES > 1) {
      const int wave = threadIdx.x >> 6, first = wave / WAVES * WAVES;
      float* const to = lds + turn * (THREADS / 64) * 2;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) to[wave * 2 + i] = x[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[i] = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) x[i] += to[(first + w) * 2 + i];
      }
    }
  }
};

// Normalises N (1 or 2) rows in place, z to z^; r: 1 / deviation.  Lanes past the row hold zeros
// and keep them.
template <int TEAM, bool LAYER, int N>
__device__ __forceinline__ void unit(float (&z)[N][8], float (&r)[N], bool in, float inv_w, float eps,
                                     float* lds, int& turn) {
  float s[N];
  if constexpr (LAYER) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      s[n] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s[n] += z[n][e];
    }
    Team<TEAM>::sum(s, lds, turn);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) z[n][e] = in ? z[n][e] - s[n] * inv_w : 0.f;
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    s[n] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s[n] = fmaf(z[n][e], z[n][e], s[n]);
  }
  Team<TEAM>::sum(s, lds, turn);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    r[n] = rsqrtf(s[n] * inv_w + eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) z[n][e] *= r[n];
  }
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

// 2 reads and 2 writes an element and nothing between them but the row's sums: 16384 x 4096 bf16
// with dropout in 113 us, 4.7 TB/s (a copy of that size: 5.3).
template <typename T, int TEAM, bool LAYER, bool DROP>
__global__ __launch_bounds__(Team<TEAM>::THREADS) void couple_forward_kernel(CoupleArgs a) {
  using Tm = Team<TEAM>;
  __shared__ float lds[Tm::LDS];
  int turn = 0;
  const int col = 8 * (threadIdx.x % TEAM);
  const long w = a.width;
  const long row = a.row0 + static_cast<long>(blockIdx.x) * Tm::TEAMS + threadIdx.x / TEAM;
  const bool in = row < a.rows && col < w;
  const long at = row * w + col;
  float y[1][8], r[1];
  load_or_zero(static_cast<const T*>(a.x) + at, in, y[0]);
  if (a.f != nullptr) {
    float n[1][8];
    load_or_zero(static_cast<const T*>(a.f) + at, in, n[0]);
    uint32_t bits[4];
    if (DROP) philox(load_rng(a.rng), static_cast<uint64_t>(at) >> 3, bits);
    unit<TEAM, LAYER>(n, r, in, a.inv_width, a.eps, lds, turn);
    if (in) {
      float gm[8], gg[8], bb[8] = {};
      Vec8<float>::load(a.post_gamma + col, gm);
      if (a.post_beta != nullptr) Vec8<float>::load(a.post_beta + col, bb);
      Vec8<float>::load(a.gate + row / a.rows_per_gate * w + col, gg);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float t = fmaf(n[0][e], gm[e], bb[e]);
        if (DROP) t = kept(bits, e, a.cut) ? t * a.inv_keep : 0.f;
        y[0][e] = quant(fmaf(gg[e], t, a.scale * y[0][e]), static_cast<const T*>(nullptr));
      }
      Vec8<T>::store(static_cast<T*>(a.y) + at, y[0]);
    }
  }
  if (a.u != nullptr) {
    unit<TEAM, LAYER>(y, r, in, a.inv_width, a.eps, lds, turn);
    if (in) {
      float gm[8], bb[8] = {};
      Vec8<float>::load(a.pre_gamma + col, gm);
      if (a.pre_beta != nullptr) Vec8<float>::load(a.pre_beta + col, bb);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[0][e] = fmaf(y[0][e], gm[e], bb[e]);
      Vec8<T>::store(static_cast<T*>(a.u) + at, y[0]);
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
// a gate a row, a row's dgate is written with the row.  The next row's tensors are
// asked for before this one's sums, which wait for the team's waves.  All teams of a
// workgroup are at one gate: gates of fewer rows than it has teams leave some idle (524288 x
// 64 bf16, 32 teams: 1012 us with 2 rows a gate, 531 with 4, 172 with 16; one gate 100, a
// gate a row 153).
// FULL: a layer norm or a beta (the sums that only those need).
// 4 reads and 3 writes an element: 16384 x 2048 bf16 with dropout in 95 us and 4.8 for the second
// kernel, 4.7 TB/s; without the next row fetched ahead, and with a barrier more for each sum, 188.
template <typename T, int TEAM, bool FULL, bool DROP, bool PRE>
__global__ __launch_bounds__(Team<TEAM>::THREADS) void couple_backward_kernel(CoupleArgs a) {
  using Tm = Team<TEAM>;
  constexpr int TEAMS = Tm::TEAMS, THREADS = Tm::THREADS;
  // 1024 lanes have 128 registers each: no room for the next row, nor for the parameters.  The sums alone
  // leave too few: all but the forms without u, layer norm and beta spill, up to 122 registers (4096 x 8192
  // bf16: rms 174 us, layer 434, memory's share 89; 8192 x 4096, by 512 lanes, 105)
  constexpr bool LEAN = TEAM == 1024;
  // partial sums of the teams, one parameter at a time
  __shared__ float joined[TEAMS > 1 ? THREADS * 8 : 1];
  __shared__ float lds[Tm::LDS];
  int turn = 0;
  const int team = threadIdx.x / TEAM, col = 8 * (threadIdx.x % TEAM);
  const long w = a.width;
  const bool col_in = col < w;
  const bool layer = FULL && a.layer != 0;
  const bool has_f = a.has_f != 0;
  Rng rng{};
  if (DROP) rng = load_rng(a.rng);
  float gpost[8] = {}, bpost[8] = {}, gpre[8] = {}, bpre[8] = {};

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
  auto flush = [&](const float (&x)[8], float* to) {
    if constexpr (TEAMS > 1) {
      __syncthreads();
      Vec8<float>::store(joined + team * (TEAM * 8) + col, x);
      __syncthreads();
      for (int c = threadIdx.x; c < w; c += THREADS) {
        float s = 0.f;
#pragma unroll
        for (int t = 0; t < TEAMS; ++t) s += joined[t * (TEAM * 8) + c];
        to[c] = s;
      }
    } else if (col_in) {
      Vec8<float>::store(to + col, x);
    }
  };

  float post_gamma[8] = {}, post_beta[8] = {}, pre_gamma[8] = {};
  auto load_post = [&] {
    Vec8<float>::load(a.post_gamma + col, post_gamma);
    if (FULL && a.post_beta != nullptr) Vec8<float>::load(a.post_beta + col, post_beta);
  };
  if (col_in && !LEAN) {
    if (has_f) load_post();
    if (PRE) Vec8<float>::load(a.pre_gamma + col, pre_gamma);
  }

  Raw8<T> next[4];
  auto fetch = [&](long row, bool live) {
    const long at = row * w + col;
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i].zero();
    if (!live || !col_in) return;
    next[0].load(static_cast<const T*>(a.y_in) + at);
    next[1].load(static_cast<const T*>(a.dy) + at);
    if (PRE) next[2].load(static_cast<const T*>(a.du) + at);
    if (has_f) next[3].load(static_cast<const T*>(a.f) + at);
  };

  for (long g = gate0; g < gate1; ++g) {
    float dg[8] = {};
    first = g * a.rows_per_gate;
    last = first + a.rows_per_gate;
    if (gate_a_row) {
      first = static_cast<long>(blockIdx.x) * a.rows_per_chunk;
      last = first + a.rows_per_chunk < a.rows ? first + a.rows_per_chunk : a.rows;
    } else if (a.chunks_per_gate > 1) {
      first += part * a.rows_per_chunk;
      if (first + a.rows_per_chunk < last) last = first + a.rows_per_chunk;
    }
    float gate[8] = {};
    if (!LEAN && has_f && !gate_a_row && col_in) Vec8<float>::load(a.gate + g * w + col, gate);
    if (!LEAN) fetch(first + team, first + team < last);
    // every team makes as many rounds: the sums over a team wait for its waves
    for (long base = first; base < last; base += TEAMS) {
      const long row = base + team;
      const bool in = row < last && col_in;
      const long at = row * w + col;
      if (LEAN) fetch(row, row < last);
      float y[8], t[8], z[2][8], h[8], r[2];   // z: y^ and f^
      next[0].to_f32(y);
      next[1].to_f32(t);
      if (PRE) next[2].to_f32(h);
      next[0].to_f32(z[0]);
      next[3].to_f32(z[1]);
      if (has_f && gate_a_row && in) Vec8<float>::load(a.gate + at, gate);
      if (!LEAN && base + TEAMS < last) fetch(row + TEAMS, row + TEAMS < last);
      if (layer)
        unit<TEAM, true>(z, r, in, a.inv_width, a.eps, lds, turn);
      else
        unit<TEAM, false>(z, r, in, a.inv_width, a.eps, lds, turn);
      if constexpr (PRE) {
        if (LEAN && col_in) Vec8<float>::load(a.pre_gamma + col, pre_gamma);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          gpre[e] = fmaf(h[e], z[0][e], gpre[e]);
          if (FULL) bpre[e] += h[e];
          h[e] *= pre_gamma[e];
          s[0] = fmaf(h[e], z[0][e], s[0]);
          s[1] += h[e];
        }
        Tm::sum(s, lds, turn);
        const float c0 = s[0] * a.inv_width, c1 = layer ? s[1] * a.inv_width : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = fmaf(r[0], h[e] - z[0][e] * c0 - c1, t[e]);
      }
      if (has_f) {
        if (LEAN && col_in) {
          load_post();
          if (!gate_a_row) Vec8<float>::load(a.gate + g * w + col, gate);
        }
        float s[2] = {0.f, 0.f};
        uint32_t bits[4];
        if (DROP) philox(rng, static_cast<uint64_t>(at) >> 3, bits);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float nm = z[1][e] * post_gamma[e], d = gate[e] * t[e];
          if (FULL) nm += post_beta[e];
          if (DROP) {
            const bool k = kept(bits, e, a.cut);
            nm = k ? nm * a.inv_keep : 0.f;
            d = k ? d * a.inv_keep : 0.f;
          }
          if (!in) d = 0.f, nm = 0.f;   // past the row: t is (nothing - mean) there
          dg[e] = gate_a_row ? t[e] * nm : fmaf(t[e], nm, dg[e]);
          gpost[e] = fmaf(d, z[1][e], gpost[e]);
          if (FULL) bpost[e] += d;
          h[e] = d * post_gamma[e];
          s[0] = fmaf(h[e], z[1][e], s[0]);
          s[1] += h[e];
          y[e] = fmaf(-gate[e], nm, y[e]) * a.inv_scale;
        }
        Tm::sum(s, lds, turn);
        const float c0 = s[0] * a.inv_width, c1 = layer ? s[1] * a.inv_width : 0.f;
        if (in) {
#pragma unroll
          for (int e = 0; e < 8; ++e) h[e] = r[1] * (h[e] - z[1][e] * c0 - c1);
          Vec8<T>::store(static_cast<T*>(a.df) + at, h);
          if (a.x_out != nullptr) Vec8<T>::store(static_cast<T*>(a.x_out) + at, y);
          if (gate_a_row) Vec8<float>::store(a.dgate + at, dg);
        }
      }
      if (in) {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] *= a.scale;
        Vec8<T>::store(static_cast<T*>(a.dx) + at, t);
      }
    }
    if (has_f && !gate_a_row)
      flush(dg, a.chunks_per_gate > 1 ? a.part_gate + static_cast<long>(blockIdx.x) * w : a.dgate + g * w);
  }
  const long block = blockIdx.x;
  if (has_f) {
    flush(gpost, a.part_post_gamma + block * w);
    if (FULL && a.post_beta != nullptr) flush(bpost, a.part_post_beta + block * w);
  }
  if (PRE) {
    flush(gpre, a.part_pre_gamma + block * w);
    if (FULL && a.pre_beta != nullptr) flush(bpre, a.part_pre_beta + block * w);
  }
}

// Adds rows of partial sums: out[o][c] = sum over r of part[o * rows + r][c], in 16
// interleaved sums a column, then joined.  blockIdx.y counts the outputs of all sets.
struct JoinSet {
  const float* part;
  float* out;
  long outs, rows;
};
struct JoinArgs {
  JoinSet set[6];
  int sets;
  long width;
};

__global__ __launch_bounds__(1024) void couple_join_kernel(JoinArgs a) {
  __shared__ float lds[16][64];
  const long c = static_cast<long>(blockIdx.x) * 64 + (threadIdx.x & 63);
  const int lane = threadIdx.x >> 6;
  long o = blockIdx.y;
  int n = 0;
  while (n + 1 < a.sets && o >= a.set[n].outs) o -= a.set[n++].outs;
  const JoinSet s = a.set[n];
  float v = 0.f;
  if (c < a.width) {
    const float* p = s.part + (o * s.rows) * a.width + c;
#pragma unroll 8
    for (long r = lane; r < s.rows; r += 16) v += p[r * a.width];
  }
  lds[lane][threadIdx.x & 63] = v;
  __syncthreads();
  if (lane == 0 && c < a.width) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += lds[i][threadIdx.x & 63];
    s.out[o * a.width + c] = t;
  }
}

// ---------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------

// y = residual + alpha m x, 8 elements a thread (a group of the generator): 16 or 32
// bytes a load.  Bound by memory, the generator's products beside it: 2^27 bf16 with
// a residual in 146 us, 5.5 TB/s.  The last, partial group goes element by element.
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, const T* residual, T* y, long n,
                                                      float factor, uint32_t cut, const uint64_t* rng_at) {
  const Rng rng = rng_at != nullptr ? load_rng(rng_at) : Rng{};   // (nothing is dropped without)
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

template <typename T, int TEAM>
void forward_launch(const CoupleArgs& a, hipStream_t s) {
  using Tm = Team<TEAM>;
  // a grid has fewer than 2^32 lanes: more rows than that holds go in several launches
  const long most = static_cast<long>(1 << 20) * Tm::TEAMS;
  CoupleArgs part = a;
  for (part.row0 = 0; part.row0 < a.rows; part.row0 += most) {
    const long rows = a.rows - part.row0 < most ? a.rows - part.row0 : most;
    const unsigned n = static_cast<unsigned>((rows + Tm::TEAMS - 1) / Tm::TEAMS);
    if (a.layer) {
      if (a.rng != nullptr) couple_forward_kernel<T, TEAM, true, true><<<n, Tm::THREADS, 0, s>>>(part);
      else couple_forward_kernel<T, TEAM, true, false><<<n, Tm::THREADS, 0, s>>>(part);
    } else {
      if (a.rng != nullptr) couple_forward_kernel<T, TEAM, false, true><<<n, Tm::THREADS, 0, s>>>(part);
      else couple_forward_kernel<T, TEAM, false, false><<<n, Tm::THREADS, 0, s>>>(part);
    }
  }
}

template <typename T, int TEAM, bool FULL>
void backward_by(const CoupleArgs& a, hipStream_t s) {
  using Tm = Team<TEAM>;
  const unsigned n = static_cast<unsigned>(a.blocks);
  if (a.rng != nullptr) {
    if (a.has_u) couple_backward_kernel<T, TEAM, FULL, true, true><<<n, Tm::THREADS, 0, s>>>(a);
    else couple_backward_kernel<T, TEAM, FULL, true, false><<<n, Tm::THREADS, 0, s>>>(a);
  } else {
    if (a.has_u) couple_backward_kernel<T, TEAM, FULL, false, true><<<n, Tm::THREADS, 0, s>>>(a);
    else couple_backward_kernel<T, TEAM, FULL, false, false><<<n, Tm::THREADS, 0, s>>>(a);
  }
}

template <typename T, int TEAM>
void backward_launch(const CoupleArgs& a, hipStream_t s) {
  if (a.layer || a.post_beta != nullptr || a.pre_beta != nullptr) backward_by<T, TEAM, true>(a, s);
  else backward_by<T, TEAM, false>(a, s);
}

// Lanes a row: the fewest powers of two that hold it, 8 elements each (2159903 x 8 bf16 with a gate a row:
// 88 us backward, 242 by 8 lanes).
int team(int width) {
  int n = 1;
  while (8 * n < width) n *= 2;
  return n;
}

#define PETRA_BY_WIDTH(LAUNCH, T)             \
  switch (team(a.width)) {                    \
    case 1: LAUNCH<T, 1>(a, s); break;        \
    case 2: LAUNCH<T, 2>(a, s); break;        \
    case 4: LAUNCH<T, 4>(a, s); break;        \
    case 8: LAUNCH<T, 8>(a, s); break;        \
    case 16: LAUNCH<T, 16>(a, s); break;      \
    case 32: LAUNCH<T, 32>(a, s); break;      \
    case 64: LAUNCH<T, 64>(a, s); break;      \
    case 128: LAUNCH<T, 128>(a, s); break;    \
    case 256: LAUNCH<T, 256>(a, s); break;    \
    case 512: LAUNCH<T, 512>(a, s); break;    \
    default: LAUNCH<T, 1024>(a, s); break;    \
  }

}  // namespace

void couple_plan(CoupleArgs& a) {
  // rows that a workgroup works on at once
  const int lanes = team(a.width);
  const long teams = lanes < 256 ? 256 / lanes : 1;
  // two workgroups a CU (one of 1024 lanes): partial sums are a row of the width for each of them, and a count
  // that the 256 CUs do not share evenly ends late (16384 x 2048 bf16: 512 workgroups 95 us, 256 115, 640
  // 115, 768 112, 1024 97 and a longer join)
  const long most = lanes <= 512 ? 512 : 256;
  long span = (a.rows + most - 1) / most;
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
  long outs = 0;
  j.width = a.width;
  auto add = [&](const float* part, float* out, long n, long rows) {
    if (n == 0) return;
    j.set[j.sets++] = {part, out, n, rows};
    outs += n;
  };
  if (a.has_f) {
    add(a.part_post_gamma, a.dpost_gamma, 1, a.blocks);
    if (a.post_beta != nullptr) add(a.part_post_beta, a.dpost_beta, 1, a.blocks);
  }
  if (a.has_u) {
    add(a.part_pre_gamma, a.dpre_gamma, 1, a.blocks);
    if (a.pre_beta != nullptr) add(a.part_pre_beta, a.dpre_beta, 1, a.blocks);
  }
  if (a.has_f) {
    // without rows the sums are zeros, that of the one gate too
    if (a.blocks == 0) add(nullptr, a.dgate, a.gates, 0);
    if (a.chunks_per_gate > 1) add(a.part_gate, a.dgate, a.gates, a.chunks_per_gate);
  }
  // (gates are joined where each has more rows than a workgroup's share, a 512th of all: fewer than 512)
  if (j.sets > 0)
    couple_join_kernel<<<dim3(static_cast<unsigned>((a.width + 63) / 64), static_cast<unsigned>(outs)), 1024, 0, s>>>(j);
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
