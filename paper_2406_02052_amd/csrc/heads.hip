// Norms of query and key heads with the rotation by their tokens' positions, and
// their backward.
//
//   z = n(x) gamma (+ beta),  (y_a, y_b) = (z_a cos t - z_b sin t, z_a sin t + z_b cos t)
// for the pairs (a, b) of a head's channels, t = freq_i position[axis_i]; n is over
// the head's channels.  Backward, with g the rotation of dy by -t:
//   dgamma = sum g x^,  dbeta = sum g,  dx = r (g gamma - x^ mean(g gamma x^) (- mean(g gamma)))
//
// Bound by memory: a read and a write an element forward, two and one backward.
//
// Angles are held in turns, as 64-bit fractions: position times round(2^64 freq / 2 pi),
// whose wrap is the wrap of the angle, so that far positions lose nothing (an fp32
// product would be off by 0.1 at 10^6).  The upper 32 bits give the quarter turn and a rest of at
// most pi / 4, whose sine and cosine are their Taylor polynomials of degree 9 and 10 (the
// next terms are 2e-9 and 1e-10).
#include <type_traits>

#include "common.h"
#include "ops.h"

namespace petra {

namespace {

constexpr int THREADS = 256;

// cos and sin of u / 2^32 turns.
__device__ __forceinline__ void turn(uint32_t u, float& c, float& s) {
  const uint32_t q = (u + 0x20000000u) >> 30;
  const float x = static_cast<float>(static_cast<int32_t>(u - (q << 30))) * 1.46291807926715968105e-9f;   // 2 pi / 2^32
  const float x2 = x * x;
  float sn = fmaf(x2, 2.75573192239858907e-6f, -1.98412698412698413e-4f);
  sn = fmaf(x2, sn, 8.33333333333333333e-3f);
  sn = fmaf(x2, sn, -1.66666666666666667e-1f);
  sn = fmaf(x * x2, sn, x);
  float cs = fmaf(x2, -2.75573192239858907e-7f, 2.48015873015873016e-5f);
  cs = fmaf(x2, cs, -1.38888888888888889e-3f);
  cs = fmaf(x2, cs, 4.16666666666666667e-2f);
  cs = fmaf(x2, cs, -0.5f);
  cs = fmaf(x2, cs, 1.f);
  const bool odd = (q & 1) != 0;
  const float a = odd ? sn : cs, b = odd ? cs : sn;
  c = (q == 1 || q == 2) ? -a : a;
  s = (q & 2) ? -b : b;
}

// Sum over the LANES lanes (a power of two, at most 16) of a team, in every lane.
template <int LANES>
__device__ __forceinline__ float team_sum(float v) {
  if constexpr (LANES == 16) return sum16(v);
  auto swapped = [](float x, auto dpp) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(dpp)::value, 0xF, 0xF, false));
  };
  if constexpr (LANES >= 2) v += swapped(v, std::integral_constant<int, 0xB1>{});    // [1,0,3,2]
  if constexpr (LANES >= 4) v += swapped(v, std::integral_constant<int, 0x4E>{});    // [2,3,0,1]
  if constexpr (LANES >= 8) v += swapped(v, std::integral_constant<int, 0x141>{});   // half mirror
  return v;
}

// Sum over a wave's teams, of the lanes at one place in theirs: rows of 16 lanes turned by multiples of a team, then the rows.
template <int LANES>
__device__ __forceinline__ float over_teams(float v) {
  auto turned = [](float x, auto dpp) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(dpp)::value, 0xF, 0xF, false));
  };
  if constexpr (LANES <= 8) v += turned(v, std::integral_constant<int, 0x128>{});
  if constexpr (LANES <= 4) v += turned(v, std::integral_constant<int, 0x124>{});
  if constexpr (LANES <= 2) v += turned(v, std::integral_constant<int, 0x122>{});
  if constexpr (LANES <= 1) v += turned(v, std::integral_constant<int, 0x121>{});
  return sum_halves(sum_quarters(v));
}

// C consecutive elements (4 or 8) as they lie in memory.
template <typename T, int C> struct Chunk;
template <> struct Chunk<bf16_t, 8> {
  uint4 w;
  __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float* o) const {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) o[2 * i] = __uint_as_float(v[i] << 16), o[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
  }
  static __device__ __forceinline__ void store(bf16_t* p, const float* o) { Vec8<bf16_t>::store(p, o); }
};
template <> struct Chunk<bf16_t, 4> {
  uint2 w;
  __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void get(float* o) const {
    o[0] = __uint_as_float(w.x << 16), o[1] = __uint_as_float(w.x & 0xffff0000u);
    o[2] = __uint_as_float(w.y << 16), o[3] = __uint_as_float(w.y & 0xffff0000u);
  }
  static __device__ __forceinline__ void store(bf16_t* p, const float* o) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
  }
};
template <int C> struct Chunk<float, C> {
  float4 w[C / 4];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < C / 4; ++i) w[i] = reinterpret_cast<const float4*>(p)[i];
  }
  __device__ __forceinline__ void get(float* o) const {
#pragma unroll
    for (int i = 0; i < C / 4; ++i) o[4 * i] = w[i].x, o[4 * i + 1] = w[i].y, o[4 * i + 2] = w[i].z, o[4 * i + 3] = w[i].w;
  }
  static __device__ __forceinline__ void store(float* p, const float* o) {
#pragma unroll
    for (int i = 0; i < C / 4; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
  }
};

// What a lane of a head's team holds: two chunks of C channels, at a and b.  With halves the channels of a
// pair are in the two chunks, and a lane past the pairs has two chunks in a row; with neighbours all lanes have.
template <int C, bool HALVES>
struct Place {
  int a, b;                  // (the lane's C pairs begin at C lane in either layout)
  bool in_a, in_b, turn_a, turn_b;
  __device__ __forceinline__ Place(int lane, int dim, int pairs) {
    if constexpr (HALVES) {
      const int n = pairs / C;
      turn_a = turn_b = lane < n;
      a = lane < n ? lane * C : 2 * pairs + (lane - n) * 2 * C;
      b = lane < n ? pairs + lane * C : a + C;
    } else {
      a = lane * 2 * C;
      b = a + C;
      turn_a = a < 2 * pairs;
      turn_b = b < 2 * pairs;
    }
    in_a = a < dim;
    in_b = b < dim;
  }
};

// The angles of a wave's tokens.  Each is formed by one lane, an entry (token, pair) each, and read by all heads' teams from LDS:
// forming them in every team takes as long as memory does (16384 tokens x 20 heads of 128 bf16: 46 us in all).
template <int C>
struct Angles {
  int count, split;          // entries of the wave; 2^16 / pairs, rounded up
  int first;                 // position of the lane's first entry of the next tokens
  float c[C], s[C];

  __device__ __forceinline__ void begin(const HeadsArgs& a, int tokens) {
    count = tokens * a.pairs;
    split = a.pairs > 0 ? (65535 + a.pairs) / a.pairs : 0;
    first = 0;
  }
  // Entry e's token of the wave (e < 512: exact) and pair.
  __device__ __forceinline__ int token(int e) const { return (e * split) >> 16; }
  __device__ __forceinline__ int position(const HeadsArgs& a, long base, int e) const {
    const int t = token(e), pair = e - t * a.pairs;
    const long at = base + t;
    if (e >= count || at >= a.tokens) return 0;
    const int axis = a.axes == 1 ? 0 : (a.axes4[pair >> 3] >> (pair % 8 * 4)) & 15;
    return a.positions != nullptr ? a.positions[axis * a.tokens + at] : static_cast<int>(static_cast<uint32_t>(at) % a.len);
  }
  // Asks for the first position of the tokens from `base` on: where heads fill a wave it is all.
  __device__ __forceinline__ void fetch(const HeadsArgs& a, long base) { first = position(a, base, threadIdx.x & 63); }
  // Forms the angles of the tokens from `base` on, whose first positions have been asked for.
  __device__ __forceinline__ void form(const HeadsArgs& a, long base, const uint64_t* freq, float2* table) const {
    __builtin_amdgcn_wave_barrier();
    int v = first;
#pragma unroll 1
    for (int k = 0; 64 * k < count; ++k) {
      const int e = 64 * k + (threadIdx.x & 63);
      if (k > 0) v = position(a, base, e);
      const int t = token(e);
      const uint64_t f = freq[e < count ? e - t * a.pairs : 0];
      const uint32_t lo = static_cast<uint32_t>(f), hi = static_cast<uint32_t>(f >> 32), u = static_cast<uint32_t>(v);
      float2 r;
      turn(__umulhi(u, lo) + u * hi - (v < 0 ? lo : 0u), r.x, r.y);
      table[e] = r;
    }
    __builtin_amdgcn_wave_barrier();
  }
  // Those of the lane's pairs, of the wave's token `token`.
  __device__ __forceinline__ void read(const HeadsArgs& a, const float2* table, int token, int lane) {
#pragma unroll
    for (int j = 0; j < C; ++j) {
      const float2 t = lane * C + j < a.pairs ? table[token * a.pairs + lane * C + j] : make_float2(1.f, 0.f);
      c[j] = t.x;
      s[j] = t.y;
    }
  }
};

// Rotates the lane's channels in place, by the angle or (BACK) against it.
template <int C, bool HALVES, bool BACK>
__device__ __forceinline__ void rotate(float (&x)[2 * C], const Angles<C>& t, const Place<C, HALVES>& p) {
#pragma unroll
  for (int j = 0; j < C; ++j) {
    const int i = HALVES ? j : 2 * j, k = HALVES ? C + j : 2 * j + 1;
    const float s = BACK ? -t.s[j] : t.s[j], a = x[i], b = x[k];
    const float u = fmaf(a, t.c[j], -b * s), v = fmaf(a, s, b * t.c[j]);
    const bool on = HALVES ? p.turn_a : (j < C / 2 ? p.turn_a : p.turn_b);
    x[i] = on ? u : a;
    x[k] = on ? v : b;
  }
}

// Normalises the lane's channels of a head in place; returns 1 / the deviation.
template <int C, int LANES>
__device__ __forceinline__ float unit(float (&x)[2 * C], bool layer, bool in_a, bool in_b, float inv_dim, float eps) {
  if (layer) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 2 * C; ++e) s += x[e];
    const float mean = team_sum<LANES>(s) * inv_dim;
#pragma unroll
    for (int e = 0; e < 2 * C; ++e) x[e] = (e < C ? in_a : in_b) ? x[e] - mean : 0.f;
  }
  float q = 0.f;
#pragma unroll
  for (int e = 0; e < 2 * C; ++e) q = fmaf(x[e], x[e], q);
  const float r = rsqrtf(fmaf(team_sum<LANES>(q), inv_dim, eps));
#pragma unroll
  for (int e = 0; e < 2 * C; ++e) x[e] *= r;
  return r;
}

// How a workgroup's lanes lie over tokens and heads: a team of LANES lanes a head, 2^head_bits heads and the
// rest of a wave's teams tokens beside each other.  A wave takes a group of tokens and `rounds` times its heads, so
// that a token's angles are formed once for them.
struct Lane {
  int lane, head, token;     // token: of the wave's
  int tokens;                // of a wave
  long base, step;           // the wave's first token, and how far the next group is
};
template <int LANES>
__device__ __forceinline__ Lane my_lane(const HeadsPart& p, int block) {
  const int in_wave = (threadIdx.x & 63) / LANES, wave = threadIdx.x >> 6;
  Lane l;
  l.tokens = (64 / LANES) >> p.head_bits;
  l.lane = threadIdx.x & (LANES - 1);
  l.head = in_wave & ((1 << p.head_bits) - 1);
  const int group = block / p.splits, split = block - group * p.splits;
  l.head += split * (p.rounds << p.head_bits);
  l.token = in_wave >> p.head_bits;
  l.base = (static_cast<long>(group) * (THREADS / 64) + __builtin_amdgcn_readfirstlane(wave)) * l.tokens;
  l.step = static_cast<long>(p.groups) * (THREADS / 64) * l.tokens;
  return l;
}

// 16384 tokens of 16 + 4 heads of 128 bf16 in 39 us, 4.3 TB/s (30 from the last cache).
template <typename T, int C, int LANES, bool HALVES>
__global__ __launch_bounds__(THREADS) void heads_forward_kernel(HeadsArgs a) {
  __shared__ uint64_t freq[HEADS_PAIRS];
  __shared__ float2 turns[THREADS / 64][64 * C];
  if (threadIdx.x < HEADS_PAIRS) freq[threadIdx.x] = a.freq[threadIdx.x];
  __syncthreads();
  const bool second = static_cast<int>(blockIdx.x) >= a.part[0].blocks;
  const HeadsPart& p = a.part[second];
  const Lane l = my_lane<LANES>(p, blockIdx.x - (second ? a.part[0].blocks : 0));
  const Place<C, HALVES> at(l.lane, a.dim, a.pairs);
  Angles<C> angles;
  angles.begin(a, l.tokens);
  float2* const mine_turns = turns[threadIdx.x >> 6];
  float gamma[2 * C];
#pragma unroll
  for (int e = 0; e < 2 * C; ++e) gamma[e] = 1.f;
  if (p.gamma != nullptr) {
    Chunk<float, C> t;
    if (at.in_a) t.load(p.gamma + at.a), t.get(gamma);
    if (at.in_b) t.load(p.gamma + at.b), t.get(gamma + C);
  }
  // the next head's channels are asked for before these are worked on
  struct Item {
    Chunk<T, C> a, b;
    uint32_t row, index;     // batch row, token of it
    long base;               // the wave's first token: all its lanes take as many turns
    bool in;
    int round;
  } next{};
  auto fetch = [&](long base, int round) {
    const long token = base + l.token;
    if (round == 0 && base < a.tokens) {
      next.row = static_cast<uint32_t>(token) / a.len;
      next.index = static_cast<uint32_t>(token) - next.row * a.len;
      angles.fetch(a, base);
    }
    next.base = base;
    next.round = round;
    const int h = l.head + (round << p.head_bits);
    const T* const x = static_cast<const T*>(p.x) + next.row * p.x_stride[0] + next.index * p.x_stride[1] + h * p.x_stride[2];
    next.a = next.b = Chunk<T, C>{};
    const bool in = next.in = token < a.tokens && h < p.heads;
    if (in && at.in_a) next.a.load(x + at.a);
    if (in && at.in_b) next.b.load(x + at.b);
  };
  fetch(l.base, 0);
  while (next.base < a.tokens) {
    const Item now = next;
    if (now.round == 0) {
      angles.form(a, now.base, freq, mine_turns);
      angles.read(a, mine_turns, l.token, l.lane);
    }
    const bool more = now.round + 1 < p.rounds;
    fetch(more ? now.base : now.base + l.step, more ? now.round + 1 : 0);
    float x[2 * C];
    now.a.get(x);
    now.b.get(x + C);
    if (p.gamma != nullptr) {
      unit<C, LANES>(x, a.layer, at.in_a, at.in_b, a.inv_dim, a.eps);
#pragma unroll
      for (int e = 0; e < 2 * C; ++e) x[e] *= gamma[e];
      if (p.beta != nullptr) {
        float beta[2 * C] = {};
        Chunk<float, C> t;
        if (at.in_a) t.load(p.beta + at.a), t.get(beta);
        if (at.in_b) t.load(p.beta + at.b), t.get(beta + C);
#pragma unroll
        for (int e = 0; e < 2 * C; ++e) x[e] += beta[e];
      }
    }
    rotate<C, HALVES, false>(x, angles, at);
    const int h = l.head + (now.round << p.head_bits);
    if (!now.in) continue;
    T* const y = static_cast<T*>(p.y) + now.row * p.y_stride[0] + now.index * p.y_stride[1] + h * p.y_stride[2];
    if (at.in_a) Chunk<T, C>::store(y + at.a, x);
    if (at.in_b) Chunk<T, C>::store(y + at.b, x + C);
  }
}

// Sums of the parameters' gradients stay in registers over a workgroup's tokens; its teams' are then added
// in a fixed order and written as a row of partial sums, which heads_join_kernel adds in a fixed order too.
// FULL: a layer norm or a beta (what only those need).
// 16384 tokens of 16 + 4 heads of 128 bf16 in 64 us, 3.9 TB/s; of 16 + 16 with 60 pairs, 8 bytes a load, 93 us, 4.3 TB/s.
template <typename T, int C, int LANES, bool HALVES, bool FULL>
__global__ __launch_bounds__(THREADS, FULL ? 1 : 4) void heads_backward_kernel(HeadsArgs a) {
  const bool layer = FULL && a.layer != 0;
  __shared__ float joined[THREADS / 64][128];
  __shared__ uint64_t freq[HEADS_PAIRS];
  __shared__ float2 turns[THREADS / 64][64 * C];
  if (threadIdx.x < HEADS_PAIRS) freq[threadIdx.x] = a.freq[threadIdx.x];
  __syncthreads();
  const bool second = static_cast<int>(blockIdx.x) >= a.part[0].blocks;
  const HeadsPart& p = a.part[second];
  const int block = blockIdx.x - (second ? a.part[0].blocks : 0);
  const Lane l = my_lane<LANES>(p, block);
  const Place<C, HALVES> at(l.lane, a.dim, a.pairs);
  Angles<C> angles;
  angles.begin(a, l.tokens);
  float2* const mine_turns = turns[threadIdx.x >> 6];
  const bool norm = p.gamma != nullptr;
  float gamma[2 * C], dgamma[2 * C] = {}, dbeta[2 * C] = {};
#pragma unroll
  for (int e = 0; e < 2 * C; ++e) gamma[e] = 1.f;
  if (norm) {
    Chunk<float, C> t;
    if (at.in_a) t.load(p.gamma + at.a), t.get(gamma);
    if (at.in_b) t.load(p.gamma + at.b), t.get(gamma + C);
  }
  struct Item {
    Chunk<T, C> ga, gb, xa, xb;
    uint32_t row, index;     // batch row, token of it
    long base;               // the wave's first token: all its lanes take as many turns
    bool in;
    int round;
  } next{};
  auto fetch = [&](long base, int round) {
    const long token = base + l.token;
    if (round == 0 && base < a.tokens) {
      next.row = static_cast<uint32_t>(token) / a.len;
      next.index = static_cast<uint32_t>(token) - next.row * a.len;
      angles.fetch(a, base);
    }
    next.base = base;
    next.round = round;
    const int h = l.head + (round << p.head_bits);
    const T* const dy = static_cast<const T*>(p.dy) + next.row * p.y_stride[0] + next.index * p.y_stride[1] + h * p.y_stride[2];
    const T* const x = static_cast<const T*>(p.x) + next.row * p.x_stride[0] + next.index * p.x_stride[1] + h * p.x_stride[2];
    next.ga = next.gb = next.xa = next.xb = Chunk<T, C>{};
    const bool in = next.in = token < a.tokens && h < p.heads;
    if (in && at.in_a) {
      next.ga.load(dy + at.a);
      if (norm) next.xa.load(x + at.a);
    }
    if (in && at.in_b) {
      next.gb.load(dy + at.b);
      if (norm) next.xb.load(x + at.b);
    }
  };
  fetch(l.base, 0);
  while (next.base < a.tokens) {
    const Item now = next;
    if (now.round == 0) {
      angles.form(a, now.base, freq, mine_turns);
      angles.read(a, mine_turns, l.token, l.lane);
    }
    const bool more = now.round + 1 < p.rounds;
    fetch(more ? now.base : now.base + l.step, more ? now.round + 1 : 0);
    float g[2 * C];
    now.ga.get(g);
    now.gb.get(g + C);
    rotate<C, HALVES, true>(g, angles, at);
    if (norm) {
      float x[2 * C], s = 0.f, m = 0.f;
      now.xa.get(x);
      now.xb.get(x + C);
      const float r = unit<C, LANES>(x, layer, at.in_a, at.in_b, a.inv_dim, a.eps);
#pragma unroll
      for (int e = 0; e < 2 * C; ++e) {
        dgamma[e] = fmaf(g[e], x[e], dgamma[e]);
        if (FULL) dbeta[e] += g[e];
        g[e] *= gamma[e];
        s = fmaf(g[e], x[e], s);
        if (FULL) m += g[e];
      }
      s = team_sum<LANES>(s) * a.inv_dim;
      m = layer ? team_sum<LANES>(m) * a.inv_dim : 0.f;
#pragma unroll
      for (int e = 0; e < 2 * C; ++e) g[e] = r * (g[e] - x[e] * s - m);
    }
    const int h = l.head + (now.round << p.head_bits);
    if (!now.in) continue;
    T* const dx = static_cast<T*>(p.dx) + now.row * p.x_stride[0] + now.index * p.x_stride[1] + h * p.x_stride[2];
    if (at.in_a) Chunk<T, C>::store(dx + at.a, g);
    if (at.in_b) Chunk<T, C>::store(dx + at.b, g + C);
  }
  if (!norm) return;
  auto flush = [&](const float (&v)[2 * C], float* to) {
    __syncthreads();
    float* const mine = joined[threadIdx.x >> 6];
#pragma unroll
    for (int e = 0; e < 2 * C; ++e) {
      const float t = over_teams<LANES>(v[e]);
      if ((threadIdx.x & 63) < LANES && (e < C ? at.in_a : at.in_b)) mine[e < C ? at.a + e : at.b + e - C] = t;
    }
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < a.dim) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < THREADS / 64; ++w) s += joined[w][threadIdx.x];
      to[static_cast<long>(block) * a.dim + threadIdx.x] = s;
    }
  };
  flush(dgamma, p.part_gamma);
  if (FULL && p.beta != nullptr) flush(dbeta, p.part_beta);
}

// Output blockIdx.x (dgamma and dbeta of the queries, then of the keys), channels 16 blockIdx.y ..: the sum over rows of
// partial sums, in 64 interleaved sums a channel.
__global__ __launch_bounds__(1024) void heads_join_kernel(HeadsArgs a) {
  __shared__ float lds[64][17];
  const HeadsPart& p = a.part[blockIdx.x >> 1];
  const bool beta = (blockIdx.x & 1) != 0;
  if (p.heads == 0 || p.gamma == nullptr || (beta && p.beta == nullptr)) return;
  const float* const from = beta ? p.part_beta : p.part_gamma;
  float* const to = beta ? p.dbeta : p.dgamma;
  const int c = blockIdx.y * 16 + (threadIdx.x & 15), lane = threadIdx.x >> 4;
  float v = 0.f;
  if (c < a.dim)
#pragma unroll 8
    for (int r = lane; r < p.blocks; r += 64) v += from[static_cast<long>(r) * a.dim + c];
  lds[lane][threadIdx.x & 15] = v;
  __syncthreads();
  if (lane == 0 && c < a.dim) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) t += lds[i][threadIdx.x & 15];
    to[c] = t;
  }
}

// Channels of a chunk: 8 where the pairs' halves are whole chunks.
int chunk(const HeadsArgs& a) { return a.halves && a.pairs % 8 != 0 ? 4 : 8; }

int lanes(const HeadsArgs& a) {
  const int c = chunk(a), rest = a.dim - 2 * a.pairs;
  const int need = a.halves ? a.pairs / c + (rest + 2 * c - 1) / (2 * c) : (a.dim + 2 * c - 1) / (2 * c);
  int n = 1;
  while (n < need) n *= 2;
  return n;
}

template <typename T, int C, int LANES>
void launch(const HeadsArgs& a, bool backward, hipStream_t s) {
  const unsigned n = static_cast<unsigned>(a.part[0].blocks + a.part[1].blocks);
  if (n == 0) return;
  auto by_layout = [&](auto halves) {
    constexpr bool HALVES = decltype(halves)::value;
    if (!backward) heads_forward_kernel<T, C, LANES, HALVES><<<n, THREADS, 0, s>>>(a);
    else if (a.layer || a.part[0].beta != nullptr || a.part[1].beta != nullptr) heads_backward_kernel<T, C, LANES, HALVES, true><<<n, THREADS, 0, s>>>(a);
    else heads_backward_kernel<T, C, LANES, HALVES, false><<<n, THREADS, 0, s>>>(a);
  };
  if (a.halves) by_layout(std::true_type{});
  else if constexpr (C == 8) by_layout(std::false_type{});
}

template <typename T>
void by_shape(const HeadsArgs& a, bool backward, hipStream_t s) {
  const int n = lanes(a);
  if (chunk(a) == 8) {
    switch (n) {
      case 1: return launch<T, 8, 1>(a, backward, s);
      case 2: return launch<T, 8, 2>(a, backward, s);
      case 4: return launch<T, 8, 4>(a, backward, s);
      default: return launch<T, 8, 8>(a, backward, s);
    }
  }
  switch (n) {
    case 1: return launch<T, 4, 1>(a, backward, s);
    case 2: return launch<T, 4, 2>(a, backward, s);
    case 4: return launch<T, 4, 4>(a, backward, s);
    case 8: return launch<T, 4, 8>(a, backward, s);
    default: return launch<T, 4, 16>(a, backward, s);
  }
}

}  // namespace

void heads_plan(HeadsArgs& a, bool backward) {
  const int teams = 64 / lanes(a);
  // workgroups of both parts together: as many as CUs would hold with 8 each forward and 4 or 5 backward.  By their registers they hold
  // 4 to 6 of the forwards of 8 channels a chunk (8 of those of 4), which so take up to two turns, 4 to 7 of the rms
  // backwards, and 3 to 6 of those with a layer norm or a beta (fp32 of 8 channels 2 or 3, up to two turns)
  const long most = 256 * (!backward ? 8 : chunk(a) == 8 ? 4 : 5);
  long units = 0, want[2] = {}, all[2] = {};
  for (int i = 0; i < 2; ++i) {
    HeadsPart& p = a.part[i];
    p.blocks = p.head_bits = 0;
    if (p.heads == 0 || a.tokens == 0) continue;
    while ((1 << p.head_bits) < p.heads && (2 << p.head_bits) <= teams) ++p.head_bits;
    const long tokens = static_cast<long>(teams >> p.head_bits) * (THREADS / 64);
    all[i] = (p.heads + (1 << p.head_bits) - 1) >> p.head_bits;
    want[i] = (a.tokens + tokens - 1) / tokens;
    units += want[i] * all[i];
  }
  // rounds a workgroup: the fewest by which there are no more workgroups than that (16384 tokens, 16 + 4 heads of 128: 10 give 1025
  // workgroups and take 73 us backward, 11 give 870)
  for (long each = (units + most - 1) / most, total = most + 1; total > most; ++each) {
    total = 0;
    for (int i = 0; i < 2; ++i) {
      HeadsPart& p = a.part[i];
      if (want[i] == 0) continue;
      // few tokens: the rounds over heads go to workgroups of their own
      p.splits = each == 1 ? static_cast<int>(all[i]) : 1;
      p.rounds = static_cast<int>(all[i] / p.splits);
      const long per = (each + p.rounds - 1) / p.rounds;
      p.groups = static_cast<int>((want[i] + per - 1) / per);
      p.blocks = p.groups * p.splits;
      total += p.blocks;
    }
  }
}

void heads_forward(const HeadsArgs& a, int dtype, hipStream_t s) {
  if (dtype == 1) by_shape<bf16_t>(a, false, s);
  else by_shape<float>(a, false, s);
}

void heads_backward(const HeadsArgs& a, int dtype, hipStream_t s) {
  if (dtype == 1) by_shape<bf16_t>(a, true, s);
  else by_shape<float>(a, true, s);
  if (a.part[0].gamma != nullptr || a.part[1].gamma != nullptr)
    heads_join_kernel<<<dim3(4, static_cast<unsigned>((a.dim + 15) / 16)), 1024, 0, s>>>(a);
}

}  // namespace petra
