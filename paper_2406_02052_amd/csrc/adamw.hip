// AdamW over many tensors in one launch, its states in fp32 or in 8 bits.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  t = steps + 1
//   theta -= lr (m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps) + decay theta)
//
// Bound by memory: 28 bytes an element with fp32 states and gradients, 16.25 with states
// in 8 bits, 2 more with a bf16 copy.
//
// In 8 bits a block of 64 elements holds m, and r = sqrt(v), as e4m3 numbers times a power
// of two that brings the block's largest into [128, 256): 17 binades below it, for v twice as many.
// v moves by a thousandth a step, where the format's step is a sixteenth: rounded to nearest
// it would stand still.  Both are rounded up or down at random, m so that its mean is kept and
// r so that its square's is; r of v > 0 is never rounded to 0, which would leave m over eps.
// A block is 16 lanes of 4 elements, one group of the generator a lane.
#include "common.h"
#include "ops.h"
#include "philox.h"

namespace petra {

namespace {

constexpr int PER_THREAD = 4, ROUND = 256 * PER_THREAD, ROUNDS = ADAMW_CHUNK / ROUND;

// Advances the step count; corrections for it, in 64 bits: 1 - b2^t loses ten bits at the first steps.
__global__ void adamw_begin_kernel(int64_t* steps, double log_b1, double log_b2, float* hyper) {
  const int64_t t = *steps + 1;
  *steps = t;
  hyper[0] = static_cast<float>(1.0 / -expm1(static_cast<double>(t) * log_b1));
  hyper[1] = static_cast<float>(1.0 / sqrt(-expm1(static_cast<double>(t) * log_b2)));
}

// The largest of the 16 lanes of a DPP row, in all of them.
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  uint32_t o;
  o = __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, false);    // [1,0,3,2]
  v = v > o ? v : o;
  o = __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, false);    // [2,3,0,1]
  v = v > o ? v : o;
  o = __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, false);   // half mirror
  v = v > o ? v : o;
  o = __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, false);   // mirror
  return v > o ? v : o;
}

// The bits of the power of two that brings a magnitude with these bits into [128, 256) (0 for 0), not below 2^-126.
__device__ __forceinline__ uint32_t scale_bits(uint32_t top) {
  const uint32_t e = top >> 23;
  return top == 0 ? 0u : (e > 8 ? e - 7 : 1u) << 23;
}
// The bits of 1 / a power of two (0 for 0).
__device__ __forceinline__ float inverse(uint32_t scale) {
  return scale == 0 ? 0.f : __uint_as_float((254u << 23) - scale);
}

// e4m3 code of the number at or below x (0 <= x), the number, and the step to the next.
__device__ __forceinline__ uint32_t below(float x, float& lo, float& ulp) {
  const uint32_t b = __float_as_uint(x), e = b >> 23;
  const bool tiny = e < 121;                       // below 2^-6 steps are 2^-9
  const float steps = floorf(x * 512.f);
  ulp = __uint_as_float(((tiny ? 121u : e) - 3u) << 23);
  lo = tiny ? steps * 0.001953125f : __uint_as_float(b & 0xfff00000u);
  return tiny ? static_cast<uint32_t>(steps) : (b >> 20) - 960u;
}

// Four consecutive elements at p, of which `left` exist.
__device__ __forceinline__ void load4(const float* p, int left, float* o) {
  if (left >= 4) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    o[0] = v.x, o[1] = v.y, o[2] = v.z, o[3] = v.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = i < left ? p[i] : 0.f;
  }
}
__device__ __forceinline__ void load4(const bf16_t* p, int left, float* o) {
  if (left >= 4) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    o[0] = __uint_as_float(v.x << 16), o[1] = __uint_as_float(v.x & 0xffff0000u);
    o[2] = __uint_as_float(v.y << 16), o[3] = __uint_as_float(v.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = i < left ? load1(p + i) : 0.f;
  }
}
__device__ __forceinline__ void store4(float* p, int left, const float* v) {
  if (left >= 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = v[i];
  }
}
__device__ __forceinline__ void store4(bf16_t* p, int left, const float* v) {
  if (left >= 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < left) store1(p + i, v[i]);
  }
}

// A chunk of ADAMW_CHUNK elements of one tensor a workgroup, in rounds whose loads are all asked for first.  64M elements with fp32
// states, bf16 gradients and copies in 237 us, 5.0 TB/s; 134M in 8 bits with copies in 332 us, 5.3 TB/s; 300 tensors of 2M in all 10.
template <typename G, bool FP8>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwArgs a) {
#pragma clang fp contract(off)
  const AdamwEntry t = a.entries[a.chunk_of[blockIdx.x]];
  const long first = (static_cast<long>(blockIdx.x) - t.first_chunk) * ADAMW_CHUNK + threadIdx.x * PER_THREAD;
  const float fix1 = a.hyper[0], fix2 = a.hyper[1], lr = *a.lr, gs = a.grad_scale != nullptr ? *a.grad_scale : 1.f;
  const Rng rng = FP8 ? load_rng(a.rng) : Rng{};
  float th[ROUNDS][4], g[ROUNDS][4], m[ROUNDS][4], v[ROUNDS][4];
  uint32_t cm[ROUNDS], cv[ROUNDS];
  float sm[ROUNDS], sv[ROUNDS];
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const long at = first + i * ROUND;
    const long rest = t.n - at;
    const int left = rest < 4 ? static_cast<int>(rest) : 4;
    load4(t.theta + at, left, th[i]);
    load4(static_cast<const G*>(t.grad) + at, left, g[i]);
    if constexpr (FP8) {
      cm[i] = cv[i] = 0;
      sm[i] = sv[i] = 0.f;
      if (at < t.padded) {   // whole blocks
        cm[i] = reinterpret_cast<const uint32_t*>(t.m)[at >> 2];
        cv[i] = reinterpret_cast<const uint32_t*>(t.v)[at >> 2];
        sm[i] = t.m_scale[at >> 6];
        sv[i] = t.v_scale[at >> 6];
      }
    } else {
      load4(static_cast<const float*>(t.m) + at, left, m[i]);
      load4(static_cast<const float*>(t.v) + at, left, v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < ROUNDS; ++i) {
    const long at = first + i * ROUND;
    const long rest = t.n - at;
    const int left = rest < 4 ? static_cast<int>(rest) : 4;
    if (FP8 ? at - (at & 63) >= t.padded : left <= 0) continue;   // whole blocks go together
    if constexpr (FP8) {
      const f32x2_t m0 = __builtin_amdgcn_cvt_pk_f32_fp8(cm[i], false), m1 = __builtin_amdgcn_cvt_pk_f32_fp8(cm[i], true);
      const f32x2_t r0 = __builtin_amdgcn_cvt_pk_f32_fp8(cv[i], false), r1 = __builtin_amdgcn_cvt_pk_f32_fp8(cv[i], true);
      m[i][0] = m0[0] * sm[i], m[i][1] = m0[1] * sm[i], m[i][2] = m1[0] * sm[i], m[i][3] = m1[1] * sm[i];
      v[i][0] = r0[0] * sv[i], v[i][1] = r0[1] * sv[i], v[i][2] = r1[0] * sv[i], v[i][3] = r1[1] * sv[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = v[i][e] * v[i][e];
    }
    float root[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // three roundings each, in this order: what is held in 8 bits is then a function of the inputs alone
      const float x = g[i][e] * gs;
      m[i][e] = m[i][e] * a.b1 + x * a.c1;
      v[i][e] = v[i][e] * a.b2 + x * x * a.c2;
      root[e] = __builtin_amdgcn_sqrtf(v[i][e]);
      const float step = m[i][e] * fix1 * __builtin_amdgcn_rcpf(fmaf(root[e], fix2, a.eps));
      th[i][e] = fmaf(-lr, fmaf(t.decay, th[i][e], step), th[i][e]);
    }
    store4(t.theta + at, left, th[i]);
    if (t.copy != nullptr) store4(static_cast<bf16_t*>(t.copy) + at, left, th[i]);
    if (a.zero_grads) {
      const float none[4] = {};
      store4(static_cast<G*>(t.grad) + at, left, none);
    }
    if constexpr (FP8) {
      uint32_t top_m = 0, top_v = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // finite values only: an infinity or NaN is held as NaN whatever the scale, and leaves the others theirs
        const uint32_t x = __float_as_uint(m[i][e]) & 0x7fffffffu, y = __float_as_uint(v[i][e]);
        if (x < 0x7f800000u) top_m = top_m > x ? top_m : x;
        if (y < 0x7f800000u) top_v = top_v > y ? top_v : y;
      }
      top_m = max16(top_m);
      top_v = max16(top_v);
      const uint32_t bm = scale_bits(top_m), bv = scale_bits(__float_as_uint(sqrtf(__uint_as_float(top_v))));
      const float im = inverse(bm), iv = inverse(bv);
      uint32_t bits[4], wm = 0, wv = 0;
      philox(rng, static_cast<uint64_t>(t.first_group + (at >> 2)), bits);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float um = static_cast<float>(bits[e] & 0xffffu) * 1.52587890625e-5f;
        const float uv = static_cast<float>(bits[e] >> 16) * 1.52587890625e-5f;
        float lo, ulp;
        const float x = fabsf(m[i][e]) * im;
        uint32_t c = below(x, lo, ulp);
        c += um * ulp < x - lo;
        c = x < 256.f ? c : 0x7fu;   // infinities and NaN
        wm |= (c | (__float_as_uint(m[i][e]) >> 31 << 7)) << (8 * e);
        const float w = v[i][e] * iv * iv;
        c = below(root[e] * iv, lo, ulp);
        c += uv * (ulp * (2.f * lo + ulp)) < w - lo * lo;
        c = c == 0 && v[i][e] > 0.f ? 1u : c;
        c = w < 65536.f ? c : 0x7fu;
        wv |= c << (8 * e);
      }
      reinterpret_cast<uint32_t*>(t.m)[at >> 2] = wm;
      reinterpret_cast<uint32_t*>(t.v)[at >> 2] = wv;
      if ((threadIdx.x & 15) == 0) {
        t.m_scale[at >> 6] = __uint_as_float(bm);
        t.v_scale[at >> 6] = __uint_as_float(bv);
      }
    } else {
      store4(static_cast<float*>(t.m) + at, left, m[i]);
      store4(static_cast<float*>(t.v) + at, left, v[i]);
    }
  }
}

}  // namespace

void adamw_step(const AdamwArgs& a, bool bf16_grads, bool fp8, hipStream_t s) {
  adamw_begin_kernel<<<1, 1, 0, s>>>(a.steps, a.log_b1, a.log_b2, a.hyper);
  if (a.chunks == 0) return;
  const unsigned n = static_cast<unsigned>(a.chunks);
  if (bf16_grads) {
    if (fp8) adamw_kernel<bf16_t, true><<<n, 256, 0, s>>>(a);
    else adamw_kernel<bf16_t, false><<<n, 256, 0, s>>>(a);
  } else {
    if (fp8) adamw_kernel<float, true><<<n, 256, 0, s>>>(a);
    else adamw_kernel<float, false><<<n, 256, 0, s>>>(a);
  }
}

}  // namespace petra
