// Attention over tokens, forward and backward, without a length x length tensor.
//
//   s_ij = scale q_i . k_j over the visible keys j of query i
//   lse_i = log sum_j exp s_ij,  p_ij = exp(s_ij - lse_i),  o_i = sum_j m_ij p_ij v_j
//   D_i = do_i . o_i,  dp_ij = m_ij do_i . v_j,  ds_ij = scale p_ij (dp_ij - D_i)
//   dq_i = sum_j ds_ij k_j,  dk_j = sum_i ds_ij q_i,  dv_j = sum_i m_ij p_ij do_i
//
// m is dropout's 0 or 1/keep.  The forward makes one pass over the keys with the
// running maximum and sum of each query's softmax; the backward takes p from s and
// lse again.  It has one kernel for dq (keys inside, a tile of queries a workgroup)
// and one for dk and dv (queries inside, a tile of keys a workgroup): 7 products of
// the pairs in place of 5, but no sum crosses workgroups, so results do not depend
// on timing and dq is not read and written once per tile of keys.
//
// Matrix instructions are 32x32x16 (bf16; fp32 by eight 32x32x2).  Their result has
// a column a lane and, in lane half h, rows 8 g + 4 h + {0..3}.  Scores are formed
// with the dimension that the next product keeps as the column, so that p or ds goes
// into that product from the registers that hold it: the product's inner index runs
// over 16 rows in the order (h, g, 0..3), and the other operand is read from LDS in
// the same order (bf16: by transposing LDS loads).
//
// Scores, sums, statistics and accumulators are fp32.  p and ds are rounded to the
// storage type as operands of the products (the matrix unit takes bf16): an error of
// each term of 2^-9 at most, as of the result's own rounding.
#include "common.h"
#include "ops.h"
#include "philox.h"

namespace petra {

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

__device__ __forceinline__ f32x16_t mfma32(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mfma32(const Frag<float>& a, const Frag<float>& b, f32x16_t c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
// Value of the lane in the other half of the wave.
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, 64); }

__device__ __forceinline__ void zero(f32x16_t& c) {
#pragma unroll
  for (int i = 0; i < 16; ++i) c[i] = 0.f;
}

// Eight consecutive accumulator registers (16 rows of a result) as an operand.
__device__ __forceinline__ void operand(const f32x16_t& c, int half, Frag<bf16_t>& f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(c[8 * half + 2 * i], c[8 * half + 2 * i + 1]);
  f.v = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
}
__device__ __forceinline__ void operand(const f32x16_t& c, int half, Frag<float>& f) {
#pragma unroll
  for (int i = 0; i < 8; ++i) f.v[i] = c[8 * half + i];
}

// A tile of rows of DP elements in LDS, in chunks of 16 bytes.  Chunks are moved
// within a row by an exclusive or with a key of the row: eight consecutive rows at
// one chunk (a straight read) and four consecutive rows at two chunks (a transposing
// read) then lie in different banks.
template <typename T, int DP>
struct Tile {
  static constexpr int CHUNKS = DP * static_cast<int>(sizeof(T)) / 16;
  static constexpr int ROW_BYTES = CHUNKS * 16;
  static constexpr int STEPS = DP / 16;
  static __device__ __forceinline__ int at(int row, int chunk) {
    if constexpr (CHUNKS % 8 == 0)
      return row * ROW_BYTES + ((chunk ^ (((row & 3) << 1) | ((row >> 2) & 1))) << 4);
    else
      return row * ROW_BYTES + ((chunk ^ ((row & 2) | ((row >> 2) & 1))) << 4);
  }
  // Operand whose free index is the row (this lane's `row`) and inner index the
  // channels 16 step .. 16 step + 15.
  static __device__ __forceinline__ Frag<T> straight(const char* lds, int row, int step, int h) {
    Frag<T> f;
    if constexpr (sizeof(T) == 2) {
      f.v = *reinterpret_cast<const bf16x8_t*>(lds + at(row, 2 * step + h));
    } else {
      const float4 a = *reinterpret_cast<const float4*>(lds + at(row, 4 * step + 2 * h));
      const float4 b = *reinterpret_cast<const float4*>(lds + at(row, 4 * step + 2 * h + 1));
      f.v[0] = a.x; f.v[1] = a.y; f.v[2] = a.z; f.v[3] = a.w;
      f.v[4] = b.x; f.v[5] = b.y; f.v[6] = b.z; f.v[7] = b.w;
    }
    return f;
  }
  // Operand whose free index is the channel d0 + (lane & 31) and inner index the 16
  // rows row0 .. in the order of a result's registers.
  static __device__ __forceinline__ Frag<T> across(char* lds, int row0, int d0, int lane) {
    Frag<T> f;
    const int h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      const int row = row0 + 4 * h + ((lane & 15) >> 2), col = d0 + (lane & 16) + 4 * (lane & 3);
      const int in = (col & 7) * 2;
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4_t*)(lds + at(row, col >> 3) + in));
      const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4_t*)(lds + at(row + 8, col >> 3) + in));
      typedef short s16x8_t __attribute__((ext_vector_type(8)));
      f.v = __builtin_bit_cast(bf16x8_t, s16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    } else {
      const int d = d0 + (lane & 31);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        f.v[j] = *reinterpret_cast<const float*>(lds + at(row0 + 8 * (j >> 2) + 4 * h + (j & 3), d >> 2) + 4 * (d & 3));
    }
    return f;
  }
};

// A tile of ROWS rows on its way from memory to LDS, THREADS threads.
template <typename T, int DP, int ROWS, int THREADS>
struct Mover {
  using Tl = Tile<T, DP>;
  static constexpr int N = (ROWS * Tl::CHUNKS + THREADS - 1) / THREADS;
  static_assert(ROWS * Tl::CHUNKS % THREADS == 0, "whole chunks a thread");
  u32x4_t v[N];

  // Keys first .. first + ROWS - 1 of one head (base: its key 0); keys at or past `end` and channels
  // past dim as zeros.  The resource starts at the tile, so offsets stay small however long the cache.
  __device__ __forceinline__ void keys(const T* base, int64_t stride, int first, int end, int dim) {
    const int left = end - first < ROWS ? end - first : ROWS;
    const __amdgpu_buffer_rsrc_t r =
        make_rsrc(base + static_cast<int64_t>(first) * stride, left > 0 ? (left - 1) * stride * sizeof(T) + dim * sizeof(T) : 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = threadIdx.x + i * THREADS, row = c / Tl::CHUNKS, chunk = c % Tl::CHUNKS;
      const bool in = row < left && chunk * 16 < dim * static_cast<int>(sizeof(T));
      v[i] = buf_load16(r, in ? static_cast<uint32_t>(row * stride * sizeof(T)) + chunk * 16 : BUF_OOB);
    }
  }
  // Rows first .. of a key head's queries: token row / group, head row % group.
  __device__ __forceinline__ void queries(const T* base, int64_t st, int64_t sh, int first, int end, int group, int dim) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = threadIdx.x + i * THREADS, row = first + c / Tl::CHUNKS, chunk = c % Tl::CHUNKS;
      v[i] = u32x4_t{0u, 0u, 0u, 0u};
      if (row < end && chunk * 16 < dim * static_cast<int>(sizeof(T))) {
        const int token = row / group, head = row - token * group;
        v[i] = *reinterpret_cast<const u32x4_t*>(reinterpret_cast<const char*>(base + token * st + head * sh) + chunk * 16);
      }
    }
  }
  __device__ __forceinline__ void put(char* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = threadIdx.x + i * THREADS;
      *reinterpret_cast<u32x4_t*>(lds + Tl::at(c / Tl::CHUNKS, c % Tl::CHUNKS)) = v[i];
    }
  }
};

// This lane's row of an operand, straight from memory: channels 16 step + 8 h .. + 7 of each step.
template <typename T, int DP>
__device__ __forceinline__ void load_row(const T* p, bool live, int h, int dim, Frag<T> (&f)[DP / 16]) {
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    Raw8<T> r;
    r.zero();
    if (live && 16 * s + 8 * h < dim) r.load(p + 16 * s + 8 * h);
    f[s].set(r);
  }
}

// What a workgroup works on.
struct Where {
  int b, kvh, q_len, kv_len;   // batch row, key head, lengths of this batch row
  int64_t head0;               // batch row's first head in [batch][heads] arrays, at this key head
};

__device__ __forceinline__ Where where(const AttnArgs& a, int bh) {
  Where w;
  w.b = bh / a.kv_heads;
  w.kvh = bh - w.b * a.kv_heads;
  const int ql = a.q_lens != nullptr ? a.q_lens[w.b] : a.q_len;
  const int kl = a.kv_lens != nullptr ? a.kv_lens[w.b] : a.kv_len;
  w.q_len = ql < 0 ? 0 : ql > a.q_len ? a.q_len : ql;
  w.kv_len = kl < 0 ? 0 : kl > a.kv_len ? a.kv_len : kl;
  w.head0 = static_cast<int64_t>(w.b) * a.heads + static_cast<int64_t>(w.kvh) * a.group;
  return w;
}

template <typename T>
__device__ __forceinline__ const T* at(const void* p, const int64_t (&st)[3], int b, int64_t token, int head) {
  return static_cast<const T*>(p) + b * st[0] + token * st[1] + head * st[2];
}
template <typename T>
__device__ __forceinline__ T* at(void* p, const int64_t (&st)[3], int b, int64_t token, int head) {
  return static_cast<T*>(p) + b * st[0] + token * st[1] + head * st[2];
}

// Keys that token i sees: 0 .. result - 1.
__device__ __forceinline__ int seen(const AttnArgs& a, const Where& w, int i) {
  int n = w.kv_len;
  if (a.causal) {
    n = i + w.kv_len - w.q_len + 1;
    n = n < 0 ? 0 : n > w.kv_len ? w.kv_len : n;
  }
  return i < w.q_len ? n : 0;
}

// Bits of the generator for this lane's row and the 16 keys from 16 block: keys 4 h + {0..3, 8..11}.
__device__ __forceinline__ void drop_bits(const AttnArgs& a, const Rng& rng, int64_t row, int block, int h, uint32_t w[4]) {
  philox(rng, static_cast<uint64_t>((row * ((a.kv_len + 15) >> 4) + block) * 2 + h), w);
}

// The accumulators of one row (column `lane & 31`): channels 32 m + 8 g + 4 h + {0..3}.
template <typename T, int DP>
__device__ __forceinline__ void store_row(T* p, const f32x16_t (&acc)[DP / 32], float f, int h, int dim) {
#pragma unroll
  for (int m = 0; m < DP / 32; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int d = 32 * m + 8 * g + 4 * h;
      if (d >= dim) continue;
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = acc[m][4 * g + i] * f;
      if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(p + d) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
      else
        *reinterpret_cast<float4*>(p + d) = make_float4(v[0], v[1], v[2], v[3]);
    }
}

// ---------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------

// WR waves side by side over rows (32 each), WK over keys (KB blocks of 32 each in a tile).
template <typename T, int DP, int WR, int WK, int KB, bool DROP>
__global__ __launch_bounds__(64 * WR * WK) void attn_forward_kernel(AttnArgs a) {
  using Tl = Tile<T, DP>;
  constexpr int THREADS = 64 * WR * WK, ROWS = 32 * WR, KT = 32 * KB * WK;
  constexpr int TILE_BYTES = KT * Tl::ROW_BYTES;
  constexpr int JOIN_BYTES = WK > 1 ? WK * WR * 32 * (DP + 2) * 4 : 0;
  __shared__ __attribute__((aligned(16))) char lds[2 * TILE_BYTES > JOIN_BYTES ? 2 * TILE_BYTES : JOIN_BYTES];
  char* const kt = lds;
  char* const vt = lds + TILE_BYTES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
  const int wr = wave % WR, wk = wave / WR;
  const Where w = where(a, blockIdx.y);
  const int rows = a.q_len * a.group;
  const int row0 = blockIdx.x * ROWS;
  const int row = row0 + wr * 32 + (lane & 31);
  const int token = row / a.group, head = w.kvh * a.group + row % a.group;
  const bool in_q = row < rows;
  const int limit = in_q ? seen(a, w, token) : 0;

  Frag<T> q[Tl::STEPS];
  load_row<T, DP>(at<T>(a.q, a.q_stride, w.b, in_q ? token : 0, head), in_q && token < w.q_len, h, a.dim, q);

  // keys that any row of the workgroup and of the wave sees, and that every row of the wave sees
  const int last_row = (row0 + ROWS < rows ? row0 + ROWS : rows) - 1;
  int last_token = last_row / a.group;
  if (last_token > w.q_len - 1) last_token = w.q_len - 1;
  const int end = row0 / a.group < w.q_len ? seen(a, w, last_token) : 0;
  int all = w.kv_len;
  if (a.causal) {
    all = (row0 + wr * 32) / a.group + w.kv_len - w.q_len + 1;
    all = all < w.kv_len ? all : w.kv_len;
  }
  const int tiles = (end + KT - 1) / KT;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int t0 = blockIdx.z * per, t1 = t0 + per < tiles ? t0 + per : tiles;

  f32x16_t acc[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) zero(acc[m]);
  float top = -INFINITY, sum = 0.f;
  const float c = a.scale_log2;
  Rng rng{};
  if (DROP) rng = load_rng(a.rng);
  const int64_t drop_row = (static_cast<int64_t>(w.b) * a.heads + head) * a.q_len + token;

  const T* const kb = at<T>(a.k, a.k_stride, w.b, 0, w.kvh);
  const T* const vb = at<T>(a.v, a.v_stride, w.b, 0, w.kvh);
  Mover<T, DP, KT, THREADS> mk, mv;
  if (t0 < t1) {
    mk.keys(kb, a.k_stride[1], t0 * KT, end, a.dim);
    mv.keys(vb, a.v_stride[1], t0 * KT, end, a.dim);
  }
  for (int t = t0; t < t1; ++t) {
    __syncthreads();
    mk.put(kt);
    mv.put(vt);
    __syncthreads();
    if (t + 1 < t1) {
      mk.keys(kb, a.k_stride[1], (t + 1) * KT, end, a.dim);
      mv.keys(vb, a.v_stride[1], (t + 1) * KT, end, a.dim);
    }
    const int at0 = wk * 32 * KB;          // this wave's keys in the tile
    const int key0 = t * KT + at0;
    f32x16_t s[KB];
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      zero(s[b]);
#pragma unroll
      for (int i = 0; i < Tl::STEPS; ++i)
        s[b] = mfma32(Tl::straight(kt, at0 + 32 * b + (lane & 31), i, h), q[i], s[b]);
    }
    if (key0 + 32 * KB > all) {
#pragma unroll
      for (int b = 0; b < KB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key0 + 32 * b + 8 * (i >> 2) + 4 * h + (i & 3);
          s[b][i] = key < limit ? s[b][i] : -INFINITY;
        }
    }
    float m = s[0][0];
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) m = fmaxf(m, s[b][i]);
    m = fmaxf(m, other_half(m));
    // the running maximum moves only when some row's grew by more than 2^8: exp stays far inside fp32
    if (__any(fmaf(m, c, -8.f) > top * c)) {
      const float n = fmaxf(top, m);
      const float f = n == -INFINITY ? 1.f : exp2_((top - n) * c);
      top = n;
      sum *= f;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] *= f;
    }
    const float base = top == -INFINITY ? 0.f : top * c;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[b][i] = exp2_(fmaf(s[b][i], c, -base));
        sum += s[b][i];
      }
#pragma unroll
      for (int k16 = 0; k16 < 2; ++k16) {
        if (DROP) {
          uint32_t bits[4];
          drop_bits(a, rng, drop_row, ((key0 + 32 * b) >> 4) + k16, h, bits);
#pragma unroll
          for (int i = 0; i < 8; ++i) s[b][8 * k16 + i] = kept(bits, i, a.cut) ? s[b][8 * k16 + i] : 0.f;
        }
        Frag<T> p;
        operand(s[b], k16, p);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
          acc[d] = mfma32(Tl::across(vt, at0 + 32 * b + 16 * k16, 32 * d, lane), p, acc[d]);
      }
    }
  }
  sum += other_half(sum);

  if constexpr (WK > 1) {
    // join the waves that shared the rows: statistics, then the scaled accumulators, in a fixed order
    float* const stat = reinterpret_cast<float*>(lds);              // [WK][WR][32][2]
    float* const part = stat + WK * WR * 32 * 2;                     // [WK][WR][32][DP]
    const int at_row = wr * 32 + (lane & 31);
    __syncthreads();
    if (h == 0) {
      stat[(wk * ROWS + at_row) * 2] = top;
      stat[(wk * ROWS + at_row) * 2 + 1] = sum;
    }
    __syncthreads();
    float n = -INFINITY;
#pragma unroll
    for (int i = 0; i < WK; ++i) n = fmaxf(n, stat[(i * ROWS + at_row) * 2]);
    const float f = n == -INFINITY ? 0.f : exp2_((top - n) * c);
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < WK; ++i) {
      const float ti = stat[(i * ROWS + at_row) * 2];
      sum += ti == -INFINITY ? 0.f : stat[(i * ROWS + at_row) * 2 + 1] * exp2_((ti - n) * c);
    }
    top = n;
    if (wk > 0) store_row<float, DP>(part + (wk * ROWS + at_row) * DP, acc, f, h, DP);
    __syncthreads();
    if (wk > 0) return;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float4 v = make_float4(acc[d][4 * g] * f, acc[d][4 * g + 1] * f, acc[d][4 * g + 2] * f, acc[d][4 * g + 3] * f);
#pragma unroll
        for (int i = 1; i < WK; ++i) {
          const float4 u = *reinterpret_cast<const float4*>(part + (i * ROWS + at_row) * DP + 32 * d + 8 * g + 4 * h);
          v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
        }
        acc[d][4 * g] = v.x; acc[d][4 * g + 1] = v.y; acc[d][4 * g + 2] = v.z; acc[d][4 * g + 3] = v.w;
      }
  }
  if (!in_q) return;
  if (a.splits > 1) {
    // [split][batch x key heads][rows][DP], and the statistics as [..][rows][2]
    const int64_t at_part = (static_cast<int64_t>(blockIdx.z) * gridDim.y + blockIdx.y) * rows + row;
    store_row<float, DP>(a.part + at_part * DP, acc, 1.f, h, DP);
    if (h == 0) {   // a row without keys: as if it had met none
      a.part_ml[at_part * 2] = limit > 0 ? top : -INFINITY;
      a.part_ml[at_part * 2 + 1] = limit > 0 ? sum : 0.f;
    }
    return;
  }
  const bool any = sum > 0.f || sum != sum;
  store_row<T, DP>(at<T>(a.out, a.o_stride, w.b, token, head), acc, limit > 0 && any ? a.inv_keep / sum : 0.f, h, a.dim);
  if (h == 0)
    a.lse[(w.head0 + row % a.group) * a.q_len + token] =
        limit > 0 && any ? fmaf(top, a.scale, __builtin_amdgcn_logf(sum) * LN2) : -INFINITY;
}

// Joins the splits of one row: a wave a row, DP / 64 channels a lane.
template <typename T, int DP>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  const int lane = threadIdx.x & 63;
  const int rows = a.q_len * a.group;
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const Where w = where(a, blockIdx.y);
  const int64_t step = static_cast<int64_t>(gridDim.y) * rows, first = static_cast<int64_t>(blockIdx.y) * rows + row;
  float n = -INFINITY;
  for (int s = 0; s < a.splits; ++s) n = fmaxf(n, a.part_ml[(first + s * step) * 2]);
  constexpr int PER = (DP + 63) / 64;
  float acc[PER] = {}, sum = 0.f;
  for (int s = 0; s < a.splits; ++s) {
    const int64_t i = first + s * step;
    const float t = a.part_ml[i * 2];
    if (t == -INFINITY) continue;
    const float f = exp2_((t - n) * a.scale_log2);
    sum = fmaf(a.part_ml[i * 2 + 1], f, sum);
#pragma unroll
    for (int e = 0; e < PER; ++e)
      if (lane + 64 * e < DP) acc[e] = fmaf(a.part[i * DP + lane + 64 * e], f, acc[e]);
  }
  const int token = row / a.group, head = w.kvh * a.group + row % a.group;
  const bool any = sum > 0.f || sum != sum;
  const float f = any ? a.inv_keep / sum : 0.f;
  T* const o = at<T>(a.out, a.o_stride, w.b, token, head);
#pragma unroll
  for (int e = 0; e < PER; ++e)
    if (lane + 64 * e < a.dim) store1(o + lane + 64 * e, acc[e] * f);
  if (lane == 0)
    a.lse[(w.head0 + row % a.group) * a.q_len + token] = any ? fmaf(n, a.scale, __builtin_amdgcn_logf(sum) * LN2) : -INFINITY;
}

// ---------------------------------------------------------------------------
// backward: query gradient
// ---------------------------------------------------------------------------

template <typename T, int DP, int WR, int KB, bool DROP>
__global__ __launch_bounds__(64 * WR) void attn_dq_kernel(AttnArgs a) {
  using Tl = Tile<T, DP>;
  constexpr int THREADS = 64 * WR, ROWS = 32 * WR, KT = 32 * KB;
  constexpr int TILE_BYTES = KT * Tl::ROW_BYTES;
  __shared__ __attribute__((aligned(16))) char lds[2 * TILE_BYTES];
  char* const kt = lds;
  char* const vt = lds + TILE_BYTES;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
  const Where w = where(a, blockIdx.y);
  const int rows = a.q_len * a.group;
  const int row0 = blockIdx.x * ROWS;
  const int row = row0 + wave * 32 + (lane & 31);
  const int token = row / a.group, head = w.kvh * a.group + row % a.group;
  const bool in_q = row < rows, live = in_q && token < w.q_len;
  const int limit = in_q ? seen(a, w, token) : 0;
  const int from = in_q ? token : 0;

  Frag<T> q[Tl::STEPS], g[Tl::STEPS];
  load_row<T, DP>(at<T>(a.q, a.q_stride, w.b, from, head), live, h, a.dim, q);
  load_row<T, DP>(at<T>(a.d_o, a.o_stride, w.b, from, head), live, h, a.dim, g);
  // D = do . o: each half of the lanes has half the channels
  float delta = 0.f;
  {
    const T* const o = at<T>(a.o, a.o_stride, w.b, from, head);
    const T* const d = at<T>(a.d_o, a.o_stride, w.b, from, head);
#pragma unroll
    for (int s = 0; s < Tl::STEPS; ++s)
      if (live && 16 * s + 8 * h < a.dim) {
        float x[8], y[8];
        Vec8<T>::load(o + 16 * s + 8 * h, x);
        Vec8<T>::load(d + 16 * s + 8 * h, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) delta = fmaf(x[i], y[i], delta);
      }
    delta += other_half(delta);
  }
  const int64_t stat = (w.head0 + row % a.group) * a.q_len + token;
  // a row without keys: lse +inf makes every p zero
  const float lse = limit > 0 ? a.lse[stat] * LOG2E : INFINITY;
  if (in_q && h == 0) a.delta[stat] = delta;

  const int last_row = (row0 + ROWS < rows ? row0 + ROWS : rows) - 1;
  int last_token = last_row / a.group;
  if (last_token > w.q_len - 1) last_token = w.q_len - 1;
  const int end = row0 / a.group < w.q_len ? seen(a, w, last_token) : 0;
  int all = w.kv_len;
  if (a.causal) {
    all = (row0 + wave * 32) / a.group + w.kv_len - w.q_len + 1;
    all = all < w.kv_len ? all : w.kv_len;
  }
  const int tiles = (end + KT - 1) / KT;

  f32x16_t acc[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) zero(acc[m]);
  const float c = a.scale_log2;
  Rng rng{};
  if (DROP) rng = load_rng(a.rng);
  const int64_t drop_row = (static_cast<int64_t>(w.b) * a.heads + head) * a.q_len + token;

  const T* const kb = at<T>(a.k, a.k_stride, w.b, 0, w.kvh);
  const T* const vb = at<T>(a.v, a.v_stride, w.b, 0, w.kvh);
  Mover<T, DP, KT, THREADS> mk, mv;
  if (tiles > 0) {
    mk.keys(kb, a.k_stride[1], 0, end, a.dim);
    mv.keys(vb, a.v_stride[1], 0, end, a.dim);
  }
  for (int t = 0; t < tiles; ++t) {
    __syncthreads();
    mk.put(kt);
    mv.put(vt);
    __syncthreads();
    if (t + 1 < tiles) {
      mk.keys(kb, a.k_stride[1], (t + 1) * KT, end, a.dim);
      mv.keys(vb, a.v_stride[1], (t + 1) * KT, end, a.dim);
    }
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const int key0 = t * KT + 32 * b;
      f32x16_t s, dp;
      zero(s);
      zero(dp);
#pragma unroll
      for (int i = 0; i < Tl::STEPS; ++i) {
        s = mfma32(Tl::straight(kt, 32 * b + (lane & 31), i, h), q[i], s);
        dp = mfma32(Tl::straight(vt, 32 * b + (lane & 31), i, h), g[i], dp);
      }
#pragma unroll
      for (int k16 = 0; k16 < 2; ++k16) {
        uint32_t bits[4];
        if (DROP) drop_bits(a, rng, drop_row, (key0 >> 4) + k16, h, bits);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = 8 * k16 + j;
          const float p = exp2_(fmaf(s[i], c, -lse));
          float d = dp[i];
          if (DROP) d = kept(bits, j, a.cut) ? d * a.inv_keep : 0.f;
          s[i] = p * (d - delta);
        }
      }
      if (key0 + 32 > all) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key0 + 8 * (i >> 2) + 4 * h + (i & 3);
          s[i] = key < limit ? s[i] : 0.f;
        }
      }
#pragma unroll
      for (int k16 = 0; k16 < 2; ++k16) {
        Frag<T> p;
        operand(s, k16, p);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
          acc[d] = mfma32(Tl::across(kt, 32 * b + 16 * k16, 32 * d, lane), p, acc[d]);
      }
    }
  }
  if (!in_q) return;
  store_row<T, DP>(at<T>(a.dq, a.q_stride, w.b, token, head), acc, limit > 0 ? a.scale : 0.f, h, a.dim);
}

// ---------------------------------------------------------------------------
// backward: key and value gradients
// ---------------------------------------------------------------------------

template <typename T, int DP, int WC, int RB, bool DROP>
__global__ __launch_bounds__(64 * WC) void attn_dkv_kernel(AttnArgs a) {
  using Tl = Tile<T, DP>;
  constexpr int THREADS = 64 * WC, KEYS = 32 * WC, RT = 32 * RB;
  constexpr int TILE_BYTES = RT * Tl::ROW_BYTES;
  __shared__ __attribute__((aligned(16))) char lds[2 * TILE_BYTES + RT * 8 + (DROP ? WC * 32 * 4 : 0)];
  char* const qt = lds;
  char* const gt = lds + TILE_BYTES;
  float* const lse_t = reinterpret_cast<float*>(lds + 2 * TILE_BYTES);
  float* const delta_t = lse_t + RT;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
  const Where w = where(a, blockIdx.y);
  const int key0 = blockIdx.x * KEYS + wave * 32, key = key0 + (lane & 31);
  const bool live = key < w.kv_len;
  const int key_at = live ? key : 0;

  Frag<T> k[Tl::STEPS], v[Tl::STEPS];
  load_row<T, DP>(at<T>(a.k, a.k_stride, w.b, key_at, w.kvh), live, h, a.dim, k);
  load_row<T, DP>(at<T>(a.v, a.v_stride, w.b, key_at, w.kvh), live, h, a.dim, v);
  f32x16_t dk[DP / 32], dv[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) {
    zero(dk[m]);
    zero(dv[m]);
  }
  const int rows = w.q_len * a.group;
  // the first token that sees the workgroup's first key
  int first = 0;
  if (a.causal) first = blockIdx.x * KEYS - (w.kv_len - w.q_len);
  first = (first < 0 ? 0 : first) * a.group;
  const int t0 = static_cast<int>(blockIdx.x) * KEYS < w.kv_len ? first / RT : 0;
  const int t1 = static_cast<int>(blockIdx.x) * KEYS < w.kv_len ? (rows + RT - 1) / RT : 0;
  const float c = a.scale_log2;
  Rng rng{};
  if (DROP) rng = load_rng(a.rng);

  const T* const qb = at<T>(a.q, a.q_stride, w.b, 0, w.kvh * a.group);
  const T* const gb = at<T>(a.d_o, a.o_stride, w.b, 0, w.kvh * a.group);
  Mover<T, DP, RT, THREADS> mq, mg;
  float lse = INFINITY, delta = 0.f;
  auto fetch = [&](int t) {
    mq.queries(qb, a.q_stride[1], a.q_stride[2], t * RT, rows, a.group, a.dim);
    mg.queries(gb, a.o_stride[1], a.o_stride[2], t * RT, rows, a.group, a.dim);
    const int r = t * RT + static_cast<int>(threadIdx.x);
    lse = INFINITY;
    delta = 0.f;
    if (threadIdx.x < RT && r < rows) {
      const int token = r / a.group;
      const int64_t stat = (w.head0 + r % a.group) * a.q_len + token;
      if (seen(a, w, token) > 0) lse = a.lse[stat] * LOG2E;
      delta = a.delta[stat];
    }
  };
  if (t0 < t1) fetch(t0);
  for (int t = t0; t < t1; ++t) {
    __syncthreads();
    mq.put(qt);
    mg.put(gt);
    if (threadIdx.x < RT) {
      lse_t[threadIdx.x] = lse;
      delta_t[threadIdx.x] = delta;
    }
    __syncthreads();
    if (t + 1 < t1) fetch(t + 1);
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      const int row0 = t * RT + 32 * b;
      f32x16_t s, dp;
      zero(s);
      zero(dp);
#pragma unroll
      for (int i = 0; i < Tl::STEPS; ++i) {
        s = mfma32(Tl::straight(qt, 32 * b + (lane & 31), i, h), k[i], s);
        dp = mfma32(Tl::straight(gt, 32 * b + (lane & 31), i, h), v[i], dp);
      }
      uint32_t keep = 0xffffffffu;   // bit n: row row0 + n keeps this lane's key
      if (DROP) {
        // the generator's groups run along the keys: each lane draws for its row, and the wave turns the
        // 32 x 32 bits round (a compare gives the bits of one key of each half for 32 rows)
        const int r = row0 + (lane & 31);
        const int token = r / a.group, head = w.kvh * a.group + r % a.group;
        const int64_t drop_row = (static_cast<int64_t>(w.b) * a.heads + head) * a.q_len + token;
        uint32_t* const turn = reinterpret_cast<uint32_t*>(delta_t + RT) + wave * 32;
#pragma unroll
        for (int k16 = 0; k16 < 2; ++k16) {
          uint32_t bits[4];
          drop_bits(a, rng, drop_row, (key0 >> 4) + k16, h, bits);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint64_t m = __ballot(kept(bits, j, a.cut));
            const int n = 16 * k16 + 8 * (j >> 2) + (j & 3);   // key of the lower half
            if (lane == 0) turn[n] = static_cast<uint32_t>(m);
            if (lane == 32) turn[n + 4] = static_cast<uint32_t>(m >> 32);
          }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        keep = turn[lane & 31];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
      f32x16_t ds;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 l4 = *reinterpret_cast<const float4*>(lse_t + 32 * b + 8 * g + 4 * h);
        const float4 d4 = *reinterpret_cast<const float4*>(delta_t + 32 * b + 8 * g + 4 * h);
        const float ll[4] = {l4.x, l4.y, l4.z, l4.w}, dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = 4 * g + j;
          float p = exp2_(fmaf(s[i], c, -ll[j]));
          if (a.causal) {
            const int r = row0 + 8 * g + 4 * h + j;
            if (row0 < (key0 + 31 - (w.kv_len - w.q_len)) * a.group)   // the block has hidden pairs
              p = key < r / a.group + w.kv_len - w.q_len + 1 ? p : 0.f;
          }
          float d = dp[i], pm = p;
          if (DROP) {
            const bool kp = (keep >> (8 * g + 4 * h + j)) & 1;
            d = kp ? d * a.inv_keep : 0.f;
            pm = kp ? p : 0.f;
          }
          ds[i] = p * (d - dd[j]);
          s[i] = pm;
        }
      }
#pragma unroll
      for (int r16 = 0; r16 < 2; ++r16) {
        Frag<T> p, d;
        operand(s, r16, p);
        operand(ds, r16, d);
#pragma unroll
        for (int m = 0; m < DP / 32; ++m) {
          dv[m] = mfma32(Tl::across(gt, 32 * b + 16 * r16, 32 * m, lane), p, dv[m]);
          dk[m] = mfma32(Tl::across(qt, 32 * b + 16 * r16, 32 * m, lane), d, dk[m]);
        }
      }
    }
  }
  if (key >= a.kv_len) return;
  // a key past its length takes no part, whatever its score was
  if (!live) {
#pragma unroll
    for (int m = 0; m < DP / 32; ++m) {
      zero(dk[m]);
      zero(dv[m]);
    }
  }
  store_row<T, DP>(at<T>(a.dk, a.k_stride, w.b, key, w.kvh), dk, a.scale, h, a.dim);
  store_row<T, DP>(at<T>(a.dv, a.v_stride, w.b, key, w.kvh), dv, a.inv_keep, h, a.dim);
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

template <typename T> struct Shape { static constexpr int KB = 2; };
template <> struct Shape<float> { static constexpr int KB = 1; };

template <typename T, int DP, bool DROP>
void forward_by(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
  const int rows = a.q_len * a.group, bh = a.batch * a.kv_heads;
  const dim3 grid((rows + p.row_tile - 1) / p.row_tile, bh, a.splits);
  if (p.row_tile == 32)
    attn_forward_kernel<T, DP, 1, 2, 1, DROP><<<grid, 128, 0, s>>>(a);
  else
    attn_forward_kernel<T, DP, 4, 1, Shape<T>::KB, DROP><<<grid, 256, 0, s>>>(a);
  if (a.splits > 1) attn_join_kernel<T, DP><<<dim3((rows + 3) / 4, bh), 256, 0, s>>>(a);
}

template <typename T, int DP, bool DROP>
void backward_by(const AttnArgs& a, const AttnPlan&, hipStream_t s) {
  const int rows = a.q_len * a.group, bh = a.batch * a.kv_heads;
  if (rows > 0)
    attn_dq_kernel<T, DP, 4, Shape<T>::KB, DROP><<<dim3((rows + 127) / 128, bh), 256, 0, s>>>(a);
  if (a.kv_len > 0)
    attn_dkv_kernel<T, DP, 4, Shape<T>::KB, DROP><<<dim3((a.kv_len + 127) / 128, bh), 256, 0, s>>>(a);
}

#define PETRA_BY_DIM(F, T)                                                       \
  if (a.rng != nullptr) {                                                        \
    if (a.dim <= 32) F<T, 32, true>(a, p, s);                                    \
    else if (a.dim <= 64) F<T, 64, true>(a, p, s);                               \
    else if (a.dim <= 96) F<T, 96, true>(a, p, s);                               \
    else F<T, 128, true>(a, p, s);                                               \
  } else {                                                                       \
    if (a.dim <= 32) F<T, 32, false>(a, p, s);                                   \
    else if (a.dim <= 64) F<T, 64, false>(a, p, s);                              \
    else if (a.dim <= 96) F<T, 96, false>(a, p, s);                              \
    else F<T, 128, false>(a, p, s);                                              \
  }

int padded(int dim) { return (dim + 31) / 32 * 32; }

}  // namespace

AttnPlan attn_plan(const AttnArgs& a, int) {
  AttnPlan p{};
  const int64_t rows = static_cast<int64_t>(a.q_len) * a.group, bh = static_cast<int64_t>(a.batch) * a.kv_heads;
  p.row_tile = rows <= 32 ? 32 : 128;
  const int64_t blocks = (rows + p.row_tile - 1) / p.row_tile * bh;
  // few workgroups: split the keys until the chip's 256 CUs have about two each, 128 keys a split at least
  int64_t splits = blocks == 0 || blocks >= 256 ? 1 : (512 + blocks - 1) / blocks;
  const int64_t most = (a.kv_len + 127) / 128;
  splits = splits < most ? splits : most;
  p.splits = static_cast<int>(splits < 1 ? 1 : splits);
  p.fwd_bytes = p.splits > 1 ? static_cast<size_t>(p.splits) * bh * rows * (padded(a.dim) + 2) * 4 : 0;
  p.bwd_bytes = static_cast<size_t>(a.batch) * a.heads * a.q_len * 4;
  return p;
}

void attn_forward(const AttnArgs& args, const AttnPlan& p, int dtype, void* workspace, hipStream_t s) {
  AttnArgs a = args;
  a.splits = p.splits;
  a.part = static_cast<float*>(workspace);
  a.part_ml = a.part + static_cast<size_t>(p.splits) * a.batch * a.heads * a.q_len * padded(a.dim);
  if (dtype == 1) {
    PETRA_BY_DIM(forward_by, bf16_t)
  } else {
    PETRA_BY_DIM(forward_by, float)
  }
}

void attn_backward(const AttnArgs& args, const AttnPlan& p, int dtype, void* workspace, hipStream_t s) {
  AttnArgs a = args;
  a.delta = static_cast<float*>(workspace);
  if (dtype == 1) {
    PETRA_BY_DIM(backward_by, bf16_t)
  } else {
    PETRA_BY_DIM(backward_by, float)
  }
}

}  // namespace petra
