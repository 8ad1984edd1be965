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

// A tile of rows of DP elements in LDS, in chunks of 16 bytes.  LDS serves 256 bytes a
// cycle if they lie in different banks: 16 lanes of a straight read (16 rows at one
// chunk), 32 of a transposing one (4 rows at 4 chunks).  Chunks are therefore moved
// within a row by an exclusive or with a key of the row.
template <typename T, int DP>
struct Tile {
  static constexpr int CHUNKS = DP * static_cast<int>(sizeof(T)) / 16;
  static constexpr int ROW_BYTES = CHUNKS * 16;
  static constexpr int STEPS = DP / 16;
  static __device__ __forceinline__ int key(int row) {
    if constexpr (CHUNKS % 16 == 0 && sizeof(T) == 2)
      return ((row & 3) << 2) | ((row >> 2) & 3);
    else if constexpr (CHUNKS % 16 == 0)   // fp32 reads across rows take a row and its fourth next
      return (((row >> 2) & 1) << 3) | ((row & 3) << 1) | ((row >> 3) & 1);
    else if constexpr (CHUNKS % 8 == 0)    // two rows to 256 bytes
      return (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    else                                   // four, or four thirds
      return (row >> 2) & 3;
  }
  static __device__ __forceinline__ int at(int row, int chunk) {
    return row * ROW_BYTES + ((chunk ^ key(row)) << 4);
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

// Brings tiles of ROWS rows from memory to LDS without passing through registers:
// each wave's load puts 64 chunks of 16 bytes in a row into LDS, so the lanes ask for
// the chunks in the order that Tile gives them.  Offsets from the tile's first row
// are the same for every whole tile; lanes without an element ask past the end of
// the resource, which brings zeros.
template <typename T, int DP, int ROWS, int THREADS>
struct Stager {
  using Tl = Tile<T, DP>;
  static constexpr int N = ROWS * Tl::CHUNKS / THREADS;
  static_assert(ROWS * Tl::CHUNKS % THREADS == 0, "whole chunks a thread");
  uint32_t off[N];

  static __device__ __forceinline__ int place(int i) { return i * THREADS + static_cast<int>(threadIdx.x); }
  static __device__ __forceinline__ int row(int i) { return place(i) / Tl::CHUNKS; }
  static __device__ __forceinline__ int chunk_offset(int i, int dim) {
    const int p = place(i), r = p / Tl::CHUNKS, c = (Tl::at(r, p % Tl::CHUNKS) >> 4) - r * Tl::CHUNKS;
    return c * 16 < dim * static_cast<int>(sizeof(T)) ? c * 16 : -1;
  }
  // Rows one stride apart.
  __device__ __forceinline__ void keys(int64_t stride, int dim) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = chunk_offset(i, dim);
      off[i] = c < 0 ? BUF_OOB : static_cast<uint32_t>(row(i) * stride * sizeof(T)) + c;
    }
  }
  // Rows of a key head's queries from row `first`, of `left` rows: token row / group, head row % group.
  __device__ __forceinline__ void queries(int64_t st, int64_t sh, int first, int left, int group, int dim) {
    const int token0 = first / group;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = chunk_offset(i, dim), r = first + row(i), token = r / group;
      const int64_t o = ((token - token0) * st + (r - token * group) * sh) * static_cast<int64_t>(sizeof(T));
      off[i] = c < 0 || row(i) >= left ? BUF_OOB : static_cast<uint32_t>(o) + c;
    }
  }
  // Zeros in place of the tile's first n rows.
  __device__ __forceinline__ void skip(int n) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (row(i) < n) off[i] = BUF_OOB;
  }
  // The loads are written out: the compiler would let every later transposing LDS read wait for them,
  // those of the other buffer too.  They write no register, and arrived() waits for them.
  __device__ __forceinline__ void load(const T* first, uint32_t bytes, char* lds) const {
    const uint64_t base = reinterpret_cast<uint64_t>(first);
    const u32x4_t r = {static_cast<uint32_t>(base), static_cast<uint32_t>(base >> 32) & 0xffffu, bytes, 0x00020000u};
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t to = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds)) + wave * 1024;
#pragma unroll
    for (int i = 0; i < N; ++i)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   ::"s"(to + i * THREADS * 16), "v"(off[i]), "s"(r) : "memory");
  }
  // Keys first .. of a head whose key 0 is at base; those at or past `end` as zeros.
  __device__ __forceinline__ void load_keys(const T* base, int64_t stride, int first, int end, int dim, char* lds) const {
    const int left = end - first < ROWS ? end - first : ROWS;
    load(base + first * stride, static_cast<uint32_t>(((left - 1) * stride + dim) * sizeof(T)), lds);
  }
};

// Every load of the workgroup has arrived in LDS, and every wave has left the buffer that is next.
// The builtin tells the compiler that its own loads from before a loop have arrived too, which
// it would otherwise wait for inside the loop, with the tile that was just asked for.
__device__ __forceinline__ void arrived() {
  __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
}

// 64 consecutive floats (or zeros past `bytes`) into LDS, by the wave that calls.
__device__ __forceinline__ void stage_floats(const float* from, int bytes, float* lds) {
  const uint64_t base = reinterpret_cast<uint64_t>(from);
  const u32x4_t r = {static_cast<uint32_t>(base), static_cast<uint32_t>(base >> 32) & 0xffffu, static_cast<uint32_t>(bytes), 0x00020000u};
  const uint32_t to = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) float*)lds));
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
               ::"s"(to), "v"((threadIdx.x & 63) * 4), "s"(r) : "memory");
}

// Runs body(t, buffer) for t0 <= t < t1 with the buffers 0 and 1 in turn.  The buffer is a constant
// in each of the two copies: LDS addresses differ by immediates, where a variable buffer costs an
// addition for every operand read.
template <int N> struct Const { static constexpr int value = N; };
template <typename F>
__device__ __forceinline__ void in_turn(int t0, int t1, F body) {
  for (int t = t0; t < t1; t += 2) {
    body(t, Const<0>{});
    if (t + 1 < t1) body(t + 1, Const<1>{});
  }
}

// What this workgroup works on: (batch row, key head), split, tile.  Splits and heads run
// fastest: workgroups go to the 8 XCDs in turn, so that with a multiple of 8 heads each XCD's
// L2 has the keys of its own (2 x 4096 causal tokens, 16 heads: 147 us, 227 with the tiles
// fastest), and the workgroups of a short sequence, which end at once, lie between others';
// tiles run slowest, from the one with most visible pairs where the mask is causal, so that
// what is left for the end is short.
struct Item {
  int bh, split, tile;
};
__device__ __forceinline__ Item work_item(const AttnArgs& a, bool last_first) {
  const int rest = blockIdx.x / a.splits;
  Item i;
  i.split = blockIdx.x - rest * a.splits;
  i.tile = rest / a.bhs;
  i.bh = a.bh0 + rest - i.tile * a.bhs;
  if (last_first) i.tile = a.tiles - 1 - i.tile;
  return i;
}

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

// Bound by the exponentials beside the products: a block of 32 x 32 pairs of 128 channels has 512 cycles of
// matrix instructions a wave and about 640 of other vector ones, which overlap between waves only.  With 128
// channels of bf16 three waves a SIMD, of 32 keys at a time, take 151 us for 2 x 4096 causal tokens and 16
// heads, two waves of 64 keys 162; buffers at constant addresses then save 7.  Two blocks of rows a wave,
// which halve the reads of LDS, leave one wave a SIMD: 241 us.
// WR waves side by side over rows (32 each), WK over keys (KB blocks of 32 each in a tile).
template <typename T, int DP, int WR, int WK, int KB, bool DROP>
__global__ __launch_bounds__(64 * WR * WK, (DP * sizeof(T) > 256 ? 1 : DP * sizeof(T) == 256 && KB == 1 && WR == 4 ? 3 : 2)) void attn_forward_kernel(AttnArgs a) {
  using Tl = Tile<T, DP>;
  constexpr int THREADS = 64 * WR * WK, ROWS = 32 * WR, KT = 32 * KB * WK;
  constexpr int TILE_BYTES = KT * Tl::ROW_BYTES;
  constexpr int JOIN_ROW = DP + 4;   // floats: rows 16 bytes apart in the banks
  constexpr int JOIN_BYTES = WK > 1 ? WK * ROWS * (JOIN_ROW + 2) * 4 : 0;
  __shared__ __attribute__((aligned(16))) char lds[4 * TILE_BYTES > JOIN_BYTES ? 4 * TILE_BYTES : JOIN_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int wr = wave % WR, wk = wave / WR;
  const Item item = work_item(a, true);
  const int bh = item.bh, split = item.split, tile = item.tile;
  const Where w = where(a, bh);
  const int rows = a.q_len * a.group;
  const int row0 = tile * ROWS, wave0 = row0 + wr * 32;
  const int row = wave0 + (lane & 31);
  const int token = row / a.group, head = w.kvh * a.group + row - token * a.group;
  const bool in_q = row < rows;
  const int limit = in_q ? seen(a, w, token) : 0;
  Frag<T> q[Tl::STEPS];
  load_row<T, DP>(at<T>(a.q, a.q_stride, w.b, in_q ? token : 0, head), in_q && token < w.q_len, h, a.dim, q);

  // keys that any row of the workgroup sees, and that every row of the wave sees
  const int last_row = (row0 + ROWS < rows ? row0 + ROWS : rows) - 1;
  int last_token = last_row / a.group;
  if (last_token > w.q_len - 1) last_token = w.q_len - 1;
  const int end = row0 / a.group < w.q_len ? seen(a, w, last_token) : 0;
  int all = w.kv_len;
  if (a.causal) {
    all = wave0 / a.group + w.kv_len - w.q_len + 1;
    all = all < w.kv_len ? all : w.kv_len;
  }
  const int tiles = (end + KT - 1) / KT;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int t0 = split * per, t1 = t0 + per < tiles ? t0 + per : tiles;

  f32x16_t acc[DP / 32];
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) zero(acc[m]);
  const float c = a.scale_log2;
  Rng rng{};
  if (DROP) rng = load_rng(a.rng);
  const int64_t stat = (static_cast<int64_t>(w.b) * a.heads + head) * a.q_len + token;   // of lse, and the generator's row

  const T* const kb = at<T>(a.k, a.k_stride, w.b, 0, w.kvh);
  const T* const vb = at<T>(a.v, a.v_stride, w.b, 0, w.kvh);
  Stager<T, DP, KT, THREADS> sk, sv;
  sk.keys(a.k_stride[1], a.dim);
  sv.keys(a.v_stride[1], a.dim);
  auto stage = [&](int t, int buffer) {
    char* const to = lds + buffer * 2 * TILE_BYTES;
    sk.load_keys(kb, a.k_stride[1], t * KT, end, a.dim, to);
    sv.load_keys(vb, a.v_stride[1], t * KT, end, a.dim, to + TILE_BYTES);
  };
  if (t0 < t1) stage(t0, 0);
  in_turn(t0, t1, [&](int t, auto buffer) {
    constexpr int B = decltype(buffer)::value;
    arrived();
    if (t + 1 < t1) stage(t + 1, 1 - B);
    char* const kt = lds + B * 2 * TILE_BYTES;
    char* const vt = kt + TILE_BYTES;
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
    // the running maximum moves only when some row's grew by more than 2^8: exp stays far inside fp32
    float m = s[0][0];
#pragma unroll
    for (int b = 0; b < KB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) m = fmaxf(m, s[b][i]);
    m = max_halves(m);
    if (__any(fmaf(m, c, -8.f) > top * c)) {
      const float to = fmaxf(top, m);
      const float f = to == -INFINITY ? 1.f : exp2_((top - to) * c);
      top = to;
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
          drop_bits(a, rng, stat, ((key0 + 32 * b) >> 4) + k16, h, bits);
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
  });
  sum = sum_halves(sum);

  if constexpr (WK > 1) {
    // join the waves that shared the rows: statistics, then the scaled accumulators, in a fixed order
    float* const stat = reinterpret_cast<float*>(lds);              // [WK][ROWS][2]
    float* const part = stat + WK * ROWS * 2;                       // [WK][ROWS][JOIN_ROW]
    const int at_row = wr * 32 + (lane & 31);
    __syncthreads();
    if (h == 0) {
      stat[(wk * ROWS + at_row) * 2] = top;
      stat[(wk * ROWS + at_row) * 2 + 1] = sum;
    }
    __syncthreads();
    float to = -INFINITY;
#pragma unroll
    for (int i = 0; i < WK; ++i) to = fmaxf(to, stat[(i * ROWS + at_row) * 2]);
    const float f = to == -INFINITY ? 0.f : exp2_((top - to) * c);
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < WK; ++i) {
      const float ti = stat[(i * ROWS + at_row) * 2];
      const float si = stat[(i * ROWS + at_row) * 2 + 1];
      sum += ti == -INFINITY ? si : si * exp2_((ti - to) * c);   // NaN (a maximum leaves it out) or 0 beside -inf
    }
    top = to;
    if (wk > 0) store_row<float, DP>(part + (wk * ROWS + at_row) * JOIN_ROW, acc, f, h, DP);
    __syncthreads();
    if (wk > 0) return;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float4 v = make_float4(acc[d][4 * g] * f, acc[d][4 * g + 1] * f, acc[d][4 * g + 2] * f, acc[d][4 * g + 3] * f);
#pragma unroll
        for (int i = 1; i < WK; ++i) {
          const float4 u = *reinterpret_cast<const float4*>(part + (i * ROWS + at_row) * JOIN_ROW + 32 * d + 8 * g + 4 * h);
          v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
        }
        acc[d][4 * g] = v.x; acc[d][4 * g + 1] = v.y; acc[d][4 * g + 2] = v.z; acc[d][4 * g + 3] = v.w;
      }
  }
  if (row >= rows) return;
  if (a.splits > 1) {
    // [split][batch x key heads][rows][DP], and the statistics as [..][rows][2]; nothing for a row without keys
    if (limit == 0) return;
    const int64_t at_part = (static_cast<int64_t>(split) * a.batch * a.kv_heads + bh) * rows + row;
    store_row<float, DP>(a.part + at_part * DP, acc, 1.f, h, DP);
    if (h == 0) {
      a.part_ml[at_part * 2] = top;
      a.part_ml[at_part * 2 + 1] = sum;
    }
    return;
  }
  const bool any = limit > 0 && (sum > 0.f || sum != sum);
  if (!any) {   // not zero times them: what others see may be infinite
#pragma unroll
    for (int m = 0; m < DP / 32; ++m) zero(acc[m]);
  }
  store_row<T, DP>(at<T>(a.out, a.o_stride, w.b, token, head), acc, any ? a.inv_keep / sum : 0.f, h, a.dim);
  if (h == 0) a.lse[stat] = any ? fmaf(top, a.scale, __builtin_amdgcn_logf(sum) * LN2) : -INFINITY;
}

// Joins the splits of one row, a wave a row: lane s takes the statistics of split s, then groups
// of DP / 4 lanes add splits side by side, 4 channels a lane, and the groups are added in order.
constexpr int MOST_SPLITS = 64;

template <typename T, int DP>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a) {
  constexpr int WIDE = DP / 4, GROUPS = 64 / WIDE;
  const int lane = threadIdx.x & 63;
  const int rows = a.q_len * a.group;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t step = static_cast<int64_t>(a.batch) * a.kv_heads * rows;
  if (item >= step) return;
  const int bh = static_cast<int>(item / rows), row = static_cast<int>(item - static_cast<int64_t>(bh) * rows);
  const Where w = where(a, bh);
  const int token = row / a.group, head = w.kvh * a.group + row - token * a.group;
  const bool keys = seen(a, w, token) > 0;
  const int g = lane / WIDE, c = (lane - g * WIDE) * 4;
  const float* const part = a.part + item * DP + c;
  // the first splits' values are asked for with the statistics
  constexpr int AHEAD = 4;
  float4 v[AHEAD] = {};
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (keys && g < GROUPS && i * GROUPS + g < a.splits)
      v[i] = *reinterpret_cast<const float4*>(part + (i * GROUPS + g) * step * DP);
  float2 ml = make_float2(-INFINITY, 0.f);
  if (keys && lane < a.splits) ml = *reinterpret_cast<const float2*>(a.part_ml + (item + lane * step) * 2);
  float top = ml.x;
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  top = fmaxf(top, __shfl_xor(top, 16, 64));
  top = max_halves(top);
  const float f = ml.x == -INFINITY ? 0.f : exp2_((ml.x - top) * a.scale_log2);
  const float sum = sum_halves(sum_quarters(sum16(f * ml.y)));
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](int s, const float4& x) {
    const float f_s = __shfl(f, s < MOST_SPLITS ? s : 0, 64);
    if (g < GROUPS && s < a.splits && f_s > 0.f) {
      acc.x = fmaf(x.x, f_s, acc.x);
      acc.y = fmaf(x.y, f_s, acc.y);
      acc.z = fmaf(x.z, f_s, acc.z);
      acc.w = fmaf(x.w, f_s, acc.w);
    }
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) add(i * GROUPS + g, v[i]);
#pragma unroll 4
  for (int s0 = AHEAD * GROUPS; s0 < a.splits; s0 += GROUPS) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (keys && g < GROUPS && s0 + g < a.splits) x = *reinterpret_cast<const float4*>(part + (s0 + g) * step * DP);
    add(s0 + g, x);
  }
#pragma unroll
  for (int n = GROUPS / 2; n >= 1; n >>= 1) {
    acc.x += __shfl_down(acc.x, n * WIDE, 64);
    acc.y += __shfl_down(acc.y, n * WIDE, 64);
    acc.z += __shfl_down(acc.z, n * WIDE, 64);
    acc.w += __shfl_down(acc.w, n * WIDE, 64);
  }
  const bool any = sum > 0.f || sum != sum;
  const float n = any ? a.inv_keep / sum : 0.f;
  if (lane < WIDE && c < a.dim) {
    T* const o = at<T>(a.out, a.o_stride, w.b, token, head) + c;
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(acc.x * n, acc.y * n), pack_bf16x2(acc.z * n, acc.w * n));
    else
      *reinterpret_cast<float4*>(o) = make_float4(acc.x * n, acc.y * n, acc.z * n, acc.w * n);
  }
  if (lane == 0)
    a.lse[(static_cast<int64_t>(w.b) * a.heads + head) * a.q_len + token] =
        any ? fmaf(top, a.scale, __builtin_amdgcn_logf(sum) * LN2) : -INFINITY;
}

// The same for up to FEW_SPLITS splits, 4 channels a thread, which takes the row's statistics itself: the
// exchange between lanes above costs more than reading a few of them again (30000 rows of 80 channels in
// 3 splits: 15 us against 7).
constexpr int FEW_SPLITS = 8;

template <typename T, int DP>
__global__ __launch_bounds__(256) void attn_join_few_kernel(AttnArgs a) {
  constexpr int WIDE = DP / 4;
  const int rows = a.q_len * a.group;
  const int64_t step = static_cast<int64_t>(a.batch) * a.kv_heads * rows;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t item = i / WIDE;
  if (item >= step) return;
  const int c = static_cast<int>(i - item * WIDE) * 4;
  const int bh = static_cast<int>(item / rows), row = static_cast<int>(item - static_cast<int64_t>(bh) * rows);
  const Where w = where(a, bh);
  const int token = row / a.group, head = w.kvh * a.group + row - token * a.group;
  float top = -INFINITY, sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (seen(a, w, token) > 0) {
    float2 ml[FEW_SPLITS];
    float4 v[FEW_SPLITS];
#pragma unroll
    for (int s = 0; s < FEW_SPLITS; ++s) {
      ml[s] = make_float2(-INFINITY, 0.f);
      if (s < a.splits) {
        ml[s] = *reinterpret_cast<const float2*>(a.part_ml + (item + s * step) * 2);
        v[s] = *reinterpret_cast<const float4*>(a.part + (item + s * step) * DP + c);
        top = fmaxf(top, ml[s].x);
      }
    }
#pragma unroll
    for (int s = 0; s < FEW_SPLITS; ++s) {
      // nothing seen is a sum of 0: the maximum of scores that are all NaN is -inf too
      if (s >= a.splits || (ml[s].x == -INFINITY && ml[s].y == 0.f)) continue;
      const float f = ml[s].x == -INFINITY ? 0.f : exp2_((ml[s].x - top) * a.scale_log2);
      sum = fmaf(ml[s].y, f, sum);
      acc.x = fmaf(v[s].x, f, acc.x);
      acc.y = fmaf(v[s].y, f, acc.y);
      acc.z = fmaf(v[s].z, f, acc.z);
      acc.w = fmaf(v[s].w, f, acc.w);
    }
  }
  const bool any = sum > 0.f || sum != sum;
  const float n = any ? a.inv_keep / sum : 0.f;
  if (c < a.dim) {
    T* const o = at<T>(a.out, a.o_stride, w.b, token, head) + c;
    if constexpr (sizeof(T) == 2)
      *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(acc.x * n, acc.y * n), pack_bf16x2(acc.z * n, acc.w * n));
    else
      *reinterpret_cast<float4*>(o) = make_float4(acc.x * n, acc.y * n, acc.z * n, acc.w * n);
  }
  if (c == 0)
    a.lse[(static_cast<int64_t>(w.b) * a.heads + head) * a.q_len + token] =
        any ? fmaf(top, a.scale, __builtin_amdgcn_logf(sum) * LN2) : -INFINITY;
}

// ---------------------------------------------------------------------------
// backward: query gradient
// ---------------------------------------------------------------------------

// Three products a pair, each with one operand in registers (q, do, or what the last two left) and one from
// LDS; two waves a SIMD (one for the 64-row kernel of 128 channels, whose two waves have 64 KB of LDS between
// them).  2 x 4096 causal tokens, 16 heads of 128 over 4: 210 us, 980 TFLOP/s, matrix instructions busy 60 % of
// the time.
template <typename T, int DP, int WR, int KB, bool DROP>
__global__ __launch_bounds__(64 * WR, (DP * sizeof(T) > 256 ? 1 : 2)) void attn_dq_kernel(AttnArgs a) {
  using Tl = Tile<T, DP>;
  constexpr int THREADS = 64 * WR, ROWS = 32 * WR, KT = 32 * KB;
  constexpr int TILE_BYTES = KT * Tl::ROW_BYTES;
  __shared__ __attribute__((aligned(16))) char lds[4 * TILE_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const Item item = work_item(a, true);
  const int bh = item.bh, split = item.split, tile = item.tile;
  const Where w = where(a, bh);
  const int rows = a.q_len * a.group;
  const int row0 = tile * ROWS, wave0 = row0 + wave * 32;
  const int row = wave0 + (lane & 31);
  const int token = row / a.group, head = w.kvh * a.group + row - token * a.group;
  const bool in_q = row < rows;
  const int limit = in_q ? seen(a, w, token) : 0;
  const bool live = limit > 0;   // a row without keys counts as zeros, whatever it holds
  const int from = in_q ? token : 0;

  const int last_row = (row0 + ROWS < rows ? row0 + ROWS : rows) - 1;
  int last_token = last_row / a.group;
  if (last_token > w.q_len - 1) last_token = w.q_len - 1;
  const int end = row0 / a.group < w.q_len ? seen(a, w, last_token) : 0;
  int all = w.kv_len;
  if (a.causal) {
    all = wave0 / a.group + w.kv_len - w.q_len + 1;
    all = all < w.kv_len ? all : w.kv_len;
  }
  const int tiles = (end + KT - 1) / KT;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int t0 = split * per, t1 = t0 + per < tiles ? t0 + per : tiles;

  const T* const kb = at<T>(a.k, a.k_stride, w.b, 0, w.kvh);
  const T* const vb = at<T>(a.v, a.v_stride, w.b, 0, w.kvh);
  Stager<T, DP, KT, THREADS> sk, sv;
  sk.keys(a.k_stride[1], a.dim);
  sv.keys(a.v_stride[1], a.dim);
  auto stage = [&](int t, int buffer) {
    char* const to = lds + buffer * 2 * TILE_BYTES;
    sk.load_keys(kb, a.k_stride[1], t * KT, end, a.dim, to);
    sv.load_keys(vb, a.v_stride[1], t * KT, end, a.dim, to + TILE_BYTES);
  };
  // A row that sees at most the first tile takes D from that tile's own products: with few keys
  // p is large and o's rounding, which do . o would bring in, does not average out over them.
  const bool few = sizeof(T) == 2 && all <= KT && tiles > 0;
  const bool few_any = sizeof(T) == 2 && tiles > 0 && (w.kv_len <= KT || (a.causal && row0 / a.group + w.kv_len - w.q_len < KT));
  const int few_buffer = t0 == 0 ? 0 : 1;   // the first split has that tile anyway
  if (few_any && few_buffer == 1) stage(0, 1);
  if (t0 < t1) stage(t0, 0);

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
    delta = sum_halves(delta);
  }
  const int64_t stat = (static_cast<int64_t>(w.b) * a.heads + head) * a.q_len + token;
  // a row without keys, or whose scores are all -inf, which the forward took as such: lse +inf makes every p zero
  float lse = limit > 0 ? a.lse[stat] * LOG2E : INFINITY;
  if (lse == -INFINITY) lse = INFINITY;
  const float c = a.scale_log2;
  Rng rng{};
  if (DROP) rng = load_rng(a.rng);
  const int64_t drop_row = stat;

  // s = p and dp (with dropout's factor) of a block of keys
  auto products = [&](char* kt, int b, int key0, f32x16_t& s, f32x16_t& dp) {
    zero(s);
    zero(dp);
#pragma unroll
    for (int i = 0; i < Tl::STEPS; ++i) {
      s = mfma32(Tl::straight(kt, 32 * b + (lane & 31), i, h), q[i], s);
      dp = mfma32(Tl::straight(kt + TILE_BYTES, 32 * b + (lane & 31), i, h), g[i], dp);
    }
#pragma unroll
    for (int k16 = 0; k16 < 2; ++k16) {
      uint32_t bits[4];
      if (DROP) drop_bits(a, rng, drop_row, (key0 >> 4) + k16, h, bits);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = 8 * k16 + j;
        s[i] = exp2_(fmaf(s[i], c, -lse));
        if (DROP) dp[i] = kept(bits, j, a.cut) ? dp[i] * a.inv_keep : 0.f;
      }
    }
    if (key0 + 32 > all) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = key0 + 8 * (i >> 2) + 4 * h + (i & 3);
        s[i] = key < limit ? s[i] : 0.f;
      }
    }
  };

  if (few_any) {
    arrived();
    if (few) {
      float own = 0.f;
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        f32x16_t s, dp;
        products(lds + few_buffer * 2 * TILE_BYTES, b, 32 * b, s, dp);
#pragma unroll
        for (int i = 0; i < 16; ++i) own = s[i] > 0.f ? fmaf(s[i], dp[i], own) : own;
      }
      own = sum_halves(own);
      delta = limit <= KT ? own : delta;
    }
  }
  if (in_q && h == 0 && split == 0) {   // for the key gradients, by row
    a.stat_lse[static_cast<int64_t>(bh) * rows + row] = lse;
    a.stat_delta[static_cast<int64_t>(bh) * rows + row] = delta;
  }

  f32x16_t acc[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) zero(acc[m]);
  in_turn(t0, t1, [&](int t, auto buffer) {
    constexpr int B = decltype(buffer)::value;
    arrived();
    if (t + 1 < t1) stage(t + 1, 1 - B);
    char* const kt = lds + B * 2 * TILE_BYTES;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      f32x16_t s, dp;
      products(kt, b, t * KT + 32 * b, s, dp);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = s[i] * (dp[i] - delta);
#pragma unroll
      for (int k16 = 0; k16 < 2; ++k16) {
        Frag<T> p;
        operand(s, k16, p);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
          acc[d] = mfma32(Tl::across(kt, 32 * b + 16 * k16, 32 * d, lane), p, acc[d]);
      }
    }
  });
  if (!in_q) return;
  if (!live) {
#pragma unroll
    for (int m = 0; m < DP / 32; ++m) zero(acc[m]);
  }
  if (a.splits > 1) {
    if (token < w.q_len)
      store_row<float, DP>(a.part + ((static_cast<int64_t>(split) * a.batch * a.kv_heads + bh) * rows + row) * DP, acc, a.scale, h, DP);
  } else {
    store_row<T, DP>(at<T>(a.dq, a.q_stride, w.b, token, head), acc, a.scale, h, a.dim);
  }
}

// ---------------------------------------------------------------------------
// backward: key and value gradients
// ---------------------------------------------------------------------------

// One wave a SIMD above 64 channels of bf16: its key and value rows, and their gradients, take 192
// registers.  With the value rows in LDS and two waves a SIMD it has too few left to ask for its
// operands early: 439 us against 353 for 2 x 4096 causal tokens, 16 heads of 128 over 4, where the
// matrix instructions are busy 40 % of the time (780 TFLOP/s).
template <typename T, int DP, int WC, int RB, bool DROP>
__global__ __launch_bounds__(64 * WC, (DP * sizeof(T) > 128 ? 1 : 2)) void attn_dkv_kernel(AttnArgs a) {
  using Tl = Tile<T, DP>;
  constexpr int THREADS = 64 * WC, KEYS = 32 * WC, RT = 32 * RB;
  constexpr int TILE_BYTES = RT * Tl::ROW_BYTES, STAT_BYTES = 512;
  constexpr int BUFFER = 2 * TILE_BYTES + STAT_BYTES;
  __shared__ __attribute__((aligned(16))) char lds[2 * BUFFER];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const Item item = work_item(a, false);
  const int bh = item.bh, split = item.split, tile = item.tile;
  const Where w = where(a, bh);
  const int key0 = tile * KEYS + wave * 32, key = key0 + (lane & 31);
  const bool live = key < w.kv_len;
  const int key_at = live ? key : 0;

  const int rows = w.q_len * a.group;
  // the first token that sees the workgroup's first key
  int first = 0;
  if (a.causal) first = tile * KEYS - (w.kv_len - w.q_len);
  first = first < 0 ? 0 : first;
  const bool any = tile * KEYS < w.kv_len && first < w.q_len;
  const int from = any ? first * a.group / RT : 0, tiles = any ? (rows + RT - 1) / RT - from : 0;
  const int per = (tiles + a.splits - 1) / a.splits;
  const int t0 = from + split * per, t1 = split * per + per < tiles ? t0 + per : from + tiles;
  const float c = a.scale_log2;
  Rng rng{};
  if (DROP) rng = load_rng(a.rng);

  const T* const qb = at<T>(a.q, a.q_stride, w.b, 0, w.kvh * a.group);
  const T* const gb = at<T>(a.d_o, a.o_stride, w.b, 0, w.kvh * a.group);
  Stager<T, DP, RT, THREADS> sq, sg;
  const bool same = RT % a.group == 0;   // every whole tile has the same offsets
  auto lay = [&](int r0, int left) {
    sq.queries(a.q_stride[1], a.q_stride[2], r0, left, a.group, a.dim);
    sg.queries(a.o_stride[1], a.o_stride[2], r0, left, a.group, a.dim);
  };
  const int64_t stat0 = static_cast<int64_t>(bh) * a.q_len * a.group;
  auto stage = [&](int t, bool first_tile) {
    const int r0 = t * RT, left = rows - r0, token0 = r0 / a.group;
    if (first_tile || !same || left < RT) lay(r0, left);
    // rows that see no key at all are staged as zeros: only the first tile can have such
    const int blind = first_tile && a.causal && w.q_len > w.kv_len ? (w.q_len - w.kv_len) * a.group - r0 : 0;
    if (blind > 0) {
      sq.skip(blind);
      sg.skip(blind);
    }
    char* const to = lds + (t & 1) * BUFFER;
    sq.load(qb + token0 * a.q_stride[1], 0x7fffffffu, to);
    sg.load(gb + token0 * a.o_stride[1], 0x7fffffffu, to + TILE_BYTES);
    float* const st = reinterpret_cast<float*>(to + 2 * TILE_BYTES);
    const int bytes = (left < RT ? left : RT) * 4;
    if (wave == 0) stage_floats(a.stat_lse + stat0 + r0, bytes, st);
    if (wave == 1) stage_floats(a.stat_delta + stat0 + r0, bytes, st + 64);
    if (blind > 0) lay(r0, left);
  };
  if (t0 < t1) stage(t0, true);

  Frag<T> k[Tl::STEPS], v[Tl::STEPS];
  load_row<T, DP>(at<T>(a.k, a.k_stride, w.b, key_at, w.kvh), live, h, a.dim, k);
  load_row<T, DP>(at<T>(a.v, a.v_stride, w.b, key_at, w.kvh), live, h, a.dim, v);
  f32x16_t dk[DP / 32], dv[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) {
    zero(dk[m]);
    zero(dv[m]);
  }
  for (int t = t0; t < t1; ++t) {
    arrived();
    if (t + 1 < t1) stage(t + 1, false);
    char* const qt = lds + (t & 1) * BUFFER;
    char* const gt = qt + TILE_BYTES;
    const float* const lse_t = reinterpret_cast<const float*>(gt + TILE_BYTES);
    const float* const delta_t = lse_t + 64;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      const int row0 = t * RT + 32 * b;
      uint32_t keep = 0xffffffffu;   // bit n: row row0 + n keeps this lane's key
      if (DROP) {
        // the generator's groups run along the keys: each lane draws for its row, and the wave turns the
        // 32 x 32 bits round (a compare gives the bits of one key of each half for 32 rows)
        const int r = row0 + (lane & 31);
        const int token = r / a.group, head = w.kvh * a.group + r - token * a.group;
        const int64_t drop_row = (static_cast<int64_t>(w.b) * a.heads + head) * a.q_len + token;
        int turned = 0;   // lane n < 32: the bits of key n
#pragma unroll
        for (int k16 = 0; k16 < 2; ++k16) {
          uint32_t bits[4];
          drop_bits(a, rng, drop_row, (key0 >> 4) + k16, h, bits);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const uint64_t m = __ballot(kept(bits, j, a.cut));
            const int n = 16 * k16 + 8 * (j >> 2) + (j & 3);   // key of the lower half
            // (two wait states after the compare that wrote m)
            asm("s_nop 1\n\tv_writelane_b32 %0, %1, %3\n\tv_writelane_b32 %0, %2, %4"
                : "+v"(turned) : "s"(static_cast<int>(m)), "s"(static_cast<int>(m >> 32)), "i"(n), "i"(n + 4));
          }
        }
        keep = __builtin_amdgcn_permlane32_swap(turned, turned, false, false)[0];   // the lower half's, in both
        __builtin_amdgcn_sched_barrier(0);   // before the products: their registers are not yet in use
      }
      f32x16_t s, dp;
      zero(s);
      zero(dp);
#pragma unroll
      for (int i = 0; i < Tl::STEPS; ++i) {
        s = mfma32(Tl::straight(qt, 32 * b + (lane & 31), i, h), k[i], s);
        dp = mfma32(Tl::straight(gt, 32 * b + (lane & 31), i, h), v[i], dp);
      }
      // the block has pairs that are hidden
      const int before = key - (w.kv_len - w.q_len);      // tokens that do not see this lane's key
      const bool hidden = a.causal && row0 < max(key0 + 31 - (w.kv_len - w.q_len), 0) * a.group;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 l4 = *reinterpret_cast<const float4*>(lse_t + 32 * b + 8 * g + 4 * h);
        const float ll[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) s[4 * g + j] = exp2_(fmaf(s[4 * g + j], c, -ll[j]));
      }
      if (hidden) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int r = row0 + 8 * (i >> 2) + 4 * h + (i & 3);
          s[i] = r >= max(before, 0) * a.group ? s[i] : 0.f;
        }
      }
      // dp becomes ds, and s what multiplies do
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 d4 = *reinterpret_cast<const float4*>(delta_t + 32 * b + 8 * g + 4 * h);
        const float dd[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = 4 * g + j;
          float d = dp[i], pm = s[i];
          if (DROP) {
            const bool kp = (keep >> (8 * g + 4 * h + j)) & 1;
            d = kp ? d * a.inv_keep : 0.f;
            pm = kp ? pm : 0.f;
          }
          dp[i] = s[i] * (d - dd[j]);
          s[i] = pm;
        }
      }
#pragma unroll
      for (int r16 = 0; r16 < 2; ++r16) {
        Frag<T> p, d;
        operand(s, r16, p);
        operand(dp, r16, d);
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
  if (a.splits > 1) {
    // [dk, dv][split][batch x key heads][keys][DP]
    if (!live) return;
    const int64_t bhs = static_cast<int64_t>(a.batch) * a.kv_heads;
    float* const to = a.part + ((split * bhs + bh) * a.kv_len + key) * DP;
    store_row<float, DP>(to, dk, a.scale, h, DP);
    store_row<float, DP>(to + a.splits * bhs * a.kv_len * DP, dv, a.inv_keep, h, DP);
  } else {
    store_row<T, DP>(at<T>(a.dk, a.k_stride, w.b, key, w.kvh), dk, a.scale, h, a.dim);
    store_row<T, DP>(at<T>(a.dv, a.v_stride, w.b, key, w.kvh), dv, a.inv_keep, h, a.dim);
  }
}

// Adds the splits of a gradient, 4 channels a thread, in their order: rows of [batch x key heads][rows].
struct SumArgs {
  const float* part;
  void* out;
  int64_t stride[3];
  const int32_t* lens;   // of the rows' tokens: those past them have no partial results
  int64_t items, step;   // rows x DP / 4, elements between splits
  int rows, splits, kv_heads, group, dim;
};

template <typename T, int DP>
__global__ __launch_bounds__(256) void attn_sum_kernel(SumArgs a0, SumArgs a1) {
  const SumArgs& a = blockIdx.y == 0 ? a0 : a1;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= a.items) return;
  const int64_t r = i / (DP / 4);
  const int d = static_cast<int>(i - r * (DP / 4)) * 4;
  if (d >= a.dim) return;
  const int bh = static_cast<int>(r / a.rows), row = static_cast<int>(r - static_cast<int64_t>(bh) * a.rows);
  const int b = bh / a.kv_heads, kvh = bh - b * a.kv_heads, token = row / a.group;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (a.lens == nullptr || token < a.lens[b])
#pragma unroll 4
    for (int n = 0; n < a.splits; ++n) {
      const float4 v = *reinterpret_cast<const float4*>(a.part + n * a.step + r * DP + d);
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
  T* const to = at<T>(a.out, a.stride, b, token, kvh * a.group + row - token * a.group) + d;
  if constexpr (sizeof(T) == 2)
    *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(s.x, s.y), pack_bf16x2(s.z, s.w));
  else
    *reinterpret_cast<float4*>(to) = s;
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

template <typename T> struct Shape { static constexpr int KB = 2; };
template <> struct Shape<float> { static constexpr int KB = 1; };

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Launches tiles x splits workgroups for each (batch row, key head).  A grid has fewer than 2^32 lanes: more
// heads than that holds go in several launches.  (One head always fits: 2^23 tiles at most, and splits only
// where there are few workgroups.)
void launch(AttnArgs& a, int64_t tiles, int splits, int threads, hipStream_t s, void (*kernel)(AttnArgs)) {
  a.tiles = static_cast<int>(tiles);
  a.splits = splits;
  const int64_t bh = static_cast<int64_t>(a.batch) * a.kv_heads, most = 0xffffffffll / threads / (tiles * splits);
  for (int64_t first = 0; first < bh; first += most) {
    a.bh0 = static_cast<int>(first);
    a.bhs = static_cast<int>(bh - first < most ? bh - first : most);
    kernel<<<static_cast<unsigned>(tiles * splits * a.bhs), threads, 0, s>>>(a);
  }
}

template <typename T, int DP, bool DROP>
void forward_by(AttnArgs& a, const AttnPlan& p, hipStream_t s) {
  const int rows = a.q_len * a.group, bh = a.batch * a.kv_heads;
  const int64_t tiles = ceil_div(rows, p.row_tile);
  if (p.row_tile == 32)
    launch(a, tiles, p.splits, 128, s, attn_forward_kernel<T, DP, 1, 2, 1, DROP>);
  else if (p.row_tile == 64)
    launch(a, tiles, p.splits, 128, s, attn_forward_kernel<T, DP, 2, 1, Shape<T>::KB, DROP>);
  else
    launch(a, tiles, p.splits, 256, s, attn_forward_kernel<T, DP, 4, 1, DP == 128 ? 1 : Shape<T>::KB, DROP>);
  const int64_t out = static_cast<int64_t>(rows) * bh;
  if (a.splits > FEW_SPLITS)
    attn_join_kernel<T, DP><<<static_cast<unsigned>(ceil_div(out, 4)), 256, 0, s>>>(a);
  else if (a.splits > 1)
    attn_join_few_kernel<T, DP><<<static_cast<unsigned>(ceil_div(out * (DP / 4), 256)), 256, 0, s>>>(a);
}

template <typename T, int DP, bool DROP>
void backward_by(AttnArgs& a, const AttnPlan& p, hipStream_t s) {
  const int rows = a.q_len * a.group, bh = a.batch * a.kv_heads;
  auto sum = [&](void* out, const int64_t (&st)[3], const int32_t* lens, int n, int splits, int group) {
    SumArgs r{a.part, out, {st[0], st[1], st[2]}, lens, static_cast<int64_t>(bh) * n * (DP / 4),
              static_cast<int64_t>(bh) * n * DP, n, splits, a.kv_heads, group, a.dim};
    return r;
  };
  if (rows > 0) {
    const int64_t tiles = ceil_div(rows, p.dq_tile);
    if (p.dq_tile == 64) launch(a, tiles, p.dq_splits, 128, s, attn_dq_kernel<T, DP, 2, Shape<T>::KB, DROP>);
    else launch(a, tiles, p.dq_splits, 256, s, attn_dq_kernel<T, DP, 4, Shape<T>::KB, DROP>);
    if (a.splits > 1) {
      const SumArgs r = sum(a.dq, a.q_stride, a.q_lens, rows, a.splits, a.group);
      attn_sum_kernel<T, DP><<<static_cast<unsigned>(ceil_div(r.items, 256)), 256, 0, s>>>(r, r);
    }
  }
  if (a.kv_len > 0) {
    const int64_t tiles = ceil_div(a.kv_len, p.key_tile);
    if (p.key_tile == 64) launch(a, tiles, p.dkv_splits, 128, s, attn_dkv_kernel<T, DP, 2, Shape<T>::KB, DROP>);
    else launch(a, tiles, p.dkv_splits, 256, s, attn_dkv_kernel<T, DP, 4, Shape<T>::KB, DROP>);
    if (a.splits > 1) {
      const SumArgs rk = sum(a.dk, a.k_stride, a.kv_lens, a.kv_len, a.splits, 1);
      SumArgs rv = sum(a.dv, a.v_stride, a.kv_lens, a.kv_len, a.splits, 1);
      rv.part += a.splits * rv.step;
      attn_sum_kernel<T, DP><<<dim3(static_cast<unsigned>(ceil_div(rk.items, 256)), 2), 256, 0, s>>>(rk, rv);
    }
  }
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

// Few workgroups for the chip, which holds `slots` at a time: their inner axis is split until
// they fill it twice (ragged lengths and causal masks leave some short), with at least `least`
// of `length` a split.  More splits cost more than they give: each writes its results in fp32.
int splits_for(int64_t blocks, int64_t slots, int64_t length, int64_t least) {
  if (blocks == 0 || 2 * blocks >= 3 * slots) return 1;
  int64_t n = ceil_div(2 * slots, blocks);
  const int64_t most = ceil_div(length, least);
  n = n < most ? n : most;
  n = n < MOST_SPLITS ? n : MOST_SPLITS;
  return static_cast<int>(n < 1 ? 1 : n);
}

}  // namespace

AttnPlan attn_plan(const AttnArgs& a) {
  AttnPlan p{};
  const int64_t rows = static_cast<int64_t>(a.q_len) * a.group, bh = static_cast<int64_t>(a.batch) * a.kv_heads;
  // 128 rows or keys a workgroup share what it brings to LDS; more small workgroups in place of splits
  // are slower (5 x 1000 ragged tokens: dk and dv 72 us by 64 keys, 46 by 128), unless 64 is all there is
  p.row_tile = rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  // 256 slots by 64 and 128 rows, where 512 are slower (777 over 1023 fp32 ragged 40 us against 30, 1000 over 4000, 8
  // heads of 64, 29 against 26, its gradients by 32 channels 75 against 66).  By 32 rows neither is best throughout,
  // whatever the type and width: single tokens over 4097 keys, 4 key heads, 512 against 256: 8 requests 15 / 14
  // (128 channels 25 / 21, fp32 79 / 62); 48: 42 / 38 (fp32 99 / 119; 128 channels 84 / 93, fp32 294 / 328); 160: 153 / 129
  // (fp32 282 / 350; 128 channels 253 / 290, fp32 822 / 941), ragged 73 / 76; 128 ragged 56 / 60.
  p.splits = splits_for(ceil_div(rows, p.row_tile) * bh, p.row_tile == 32 ? 512 : 256, a.kv_len, 128);
  p.dq_tile = rows <= 64 ? 64 : 128;
  p.key_tile = a.kv_len <= 64 ? 64 : 128;
  const size_t row = static_cast<size_t>(padded(a.dim)) * 4;
  p.fwd_bytes = p.splits > 1 ? p.splits * bh * rows * (row + 8) : 0;
  p.dq_splits = splits_for(ceil_div(rows, p.dq_tile) * bh, 256, a.kv_len, 256);
  p.dkv_splits = splits_for(ceil_div(a.kv_len, p.key_tile) * bh, 256, rows, 256);
  const size_t dq = p.dq_splits > 1 ? p.dq_splits * bh * rows * row : 0;
  const size_t dkv = p.dkv_splits > 1 ? 2 * p.dkv_splits * bh * a.kv_len * row : 0;
  p.stat_bytes = 2 * ((static_cast<size_t>(bh) * rows * 4 + 15) / 16 * 16);
  p.bwd_bytes = p.stat_bytes + (dq > dkv ? dq : dkv);
  return p;
}

void attn_forward(const AttnArgs& args, const AttnPlan& p, int dtype, void* workspace, hipStream_t s) {
  AttnArgs a = args;
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
  a.stat_lse = static_cast<float*>(workspace);
  a.stat_delta = a.stat_lse + p.stat_bytes / 8;
  a.part = a.stat_lse + p.stat_bytes / 4;
  if (dtype == 1) {
    PETRA_BY_DIM(backward_by, bf16_t)
  } else {
    PETRA_BY_DIM(backward_by, float)
  }
}

}  // namespace petra
