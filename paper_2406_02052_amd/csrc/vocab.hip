// The loss over a large vocabulary and its gradients, without a rows x vocabulary tensor.
//
//   s_ij = scale x_i . w_j,  lse_i = log sum_j exp s_ij,  loss_i = lse_i - s_it  (t: the row's target)
//   dx_i = scale weight_i sum_j (p_ij - [j = t]) w_j,  dw_j = scale sum_i weight_i (p_ij - [j = t]) x_i
//
// Three products of 2 rows width vocabulary operations each; bound by them for all but a few rows.
// The rows go in pieces, of which one at a time is held as e_ij = exp(s_ij - s_it) in the storage type: the
// target's score is known before the product and a softmax may take any reference, so that with R_i = sum_{j != t} e_ij
// loss_i = log(1 + R_i), and both gradients are products of e as it lies:
//   f_i = scale weight_i / (1 + R_i),  e_it = -R_i,  dx_i = f_i sum_j e_ij w_j,  dw_j = sum_i e_ij (f_i x_i)
// where a maximum as the reference would have e rescaled, or the first product made twice.  The product's own e_it is left
// out of the sums: its score is the reference's sum in another order, and what they differ by (1e-5 at scores of 30) would be
// the loss and gradient of a row whose target has all but 1e-5 of the softmax.  bf16 has the exponents of fp32; a tile
// whose sum of a row passes 2^86 takes its own largest as the reference, and the row's e are brought to one when all are
// known.
//
// Scores, sums, statistics and accumulators are fp32.  With bf16 tensors e and f x are rounded to bf16 as
// operands of the products (the matrix unit takes bf16), 2^-8 of each term at most each, e of a row with a reference of its own once
// more.  The targets' terms are most of both gradients: what rounding them left is added to the sums from the fp32 values, for dw by
// lists of the rows of each column.  Rows of dw whose column is no row's target have none: at 2048 x 1024 over 32768 they are off
// by 1.6 times what rounding them alone would leave (median), 3 at most, the others and dx by 1.0.
#include "common.h"
#include "ops.h"

namespace petra {

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

constexpr float LN2 = 0.69314718055994530942f;
// How large a tile's sum of a row may be (sums of all tiles fit fp32), and log2 of the least largest e that makes a reference of its own.
constexpr float MOST = 0x1p86f, REACH = 70.f;
constexpr float INF = __builtin_huge_valf();

__device__ __forceinline__ f32x16_t mfma32(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mfma32(const Frag<float>& a, const Frag<float>& b, f32x16_t c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
  return c;
}

// ---------------------------------------------------------------------------
// tiles of a product's operands in LDS
// ---------------------------------------------------------------------------

// FREE free indices by 128 bytes of the inner index, as they lie in memory: lines of the inner index (ALONG), or lines of
// the free one.  Chunks of 16 bytes are moved within a line by an exclusive or with a key of the line, so that the 16
// lanes of a straight read (16 lines at one chunk) and the 32 of a transposing one (4 lines at 4 chunks) meet different banks.
template <typename T, int FREE, bool ALONG, int THREADS>
struct Panel {
  static constexpr int INNER = 128 / static_cast<int>(sizeof(T));
  static constexpr int LINES = ALONG ? FREE : INNER, CHUNKS = ALONG ? 8 : FREE * static_cast<int>(sizeof(T)) / 16;
  static constexpr int BYTES = FREE * 128, N = BYTES / 16 / THREADS, PER = 16 / static_cast<int>(sizeof(T));
  static_assert(BYTES % (16 * THREADS) == 0, "whole chunks a thread");
  uint32_t off[N];
  const T* base;
  int64_t ld, step;
  int64_t left;              // elements of the tensor from `base` on

  static __device__ __forceinline__ int key(int line) {
    if constexpr (ALONG) return (line >> 1) & 7;
    else if constexpr (sizeof(T) == 2) return ((line & 3) << 2) & (CHUNKS - 1);
    else return line & 8;
  }
  static __device__ __forceinline__ int at(int line, int chunk) { return (line * CHUNKS + (chunk ^ key(line))) << 4; }
  static __device__ __forceinline__ int line(int i) { return (i * THREADS + static_cast<int>(threadIdx.x)) / CHUNKS; }
  static __device__ __forceinline__ int chunk(int i) {
    const int place = i * THREADS + static_cast<int>(threadIdx.x), l = place / CHUNKS;
    return (place - l * CHUNKS) ^ key(l);
  }

  // Free indices first .. of `free` and inner ones from k0 of a matrix at p, `inner` wide, lines ld apart.
  __device__ __forceinline__ void begin(const T* p, int64_t ld_, long first, long free, long k0, long inner) {
    ld = ld_;
    if constexpr (ALONG) {
      base = p + first * ld + k0;
      left = (free - first - 1) * ld + inner - k0;
      step = INNER;
    } else {
      base = p + k0 * ld + first;
      left = (inner - k0 - 1) * ld + free - first;
      step = INNER * ld;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t o = (static_cast<uint32_t>(line(i)) * static_cast<uint32_t>(ld) + chunk(i) * PER) * static_cast<uint32_t>(sizeof(T));
      // (past the last line: past `left`)
      off[i] = !ALONG && first + chunk(i) * PER >= free ? BUF_OOB : o;
    }
  }
  // The next tile, of which `inner` inner indices exist: a resource that ends with the tensor, and the buffer it goes to.
  struct Next {
    u32x4_t from;
    uint32_t to;
    long inner;
  };
  __device__ __forceinline__ Next next(char* lds, long inner) {
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    const int64_t bytes = left * static_cast<int64_t>(sizeof(T));
    const uint32_t most = inner <= 0 || bytes <= 0 ? 0u : bytes < 0x7fffffff ? static_cast<uint32_t>(bytes) : 0x7fffffffu;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    base += step;
    left -= step;
    return {{static_cast<uint32_t>(at), static_cast<uint32_t>(at >> 32) & 0xffffu, most, 0x00020000u},
            static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds)) + wave * 1024, inner};
  }
  // Asks for this thread's chunk i of it (CUT: a last, partial tile).  The loads are written out: the compiler would let every
  // later transposing LDS read wait for them.  They write no register, and a buffer that is not read before the next arrived(),
  // which waits for them.
  template <bool CUT>
  __device__ __forceinline__ void load(const Next& n, int i) const {
    const uint32_t o = CUT && ALONG && chunk(i) * PER >= n.inner ? BUF_OOB : off[i];
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(n.to + i * THREADS * 16), "v"(o), "s"(n.from));
  }
};

// Where in a panel a lane finds its operands: free index free0 + 32 i + (lane & 31) for i < BLOCKS, inner ones 16 k + 8 (lane >> 5) .. + 7.
// The keys leave few places that differ by lane; the rest are constants.
template <typename T, typename P, bool ALONG, int BLOCKS>
struct Reader {
  static constexpr int LINE = P::CHUNKS * 16;
  int at[ALONG ? 4 : BLOCKS];

  __device__ __forceinline__ Reader(int free0, int lane) {
    const int h = lane >> 5;
    if constexpr (ALONG) {
      const int l = free0 + (lane & 31);   // (its key does not go by 32 i)
#pragma unroll
      for (int q = 0; q < 4; ++q) at[q] = P::at(l, sizeof(T) == 2 ? 2 * q + h : 4 * (q >> 1) + 2 * h + (q & 1));
    } else if constexpr (sizeof(T) == 2) {
      const int l = 8 * h + ((lane & 15) >> 2);   // (nor by 16 k or 4)
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i) {
        const int col = free0 + 32 * i + (lane & 16) + 4 * (lane & 3);
        at[i] = P::at(l, col >> 3) + (col & 7) * 2;
      }
    } else {
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i) {
        const int col = free0 + 32 * i + (lane & 31);
        at[i] = P::at(8 * h, col >> 2) + (col & 3) * 4;
      }
    }
  }
  __device__ __forceinline__ Frag<T> get(char* lds, int i, int k) const {
    Frag<T> f;
    if constexpr (ALONG && sizeof(T) == 2) {
      f.v = *reinterpret_cast<const bf16x8_t*>(lds + at[k] + i * 32 * LINE);
    } else if constexpr (ALONG) {
      const float4 a = *reinterpret_cast<const float4*>(lds + at[2 * k] + i * 32 * LINE);
      const float4 b = *reinterpret_cast<const float4*>(lds + at[2 * k + 1] + i * 32 * LINE);
      f.v[0] = a.x; f.v[1] = a.y; f.v[2] = a.z; f.v[3] = a.w;
      f.v[4] = b.x; f.v[5] = b.y; f.v[6] = b.z; f.v[7] = b.w;
    } else if constexpr (sizeof(T) == 2) {
      char* const p = lds + at[i] + k * 16 * LINE;
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)p);
      const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(p + 4 * LINE));
      f.v = __builtin_bit_cast(bf16x8_t, s16x8_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) f.v[j] = *reinterpret_cast<const float*>(lds + at[i] + (16 * k + j) * LINE);
    }
    return f;
  }
};

template <int N> struct Const { static constexpr int value = N; };

// This wave's loads to LDS have arrived but for the newest LOADS, it has read what it asked LDS for, and every wave is here.
template <int LOADS>
__device__ __forceinline__ void arrived() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LOADS) : "memory");
}

// A tile of a product: BM x BN results of A's and B's free indices, by WM x WN waves, in two buffers.  A wave has (BM / WM) x
// (BN / WN) results as blocks of 32 x 32, a row (A's free index) a lane and in lane half h the columns 8 g + 4 h + {0..3}: what a
// row needs, its sums or its factor, is then a lane's.
template <typename T, int BM_, int BN_, int WM_, int WN_, bool A_ALONG, bool B_ALONG>
struct Product {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, THREADS = 64 * WM * WN;
  static constexpr int MB = BM / WM / 32, NB = BN / WN / 32;
  using A = Panel<T, BM, A_ALONG, THREADS>;
  using B = Panel<T, BN, B_ALONG, THREADS>;
  static constexpr bool CUT = A_ALONG && B_ALONG;   // (e is padded to whole tiles)
  static constexpr int BUF = A::BYTES + B::BYTES, LDS = 2 * BUF, INNER = A::INNER, LOADS = A::N + B::N;

  // acc += the inner indices k0 .. k1 (k0 a multiple of INNER); a.begin() and b.begin() have been called at k0.  A tile is taken 16
  // inner indices at a time, and the operands of the next 16 are read while the matrix unit has these: at the tile's last 16 all
  // reads of its buffer are done, so that the next tile is waited for there, its first operands read, and the buffer given to
  // the tile after it.  Reads and loads go one by one between the matrix instructions, in the order written.
  static __device__ __forceinline__ void run(A& a, B& b, long k0, long k1, char* lds, f32x16_t (&acc)[MB][NB]) {
    constexpr int PARTS = INNER / 16, M = MB * NB, R = MB + NB;
    static_assert(PARTS % 2 == 0, "operands in turn");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m0 = wave / WN * (BM / WM), n0 = wave % WN * (BN / WN);
    // a last part of lines of the inner index goes after the whole tiles; of lines of free ones those past the end are zeros
    const int steps = static_cast<int>((k1 - k0 + (CUT ? 0 : INNER - 1)) / INNER);
    const Reader<T, A, A_ALONG, MB> ra(m0, lane);
    const Reader<T, B, B_ALONG, NB> rb(n0, lane);
    Frag<T> fa[2][MB], fb[2][NB];
    auto read = [&](char* from, int k, int r, Frag<T> (&x)[MB], Frag<T> (&y)[NB]) {
      if (r < NB) y[r < NB ? r : 0] = rb.get(from + A::BYTES, r, k);
      else x[r < NB ? 0 : r - NB] = ra.get(from, r - NB, k);
    };
    auto fetch = [&](int s, char* to) {   // (past the end: nothing)
      const long inner = s < steps ? INNER : 0;
      const typename A::Next na = a.next(to, inner);
      const typename B::Next nb = b.next(to + A::BYTES, inner);
#pragma unroll
      for (int i = 0; i < A::N; ++i) a.template load<false>(na, i);
#pragma unroll
      for (int i = 0; i < B::N; ++i) b.template load<false>(nb, i);
    };
    fetch(0, lds);
    fetch(1, lds + BUF);
    arrived<LOADS>();
#pragma unroll
    for (int r = 0; r < R; ++r) read(lds, 0, r, fa[0], fb[0]);
    auto body = [&](int s, auto buf) {
      constexpr int I = decltype(buf)::value;
      char *const at = lds + I * BUF, *const other = lds + (1 - I) * BUF;
#pragma unroll
      for (int k = 0; k < PARTS; ++k) {
        const bool last = k + 1 == PARTS;
        const int now = k & 1, then = 1 - now;
        typename A::Next na{};
        typename B::Next nb{};
        if (last) {
          const long inner = s + 2 < steps ? INNER : 0;
          na = a.next(at, inner);
          nb = b.next(at + A::BYTES, inner);
          arrived<0>();
        }
#pragma unroll
        for (int m = 0; m < M; ++m) {
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (r * M / R == m) read(last ? other : at, last ? 0 : k + 1, r, fa[then], fb[then]);
          if (last) {
#pragma unroll
            for (int i = 0; i < A::N; ++i)
              if (i * M / LOADS == m) a.template load<false>(na, i);
#pragma unroll
            for (int i = 0; i < B::N; ++i)
              if ((A::N + i) * M / LOADS == m) b.template load<false>(nb, i);
          }
          acc[m / NB][m % NB] = mfma32(fb[now][m % NB], fa[now][m / NB], acc[m / NB][m % NB]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    for (int s = 0; s < steps; s += 2) {
      body(s, Const<0>{});
      if (s + 1 < steps) body(s + 1, Const<1>{});
    }
    arrived<0>();   // LDS is free
    if constexpr (CUT) {
      const long inner = k1 - k0 - static_cast<long>(steps) * INNER;
      if (inner > 0) {
        a.base -= 2 * a.step, a.left += 2 * a.step, b.base -= 2 * b.step, b.left += 2 * b.step;   // (asked for nothing twice)
        const typename A::Next na = a.next(lds, inner);
        const typename B::Next nb = b.next(lds + A::BYTES, inner);
#pragma unroll
        for (int i = 0; i < A::N; ++i) a.template load<true>(na, i);
#pragma unroll
        for (int i = 0; i < B::N; ++i) b.template load<true>(nb, i);
        arrived<0>();
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
#pragma unroll
          for (int r = 0; r < R; ++r) read(lds, k, r, fa[0], fb[0]);
#pragma unroll
          for (int m = 0; m < M; ++m) acc[m / NB][m % NB] = mfma32(fb[0][m % NB], fa[0][m / NB], acc[m / NB][m % NB]);
        }
        arrived<0>();
      }
    }
  }
  static __device__ __forceinline__ void zero(f32x16_t (&acc)[MB][NB]) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  }
};

// The tile of workgroup `id` of ms x ns: each of the 8 XCDs, which take workgroups in turn, has a run of tiles, in groups of 8 along
// m with m fastest, so that the 32 workgroups of an XCD share 8 + 4 panels through its L2.
__device__ __forceinline__ void tile_of(int id, int ms, int ns, int& m, int& n) {
  const int all = ms * ns, per = all / 8, more = all % 8;
  const int x = id & 7;
  const int t = x * per + (x < more ? x : more) + (id >> 3);
  const int group = t / (8 * ns), in = t - group * 8 * ns;
  const int size = ms - group * 8 < 8 ? ms - group * 8 : 8;
  n = in / size;
  m = group * 8 + in - n * size;
}

// ---------------------------------------------------------------------------
// rows
// ---------------------------------------------------------------------------

// Whether a row takes part: its target is a column.
__device__ __forceinline__ bool takes_part(const VocabArgs& a, long row) {
  return static_cast<uint32_t>(a.targets[row]) < static_cast<uint32_t>(a.vocab);
}

__device__ __forceinline__ float wave_sum(float v) { return sum_halves(sum_quarters(sum16(v))); }
__device__ __forceinline__ float max16f(float v) {
  auto over = [](float x, auto dpp) {
    return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(dpp)::value, 0xF, 0xF, false)));
  };
  v = over(v, Const<0xB1>{});
  v = over(v, Const<0x4E>{});
  v = over(v, Const<0x141>{});
  return over(v, Const<0x140>{});
}

// The rows of a piece by their targets, those of one target in their own order: start[j] .. start[j + 1] of `order` are the rows with
// target j.  A workgroup takes 256 columns and reads all targets twice, a quarter each wave: how many are below its columns
// and at each of them, then where each row goes, wave after wave and a wave's rows in turn.
__device__ __forceinline__ void list_rows(const VocabArgs& a, int base) {
  __shared__ int count[4][256], below[4], sums[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t* const targets = a.targets + a.row0;
  const long part = (a.piece + 255) / 256 * 64, from = wave * part, to = from + part < a.piece ? from + part : a.piece;
#pragma unroll
  for (int w = 0; w < 4; ++w) count[w][tid] = 0;
  __syncthreads();
  int less = 0;
#pragma unroll 4
  for (long i = from + lane; i < to; i += 64) {
    const int t = targets[i], c = t - base;
    if (t < 0 || t >= a.vocab) continue;
    less += c < 0;
    if (c >= 0 && c < 256) atomicAdd(&count[wave][c], 1);   // (whole numbers: their order changes nothing)
  }
  for (int d = 32; d > 0; d >>= 1) less += __shfl_xor(less, d, 64);
  if (lane == 0) below[wave] = less;
  __syncthreads();
  const int n = count[0][tid] + count[1][tid] + count[2][tid] + count[3][tid];
  int upto = n;
  for (int d = 1; d < 64; d <<= 1) {
    const int v = __shfl_up(upto, d, 64);
    if (lane >= d) upto += v;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int at = below[0] + below[1] + below[2] + below[3] + upto - n;
  for (int w = 0; w < wave; ++w) at += sums[w];
  if (base + tid < a.vocab) a.start[base + tid] = at;
  if (base + tid == a.vocab - 1) a.start[a.vocab] = at + n;
#pragma unroll
  for (int w = 0; w < 4; ++w) {   // where the next row of this column goes, for each wave
    const int v = count[w][tid];
    count[w][tid] = at;
    at += v;
  }
  __syncthreads();
  int next = from + lane < to ? targets[from + lane] : -1;
  for (long first = from; first < to; first += 64) {
    const long i = first + lane;
    const int t = next, c = t - base;
    next = i + 64 < to ? targets[i + 64] : -1;
    const bool in = t >= 0 && t < a.vocab && c >= 0 && c < 256;
    // the lanes with the same column, by its bits: the first of them takes places for all, in the lanes' order
    uint64_t same = __ballot(in);
    if (same == 0) continue;
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const bool set = (c >> b & 1) != 0;
      const uint64_t with = __ballot(set);
      same &= set ? with : ~with;
    }
    const int leader = in ? __ffsll(static_cast<unsigned long long>(same)) - 1 : 0;
    int place = 0;
    if (in && lane == leader) place = atomicAdd(&count[wave][c], __popcll(same));
    place = __shfl(place, leader, 64);
    if (in) a.order[place + __popcll(same & ((uint64_t{1} << lane) - 1))] = static_cast<int>(i);
  }
}

// A row's reference, its target's score in binary logarithms, a wave a row of those at work.  The first `lists` workgroups list the
// rows by their targets: beside the others that takes no time of its own (7 us as a launch, at 2048 rows over 32768).
template <typename T>
__global__ __launch_bounds__(256) void vocab_target_kernel(VocabArgs a, int lists) {
  if (static_cast<int>(blockIdx.x) < lists) {
    list_rows(a, static_cast<int>(blockIdx.x) * 256);
    return;
  }
  const long of = static_cast<long>(blockIdx.x - lists) * 4 + (threadIdx.x >> 6), row = a.row0 + of;
  const int lane = threadIdx.x & 63;
  if (of >= a.piece || !takes_part(a, row)) return;
  const int t = a.targets[row];
  const T* const x = static_cast<const T*>(a.x) + row * a.width;
  const T* const w = static_cast<const T*>(a.w) + static_cast<long>(t) * a.width;
  float s = 0.f;
  for (int c = lane * 8; c < a.width; c += 512) {
    float p[8], q[8];
    Vec8<T>::load(x + c, p);
    Vec8<T>::load(w + c, q);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(p[e], q[e], s);
  }
  s = wave_sum(s);
  if (lane == 0) a.ref[row] = s * a.scale_log2;
}

// 1 / (the rows that take part).
__global__ __launch_bounds__(1024) void vocab_mean_kernel(VocabArgs a) {
  __shared__ int counts[16];
  int n = 0;
  for (long r = threadIdx.x; r < a.rows; r += 1024) n += takes_part(a, r);
  for (int d = 32; d > 0; d >>= 1) n += __shfl_xor(n, d, 64);
  if ((threadIdx.x & 63) == 0) counts[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    int all = 0;
    for (int i = 0; i < 16; ++i) all += counts[i];
    *a.mean = 1.f / static_cast<float>(all > 1 ? all : 1);
  }
}

// e of a tile (KEEP: kept; a bf16 tile goes through LDS, so that whole lines are written) and each row's sum of it.  4096 x 4096 by
// 131072 bf16 in 3.75 ms, 1.17 PFLOP/s (matrix units 65 % busy at 1.75 GHz, where power holds the clock); with 1024 inner indices the 65536
// exponentials of a tile come after 16 steps only: 2048 by 32768 in 160 to 177 us, 0.8.  With e written by the lanes that hold it, 8 bytes in a
// line each, the larger takes 4.14 ms.  The slow path's maximum and the ordinary exponentials share the scaled scores, some of which are
// kept in memory between (36 registers a lane; 20 without e).
template <typename T, typename P, bool KEEP>
__global__ __launch_bounds__(P::THREADS, 2) void vocab_scores_kernel(VocabArgs a) {
  constexpr int MB = P::MB, NB = P::NB, CHUNKS = P::BN / 8;   // chunks of 16 bytes of a line of e, moved by the line's number
  __shared__ __attribute__((aligned(16))) char lds[P::LDS + P::WN * P::BM * 4];
  float* const shared = reinterpret_cast<float*>(lds + P::LDS);   // [wave column][row of the tile]
  int mt, nt;
  tile_of(blockIdx.x, a.row_tiles, a.col_tiles, mt, nt);
  const long m0 = static_cast<long>(mt) * P::BM, n0 = static_cast<long>(nt) * P::BN;
  f32x16_t acc[MB][NB];
  P::zero(acc);
  {
    typename P::A pa;
    typename P::B pb;
    pa.begin(static_cast<const T*>(a.x) + a.row0 * a.width, a.width, m0, a.piece, 0, a.width);
    pb.begin(static_cast<const T*>(a.w), a.width, n0, a.vocab, 0, a.width);
    P::run(pa, pb, 0, a.width, lds, acc);
  }
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / P::WN * (P::BM / P::WM) + (lane & 31), wn = wave % P::WN * (P::BN / P::WN);
  if (n0 + P::BN > a.vocab) {
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (n0 + wn + 32 * j + 8 * (e >> 2) + 4 * h + (e & 3) >= a.vocab)
#pragma unroll
          for (int i = 0; i < MB; ++i) acc[i][j][e] = -INF;
  }
  float c[MB];
  uint32_t live[MB];   // all ones for a row that takes part
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const long row = m0 + wm + 32 * i;
    const bool in = row < a.piece && takes_part(a, a.row0 + row);
    live[i] = in ? ~0u : 0u;
    c[i] = in ? -a.ref[a.row0 + row] : 0.f;
    // the target's, which few waves have
    const int own = in ? a.targets[a.row0 + row] - static_cast<int>(n0) - wn : -1;
    if (__any(own >= 0 && own < 32 * NB)) {
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (own == 32 * j + 8 * (e >> 2) + 4 * h + (e & 3)) acc[i][j][e] = -INF;
    }
  }
  // e and its sums; whether a row's passed MOST
  auto exponentials = [&]() {
    bool over = false;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      const long row = m0 + wm + 32 * i;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][4 * g + e], a.scale_log2, c[i]));
            sum += v[e];
          }
          const int n = wn + 32 * j + 8 * g;
          if constexpr (KEEP && sizeof(T) == 2) {
            *reinterpret_cast<uint2*>(lds + (wm + 32 * i) * (CHUNKS * 16) + (((n >> 3) ^ (lane & 31 & (CHUNKS - 1))) << 4) + 8 * h) =
                make_uint2(pack_bf16x2(v[0], v[1]) & live[i], pack_bf16x2(v[2], v[3]) & live[i]);
          } else if constexpr (KEEP) {
            if (row < a.piece && n0 + n < a.vocab_padded)
              *reinterpret_cast<float4*>(static_cast<T*>(a.e) + row * a.vocab_padded + n0 + n + 4 * h) =
                  live[i] ? make_float4(v[0], v[1], v[2], v[3]) : make_float4(0.f, 0.f, 0.f, 0.f);
          }
        }
      sum = sum_halves(sum);
      over |= live[i] && sum > MOST;
      if (h == 0) shared[(wave % P::WN) * P::BM + wm + 32 * i] = sum;
    }
    return over;
  };
  // rows that need another reference are rare: their whole tile is done again, with their largest as the reference
  const bool slow = __syncthreads_or(exponentials());
  if (slow) {
    float top[MB];
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      top[i] = -INF;
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) top[i] = fmaxf(top[i], fmaf(acc[i][j][e], a.scale_log2, c[i]));
      top[i] = max_halves(top[i]);
      if (h == 0) shared[(wave % P::WN) * P::BM + wm + 32 * i] = top[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MB; ++i) {
#pragma unroll
      for (int w = 0; w < P::WN; ++w) top[i] = fmaxf(top[i], shared[w * P::BM + wm + 32 * i]);
      const long row = m0 + wm + 32 * i;
      const float shift = top[i] > REACH ? top[i] : 0.f;
      c[i] -= shift;
      if (h == 0 && wave % P::WN == 0 && row < a.piece) a.shift[row * a.col_tiles + nt] = shift;
    }
    __syncthreads();
    exponentials();
    __syncthreads();
  }
  for (int r = threadIdx.x; r < P::BM; r += P::THREADS) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < P::WN; ++w) s += shared[w * P::BM + r];
    if (m0 + r < a.piece) a.sums[(m0 + r) * a.col_tiles + nt] = s;
  }
  if (threadIdx.x == 0) a.slow[static_cast<long>(mt) * a.col_tiles + nt] = slow;
  if constexpr (KEEP && sizeof(T) == 2) {
    const int chunk = threadIdx.x % CHUNKS;
    const long col = n0 + chunk * 8;
    for (int r = threadIdx.x / CHUNKS; r < P::BM; r += P::THREADS / CHUNKS)
      if (m0 + r < a.piece && col < a.vocab_padded)
        *reinterpret_cast<uint4*>(static_cast<T*>(a.e) + (m0 + r) * a.vocab_padded + col) =
            *reinterpret_cast<const uint4*>(lds + r * (CHUNKS * 16) + ((chunk ^ (r & 31 & (CHUNKS - 1))) << 4));
  }
}

// A row's R, loss and lse from its tiles' sums; with gradients also its factor, f x, the target's e and what had another
// reference.  A workgroup a row: 4096 rows of 4096 over 512 tiles in 20 us.
template <typename T, bool KEEP>
__global__ __launch_bounds__(256) void vocab_join_kernel(VocabArgs a) {
  __shared__ float lds[8];
  const long row = blockIdx.x, all = a.row0 + row;
  const float* const sums = a.sums + row * a.col_tiles;
  const float* const shifts = a.shift + row * a.col_tiles;
  const int* const slow = a.slow + row / a.row_tile * a.col_tiles;
  T* const scaled = KEEP ? static_cast<T*>(a.scaled) + row * a.width : nullptr;
  if (!takes_part(a, all)) {
    if (threadIdx.x == 0) {
      a.loss[all] = 0.f;
      a.lse[all] = 0.f;
      if (KEEP) a.factor[row] = a.rest[row] = a.term[row] = 0.f;
    }
    if (KEEP) {
      const float none[8] = {};
      for (int c = threadIdx.x * 8; c < a.width; c += 2048) Vec8<T>::store(scaled + c, none);
    }
    return;
  }
  const float ref = a.ref[all];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float s = 0.f, top = 0.f;
  for (int t = threadIdx.x; t < a.col_tiles; t += 256)
    if (slow[t]) top = fmaxf(top, shifts[t]);
  top = max_halves(max16f(fmaxf(top, __shfl_xor(top, 16, 64))));
  if (lane == 0) lds[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
  for (int t = threadIdx.x; t < a.col_tiles; t += 256)
    s += top > 0.f ? sums[t] * __builtin_amdgcn_exp2f((slow[t] ? shifts[t] : 0.f) - top) : sums[t];
  s = wave_sum(s);
  if (lane == 0) lds[4 + wave] = s;
  __syncthreads();
  // of the others and the target, with 2^top as the unit (own: NaN where the target's score is no finite number)
  const float rest = lds[4] + lds[5] + lds[6] + lds[7], own = __builtin_amdgcn_exp2f(ref - ref - top), z = own + rest;
  // log(1 + rest) = log(z) rest / (z - 1) with the rounded z in all places: what rounding 1 + rest lost goes out again
  const float by = z - own, log_z = LN2 * (top + log2f(z));
  const float loss = top > 0.f ? log_z : by == 0.f ? rest : log_z * (rest * __builtin_amdgcn_rcpf(by));
  if (threadIdx.x == 0) {
    a.loss[all] = loss;
    a.lse[all] = fmaf(LN2, ref, loss);
  }
  if constexpr (KEEP) {
    const float f = a.scale * (a.weight != nullptr ? a.weight[all] : *a.mean) / z;
    if (threadIdx.x == 0) a.factor[row] = f;
    T* const e = static_cast<T*>(a.e) + row * a.vocab_padded;
    if (top > 0.f) {
      for (int t = 0; t < a.col_tiles; ++t) {
        const float d = (slow[t] ? shifts[t] : 0.f) - top;
        if (d == 0.f) continue;
        const float by = __builtin_amdgcn_exp2f(d);
        for (int c = threadIdx.x; c < a.col_tile && t * a.col_tile + c < a.vocab; c += 256) {
          T* const p = e + static_cast<long>(t) * a.col_tile + c;
          store1(p, load1(p) * by);
        }
      }
      __syncthreads();   // before the target's
    }
    // the target's, of which the gradients mostly consist: what its rounding leaves goes to them by itself
    if (threadIdx.x == 0) {
      const float t = -rest;
      store1(e + a.targets[all], t);
      a.rest[row] = f * (t - quant(t, static_cast<const T*>(nullptr)));
      a.term[row] = t;
    }
    const T* const x = static_cast<const T*>(a.x) + all * a.width;
    for (int c = threadIdx.x * 8; c < a.width; c += 2048) {
      float v[8];
      Vec8<T>::load(x + c, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= f;
      Vec8<T>::store(scaled + c, v);
    }
  }
}

// ---------------------------------------------------------------------------
// gradients
// ---------------------------------------------------------------------------

// Columns with up to FEW target rows are gone through where dw's sums leave; of the others
// there are sums of runs of rows, in lines of their own: a column whose rows are first .. last - 1 of the order has at least one place
// there that is a multiple of FEW for each of its runs, and its runs' lines are those places' / FEW.
constexpr int FEW = 4;
__device__ __forceinline__ int line_of(int first) { return (first + FEW - 1) / FEW; }

// What rounding left of 4 channels w of a row's term t x f: the product took round(t) round(f x).
__device__ __forceinline__ void add_left(float t, float f, uint2 w, float (&v)[4]) {
  const float q = quant(t, static_cast<const bf16_t*>(nullptr));
  const float x[4] = {__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                      __uint_as_float(w.y & 0xffff0000u)};
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] += fmaf(f * t, x[e], -q * quant(f * x[e], static_cast<const bf16_t*>(nullptr)));
}

// Where a gradient's sums go: times the row's factor, with what is left of its target's term, added to what earlier pieces gave, and on to the tensor or to the sums
// for the next piece.
// dw's result row is a column of the vocabulary, whose target rows are order[first .. last).
template <typename T>
__device__ __forceinline__ void finish(const VocabGrad& g, long row, long col, int first, int last, float (&v)[4]) {
  const long at = row * g.cols + col;
  if constexpr (sizeof(T) == 2) {
    if (__builtin_expect(first < last, 0)) {   // (unlikely: among the others' code it makes dw of 16 rows 6 % slower)
      if (last - first > FEW) {
        const float* const left = g.left + static_cast<long>(line_of(first)) * g.cols + col;
        const int runs = (last - first + (1 << g.run_bits) - 1) >> g.run_bits;
#pragma unroll 1
        for (int k = 0; k < runs; k += 4) {
          float4 q[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) q[u] = *reinterpret_cast<const float4*>(left + static_cast<long>(k + u < runs ? k + u : k) * g.cols);
#pragma unroll
          for (int u = 0; u < 4; ++u)
            if (k + u < runs) v[0] += q[u].x, v[1] += q[u].y, v[2] += q[u].z, v[3] += q[u].w;
        }
      } else {
#pragma unroll 1
        for (int k = first; k < last; ++k) {
          const long i = g.order[k];
          add_left(g.term[i], g.row_factor[i], *reinterpret_cast<const uint2*>(static_cast<const T*>(g.x) + i * g.cols + col), v);
        }
      }
    }
  }
  if (g.factor != nullptr) {
    const float f = g.factor[row];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= f;
    // a row that takes no part: w may hold infinities or NaN, which zeros of e do not take out of a product
    if (f == 0.f && (g.targets[row] < 0 || g.targets[row] >= g.b_inner)) v[0] = v[1] = v[2] = v[3] = 0.f;
    if constexpr (sizeof(T) == 2) {
      const float r = g.rest[row];
      if (r != 0.f) {
        const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const T*>(g.b) + static_cast<long>(g.targets[row]) * g.cols + col);
        v[0] = fmaf(r, __uint_as_float(w.x << 16), v[0]);
        v[1] = fmaf(r, __uint_as_float(w.x & 0xffff0000u), v[1]);
        v[2] = fmaf(r, __uint_as_float(w.y << 16), v[2]);
        v[3] = fmaf(r, __uint_as_float(w.y & 0xffff0000u), v[3]);
      }
    }
  }
  if (g.add) {
    const float4 o = *reinterpret_cast<const float4*>(g.acc + at);
    v[0] += o.x, v[1] += o.y, v[2] += o.z, v[3] += o.w;
  }
  if (!g.last) {
    *reinterpret_cast<float4*>(g.acc + at) = make_float4(v[0], v[1], v[2], v[3]);
  } else if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint2*>(static_cast<T*>(g.out) + at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  } else {
    *reinterpret_cast<float4*>(static_cast<T*>(g.out) + at) = make_float4(v[0], v[1], v[2], v[3]);
  }
}

// rows x cols results, inner indices split over g.splits workgroups, whose sums then go to g.part.  dx of 4096 x 4096 over 131072 bf16
// 3.3 to 3.7 ms, 1.2 to 1.3 PFLOP/s (78 % busy at 1.5 GHz; a library's product of that order 3.1); dw, whose operands both have to be
// transposed on their way from LDS, 3.9 to 4.2 (3.6 to 3.9).
template <typename T, typename P>
__global__ __launch_bounds__(P::THREADS, 2) void vocab_grad_kernel(VocabGrad g) {
  __shared__ __attribute__((aligned(16))) char lds[P::LDS];
  __shared__ int lists[P::BM + 1];
  const int id = blockIdx.x / g.splits, split = blockIdx.x - id * g.splits;
  int mt, nt;
  tile_of(id, g.row_tiles, g.col_tiles, mt, nt);
  const long m0 = static_cast<long>(mt) * P::BM, n0 = static_cast<long>(nt) * P::BN;
  const long k0 = split * g.per_split, k1 = k0 + g.per_split < g.inner ? k0 + g.per_split : g.inner;
  if (g.start != nullptr)   // (seen by all after the product's barriers)
    for (int r = threadIdx.x; r <= P::BM; r += P::THREADS) lists[r] = g.start[m0 + r < g.rows ? m0 + r : g.rows];
  f32x16_t acc[P::MB][P::NB];
  P::zero(acc);
  {
    typename P::A pa;
    typename P::B pb;
    pa.begin(static_cast<const T*>(g.a), g.a_ld, m0, g.a_free, k0, g.inner);
    pb.begin(static_cast<const T*>(g.b), g.cols, n0, g.cols, k0, g.b_inner);
    P::run(pa, pb, k0, k1, lds, acc);
  }
  // through LDS, as many of each wave's rows at a time as fit, so that whole lines are written: a lane's results are 4 columns here
  // and there
  constexpr int PASSES = P::BM * P::BN * 4 <= P::LDS ? 1 : 2;
  constexpr int CHUNKS = P::BN / 4, PART = P::BM / P::WM / PASSES, ROWS = P::BM / PASSES, MB = P::MB / PASSES;
  static_assert(ROWS * P::BN * 4 <= P::LDS && MB > 0, "a pass's rows in fp32");
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int chunk = threadIdx.x % CHUNKS;
  const long col = n0 + chunk * 4;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    if (p > 0) __syncthreads();
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < P::NB; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int r = wave / P::WN * PART + 32 * i + (lane & 31), c = (wave % P::WN * (P::BN / P::WN) + 32 * j + 8 * q) / 4 + h;
          const f32x16_t& v = acc[p * MB + i][j];
          *reinterpret_cast<float4*>(lds + r * (CHUNKS * 16) + ((c ^ (lane & 31 & (CHUNKS - 1))) << 4)) =
              make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        }
    __syncthreads();
    for (int r = threadIdx.x / CHUNKS; r < ROWS; r += P::THREADS / CHUNKS) {
      const long row = m0 + r / PART * (PASSES * PART) + p * PART + r % PART;
      if (row >= g.rows || col >= g.cols) continue;
      const float4 x = *reinterpret_cast<const float4*>(lds + r * (CHUNKS * 16) + ((chunk ^ (r & 31 & (CHUNKS - 1))) << 4));
      float v[4] = {x.x, x.y, x.z, x.w};
      if (g.splits > 1) *reinterpret_cast<float4*>(g.part + (split * g.rows + row) * g.cols + col) = x;
      else finish<T>(g, row, col, g.start != nullptr ? lists[row - m0] : 0, g.start != nullptr ? lists[row - m0 + 1] : 0, v);
    }
  }
}

// What rounding left of the targets' terms of dw for columns of more than FEW target rows: a wave a run of 2^run_bits of a
// column's rows and 256 channels, its rows on their way four at a time.  So the time goes by all rows and not by how many
// have one target: 2048 x 1024 over 32768 with one for all took 1.53 ms when dw's epilogue went through whole lists.
__global__ __launch_bounds__(256) void vocab_left_kernel(VocabArgs a, int run_bits) {
  const int lane = threadIdx.x & 63, parts = (a.width + 255) / 256;
  const long id = static_cast<long>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int line = static_cast<int>(id / parts), col = static_cast<int>(id % parts) * 256 + lane * 4;
  if (line * FEW >= a.start[a.vocab]) return;
  // whose line it is, and of which run
  const int target = a.targets[a.row0 + a.order[line * FEW]], first = a.start[target], last = a.start[target + 1];
  const int from = first + ((line - line_of(first)) << run_bits), to = from + (1 << run_bits) < last ? from + (1 << run_bits) : last;
  if (last - first <= FEW || from >= last || col >= a.width) return;
  float v[4] = {};
  for (int k = from; k < to; k += 4) {
    int row[4];
    float f[4], t[4];
    uint2 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) row[u] = a.order[k + u < to ? k + u : k];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f[u] = a.factor[row[u]];
      t[u] = a.term[row[u]];
      x[u] = *reinterpret_cast<const uint2*>(static_cast<const bf16_t*>(a.x) + (a.row0 + row[u]) * a.width + col);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (k + u < to) add_left(t[u], f[u], x[u], v);
  }
  *reinterpret_cast<float4*>(a.left + static_cast<long>(line) * a.width + col) = make_float4(v[0], v[1], v[2], v[3]);
}

// Adds the splits' sums, 4 columns a thread.
template <typename T>
__global__ __launch_bounds__(256) void vocab_add_kernel(VocabGrad g) {
  const long all = g.rows * g.cols;
  for (long at = (static_cast<long>(blockIdx.x) * 256 + threadIdx.x) * 4; at < all; at += static_cast<long>(gridDim.x) * 1024) {
    float v[4] = {};
    for (int s = 0; s < g.splits; ++s) {
      const float4 o = *reinterpret_cast<const float4*>(g.part + s * all + at);
      v[0] += o.x, v[1] += o.y, v[2] += o.z, v[3] += o.w;
    }
    const long row = at / g.cols;
    finish<T>(g, row, at - row * g.cols, g.start != nullptr ? g.start[row] : 0, g.start != nullptr ? g.start[row + 1] : 0, v);
  }
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

// Tiles of a product.  Large ones feed the matrix unit best, a workgroup a CU; smaller ones, two and four a CU, leave less of the
// chip and of their own edges idle where there are few; and few rows are bound by reading w, which needs many workgroups.
template <typename T, bool A, bool B> using Large = Product<T, 256, 256, 2, 4, A, B>;
template <typename T, bool A, bool B> using Small = Product<T, 128, 128, 2, 2, A, B>;
template <typename T, bool A, bool B> using Tiny = Product<T, 64, 64, 2, 2, A, B>;
template <typename T> using Few = Product<T, 32, 64, 1, 2, true, true>;

long up(long x, long y) { return (x + y - 1) / y; }

// How long rows x cols results over `steps` tiles of the inner index take by one kind of tile, in microseconds: the tiles of
// the fullest CU, as many at a time as it holds, each 3 steps longer than its inner index.  A step of a tile measured, with a CU
// full of them: 256 x 256 1.6 (bf16) and 6.9 (fp32), 128 x 128 0.5 and 1.7, 64 x 64 0.25 and 0.43; none is shorter than loads take
// to arrive.  Split sums are written and read again, at 4 TB/s.
double cost(int tile, int dtype, long rows, long cols, long steps, long splits) {
  const double step = dtype == 1 ? (tile == 256 ? 1.6 : tile == 128 ? 0.5 : 0.25) : (tile == 256 ? 6.9 : tile == 128 ? 1.7 : 0.43);
  const long held = tile == 256 ? 1 : tile == 128 ? 2 : 4;
  const long a_cu = up(up(rows, tile) * up(cols, tile) * splits, 256), rest = a_cu % held;
  const double latency = 0.9, full = held * step > latency ? held * step : latency;
  const double last = rest == 0 ? 0. : rest * step > latency ? rest * step : latency;
  const double sums = splits > 1 ? 4. + static_cast<double>(rows) * cols * 8 * splits / 4e6 : 0.;
  return (a_cu / held * full + last) * (up(steps, splits) + 3) + sums;
}

template <typename T>
void scores(const VocabArgs& a, bool keep, hipStream_t s) {
  const unsigned n = static_cast<unsigned>(a.row_tiles * a.col_tiles);
  auto launch = [&](auto p) {
    using P = decltype(p);
    if (keep) vocab_scores_kernel<T, P, true><<<n, P::THREADS, 0, s>>>(a);
    else vocab_scores_kernel<T, P, false><<<n, P::THREADS, 0, s>>>(a);
  };
  if (a.row_tile == 32) launch(Few<T>{});
  else if (a.row_tile == 64) launch(Tiny<T, true, true>{});
  else if (a.row_tile == 128) launch(Small<T, true, true>{});
  else launch(Large<T, true, true>{});
}

template <typename T>
void add(const VocabGrad& g, hipStream_t s) {
  const long n = up(g.rows * g.cols, 1024);
  vocab_add_kernel<T><<<static_cast<unsigned>(n < 4096 ? n : 4096), 256, 0, s>>>(g);
}

template <typename T, bool A, bool B>
void grad(VocabGrad& g, hipStream_t s) {
  auto launch = [&](auto p) {
    using P = decltype(p);
    g.row_tiles = static_cast<int>(up(g.rows, P::BM));
    g.col_tiles = static_cast<int>(up(g.cols, P::BN));
    vocab_grad_kernel<T, P><<<static_cast<unsigned>(g.row_tiles * g.col_tiles * g.splits), P::THREADS, 0, s>>>(g);
  };
  if (g.tile == 64) launch(Tiny<T, A, B>{});
  else if (g.tile == 128) launch(Small<T, A, B>{});
  else launch(Large<T, A, B>{});
  if (g.splits > 1) add<T>(g, s);
}

// Tiles and splits of a gradient's product: the cheapest.
void split(VocabGrad& g, int dtype, long inner_tile) {
  const long steps = up(g.inner, inner_tile);
  double best = 0.;
  long splits = 1;
  for (int tile : {256, 128, 64})
    for (long n = 1; n <= 64 && (n == 1 || n <= steps / 4); n = n < 4 ? n + 1 : n + n / 4) {
      const double c = cost(tile, dtype, g.rows, g.cols, steps, n);
      if (best == 0. || c < best) best = c, splits = n, g.tile = tile;
    }
  g.per_split = up(steps, splits) * inner_tile;
  g.splits = static_cast<int>(up(g.inner, g.per_split));
}

template <typename T>
void run(const VocabArgs& all, const VocabPlan& p, bool gradients, hipStream_t s) {
  VocabArgs a = all;
  if (a.rows == 0) {   // nothing but the zeros of dw
    VocabGrad none{};
    none.rows = a.vocab, none.cols = a.width, none.out = a.dw, none.last = 1;
    if (gradients) add<T>(none, s);
    return;
  }
  if (gradients && a.weight == nullptr) vocab_mean_kernel<<<1, 1024, 0, s>>>(a);
  a.row_tile = p.row_tile;
  a.col_tile = p.col_tile;
  a.col_tiles = static_cast<int>(up(a.vocab, a.col_tile));
  for (a.row0 = 0; a.row0 < a.rows; a.row0 += p.piece) {
    a.piece = a.rows - a.row0 < p.piece ? a.rows - a.row0 : p.piece;
    a.row_tiles = static_cast<int>(up(a.piece, a.row_tile));
    const int lists = p.lists ? static_cast<int>(up(a.vocab, 256)) : 0;
    vocab_target_kernel<T><<<static_cast<unsigned>(lists + up(a.piece, 4)), 256, 0, s>>>(a, lists);
    scores<T>(a, gradients, s);
    const unsigned n = static_cast<unsigned>(a.piece);
    if (!gradients) {
      vocab_join_kernel<T, false><<<n, 256, 0, s>>>(a);
      continue;
    }
    vocab_join_kernel<T, true><<<n, 256, 0, s>>>(a);
    VocabGrad x = p.dx, w = p.dw;
    x.a = a.e, x.b = a.w, x.a_ld = a.vocab_padded, x.a_free = a.piece, x.b_inner = a.vocab, x.rows = a.piece, x.cols = a.width, x.inner = a.vocab_padded;
    x.out = static_cast<T*>(a.dx) + a.row0 * a.width, x.factor = a.factor, x.rest = a.rest, x.targets = a.targets + a.row0, x.part = a.part, x.last = 1;
    grad<T, true, false>(x, s);
    w.a = a.e, w.b = a.scaled, w.a_ld = w.a_free = a.vocab_padded, w.b_inner = a.piece, w.rows = a.vocab, w.cols = a.width, w.inner = a.piece;
    w.out = a.dw, w.part = a.part, w.acc = a.acc, w.add = a.row0 > 0, w.last = a.row0 + a.piece == a.rows;
    if (p.lists) {
      const long waves = up(a.piece, FEW) * up(a.width, 256);
      vocab_left_kernel<<<static_cast<unsigned>(up(waves, 4)), 256, 0, s>>>(a, p.run_bits);
      w.start = a.start, w.order = a.order, w.term = a.term, w.row_factor = a.factor, w.left = a.left, w.run_bits = p.run_bits;
      w.x = static_cast<const T*>(a.x) + a.row0 * a.width;
    }
    if (w.per_split >= w.inner) w.splits = 1;   // a last, smaller piece
    else w.splits = static_cast<int>(up(w.inner, w.per_split));
    grad<T, false, false>(w, s);
  }
}

}  // namespace

VocabPlan vocab_plan(const VocabArgs& a, int dtype, bool gradients, long piece_rows) {
  const size_t esz = dtype == 1 ? 2 : 4;
  const long inner_tile = 128 / static_cast<long>(esz);
  VocabPlan p{};
  // 2^30 bytes of e at a time, in whole tiles; without it 2^30 of sums
  long most = gradients ? (1L << 30) / (a.vocab_padded * static_cast<long>(esz)) : (1L << 30) / (8 * up(a.vocab, 64));
  most = most < 256 ? 256 : most / 256 * 256;
  if (most > 1L << 23) most = 1L << 23;   // (a grid has fewer than 2^32 lanes, and some have a workgroup a row)
  if (piece_rows > 0 && piece_rows < most) most = piece_rows;
  const long rows = a.rows > 0 ? a.rows : 1;
  p.piece = rows < most ? rows : most;
  if (piece_rows <= 0) {   // pieces of one size
    const long even = up(up(rows, up(rows, p.piece)), 256) * 256;
    if (even < p.piece) p.piece = even;
  }
  const long steps = up(a.width, inner_tile);
  p.row_tile = p.col_tile = 256;
  for (int tile : {128, 64})
    if (cost(tile, dtype, p.piece, a.vocab, steps, 1) < cost(p.row_tile, dtype, p.piece, a.vocab, steps, 1)) p.row_tile = p.col_tile = tile;
  if (p.piece <= 32) p.row_tile = 32, p.col_tile = 64;
  const long tiles = up(a.vocab, p.col_tile);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  p.ref = take(static_cast<size_t>(a.rows) * 4);
  p.sums = take(static_cast<size_t>(p.piece) * tiles * 4);
  p.shift = take(static_cast<size_t>(p.piece) * tiles * 4);
  p.slow = take(static_cast<size_t>(up(p.piece, p.row_tile)) * tiles * 4);
  if (gradients) {
    p.mean = take(4);
    p.factor = take(static_cast<size_t>(p.piece) * 4);
    p.rest = take(static_cast<size_t>(p.piece) * 4);
    p.term = take(static_cast<size_t>(p.piece) * 4);
    // fp32 has no rounding to take back; and where many rows share few columns, and few workgroups list them, that would take as
    // long as the products
    p.lists = esz == 2 && p.piece <= 65536 && p.piece <= 16L * a.vocab;
    // runs of 16 rows, and of more where a column of all rows would have over 256; their sums where the tiles' have been, if they fit
    for (p.run_bits = 4; p.piece > 256L << p.run_bits; ++p.run_bits) {}
    const size_t left = p.lists ? static_cast<size_t>(up(p.piece, FEW)) * a.width * 4 : 0;
    p.left = left <= p.mean - p.sums ? p.sums : take(left);
    p.start = take(p.lists ? (static_cast<size_t>(a.vocab) + 1) * 4 : 0);
    p.order = take(p.lists ? static_cast<size_t>(p.piece) * 4 : 0);
    p.scaled = take(static_cast<size_t>(p.piece) * a.width * esz);
    p.e = take(static_cast<size_t>(p.piece) * a.vocab_padded * esz);
    p.dx.rows = p.piece, p.dx.cols = a.width, p.dx.inner = a.vocab_padded;
    p.dw.rows = a.vocab, p.dw.cols = a.width, p.dw.inner = p.piece;
    size_t part = 0;
    for (VocabGrad* g : {&p.dx, &p.dw}) {
      split(*g, dtype, inner_tile);
      const size_t bytes = g->splits > 1 ? static_cast<size_t>(g->splits) * g->rows * g->cols * 4 : 0;
      if (bytes > part) part = bytes;
    }
    p.part = take(part);
    // sums over pieces; fp32 has them in dw itself
    p.acc = take(esz == 2 && p.piece < a.rows ? static_cast<size_t>(a.vocab) * a.width * 4 : 0);
  }
  p.bytes = at;
  return p;
}

void vocab_run(VocabArgs a, const VocabPlan& p, int dtype, bool gradients, void* workspace, hipStream_t s) {
  char* const ws = static_cast<char*>(workspace);
  a.ref = reinterpret_cast<float*>(ws + p.ref);
  a.sums = reinterpret_cast<float*>(ws + p.sums);
  a.shift = reinterpret_cast<float*>(ws + p.shift);
  a.slow = reinterpret_cast<int*>(ws + p.slow);
  if (gradients) {
    a.mean = reinterpret_cast<float*>(ws + p.mean);
    a.factor = reinterpret_cast<float*>(ws + p.factor);
    a.rest = reinterpret_cast<float*>(ws + p.rest);
    a.term = reinterpret_cast<float*>(ws + p.term);
    a.start = reinterpret_cast<int*>(ws + p.start);
    a.order = reinterpret_cast<int*>(ws + p.order);
    a.left = reinterpret_cast<float*>(ws + p.left);
    a.scaled = ws + p.scaled;
    a.e = ws + p.e;
    a.part = reinterpret_cast<float*>(ws + p.part);
    a.acc = dtype == 1 ? reinterpret_cast<float*>(ws + p.acc) : static_cast<float*>(a.dw);
  }
  if (dtype == 1) run<bf16_t>(a, p, gradients, s);
  else run<float>(a, p, gradients, s);
}

}  // namespace petra
