// Attention over packed sequences of tokens, with grouped heads, a causal mask and a learned relative position bias by buckets,
// and its backward pass.  For head a of a sequence with Lq queries and Lk keys, r = j - (i + Lk - Lq) the position of key j
// relative to query i (the queries are the sequence's last positions):
//
//   s_ij = scale <q_i, k_j> + bias[a][bucket(r)]     (causal: only r <= 0)
//   o_i  = sum_j P_ij v_j,   P_ij = exp(s_ij - lse_i),   lse_i = log sum_j exp s_ij
//   dP_ij = <do_i, v_j>,  dS_ij = P_ij (dP_ij - <do_i, o_i>),  dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,
//   dv_j = sum_i P_ij do_i,  dbias[a][b] = sum over the pairs of bucket b of dS_ij
//
// Scores, softmax statistics and sums are fp32; for bf16 tensors P and dS are rounded to bf16 once, as operands of the matrix
// instructions (their sums of products are fp32).  Exponentials are taken to base 2 of scores scaled by log2(e).
//
// Layout shared by all kernels here: products are formed so that the 16 columns of an accumulator block are the rows a wavefront
// owns (queries, or keys in k_attend_dkv) and its 16 rows are those of the tile that lies in LDS: lane l holds, for its own row
// l % 16, the tile rows 4 (l / 16) + 0..3.  A softmax row is then in-lane work plus two lane exchanges, rescaling is one factor
// a lane, and two such blocks are, without any exchange, the operand of the next product over 32 tile rows in the order
// {4 g + 0..3, 16 + 4 g + 0..3}, g = l / 16; the other operand is read from LDS in the same order (transposing reads).
#pragma once
#include <type_traits>

#include "dchag_dev.h"

namespace dchag {

constexpr int kMaxBorders = 63;
constexpr int kMaxDistance = 1024;     // of the last border: bounds the tables in LDS
constexpr int kTileKeys = 64;          // rows of a tile in LDS
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.4028234663852886e38f;
constexpr float kNegInf = -__builtin_inff();
// A bias entry at or below this masks its pairs, like -inf (a mask written as a type's lowest value would not survive the scaling).
constexpr float kMaskBias = -1e30f;
// The running maximum is moved only when a tile's exceeds it by this much (base 2): what is added up stays below 2^8 of it.
constexpr float kMaxSlack = 8.f;

struct AttendArgs {
  const int *q_starts, *k_starts, *k_used;
  const int* firsts;                   // of each sequence its first item, [sequences + 1] (k_attend_plan), or NULL: found in the kernel
  int sequences, rows_q, rows_k, heads, kv_heads, d, causal;
  long ld_q, ld_k, ld_v, ld_o, ld_do, ld_dq, ld_dk, ld_dv;   // elements from one row to the next
  float scale, c;                      // c = scale * log2(e)
  const void* bias;                    // [heads][buckets] or NULL
  int n_borders, last, side, buckets;  // last: the last border; side: buckets of one side
  int borders[kMaxBorders];
};

typedef __attribute__((ext_vector_type(8))) float f32x8;
template <typename T> struct Frag;
template <> struct Frag<bf16> { typedef bf16x8 type; };
template <> struct Frag<float> { typedef f32x8 type; };

// c += a x b over 32 contraction elements, eight of them a lane (8 g + 0..7 of it): one bf16 instruction, or eight fp32 ones,
// each of which takes the same element of the four lanes g.
__device__ __forceinline__ f32x4 mma(f32x4 c, bf16x8 a, bf16x8 b) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(f32x4 c, f32x8 a, f32x8 b) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

static __device__ __align__(16) const unsigned char kZeros[16] = {0};

// A tile of rows of DP elements in LDS, 16-byte chunks XOR-swizzled by the row.  A 16-byte read serves 16 lanes at a time, eight of one chunk's rows
// 0..3 and 12..15 and eight of the next chunk's rows 4..11 (and so on): the rows' low bits move the chunk by two, so these lie in different banks,
// and so do the eight half-rows of 32 bytes that half a wavefront reads transposed.  (Rows 8 apart moved by one as well: a third of the LDS
// cycles were conflicts, none is now; key gradients of packed causal rows 747 -> 697 us.)
template <typename T, int DP>
struct Tile {
  static constexpr int kPitch = DP * (int)sizeof(T), kChunks = kPitch / 16, kElems = 16 / (int)sizeof(T);
  static constexpr int kBytes = kTileKeys * kPitch;
  static __device__ __forceinline__ int swz(int row) {
    constexpr int per = kChunks >= 16 ? 1 : 16 / kChunks, wide = kChunks >= 16 ? 16 : kChunks;
    return ((row / per) & (wide / 2 - 1)) << 1;
  }
  // Eight elements 32 ks + 8 g .. of row 16 blk + l % 16.
  static __device__ __forceinline__ typename Frag<T>::type row_frag(const unsigned char* t, int blk, int ks, int lane) {
    const int l16 = lane & 15, g = lane >> 4;
    const unsigned char* p = t + (blk * 16 + l16) * kPitch;
    if constexpr (sizeof(T) == 2) {
      return *reinterpret_cast<const bf16x8*>(p + ((ks * 4 + g) ^ swz(l16)) * 16);
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(p + ((ks * 8 + 2 * g) ^ swz(l16)) * 16);
      const f32x4 b = *reinterpret_cast<const f32x4*>(p + ((ks * 8 + 2 * g + 1) ^ swz(l16)) * 16);
      return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
  // Column 16 blk + l % 16 of the rows 32 s + {4 g + 0..3, 16 + 4 g + 0..3}.
  static __device__ __forceinline__ typename Frag<T>::type col_frag(const unsigned char* t, int blk, int s, int lane) {
    const int l16 = lane & 15, g = lane >> 4;
    if constexpr (sizeof(T) == 2) {
      typedef __attribute__((ext_vector_type(4))) short s16x4;
      typedef __attribute__((address_space(3))) s16x4* tptr;
      const int row = 4 * g + (l16 >> 2);
      const unsigned char* p = t + row * kPitch + (((blk * 2 + ((l16 & 3) >> 1)) ^ swz(row)) * 16) + (l16 & 1) * 8 + s * 32 * kPitch;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tptr)p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tptr)(p + 16 * kPitch));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      f32x8 r;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int row = 4 * g + (j & 3) + (j >> 2) * 16;
        r[j] = *reinterpret_cast<const float*>(t + (row + s * 32) * kPitch + (((blk * 4 + (l16 >> 2)) ^ swz(row)) * 16) + (l16 & 3) * 4);
      }
      return r;
    }
  }
  // Elements col .. col + 3 of a row; col a multiple of 4.
  static __device__ __forceinline__ f32x4 four(const unsigned char* t, int row, int col) {
    const unsigned char* p = t + row * kPitch + ((col / kElems) ^ swz(row)) * 16 + (col % kElems) * (int)sizeof(T);
    if constexpr (sizeof(T) == 2) {
      const bf16x4 v = *reinterpret_cast<const bf16x4*>(p);
      return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
    } else {
      return *reinterpret_cast<const f32x4*>(p);
    }
  }
  // Fills ROWS rows of a tile from rows base + row * ld (direct-to-LDS loads; NT threads take part, tid among them); rows from
  // `rows` on and columns from d on come from zeros, so nothing outside the sequence and the head is read.
  template <int ROWS, int NT>
  static __device__ __forceinline__ void stage(const T* base, long ld, int rows, int d, unsigned char* lds, int tid) {
    constexpr int kLoads = ROWS * kChunks / NT;
    static_assert(kLoads * NT == ROWS * kChunks, "rows do not split over the threads");
    if (rows >= ROWS && d == DP) {
      const unsigned lds0 = __builtin_amdgcn_readfirstlane((unsigned)(size_t)(lptr_t)(lds + (tid & ~63) * 16));
      const uint64_t at = reinterpret_cast<uint64_t>(base);                   // the same in every lane, which the compiler does not always see
      const unsigned low = __builtin_amdgcn_readfirstlane((unsigned)at), high = __builtin_amdgcn_readfirstlane((unsigned)(at >> 32));
      const void* first = reinterpret_cast<const void*>((uint64_t)high << 32 | low);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int idx = i * NT + tid, row = idx / kChunks, chunk = (idx % kChunks) ^ swz(row);
        load16_to_lds_at(first, (unsigned)(row * (int)ld * (int)sizeof(T) + chunk * 16), __builtin_amdgcn_readfirstlane(lds0 + i * NT * 16));
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int idx = i * NT + tid, row = idx / kChunks, chunk = (idx % kChunks) ^ swz(row);
        const bool in = row < rows && chunk * kElems < d;
        const void* src = in ? static_cast<const void*>(base + row * ld + chunk * kElems) : static_cast<const void*>(kZeros);
        load16_to_lds(src, lds + (i * NT + (tid & ~63)) * 16);
      }
    }
  }
};

// Eight elements 32 ks + 8 g .. of a row in global memory; zeros past the head's d.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type load_frag(const T* row, bool in, int ks, int g, int d) {
  const int e = ks * 32 + g * 8;
  typename Frag<T>::type r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r[j] = (T)0.f;
  if (in && e < d) {
    if constexpr (sizeof(T) == 2) {
      r = *reinterpret_cast<const bf16x8*>(row + e);
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(row + e), b = *reinterpret_cast<const f32x4*>(row + e + 4);
      r = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  }
  return r;
}
// Four adjacent elements.
__device__ __forceinline__ void store4(float* p, f32x4 v) { *reinterpret_cast<f32x4*>(p) = v; }
__device__ __forceinline__ void store4(bf16* p, f32x4 v) { *reinterpret_cast<bf16x4*>(p) = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]}; }

// The values of lanes l and l ^ 32 (l ^ 16), the lower one first.
struct LanePair {
  float low, high;
};
template <class Two>
__device__ __forceinline__ LanePair lane_pair(Two p) {
  const unsigned low = p[0], high = p[1];                                    // a bit cast of a vector's element takes its first one
  return {__builtin_bit_cast(float, low), __builtin_bit_cast(float, high)};
}
__device__ __forceinline__ LanePair pair32(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  return lane_pair(__builtin_amdgcn_permlane32_swap(u, u, false, false));
}
__device__ __forceinline__ LanePair pair16(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  return lane_pair(__builtin_amdgcn_permlane16_swap(u, u, false, false));
}
// The larger of two numbers, NaN if one is (fmaxf would first quiet every operand, an instruction each).
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// Maximum and sum over the four lanes of a row (lane, lane ^ 16, lane ^ 32, lane ^ 48); every one of them gets it.
__device__ __forceinline__ float row_max(float v) {
  LanePair p = pair32(v);
  p = pair16(larger(p.low, p.high));
  return larger(p.low, p.high);
}
__device__ __forceinline__ float row_sum(float v) {
  LanePair p = pair32(v);
  p = pair16(p.low + p.high);
  return p.low + p.high;
}

// One sequence: rows q0 .. q0 + nq of the queries, k0 .. k0 + nk of the keys, and a tile of it.  The starts are data of the
// device: whatever they hold, rows stay inside the tensors.
struct Span {
  int q0, nq, k0, nk, tile, tiles;
};
__device__ __forceinline__ void read_span(const AttendArgs& a, int s, int& q0, int& nq, int& k0, int& nk) {
  q0 = min(max(a.q_starts[s], 0), a.rows_q);
  nq = min(max(a.q_starts[s + 1], q0), a.rows_q) - q0;
  k0 = min(max(a.k_starts[s], 0), a.rows_k);
  nk = min(max(a.k_starts[s + 1], k0), a.rows_k) - k0;
  if (a.k_used) nk = min(max(a.k_used[s], 0), nk);
}
// The sequence that item `at` belongs to: the last one whose first item is not behind it.  64 places are looked at in one turn.
__device__ __forceinline__ int find_sequence(const int* firsts, int sequences, int at) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = sequences;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, i = lo + (lane + 1) * step;
    const bool behind = i < hi && firsts[i] <= at;
    lo += __popcll(__ballot(behind)) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}
// The sequence and tile that item idx is, the items of a sequence being count(nq, nk).  False if there are not as many items.  Every wavefront finds
// it for itself: up to kPlanFrom sequences by going through them 64 at a time, one a lane, beyond by a search in what k_attend_plan
// has left (1024 sequences of 64 rows, 16 heads of 64, training step, us: 1262 / 701; 4096 single tokens against 128 keys: 4070 / 528).
constexpr int kPlanFrom = 128;
template <class Count>
__device__ __forceinline__ bool find_span(const AttendArgs& a, int idx, Count count, Span& sp) {
  const int lane = threadIdx.x & 63;
  if (a.firsts) {
    if (idx >= a.firsts[a.sequences]) return false;
    const int s = find_sequence(a.firsts, a.sequences, idx);
    read_span(a, s, sp.q0, sp.nq, sp.k0, sp.nk);
    sp.tiles = count(sp.nq, sp.nk);
    sp.tile = idx - a.firsts[s];
    return sp.tile >= 0 && sp.tile < sp.tiles;                               // false only where overlapping sequences have more items than 32 bits count
  }
  for (int s0 = 0; s0 < a.sequences; s0 += 64) {
    int q0 = 0, nq = 0, k0 = 0, nk = 0, n = 0;
    if (s0 + lane < a.sequences) {
      read_span(a, s0 + lane, q0, nq, k0, nk);
      n = count(nq, nk);
    }
    int upto = n;
#pragma unroll
    for (int w = 1; w < 64; w *= 2) {
      const int v = __shfl_up(upto, w);
      if (lane >= w) upto += v;
    }
    const int total = __builtin_amdgcn_readlane(upto, 63);
    if (idx < total) {
      const int l = __builtin_ctzll(__ballot(idx < upto));
      sp.q0 = __builtin_amdgcn_readlane(q0, l);
      sp.nq = __builtin_amdgcn_readlane(nq, l);
      sp.k0 = __builtin_amdgcn_readlane(k0, l);
      sp.nk = __builtin_amdgcn_readlane(nk, l);
      sp.tiles = __builtin_amdgcn_readlane(n, l);
      sp.tile = idx - (__builtin_amdgcn_readlane(upto, l) - sp.tiles);
      return true;
    }
    idx -= total;
  }
  return false;
}

// Which heads and which item a workgroup takes: key heads fastest, so that one XCD's workgroups (id % 8) share few of them.
struct HeadItem {
  int h, kvh, idx;
};
__device__ __forceinline__ HeadItem head_item(const AttendArgs& a, int id) {
  const int group = a.heads / a.kv_heads, kvh = id % a.kv_heads, rest = id / a.kv_heads;
  return {kvh * group + rest % group, kvh, rest / group};
}

// ---- the bias -------------------------------------------------------------------------------------------------------------
// A pair whose distance is at least the last border has the last bucket of its side: a tile of such pairs only adds a constant.
// The others look their value up by r in a table of the head in LDS that reaches kPad beyond the last border on both sides, as far
// as a tile with one nearer pair can.
constexpr int kPad = 128;
__host__ __device__ inline int bias_table_size(int last) { return 2 * (last + kPad) + 1; }
__device__ __forceinline__ int bucket_of(const AttendArgs& a, int r) {
  const int dist = r < 0 ? -r : r;
  int n = 0;
  for (int b = 0; b < a.n_borders; ++b) n += dist >= a.borders[b];
  return n + (r > 0 && !a.causal ? a.side : 0);
}
// An entry as it is added to scores to base 2.
template <typename T>
__device__ __forceinline__ float bias_value(const AttendArgs& a, int h, int bucket) {
  const float v = to_f32(static_cast<const T*>(a.bias)[(size_t)h * a.buckets + bucket]);
  return v <= kMaskBias ? kNegInf : v * kLog2e;
}
template <typename T, int NT>
__device__ __forceinline__ void fill_bias_table(const AttendArgs& a, int h, float* table, int tid) {
  const int n = bias_table_size(a.last), mid = a.last + kPad;
  for (int i = tid; i < n; i += NT) table[i] = bias_value<T>(a, h, bucket_of(a, i - mid));
}

// acc += p v over the 32 rows row0 .. of a tile, as mma(acc, column fragments, p) does but pair by pair, leaving out the pairs with p = 0:
// what a masked pair's v holds then does not matter, not even a NaN.  For tiles with masked pairs and with values that are not finite.
template <typename T, int DP, int NB>
__device__ __forceinline__ void accumulate_pairs(f32x4 (&acc)[DP / 16][NB], const typename Frag<T>::type (&p)[NB], const unsigned char* t, int row0, int lane) {
  const int l16 = lane & 15, g = lane >> 4;
#pragma unroll 1
  for (int j = 0; j < 32; ++j) {
    float w[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float own = 0.f;
#pragma unroll
      for (int m = 0; m < 8; ++m)
        if (m == (j >> 4) * 4 + (j & 3)) own = to_f32(p[nb][m]);
      w[nb] = __shfl(own, l16 + 16 * ((j >> 2) & 3));
    }
#pragma unroll
    for (int b = 0; b < DP / 16; ++b) {
      const f32x4 v = Tile<T, DP>::four(t, row0 + j, b * 16 + 4 * g);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (w[nb] != 0.f) acc[b][nb][r] += w[nb] * v[r];
      __builtin_amdgcn_sched_barrier(0);                                     // four values at a time: the registers are the accumulators'
    }
  }
}
// Whether a tile's rows row0 .. row0 + ROWS hold a value that is not finite (the same answer in every lane).
template <typename T, int DP, int ROWS>
__device__ __forceinline__ bool any_not_finite(const unsigned char* t, int row0, int lane) {
  unsigned bad = 0;
  asm volatile("");                                                          // only where it is asked for, not ahead of the branch
#pragma unroll
  for (int i = 0; i < ROWS * Tile<T, DP>::kChunks / 64; ++i) {
    const uint4 w = *reinterpret_cast<const uint4*>(t + row0 * Tile<T, DP>::kPitch + (i * 64 + lane) * 16);
    const unsigned x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 2) bad |= ((x[k] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;   // exponent all ones carries into the sign
      else bad |= ((x[k] & 0x7f800000u) + 0x00800000u) & 0x80000000u;
    }
  }
  return __ballot(bad != 0) != 0;
}

// Scheduling hint for a run of N fragments, READS LDS reads each, every one used by USES products: AHEAD fragments are read before the first
// product and one more behind each fragment's products.  Without it the compiler reads them all first, more than the registers hold.
template <typename T, int N, int READS, int USES, int AHEAD>
__device__ __forceinline__ void interleave_reads() {
  if constexpr (sizeof(T) == 2) {
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * READS, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, USES, 0);
      if (i + AHEAD < N) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
    }
  }
}

// Where there are too few rows for all SIMDs, two wavefronts (SPLIT = 2) share 16 NB rows: each takes half of every tile, and the second leaves
// what it has in LDS for the first.  The place of a wavefront's accumulators there: 16 bytes a lane and block.
template <int DB, int NB>
struct Handover {
  static constexpr int kBytes = (DB * NB * 4 + 2 * NB) * 64 * 4;
  unsigned char* at;
  int lane;
  __device__ __forceinline__ f32x4& block(int b, int nb) const { return *reinterpret_cast<f32x4*>(at + ((b * NB + nb) * 64 + lane) * 16); }
  __device__ __forceinline__ float& number(int i) const { return *reinterpret_cast<float*>(at + DB * NB * 1024 + (i * 64 + lane) * 4); }
};

// Workgroup: NW / SPLIT groups of 16 NB queries of one head, SPLIT wavefronts each; the keys pass by in tiles of 64, two tiles of K and V in
// LDS, the next one on its way (direct-to-LDS) while one is worked on.
template <typename T, int DP, int NB, int NW, int SPLIT, bool BIAS>
__global__ __launch_bounds__(NW * 64, sizeof(T) == 2 ? 2 : 1) void k_attend(AttendArgs a, const T* __restrict__ q, const T* __restrict__ k, const T* __restrict__ v,
                                                       T* __restrict__ out, float* __restrict__ lse) {
  typedef Tile<T, DP> TL;
  typedef typename Frag<T>::type frag;
  constexpr int KS = DP / 32, DB = DP / 16, HALVES = 2 / SPLIT, MB = 2 * HALVES, ROWS = NW / SPLIT * NB * 16, NT = NW * 64;   // MB: of a wavefront's part of a tile
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float* table = reinterpret_cast<float*>(smem + 4 * TL::kBytes);
  const HeadItem hi = head_item(a, blockIdx.x);
  Span sp;
  if (!find_span(a, hi.idx, [](int nq, int) { return (nq + ROWS - 1) / ROWS; }, sp)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  const int i0 = (a.causal ? sp.tiles - 1 - sp.tile : sp.tile) * ROWS;      // causal: the longest rows first
  const int iw = i0 + wave / SPLIT * NB * 16, off = sp.nk - sp.nq, h0 = SPLIT == 2 ? wave & 1 : 0;
  const int kend = a.causal ? min(sp.nk, max(0, min(i0 + ROWS, sp.nq) + off)) : sp.nk;
  const int tiles = (kend + kTileKeys - 1) / kTileKeys;
  const T* kb_ = k + (long)sp.k0 * a.ld_k + hi.kvh * a.d;
  const T* vb_ = v + (long)sp.k0 * a.ld_v + hi.kvh * a.d;
  auto stage = [&](int t) {
    unsigned char* to = smem + (t & 1) * 2 * TL::kBytes;
    TL::template stage<kTileKeys, NT>(kb_ + (long)t * kTileKeys * a.ld_k, a.ld_k, sp.nk - t * kTileKeys, a.d, to, tid);
    TL::template stage<kTileKeys, NT>(vb_ + (long)t * kTileKeys * a.ld_v, a.ld_v, sp.nk - t * kTileKeys, a.d, to + TL::kBytes, tid);
  };
  if (tiles > 0) stage(0);
  float far_left = 0.f, far_right = 0.f;
  if (BIAS) {
    fill_bias_table<T, NT>(a, hi.h, table, tid);
    far_left = bias_value<T>(a, hi.h, a.side - 1);
    far_right = a.causal ? 0.f : bias_value<T>(a, hi.h, 2 * a.side - 1);
  }
  frag qf[NB][KS];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int i = iw + nb * 16 + l16;
    const T* row = q + (long)(sp.q0 + min(i, sp.nq - 1)) * a.ld_q + hi.h * a.d;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[nb][ks] = load_frag<T>(row, i < sp.nq, ks, g, a.d);
  }
  f32x4 acc[DB][NB];
  float m[NB], l[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb] = kLowest;
    l[nb] = 0.f;
#pragma unroll
    for (int b = 0; b < DB; ++b) acc[b][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int lo = iw + off, top = lo + NB * 16 - 1;                          // positions of the wavefront's rows
  // A tile; MASKED: some pair of the workgroup's may not be visible.  Two loops and not one with a branch: with both ways of adding up in
  // one loop the compiler keeps two sets of accumulators.
  auto step = [&](int t, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    wait_vmcnt<0>();
    __syncthreads();
    if (t + 1 < tiles) stage(t + 1);
    const int kb = t * kTileKeys;
    if (iw >= sp.nq || (MASKED && a.causal && kb > top)) return;
    const unsigned char* K = smem + (t & 1) * 2 * TL::kBytes;
    const unsigned char* V = K + TL::kBytes;
    f32x4 s[MB][NB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) s[mb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const frag kf = TL::row_frag(K, h0 * 2 + mb, ks, lane);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[mb][nb] = mma(s[mb][nb], kf, qf[nb][ks]);
      }
    }
    interleave_reads<T, MB * KS, 1, NB, 4>();
    float mul = a.c, add = 0.f;
    if (BIAS) {
      const int rmax = kb + kTileKeys - 1 - lo, rmin = kb - top;
      if (rmax <= -a.last) add = far_left;
      else if (rmin >= a.last) add = far_right;
      else {
        mul = 1.f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const float* tb = table + kb + h0 * 32 + 4 * g - (lo + nb * 16 + l16) + a.last + kPad;
#pragma unroll
          for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[mb][nb][r] = fmaf(s[mb][nb][r], a.c, tb[mb * 16 + r]);
        }
      }
    }
    if (MASKED) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int end = a.causal ? min(sp.nk, lo + nb * 16 + l16 + 1) : sp.nk;   // keys before it are visible
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (kb + h0 * 32 + mb * 16 + 4 * g + r >= end) s[mb][nb][r] = kNegInf;
      }
    }
    float mx[NB];
    bool grow = false;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      mx[nb] = kNegInf;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) mx[nb] = larger(larger(larger(larger(mx[nb], s[mb][nb][0]), s[mb][nb][1]), s[mb][nb][2]), s[mb][nb][3]);
      mx[nb] = fmaf(row_max(mx[nb]), mul, add);
      grow |= mx[nb] > m[nb] + kMaxSlack;
    }
    if (__ballot(grow)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float next = fmaxf(m[nb], mx[nb]), f = __builtin_amdgcn_exp2f(m[nb] - next);
        m[nb] = next;
        l[nb] *= f;
#pragma unroll
        for (int b = 0; b < DB; ++b) acc[b][nb] *= f;
      }
    }
    const bool slow = MASKED && any_not_finite<T, DP, 32 * HALVES>(V, h0 * 32, lane);
    auto exps = [&](int h2) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float sub = add - m[nb];
#pragma unroll
        for (int mb = 2 * h2; mb < 2 * h2 + 2; ++mb) {
#pragma unroll
          for (int r = 0; r < 4; ++r) s[mb][nb][r] = __builtin_amdgcn_exp2f(fmaf(s[mb][nb][r], mul, sub));
          l[nb] += (s[mb][nb][0] + s[mb][nb][1]) + (s[mb][nb][2] + s[mb][nb][3]);
        }
      }
    };
    exps(0);
#pragma unroll
    for (int h2 = 0; h2 < HALVES; ++h2) {
      frag pf[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 8; ++j) pf[nb][j] = (T)s[h2 * 2 + (j >> 2)][nb][j & 3];
      if constexpr (HALVES == 2)
        if (h2 == 0) exps(1);
      if (MASKED && slow) {
        accumulate_pairs<T, DP, NB>(acc, pf, V, (h0 + h2) * 32, lane);
        continue;
      }
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const frag vf = TL::col_frag(V, b, h0 + h2, lane);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[b][nb] = mma(acc[b][nb], vf, pf[nb]);
      }
    }
    if (!MASKED) interleave_reads<T, DB * HALVES, 2, NB, 3>();
  };
  const int full = min(sp.nk, a.causal ? max(0, i0 + off + 1) : sp.nk) / kTileKeys;         // tiles all of whose pairs are visible
  int t = 0;
  for (; t < min(full, tiles); ++t) step(t, std::false_type{});
  for (; t < tiles; ++t) step(t, std::true_type{});
  if constexpr (SPLIT == 2) {
    __syncthreads();
    const Handover<DB, NB> there{smem + (wave >> 1) * Handover<DB, NB>::kBytes, lane};
    if (h0) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        there.number(2 * nb) = m[nb];
        there.number(2 * nb + 1) = l[nb];
#pragma unroll
        for (int b = 0; b < DB; ++b) there.block(b, nb) = acc[b][nb];
      }
    }
    __syncthreads();
    if (h0) return;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float other = there.number(2 * nb), next = fmaxf(m[nb], other);
      const float f = __builtin_amdgcn_exp2f(m[nb] - next), fo = __builtin_amdgcn_exp2f(other - next);
      m[nb] = next;
      l[nb] = l[nb] * f + there.number(2 * nb + 1) * fo;
#pragma unroll
      for (int b = 0; b < DB; ++b) acc[b][nb] = acc[b][nb] * f + there.block(b, nb) * fo;
    }
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int i = iw + nb * 16 + l16;
    const float sum = row_sum(l[nb]), inv = sum == 0.f ? 0.f : 1.f / sum;     // sum 0: the row sees no key
    if (i >= sp.nq) continue;
    T* o = out + (long)(sp.q0 + i) * a.ld_o + hi.h * a.d;
#pragma unroll
    for (int b = 0; b < DB; ++b)
      if (b * 16 + 4 * g < a.d) store4(o + b * 16 + 4 * g, acc[b][nb] * inv);
    if (g == 0) lse[(size_t)hi.h * a.rows_q + sp.q0 + i] = sum == 0.f ? kNegInf : (m[nb] + __builtin_amdgcn_logf(sum)) * kLn2;
  }
}

// The same for few query rows a key head (single tokens against a cache): the rows of a workgroup are 16 of the pairs (query, head of
// the group), so that a key head's rows are read once for its whole group, and the keys are dealt out: to workgroups in
// stretches, inside one to its wavefronts tile by tile.  A wavefront streams its tiles of 32 keys through LDS of its own, without
// a barrier, the next K on its way while V is worked on and the reverse; what the wavefronts have is joined in LDS, what the workgroups have by k_attend_join.  HBM-bound.
constexpr int kFewRows = 16;
constexpr int kFewKeys = 32;
template <typename T, int DP>
constexpr int few_waves() { return DP * (int)sizeof(T) > 256 ? 2 : 4; }
template <typename T, int DP>
constexpr int few_lds() { return few_waves<T, DP>() * 2 * kFewKeys * DP * (int)sizeof(T); }

// How the keys are dealt out: all row tiles' key counts together make `stretches` stretches of about equal length, a row tile having at least
// one to itself (stretches = 0: exactly one).  A stretch then is a row tile and a part of its keys; the partial results lie in the order of the
// stretches.
struct Stretch {
  Span sp;                   // tile: the row tile
  int part, parts, keys;     // which part of the row tile's keys, of how many, of how many keys each
  int first;                 // stretch of the row tile's first part
};
__device__ __forceinline__ int wave_total(int v) {
#pragma unroll
  for (int w = 1; w < 64; w *= 2) v += __shfl_xor(v, w);
  return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ long wave_total(long v) {
#pragma unroll
  for (int w = 1; w < 64; w *= 2) v += __shfl_xor(v, w);
  return (long)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}
// The keys of a part, of `keys` in all row tiles together.
__device__ __forceinline__ int part_keys(const AttendArgs& a, int stretches, int tiles, long keys) {
  const int spare = stretches - tiles;
  const long even = spare > 0 ? (keys + spare - 1) / spare : (long)a.rows_k + 1;
  return (int)min(max((even + kFewKeys - 1) / kFewKeys * kFewKeys, 4L * kFewKeys), 1L << 30);
}
// The stretch of index `at`, or (by_tile) the first one of row tile `at`; false if there are not as many.  By a plan, the row tiles' first items lie
// behind the stretches', and the keys of a part behind those.
__device__ __forceinline__ bool find_stretch(const AttendArgs& a, int stretches, int at, bool by_tile, Stretch& st) {
  if (a.firsts) {
    const int *tiles = a.firsts + a.sequences + 1, *of = by_tile ? tiles : a.firsts, group = a.heads / a.kv_heads;
    if (at >= of[a.sequences]) return false;
    const int s = find_sequence(of, a.sequences, at);
    st.keys = tiles[a.sequences + 1];
    read_span(a, s, st.sp.q0, st.sp.nq, st.sp.k0, st.sp.nk);
    st.sp.tiles = (st.sp.nq * group + kFewRows - 1) / kFewRows;
    st.parts = max(1, (st.sp.nk + st.keys - 1) / st.keys);
    const int inside = at - of[s];
    if (inside < 0) return false;                                            // see find_span
    st.sp.tile = by_tile ? inside : inside / st.parts;
    st.part = by_tile ? 0 : inside % st.parts;
    st.first = a.firsts[s] + st.sp.tile * st.parts;
    return st.sp.tile < st.sp.tiles;
  }
  const int lane = threadIdx.x & 63, group = a.heads / a.kv_heads;
  long keys = 0;
  int tiles = 0;
  int q0 = 0, nq = 0, k0 = 0, nk = 0;
  for (int s0 = 0; s0 < a.sequences; s0 += 64) {
    q0 = nq = k0 = nk = 0;
    if (s0 + lane < a.sequences) read_span(a, s0 + lane, q0, nq, k0, nk);
    const int n = (nq * group + kFewRows - 1) / kFewRows;
    tiles += wave_total(n);
    keys += wave_total((long)n * nk);                                        // overlapping sequences: more than 32 bits even in 1024s
  }
  st.keys = part_keys(a, stretches, tiles, keys);
  int first = 0;
  for (int s0 = 0; s0 < a.sequences; s0 += 64) {
    if (a.sequences > 64) {
      q0 = nq = k0 = nk = 0;
      if (s0 + lane < a.sequences) read_span(a, s0 + lane, q0, nq, k0, nk);
    }
    const int n = (nq * group + kFewRows - 1) / kFewRows, parts = max(1, (nk + st.keys - 1) / st.keys);
    int upto = n * parts, upto_tiles = n;
#pragma unroll
    for (int w = 1; w < 64; w *= 2) {
      const int v = __shfl_up(upto, w), u = __shfl_up(upto_tiles, w);
      if (lane >= w) {
        upto += v;
        upto_tiles += u;
      }
    }
    const int total = __builtin_amdgcn_readlane(by_tile ? upto_tiles : upto, 63);
    if (at < total) {
      const int l = __builtin_ctzll(__ballot(at < (by_tile ? upto_tiles : upto)));
      st.sp.q0 = __builtin_amdgcn_readlane(q0, l);
      st.sp.nq = __builtin_amdgcn_readlane(nq, l);
      st.sp.k0 = __builtin_amdgcn_readlane(k0, l);
      st.sp.nk = __builtin_amdgcn_readlane(nk, l);
      st.sp.tiles = __builtin_amdgcn_readlane(n, l);
      st.parts = __builtin_amdgcn_readlane(parts, l);
      const int before = __builtin_amdgcn_readlane(upto, l) - st.sp.tiles * st.parts;   // stretches of the sequences before, of these 64
      if (by_tile) {
        st.sp.tile = at - (__builtin_amdgcn_readlane(upto_tiles, l) - st.sp.tiles);
        st.part = 0;
      } else {
        st.sp.tile = (at - before) / st.parts;
        st.part = (at - before) % st.parts;
      }
      st.first = first + before + st.sp.tile * st.parts;
      return true;
    }
    at -= total;
    first += __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// The first items of many sequences, for find_span (rows > 0: an item is a tile of so many query rows, or with block 1 of key_rows key rows,
// into `keys`) and find_stretch (rows = 0).  A workgroup of 1024 threads a table; a thread takes a run of sequences.
struct Total1024 {
  int sums[16];
  long keys[16];
};
__device__ __forceinline__ int scan1024(int v, int& total, int* sums) {     // the sum of the threads before, and of all
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = v;
#pragma unroll
  for (int w = 1; w < 64; w *= 2) {
    const int u = __shfl_up(upto, w);
    if (lane >= w) upto += u;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    if (w < wave) before += sums[w];
    total += sums[w];
  }
  return before + upto - v;
}
static __global__ __launch_bounds__(1024) void k_attend_plan(AttendArgs a, int rows, int key_rows, int stretches, int* __restrict__ firsts, int* __restrict__ keys) {
  __shared__ Total1024 sh;
  const int per = (a.sequences + 1023) / 1024, s0 = min((int)threadIdx.x * per, a.sequences), s1 = min(s0 + per, a.sequences);
  const int group = a.heads / a.kv_heads;
  const bool by_keys = blockIdx.x == 1;
  int q0, nq, k0, nk, n = 0, total;
  long some = 0;
  for (int s = s0; s < s1; ++s) {
    read_span(a, s, q0, nq, k0, nk);
    const int t = by_keys ? (nk + key_rows - 1) / key_rows : rows ? (nq + rows - 1) / rows : (nq * group + kFewRows - 1) / kFewRows;
    n += t;
    some += (long)t * nk;
  }
  int at = scan1024(n, total, sh.sums);
  int* to = by_keys ? keys : rows ? firsts : firsts + a.sequences + 1;
  for (int s = s0; s < s1; ++s) {
    to[s] = at;
    read_span(a, s, q0, nq, k0, nk);
    at += by_keys ? (nk + key_rows - 1) / key_rows : rows ? (nq + rows - 1) / rows : (nq * group + kFewRows - 1) / kFewRows;
  }
  if (threadIdx.x == 0) to[a.sequences] = total;
  if (rows) return;
#pragma unroll
  for (int w = 1; w < 64; w *= 2) some += __shfl_xor(some, w);
  if ((threadIdx.x & 63) == 0) sh.keys[threadIdx.x >> 6] = some;
  __syncthreads();
  long all = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) all += sh.keys[w];
  const int part = part_keys(a, stretches, total, all);
  n = 0;
  for (int s = s0; s < s1; ++s) {
    read_span(a, s, q0, nq, k0, nk);
    n += (nq * group + kFewRows - 1) / kFewRows * max(1, (nk + part - 1) / part);
  }
  at = scan1024(n, total, sh.sums);
  for (int s = s0; s < s1; ++s) {
    firsts[s] = at;
    read_span(a, s, q0, nq, k0, nk);
    at += (nq * group + kFewRows - 1) / kFewRows * max(1, (nk + part - 1) / part);
  }
  if (threadIdx.x == 0) {
    firsts[a.sequences] = total;
    to[a.sequences + 1] = part;
  }
}

template <typename T, int DP, bool BIAS>
__global__ __launch_bounds__((few_waves<T, DP>() * 64)) void k_attend_few(AttendArgs a, int stretches, const T* __restrict__ q, const T* __restrict__ k,
                                                                        const T* __restrict__ v, T* __restrict__ out, float* __restrict__ lse,
                                                                        float* __restrict__ part, float* __restrict__ part_ml) {
  typedef Tile<T, DP> TL;
  typedef typename Frag<T>::type frag;
  constexpr int KS = DP / 32, DB = DP / 16, NW = few_waves<T, DP>(), kHalf = kFewKeys * TL::kPitch, kLoads = kFewKeys * TL::kChunks / 64;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ float ml[NW][2][kFewRows];
  const int group = a.heads / a.kv_heads, kvh = blockIdx.x % a.kv_heads;
  Stretch where;
  if (!find_stretch(a, stretches, blockIdx.x / a.kv_heads, false, where)) return;
  const Span& sp = where.sp;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  const int rows = sp.nq * group, off = sp.nk - sp.nq;
  const int row = min(sp.tile * kFewRows + l16, rows - 1);                   // past the end: the last one again, not written
  const int i = row / group, h = kvh * group + row % group, pos = i + off;
  const int first_pos = sp.tile * kFewRows / group + off, last_pos = min((sp.tile + 1) * kFewRows - 1, rows - 1) / group + off;
  const int kend = a.causal ? min(sp.nk, max(0, last_pos + 1)) : sp.nk;
  const int c0 = min(where.part * where.keys, kend), c1 = min(c0 + where.keys, kend);
  const int tiles = (c1 - c0 + kFewKeys - 1) / kFewKeys;
  const T* kb_ = k + (long)sp.k0 * a.ld_k + kvh * a.d;
  const T* vb_ = v + (long)sp.k0 * a.ld_v + kvh * a.d;
  unsigned char* mine = smem + wave * 2 * kHalf;
  const unsigned char* K = mine;
  const unsigned char* V = mine + kHalf;
  // past the last tile there is nothing to load, but as many loads are issued (of zeros): the waits count them
  auto stage_k = [&](int t) {
    const int kb = c0 + t * kFewKeys;
    TL::template stage<kFewKeys, 64>(kb_ + (long)kb * a.ld_k, a.ld_k, c1 - kb, a.d, mine, lane);
  };
  auto stage_v = [&](int t) {
    const int kb = c0 + t * kFewKeys;
    TL::template stage<kFewKeys, 64>(vb_ + (long)kb * a.ld_v, a.ld_v, c1 - kb, a.d, mine + kHalf, lane);
  };
  if (wave < tiles) {
    stage_k(wave);
    stage_v(wave);
  }
  frag qf[KS];
  const T* qrow = q + (long)(sp.q0 + i) * a.ld_q + h * a.d;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) qf[ks] = load_frag<T>(qrow, true, ks, g, a.d);
  float far_left = 0.f, far_right = 0.f;
  if (BIAS) {
    far_left = bias_value<T>(a, h, a.side - 1);
    far_right = a.causal ? 0.f : bias_value<T>(a, h, 2 * a.side - 1);
  }
  f32x4 acc[DB][1];
#pragma unroll
  for (int b = 0; b < DB; ++b) acc[b][0] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = kLowest, l = 0.f;
  for (int t = wave; t < tiles; t += NW) {
    wait_vmcnt<kLoads>();                                                    // K is here, V may be on its way
    __builtin_amdgcn_sched_barrier(0);
    const int kb = c0 + t * kFewKeys;
    f32x4 s[2][1];
#pragma unroll
    for (int mb = 0; mb < 2; ++mb) {
      s[mb][0] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[mb][0] = mma(s[mb][0], TL::row_frag(K, mb, ks, lane), qf[ks]);
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);                                      // lgkmcnt(0): K is read, its place takes the next one
    stage_k(t + NW);
    float mul = a.c, add = 0.f;
    if (BIAS) {
      if (kb + kFewKeys - 1 - first_pos <= -a.last) add = far_left;
      else if (kb - last_pos >= a.last) add = far_right;
      else {
        mul = 1.f;
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s[mb][0][r] = fmaf(s[mb][0][r], a.c, bias_value<T>(a, h, bucket_of(a, kb + mb * 16 + 4 * g + r - pos)));
      }
    }
    const bool masked = kb + kFewKeys > c1 || (a.causal && kb + kFewKeys - 1 > first_pos);
    if (masked) {
      const int end = a.causal ? min(c1, pos + 1) : c1;
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (kb + mb * 16 + 4 * g + r >= end) s[mb][0][r] = kNegInf;
    }
    float mx = kNegInf;
#pragma unroll
    for (int mb = 0; mb < 2; ++mb) mx = larger(larger(larger(larger(mx, s[mb][0][0]), s[mb][0][1]), s[mb][0][2]), s[mb][0][3]);
    mx = fmaf(row_max(mx), mul, add);
    if (__ballot(mx > m + kMaxSlack)) {
      const float next = fmaxf(m, mx), f = __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (int b = 0; b < DB; ++b) acc[b][0] *= f;
    }
    const float sub = add - m;
#pragma unroll
    for (int mb = 0; mb < 2; ++mb)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[mb][0][r], mul, sub));
        l += p;
        s[mb][0][r] = p;
      }
    frag pf[1];
#pragma unroll
    for (int j = 0; j < 8; ++j) pf[0][j] = (T)s[j >> 2][0][j & 3];
    wait_vmcnt<kLoads>();                                                    // V is here, the next K may be on its way
    __builtin_amdgcn_sched_barrier(0);
    if (masked && any_not_finite<T, DP, kFewKeys>(V, 0, lane)) {
      accumulate_pairs<T, DP, 1>(acc, pf, V, 0, lane);
    } else {
#pragma unroll
      for (int b = 0; b < DB; ++b) acc[b][0] = mma(acc[b][0], TL::col_frag(V, b, 0, lane), pf[0]);
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);
    stage_v(t + NW);
  }
  __builtin_amdgcn_s_waitcnt((0 << 8) | (7 << 4));                           // nothing may still be on its way into LDS
  // join the wavefronts: each leaves its sums [16][DP] where its tiles were
  l = row_sum(l);
  float* own = reinterpret_cast<float*>(mine);
#pragma unroll
  for (int b = 0; b < DB; ++b) *reinterpret_cast<f32x4*>(own + l16 * DP + ((b * 4 + g) ^ (l16 & 7)) * 4) = acc[b][0];
  if (g == 0) {
    ml[wave][0][l16] = m;
    ml[wave][1][l16] = l;
  }
  __syncthreads();
  for (int e = tid; e < kFewRows * DP / 4; e += NW * 64) {
    const int rr = e / (DP / 4), d4 = e % (DP / 4);
    float mm = ml[0][0][rr], sum = 0.f;
#pragma unroll
    for (int w = 1; w < NW; ++w) mm = fmaxf(mm, ml[w][0][rr]);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml[w][0][rr] - mm);
      sum += ml[w][1][rr] * f;
      o += *reinterpret_cast<const f32x4*>(smem + w * 2 * kHalf + (rr * DP + (d4 ^ (rr & 7)) * 4) * 4) * f;
    }
    const int at = sp.tile * kFewRows + rr;
    if (at >= rows) continue;
    if (where.parts > 1) {
      const size_t item = (size_t)(where.first + where.part) * a.kv_heads + kvh;
      *reinterpret_cast<f32x4*>(part + (item * kFewRows + rr) * DP + d4 * 4) = o;
      if (d4 == 0) {
        part_ml[(item * kFewRows + rr) * 2] = mm;
        part_ml[(item * kFewRows + rr) * 2 + 1] = sum;
      }
    } else {
      const int qi = sp.q0 + at / group, hh = kvh * group + at % group;
      if (d4 * 4 < a.d) store4(out + (long)qi * a.ld_o + hh * a.d + d4 * 4, o * (sum == 0.f ? 0.f : 1.f / sum));
      if (d4 == 0) lse[(size_t)hh * a.rows_q + qi] = sum == 0.f ? kNegInf : (mm + __builtin_amdgcn_logf(sum)) * kLn2;
    }
  }
}

// Joins the parts of k_attend_few's row tiles, in their order.  A thread takes four columns of a row.
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attend_join(AttendArgs a, int stretches, const float* __restrict__ part, const float* __restrict__ part_ml,
                                                     T* __restrict__ out, float* __restrict__ lse) {
  const int group = a.heads / a.kv_heads, kvh = blockIdx.x % a.kv_heads;
  Stretch where;
  if (!find_stretch(a, stretches, blockIdx.x / a.kv_heads, true, where) || where.parts == 1) return;
  if (where.first < 0 || where.parts > stretches - where.first) return;      // as in find_span
  const Span& sp = where.sp;
  const size_t pitch = (size_t)a.kv_heads * kFewRows;                        // rows of partial results from one part to the next
  for (int e = threadIdx.x; e < kFewRows * DP / 4; e += 256) {
    const int rr = e / (DP / 4), d4 = e % (DP / 4), at = sp.tile * kFewRows + rr;
    if (at >= sp.nq * group || d4 * 4 >= a.d) continue;
    const size_t row = ((size_t)where.first * a.kv_heads + kvh) * kFewRows + rr;
    float mm = kLowest, sum = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < where.parts; ++s) mm = fmaxf(mm, part_ml[(row + s * pitch) * 2]);
#pragma unroll 8
    for (int s = 0; s < where.parts; ++s) {
      const float f = __builtin_amdgcn_exp2f(part_ml[(row + s * pitch) * 2] - mm);
      sum += part_ml[(row + s * pitch) * 2 + 1] * f;
      o += *reinterpret_cast<const f32x4*>(part + (row + s * pitch) * DP + d4 * 4) * f;
    }
    const int qi = sp.q0 + at / group, hh = kvh * group + at % group;
    store4(out + (long)qi * a.ld_o + hh * a.d + d4 * 4, o * (sum == 0.f ? 0.f : 1.f / sum));
    if (d4 == 0) lse[(size_t)hh * a.rows_q + qi] = sum == 0.f ? kNegInf : (mm + __builtin_amdgcn_logf(sum)) * kLn2;
  }
}

// ---- backward -------------------------------------------------------------------------------------------------------------
// Two kernels, each with sums of its own in registers and no atomics: k_attend_dq (a workgroup has queries, the keys pass by) and
// k_attend_dkv (a workgroup has keys, the queries of all heads of the group pass by).  Scores and dP are formed in both: seven
// products for the formula's five, instead of partial sums of dq in memory or atomics whose order changes results.

// Bias gradient of a wavefront in LDS: sums of dS by r (as in the bias table), and 32 x 32 pairs at a time to sum along diagonals.
template <int NB>
struct BiasGrad {
  static constexpr int kPairs = NB * 16 * 32;                                // floats
  // dS of 32 keys (key 16 mb + 4 g + r of row nb * 16 + l16) into the buffer; row n holds its keys in chunks of four, swizzled.
  static __device__ __forceinline__ void put(float* buf, const f32x4 (&ds)[2][NB], int lane) {
    const int l16 = lane & 15, g = lane >> 4;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int mb = 0; mb < 2; ++mb) {
        const int n = nb * 16 + l16;
        *reinterpret_cast<f32x4*>(buf + n * 32 + ((mb * 4 + g) ^ ((n >> 1) & 7)) * 4) = ds[mb][nb];
      }
  }
  // Adds the diagonals to sums[]: key x of row n is r = x - n further right than sums' first.  A lane takes diagonal x = lane % 32
  // and, where that leaves the block, diagonal x - 32; the halves of the wavefront take the odd and the even rows.
  static __device__ __forceinline__ void diagonals(const float* buf, float* sums, int lane) {
    const int x = lane & 31, half = lane >> 5;
    float here = 0.f, wrapped = 0.f;
#pragma unroll
    for (int n2 = 0; n2 < NB * 8; ++n2) {
      const int n = 2 * n2 + half, key = (x + n) & 31;
      const float v = buf[n * 32 + (((key >> 2) ^ ((n >> 1) & 7)) << 2) + (key & 3)];
      const bool in = x + n < 32;
      here += in ? v : 0.f;
      wrapped += in ? 0.f : v;
    }
    const float other = half ? here : wrapped;                               // what the partner lane keeps
    const float got = __shfl_xor(other, 32);
    // lanes 0..31 keep diagonal x, lanes 32..63 diagonal x - 32; even rows first in both
    float* to = sums + (half ? x - 32 : x);
    *to += half ? got + wrapped : here + got;
  }
};

template <typename T, int DP, int NB, int NW, int SPLIT, bool BIAS>
__global__ __launch_bounds__(NW * 64, sizeof(T) == 2 ? 2 : 1) void k_attend_dq(AttendArgs a, const T* __restrict__ q, const T* __restrict__ k,
                                                      const T* __restrict__ v, const T* __restrict__ out, const float* __restrict__ lse,
                                                      const T* __restrict__ dout, T* __restrict__ dq, float* __restrict__ stat,
                                                      float* __restrict__ dbias_part, int want_dbias) {
  typedef Tile<T, DP> TL;
  typedef typename Frag<T>::type frag;
  constexpr int KS = DP / 32, DB = DP / 16, HALVES = 2 / SPLIT, ROWS = NW / SPLIT * NB * 16, NT = NW * 64;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  const int entries = BIAS ? bias_table_size(a.last) : 0;
  __shared__ float shared[NW][16];
  float* table = reinterpret_cast<float*>(smem + 4 * TL::kBytes);
  float* sums = table + ((entries + 3) & ~3) + wave * ((entries + 3) & ~3);
  float* pairs = table + ((entries + 3) & ~3) * (NW + 1) + wave * BiasGrad<NB>::kPairs;
  const HeadItem hi = head_item(a, blockIdx.x);
  float* part = BIAS ? dbias_part + ((size_t)hi.idx * a.heads + hi.h) * a.buckets : nullptr;
  Span sp;
  if (!find_span(a, hi.idx, [](int nq, int) { return (nq + ROWS - 1) / ROWS; }, sp)) {
    if (BIAS && want_dbias)
      for (int b = tid; b < a.buckets; b += NT) part[b] = 0.f;
    return;
  }
  const int i0 = (a.causal ? sp.tiles - 1 - sp.tile : sp.tile) * ROWS;
  const int iw = i0 + wave / SPLIT * NB * 16, off = sp.nk - sp.nq, h0 = SPLIT == 2 ? wave & 1 : 0;
  const int kend = a.causal ? min(sp.nk, max(0, min(i0 + ROWS, sp.nq) + off)) : sp.nk;
  const int tiles = (kend + kTileKeys - 1) / kTileKeys;
  const T* kb_ = k + (long)sp.k0 * a.ld_k + hi.kvh * a.d;
  const T* vb_ = v + (long)sp.k0 * a.ld_v + hi.kvh * a.d;
  auto stage = [&](int t) {
    unsigned char* to = smem + (t & 1) * 2 * TL::kBytes;
    TL::template stage<kTileKeys, NT>(kb_ + (long)t * kTileKeys * a.ld_k, a.ld_k, sp.nk - t * kTileKeys, a.d, to, tid);
    TL::template stage<kTileKeys, NT>(vb_ + (long)t * kTileKeys * a.ld_v, a.ld_v, sp.nk - t * kTileKeys, a.d, to + TL::kBytes, tid);
  };
  if (tiles > 0) stage(0);
  float far_left = 0.f, far_right = 0.f, sum_left = 0.f, sum_right = 0.f;
  if (BIAS) {
    fill_bias_table<T, NT>(a, hi.h, table, tid);
    if (want_dbias)
      for (int e = lane; e < entries; e += 64) sums[e] = 0.f;
    far_left = bias_value<T>(a, hi.h, a.side - 1);
    far_right = a.causal ? 0.f : bias_value<T>(a, hi.h, 2 * a.side - 1);
  }
  frag qf[NB][KS], dof[NB][KS];
  f32x4 acc[DB][NB];
  float lse2[NB], delta[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int i = iw + nb * 16 + l16, row = sp.q0 + min(i, sp.nq - 1);
    const bool in = i < sp.nq;
    float dot = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      qf[nb][ks] = load_frag<T>(q + (long)row * a.ld_q + hi.h * a.d, in, ks, g, a.d);
      dof[nb][ks] = load_frag<T>(dout + (long)row * a.ld_do + hi.h * a.d, in, ks, g, a.d);
      const frag of = load_frag<T>(out + (long)row * a.ld_o + hi.h * a.d, in, ks, g, a.d);
#pragma unroll
      for (int j = 0; j < 8; ++j) dot = fmaf(to_f32(dof[nb][ks][j]), to_f32(of[j]), dot);
    }
    const float sum = row_sum(dot), e = lse[(size_t)hi.h * a.rows_q + row];
    const bool sees = in && e != kNegInf;
    delta[nb] = sees ? sum : 0.f;                                            // a row that sees no key: P = 0, and what its dout holds has no part
    lse2[nb] = sees ? e * kLog2e : __builtin_inff();
#pragma unroll
    for (int b = 0; b < DB; ++b) acc[b][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int lo = iw + off, top = lo + NB * 16 - 1;
  // P (into s) and dP of 32 keys of tile t, the second half of it if h2; P of a pair that is not visible is 0, and so is its dP.
  auto pairs_of = [&](int t, int h2, auto masked, auto near, f32x4 (&s)[2][NB], f32x4 (&dp)[2][NB], int side) {
    constexpr bool MASKED = decltype(masked)::value, NEAR = BIAS && decltype(near)::value;
    const unsigned char* K = smem + (t & 1) * 2 * TL::kBytes;
    const unsigned char* V = K + TL::kBytes;
    const int kb = t * kTileKeys;
#pragma unroll
    for (int mb = 0; mb < 2; ++mb) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) s[mb][nb] = dp[mb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const frag kf = TL::row_frag(K, h2 * 2 + mb, ks, lane);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[mb][nb] = mma(s[mb][nb], kf, qf[nb][ks]);
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const frag vf = TL::row_frag(V, h2 * 2 + mb, ks, lane);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) dp[mb][nb] = mma(dp[mb][nb], vf, dof[nb][ks]);
      }
    }
    interleave_reads<T, 4 * KS, 1, NB, 4>();
    if (NEAR && !side) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float* tb = table + kb + h2 * 32 + 4 * g - (lo + nb * 16 + l16) + a.last + kPad;
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[mb][nb][r] = fmaf(s[mb][nb][r], a.c, tb[mb * 16 + r]);
      }
    }
    const float mul = NEAR && !side ? 1.f : a.c, far = side < 0 ? far_left : side > 0 ? far_right : 0.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float sub = far - lse2[nb];
      const int end = a.causal ? min(sp.nk, lo + nb * 16 + l16 + 1) : sp.nk;
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          s[mb][nb][r] = __builtin_amdgcn_exp2f(fmaf(s[mb][nb][r], mul, sub));
          if (MASKED && kb + h2 * 32 + mb * 16 + 4 * g + r >= end) s[mb][nb][r] = dp[mb][nb][r] = 0.f;
        }
    }
  };
  // -1, 1: all pairs of the tile are in the last bucket of that side
  auto side_of = [&](int kb) { return !BIAS ? 0 : kb + kTileKeys - 1 - lo <= -a.last ? -1 : kb - top >= a.last ? 1 : 0; };
  // A row's number summed over the wavefronts that share it (every wavefront of the workgroup comes here).
  auto both = [&](float v) {
    if constexpr (SPLIT == 1) return v;
    if (g == 0) shared[wave][l16] = v;
    __syncthreads();
    const float sum = shared[wave & ~1][l16] + shared[wave | 1][l16];
    __syncthreads();
    return sum;
  };
  // delta from out as it was rounded to bf16 is off by up to 2^-8 <|do|, |out|>, which counts where few keys share a row's weight (dq's and dk's
  // error against 64 bits, 16 to 100 keys: 1.85 times that of the two roundings of P and dS alone).  So where a row has at most two tiles of
  // keys, which then both lie in LDS, it is added up from the pairs first: sum of P dP.
  if (sizeof(T) == 2 && tiles <= 2) {
    if (tiles == 2) stage(1);
    wait_vmcnt<0>();
    __syncthreads();
    float sum[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) sum[nb] = 0.f;
#pragma unroll 1
    for (int u = 0; u < HALVES * tiles; ++u) {
      f32x4 s[2][NB], dp[2][NB];
      const int t = u / HALVES;
      pairs_of(t, h0 + u % HALVES, std::true_type{}, std::true_type{}, s, dp, side_of(t * kTileKeys));
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
          for (int r = 0; r < 4; ++r) sum[nb] = fmaf(s[mb][nb][r], dp[mb][nb][r], sum[nb]);
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) delta[nb] = both(row_sum(sum[nb]));
  }
  // With a bias: rows' sums of dS, which delta's error alone makes differ from 0, and of P in the last bucket of each side.  At the end the error's share
  // of the last buckets is taken out (2048 rows, 32 heads of 128: dbias' error against 64 bits 0.0031 -> 0.0016), and delta goes to k_attend_dkv
  // without it, whether dbias is wanted or not: dk does not depend on that.  (The near buckets keep their share, and so does dq.)
  float rest[NB], far_p[NB][2];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) rest[nb] = far_p[nb][0] = far_p[nb][1] = 0.f;
  auto step = [&](int t, auto masked, auto near) {                           // as in k_attend; near: some pair may need the table
    constexpr bool MASKED = decltype(masked)::value, NEAR = decltype(near)::value;
    wait_vmcnt<0>();
    __syncthreads();
    if (t + 1 < tiles) stage(t + 1);
    const int kb = t * kTileKeys;
    if (iw >= sp.nq || (MASKED && a.causal && kb > top)) return;
    const unsigned char* K = smem + (t & 1) * 2 * TL::kBytes;
    int side = side_of(kb);
    if (!NEAR && BIAS) side = side < 0 ? -1 : 1;
    const bool slow = MASKED && any_not_finite<T, DP, 32 * HALVES>(K, h0 * 32, lane);
#pragma unroll
    for (int hh = 0; hh < HALVES; ++hh) {
      const int h2 = h0 + hh;
      f32x4 s[2][NB], dp[2][NB];
      pairs_of(t, h2, masked, near, s, dp, side);
      if (BIAS && want_dbias && side) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float sum = 0.f;
#pragma unroll
          for (int mb = 0; mb < 2; ++mb) sum += (s[mb][nb][0] + s[mb][nb][1]) + (s[mb][nb][2] + s[mb][nb][3]);
          if (side < 0) far_p[nb][0] += sum;
          else far_p[nb][1] += sum;
        }
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[mb][nb][r] *= dp[mb][nb][r] - delta[nb];
      if (BIAS) {
        float all = 0.f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          float sum = 0.f;
#pragma unroll
          for (int mb = 0; mb < 2; ++mb) sum += (s[mb][nb][0] + s[mb][nb][1]) + (s[mb][nb][2] + s[mb][nb][3]);
          rest[nb] += sum;
          all += sum;
        }
        if (!NEAR || side) {
          if (side < 0) sum_left += all;
          else sum_right += all;
        } else if (want_dbias) {
          asm volatile("" ::: "memory");                                     // lanes read what other lanes of the wavefront wrote: in program order
          BiasGrad<NB>::put(pairs, s, lane);
          asm volatile("" ::: "memory");
          BiasGrad<NB>::diagonals(pairs, sums + kb + h2 * 32 - lo + a.last + kPad, lane);
        }
      }
      frag df[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int j = 0; j < 8; ++j) df[nb][j] = (T)s[j >> 2][nb][j & 3];
      if (MASKED && slow) {
        accumulate_pairs<T, DP, NB>(acc, df, K, h2 * 32, lane);
        continue;
      }
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const frag kf = TL::col_frag(K, b, h2, lane);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[b][nb] = mma(acc[b][nb], kf, df[nb]);
      }
      if (!MASKED) interleave_reads<T, DB, 2, NB, 3>();
    }
  };
  const int full = min(sp.nk, a.causal ? max(0, i0 + off + 1) : sp.nk) / kTileKeys;
  // tiles all of whose pairs with the workgroup's rows are in the last bucket: those before `left`, those from `right` on
  const int left = max(0, i0 + off - a.last + 1) / kTileKeys, right = (max(0, i0 + ROWS - 1 + off + a.last) + kTileKeys - 1) / kTileKeys;
  int t = 0;
  if (BIAS) {
    for (; t < min(left, min(full, tiles)); ++t) step(t, std::false_type{}, std::false_type{});
    for (; t < min(right, min(full, tiles)); ++t) step(t, std::false_type{}, std::true_type{});
  }
  for (; t < min(full, tiles); ++t) step(t, std::false_type{}, std::false_type{});
  for (; t < tiles; ++t) step(t, std::true_type{}, std::true_type{});
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int i = iw + nb * 16 + l16;
    if (BIAS) {
      const float off_by = both(row_sum(rest[nb]));
      sum_left -= off_by * far_p[nb][0];
      sum_right -= off_by * far_p[nb][1];
      delta[nb] += off_by;
    }
    if (g == 0 && h0 == 0 && i < sp.nq) {
      stat[(size_t)hi.h * a.rows_q + sp.q0 + i] = lse2[nb];
      stat[(size_t)(a.heads + hi.h) * a.rows_q + sp.q0 + i] = delta[nb];
    }
  }
  if constexpr (SPLIT == 2) {
    __syncthreads();
    const Handover<DB, NB> there{smem + (wave >> 1) * Handover<DB, NB>::kBytes, lane};
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int b = 0; b < DB; ++b)
        if (h0) there.block(b, nb) = acc[b][nb];
    __syncthreads();
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int b = 0; b < DB; ++b)
        if (!h0) acc[b][nb] += there.block(b, nb);
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int i = iw + nb * 16 + l16;
    if (i >= sp.nq || h0) continue;
    T* o = dq + (long)(sp.q0 + i) * a.ld_dq + hi.h * a.d;
#pragma unroll
    for (int b = 0; b < DB; ++b)
      if (b * 16 + 4 * g < a.d) store4(o + b * 16 + 4 * g, acc[b][nb] * a.scale);
  }
  if (BIAS && want_dbias) {                                                  // sums by r -> sums by bucket, in a fixed order
    float* far_sums = reinterpret_cast<float*>(smem);                        // [2][NW], over the tiles
    sum_left = wave_sum(sum_left);
    sum_right = wave_sum(sum_right);
    __syncthreads();
    if (lane == 0) {
      far_sums[wave] = sum_left;
      far_sums[NW + wave] = sum_right;
    }
    __syncthreads();
    const int pitch = (entries + 3) & ~3, mid = a.last + kPad;
    const float* all = table + pitch;
    for (int b = wave; b < a.buckets; b += NW) {
      const bool right = b >= a.side;
      const int n = right ? b - a.side : b;
      const int from = n ? a.borders[n - 1] : (right ? 1 : 0), to = n < a.n_borders ? a.borders[n] : mid + 1;
      float sum = 0.f;
      for (int dist = from + lane; dist < to; dist += 64)
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += all[w * pitch + mid + (right ? dist : -dist)];
      sum = wave_sum(sum);
      if (n == a.n_borders)
#pragma unroll
        for (int w = 0; w < NW; ++w) sum += far_sums[(right ? NW : 0) + w];
      if (lane == 0) part[b] = sum;
    }
  }
}

// dbias[h][b] = sum over the items of their parts, in their order: 64 threads an entry.
template <typename T>
__global__ __launch_bounds__(64) void k_attend_dbias(int items, int entries, const float* __restrict__ part, T* __restrict__ dbias) {
  const int e = blockIdx.x;
  float sum = 0.f;
  for (int i = threadIdx.x; i < items; i += 64) sum += part[(size_t)i * entries + e];
  sum = wave_sum(sum);
  if (threadIdx.x == 0) dbias[e] = from_f32<T>(sum);
}

// Keys' and values' gradients.  Workgroup: NW wavefronts of 16 NB keys of one key head; the queries of the group's heads pass by in
// tiles of 64, Q and dO of two tiles in LDS with the rows' lse (base 2) and delta.
template <typename T, int DP>
constexpr int dkv_stage_bytes() { return 2 * Tile<T, DP>::kBytes + 2 * 64 * 4; }

template <typename T, int DP, int NB, int NW, int SPLIT, bool BIAS>
__global__ __launch_bounds__(NW * 64, sizeof(T) == 2 ? 2 : 1) void k_attend_dkv(AttendArgs a, const T* __restrict__ q, const T* __restrict__ k,
                                                       const T* __restrict__ v, const T* __restrict__ dout, const float* __restrict__ stat,
                                                       T* __restrict__ dk, T* __restrict__ dv) {
  typedef Tile<T, DP> TL;
  typedef typename Frag<T>::type frag;
  constexpr int KS = DP / 32, DB = DP / 16, HALVES = 2 / SPLIT, ROWS = NW / SPLIT * NB * 16, NT = NW * 64, kStage = dkv_stage_bytes<T, DP>();
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float* table = reinterpret_cast<float*>(smem + 2 * kStage);
  const int group = a.heads / a.kv_heads, kvh = blockIdx.x % a.kv_heads;
  Span sp;
  if (!find_span(a, blockIdx.x / a.kv_heads, [](int, int nk) { return (nk + ROWS - 1) / ROWS; }, sp)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  const int j0 = sp.tile * ROWS, jw = j0 + wave / SPLIT * NB * 16, jtop = jw + NB * 16 - 1, off = sp.nk - sp.nq;
  const int h0 = SPLIT == 2 ? wave & 1 : 0;                                  // SPLIT = 2: of every tile, the half that this wavefront takes
  const int first = a.causal ? max(0, j0 - off) / kTileKeys : 0, per = max(0, (sp.nq + kTileKeys - 1) / kTileKeys - first);
  const int steps = per * group;
  auto stage = [&](int it) {
    const int h = kvh * group + it / per, r0 = (first + it % per) * kTileKeys, rows = sp.nq - r0;
    unsigned char* to = smem + (it & 1) * kStage;
    TL::template stage<kTileKeys, NT>(q + (long)(sp.q0 + r0) * a.ld_q + h * a.d, a.ld_q, rows, a.d, to, tid);
    TL::template stage<kTileKeys, NT>(dout + (long)(sp.q0 + r0) * a.ld_do + h * a.d, a.ld_do, rows, a.d, to + TL::kBytes, tid);
    if (wave < 2) {                                                          // lse by the first wavefront, delta by the second
      const float* src = stat + (size_t)(wave * a.heads + h) * a.rows_q + sp.q0 + r0 + min(lane, rows - 1);
      load4_to_lds(src, to + 2 * TL::kBytes + wave * 256);
    }
  };
  if (steps > 0) stage(0);
  frag kf[NB][KS], vf[NB][KS];
  f32x4 ak[DB][NB], av[DB][NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int j = jw + nb * 16 + l16;
    const long row = sp.k0 + min(j, sp.nk - 1);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kf[nb][ks] = load_frag<T>(k + row * a.ld_k + kvh * a.d, j < sp.nk, ks, g, a.d);
      vf[nb][ks] = load_frag<T>(v + row * a.ld_v + kvh * a.d, j < sp.nk, ks, g, a.d);
    }
#pragma unroll
    for (int b = 0; b < DB; ++b) ak[b][nb] = av[b][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  float far_left = 0.f, far_right = 0.f;
  auto step = [&](int it, int tile, auto masked) {
    constexpr bool MASKED = decltype(masked)::value;
    wait_vmcnt<0>();
    __syncthreads();
    if (BIAS && tile == 0) {
      const int h = kvh * group + it / per;
      fill_bias_table<T, NT>(a, h, table, tid);
      far_left = bias_value<T>(a, h, a.side - 1);
      far_right = a.causal ? 0.f : bias_value<T>(a, h, 2 * a.side - 1);
      __syncthreads();
    }
    if (it + 1 < steps) stage(it + 1);
    const int qb = (first + tile) * kTileKeys, lo = qb + off, top = lo + kTileKeys - 1;   // positions of the tile's queries
    if (jw >= sp.nk || (MASKED && a.causal && jw > top)) return;
    const unsigned char* Q = smem + (it & 1) * kStage;
    const unsigned char* dO = Q + TL::kBytes;
    const float* st = reinterpret_cast<const float*>(dO + TL::kBytes);
    int side = 0;
    if (BIAS) side = jtop - lo <= -a.last ? -1 : (jw - top >= a.last ? 1 : 0);
    const float far = side < 0 ? far_left : side > 0 ? far_right : 0.f;
    const bool slow = MASKED && (any_not_finite<T, DP, 32 * HALVES>(dO, h0 * 32, lane) || any_not_finite<T, DP, 32 * HALVES>(Q, h0 * 32, lane));
#pragma unroll
    for (int hh = 0; hh < HALVES; ++hh) {
      const int h2 = h0 + hh;
      frag pf[NB], df[NB];
#pragma unroll
      for (int mb = 0; mb < 2; ++mb) {
        f32x4 s[NB], dp[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[nb] = dp[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const frag qf = TL::row_frag(Q, h2 * 2 + mb, ks, lane);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) s[nb] = mma(s[nb], qf, kf[nb][ks]);
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const frag of = TL::row_frag(dO, h2 * 2 + mb, ks, lane);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) dp[nb] = mma(dp[nb], of, vf[nb][ks]);
        }
        const int row = (h2 * 2 + mb) * 16 + 4 * g;
        const f32x4 e = *reinterpret_cast<const f32x4*>(st + row), dl = *reinterpret_cast<const f32x4*>(st + 64 + row);
        if (BIAS && !side) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            const float* tb = table + jw + nb * 16 + l16 - (lo + row) + a.last + kPad;
#pragma unroll
            for (int r = 0; r < 4; ++r) s[nb][r] = fmaf(s[nb][r], a.c, tb[-r]);
          }
        }
        const float mul = BIAS && !side ? 1.f : a.c;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float p = __builtin_amdgcn_exp2f(fmaf(s[nb][r], mul, far - e[r]));
            float ds = p * (dp[nb][r] - dl[r]);
            if (MASKED && (qb + row + r >= sp.nq || (a.causal && jw + nb * 16 + l16 > lo + row + r))) p = ds = 0.f;
            pf[nb][mb * 4 + r] = (T)p;
            df[nb][mb * 4 + r] = (T)ds;
          }
      }
      if (MASKED && slow) {
        accumulate_pairs<T, DP, NB>(av, pf, dO, h2 * 32, lane);
        accumulate_pairs<T, DP, NB>(ak, df, Q, h2 * 32, lane);
        continue;
      }
#pragma unroll
      for (int b = 0; b < DB; ++b) {
        const frag of = TL::col_frag(dO, b, h2, lane), qf = TL::col_frag(Q, b, h2, lane);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          av[b][nb] = mma(av[b][nb], of, pf[nb]);
          ak[b][nb] = mma(ak[b][nb], qf, df[nb]);
        }
      }
      if (!MASKED) interleave_reads<T, 2 * DB, 2, NB, 3>();
    }
  };
  // of a head's tiles: those with queries before some of the workgroup's keys, those all of whose pairs are visible, a short last one
  const int whole = sp.nq / kTileKeys - first;                               // tiles before the short one
  const int diag = a.causal ? max(0, min(per, (j0 + ROWS - 1 - off + kTileKeys - 1) / kTileKeys - first)) : 0;
  int it = 0;
  for (int hh = 0; hh < (steps > 0 ? group : 0); ++hh) {
    for (int tile = 0; tile < per;) {
      while (tile < per && (tile < diag || tile >= whole)) step(it++, tile++, std::true_type{});
      while (tile < whole) step(it++, tile++, std::false_type{});
    }
  }
  if constexpr (SPLIT == 2) {
    const Handover<DB, NB> there{smem + (wave >> 1) * Handover<DB, NB>::kBytes, lane};
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int b = 0; b < DB; ++b)
          if (h0) there.block(b, nb) = which ? av[b][nb] : ak[b][nb];
      __syncthreads();
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int b = 0; b < DB; ++b)
          if (!h0) (which ? av : ak)[b][nb] += there.block(b, nb);
    }
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int j = jw + nb * 16 + l16;
    if (j >= sp.nk || h0) continue;
    T* ok = dk + (long)(sp.k0 + j) * a.ld_dk + kvh * a.d;
    T* ov = dv + (long)(sp.k0 + j) * a.ld_dv + kvh * a.d;
#pragma unroll
    for (int b = 0; b < DB; ++b)
      if (b * 16 + 4 * g < a.d) {
        store4(ok + b * 16 + 4 * g, ak[b][nb] * a.scale);
        store4(ov + b * 16 + 4 * g, av[b][nb]);
      }
  }
}

}  // namespace dchag
