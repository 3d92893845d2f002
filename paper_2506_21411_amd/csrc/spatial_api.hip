// C ABI of the spatial block's operators: attention over packed sequences with its backward pass, and activations kept in 8 bits
// with the weight gradient that reads them.  Argument validation, workspace layout and kernel launches.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "host_base.h"
#include "k_attend.h"
#include "k_keep8.h"

using namespace dchag;

namespace {

// The threads of a launch are counted in 32 bits.
constexpr long kMostThreads = 0xffffffffL;
bool too_large(long workgroups, int threads) { return workgroups > kMostThreads / threads; }

// ---- attention ------------------------------------------------------------------------------------------------------------
// Rows and sequences are counted in 32 bits in the kernels, and so are a row's end plus a tile, a part of the keys plus another, and a key head's
// pairs of (query, head of the group) where rows are few.  A part holds up to 2^30 keys: a sequence of more would be two parts where the workspace has
// no room for parts (part_keys).
constexpr int kMostRows = 1 << 30;
int check_attention(dchag_dtype dt, const dchag_attention* a) {
  if (dt != DCHAG_F32 && dt != DCHAG_BF16) return DCHAG_ERR_DTYPE;
  if (!a || !a->q_starts || !a->k_starts) return DCHAG_ERR_NULL;
  if (a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads || a->heads > 4096) return DCHAG_ERR_SHAPE;
  if (a->head_dim < 8 || a->head_dim > 128 || a->head_dim % 8) return DCHAG_ERR_SHAPE;
  if (a->sequences < 0 || a->rows_q < 0 || a->rows_k < 0 || (a->causal != 0 && a->causal != 1)) return DCHAG_ERR_SHAPE;
  if (a->sequences > kMostRows || a->rows_q > kMostRows || a->rows_k > kMostRows) return DCHAG_ERR_SHAPE;
  if (!(a->scale >= 0.f) || !(a->scale < INFINITY)) return DCHAG_ERR_SHAPE;
  const int64_t lds[8] = {a->ld_q, a->ld_k, a->ld_v, a->ld_out, a->ld_dout, a->ld_dq, a->ld_dk, a->ld_dv};
  const int heads_of[8] = {a->heads, a->kv_heads, a->kv_heads, a->heads, a->heads, a->heads, a->kv_heads, a->kv_heads};
  for (int i = 0; i < 8; ++i)
    if (lds[i] != 0 && (lds[i] < (int64_t)heads_of[i] * a->head_dim || lds[i] % 8 || lds[i] > (1 << 23))) return DCHAG_ERR_SHAPE;
  if (a->bias) {
    if (!a->borders) return DCHAG_ERR_NULL;
    if (a->n_borders < 1 || a->n_borders > kMaxBorders) return DCHAG_ERR_SHAPE;
    for (int i = 0; i < a->n_borders; ++i)
      if (a->borders[i] < 1 || a->borders[i] > kMaxDistance || (i && a->borders[i] <= a->borders[i - 1])) return DCHAG_ERR_SHAPE;
    if (misaligned(a->bias)) return DCHAG_ERR_ALIGN;
  }
  if ((reinterpret_cast<uintptr_t>(a->q_starts) | reinterpret_cast<uintptr_t>(a->k_starts) | reinterpret_cast<uintptr_t>(a->k_used)) & 3u)
    return DCHAG_ERR_ALIGN;
  return DCHAG_OK;
}

AttendArgs kernel_args(const dchag_attention* a) {
  AttendArgs k;
  memset(&k, 0, sizeof k);
  k.q_starts = a->q_starts;
  k.k_starts = a->k_starts;
  k.k_used = a->k_used;
  k.sequences = a->sequences;
  k.rows_q = a->rows_q;
  k.rows_k = a->rows_k;
  k.heads = a->heads;
  k.kv_heads = a->kv_heads;
  k.d = a->head_dim;
  k.causal = a->causal;
  const long dq = (long)a->heads * a->head_dim, dk = (long)a->kv_heads * a->head_dim;
  k.ld_q = a->ld_q ? a->ld_q : dq;
  k.ld_k = a->ld_k ? a->ld_k : dk;
  k.ld_v = a->ld_v ? a->ld_v : dk;
  k.ld_o = a->ld_out ? a->ld_out : dq;
  k.ld_do = a->ld_dout ? a->ld_dout : dq;
  k.ld_dq = a->ld_dq ? a->ld_dq : dq;
  k.ld_dk = a->ld_dk ? a->ld_dk : dk;
  k.ld_dv = a->ld_dv ? a->ld_dv : dk;
  k.scale = a->scale > 0.f ? a->scale : 1.f / sqrtf((float)a->head_dim);
  k.c = k.scale * kLog2e;
  k.bias = a->bias;
  if (a->bias) {
    k.n_borders = a->n_borders;
    k.last = a->borders[a->n_borders - 1];
    k.side = a->n_borders + 1;
    k.buckets = a->causal ? k.side : 2 * k.side;
    memcpy(k.borders, a->borders, sizeof(int) * a->n_borders);
  }
  return k;
}

// Most tiles of `rows` rows that sequences of `total` rows can have.
long tiles_bound(long total, long sequences, int rows) { return total / rows + std::min(sequences, total); }

// Many sequences: tables of their first items, made by a launch of its own before the others.
bool planned(const AttendArgs& a) { return a.sequences > kPlanFrom; }
size_t plan_bytes(const AttendArgs& a, int tables) { return planned(a) ? align_up(((size_t)a.sequences + 2) * tables * 4) : 0; }

int padded_dim(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }

// Rows of a workgroup: 16 nb for every `split` of its nw wavefronts.
struct TileShape {
  int nb, nw, split;
  int rows() const { return 16 * nb * nw / split; }
};
// Tiles of 32, two wavefronts to a row, where tiles of 128 rows would leave compute units without work (64 rows gave every SIMD one wavefront: training
// step, 4 x 256 rows, 16 heads of 64, kernels' us 44 / 36), and for sequences that they hold whole (2048 of 24 rows, us: 1193 / 915).
// fp32, whose fragments fill the registers, has 16 rows a wavefront: tiles of 64, or of 32 as above where 64 leave SIMDs with less than two
// wavefronts (2 x 512 rows, 8 heads of 64, us: 120 / 82).  bf16 otherwise: tiles of 256 for long sequences whose rows see every key (heads of more
// than 32: a tile of keys is a load for each of 512 threads), else of 128, since a causal tile's work grows with its rows and short sequences
// fill large tiles badly (eight of 77 to 2048 rows, us, 128 / 256: 55 / 74).
// 16 heads, 8192 rows, TFLOP/s with tiles of 64 / 128 / 256: heads of 64 714 / 799 / 839, heads of 128 836 / 1107 / 1152; causal, 32 heads of 128
// 832 / 1069 / 1046.
TileShape tile_shape(dchag_dtype dt, int d, long rows, long sequences, long heads, bool causal) {
  const long cus = compute_units();
  if (dt != DCHAG_BF16) return {1, 4, tiles_bound(rows, sequences, 64) * heads < 2 * cus ? 2 : 1};
  if (tiles_bound(rows, sequences, 128) * heads < cus || rows <= 32 * sequences) return {1, 4, 2};
  if (causal || d <= 32 || rows < 1024 * sequences || tiles_bound(rows, sequences, 256) * heads < cus) return {2, 4, 1};
  return {2, 8, 1};
}

template <int N> using Const = std::integral_constant<int, N>;

// How a forward call goes about its rows: few (k_attend_few) or tiles of query rows.
struct ForwardPlan {
  bool few;
  TileShape tile;
  long items, stretches;      // row tiles at most; few: parts that their keys are dealt to, 0: not split
  size_t part, part_ml, plan, total;
};
ForwardPlan forward_plan(dchag_dtype dt, const AttendArgs& a) {
  ForwardPlan p;
  memset(&p, 0, sizeof p);
  const int group = a.heads / a.kv_heads;
  const long rows = (long)a.rows_q * group, seqs = std::min<long>(a.sequences, a.rows_q);
  // Few rows: on average at most as many as a row tile has, of grouped heads two tiles' (the other kernel reads the keys once a head), and
  // many keys or hardly any rows.  us, few / tiles of 32 rows: 64 sequences, 2000 keys, 16 heads, 10 rows 104 / 105, 20 rows 133 / 106; 32 heads on 8,
  // 5 rows 56 / 73; 2048 sequences of 10 rows and keys 200 / 132.
  p.few = rows <= (group > 1 ? 2L : 1L) * kFewRows * seqs && (a.rows_k >= 128 * seqs || rows <= 4 * seqs) && rows <= kMostRows;
  if (p.few) {
    p.items = rows / kFewRows + std::min<long>(a.sequences, rows);
    const long fill = 4L * compute_units() / a.kv_heads;                     // twice the workgroups that the chip holds at once
    const bool split = p.items > 0 && p.items * 2 < fill && a.rows_k / std::max(1, a.sequences) >= 1024;
    p.stretches = split ? fill : 0;
    if (split) {
      const size_t n = (size_t)p.stretches * a.kv_heads * kFewRows;
      p.part_ml = align_up(n * padded_dim(a.d) * 4);
      p.plan = p.part_ml + align_up(n * 8);
    }
    p.total = p.plan + plan_bytes(a, 2) + 256;
    return p;
  }
  p.tile = tile_shape(dt, a.d, a.rows_q, a.sequences, a.heads, a.causal);
  p.items = tiles_bound(a.rows_q, a.sequences, p.tile.rows());
  p.total = p.plan + plan_bytes(a, 1) + 256;
  return p;
}

template <typename T, int DP, int NB, int NW, int SPLIT, bool BIAS>
int launch_attend(const AttendArgs& a, const ForwardPlan& p, const void* q, const void* k, const void* v, void* out, float* lse, hipStream_t st) {
  const int lds = 4 * Tile<T, DP>::kBytes + (BIAS ? bias_table_size(a.last) * 4 : 0);
  auto kern = k_attend<T, DP, NB, NW, SPLIT, BIAS>;
  if (ensure_dynamic_lds(reinterpret_cast<const void*>(kern), lds)) return DCHAG_ERR_LAUNCH;
  StageTimer tm(DCHAG_STAGE_ATTEND, st);
  kern<<<dim3((unsigned)(p.items * a.heads)), NW * 64, lds, st>>>(a, static_cast<const T*>(q), static_cast<const T*>(k), static_cast<const T*>(v),
                                                                  static_cast<T*>(out), lse);
  return launch_status();
}

template <typename T, int DP, bool BIAS>
int launch_few(const AttendArgs& a, const ForwardPlan& p, const void* q, const void* k, const void* v, void* out, float* lse, unsigned char* ws,
               hipStream_t st) {
  auto kern = k_attend_few<T, DP, BIAS>;
  constexpr int lds = few_lds<T, DP>();
  if (ensure_dynamic_lds(reinterpret_cast<const void*>(kern), lds)) return DCHAG_ERR_LAUNCH;
  float* part = reinterpret_cast<float*>(ws + p.part);
  float* ml = reinterpret_cast<float*>(ws + p.part_ml);
  {
    StageTimer tm(DCHAG_STAGE_ATTEND, st);
    kern<<<dim3((unsigned)(std::max(p.items, p.stretches) * a.kv_heads)), few_waves<T, DP>() * 64, lds, st>>>(
        a, (int)p.stretches, static_cast<const T*>(q), static_cast<const T*>(k), static_cast<const T*>(v), static_cast<T*>(out), lse, part, ml);
  }
  if (p.stretches) {
    StageTimer tm(DCHAG_STAGE_ATTEND_JOIN, st);
    k_attend_join<T, DP><<<dim3((unsigned)(p.items * a.kv_heads)), 256, 0, st>>>(a, (int)p.stretches, part, ml, static_cast<T*>(out), lse);
  }
  return launch_status();
}

template <typename T, int DP>
int attend_dim(const AttendArgs& a, const ForwardPlan& p, const void* q, const void* k, const void* v, void* out, float* lse, unsigned char* ws,
               hipStream_t st) {
  if (p.few) return a.bias ? launch_few<T, DP, true>(a, p, q, k, v, out, lse, ws, st) : launch_few<T, DP, false>(a, p, q, k, v, out, lse, ws, st);
  const auto go = [&](auto nb, auto nw, auto split) {
    return a.bias ? launch_attend<T, DP, nb.value, nw.value, split.value, true>(a, p, q, k, v, out, lse, st)
                  : launch_attend<T, DP, nb.value, nw.value, split.value, false>(a, p, q, k, v, out, lse, st);
  };
  if constexpr (sizeof(T) == 2) {
    if constexpr (DP > 32)
      if (p.tile.nw == 8) return go(Const<2>{}, Const<8>{}, Const<1>{});
    if (p.tile.nb == 2) return go(Const<2>{}, Const<4>{}, Const<1>{});
  } else {
    if (p.tile.split == 1) return go(Const<1>{}, Const<4>{}, Const<1>{});
  }
  return go(Const<1>{}, Const<4>{}, Const<2>{});
}

struct BackwardPlan {
  TileShape q, k;
  long items_q, items_k;
  size_t stat, dbias, plan, total;
};
// Query tiles as in the forward pass, but of 256 for heads of 128 with a bias, whose sums leave room for one workgroup a compute unit (2048 rows, 32
// heads, us, tiles of 16 x 8 / 32 x 8 rows: 166 / 130).  Key tiles of heads of 128 have 16 keys a wavefront, as two
// sums and two operands of 32 do not fit its registers (4096 rows, 16 heads, us: 16 x 4 296, 16 x 8 291, 32 x 4 755, or 377 with one wavefront a SIMD; causal with
// grouped heads, 10374 rows: 745, 867, 2905).
// The bias gradient's sums by distance, one set a wavefront, may leave no room for that many of them (heads of 128: borders beyond some 700; fp32 460):
// then fewer.
template <typename T, int DP, int NB, int NW>
constexpr int dq_lds(int last) {
  return 4 * Tile<T, DP>::kBytes + (last ? ((bias_table_size(last) + 3) & ~3) * 4 * (NW + 1) + NW * BiasGrad<NB>::kPairs * 4 : 0);
}
constexpr int kLdsLimit = 160 * 1024 - 1024;                                 // 1024: what the kernels have beside it
BackwardPlan backward_plan(dchag_dtype dt, const AttendArgs& a) {
  BackwardPlan p;
  p.q = tile_shape(dt, a.d, a.rows_q, a.sequences, a.heads, a.causal);
  p.k = tile_shape(dt, a.d, a.rows_k, a.sequences, a.kv_heads, true);
  if (a.d > 64) {
    if (a.bias && p.q.nb == 2) p.q = {2, 8, 1};
    if (p.q.nb == 2 && a.bias && dq_lds<bf16, 128, 2, 8>(a.last) > kLdsLimit) p.q = {1, 4, 2};
    if (dt == DCHAG_F32 && a.bias && dq_lds<float, 128, 1, 4>(a.last) > kLdsLimit) p.q = {1, 2, 1};
    if (p.k.nb == 2) p.k = {1, 4, 1};
  }
  p.items_q = tiles_bound(a.rows_q, a.sequences, p.q.rows());
  p.items_k = tiles_bound(a.rows_k, a.sequences, p.k.rows());
  p.stat = 0;
  p.dbias = align_up((size_t)2 * a.heads * a.rows_q * 4);
  p.plan = p.dbias + align_up((size_t)p.items_q * a.heads * a.buckets * 4);
  p.total = p.plan + plan_bytes(a, 2) + 256;
  return p;
}

struct BackwardPtrs {
  const void *q, *k, *v, *out, *dout;
  const float* lse;
  void *dq, *dk, *dv, *dbias;
  const int *firsts_q, *firsts_k;
};

template <typename T, int DP, int NB, int NW, int SPLIT, bool BIAS>
int launch_dq(AttendArgs a, const BackwardPlan& p, const BackwardPtrs& t, unsigned char* ws, hipStream_t st) {
  const int lds = dq_lds<T, DP, NB, NW>(BIAS ? a.last : 0);
  auto kern = k_attend_dq<T, DP, NB, NW, SPLIT, BIAS>;
  if (ensure_dynamic_lds(reinterpret_cast<const void*>(kern), lds)) return DCHAG_ERR_LAUNCH;
  a.firsts = t.firsts_q;
  StageTimer tm(DCHAG_STAGE_BWD_ATTEND_QUERY, st);
  if (p.items_q > 0)
    kern<<<dim3((unsigned)(p.items_q * a.heads)), NW * 64, lds, st>>>(
        a, static_cast<const T*>(t.q), static_cast<const T*>(t.k), static_cast<const T*>(t.v), static_cast<const T*>(t.out), t.lse,
        static_cast<const T*>(t.dout), static_cast<T*>(t.dq), reinterpret_cast<float*>(ws + p.stat), reinterpret_cast<float*>(ws + p.dbias),
        t.dbias != nullptr);
  return launch_status();
}
template <typename T, int DP, int NB, int NW, int SPLIT, bool BIAS>
int launch_dkv(AttendArgs a, const BackwardPlan& p, const BackwardPtrs& t, unsigned char* ws, hipStream_t st) {
  const int lds = 2 * dkv_stage_bytes<T, DP>() + (BIAS ? bias_table_size(a.last) * 4 : 0);
  auto kern = k_attend_dkv<T, DP, NB, NW, SPLIT, BIAS>;
  if (ensure_dynamic_lds(reinterpret_cast<const void*>(kern), lds)) return DCHAG_ERR_LAUNCH;
  a.firsts = t.firsts_k;
  StageTimer tm(DCHAG_STAGE_BWD_ATTEND_KEY, st);
  if (p.items_k > 0)
    kern<<<dim3((unsigned)(p.items_k * a.kv_heads)), NW * 64, lds, st>>>(
        a, static_cast<const T*>(t.q), static_cast<const T*>(t.k), static_cast<const T*>(t.v), static_cast<const T*>(t.dout),
        reinterpret_cast<const float*>(ws + p.stat), static_cast<T*>(t.dk), static_cast<T*>(t.dv));
  return launch_status();
}

// What follows the queries' gradients: the keys', and the sum of the bias gradient's parts.
template <typename T, int DP, bool BIAS>
int rest_of_backward(const AttendArgs& a, const BackwardPlan& p, const BackwardPtrs& t, unsigned char* ws, hipStream_t st) {
  const auto keys = [&](auto nb, auto split) { return launch_dkv<T, DP, nb.value, 4, split.value, BIAS>(a, p, t, ws, st); };
  int rc;
  if (p.k.split == 2) rc = keys(Const<1>{}, Const<2>{});
  else if constexpr (sizeof(T) == 4 || DP == 128) rc = keys(Const<1>{}, Const<1>{});
  else rc = keys(Const<2>{}, Const<1>{});
  if (rc || !BIAS || !t.dbias) return rc;
  StageTimer tm(DCHAG_STAGE_BWD_ATTEND_BIAS, st);
  const int entries = a.heads * a.buckets;
  k_attend_dbias<T><<<dim3(entries), 64, 0, st>>>((int)p.items_q, entries, reinterpret_cast<const float*>(ws + p.dbias), static_cast<T*>(t.dbias));
  return launch_status();
}
template <typename T, int DP, bool BIAS>
int backward_bias(const AttendArgs& a, const BackwardPlan& p, const BackwardPtrs& t, unsigned char* ws, hipStream_t st) {
  const auto queries = [&](auto nb, auto nw, auto split) { return launch_dq<T, DP, nb.value, nw.value, split.value, BIAS>(a, p, t, ws, st); };
  int rc;
  if constexpr (sizeof(T) == 4 && DP == 128 && BIAS)
    if (p.q.nw == 2) {
      rc = queries(Const<1>{}, Const<2>{}, Const<1>{});
      return rc ? rc : rest_of_backward<T, DP, BIAS>(a, p, t, ws, st);
    }
  if (p.q.split == 2) rc = queries(Const<1>{}, Const<4>{}, Const<2>{});
  else if constexpr (sizeof(T) == 4) rc = queries(Const<1>{}, Const<4>{}, Const<1>{});
  else if constexpr (DP == 128 && BIAS) rc = queries(Const<2>{}, Const<8>{}, Const<1>{});
  else if constexpr (DP == 32) rc = queries(Const<2>{}, Const<4>{}, Const<1>{});
  else rc = p.q.nw == 8 ? queries(Const<2>{}, Const<8>{}, Const<1>{}) : queries(Const<2>{}, Const<4>{}, Const<1>{});
  return rc ? rc : rest_of_backward<T, DP, BIAS>(a, p, t, ws, st);
}
template <typename T, int DP>
int backward_dim(const AttendArgs& a, const BackwardPlan& p, const BackwardPtrs& t, unsigned char* ws, hipStream_t st) {
  return a.bias ? backward_bias<T, DP, true>(a, p, t, ws, st) : backward_bias<T, DP, false>(a, p, t, ws, st);
}

bool bad_workspace(const void* ws, size_t have, size_t need) {
  return !ws || (reinterpret_cast<uintptr_t>(ws) & (kAlign - 1)) || have < need;
}

// ---- weight gradient from 8 bits ------------------------------------------------------------------------------------------
struct GradPlan {
  int side, tiles, splits, stretch;
  size_t total;
};
// Squares of dW of 256 (bf16; a compute unit holds one), 128 (two) or 64, the largest that give every compute unit one, over as many stretches
// of the rows as the chip holds.  1536 x 1024 over 32768 rows, us: squares of 128 156, of 256 123.
GradPlan grad_plan(dchag_dtype dt, long rows, int d_out, int d_in) {
  GradPlan p;
  const int cus = compute_units();
  const long most = std::max(1L, (rows + 255) / 256);                        // a stretch of fewer rows costs more in partial sums than it gains
  const auto count = [&](int side) { return (long)((d_out + side - 1) / side) * ((d_in + side - 1) / side); };
  p.side = dt == DCHAG_BF16 && count(256) * most >= cus ? 256 : count(128) * most >= cus ? 128 : 64;
  p.tiles = (int)count(p.side);
  p.splits = (int)std::max(1L, std::min({(p.side == 256 ? 1L : 2L) * cus / p.tiles, most, 64L}));
  p.stretch = (int)(((rows + p.splits - 1) / p.splits + 63) / 64 * 64);
  if (p.stretch < 64) p.stretch = 64;
  p.splits = (int)std::max(1L, (rows + p.stretch - 1) / p.stretch);
  p.total = p.splits > 1 ? align_up(((size_t)p.splits * d_out * d_in + (size_t)p.splits * d_out) * 4) : 256;
  return p;
}
int check_rows8(dchag_dtype dt, int64_t rows, int D, int64_t ld, int turns) {
  if (dt != DCHAG_F32 && dt != DCHAG_BF16) return DCHAG_ERR_DTYPE;
  if (rows < 0 || D < 8 || D % 8 || D > (1 << 20) || (ld != 0 && (ld < D || ld % 8 || ld > (1 << 23)))) return DCHAG_ERR_SHAPE;
  if (rows > kMostThreads / 1024 * 256 * turns / ((D + 31) / 32)) return DCHAG_ERR_SHAPE;   // four threads a block of 32, of whole workgroups
  return DCHAG_OK;
}
Rows8 rows8(int64_t rows, int D, int64_t ld) {
  if (D % 32 == 0 && (ld == 0 || ld == D)) return Rows8{1, (long)rows * D, (long)rows * D, (long)rows * (D / 32)};
  return Rows8{(long)rows, D, ld ? (long)ld : D, (D + 31) / 32};
}
unsigned rows8_grid(const Rows8& r, int turns) { return (unsigned)((r.rows * r.blocks * 4 + 256 * turns - 1) / (256 * turns)); }
int check_grad8(dchag_dtype dt, int rows, int d_out, int d_in, int64_t ld) {
  if (dt != DCHAG_F32 && dt != DCHAG_BF16) return DCHAG_ERR_DTYPE;
  if (rows < 0 || rows > (1 << 30) || d_out < 8 || d_in < 8 || d_out % 8 || d_in % 8 || d_out > (1 << 20) || d_in > (1 << 20)) return DCHAG_ERR_SHAPE;
  if (ld != 0 && (ld < d_out || ld % 8 || ld > (1 << 23))) return DCHAG_ERR_SHAPE;
  if ((int64_t)((d_out + 63) / 64) * ((d_in + 63) / 64) > (1 << 22)) return DCHAG_ERR_SHAPE;
  return DCHAG_OK;
}

template <typename T, int WO, int WI, int NO, int NI>
int launch_grad8(const GradPlan& p, int rows, int d_out, int d_in, long ld, const void* dy, const void* codes, const void* scales, void* dW, void* db,
                 float* part, hipStream_t st) {
  typedef GradTile<T, WO, WI, NO, NI> GT;
  auto kern = k_weight_grad8<T, WO, WI, NO, NI>;
  constexpr int lds = GT::kLds;
  if (ensure_dynamic_lds(reinterpret_cast<const void*>(kern), lds)) return DCHAG_ERR_LAUNCH;
  {
    StageTimer tm(DCHAG_STAGE_WEIGHT_GRAD8, st);
    kern<<<dim3((unsigned)((p.tiles * p.splits + kXcds - 1) / kXcds * kXcds)), GT::kThreads, lds, st>>>(
        rows, d_out, d_in, ld, p.stretch, p.splits, static_cast<const T*>(dy), static_cast<const unsigned char*>(codes),
        static_cast<const unsigned char*>(scales), static_cast<T*>(dW), static_cast<T*>(db), p.splits > 1 ? part : nullptr);
  }
  if (p.splits > 1) {
    StageTimer tm(DCHAG_STAGE_WEIGHT_GRAD8, st);
    const size_t n = (size_t)d_out * d_in, all = n + d_out;
    k_grad_join<T><<<dim3((unsigned)((all / 4 + 255) / 256)), 256, 0, st>>>(n, d_out, p.splits, part, static_cast<T*>(dW), static_cast<T*>(db));
  }
  return launch_status();
}

}  // namespace

extern "C" {

size_t dchag_attend_workspace_bytes(dchag_dtype dt, const dchag_attention* att, int which) {
  if (check_attention(dt, att)) return 0;
  const AttendArgs a = kernel_args(att);
  if (which == 0) return forward_plan(dt, a).total;
  if (which == 1) return backward_plan(dt, a).total;
  return 0;
}

int dchag_attend(dchag_dtype dt, const dchag_attention* att, const void* q, const void* k, const void* v, void* out, float* lse, void* workspace,
                 size_t workspace_bytes, void* stream) {
  int rc = check_attention(dt, att);
  if (rc) return rc;
  AttendArgs a = kernel_args(att);
  if (a.rows_q > 0 && (!q || !out || !lse)) return DCHAG_ERR_NULL;
  if (a.rows_q > 0 && a.rows_k > 0 && (!k || !v)) return DCHAG_ERR_NULL;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out) || misaligned(lse)) return DCHAG_ERR_ALIGN;
  const ForwardPlan p = forward_plan(dt, a);
  if (bad_workspace(workspace, workspace_bytes, p.total)) return DCHAG_ERR_WORKSPACE;
  if (p.few ? too_large(std::max(p.items, p.stretches) * a.kv_heads, 256) : too_large(p.items * a.heads, p.tile.nw * 64)) return DCHAG_ERR_SHAPE;
  if (p.items == 0) return DCHAG_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  set_level(0);
  if (planned(a)) {
    int* firsts = reinterpret_cast<int*>(ws + p.plan);
    StageTimer tm(DCHAG_STAGE_ATTEND_PLAN, st);
    k_attend_plan<<<dim3(1), 1024, 0, st>>>(a, p.few ? 0 : p.tile.rows(), 0, (int)p.stretches, firsts, nullptr);
    a.firsts = firsts;
  }
  const int dp = padded_dim(a.d);
  if (dt == DCHAG_F32)
    return dp == 32 ? attend_dim<float, 32>(a, p, q, k, v, out, lse, ws, st)
         : dp == 64 ? attend_dim<float, 64>(a, p, q, k, v, out, lse, ws, st) : attend_dim<float, 128>(a, p, q, k, v, out, lse, ws, st);
  return dp == 32 ? attend_dim<bf16, 32>(a, p, q, k, v, out, lse, ws, st)
       : dp == 64 ? attend_dim<bf16, 64>(a, p, q, k, v, out, lse, ws, st) : attend_dim<bf16, 128>(a, p, q, k, v, out, lse, ws, st);
}

int dchag_attend_backward(dchag_dtype dt, const dchag_attention* att, const void* q, const void* k, const void* v, const void* out, const float* lse,
                          const void* dout, void* dq, void* dk, void* dv, void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_attention(dt, att);
  if (rc) return rc;
  AttendArgs a = kernel_args(att);
  if (a.rows_q > 0 && (!q || !out || !lse || !dout || !dq)) return DCHAG_ERR_NULL;
  if (a.rows_k > 0 && (!k || !v || !dk || !dv)) return DCHAG_ERR_NULL;
  if (dbias && !att->bias) return DCHAG_ERR_SHAPE;
  if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(out) || misaligned(lse) || misaligned(dout) || misaligned(dq) || misaligned(dk) ||
      misaligned(dv) || misaligned(dbias))
    return DCHAG_ERR_ALIGN;
  const BackwardPlan p = backward_plan(dt, a);
  if (bad_workspace(workspace, workspace_bytes, p.total)) return DCHAG_ERR_WORKSPACE;
  if (too_large(p.items_q * a.heads, p.q.nw * 64) || too_large(p.items_k * a.kv_heads, 256)) return DCHAG_ERR_SHAPE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  unsigned char* ws = static_cast<unsigned char*>(workspace);
  BackwardPtrs t{q, k, v, out, dout, lse, dq, dk, dv, dbias, nullptr, nullptr};
  set_level(0);
  if (planned(a)) {
    int* firsts = reinterpret_cast<int*>(ws + p.plan);
    t.firsts_q = firsts;
    t.firsts_k = firsts + a.sequences + 2;
    StageTimer tm(DCHAG_STAGE_ATTEND_PLAN, st);
    k_attend_plan<<<dim3(2), 1024, 0, st>>>(a, p.q.rows(), p.k.rows(), 0, firsts, firsts + a.sequences + 2);
  }
  const int dp = padded_dim(a.d);
  if (dt == DCHAG_F32)
    return dp == 32 ? backward_dim<float, 32>(a, p, t, ws, st) : dp == 64 ? backward_dim<float, 64>(a, p, t, ws, st) : backward_dim<float, 128>(a, p, t, ws, st);
  return dp == 32 ? backward_dim<bf16, 32>(a, p, t, ws, st) : dp == 64 ? backward_dim<bf16, 64>(a, p, t, ws, st) : backward_dim<bf16, 128>(a, p, t, ws, st);
}

int dchag_pack8(dchag_dtype dt, int64_t rows, int D, int64_t ld, const void* x, void* codes, void* scales, void* stream) {
  int rc = check_rows8(dt, rows, D, ld, kTurns);
  if (rc) return rc;
  if (rows == 0) return DCHAG_OK;
  if (!x || !codes || !scales) return DCHAG_ERR_NULL;
  if (misaligned(x) || misaligned(codes) || misaligned(scales)) return DCHAG_ERR_ALIGN;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const Rows8 r = rows8(rows, D, ld);
  unsigned char *c = static_cast<unsigned char*>(codes), *e = static_cast<unsigned char*>(scales);
  set_level(0);
  StageTimer tm(DCHAG_STAGE_PACK8, st);
  if (dt == DCHAG_F32) k_pack8<float><<<rows8_grid(r, kTurns), 256, 0, st>>>(r, static_cast<const float*>(x), c, e);
  else k_pack8<bf16><<<rows8_grid(r, kTurns), 256, 0, st>>>(r, static_cast<const bf16*>(x), c, e);
  return launch_status();
}

int dchag_unpack8(dchag_dtype dt, int64_t rows, int D, int64_t ld, const void* codes, const void* scales, void* x, void* stream) {
  int rc = check_rows8(dt, rows, D, ld, 1);
  if (rc) return rc;
  if (rows == 0) return DCHAG_OK;
  if (!x || !codes || !scales) return DCHAG_ERR_NULL;
  if (misaligned(x) || misaligned(codes) || misaligned(scales)) return DCHAG_ERR_ALIGN;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const Rows8 r = rows8(rows, D, ld);
  const unsigned char *c = static_cast<const unsigned char*>(codes), *e = static_cast<const unsigned char*>(scales);
  set_level(0);
  StageTimer tm(DCHAG_STAGE_UNPACK8, st);
  if (dt == DCHAG_F32) k_unpack8<float><<<rows8_grid(r, 1), 256, 0, st>>>(r, c, e, static_cast<float*>(x));
  else k_unpack8<bf16><<<rows8_grid(r, 1), 256, 0, st>>>(r, c, e, static_cast<bf16*>(x));
  return launch_status();
}

size_t dchag_weight_grad8_workspace_bytes(dchag_dtype dt, int rows, int d_out, int d_in) {
  if (check_grad8(dt, rows, d_out, d_in, 0)) return 0;
  return grad_plan(dt, rows, d_out, d_in).total;
}

int dchag_weight_grad8(dchag_dtype dt, int rows, int d_out, int d_in, int64_t ld, const void* dy, const void* codes, const void* scales, void* dW,
                       void* db, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_grad8(dt, rows, d_out, d_in, ld);
  if (rc) return rc;
  if (!dW || (rows > 0 && (!dy || !codes || !scales))) return DCHAG_ERR_NULL;
  if (misaligned(dy) || misaligned(codes) || misaligned(scales) || misaligned(dW) || misaligned(db)) return DCHAG_ERR_ALIGN;
  const GradPlan p = grad_plan(dt, rows, d_out, d_in);
  if (bad_workspace(workspace, workspace_bytes, p.total)) return DCHAG_ERR_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  set_level(0);
  float* part = static_cast<float*>(workspace);
  const auto launch = dt == DCHAG_F32 ? (p.side == 64 ? launch_grad8<float, 2, 2, 2, 2> : launch_grad8<float, 4, 4, 2, 2>)
                      : p.side == 64  ? launch_grad8<bf16, 2, 2, 2, 2>
                      : p.side == 128 ? launch_grad8<bf16, 4, 4, 2, 2> : launch_grad8<bf16, 8, 4, 2, 4>;
  return launch(p, rows, d_out, d_in, ld ? ld : d_out, dy, codes, scales, dW, db, part, st);
}

}  // extern "C"
