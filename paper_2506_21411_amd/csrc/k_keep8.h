// Activations kept in 8 bits between the passes, and the weight gradient that reads them.
//
// A row of D values is held as e4m3 codes and one exponent byte for every 32 of them: value = code * 2^(byte - 127).  The exponent
// is the smallest with which the block's largest finite magnitude does not exceed e4m3's largest number, 448 = 1.75 * 2^8, so
// nothing saturates and scaling is exact; the one rounding (to nearest even, 3 mantissa bits) is off by at most 2^-4 of a value, or
// by 2^-10 * 2^(byte - 127) for the values too small for a normal code.  Values beyond 1.875 * 2^127, which would be rounded to 2^128,
// are held as that.  A value that is not finite is held as NaN and has no part in the exponent.
#pragma once
#include "k_attend.h"

namespace dchag {

// 2^(byte - 127) and its reciprocal.  Byte 0 is 2^-127, below the normal numbers.
__device__ __forceinline__ float scale_of(unsigned byte) { return __builtin_bit_cast(float, byte ? byte << 23 : 0x00400000u); }
__device__ __forceinline__ float unscale_of(unsigned byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

// Eight codes of two words as numbers of the block's scale.
__device__ __forceinline__ void decode8(uint2 w, float sc, float (&v)[8]) {
  typedef __attribute__((ext_vector_type(2))) float f2;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int word = (int)(k ? w.y : w.x);
    const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(word, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(word, true);
    v[4 * k] = lo[0] * sc;
    v[4 * k + 1] = lo[1] * sc;
    v[4 * k + 2] = hi[0] * sc;
    v[4 * k + 3] = hi[1] * sc;
  }
}
// The same as bf16 numbers: one instruction for two, which takes the scale's exponent (0 stands for 2^-127).
__device__ __forceinline__ bf16x8 decode8_bf16(uint2 w, unsigned byte) {
  typedef __attribute__((ext_vector_type(2))) __bf16 b2;
  const float sc = __builtin_bit_cast(float, byte << 23);
  const b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, sc, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, sc, true);
  const b2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, sc, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, sc, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const f32x4 a = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p)), b = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p + 4));
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = a[j];
    v[4 + j] = b[j];
  }
}
__device__ __forceinline__ void load8(const bf16* p, float (&v)[8]) {
  const bf16x8 a = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(p));
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)a[j];
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(bf16* p, const float (&v)[8]) {
  bf16x8 o;
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = (bf16)v[j];
  *reinterpret_cast<bf16x8*>(p) = o;
}

// Both HBM-bound.  Four threads share a block of 32 values, eight each.  A thread packs kTurns of its eights, whose loads are all on their way
// before the first is used and pass the caches by, as do the codes (neither is needed again soon); it unpacks one, into the caches
// (2^29 bf16 values, us: packing 259 this way, 292 one at a time through the caches; unpacking 253, four at a time 262).  Rows
// without gaps whose blocks are all whole are one long row to the kernels (the host passes them so), which saves the division.
constexpr int kTurns = 4;
struct Rows8 {
  long rows, D, ld, blocks;            // blocks of a row
  // Element offsets in x (ld) and in the codes (D) of thread chunk id, and the block's index; false past the end.
  __device__ __forceinline__ bool at(long id, long& x, long& code, long& block) const {
    block = id >> 2;
    const long row = rows == 1 ? 0 : block / blocks, e = (block - row * blocks) * 32 + (id & 3) * 8;
    x = row * ld + e;
    code = row * D + e;
    return row < rows && e < D;
  }
};

template <typename T>
__global__ __launch_bounds__(256) void k_pack8(Rows8 r, const T* __restrict__ x, unsigned char* __restrict__ codes, unsigned char* __restrict__ scales) {
  const long first = (long)blockIdx.x * (256 * kTurns) + threadIdx.x;
  long code[kTurns], block[kTurns];
  bool in[kTurns];
  float v[kTurns][8];
#pragma unroll
  for (int u = 0; u < kTurns; ++u) {
    long at;
    in[u] = r.at(first + u * 256, at, code[u], block[u]);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[u][j] = 0.f;
    if (in[u]) load8(x + at, v[u]);
  }
#pragma unroll
  for (int u = 0; u < kTurns; ++u) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float m = fabsf(v[u][j]);
      if (m <= -kLowest) top = fmaxf(top, m);
      else v[u][j] = __builtin_nanf("");
    }
    top = fmaxf(top, dpp_move<kDppSwapPairs>(top));
    top = fmaxf(top, dpp_move<kDppSwapHalves>(top));
    const unsigned bits = __builtin_bit_cast(unsigned, top);
    const int byte = max((int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), 0);
    if (!in[u]) continue;
    const float sc = unscale_of(byte);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[u][j] *= sc;
    if (byte == 247)                                                         // 256 * 2^120 is no number of T
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (fabsf(v[u][j]) > 240.f) v[u][j] = copysignf(240.f, v[u][j]);
    int w0 = 0, w1 = 0;
    w0 = __builtin_amdgcn_cvt_pk_fp8_f32(v[u][0], v[u][1], w0, false);
    w0 = __builtin_amdgcn_cvt_pk_fp8_f32(v[u][2], v[u][3], w0, true);
    w1 = __builtin_amdgcn_cvt_pk_fp8_f32(v[u][4], v[u][5], w1, false);
    w1 = __builtin_amdgcn_cvt_pk_fp8_f32(v[u][6], v[u][7], w1, true);
    typedef __attribute__((ext_vector_type(2))) int i2;
    __builtin_nontemporal_store(i2{w0, w1}, reinterpret_cast<i2*>(codes + code[u]));
    if ((threadIdx.x & 3) == 0) scales[block[u]] = (unsigned char)byte;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_unpack8(Rows8 r, const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales, T* __restrict__ x) {
  long at, code, block;
  if (!r.at((long)blockIdx.x * 256 + threadIdx.x, at, code, block)) return;
  float v[8];
  decode8(*reinterpret_cast<const uint2*>(codes + code), scale_of(scales[block]), v);
  store8(x + at, v);
}

// dW[o][i] = sum over rows of dy[row][o] x[row][i], db[o] = sum of dy[row][o], x held in 8 bits.  For long inputs no unit is full: matrix instructions
// take 52 % of the busy cycles, LDS 27 % (1536 x 1024 over 32768 rows), and the loop without its loads 95 of 107 us.
// Workgroup: OS x IS of dW over one stretch of the rows, its wavefronts NO x NI parts of 16 WO x 16 WI; slices of 64 rows of
// both operands lie in LDS as they lie in memory (both have the sum's index as their row) and are read transposed.  dy comes by
// direct-to-LDS loads; of x a thread takes half a block of 32 codes or a whole one, which it turns into numbers of T once for all that read them: every
// e4m3 value times a power of two is a bf16 number (below 2^-126 it is rounded).  Stretches beyond one leave partial sums that
// k_grad_join adds up in their order.  An XCD takes neighbouring parts of dW and one stretch, so that its L2 serves most of both operands.
template <typename T, int WO, int WI, int NO, int NI>
struct GradTile {
  static constexpr int kThreads = 64 * NO * NI, kOut = 16 * WO * NO, kIn = 16 * WI * NI;
  static constexpr int kLds = 3 * Tile<T, kOut>::kBytes + 2 * Tile<T, kIn>::kBytes;
};
template <typename T, int WO, int WI, int NO, int NI>
__global__ __launch_bounds__((64 * NO * NI), sizeof(T) == 2 ? 2 : 1) void k_weight_grad8(int rows, int d_out, int d_in, long ld, int stretch, int splits,
                                                          const T* __restrict__ dy, const unsigned char* __restrict__ codes,
                                                          const unsigned char* __restrict__ scales, T* __restrict__ dW, T* __restrict__ db,
                                                          float* __restrict__ part) {
  typedef GradTile<T, WO, WI, NO, NI> GT;
  constexpr int NT = GT::kThreads, OS = GT::kOut, IS = GT::kIn, CH = 64 * IS / 8 / NT;   // CH: chunks of 8 codes a thread takes
  typedef Tile<T, OS> TO;
  typedef Tile<T, IS> TI;
  typedef typename Frag<T>::type frag;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  const int ni = (d_in + IS - 1) / IS, no = (d_out + OS - 1) / OS;
  const int total = ni * no * splits, per = (total + kXcds - 1) / kXcds, work = blockIdx.x % kXcds * per + blockIdx.x / kXcds;
  if ((int)blockIdx.x / kXcds >= per || work >= total) return;
  const int it = work % ni, ot = work / ni % no, sp = work / ni / no;
  const int o0 = ot * OS, i0 = it * IS, r0 = sp * stretch, r1 = min(rows, r0 + stretch);
  const int wo = wave / NI * WO, wi = wave % NI * WI, blocks = (d_in + 31) / 32;         // wo, wi in blocks of 16
  const int tiles = (r1 - r0 + 63) / 64;
  constexpr int kPerRow = IS / 8 / CH;                                       // threads a row of x; a thread's chunks lie kPerRow apart
  const int xrow = tid / kPerRow, xc = tid % kPerRow;
  uint2 cw[CH];
  unsigned sc[CH];
  auto load_x = [&](int t) {
    const int r = r0 + t * 64 + xrow;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int e = i0 + (xc + c * kPerRow) * 8;
      const bool in = r < r1 && e < d_in;
      cw[c] = in ? *reinterpret_cast<const uint2*>(codes + (size_t)r * d_in + e) : make_uint2(0, 0);
      sc[c] = in ? scales[(size_t)r * blocks + e / 32] : 0;
    }
  };
  auto put_x = [&](int t) {
    unsigned char* to = smem + 3 * TO::kBytes + (t & 1) * TI::kBytes + xrow * TI::kPitch;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int chunk = xc + c * kPerRow;
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<bf16x8*>(to + (chunk ^ TI::swz(xrow)) * 16) = decode8_bf16(cw[c], sc[c]);
      } else {
        float v[8];
        decode8(cw[c], scale_of(sc[c]), v);
        *reinterpret_cast<f32x4*>(to + ((chunk * 2) ^ TI::swz(xrow)) * 16) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4*>(to + ((chunk * 2 + 1) ^ TI::swz(xrow)) * 16) = f32x4{v[4], v[5], v[6], v[7]};
      }
    }
  };
  auto stage_dy = [&](int t) {
    TO::template stage<64, NT>(dy + (long)(r0 + t * 64) * ld + o0, ld, r1 - r0 - t * 64, min(OS, d_out - o0), smem + t % 3 * TO::kBytes, tid);
  };
  frag ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = (T)1.f;
  // dy's sums are dealt out to the wavefronts and workgroups that share its fragments: this wavefront adds up those from slot on, ni * NI apart
  constexpr int MOST = WO / NI;                                              // with one workgroup to a row of them
  const int slot = it * NI + wave % NI, apart = ni * NI;
  f32x4 acc[WO][WI], bs[MOST];
#pragma unroll
  for (int i = 0; i < MOST; ++i) bs[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < WO; ++i)
#pragma unroll
    for (int j = 0; j < WI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  // In the middle of slice t the codes of slice t + 1, which have had a slice's time to come, go into LDS, and slice t + 2's loads are issued
  // (three places for dy, two for x).  (Loads a slice ahead and the codes' turn at a slice's end: us, 1536 x 1024 over 32768 rows 129.)
  auto advance = [&](int t) {
    wait_vmcnt<0>();
    if (t + 1 < tiles) put_x(t + 1);
    if (t + 2 < tiles) {
      load_x(t + 2);
      stage_dy(t + 2);
    }
  };
  if (tiles > 0) {
    load_x(0);
    stage_dy(0);
    wait_vmcnt<0>();
    put_x(0);
    if (tiles > 1) {
      load_x(1);
      stage_dy(1);
    }
  }
  auto run = [&](auto sums) {                                                // sums: how many fragments of dy this wavefront adds up
    for (int t = 0; t < tiles; ++t) {
      __syncthreads();
      const unsigned char* A = smem + t % 3 * TO::kBytes;
      const unsigned char* X = smem + 3 * TO::kBytes + (t & 1) * TI::kBytes;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (s == 1) advance(t);
        frag xf[WI];
#pragma unroll
        for (int j = 0; j < WI; ++j) xf[j] = TI::col_frag(X, wi + j, s, lane);
        // x as the rows of the block, dy as its columns: a lane holds four adjacent entries of a row of dW
#pragma unroll
        for (int i = 0; i < WO; ++i) {
          const frag af = TO::col_frag(A, wo + i, s, lane);
#pragma unroll
          for (int j = 0; j < WI; ++j) acc[i][j] = mma(acc[i][j], xf[j], af);
        }
#pragma unroll
        for (int i = 0; i < decltype(sums)::value; ++i) bs[i] = mma(bs[i], ones, TO::col_frag(A, wo + slot + i * apart, s, lane));
      }
    }
  };
  const int mine = db && slot < WO ? (WO - 1 - slot) / apart + 1 : 0;
  if (mine == 0) run(std::integral_constant<int, 0>{});
  else if (MOST == 1 || mine == 1) run(std::integral_constant<int, 1>{});
  else run(std::integral_constant<int, MOST>{});
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    const int o = o0 + (wo + slot + i * apart) * 16 + l16;
    if (i >= mine || g != 0 || o >= d_out) continue;
    if (part) part[(size_t)splits * d_out * d_in + (size_t)sp * d_out + o] = bs[i][0];
    else db[o] = from_f32<T>(bs[i][0]);
  }
#pragma unroll
  for (int i = 0; i < WO; ++i) {
    const int o = o0 + (wo + i) * 16 + l16;
    if (o >= d_out) continue;
#pragma unroll
    for (int j = 0; j < WI; ++j) {
      const int c = i0 + (wi + j) * 16 + 4 * g;
      if (c >= d_in) continue;
      if (part) *reinterpret_cast<f32x4*>(part + ((size_t)sp * d_out + o) * d_in + c) = acc[i][j];
      else store4(dW + (size_t)o * d_in + c, acc[i][j]);
    }
  }
}

// Adds up the stretches' partial sums; a thread takes four entries.  n, m: entries of dW (a multiple of 8) and of db.
template <typename T>
__global__ __launch_bounds__(256) void k_grad_join(size_t n, int m, int splits, const float* __restrict__ part, T* __restrict__ dW, T* __restrict__ db) {
  const size_t e = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (e < n) {
    f32x4 sum = *reinterpret_cast<const f32x4*>(part + e);
    for (int s = 1; s < splits; ++s) sum += *reinterpret_cast<const f32x4*>(part + s * n + e);
    store4(dW + e, sum);
  } else if (db && e - n < (size_t)m) {
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < splits; ++s) sum += *reinterpret_cast<const f32x4*>(part + splits * n + (size_t)s * m + (e - n));
    store4(db + (e - n), sum);
  }
}

}  // namespace dchag
