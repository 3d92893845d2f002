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
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = a[j];
    v[4 + j] = b[j];
  }
}
__device__ __forceinline__ void load8(const bf16* p, float (&v)[8]) {
  const bf16x8 a = *reinterpret_cast<const bf16x8*>(p);
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

// HBM-bound.  Four threads share a block of 32 values, eight each: a wavefront reads 16 blocks one behind the other.
template <typename T>
__global__ __launch_bounds__(256) void k_pack8(long rows, int D, long ld, const T* __restrict__ x, unsigned char* __restrict__ codes,
                                               unsigned char* __restrict__ scales) {
  const int blocks = (D + 31) / 32;
  const long id = (long)blockIdx.x * 256 + threadIdx.x;
  const long row = (id >> 2) / blocks;
  const int blk = (int)((id >> 2) - row * blocks), e = blk * 32 + (int)(id & 3) * 8;
  const bool in = row < rows && e < D;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (in) load8(x + row * ld + e, v);
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float m = fabsf(v[j]);
    if (m <= -kLowest) top = fmaxf(top, m);
    else v[j] = __builtin_nanf("");
  }
  top = fmaxf(top, dpp_move<kDppSwapPairs>(top));
  top = fmaxf(top, dpp_move<kDppSwapHalves>(top));
  const unsigned bits = __builtin_bit_cast(unsigned, top);
  const int byte = max((int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), 0);
  if (!in) return;
  const float sc = unscale_of(byte);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= sc;
  if (byte == 247)                                                           // 256 * 2^120 is no number of T
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (fabsf(v[j]) > 240.f) v[j] = copysignf(240.f, v[j]);
  int w0 = 0, w1 = 0;
  w0 = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], w0, false);
  w0 = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w0, true);
  w1 = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], w1, false);
  w1 = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], w1, true);
  *reinterpret_cast<uint2*>(codes + row * D + e) = make_uint2(w0, w1);
  if ((id & 3) == 0) scales[row * blocks + blk] = (unsigned char)byte;
}

template <typename T>
__global__ __launch_bounds__(256) void k_unpack8(long rows, int D, long ld, const unsigned char* __restrict__ codes,
                                                 const unsigned char* __restrict__ scales, T* __restrict__ x) {
  const int blocks = (D + 31) / 32;
  const long id = (long)blockIdx.x * 256 + threadIdx.x;
  const long row = (id >> 2) / blocks;
  const int blk = (int)((id >> 2) - row * blocks), e = blk * 32 + (int)(id & 3) * 8;
  if (row >= rows || e >= D) return;
  float v[8];
  decode8(*reinterpret_cast<const uint2*>(codes + row * D + e), scale_of(scales[row * blocks + blk]), v);
  store8(x + row * ld + e, v);
}

// dW[o][i] = sum over rows of dy[row][o] x[row][i], db[o] = sum of dy[row][o], x held in 8 bits.  MFMA-bound for long inputs.
// Workgroup: 128 x 128 of dW over one stretch of the rows, four wavefronts of 64 x 64; slices of 64 rows of both operands lie in LDS as they
// lie in memory (both have the sum's index as their row) and are read transposed.  dy comes by direct-to-LDS loads; of x a
// thread takes one block of 32 codes, which it turns into numbers of T once for all that read them: every e4m3 value times a power of
// two is a bf16 number (below 2^-126 it is rounded).  Stretches beyond one leave partial sums that k_grad_join adds up in their order.
template <typename T>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void k_weight_grad8(int rows, int d_out, int d_in, long ld, int stretch,
                                                          const T* __restrict__ dy, const unsigned char* __restrict__ codes,
                                                          const unsigned char* __restrict__ scales, T* __restrict__ dW, T* __restrict__ db,
                                                          float* __restrict__ part) {
  typedef Tile<T, 128> TL;
  typedef typename Frag<T>::type frag;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g = lane >> 4;
  const int ni = (d_in + 127) / 128, no = (d_out + 127) / 128;
  const int it = blockIdx.x % ni, ot = blockIdx.x / ni % no, sp = blockIdx.x / ni / no;
  const int o0 = ot * 128, i0 = it * 128, r0 = sp * stretch, r1 = min(rows, r0 + stretch);
  const int wo = (wave >> 1) * 64, wi = (wave & 1) * 64, blocks = (d_in + 31) / 32;
  const int tiles = (r1 - r0 + 63) / 64;
  const int xrow = tid >> 2, xblk = tid & 3, xe = i0 + xblk * 32;            // this thread's block of a slice
  uint2 cw[4];
  unsigned sc = 0;
  auto load_x = [&](int t) {
    const int r = r0 + t * 64 + xrow;
    const bool in = r < r1 && xe < d_in;
    sc = in ? scales[(size_t)r * blocks + xe / 32] : 0;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      cw[c] = in && xe + c * 8 < d_in ? *reinterpret_cast<const uint2*>(codes + (size_t)r * d_in + xe + c * 8) : make_uint2(0, 0);
  };
  auto put_x = [&](int t) {
    unsigned char* to = smem + (t & 1) * 2 * TL::kBytes + TL::kBytes + xrow * TL::kPitch;
    const float s = scale_of(sc);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float v[8];
      decode8(cw[c], s, v);
      if constexpr (sizeof(T) == 2) {
        store8(reinterpret_cast<bf16*>(to + ((xblk * 4 + c) ^ TL::swz(xrow)) * 16), v);
      } else {
        *reinterpret_cast<f32x4*>(to + ((xblk * 8 + 2 * c) ^ TL::swz(xrow)) * 16) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4*>(to + ((xblk * 8 + 2 * c + 1) ^ TL::swz(xrow)) * 16) = f32x4{v[4], v[5], v[6], v[7]};
      }
    }
  };
  auto stage_dy = [&](int t) {
    TL::template stage<64, 256>(dy + (long)(r0 + t * 64) * ld + o0, ld, r1 - r0 - t * 64, min(128, d_out - o0), smem + (t & 1) * 2 * TL::kBytes, tid);
  };
  const bool sums = it == 0 && (wave & 1) == 0;                              // these wavefronts also add up dy
  frag ones;
#pragma unroll
  for (int j = 0; j < 8; ++j) ones[j] = (T)1.f;
  f32x4 acc[4][4], bs[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    bs[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (tiles > 0) {
    load_x(0);
    stage_dy(0);
    put_x(0);
  }
  for (int t = 0; t < tiles; ++t) {
    wait_vmcnt<0>();
    __syncthreads();
    if (t + 1 < tiles) {
      stage_dy(t + 1);
      load_x(t + 1);
    }
    const unsigned char* A = smem + (t & 1) * 2 * TL::kBytes;
    const unsigned char* X = A + TL::kBytes;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      frag xf[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) xf[j] = TL::col_frag(X, wi / 16 + j, s, lane);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const frag af = TL::col_frag(A, wo / 16 + i, s, lane);
        // x as the rows of the block, dy as its columns: a lane holds four adjacent entries of a row of dW
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = mma(acc[i][j], xf[j], af);
        if (sums) bs[i] = mma(bs[i], ones, af);
      }
    }
    if (t + 1 < tiles) put_x(t + 1);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int o = o0 + wo + i * 16 + l16;
    if (o >= d_out) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = i0 + wi + j * 16 + 4 * g;
      if (c >= d_in) continue;
      if (part) *reinterpret_cast<f32x4*>(part + ((size_t)sp * d_out + o) * d_in + c) = acc[i][j];
      else store4(dW + (size_t)o * d_in + c, acc[i][j]);
    }
    if (sums && g == 0 && db) {
      if (part) part[(size_t)gridDim.x / ni / no * d_out * d_in + (size_t)sp * d_out + o] = bs[i][0];
      else db[o] = from_f32<T>(bs[i][0]);
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
