// archead_matmul_i8: arguments of its kernels and their outputs.
//
// v_mfma_i32_16x16x64_i8 (32x32x32): lane l holds 16 consecutive k of row l % 16
// (l % 32) of an operand, from 16 (l / 16) (16 (l / 32)) on; of the result
// column l % 16 (l % 32) of the second operand, and of the first operand rows
// 4 (l / 16) + i (8 (i / 4) + 4 (l / 32) + i % 4).  The channels (b) go first, so
// a lane's results come as four neighbouring channels of one token.
#pragma once

#include "dev_rows.cuh"

namespace archead {
namespace i8 {

using namespace archead::rows;

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct I8Args {
  const int8_t* a;
  const int8_t* b;
  const float* sa;
  const float* sb;
  const float* bias;   // may be null
  uint8_t* out;
  int64_t lda, ldb, ldo;
  int64_t M, N;
  int K;
};

// an output before its last rounding (bias 0 where there is none)
__device__ __forceinline__ float scaled(int acc, float sa, float sb, float bias) {
  return fmaf(float(acc) * sa, sb, bias);
}

// four fp32 values to the output's type, at p
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4v __attribute__((ext_vector_type(4)));
template <int DT>
__device__ __forceinline__ void put4(uint8_t* p, const float (&y)[4]) {
  const f32x4v v{y[0], y[1], y[2], y[3]};
  if constexpr (DT == ARCHEAD_F32) *reinterpret_cast<f32x4v*>(p) = v;
  else if constexpr (DT == ARCHEAD_BF16) *reinterpret_cast<bf16x4*>(p) = __builtin_convertvector(v, bf16x4);
  else *reinterpret_cast<f16x4*>(p) = __builtin_convertvector(v, f16x4);
}

// the first `left` (at least all that fit) elements of EB bytes of v, at any address
template <int EB, typename V>
__device__ __forceinline__ void store_part(uint8_t* p, const V& v, int64_t left) {
  constexpr int PER = sizeof(V) / EB;
  if (left >= PER) {
    store_any(p, v);
    return;
  }
  uint32_t w[sizeof(V) / 4];
  __builtin_memcpy(w, &v, sizeof(V));
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (i >= left) continue;
    if constexpr (EB == 4) *reinterpret_cast<uint32_t*>(p + 4 * i) = w[i];
    else *reinterpret_cast<uint16_t*>(p + 2 * i) = uint16_t(w[i / 2] >> (16 * (i & 1)));
  }
}

// the outputs of channels n .. n + 3 of token m
template <int DT>
__device__ __forceinline__ void finish4(const I8Args& g, int64_t m, int64_t n, const i32x4& acc) {
  if (m >= g.M || n >= g.N) return;
  constexpr int EB = DT == ARCHEAD_F32 ? 4 : 2;
  const float s = g.sa[m];
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t c = n + i < g.N ? n + i : n;
    y[i] = scaled(acc[i], s, g.sb[c], g.bias ? g.bias[c] : 0.f);
  }
  alignas(16) uint32_t w[EB];
  put4<DT>(reinterpret_cast<uint8_t*>(w), y);
  if constexpr (EB == 4) store_part<EB>(g.out + (m * g.ldo + n) * EB, uint4{w[0], w[1], w[2], w[3]}, g.N - n);
  else store_part<EB>(g.out + (m * g.ldo + n) * EB, uint2{w[0], w[1]}, g.N - n);
}

// bytes k .. k + 15 of a row of K (k < K) at any address, zeros past K
__device__ __forceinline__ uint4 row_piece(const int8_t* row, int k, int K) {
  if (__builtin_expect(K < 16, 0)) {
    uint32_t d[4] = {};
    for (int j = 0; j < K; ++j) d[j / 4] |= uint32_t(uint8_t(row[j])) << (8 * (j % 4));
    return uint4{d[0], d[1], d[2], d[3]};
  }
  // the row's last 16 bytes, moved down, where fewer are left
  const int over = max(k + 16 - K, 0);
  uint4 w = load_any<uint4>(row + k - over);
  if (over) {
    uint64_t lo = uint64_t(w.y) << 32 | w.x, hi = uint64_t(w.w) << 32 | w.z;
    const int bits = 8 * over;
    lo = bits < 64 ? lo >> bits | hi << (64 - bits) : hi >> (bits - 64);
    hi = bits < 64 ? hi >> bits : 0;
    w = uint4{uint32_t(lo), uint32_t(lo >> 32), uint32_t(hi), uint32_t(hi >> 32)};
  }
  return w;
}

// LDS accesses of one wave stay in this order (the hardware keeps it; lanes
// read what other lanes wrote, which the compiler does not see).
__device__ __forceinline__ void wave_lds_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

constexpr int64_t kMaxLd = 1 << 22;   // a tile's rows stay within 31-bit offsets

// What the kernels below need, but for launch_loose's: 16-byte pieces that lie
// whole in a row and in aligned memory.
inline bool pieces(const I8Args& g) {
  return aligned(g.a, 16) && aligned(g.b, 16) && g.K % 16 == 0 && g.lda % 16 == 0 && g.ldb % 16 == 0;
}
// kernel launchers, one translation unit each; *_take: whether the call's sizes fit
bool few_take(const I8Args& g);
template <int DT>
hipError_t launch_few(const I8Args& g, int n_cu, hipStream_t s);
bool split_take(const I8Args& g);
template <int DT>   // in tiles of 16 f x 16 f, f = 1 or 2
hipError_t launch_split(const I8Args& g, int f, hipStream_t s);
template <int DT>   // as launch_split, rows at any byte
hipError_t launch_loose(const I8Args& g, int f, int n_cu, hipStream_t s);
bool tiles_take(const I8Args& g);
template <int DT>   // in tiles of tm x 256, tm = 64, 128, 192 or 256
hipError_t launch_tiles(const I8Args& g, int tm, int n_cu, hipStream_t s);

}  // namespace i8
}  // namespace archead
