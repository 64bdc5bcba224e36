// archead_rms_norm: the residual's addition, the root-mean-square norm of rows,
// and their rounding to 8 bits.
#include <cfloat>

#include "dev_codes.cuh"

namespace {

using namespace archead::rows;

constexpr int kNHeld = 2;            // groups of 8 elements a thread holds
constexpr int kNShort = 256;         // longest row that 16 lanes take
constexpr int64_t kNLongest = 16384;   // longest row of all: 1024 threads

struct NormArgs {
  const uint8_t* x;
  const uint8_t* r;        // may be null
  const uint8_t* w;
  uint8_t* total;          // may be null
  uint8_t* out;            // may be null
  int8_t* codes;           // may be null
  float* scales;
  int64_t M, d;
  int64_t x_row, r_row, t_row, o_row, ldc;   // bytes of the steps between rows
  double eps;
  float offset;
};

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// eight values rounded to their type, to any address
template <int DT>
__device__ __forceinline__ void store8(uint8_t* p, const float (&y)[8]) {
  f32x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = y[i];
  if constexpr (DT == ARCHEAD_F32) store_any(p, v);
  else if constexpr (DT == ARCHEAD_BF16) store_any(p, __builtin_convertvector(v, bf16x8));
  else store_any(p, __builtin_convertvector(v, f16x8));
}
// one element
template <int DT>
__device__ __forceinline__ float load1(const uint8_t* p) {
  if constexpr (DT == ARCHEAD_F32) return *reinterpret_cast<const float*>(p);
  else if constexpr (DT == ARCHEAD_BF16) return float(*reinterpret_cast<const __bf16*>(p));
  else return float(*reinterpret_cast<const _Float16*>(p));
}
template <int DT>
__device__ __forceinline__ void store1(uint8_t* p, float y) {
  if constexpr (DT == ARCHEAD_F32) *reinterpret_cast<float*>(p) = y;
  else if constexpr (DT == ARCHEAD_BF16) *reinterpret_cast<__bf16*>(p) = __bf16(y);
  else *reinterpret_cast<_Float16*>(p) = _Float16(y);
}

template <int CTRL>
__device__ __forceinline__ double dpp_f64(double v) {
  const uint64_t u = __double_as_longlong(v);
  return __longlong_as_double(int64_t(uint64_t(dpp<CTRL>(uint32_t(u >> 32))) << 32 | dpp<CTRL>(uint32_t(u))));
}
__device__ __forceinline__ double lane_f64(double v, int l) {
  const uint64_t u = __double_as_longlong(v);
  const uint32_t hi = __builtin_amdgcn_readlane(int(u >> 32), l), lo = __builtin_amdgcn_readlane(int(uint32_t(u)), l);
  return __longlong_as_double(int64_t(uint64_t(hi) << 32 | lo));
}

// s = x + r, t = s (offset + w), both rounded to fp32; 1 / sqrt(mean s^2 + eps)
// scales t in the end, so the codes are those of t, whatever the norm: a rounding
// of the norm never moves one.  SHORT: 16 lanes to a row, else a workgroup, as many
// threads as hold it in kNHeld groups of 8 elements each (and one of the up to seven
// elements behind the last whole group); a workgroup takes rows one after another
// and holds the weights.  The squares are summed in fp64: fp32 inputs may be so
// large (or so small) that they leave fp32.  A row's t stays in registers, so every
// element is read once and total may be where x or r are.  Bound by the bytes: 16384 x 8192
// bf16 with every output 218 us (5.5 TB/s), 4096 x 2560 to 16 bits 15 (5.6 TB/s).
template <int DT, bool W32, bool SHORT>
__global__ __launch_bounds__(SHORT ? 256 : kNLongest / 8 / kNHeld) void k_norm(NormArgs g) {
  using E = Eight<DT>;
  constexpr int WT = W32 ? int(ARCHEAD_F32) : DT, EB = E::kBytes, WB = Eight<WT>::kBytes, HELD = kNHeld;
  static_assert(!SHORT || HELD * 128 == kNShort, "a short row is held whole");
  const int TPR = SHORT ? 16 : int(blockDim.x), rows = SHORT ? int(blockDim.x) / 16 : 1;
  __shared__ uint32_t smax[2][kNLongest / 8 / HELD / 64];
  __shared__ double ssum[2][kNLongest / 8 / HELD / 64];
  const int tid = threadIdx.x, t = SHORT ? tid & 15 : tid;
  const int nd = int(g.d) & ~7;   // elements in whole groups; this thread's single one:
  const int one = nd + t < g.d ? nd + t : -1;
  auto at = [&](int h) { return (h * TPR + t) * 8; };
  float w[HELD][8], w1 = 0;
#pragma unroll
  for (int h = 0; h < HELD; ++h)
    if (at(h) < nd) {
      Eight<WT> e;
      e.load(g.w, at(h), INT64_MAX, 0);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[h][i] = g.offset + e.at(i);
    }
  if (one >= 0) w1 = g.offset + load1<WT>(g.w + int64_t(one) * WB);
  int turn = 0;
  for (int64_t m0 = int64_t(blockIdx.x) * rows; m0 < g.M; m0 += int64_t(gridDim.x) * rows, turn ^= 1) {
    const int64_t m = SHORT ? m0 + (tid >> 4) : m0;
    const bool live = m < g.M;
    const int n = live ? nd : 0;
    const uint8_t* const x = g.x + m * g.x_row;
    const uint8_t* const r = g.r + m * g.r_row;   // (not read where there is no residual)
    uint8_t* const total = g.total + m * g.t_row;
    const bool single = live && one >= 0;
    float v[HELD][8], v1 = 0;
    {
      E ex[HELD], er[HELD];
#pragma unroll
      for (int h = 0; h < HELD; ++h)
        if (at(h) < n) {
          ex[h].load(x, at(h), INT64_MAX, 0);
          if (g.r) er[h].load(r, at(h), INT64_MAX, 0);
        }
      if (single) {
        v1 = load1<DT>(x + one * EB);
        if (g.r) v1 += load1<DT>(r + one * EB);
      }
#pragma unroll
      for (int h = 0; h < HELD; ++h)
        if (at(h) < n) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[h][i] = ex[h].at(i);
          if (g.r) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[h][i] += er[h].at(i);
          }
        }
    }
    uint32_t top = 0;
    double sum = 0;
    auto take = [&](float& s, float weight) {
      sum = fma(double(s), double(s), sum);
      s *= weight;
      top = max(top, __float_as_uint(s) & 0x7fffffffu);
    };
#pragma unroll
    for (int h = 0; h < HELD; ++h)
      if (at(h) < n) {
        if (g.total) store8<DT>(total + at(h) * EB, v[h]);
#pragma unroll
        for (int i = 0; i < 8; ++i) take(v[h][i], w[h][i]);
      }
    if (single) {
      if (g.total) store1<DT>(total + one * EB, v1);
      take(v1, w1);
    }
    top = max(top, dpp<kDpp1>(top));
    top = max(top, dpp<kDpp2>(top));
    top = max(top, dpp<kDpp4>(top));
    top = max(top, dpp<kDpp8>(top));
    sum += dpp_f64<kDpp1>(sum);
    sum += dpp_f64<kDpp2>(sum);
    sum += dpp_f64<kDpp4>(sum);
    sum += dpp_f64<kDpp8>(sum);
    if constexpr (!SHORT) {
      auto of = [&](int l) { return uint32_t(__builtin_amdgcn_readlane(int(top), l)); };
      top = max(max(of(0), of(16)), max(of(32), of(48)));
      sum = (lane_f64(sum, 0) + lane_f64(sum, 16)) + (lane_f64(sum, 32) + lane_f64(sum, 48));
    }
    if (!SHORT && TPR > 64) {
      if ((tid & 63) == 0) {
        smax[turn][tid >> 6] = top;
        ssum[turn][tid >> 6] = sum;
      }
      __syncthreads();   // (the other of the two is read no more)
      sum = 0;
      for (int k = 0; k < TPR / 64; ++k) {
        top = max(top, smax[turn][k]);
        sum += ssum[turn][k];
      }
    }
    if (!live) continue;
    const bool finite = top < 0x7f800000u;
    const double rs = finite ? 1.0 / sqrt(sum / double(g.d) + g.eps) : double(NAN);
    if (g.out) {
      // where 1 / norm leaves fp32's normal numbers a power of two goes to t instead: t is at most
      // 2^7 norm times the weight, and above 2^156 (an eps below 2^-312) every x is 0
      const bool large = rs < 0x1p-100, small = rs > 0x1p100;
      const float pre = large ? 0x1p-40f : small ? 0x1p64f : 1.f;
      const float by = float(large ? rs * 0x1p40 : small ? fmin(rs * 0x1p-64, 0x1p120) : rs);
      uint8_t* const out = g.out + m * g.o_row;
#pragma unroll
      for (int h = 0; h < HELD; ++h) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = v[h][i] * pre * by;
        if (at(h) < nd) store8<DT>(out + at(h) * EB, y);
      }
      if (single) store1<DT>(out + one * EB, v1 * pre * by);
    }
    if (g.codes) {
      const float u = finite ? fmaxf(__uint_as_float(top) / 127.f, 0x1p-126f) : 1.f, inv = 1.f / u;
      int8_t* const codes = g.codes + m * g.ldc;
      if (t == 0) g.scales[m] = top ? float(double(u) * rs) : float(fmin(double(u) * rs, double(FLT_MAX)));
#pragma unroll
      for (int h = 0; h < HELD; ++h)
        if (at(h) < nd) store_any(codes + at(h), codes8(v[h], u, inv, finite));
      if (single) {
        const float alone[8] = {v1};
        codes[one] = int8_t(codes8(alone, u, inv, finite).x);
      }
    }
  }
}

template <int DT, bool W32, bool SHORT>
hipError_t launch_rows(const NormArgs& g, hipStream_t s) {
  const int64_t groups = SHORT ? (g.M + 15) / 16 : g.M, waves = SHORT ? 4 : (g.d + 512 * kNHeld - 1) / (512 * kNHeld);
  const int64_t most = 256 * (32 / waves > 0 ? 32 / waves : 1);   // workgroups that run at once, about
  return launch_kernel(k_norm<DT, W32, SHORT>, dim3(unsigned(groups < most ? groups : most)),
                       dim3(unsigned(64 * waves)), 0, s, g);
}

// Few waves with much in flight each gain nothing here (four groups a thread: 256 x 8192 bf16
// 6.3 us, two 5.4; 8192 x 16384 201 and 177; 65536 x 1024 fp32 159 and 164).  16 lanes to a row
// where they hold it as well (65536 rows of 128, 256: 15 and 23 us, a wave each 32 and 33; of 512
// with four groups a thread 4096 rows 7.0 us, a wave each 5.8).
template <int DT, bool W32>
hipError_t launch_norm(const NormArgs& g, hipStream_t s) {
  return g.d <= kNShort ? launch_rows<DT, W32, true>(g, s) : launch_rows<DT, W32, false>(g, s);
}

}  // namespace

extern "C" archead_status archead_rms_norm(const void* x, archead_dtype dtype, int64_t M, int64_t d, int64_t ldx,
                                           const void* residual, int64_t ldr, const void* weight,
                                           archead_dtype weight_dtype, float offset, double eps, void* total,
                                           int64_t ldt, void* out, int64_t ldo, int8_t* codes, int64_t ldc,
                                           float* scales, void* stream) {
  using archead::fail;
  archead::clear_error();
  if (!float_dtype(dtype)) return fail(ARCHEAD_E_INVALID_ARG, "dtype must be F32, BF16 or F16");
  if (weight_dtype != dtype && weight_dtype != ARCHEAD_F32)
    return fail(ARCHEAD_E_INVALID_ARG, "weight_dtype must be that of x or F32");
  if (M < 0 || M > INT32_MAX) return fail(ARCHEAD_E_INVALID_ARG, "M = %lld out of range", (long long)M);
  if (d < 1) return fail(ARCHEAD_E_INVALID_ARG, "d = %lld out of range", (long long)d);
  if (d > kNLongest) return fail(ARCHEAD_E_UNSUPPORTED, "d = %lld > %lld", (long long)d, (long long)kNLongest);
  if (!(eps > 0) || !(eps < INFINITY)) return fail(ARCHEAD_E_INVALID_ARG, "eps must be positive and finite");
  if (!(offset - offset == 0)) return fail(ARCHEAD_E_INVALID_ARG, "offset must be finite");
  if (M == 0) return ARCHEAD_OK;
  if (!x || !weight || (!out && !codes) || (codes && !scales)) return fail(ARCHEAD_E_INVALID_ARG, "null pointer");
  if (ldx < d || (residual && ldr < d) || (total && ldt < d) || (out && ldo < d) || (codes && ldc < d))
    return fail(ARCHEAD_E_INVALID_ARG, "leading dimensions must be >= d");
  // (in place each row only ever meets itself)
  const auto moved = [&](const void* o, int64_t ld) { return o && ((o == x && ld != ldx) || (o == residual && ld != ldr)); };
  if (moved(total, ldt) || moved(out, ldo)) return fail(ARCHEAD_E_INVALID_ARG, "in place, leading dimensions must agree");
  if (total && total == out) return fail(ARCHEAD_E_INVALID_ARG, "total and out must be two");
  const int eb = dtype_bytes(dtype);
  if (!aligned(x, eb) || !aligned(residual, eb) || !aligned(total, eb) || !aligned(out, eb) ||
      !aligned(weight, dtype_bytes(weight_dtype)) || !aligned(scales, 4))
    return fail(ARCHEAD_E_MISALIGNED, "a pointer is misaligned");
  const NormArgs g{static_cast<const uint8_t*>(x), static_cast<const uint8_t*>(residual), static_cast<const uint8_t*>(weight),
                   static_cast<uint8_t*>(total), static_cast<uint8_t*>(out), codes, scales, M, d,
                   ldx * eb, ldr * eb, ldt * eb, ldo * eb, ldc, eps, offset};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool w32 = weight_dtype == ARCHEAD_F32;
  const hipError_t e = dtype == ARCHEAD_F32    ? launch_norm<ARCHEAD_F32, true>(g, s)
                       : dtype == ARCHEAD_BF16 ? (w32 ? launch_norm<ARCHEAD_BF16, true>(g, s) : launch_norm<ARCHEAD_BF16, false>(g, s))
                                               : (w32 ? launch_norm<ARCHEAD_F16, true>(g, s) : launch_norm<ARCHEAD_F16, false>(g, s));
  return launch_status(e, "norm launch");
}
