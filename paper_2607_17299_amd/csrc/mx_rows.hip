// Rows into and out of microscaled codes (mx.h): the residual's addition with the RMS
// norm behind it, matrices as they are or behind a SwiGLU gate, and back.
//
// All of it is bound by memory for many rows and by a launch for few.  A lane takes
// eight neighbouring columns (16 bytes of bf16), so a block of 32 is four lanes and its
// maximum two exchanges within them.  Sums and statistics are fp32; a number is rounded
// once, to its code (bf16 output: to bf16).
#include "mx.h"

namespace {

typedef float f32x2_t __attribute__((ext_vector_type(2)));

// eight numbers at p (ONCE: non-temporal)
template <bool F32, bool ONCE = false>
WAR_DEV void load8(const void* p, int64_t at, float* x) {
  auto get = [&](int i) {
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const char*>(p) + at * (F32 ? 4 : 2)) + i;
    return ONCE ? load_once16(q) : *q;
  };
  if constexpr (F32) {
    const float4 a = __builtin_bit_cast(float4, get(0)), b = __builtin_bit_cast(float4, get(1));
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
    const uint4 a = get(0);
    x[0] = lo_f(a.x), x[1] = hi_f(a.x), x[2] = lo_f(a.y), x[3] = hi_f(a.y);
    x[4] = lo_f(a.z), x[5] = hi_f(a.z), x[6] = lo_f(a.w), x[7] = hi_f(a.w);
  }
}
template <bool F32>
WAR_DEV void store8(void* p, int64_t at, const float* x) {
  if constexpr (F32) {
    float* f = static_cast<float*>(p) + at;
    *reinterpret_cast<float4*>(f) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(f + 4) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    *reinterpret_cast<uint4*>(static_cast<bf16_t*>(p) + at) =
        make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
  }
}
template <int FMT>
WAR_DEV uint8_t* codes_at(const MxRef& m, int64_t r, int c8) {
  return m.codes + r * m.code_stride + (FMT == kMxE4M3 ? c8 * 8 : c8 * 4);
}

// h += x, y = h rsqrt(mean h^2 + eps) gain.  T threads a row (a wave's: four rows a
// workgroup), NV runs of eight columns each, kept in registers between the two passes, so
// that h is read and written once: memory bounds it, and for few rows the launch (2.4 us).
// 32768 x 4096, h in fp32, into e4m3: 270 us for 1.48 GB, 5.5 TB/s, where a plain copy of
// this card reaches 6.4.
template <int T, int NV, bool HF32, int OUT>
__global__ void __launch_bounds__(T < 256 ? 256 : T) k_residual_norm_mx(NormArgs a) {
  constexpr int RPW = T < 256 ? 256 / T : 1;
  __shared__ float red[16];
  const int t = threadIdx.x % T;
  const int64_t r = (int64_t)blockIdx.x * RPW + threadIdx.x / T;
  const int n8 = a.cols / 8;
  if (T < 256 && r >= a.rows) return;
  float h[NV][8];
  uint4 gg[NV];
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * T;
    if (c < n8) {
      gg[i] = *reinterpret_cast<const uint4*>(a.gain + c * 8);
      load8<HF32>(a.h, r * a.h_stride + c * 8, h[i]);
      if (a.x) {
        float x[8];
        load8<false>(a.x, r * a.x_stride + c * 8, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[i][e] += x[e];
        store8<HF32>(a.h, r * a.h_stride + c * 8, h[i]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += h[i][e] * h[i][e];
    }
  }
  if constexpr (T < 256) ss = wave_sum(ss);
  else ss = block_sum(ss, red);
  const float rs = 1.f / sqrtf(ss / (float)a.cols + a.eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = t + i * T;
    if (c < n8) {
      const float g[8] = {lo_f(gg[i].x), hi_f(gg[i].x), lo_f(gg[i].y), hi_f(gg[i].y),
                          lo_f(gg[i].z), hi_f(gg[i].z), lo_f(gg[i].w), hi_f(gg[i].w)};
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = h[i][e] * rs * g[e];
      if constexpr (OUT < 0) store8<false>(a.y, r * a.y_stride + c * 8, y);
      else mx_store8<OUT>(y, codes_at<OUT>(a.mx, r, c), a.mx.scales + r * a.mx.scale_stride + c / 4, c % 4 == 0);
    }
  }
}

// g / (1 + exp(-g)) to a few units of 2^-23: exp as a power of two, whose exponent's
// rounding is made up for to first order, and a reciprocal of the hardware's, of a quarter:
// 1 + exp(-g) reaches 2^128, and what is below 2^-126 comes out of the reciprocal as zero.
// (Arithmetic bounds the gate's kernel, with the library's exp and division by far.)
WAR_DEV float silu(float g) {
  constexpr float kLog2e = 1.44269502f, kLn2 = 0.693147182f;
  const float c = __builtin_amdgcn_fmed3f(g, -100.f, 128.f);  // past these: an infinite power, none
  const float t = c * -kLog2e, rest = fmaf(t, -kLn2, -c);      // exp(-c) = 2^t (1 + rest)
  return 0.25f * g * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_exp2f(t), fmaf(rest, 0.25f, 0.25f), 0.25f));
}

// row of run id < 2^31 of a matrix with `by` (rows_by) runs a row
WAR_DEV uint32_t row_of(uint32_t id, RowsBy by) { return __umulhi(id, by.magic) >> by.shift; }

// y = x, or x silu(gate), into codes: a lane a run of eight columns, four lanes a block,
// whose largest they find by two swaps.  Memory bounds it once the arithmetic is short
// (the row by a product in place of a division, silu's seven instructions) and what it
// reads does not push what others need out of the caches.  16384 x 12288 of bf16 with a
// gate into e2m1: 912 MB in 155 us, 5.9 TB/s; by ordinary loads 193 (4096 rows just written,
// which the last cache holds: 30.8 by ordinary ones, 31.9 so), and a lane with sixteen
// columns, whose loads leave out every other 16 bytes, 178.
template <bool F32, bool GATE, int FMT>
__global__ void __launch_bounds__(256) k_quantize(QuantArgs a) {
  const uint32_t id = blockIdx.x * 256 + threadIdx.x, n8 = a.cols / 8;  // (at most 2^31 runs)
  if (id >= (uint32_t)a.rows * n8) return;
  const uint32_t row = row_of(id, a.by);
  const int64_t r = row;
  const int c = (int)(id - row * n8);
  float y[8];
  load8<F32, true>(a.x, r * a.x_stride + c * 8, y);
  if constexpr (GATE) {
    float g[8];
    load8<F32, true>(a.gate, r * a.gate_stride + c * 8, g);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] *= silu(g[e]);
  }
  mx_store8<FMT>(y, codes_at<FMT>(a.mx, r, c), a.mx.scales + r * a.mx.scale_stride + c / 4, c % 4 == 0);
}

WAR_DEV void from_e4m3x4(uint32_t w, float* y) {
  y[0] = from_e4m3<0>(w, 1.f), y[1] = from_e4m3<1>(w, 1.f), y[2] = from_e4m3<2>(w, 1.f), y[3] = from_e4m3<3>(w, 1.f);
}
WAR_DEV void from_e2m1x8(uint32_t w, float* y) {
  const f32x2_t v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1);
  const f32x2_t v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3);
  y[0] = v0[0], y[1] = v0[1], y[2] = v1[0], y[3] = v1[1], y[4] = v2[0], y[5] = v2[1], y[6] = v3[0], y[7] = v3[1];
}

// the numbers that codes stand for, sixteen a lane.  16384 x 12288 of e2m1 into bf16: 85 us
// for 510 MB, 6.0 TB/s (eight a lane 92, the numbers put together from the codes' bits 135).
template <bool F32, int FMT>
__global__ void __launch_bounds__(256) k_dequantize(DequantArgs a) {
  const uint32_t id = blockIdx.x * 256 + threadIdx.x, n16 = a.cols / 16;
  if (id >= (uint32_t)a.rows * n16) return;
  const uint32_t row = row_of(id, a.by);
  const int64_t r = row;
  const int c = (int)(id - row * n16);
  const float s = mx_scale(a.mx.scales[r * a.mx.scale_stride + c / 2]);
  const uint8_t* p = codes_at<FMT>(a.mx, r, 2 * c);
  float y[16];
  if constexpr (FMT == kMxE4M3) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    from_e4m3x4(w.x, y), from_e4m3x4(w.y, y + 4), from_e4m3x4(w.z, y + 8), from_e4m3x4(w.w, y + 12);
  } else {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    from_e2m1x8(w.x, y), from_e2m1x8(w.y, y + 8);
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) y[e] *= s;
  store8<F32>(a.y, r * a.y_stride + c * 16, y);
  store8<F32>(a.y, r * a.y_stride + c * 16 + 8, y + 8);
}

template <bool HF32, int OUT>
void norm_go(const NormArgs& a, hipStream_t st) {
  const int n8 = a.cols / 8;
  auto one = [&](auto t, auto nv) {
    constexpr int T = decltype(t)::value, NV = decltype(nv)::value;
    const int grid = T < 256 ? (a.rows + 256 / T - 1) / (256 / T) : a.rows;
    k_residual_norm_mx<T, NV, HF32, OUT><<<grid, T < 256 ? 256 : T, 0, st>>>(a);
  };
  using std::integral_constant;
  if (n8 <= 64) one(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (n8 <= 256) one(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (n8 <= 512) one(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (n8 <= 1024) one(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  else if (n8 <= 2048) one(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
  else if (n8 <= 4096) one(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
  else one(integral_constant<int, 1024>{}, integral_constant<int, 8>{});
}

// id / n is (id magic >> 32) >> shift for id < 2^31, n >= 2: magic is 2^(31 + l) / n
// rounded up, 2^l >= n, which is off by less than id / 2^(31 + l) < 1 / n.
RowsBy rows_by(int n) {
  int l = 1;
  while ((1 << l) < n) ++l;
  return {(uint32_t)((((uint64_t)1 << (31 + l)) + n - 1) / n), l - 1};
}

}  // namespace

void launch_residual_norm_mx(const NormArgs& a, bool h_f32, int out, hipStream_t st) {
  if (h_f32) {
    if (out < 0) norm_go<true, -1>(a, st);
    else if (out == kMxE4M3) norm_go<true, kMxE4M3>(a, st);
    else norm_go<true, kMxE2M1>(a, st);
  } else {
    if (out < 0) norm_go<false, -1>(a, st);
    else if (out == kMxE4M3) norm_go<false, kMxE4M3>(a, st);
    else norm_go<false, kMxE2M1>(a, st);
  }
}

void launch_quantize(QuantArgs a, bool f32, int fmt, hipStream_t st) {
  const int64_t n = (int64_t)a.rows * (a.cols / 8);
  a.by = rows_by(a.cols / 8);
  const int grid = (int)((n + 255) / 256);
  auto go = [&](auto f, auto g) {
    constexpr bool F = decltype(f)::value, G = decltype(g)::value;
    if (fmt == kMxE4M3) k_quantize<F, G, kMxE4M3><<<grid, 256, 0, st>>>(a);
    else k_quantize<F, G, kMxE2M1><<<grid, 256, 0, st>>>(a);
  };
  if (f32) {
    if (a.gate) go(std::true_type{}, std::true_type{});
    else go(std::true_type{}, std::false_type{});
  } else {
    if (a.gate) go(std::false_type{}, std::true_type{});
    else go(std::false_type{}, std::false_type{});
  }
}

void launch_dequantize(DequantArgs a, bool f32, int fmt, hipStream_t st) {
  const int64_t n = (int64_t)a.rows * (a.cols / 16);
  a.by = rows_by(a.cols / 16);
  const int grid = (int)((n + 255) / 256);
  if (f32) {
    if (fmt == kMxE4M3) k_dequantize<true, kMxE4M3><<<grid, 256, 0, st>>>(a);
    else k_dequantize<true, kMxE2M1><<<grid, 256, 0, st>>>(a);
  } else {
    if (fmt == kMxE4M3) k_dequantize<false, kMxE4M3><<<grid, 256, 0, st>>>(a);
    else k_dequantize<false, kMxE2M1><<<grid, 256, 0, st>>>(a);
  }
}
