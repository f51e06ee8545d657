// y = x w^T of microscaled numbers (mx.h): weights in e2m1, activations in e4m3 or e2m1,
// fp32 sums in the scaled matrix instructions (v_mfma_scale_f32_16x16x128_f8f6f4).
//
// The weights are the instruction's first operand, so a lane's four results are four
// neighbouring columns of one row of y.  Lane l holds, of row l % 16, the 32 e2m1 numbers
// k = 32 (l / 16) .., or the 32 e4m3 numbers 16 (l / 16) .. + 15 and 64 + 16 (l / 16) ..
// + 15; the scale of row l % 16 and block l / 16 is a byte of lane l's in both.  A block's
// scale byte 255 makes NaN.  The instruction sums e4m3 products in groups of eight
// neighbours in which what lies more than 13 binary places below the largest is cut off;
// the numbers themselves carry four.  (e2m1 products span fewer places: exact.)
//
// Packed weights: 1 KB fragments of 16 rows by 128 columns, 16 bytes a lane as above, the
// fragments of a row tile one after the other; and a word a lane for four of them with
// their scale bytes.  Padded with zero codes to 256 rows and 512 columns.
#include <type_traits>

#include "mx.h"

namespace {

// grid (tile, group of 512 columns), 256 threads: fragment threadIdx / 64
__global__ void __launch_bounds__(256) k_mx_pack(MxRef w, int N, int K, int groups, uint8_t* codes, uint32_t* scales) {
  const int tile = blockIdx.x, grp = blockIdx.y, l = threadIdx.x & 63, j = threadIdx.x >> 6;
  const int row = tile * 16 + (l & 15), k = grp * 512 + j * 128 + (l >> 4) * 32;
  uint4 c = make_uint4(0, 0, 0, 0);
  if (row < N && k < K) {
    const uint8_t* p = w.codes + (int64_t)row * w.code_stride + k / 2;  // (a row may begin at any byte)
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      b[i] = 0;
      for (int q = 0; q < 4; ++q) b[i] |= (uint32_t)p[i * 4 + q] << (8 * q);
    }
    c = make_uint4(b[0], b[1], b[2], b[3]);
  }
  *reinterpret_cast<uint4*>(codes + ((int64_t)(tile * (int64_t)groups + grp) * 4 + j) * 1024 + l * 16) = c;
  if (j == 0) {
    uint32_t s = 0;
    for (int i = 0; i < 4; ++i) {
      const int kk = grp * 512 + i * 128 + (l >> 4) * 32;
      const uint32_t byte = row < N && kk < K ? w.scales[(int64_t)row * w.scale_stride + kk / 32] : 127u;
      s |= byte << (8 * i);
    }
    scales[(tile * (int64_t)groups + grp) * 64 + l] = s;
  }
}

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(4), may_alias));

// One product of fragments; J: which byte of the weights' scale word
template <int XF, int J>
WAR_DEV f32x4 mx_mfma(i32x8 w, i32x8 x, f32x4 c, uint32_t sw, uint32_t sx) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 4, XF == kMxE4M3 ? 0 : 4, J, (int)sw, 0, (int)sx);
}

// Four results y[m][n .. n + 3]
template <bool F32>
WAR_DEV void store_y(const MxGemmArgs& a, int m, int n, f32x4 v) {
  if (m >= a.M || n >= a.N) return;
  const uint2 bb = *reinterpret_cast<const uint2*>(a.bias + n);
  v[0] += lo_f(bb.x), v[1] += hi_f(bb.x), v[2] += lo_f(bb.y), v[3] += hi_f(bb.y);
  const int64_t at = (int64_t)m * a.y_stride + n;
  if constexpr (F32) {
    float* y = static_cast<float*>(a.y) + at;
    if (a.vec && n + 4 <= a.N) *reinterpret_cast<f32x4*>(y) = v;
    else
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < a.N) y[i] = v[i];
  } else {
    bf16_t* y = static_cast<bf16_t*>(a.y) + at;
    if (a.vec && n + 4 <= a.N) *reinterpret_cast<uint2*>(y) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
    else
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n + i < a.N) y[i] = f2bf(v[i]);
  }
}

// Few rows: the weights' way from memory bounds it.  A workgroup takes 16 NT columns by
// 16 MT rows; its waves share the groups of 512 k between them, every fragment straight
// from memory to registers, and their sums meet in LDS in the waves' order.
template <int MT, int NT, int WAVES, int XF, bool F32>
__global__ void __launch_bounds__(WAVES * 64) k_mx_skinny(MxGemmArgs a) {
  constexpr int XB = XF == kMxE4M3 ? 128 : 64;  // bytes of a row's k-step
  __shared__ f32x4 s_sum[WAVES][MT * NT][64];
  const int lane = threadIdx.x & 63, ln = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nt0 = blockIdx.x * NT, m0 = blockIdx.y * 16 * MT;
  const int groups = (a.K + 511) / 512;
  f32x4 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint8_t *xc[MT], *xs[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {  // rows past the last read the last one, and are not written
    const int64_t r = min(m0 + m * 16 + ln, a.M - 1);
    xc[m] = a.x.codes + r * a.x.code_stride;
    xs[m] = a.x.scales + r * a.x.scale_stride;
  }
  for (int g = wave; g < groups; g += WAVES) {
    const int k0 = g * 512;
    const bool whole = k0 + 512 <= a.K;
    uint32_t sw[NT];
    uint4 w[4][NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int64_t f = (int64_t)(nt0 + n) * groups + g;
      sw[n] = a.ws[f * 64 + lane];
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j][n] = *reinterpret_cast<const uint4*>(a.w + (f * 4 + j) * 1024 + lane * 16);
    }
    uint32_t sx[MT][4];
    uint4 x[4][MT][XF == kMxE4M3 ? 2 : 1];
    if (whole) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const u32x4_any s = *reinterpret_cast<const u32x4_any*>(xs[m] + g * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sx[m][j] = s[j];
          const uint8_t* p = xc[m] + (int64_t)(g * 4 + j) * XB + lg * 16;
          x[j][m][0] = *reinterpret_cast<const uint4*>(p);
          if constexpr (XF == kMxE4M3) x[j][m][1] = *reinterpret_cast<const uint4*>(p + 64);
        }
      }
    } else {
      // 16-byte pieces hold numbers of one block: zero codes where it lies past K
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int kj = k0 + j * 128;
          sx[m][j] = kj < a.K ? *reinterpret_cast<const uint32_t*>(xs[m] + kj / 32) : 0x7f7f7f7fu;
          if (kj + lg * 32 >= a.K) sx[m][j] = 0x7f7f7f7fu;
          const uint4 zero = make_uint4(0, 0, 0, 0);
          const uint8_t* p = xc[m] + (int64_t)(g * 4 + j) * XB + lg * 16;
          x[j][m][0] = kj + (XF == kMxE4M3 ? lg * 16 : lg * 32) < a.K ? *reinterpret_cast<const uint4*>(p) : zero;
          if constexpr (XF == kMxE4M3) x[j][m][1] = kj + 64 + lg * 16 < a.K ? *reinterpret_cast<const uint4*>(p + 64) : zero;
        }
    }
    auto step = [&](auto tag) __attribute__((always_inline)) {
      constexpr int J = decltype(tag)::value;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const uint4 lo = x[J][m][0];
        i32x8 xv = {(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, 0, 0, 0, 0};
        if constexpr (XF == kMxE4M3) {
          const uint4 hi = x[J][m][1];
          xv[4] = (int)hi.x, xv[5] = (int)hi.y, xv[6] = (int)hi.z, xv[7] = (int)hi.w;
        }
        const uint32_t s = sx[m][J] >> (8 * lg);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint4 c = w[J][n];
          acc[m][n] = mx_mfma<XF, J>(i32x8{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0}, xv, acc[m][n], sw[n], s);
        }
      }
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) s_sum[wave][m * NT + n][lane] = acc[m][n];
  __syncthreads();
  for (int t = wave; t < MT * NT; t += WAVES) {
    f32x4 v = s_sum[0][t][lane];
    for (int w = 1; w < WAVES; ++w) v += s_sum[w][t][lane];
    store_y<F32>(a, m0 + (t / NT) * 16 + ln, (nt0 + t % NT) * 16 + lg * 4, v);
  }
}

template <int MT, int NT, int WAVES>
void skinny(const MxGemmArgs& a, int fmt, bool f32, hipStream_t st) {
  const dim3 grid((a.N + 16 * NT - 1) / (16 * NT), (a.M + 16 * MT - 1) / (16 * MT));
  if (fmt == kMxE4M3) {
    if (f32) k_mx_skinny<MT, NT, WAVES, kMxE4M3, true><<<grid, WAVES * 64, 0, st>>>(a);
    else k_mx_skinny<MT, NT, WAVES, kMxE4M3, false><<<grid, WAVES * 64, 0, st>>>(a);
  } else {
    if (f32) k_mx_skinny<MT, NT, WAVES, kMxE2M1, true><<<grid, WAVES * 64, 0, st>>>(a);
    else k_mx_skinny<MT, NT, WAVES, kMxE2M1, false><<<grid, WAVES * 64, 0, st>>>(a);
  }
}

}  // namespace

void launch_mx_pack(const MxRef& w, int N, int K, uint8_t* codes, uint32_t* scales, hipStream_t st) {
  k_mx_pack<<<dim3(mx_tiles(N), mx_groups(K)), 256, 0, st>>>(w, N, K, mx_groups(K), codes, scales);
}

void launch_mx_gemm(const MxGemmArgs& a, int fmt, bool f32, hipStream_t st) {
  if (a.M <= 16) skinny<1, 1, 8>(a, fmt, f32, st);
  else skinny<2, 2, 8>(a, fmt, f32, st);
}
