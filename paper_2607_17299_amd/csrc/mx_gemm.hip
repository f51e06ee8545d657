// y = x w^T of microscaled numbers (mx.h): weights in e2m1, activations in e4m3 or e2m1,
// fp32 sums in the scaled matrix instructions
// (v_mfma_scale_f32_32x32x64_f8f6f4 for many rows, 16x16x128 for few).
//
// The weights are the instruction's first operand, so four neighbouring results of a lane
// are neighbouring columns of one row of y.  A lane holds 32 numbers of a row: lane group
// g (64 or 128 columns in two or four groups) the e2m1 numbers k = 32 g .., or the e4m3
// numbers k = 16 g .. + 15 and as many from half the columns on; the scale of a row's block
// b is a byte of lane group b's in both.  A block's scale byte 255 makes NaN.  The
// instruction sums e4m3 products in groups of eight neighbours, each cut (towards zero) at
// 13 binary places below the group's largest power of two: the sum of the two numbers'
// exponents, not the product's own, where e2m1's 0.5 has the exponent 0 and zeros none.
// (e2m1 products reach from 2^-2 to 36, powers of 2^4 at most: exact.)  Where y is fp32 the
// codes go in two parts, for twice the instructions: from 2 on, powers of 2^10 at most, whose
// last bit is 2^-3, and below 2, of 2^2 at most, whose last bit is 2^-10.  So neither part
// loses a bit.  (For a bf16 y the cut, at most 7 x 2^-13 of that power for a group, is left
// in, and the products cost half.  Next to a y as large as the group's product it is less
// than half of what rounding y to bf16 takes; of a y that cancels to little it may be all,
// though less than the 2^-4 of each number that rounding them to e4m3 took.)
//
// Packed weights: 1 KB fragments of 32 rows by 64 columns, 16 bytes a lane of the 32x32x64
// instruction, the fragments of a row tile one after the other; and for four of them a
// word a lane with their scale bytes.  Padded with zero codes to 256 rows and 512 columns.
#include <type_traits>

#include "lds_load.h"
#include "mx.h"

namespace {

// grid (tile of 32 rows, group of 512 columns), 512 threads: fragment threadIdx / 64
__global__ void __launch_bounds__(512) k_mx_pack(MxRef w, int N, int K, int groups, uint8_t* codes, uint32_t* scales) {
  const int tile = blockIdx.x, grp = blockIdx.y, l = threadIdx.x & 63, j = threadIdx.x >> 6;
  const int row = tile * 32 + (l & 31), k = grp * 512 + j * 64 + (l >> 5) * 32;
  uint32_t c[4] = {0, 0, 0, 0};
  if (row < N && k < K) {
    const uint8_t* p = w.codes + (int64_t)row * w.code_stride + k / 2;  // (a row may begin at any byte)
#pragma unroll
    for (int i = 0; i < 16; ++i) c[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
  }
  const int64_t at = (int64_t)tile * groups + grp;
  *reinterpret_cast<uint4*>(codes + (at * 8 + j) * 1024 + l * 16) = make_uint4(c[0], c[1], c[2], c[3]);
  if (j < 2) {
    uint32_t s = 0;
    for (int i = 0; i < 4; ++i) {
      const int kk = grp * 512 + (j * 4 + i) * 64 + (l >> 5) * 32;
      s |= (row < N && kk < K ? w.scales[(int64_t)row * w.scale_stride + kk / 32] : 127u) << (8 * i);
    }
    scales[(at * 2 + j) * 64 + l] = s;
  }
}

// (vector types of memory that may begin at any word, or any bf16)
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(4), may_alias));
typedef uint32_t u32x2_half __attribute__((ext_vector_type(2), aligned(2), may_alias));
typedef uint32_t u32x4_half __attribute__((ext_vector_type(4), aligned(2), may_alias));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4), may_alias));

constexpr int GM = 4;  // row blocks of a band (k_mx_tile)

typedef float f32x16 __attribute__((ext_vector_type(16)));

// One product of fragments; J: which byte of the weights' scale word, I: of x's
template <int XF, int J>
WAR_DEV f32x4 mx_mfma(i32x8 w, i32x8 x, f32x4 c, uint32_t sw, uint32_t sx) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 4, XF == kMxE4M3 ? 0 : 4, J, (int)sw, 0, (int)sx);
}
template <int XF, int I>
WAR_DEV f32x16 mx_mfma32(i32x8 w, i32x8 x, f32x16 c, uint32_t sw, uint32_t sx) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, c, 4, XF == kMxE4M3 ? 0 : 4, 0, (int)sw, I, (int)sx);
}

// e4m3 codes of 2 and more (bit 6 of the code), and the others: products of either part
// with e2m1 numbers span so few places that the instruction adds them without a cut.
WAR_DEV void split_codes(const i32x8& x, i32x8& hi, i32x8& lo) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // bit 6 of each byte, spread over it: v_perm's selectors 8 .. 11 are signs of halves
    const uint32_t c = (uint32_t)x[i], mask = __builtin_amdgcn_perm(c << 1, c << 9, 0x0b090a08u);
    hi[i] = (int)(c & mask);
    lo[i] = (int)(c ^ (c & mask));
  }
}

// Four results y[m][n .. n + 3], all of them in y (one store, which the hardware takes at
// any address)
template <bool F32>
WAR_DEV void store_whole(const MxGemmArgs& a, int m, int n, f32x4 v) {
  const uint2 b = *reinterpret_cast<const uint2*>(a.bias + n);
  v[0] += lo_f(b.x), v[1] += hi_f(b.x), v[2] += lo_f(b.y), v[3] += hi_f(b.y);
  const int64_t at = (int64_t)m * a.y_stride + n;
  if constexpr (F32) *reinterpret_cast<f32x4_any*>(static_cast<float*>(a.y) + at) = v;
  else *reinterpret_cast<u32x2_half*>(static_cast<bf16_t*>(a.y) + at) = u32x2_half{pack2(v[0], v[1]), pack2(v[2], v[3])};
}
// A 32 x 32 tile's results of a lane with the bias of their columns (from n on), into its
// row in LDS: columns 8 q + 4 half + 0 .. 3.  bf16: the lanes of a row swap halves of two
// q, so that each writes eight neighbours.
template <bool F32>
WAR_DEV void tile_row(const bf16_t* bias, int half, const f32x16& v, unsigned char* row) {
  uint32_t w[4][2];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint2 b = *reinterpret_cast<const uint2*>(bias + 8 * q + 4 * half);
    const f32x4 y = {v[4 * q] + lo_f(b.x), v[4 * q + 1] + hi_f(b.x), v[4 * q + 2] + lo_f(b.y), v[4 * q + 3] + hi_f(b.y)};
    if constexpr (F32) {
      *reinterpret_cast<f32x4*>(row + (8 * q + 4 * half) * 4) = y;
    } else {
      w[q][0] = pack2(y[0], y[1]);
      w[q][1] = pack2(y[2], y[3]);
    }
  }
  if constexpr (!F32) {
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
      const auto s0 = __builtin_amdgcn_permlane32_swap(w[q][0], w[q + 1][0], false, false);
      const auto s1 = __builtin_amdgcn_permlane32_swap(w[q][1], w[q + 1][1], false, false);
      *reinterpret_cast<uint4*>(row + 8 * (q + half) * 2) = make_uint4(s0[0], s1[0], s0[1], s1[1]);
    }
  }
}
// The same where some may lie outside
template <bool F32>
WAR_DEV void store_y(const MxGemmArgs& a, int m, int n, f32x4 v) {
  if (m >= a.M || n >= a.N) return;
  if (n + 4 <= a.N) return store_whole<F32>(a, m, n, v);
  const uint2 b = *reinterpret_cast<const uint2*>(a.bias + n);  // padded
  v[0] += lo_f(b.x), v[1] += hi_f(b.x), v[2] += lo_f(b.y), v[3] += hi_f(b.y);
  const int64_t at = (int64_t)m * a.y_stride + n;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n + i < a.N) {
      if constexpr (F32) static_cast<float*>(a.y)[at + i] = v[i];
      else static_cast<bf16_t*>(a.y)[at + i] = f2bf(v[i]);
    }
}

// Of what lanes ln (of 16) hold of rows ln % 8 (a) and 8 + ln % 8 (b), pieces g and, from
// ln = 8 on, g + 4: both pieces of row ln.
WAR_DEV void halves(uint4 a, uint4 b, uint4& lo, uint4& hi) {
  // row_ror:8 (0x128); bank masks: lanes 8 .. 15, lanes 0 .. 7
  auto low = [](uint32_t p, uint32_t q) { return (uint32_t)__builtin_amdgcn_update_dpp((int)p, (int)q, 0x128, 0xf, 0xc, false); };
  auto high = [](uint32_t p, uint32_t q) { return (uint32_t)__builtin_amdgcn_update_dpp((int)q, (int)p, 0x128, 0xf, 0x3, false); };
  lo = make_uint4(low(a.x, b.x), low(a.y, b.y), low(a.z, b.z), low(a.w, b.w));
  hi = make_uint4(high(a.x, b.x), high(a.y, b.y), high(a.z, b.z), high(a.w, b.w));
}

// Few rows: the weights' way from memory bounds it.  A workgroup takes 16 NT columns by
// 16 MT rows; its waves share the runs of 256 k between them, every fragment straight from
// memory to registers, RING - 1 runs ahead of the products, and their sums meet in LDS in
// the waves' order.  Nothing is shared between waves before that, so LDS would only add a
// wait; K goes over the waves because a tile of columns alone has too few bytes in flight
// (64 x 4096 x 12288: 256 workgroups' worth of columns at most).  What is left for few
// rows is the activations: they come from L2 once for each workgroup, by whole 128-byte
// lines (fragments read as the lanes hold them touch half lines twice: 11.7 us, now 10.4,
// for 64 x 4096 x 12288 in e2m1, 27 MB of weights; in e4m3 12.9, as twice the bytes).
// Splitting K over workgroups as well gained 15% there and 1% on average over 1 to 64 rows,
// for a workspace and a second pass; it is not done.
template <int MT, int NT, int WAVES, int RING, int XF, bool F32>
__global__ void __launch_bounds__(WAVES * 64) __attribute__((amdgpu_waves_per_eu(WAVES / 4, WAVES / 4 > 2 ? 4 : 2)))
k_mx_skinny(MxGemmArgs a) {
  constexpr bool E8 = XF == kMxE4M3, EXACT = E8 && F32;
  __shared__ f32x4 s_sum[WAVES][MT * NT][64];
  const int lane = threadIdx.x & 63, ln = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nt0 = blockIdx.x * NT, m0 = blockIdx.y * 16 * MT;
  const int groups = (a.K + 511) / 512, runs = (a.K + 255) / 256;
  f32x4 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  // x is read by whole lines: one load eight rows by 128 bytes, a lane piece pc of row ln % 8
  // (or 8 + ln % 8); lanes ln and ln ^ 8 then swap halves (see `halves`).  Rows past the
  // last read the last one, and are not written.
  const int pc = lg + (ln >> 3) * 4;
  const uint8_t *xc[MT][2], *xs[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      xc[m][h] = a.x.codes + (int64_t)min(m0 + m * 16 + h * 8 + (ln & 7), a.M - 1) * a.x.code_stride + pc * 16;
    xs[m] = a.x.scales + (int64_t)min(m0 + m * 16 + ln, a.M - 1) * a.x.scale_stride;
  }
  const uint8_t* wc[NT];
  const uint32_t* wsp[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {  // half of a tile's rows, of two of its fragments each
    const int64_t t = (int64_t)((nt0 + n) >> 1) * groups;
    const int li = ((nt0 + n) & 1) * 16 + ln + (lg & 1) * 32;
    wc[n] = a.w + (t * 8 + (lg >> 1)) * 1024 + li * 16;
    wsp[n] = a.ws + t * 128 + li;
  }
  uint4 x[RING][E8 ? 2 : 1][MT][2], w[RING][2][NT];  // x: of a line (e2m1: two steps), rows 0 .. 7 and 8 .. 15
  uint32_t sx[RING][2][MT], sw[RING][NT];
  // the fragments of run r into slot q
  auto load = [&](auto tag, int r) __attribute__((always_inline)) {
    constexpr int Q = decltype(tag)::value;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      sw[Q][n] = wsp[n][r * 64];
#pragma unroll
      for (int j = 0; j < 2; ++j) w[Q][j][n] = *reinterpret_cast<const uint4*>(wc[n] + (int64_t)(r * 2 + j) * 2048);
    }
    const int k0 = r * 256;
    if (k0 + 256 <= a.K) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const u32x2_any s = *reinterpret_cast<const u32x2_any*>(xs[m] + r * 8);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          sx[Q][j][m] = s[j];
          if (j == 0 || E8) {
#pragma unroll
            for (int h = 0; h < 2; ++h) x[Q][j][m][h] = *reinterpret_cast<const uint4*>(xc[m][h] + (int64_t)(E8 ? r * 2 + j : r) * 128);
          }
        }
      }
    } else {
      // 16-byte pieces hold numbers of one block: zero codes (and any scale but NaN's)
      // where it lies past K
      const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int kj = k0 + j * 128;
          sx[Q][j][m] = kj + lg * 32 < a.K ? *reinterpret_cast<const uint32_t*>(xs[m] + kj / 32) : 0x7f7f7f7fu;
          if (j == 0 || E8) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
              x[Q][j][m][h] = (E8 ? kj + pc * 16 : k0 + pc * 32) < a.K
                                  ? *reinterpret_cast<const uint4*>(xc[m][h] + (int64_t)(E8 ? r * 2 + j : r) * 128) : zero;
          }
        }
    }
  };
  auto products = [&](auto tag) __attribute__((always_inline)) {
    constexpr int Q = decltype(tag)::value;
    auto step = [&](auto tj) __attribute__((always_inline)) {
      constexpr int J = decltype(tj)::value;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        uint4 lo, hi;  // pieces lg and lg + 4 of row ln
        halves(x[Q][E8 ? J : 0][m][0], x[Q][E8 ? J : 0][m][1], lo, hi);
        if (!E8 && J == 1) lo = hi;
        i32x8 xv = {(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, 0, 0, 0, 0}, xl = xv;
        if constexpr (E8) {
          xv[4] = (int)hi.x, xv[5] = (int)hi.y, xv[6] = (int)hi.z, xv[7] = (int)hi.w;
          if constexpr (EXACT) {
            const i32x8 all = xv;
            split_codes(all, xv, xl);
          }
        }
        const uint32_t s = sx[Q][J][m] >> (8 * lg);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint4 c = w[Q][J][n];
          const i32x8 wv = {(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0};
          const uint32_t t = sw[Q][n] >> (8 * (lg >> 1));
          acc[m][n] = mx_mfma<XF, 2 * J>(wv, xv, acc[m][n], t, s);
          if constexpr (EXACT) acc[m][n] = mx_mfma<XF, 2 * J>(wv, xl, acc[m][n], t, s);
        }
      }
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
  };
  using std::integral_constant;
  // (every load of the loop is unconditional, so that what may stay in flight behind a
  // wait is known)
  int r = wave;
  if (r < runs) {
    load(integral_constant<int, 0>{}, r);
    if constexpr (RING == 2) {
      for (;;) {
        if (r + WAVES >= runs) {
          products(integral_constant<int, 0>{});
          break;
        }
        load(integral_constant<int, 1>{}, r += WAVES);
        products(integral_constant<int, 0>{});
        if (r + WAVES >= runs) {
          products(integral_constant<int, 1>{});
          break;
        }
        load(integral_constant<int, 0>{}, r += WAVES);
        products(integral_constant<int, 1>{});
      }
    } else if (r + WAVES >= runs) {
      products(integral_constant<int, 0>{});
    } else {
      load(integral_constant<int, 1>{}, r += WAVES);
      auto turn = [&](auto t0, auto t1, auto t2) __attribute__((always_inline)) {
        if (r + WAVES >= runs) {
          products(t0);
          products(t1);
          return false;
        }
        load(t2, r += WAVES);
        products(t0);
        return true;
      };
      while (turn(integral_constant<int, 0>{}, integral_constant<int, 1>{}, integral_constant<int, 2>{}) &&
             turn(integral_constant<int, 1>{}, integral_constant<int, 2>{}, integral_constant<int, 0>{}) &&
             turn(integral_constant<int, 2>{}, integral_constant<int, 0>{}, integral_constant<int, 1>{})) {
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) s_sum[wave][m * NT + n][lane] = acc[m][n];
  __syncthreads();
  for (int t = wave; t < MT * NT; t += WAVES) {
    f32x4 v = s_sum[0][t][lane];
#pragma unroll
    for (int q = 1; q < WAVES; ++q) v += s_sum[q][t][lane];
    store_y<F32>(a, m0 + (t / NT) * 16 + ln, (nt0 + t % NT) * 16 + lg * 4, v);
  }
}

// Many rows: the matrix cores bound it.  A workgroup computes a BM x BN tile from LDS, its
// waves as WM x WN.  A step is 128 columns, two fragments' width.  Every operand byte
// comes straight from memory to LDS, ST stages of one step each: x's rows with their
// 16-byte chunks permuted so that fragment reads fall on different banks, the weights'
// fragments as they are stored.  The scale words come for several steps at once.
//
// 256 x 256 by 8 waves: 128 sums a lane, and an LDS byte read once for 128 of a fragment's
// products, which takes 40% of the cycles.  8192 x 24576 x 4096: e2m1 435 to 480 us (3.6
// PFLOP/s; the instruction alone reaches 8.9), e4m3 590 to 640 us (2.7 of 4.95).  Over the
// whole kernel the matrix pipes are busy 52% and 76% of the cycles, in the loop 63% and
// 86%, at 1.8 GHz, to which power holds the clock: on codes of zeros the same instructions
// take 395 and 470 us, and without the loop's loads 3% less than with them.  The rest is a
// tile's first loads and its results, about 11 us each.  Not faster on this size: two
// workgroups of 128 x 256 a CU, which overlap these (582 us); one that goes on to its next
// tile and requests the first stages before it stores the results, which these then wait
// for (458 us become 492); stages requested a step later, for a barrier that waits for no
// LDS read (488, 489); bands of 8 and 16 row blocks (508, 511); stores past the caches
// (956); six stages.
template <int BM, int BN, int WM, int WN, int ST, int XF, bool F32>
__global__ void __launch_bounds__(WM * WN * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) k_mx_tile(MxGemmArgs a) {
  constexpr bool E8 = XF == kMxE4M3, EXACT = E8 && F32;
  constexpr int NW = WM * WN, MT = BM / WM / 32, NT = BN / WN / 32;
  static_assert(BM % (WM * 32) == 0 && BN % (WN * 32) == 0 && BN % (16 * NW) == 0 && BM <= NW * 64 && BN <= NW * 128 && ST <= 4,
                "whole fragments and loads");
  constexpr int RB = E8 ? 128 : 64, RPL = 1024 / RB;    // bytes of a row's step, rows of a 1 KB load
  constexpr int A_INS = (BM / RPL + NW - 1) / NW, W_INS = BN / 16 / NW, INS = A_INS + W_INS;  // loads of a wave and step
  constexpr int A_B = A_INS * NW * 1024, W_B = BN * 64, STAGE = A_B + W_B;
  // scales of four steps, requested four steps ahead, into one of two buffers: 16 bytes a
  // row of x, and a row of a weights' tile and block
  constexpr int XS_B = (BM + 63) / 64 * 1024, WS_B = BN * 16, XS = ST * STAGE, WS = XS + 2 * XS_B;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[WS + 2 * WS_B];
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, lg = lane >> 5;
  const int wi = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wi % WM, wn = wi / WM;
  const int mblocks = (a.M + BM - 1) / BM, NB = (a.N + BN - 1) / BN;
  // Workgroups are dealt to the 8 XCDs round-robin by linear id: each XCD takes an eighth of
  // the tiles, in bands of GM row blocks with the rows running fastest, so that its 32 CUs
  // work on about GM by 32 / GM blocks at a time and its L2 serves both operands.
  const int T = mblocks * NB, xcd = blockIdx.x & 7;
  const int t = xcd * (T >> 3) + min(xcd, T & 7) + (int)(blockIdx.x >> 3);
  const int band = t / (GM * NB), bm = min(mblocks - band * GM, GM), tr = t - band * GM * NB;
  const int mb = band * GM + tr % bm, nb = tr / bm;
  const int m0 = mb * BM, rows = min(BM, a.M - m0);
  const int K = a.K;
  const unsigned nsteps = (K + 127) / 128, kbytes = E8 ? K : K / 2;
  const int groups = (a.K + 511) / 512, tile_b = groups * 8192;
  const i32x4 xres = make_rsrc(a.x.codes + (int64_t)m0 * a.x.code_stride, (int64_t)(rows - 1) * a.x.code_stride + kbytes);
  const i32x4 sres = make_rsrc(a.x.scales + (int64_t)m0 * a.x.scale_stride,
                               (int64_t)(rows - 1) * a.x.scale_stride + ((K / 32 + 3) & ~3));
  const i32x4 wres = make_rsrc(a.w + (int64_t)nb * (BN / 32) * tile_b, (int64_t)(BN / 32) * tile_b);
  const i32x4 wsres = make_rsrc(a.ws + (int64_t)nb * (BN / 32) * groups * 128, (int64_t)(BN / 32) * groups * 512);
  const int xstride = (int)a.x.code_stride, sstride = (int)a.x.scale_stride;

  // x: load i of wave wi brings rows (i * NW + wi) * RPL .., a lane one 16-byte slot; slot
  // c of row r holds chunk c ^ swap(r).  Rows past the last and chunks past K are past the
  // descriptor: zero codes.
  constexpr unsigned PAST = 0x7fff0000;                 // past every descriptor (and twice that, too)
  auto swap = [](int r) { return E8 ? (r >> 1) & 7 : (r >> 2) & 3; };
  const int ar = wi * RPL + lane / (RB / 16);
  const unsigned ac = ((lane % (RB / 16)) ^ swap(ar)) * 16;
  const unsigned xv = ar * xstride + ac;
  // weights: load i brings fragment (i * NW + wi) % 2 of tile (i * NW + wi) / 2
  const unsigned wv = (wi / 2) * tile_b + (wi % 2) * 1024 + lane * 16;
  // load i of step s into stage q; steps past the last bring zeros, so that every wave
  // has the same loads in flight in every step
  auto load1 = [&](int q, unsigned s, int i) __attribute__((always_inline)) {
    const uint32_t to = lds_addr(smem) + q * STAGE;
    if (i < A_INS) {
      const unsigned o = xv + i * NW * RPL * xstride + (s < nsteps ? s * RB : PAST);
      load_lds16<false>(to + (i * NW + wi) * 1024, (int)(s * RB + ac < kbytes ? o : PAST), xres);
    } else {
      const int j = i - A_INS;
      load_lds16<false>(to + A_B + (j * NW + wi) * 1024, (int)(wv + j * (NW / 2) * tile_b + (s < nsteps ? s * 2048 : PAST)), wres);
    }
  };
  // the scale words of steps 4 g .. 4 g + 3: x's by the first waves, 64 rows each (of a row
  // in one load where rows lie and end at multiples of four words), the weights' by the
  // last, four tiles' halves each
  const int xsi = wi * 64 + lane, wsi = wi - (NW - BN / 64);
  auto load_scales = [&](unsigned g) __attribute__((always_inline)) {
    if (g * 4 >= nsteps) return;
    if (wi < XS_B / 1024) {
      if (a.scale16) {
        load_lds16<false>(lds_addr(smem) + XS + (g & 1) * XS_B + wi * 1024, (int)(xsi * sstride + g * 16), sres);
      } else {
        const uint8_t* p = a.x.scales + (int64_t)(m0 + min(xsi, rows - 1)) * a.x.scale_stride + g * 16;
        uint32_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (int)(g * 4 + e) * 128 < K ? *reinterpret_cast<const uint32_t*>(p + e * 4) : 0u;
        *reinterpret_cast<uint4*>(smem + XS + (g & 1) * XS_B + xsi * 16) = make_uint4(v[0], v[1], v[2], v[3]);
      }
    }
    if (wsi >= 0)  // (a tile's 512 bytes: 32 lanes)
      load_lds16<false>(lds_addr(smem) + WS + (g & 1) * WS_B + wsi * 1024,
                        (int)((wsi * 2 + (lane >> 5)) * groups * 512 + g * 512 + (lane & 31) * 16), wsres);
  };

  const int woff = A_B + wn * NT * 2048 + lane * 16;
  const int r0 = wm * (BM / WM) + ln;                   // swap(r0 + 32 mt) is the same for every mt
  // chunks of fragment u: e2m1 2 u + lg; e4m3 4 u + lg and 4 u + 2 + lg
  int aoff[E8 ? 4 : 2];
#pragma unroll
  for (int c = 0; c < (E8 ? 4 : 2); ++c) aoff[c] = r0 * RB + (((2 * c + lg) ^ swap(r0)) * 16);

  f32x16 acc[MT][NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[m][n][e] = 0.f;
  // own loads of the next stage arrived (`left` later ones may be in flight) and own LDS
  // reads done, then everyone's
  auto sync = [&](auto left) __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(decltype(left)::value) : "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // A step is 2 MT slots, one x fragment (and NT products) each, read LOOK slots ahead; the
  // weights of its second half are read in the first, the next step's in the last LOOK
  // slots.  Before these the next stage must be complete (sync); every read of this stage
  // is then done, and step s + ST is requested into it, a few loads a slot, on into the
  // next step's first slots.
  constexpr int SLOTS = 2 * MT, RING = SLOTS % 4 == 0 ? 4 : SLOTS % 3 == 0 ? 3 : 2, LOOK = SLOTS == 4 ? 2 : RING - 1;
  constexpr int LPS = (INS + SLOTS - 1) / SLOTS, HEAD = LPS * LOOK < INS ? LPS * LOOK : INS;
  static_assert(SLOTS % RING == 0 && RING > LOOK && LOOK <= MT, "a ring of fragments");
  uint4 ra[RING][E8 ? 2 : 1], rb[2][NT];
  uint32_t rs[MT], wsc[2][NT];                          // scales: a row's word, a fragment's byte
  // q: the step's stage, which is its place among its four steps where there are four stages
  auto of_four = [](unsigned s, int q) { return ST == 4 ? (unsigned)q : s & 3; };
  const int xsl = XS + r0 * 16, wsl = WS + wn * NT * 512 + lane * 4;
  auto read_x = [&](int q, unsigned s, int i) __attribute__((always_inline)) {
    const unsigned char* st = smem + q * STAGE;
    const int m = i % MT, u = i / MT;
    ra[i % RING][0] = *reinterpret_cast<const uint4*>(st + m * 32 * RB + aoff[E8 ? 2 * u : u]);
    if constexpr (E8) ra[i % RING][1] = *reinterpret_cast<const uint4*>(st + m * 32 * RB + aoff[2 * u + 1]);
    if (u == 0) rs[m] = *reinterpret_cast<const uint32_t*>(smem + xsl + (s >> 2 & 1) * XS_B + of_four(s, q) * 4 + m * 512);
  };
  auto read_w = [&](int q, unsigned s, int u, int n) __attribute__((always_inline)) {
    const unsigned f = of_four(s, q);
    rb[u][n] = *reinterpret_cast<const uint4*>(smem + q * STAGE + woff + (2 * n + u) * 1024);
    wsc[u][n] = smem[wsl + (s >> 2 & 1) * WS_B + f / 2 * 256 + f % 2 * 2 + n * 512 + u];
  };
  // The bytes of a row's word that are this lane's blocks, 0 and 2 of it behind the shift;
  // where a block lies past K: zero codes, and any byte but NaN's.
  uint32_t keep = 0xffffffffu, fill = 0;
  // C: the step's stage
  auto step = [&](unsigned s, auto tag) __attribute__((always_inline)) {
    constexpr int C = decltype(tag)::value, N = (C + 1) % ST, Pv = (C + ST - 1) % ST;
    if (of_four(s, C) == 0) load_scales((s >> 2) + 1);
    if (s + 1 == nsteps) {
      keep = ((int)(s * 128 + lg * 32) < K ? 0xffu : 0u) | ((int)(s * 128 + 64 + lg * 32) < K ? 0xff0000u : 0u);
      fill = ~keep & 0x7f7f7f7fu;
    }
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      const uint32_t sx = ((rs[i % MT] >> (8 * lg)) & keep) | fill;
      // stages s + 2 .. s + ST - 1 may still be in flight
      if (i == SLOTS - LOOK) sync(std::integral_constant<int, (ST - 2) * INS>{});
      if (i < SLOTS - LOOK) read_x(C, s, i + LOOK);
      else read_x(N, s + 1, i + LOOK - SLOTS);
      if (i < MT) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
          if (n * MT / NT == i) read_w(C, s, 1, n);
      }
      if (i >= SLOTS - LOOK) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
          if (n * LOOK / NT == i - (SLOTS - LOOK)) read_w(N, s + 1, 0, n);
#pragma unroll
        for (int q = 0; q < LPS; ++q)
          if ((i - (SLOTS - LOOK)) * LPS + q < INS) load1(C, s + ST, (i - (SLOTS - LOOK)) * LPS + q);
      } else {
#pragma unroll
        for (int q = 0; q < LPS; ++q)
          if (HEAD + i * LPS + q < INS) load1(Pv, s + ST - 1, HEAD + i * LPS + q);
      }
      const uint4 x0 = ra[i % RING][0];
      i32x8 xf = {(int)x0.x, (int)x0.y, (int)x0.z, (int)x0.w, 0, 0, 0, 0}, xl = xf;
      if constexpr (E8) {
        const uint4 x1 = ra[i % RING][1];
        xf[4] = (int)x1.x, xf[5] = (int)x1.y, xf[6] = (int)x1.z, xf[7] = (int)x1.w;
        if constexpr (EXACT) {
          const i32x8 whole = xf;
          split_codes(whole, xf, xl);
        }
      }
#pragma unroll
      for (int e = 0; e < (EXACT ? 2 : 1); ++e)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint4 w0 = rb[i / MT][n];
          const i32x8 wf = {(int)w0.x, (int)w0.y, (int)w0.z, (int)w0.w, 0, 0, 0, 0};
          f32x16& c = acc[i % MT][n];
          if (i < MT) c = mx_mfma32<XF, 0>(wf, e ? xl : xf, c, wsc[0][n], sx);
          else c = mx_mfma32<XF, 2>(wf, e ? xl : xf, c, wsc[1][n], sx);
        }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  load_scales(0);
#pragma unroll
  for (int q = 0; q < ST; ++q) {
    // (of the last stage only what a step leaves to the one before it: step 0 brings the rest)
#pragma unroll
    for (int i = 0; i < (q == ST - 1 ? HEAD : INS); ++i) load1(q, q, i);
  }
  sync(std::integral_constant<int, (ST - 2) * INS + HEAD>{});
#pragma unroll
  for (int n = 0; n < NT; ++n) read_w(0, 0, 0, n);
#pragma unroll
  for (int i = 0; i < LOOK; ++i) read_x(0, 0, i);
  __builtin_amdgcn_sched_barrier(0);
  // (the reads past the last step are of no use, and in bounds)
  for (unsigned s = 0; s < nsteps;) {
    step(s++, std::integral_constant<int, 0>{});
    if (s < nsteps) step(s++, std::integral_constant<int, 1>{});
    if constexpr (ST > 2)
      if (s < nsteps) step(s++, std::integral_constant<int, 2>{});
    if constexpr (ST > 3)
      if (s < nsteps) step(s++, std::integral_constant<int, 3>{});
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // no load into LDS is in flight
  __syncthreads();
  // The results go out by whole rows of the wave's columns, through LDS: as the matrix unit
  // leaves them (32 rows a store, 32 bytes each) every line of y is touched four times,
  // which took as long as a fifth of 32 steps.
  constexpr int SZ = F32 ? 4 : 2, ROW = NT * 32 * SZ, CPR = ROW / 16, RPI = 64 / CPR, PITCH = ROW + 16;
  static_assert(NW * 32 * PITCH <= WS + 2 * WS_B, "a wave's rows fit");
  unsigned char* buf = smem + wi * 32 * PITCH;
  const int n0 = nb * BN + wn * NT * 32, col = n0 + lane % CPR * (16 / SZ);
#pragma unroll
  for (int m = 0; m < MT; ++m) {
#pragma unroll
    for (int n = 0; n < NT; ++n) tile_row<F32>(a.bias + n0 + n * 32, lg, acc[m][n], buf + ln * PITCH + n * 32 * SZ);
#pragma unroll
    for (int i = 0; i < 32 / RPI; ++i) {
      const int r = i * RPI + lane / CPR, row = m0 + wm * (BM / WM) + m * 32 + r;
      const uint4 v = *reinterpret_cast<const uint4*>(buf + r * PITCH + lane % CPR * 16);
      if (row >= a.M) continue;
      unsigned char* y = static_cast<unsigned char*>(a.y) + ((int64_t)row * a.y_stride + col) * SZ;
      if (col + 16 / SZ <= a.N) {
        *reinterpret_cast<u32x4_half*>(y) = u32x4_half{v.x, v.y, v.z, v.w};
      } else {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 16 / SZ; ++e)
          if (col + e < a.N) {
            if constexpr (F32) *reinterpret_cast<uint32_t*>(y + e * 4) = w[e];
            else *reinterpret_cast<bf16_t*>(y + e * 2) = (bf16_t)(w[e / 2] >> (16 * (e & 1)));
          }
      }
    }
  }
}

template <int BM, int BN, int WM, int WN, int ST8, int ST4>
void tile(const MxGemmArgs& a, int fmt, bool f32, hipStream_t st) {
  const int grid = cdiv_i(a.N, BN) * cdiv_i(a.M, BM);
  constexpr int T = WM * WN * 64;
  if (fmt == kMxE4M3) {
    if (f32) k_mx_tile<BM, BN, WM, WN, ST8, kMxE4M3, true><<<grid, T, 0, st>>>(a);
    else k_mx_tile<BM, BN, WM, WN, ST8, kMxE4M3, false><<<grid, T, 0, st>>>(a);
  } else {
    if (f32) k_mx_tile<BM, BN, WM, WN, ST4, kMxE2M1, true><<<grid, T, 0, st>>>(a);
    else k_mx_tile<BM, BN, WM, WN, ST4, kMxE2M1, false><<<grid, T, 0, st>>>(a);
  }
}

template <int MT, int NT, int WAVES, int RING>
void skinny(const MxGemmArgs& a, int fmt, bool f32, hipStream_t st) {
  const dim3 grid((a.N + 16 * NT - 1) / (16 * NT), (a.M + 16 * MT - 1) / (16 * MT));
  if (fmt == kMxE4M3) {
    if (f32) k_mx_skinny<MT, NT, WAVES, NT < 4 ? RING : 2, kMxE4M3, true><<<grid, WAVES * 64, 0, st>>>(a);
    else k_mx_skinny<MT, NT, WAVES, RING, kMxE4M3, false><<<grid, WAVES * 64, 0, st>>>(a);
  } else {
    if (f32) k_mx_skinny<MT, NT, WAVES, RING, kMxE2M1, true><<<grid, WAVES * 64, 0, st>>>(a);
    else k_mx_skinny<MT, NT, WAVES, RING, kMxE2M1, false><<<grid, WAVES * 64, 0, st>>>(a);
  }
}

// What a kernel takes by estimate (us): `start`, then the rounds of its workgroups over the
// 256 CUs, `step` for a step of one workgroup a CU (few rows: of 2048 columns), `full`
// where the CUs hold all they can, `more` for a round behind the first; at least the
// weights' bytes at 4.6 TB/s (few rows: `more` times as long).
struct Cost {
  float start, step, full, more;
};
struct Shape {
  int bm, bn, occ;  // rows and columns of a workgroup, workgroups a CU
};
constexpr int kShapes = kMxShapes, kSkinny = 3;
constexpr Shape kShape[kShapes] = {{16, 16, 2}, {16, 32, 1}, {16, 64, 1}, {32, 128, 2}, {64, 128, 2}, {128, 128, 1},
                                   {96, 256, 2}, {128, 256, 1}, {192, 256, 1}, {256, 256, 1}};
// x in e4m3 for a bf16 y, for an fp32 y, in e2m1; fitted to the times of 677 products of 1 to
// 4096 rows, 128 to 151936 columns and K of 256 to 12288, the weights of up to eight in turn.
// Over these the choice takes 0.5% more than the best of the shapes on average, and 24% at
// most (16 rows of 24576 by 4096 in e4m3: 17.4 us for 14.0).
constexpr Cost kCost[3][kShapes] = {
    {{2.70f, 1.00f, 1.42f, 1.28f}, {2.66f, 1.29f, 1.61f, 1.13f}, {2.82f, 1.67f, 2.20f, 1.05f}, {4.04f, 0.19f, 0.18f, 0.91f},
     {4.42f, 0.25f, 0.26f, 1.23f}, {5.02f, 0.34f, 0.46f, 2.92f}, {5.97f, 0.68f, 0.57f, 2.54f},
     {6.30f, 0.56f, 0.67f, 4.82f}, {7.44f, 0.84f, 0.95f, 6.52f}, {8.00f, 1.10f, 1.35f, 8.00f}},
    {{2.50f, 0.47f, 1.72f, 1.39f}, {2.94f, 0.30f, 1.85f, 1.23f}, {3.65f, 0.23f, 2.40f, 1.08f}, {3.23f, 0.37f, 0.27f, 0.65f},
     {4.07f, 0.55f, 0.44f, 0.66f}, {3.38f, 0.89f, 0.60f, 2.88f}, {5.92f, 1.05f, 0.97f, 0.55f},
     {6.18f, 1.12f, 1.28f, 2.19f}, {6.65f, 1.69f, 1.34f, 3.96f}, {7.62f, 2.14f, 1.09f, 5.14f}},
    {{3.31f, 0.54f, 0.96f, 0.74f}, {2.92f, 0.71f, 1.22f, 0.97f}, {2.97f, 1.03f, 1.66f, 1.19f}, {4.05f, 0.18f, 0.16f, 0.96f},
     {4.30f, 0.23f, 0.22f, 1.17f}, {4.97f, 0.27f, 0.35f, 2.97f}, {6.36f, 0.40f, 0.48f, 4.02f},
     {5.95f, 0.41f, 0.62f, 4.85f}, {7.61f, 0.52f, 0.68f, 7.24f}, {8.00f, 0.68f, 0.85f, 8.00f}}};

bool fits_launch(const MxGemmArgs& a, int c) {  // its work items below 2^32
  return (int64_t)cdiv_i(a.M, kShape[c].bm) * cdiv_i(a.N, kShape[c].bn) * 512 < (int64_t)1 << 32;
}

int choose(const MxGemmArgs& a, int fmt, bool f32) {
  const Cost* cost = kCost[fmt == kMxE2M1 ? 2 : f32 ? 1 : 0];
  const float floor = (float)a.N * (float)a.K * (17.f / 32.f / 4.6e6f);
  int best = kShapes - 1;
  float least = 1e30f;
  for (int c = a.M <= 64 ? 0 : kSkinny; c < kShapes; ++c) {
    const Shape& s = kShape[c];
    const int64_t wgs = (int64_t)cdiv_i(a.M, s.bm) * cdiv_i(a.N, s.bn);
    if (!fits_launch(a, c)) continue;
    const int steps = c < kSkinny ? cdiv_i(a.K, 2048) : cdiv_i(a.K, 128);
    const float rounds = (float)((wgs + 255) / 256), few = (float)((wgs + 256 * s.occ - 1) / (256 * s.occ));
    float t = cost[c].step * steps * few;
    if (wgs > 256) t = fmaxf(t, cost[c].full * steps * rounds);
    t = cost[c].start + (c < kSkinny ? fmaxf(t, floor * cost[c].more) : fmaxf(t, floor) + cost[c].more * (rounds - 1.f));
    if (t < least) {
      least = t;
      best = c;
    }
  }
  return best;
}

}  // namespace

void launch_mx_pack(const MxRef& w, int N, int K, uint8_t* codes, uint32_t* scales, hipStream_t st) {
  k_mx_pack<<<dim3(mx_tiles(N), mx_groups(K)), 512, 0, st>>>(w, N, K, mx_groups(K), codes, scales);
}

int plan_mx_gemm(int M, int N, int K, int fmt, bool f32) {
  MxGemmArgs a{};
  a.M = M;
  a.N = N;
  a.K = K;
  return choose(a, fmt, f32);
}

bool launch_mx_gemm(const MxGemmArgs& a, int fmt, bool f32, int shape, hipStream_t st) {
  if (shape < 0) shape = choose(a, fmt, f32);
  if (shape >= kShapes || !fits_launch(a, shape) || (shape < kSkinny && a.M > 65535 * 16)) return false;
  switch (shape) {
    case 0: skinny<1, 1, 8, 3>(a, fmt, f32, st); break;
    case 1: skinny<1, 2, 8, 3>(a, fmt, f32, st); break;
    case 2: skinny<1, 4, 8, 3>(a, fmt, f32, st); break;
    case 3: tile<32, 128, 1, 4, 4, 4>(a, fmt, f32, st); break;
    case 4: tile<64, 128, 1, 4, 4, 4>(a, fmt, f32, st); break;
    case 5: tile<128, 128, 2, 4, 4, 4>(a, fmt, f32, st); break;
    case 6: tile<96, 256, 1, 4, 2, 3>(a, fmt, f32, st); break;
    case 7: tile<128, 256, 2, 4, 4, 4>(a, fmt, f32, st); break;
    case 8: tile<192, 256, 2, 4, 3, 4>(a, fmt, f32, st); break;
    default: tile<256, 256, 2, 4, 3, 4>(a, fmt, f32, st); break;
  }
  return true;
}
