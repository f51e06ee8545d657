// Rotary positions of several axes over a step's rows: queries are turned, keys are
// turned and go into the cache's pages with their values (bf16 or e4m3, kv_page.h).
//
// Pair j of a head turns by position a(j) of its row times a frequency.  The product is
// taken in double in units of a full turn, so that dropping whole turns is exact at any
// position; sine and cosine are double, too, and so are the keys' turns, as these are
// rounded twice (bf16, then a code).  Queries turn in fp32.
// Memory bounds it for many rows and a launch's latency for few: a workgroup takes a
// page of one kv-head with the same tokens' query heads of its group, eight numbers of a
// head a lane; a lane's four angles are taken once for all of them, behind the loads.
// 28300 rows of 32 and 8 heads of 128 into bf16 pages: 148 us for 695 MB, 4.7 TB/s; 134
// with sine, cosine and keys in fp32, of whose codes one in some 10^5 was another.  (By
// ordinary loads and stores of what it turns 163 for these 134, and less of the pages stays
// in the caches for who reads them next, 56 us for 40; with workgroups of their own for
// the query heads, and the angles before the loads, 188.)  192 rows into e4m3 pages: 7.6
// us, of which the angles are about 3.
#include <type_traits>

#include "e4m3.h"
#include "kv_page.h"

namespace {

constexpr int kMostGroup = 8;  // query heads of a kv-head

// A lane's eight dims of a head: four at d1 and four at d2.  Turning, they are pairs
// 4 u + e: (d1 + e, d2 + e), or neighbours of d1 .. and then of d2 ...
struct Dims {
  int d1, d2;
  bool turn;
};
WAR_DEV Dims dims_of(const RopeArgs& a, int u) {
  const int R = a.rotary;
  if (8 * u >= R) return {8 * u, 8 * u + 4, false};
  if (a.adjacent) return {8 * u, 8 * u + 4, true};
  return {4 * u, R / 2 + 4 * u, true};
}
WAR_DEV void unpack4(uint2 w, float (&x)[4]) { x[0] = lo_f(w.x), x[1] = hi_f(w.x), x[2] = lo_f(w.y), x[3] = hi_f(w.y); }

// cos and sin of the lane's four pairs, whose positions are p
WAR_DEV void angles(const double (&turns)[4], const int (&p)[4], double (&c)[4], double (&s)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const double t = (double)p[e] * turns[e];
    sincospi(2. * (t - rint(t)), &s[e], &c[e]);
  }
}
// d as a float that rounds to the bf16 that d rounds to: cut towards an odd last bit
WAR_DEV float sticky(double d) {
  const float f = (float)d;
  const double rest = d - (double)f;
  const uint32_t u = __float_as_uint(f);
  if (!(rest < 0. || rest > 0.) || (u & 1)) return f;  // exact, not finite, or no tie of a bf16's
  return __uint_as_float((rest < 0.) == (bool)(u >> 31) ? u + 1 : u - 1);
}
// the two runs turned and rounded to bf16
WAR_DEV void turn8(const RopeArgs& a, bool turn, const float (&c)[4], const float (&s)[4], uint2& w1, uint2& w2) {
  if (!turn) return;
  float x[4], y[4], o1[4], o2[4];
  unpack4(w1, x);
  unpack4(w2, y);
  if (a.adjacent) {
    o1[0] = x[0] * c[0] - x[1] * s[0], o1[1] = x[1] * c[0] + x[0] * s[0];
    o1[2] = x[2] * c[1] - x[3] * s[1], o1[3] = x[3] * c[1] + x[2] * s[1];
    o2[0] = y[0] * c[2] - y[1] * s[2], o2[1] = y[1] * c[2] + y[0] * s[2];
    o2[2] = y[2] * c[3] - y[3] * s[3], o2[3] = y[3] * c[3] + y[2] * s[3];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o1[e] = x[e] * c[e] - y[e] * s[e];
      o2[e] = y[e] * c[e] + x[e] * s[e];
    }
  }
  w1 = make_uint2(pack2(o1[0], o1[1]), pack2(o1[2], o1[3]));
  w2 = make_uint2(pack2(o2[0], o2[1]), pack2(o2[2], o2[3]));
}

// The same in double, for keys: they are rounded again, to their code, and a bf16 on the
// wrong side of a tie (in fp32 one of 10^5) may be the next code.
WAR_DEV void turn8(const RopeArgs& a, bool turn, const double (&c)[4], const double (&s)[4], uint2& w1, uint2& w2) {
  if (!turn) return;
  float x[4], y[4], o1[4], o2[4];
  unpack4(w1, x);
  unpack4(w2, y);
  auto pair = [](float x, float y, double c, double s, float& p, float& q) {
    p = sticky((double)x * c - (double)y * s);
    q = sticky((double)y * c + (double)x * s);
  };
  if (a.adjacent) {
    pair(x[0], x[1], c[0], s[0], o1[0], o1[1]), pair(x[2], x[3], c[1], s[1], o1[2], o1[3]);
    pair(y[0], y[1], c[2], s[2], o2[0], o2[1]), pair(y[2], y[3], c[3], s[3], o2[2], o2[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) pair(x[e], y[e], c[e], s[e], o1[e], o2[e]);
  }
  w1 = make_uint2(pack2(o1[0], o1[1]), pack2(o1[2], o1[3]));
  w2 = make_uint2(pack2(o2[0], o2[1]), pack2(o2[2], o2[3]));
}

template <bool Q8, int HD, int G>
__global__ void __launch_bounds__(2 * HD) k_rope_write(RopeArgs a) {
  using O = PageOrder<Q8, HD>;
  constexpr int L = HD / 8;  // lanes a token
  __shared__ __attribute__((aligned(16))) unsigned char s_pg[2 * O::kBytes];
  __shared__ unsigned char s_sc[32];
  const int b = blockIdx.x / a.pages, jp = blockIdx.x % a.pages, kvh = blockIdx.y;
  const int slot = threadIdx.x / L, u = threadIdx.x % L;
  const Dims d = dims_of(a, u);
  const int pos0 = a.pos0[b], seq = a.seq[b], n = a.n ? a.n[b] : a.n_max;
  double turns[4];
  int axis[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) turns[e] = a.turns[4 * u + e], axis[e] = a.axis[4 * u + e];
  // a token's numbers are read before its request is known to fit its pages (the rows are
  // there in any case), so that one memory round trip follows the request's numbers
  const int i = jp * kPageSlots + slot - (pos0 & (kPageSlots - 1));  // token of the request
  const bool live = pos0 >= 0 && i >= 0 && i < min(n, a.n_max);
  const int64_t row = (int64_t)b * a.n_max + i;
  uint2 k1 = {}, k2 = {}, q1[G], q2[G];
  uint4 vw = {};
  int p[4] = {};
  if (live) {
    const bf16_t* k = a.k + row * a.k_stride + kvh * HD;
    k1 = load_once8(k + d.d1);
    k2 = load_once8(k + d.d2);
    vw = load_once16(a.v + row * a.v_stride + kvh * HD + 8 * u);
    const bf16_t* q = a.q + row * a.q_stride + kvh * a.group * HD;
#pragma unroll
    for (int h = 0; h < G; ++h)
      if (h < a.group) {
        q1[h] = load_once8(q + h * HD + d.d1);
        q2[h] = load_once8(q + h * HD + d.d2);
      }
    const int64_t rows = (int64_t)a.B * a.n_max;
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = a.positions ? a.positions[axis[e] * rows + row] : pos0 + i;
  }
  PageSpan sp;
  if (!page_span(a.p, b, jp, seq, pos0, n, a.n_max, jp == 0 && kvh == 0 && threadIdx.x == 0, sp)) return;
  if (live) {
    float c[4], s[4];
    double c64[4] = {}, s64[4] = {};
    if (d.turn) angles(turns, p, c64, s64);
    turn8(a, d.turn, c64, s64, k1, k2);
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = (float)c64[e], s[e] = (float)s64[e];
    bf16_t* o = a.qo + row * a.qo_stride + kvh * a.group * HD;
#pragma unroll
    for (int h = 0; h < G; ++h)
      if (h < a.group) {
        turn8(a, d.turn, c, s, q1[h], q2[h]);
        store_once8(o + h * HD + d.d1, q1[h]);
        store_once8(o + h * HD + d.d2, q2[h]);
      }
    const uint2 w1 = k1, w2 = k2;
    const uint32_t vv[4] = {vw.x, vw.y, vw.z, vw.w};
    if constexpr (Q8) {
      float x1[4], x2[4], v[8];
      unpack4(w1, x1);
      unpack4(w2, x2);
      float ktop = 0.f, vtop = 0.f;
      int bad = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = lo_f(vv[e]);
        v[2 * e + 1] = hi_f(vv[e]);
        ktop = fmaxf(ktop, fmaxf(fabsf(x1[e]), fabsf(x2[e])));
        vtop = fmaxf(vtop, fmaxf(fabsf(v[2 * e]), fabsf(v[2 * e + 1])));
        bad |= !(fabsf(x1[e]) < INFINITY) | !(fabsf(x2[e]) < INFINITY) | !(fabsf(v[2 * e]) < INFINITY) |
               !(fabsf(v[2 * e + 1]) < INFINITY);
      }
#pragma unroll
      for (int o = 1; o < L; o <<= 1) {
        ktop = fmaxf(ktop, __shfl_xor(ktop, o, 64));
        vtop = fmaxf(vtop, __shfl_xor(vtop, o, 64));
        bad |= __shfl_xor(bad, o, 64);
      }
      // what marks a token that is not finite: as in kv8.hip
      const int ke = block_exp8(bad ? 0.f : ktop), ve = block_exp8(bad ? 0.f : vtop);
      const float kf = exp2_int(-ke), vf = exp2_int(-ve);
      const uint32_t nan4 = kNanCode8 * 0x01010101u;
      *reinterpret_cast<uint32_t*>(&s_pg[O::key(slot, d.d1)]) =
          bad ? nan4 : to_e4m3x4(x1[0] * kf, x1[1] * kf, x1[2] * kf, x1[3] * kf);
      *reinterpret_cast<uint32_t*>(&s_pg[O::key(slot, d.d2)]) =
          bad ? nan4 : to_e4m3x4(x2[0] * kf, x2[1] * kf, x2[2] * kf, x2[3] * kf);
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const uint32_t vc = bad ? 0 : to_e4m3x4(v[e] * vf, v[e + 1] * vf, v[e + 2] * vf, v[e + 3] * vf);
#pragma unroll
        for (int t = 0; t < 4; ++t) s_pg[O::kBytes + O::val(slot, 8 * u + e + t)] = (vc >> (8 * t)) & 0xff;
      }
      if (u == 0) {
        s_sc[key_scale8(slot)] = bad ? 127 : ke + 127;
        s_sc[val_scale8(slot)] = bad ? 0 : ve + 127;
      }
    } else {
      *reinterpret_cast<uint2*>(&s_pg[O::key(slot, d.d1)]) = w1;
      *reinterpret_cast<uint2*>(&s_pg[O::key(slot, d.d2)]) = w2;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        *reinterpret_cast<bf16_t*>(&s_pg[O::kBytes + O::val(slot, 8 * u + 2 * e)]) = (bf16_t)vv[e];
        *reinterpret_cast<bf16_t*>(&s_pg[O::kBytes + O::val(slot, 8 * u + 2 * e + 1)]) = (bf16_t)(vv[e] >> 16);
      }
    }
  }
  __syncthreads();
  store_page<Q8, HD, 2 * HD>(a.g, a.layer, kvh, sp, s_pg, s_sc);
}

}  // namespace

void launch_rope_write(const RopeArgs& a, hipStream_t st) {
  const dim3 grid(a.B * a.pages, a.g.n_kv_heads);
  auto go = [&](auto hd, auto g) {
    constexpr int HD = decltype(hd)::value, G = decltype(g)::value;
    if (a.g.q8) k_rope_write<true, HD, G><<<grid, 2 * HD, 0, st>>>(a);
    else k_rope_write<false, HD, G><<<grid, 2 * HD, 0, st>>>(a);
  };
  using std::integral_constant;
  if (a.g.head_dim == 128) {
    if (a.group <= 4) go(integral_constant<int, 128>{}, integral_constant<int, 4>{});
    else go(integral_constant<int, 128>{}, integral_constant<int, kMostGroup>{});
  } else {
    if (a.group <= 4) go(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else go(integral_constant<int, 64>{}, integral_constant<int, kMostGroup>{});
  }
}
