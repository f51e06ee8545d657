// Rotary positions of several axes over a step's rows: queries are turned, keys are
// turned and go into the cache's pages with their values (bf16 or e4m3, kv_page.h).
//
// Pair j of a head turns by position a(j) of its row times a frequency.  The product is
// taken in double in units of a full turn, so that dropping whole turns is exact and
// positions near 2^31 keep the angle to 2^-24 of a turn; sine and cosine are fp32.
// Memory bounds it for many rows and a launch's latency for few: a workgroup takes a
// page of one kv-head, or the same tokens' query heads, eight numbers a lane; a lane's
// four angles are taken once for all its heads.
#include <type_traits>

#include "e4m3.h"
#include "kv_page.h"

namespace {

constexpr int kQHeads = 8;  // query heads a workgroup takes, one after the other

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

// cos and sin of the lane's four pairs for row `row`
WAR_DEV void angles(const RopeArgs& a, int u, int64_t row, int pos, float (&c)[4], float (&s)[4]) {
  const int64_t rows = (int64_t)a.B * a.n_max;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int j = 4 * u + e;
    const double p = a.positions ? (double)a.positions[a.axis[j] * rows + row] : (double)pos;
    const double t = p * a.turns[j];
    sincospif(2.f * (float)(t - rint(t)), &s[e], &c[e]);
  }
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

template <bool Q8, int HD>
__global__ void __launch_bounds__(2 * HD) k_rope_write(RopeArgs a) {
  using O = PageOrder<Q8, HD>;
  constexpr int L = HD / 8;  // lanes a token
  __shared__ __attribute__((aligned(16))) unsigned char s_pg[2 * O::kBytes];
  __shared__ unsigned char s_sc[32];
  const int b = blockIdx.x / a.pages, jp = blockIdx.x % a.pages;
  const int pos0 = a.pos0[b];
  PageSpan sp;
  if (!page_span(a.p, b, jp, a.seq[b], pos0, a.n ? a.n[b] : a.n_max, a.n_max, jp == 0 && blockIdx.y == 0 && threadIdx.x == 0, sp))
    return;
  const int slot = threadIdx.x / L, u = threadIdx.x % L;
  const bool live = slot >= sp.lo && slot < sp.hi;
  const int i = sp.t0 + slot - sp.lo;  // token of the request
  const int64_t row = (int64_t)b * a.n_max + i;
  const Dims d = dims_of(a, u);
  float c[4], s[4];
  if (live && d.turn) angles(a, u, row, pos0 + i, c, s);
  const int kvh = blockIdx.y;
  if (kvh >= a.g.n_kv_heads) {
    if (!live) return;
    const int h0 = (kvh - a.g.n_kv_heads) * kQHeads, h1 = min(h0 + kQHeads, a.n_q_heads);
#pragma unroll 4
    for (int h = h0; h < h1; ++h) {
      const bf16_t* q = a.q + row * a.q_stride + h * HD;
      bf16_t* o = a.qo + row * a.qo_stride + h * HD;
      uint2 w1 = *reinterpret_cast<const uint2*>(q + d.d1), w2 = *reinterpret_cast<const uint2*>(q + d.d2);
      turn8(a, d.turn, c, s, w1, w2);
      *reinterpret_cast<uint2*>(o + d.d1) = w1;
      *reinterpret_cast<uint2*>(o + d.d2) = w2;
    }
    return;
  }
  if (live) {
    const bf16_t* k = a.k + row * a.k_stride + kvh * HD;
    uint2 w1 = *reinterpret_cast<const uint2*>(k + d.d1), w2 = *reinterpret_cast<const uint2*>(k + d.d2);
    const uint4 vw = *reinterpret_cast<const uint4*>(a.v + row * a.v_stride + kvh * HD + 8 * u);
    turn8(a, d.turn, c, s, w1, w2);
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
  const dim3 grid(a.B * a.pages, a.g.n_kv_heads + cdiv_i(a.n_q_heads, kQHeads));
  if (a.g.head_dim == 128) {
    if (a.g.q8) k_rope_write<true, 128><<<grid, 256, 0, st>>>(a);
    else k_rope_write<false, 128><<<grid, 256, 0, st>>>(a);
  } else {
    if (a.g.q8) k_rope_write<true, 64><<<grid, 128, 0, st>>>(a);
    else k_rope_write<false, 64><<<grid, 128, 0, st>>>(a);
  }
}
