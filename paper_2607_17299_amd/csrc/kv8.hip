// Keys and values of given tokens into and out of a pool's pages, for many sequences
// at once, in the pool's own format: bf16, or e4m3 with a scale for each token and
// kv-head (e4m3.h).
//
// Memory bounds them for many tokens and a launch's latency for few.  A workgroup
// takes one page of one kv-head: 16 threads a token, so that a block's maximum is four
// exchanges within a wave, and the page passes through LDS in its own order, so that
// both sides move 16-byte pieces.  A page's other slots hold other tokens: of a piece
// that covers some of them only the new tokens' bytes are written.
// 28,300 tokens of 16 requests, 8 heads of 128, e4m3 (175 MB): written in 33 us (5.3 TB/s),
// read in 31.5 (5.5); bf16 (232 MB): 40 us (5.8) and 48 (4.8); 64 requests' three tokens
// 4.3 and 3.5 us, a launch.  (A copy kernel of that size reaches 6.4 TB/s.)
#include <type_traits>

#include "e4m3.h"
#include "kernels.h"

namespace {

constexpr int kPage = 16;

// Element (bf16) or byte (e4m3) of a page's keys and values.
template <bool Q8, int HD>
struct PageOrder {
  static constexpr int kElem = Q8 ? 1 : 2;            // bytes a number
  static constexpr int kBytes = kPage * HD * kElem;   // of the keys; as many of the values
  static constexpr int kPieces = kBytes / 16;
  __device__ static int key(int s, int d) { return Q8 ? key_elem8(s, d, HD) : key_elem(s, d, HD) * 2; }
  __device__ static int val(int s, int d) { return Q8 ? val_elem8(s, d) : (d * kPage + s) * 2; }
  // slot of 16-byte piece c of the keys (in 64-byte rows), first of the eight slots of
  // piece c of the values
  __device__ static int key_slot(int c) {
    const int row = c >> 2, s8 = row & 7, t = row >> 3 >= HD * kElem / 64;
    return ((s8 >> 2) << 3) | (t << 2) | (s8 & 3);
  }
  __device__ static int val_slot(int c) { return (Q8 ? c >> 4 : c) & 1 ? 8 : 0; }
};

struct KvMoveArgs {
  PoolDev p;
  KvGeom g;
  int pages;  // most pages that n_max tokens touch
  KvMove m;
};

// This workgroup's page: false where it has none.  A request that its pages cannot
// hold is flagged and left out as a whole.
struct Span {
  int b, page, lo, hi, t0;  // slots [lo, hi) are tokens t0 + 0 ..
};
__device__ bool span_of(const KvMoveArgs& a, Span& s) {
  s.b = blockIdx.x / a.pages;
  const int j = blockIdx.x % a.pages;
  const KvMove& m = a.m;
  const int n = m.n ? m.n[s.b] : m.n_max, seq = m.seq ? m.seq[s.b] : m.seq0, pos = m.pos ? m.pos[s.b] : m.pos0;
  if (seq < 0 || seq >= a.p.max_seqs || pos < 0 || n < 0 || n > m.n_max ||
      (int64_t)pos + n > (int64_t)a.p.held[seq] * kPage) {
    if (j == 0 && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(&a.p.scalars[1], ERR_BAD_TOKEN);
    return false;
  }
  const int first = pos / kPage + j, base = first * kPage;
  s.lo = max(pos - base, 0);
  s.hi = min(pos + n - base, kPage);
  s.t0 = base + s.lo - pos;
  if (s.lo >= s.hi) return false;
  s.page = a.p.table[(int64_t)seq * a.p.max_pages + first];
  return true;
}

// R numbers (8, or 4 at head_dim 64) of a row, which may begin at any element (an import's
// source): still one load, which the hardware takes at any address
template <int R>
WAR_DEV void load_row(const bf16_t* p, float* x) {
  typedef uint32_t words_t __attribute__((ext_vector_type(R / 2)));
  typedef words_t any_t __attribute__((aligned(2), may_alias));
  const words_t w = *reinterpret_cast<const any_t*>(p);
#pragma unroll
  for (int i = 0; i < R / 2; ++i) x[2 * i] = lo_f(w[i]), x[2 * i + 1] = hi_f(w[i]);
}

template <bool Q8, int HD>
__global__ void __launch_bounds__(256) k_kv_write(KvMoveArgs a) {
  using O = PageOrder<Q8, HD>;
  constexpr int R = HD / 16;  // dims a thread
  __shared__ __attribute__((aligned(16))) unsigned char s_pg[2 * O::kBytes];
  __shared__ unsigned char s_sc[32];
  Span s;
  if (!span_of(a, s)) return;
  const int kvh = blockIdx.y, slot = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * R;
  if (slot >= s.lo && slot < s.hi) {
    const int64_t row = (int64_t)s.b * a.m.n_max + s.t0 + slot - s.lo;
    float x[2][R];
    load_row<R>(a.m.k + row * a.m.k_stride + kvh * a.m.head_stride + d0, x[0]);
    load_row<R>(a.m.v + row * a.m.v_stride + kvh * a.m.head_stride + d0, x[1]);
    if constexpr (Q8) {
      float top[2];
      bool bad = false;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < R; ++e) {
          m = fmaxf(m, fabsf(x[i][e]));
          bad = bad || !(fabsf(x[i][e]) < INFINITY);
        }
        top[i] = m;
      }
      int any = bad;
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) {
        top[0] = fmaxf(top[0], __shfl_xor(top[0], o, 64));
        top[1] = fmaxf(top[1], __shfl_xor(top[1], o, 64));
        any |= __shfl_xor(any, o, 64);
      }
      const int e0 = block_exp8(top[0]), e1 = block_exp8(top[1]);
      const float f0 = exp2_int(-e0), f1 = exp2_int(-e1);
      // a token with a number that is not finite: NaN keys make NaN scores for the rows
      // that see it, zero values and a zero scale leave all others alone
#pragma unroll
      for (int e = 0; e < R; e += 4) {
        const uint32_t kc = to_e4m3x4(x[0][e] * f0, x[0][e + 1] * f0, x[0][e + 2] * f0, x[0][e + 3] * f0);
        const uint32_t vc = to_e4m3x4(x[1][e] * f1, x[1][e + 1] * f1, x[1][e + 2] * f1, x[1][e + 3] * f1);
        *reinterpret_cast<uint32_t*>(&s_pg[O::key(slot, d0 + e)]) = any ? kNanCode8 * 0x01010101u : kc;
#pragma unroll
        for (int q = 0; q < 4; ++q) s_pg[O::kBytes + O::val(slot, d0 + e + q)] = any ? 0 : (vc >> (8 * q)) & 0xff;
      }
      if (d0 == 0) {
        s_sc[key_scale8(slot)] = any ? 127 : e0 + 127;
        s_sc[val_scale8(slot)] = any ? 0 : e1 + 127;
      }
    } else {
#pragma unroll
      for (int e = 0; e < R; ++e) {
        *reinterpret_cast<bf16_t*>(&s_pg[O::key(slot, d0 + e)]) = f2bf(x[0][e]);
        *reinterpret_cast<bf16_t*>(&s_pg[O::kBytes + O::val(slot, d0 + e)]) = f2bf(x[1][e]);
      }
    }
  }
  __syncthreads();
  const int64_t at = a.g.page_elems(a.m.layer, s.page, kvh, 0) * O::kElem;
  unsigned char* pg = (Q8 ? a.g.q8 : reinterpret_cast<unsigned char*>(a.g.kv)) + at;
  for (int c = threadIdx.x; c < O::kPieces; c += 256) {
    const int sl = O::key_slot(c);
    if (sl >= s.lo && sl < s.hi)
      *reinterpret_cast<uint4*>(pg + c * 16) = *reinterpret_cast<const uint4*>(&s_pg[c * 16]);
  }
  for (int c = threadIdx.x; c < O::kPieces; c += 256) {
    const int s0 = O::val_slot(c), lo = max(s.lo - s0, 0), hi = min(s.hi - s0, 8);
    unsigned char* dst = pg + O::kBytes + c * 16;
    const unsigned char* src = &s_pg[O::kBytes + c * 16];
    if (lo == 0 && hi == 8) {
      *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
    } else {
      for (int i = lo; i < hi; ++i) {
        if constexpr (Q8) {
          dst[i] = src[i];
          dst[8 + i] = src[8 + i];
        } else {
          *reinterpret_cast<bf16_t*>(dst + 2 * i) = *reinterpret_cast<const bf16_t*>(src + 2 * i);
        }
      }
    }
  }
  if constexpr (Q8) {
    unsigned char* sc = a.g.scale + a.g.scale_bytes(a.m.layer, s.page, kvh);
    if (threadIdx.x < 2 * kPage) {
      const int sl = threadIdx.x & 15, i = threadIdx.x < kPage ? key_scale8(sl) : val_scale8(sl);
      if (sl >= s.lo && sl < s.hi) sc[i] = s_sc[i];
    }
  }
}

template <bool Q8, int HD>
__global__ void __launch_bounds__(256) k_kv_read(KvMoveArgs a) {
  using O = PageOrder<Q8, HD>;
  constexpr int R = HD / 16;
  __shared__ __attribute__((aligned(16))) unsigned char s_pg[2 * O::kBytes];
  Span s;
  if (!span_of(a, s)) return;
  const int kvh = blockIdx.y, slot = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * R;
  const int64_t at = a.g.page_elems(a.m.layer, s.page, kvh, 0) * O::kElem;
  const unsigned char* pg = (Q8 ? a.g.q8 : reinterpret_cast<const unsigned char*>(a.g.kv)) + at;
  for (int c = threadIdx.x; c < 2 * O::kPieces; c += 256)
    *reinterpret_cast<uint4*>(&s_pg[c * 16]) = *reinterpret_cast<const uint4*>(pg + c * 16);
  float ks = 0.f, vs = 0.f;
  if constexpr (Q8) {
    const unsigned char* sc = a.g.scale + a.g.scale_bytes(a.m.layer, s.page, kvh);
    ks = scale_of<0>(sc[key_scale8(slot)]);
    vs = scale_of<0>(sc[val_scale8(slot)]);  // 0: not finite
  }
  __syncthreads();
  if (slot < s.lo || slot >= s.hi) return;
  const int64_t row = (int64_t)s.b * a.m.n_max + s.t0 + slot - s.lo;
  bf16_t* kd = a.m.k + row * a.m.k_stride + kvh * a.m.head_stride + d0;
  bf16_t* vd = a.m.v + row * a.m.v_stride + kvh * a.m.head_stride + d0;
  const bool not_finite = Q8 && vs == 0.f;
#pragma unroll
  for (int e = 0; e < R; e += 4) {
    uint2 ko, vo;
    if constexpr (Q8) {
      const uint32_t kc = *reinterpret_cast<const uint32_t*>(&s_pg[O::key(slot, d0 + e)]);
      uint32_t vc = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) vc |= (uint32_t)s_pg[O::kBytes + O::val(slot, d0 + e + q)] << (8 * q);
      if (not_finite) vc = kNanCode8 * 0x01010101u;
      ko = make_uint2(from_e4m3x2<false>(kc, ks), from_e4m3x2<true>(kc, ks));
      const float f = not_finite ? 1.f : vs;
      vo = make_uint2(from_e4m3x2<false>(vc, f), from_e4m3x2<true>(vc, f));
    } else {
      ko = *reinterpret_cast<const uint2*>(&s_pg[O::key(slot, d0 + e)]);
      uint32_t w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) w[q] = *reinterpret_cast<const bf16_t*>(&s_pg[O::kBytes + O::val(slot, d0 + e + q)]);
      vo = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    }
    *reinterpret_cast<uint2*>(kd + e) = ko;
    *reinterpret_cast<uint2*>(vd + e) = vo;
  }
}

}  // namespace

void launch_kv_move(bool write, const PoolDev& p, const KvGeom& g, const KvMove& m, hipStream_t st) {
  const KvMoveArgs a{p, g, cdiv_i(m.n_max + kPage - 1, kPage), m};
  const dim3 grid(m.B * a.pages, g.n_kv_heads);
  auto go = [&](auto hd) {
    constexpr int HD = decltype(hd)::value;
    if (g.q8) {
      if (write) k_kv_write<true, HD><<<grid, 256, 0, st>>>(a);
      else k_kv_read<true, HD><<<grid, 256, 0, st>>>(a);
    } else {
      if (write) k_kv_write<false, HD><<<grid, 256, 0, st>>>(a);
      else k_kv_read<false, HD><<<grid, 256, 0, st>>>(a);
    }
  };
  if (g.head_dim == 128) go(std::integral_constant<int, 128>{});
  else go(std::integral_constant<int, 64>{});
}
