// Pages as the kernels that move given tokens' keys and values see them: a workgroup
// takes one page of one kv-head, which passes through LDS in its own order.
#pragma once

#include "kernels.h"

constexpr int kPageSlots = 16;

// Element (bf16) or byte (e4m3) of a page's keys and values.
template <bool Q8, int HD>
struct PageOrder {
  static constexpr int kElem = Q8 ? 1 : 2;            // bytes a number
  static constexpr int kBytes = kPageSlots * HD * kElem;   // of the keys; as many of the values
  static constexpr int kPieces = kBytes / 16;
  __device__ static int key(int s, int d) { return Q8 ? key_elem8(s, d, HD) : key_elem(s, d, HD) * 2; }
  __device__ static int val(int s, int d) { return Q8 ? val_elem8(s, d) : (d * kPageSlots + s) * 2; }
  // slot of 16-byte piece c of the keys (in 64-byte rows), first of the eight slots of
  // piece c of the values
  __device__ static int key_slot(int c) {
    const int row = c >> 2, s8 = row & 7, t = row >> 3 >= HD * kElem / 64;
    return ((s8 >> 2) << 3) | (t << 2) | (s8 & 3);
  }
  __device__ static int val_slot(int c) { return (Q8 ? c >> 4 : c) & 1 ? 8 : 0; }
};

// The slots [lo, hi) of a page that a workgroup moves: tokens t0 + 0 .. of request b.
struct PageSpan {
  int b, page, lo, hi, t0;
};
// Page j of the pages that request b's n tokens from `pos` on touch: false where it holds
// none of them.  A request that its pages cannot hold is flagged (by one thread) and
// left out as a whole.
WAR_DEV bool page_span(const PoolDev& p, int b, int j, int seq, int pos, int n, int n_max, bool flags, PageSpan& s) {
  s.b = b;
  if (seq < 0 || seq >= p.max_seqs || pos < 0 || n < 0 || n > n_max ||
      (int64_t)pos + n > (int64_t)p.held[seq] * kPageSlots) {
    if (flags) atomicOr(&p.scalars[1], ERR_BAD_TOKEN);
    return false;
  }
  const int first = pos / kPageSlots + j, base = first * kPageSlots;
  s.lo = max(pos - base, 0);
  s.hi = min(pos + n - base, kPageSlots);
  s.t0 = base + s.lo - pos;
  if (s.lo >= s.hi) return false;
  s.page = p.table[(int64_t)seq * p.max_pages + first];
  return true;
}

// The tokens [lo, hi) of a page and kv-head from LDS (s_pg in the page's order, s_sc its
// scale bytes) to memory, by T threads after a barrier.  Both sides move 16-byte pieces;
// of a piece that covers other tokens too only the new ones' bytes are written.
template <bool Q8, int HD, int T>
WAR_DEV void store_page(const KvGeom& g, int layer, int kvh, const PageSpan& s, const unsigned char* s_pg,
                        const unsigned char* s_sc) {
  using O = PageOrder<Q8, HD>;
  const int64_t at = g.page_elems(layer, s.page, kvh, 0) * O::kElem;
  unsigned char* pg = (Q8 ? g.q8 : reinterpret_cast<unsigned char*>(g.kv)) + at;
  for (int c = threadIdx.x; c < O::kPieces; c += T) {
    const int sl = O::key_slot(c);
    if (sl >= s.lo && sl < s.hi)
      *reinterpret_cast<uint4*>(pg + c * 16) = *reinterpret_cast<const uint4*>(&s_pg[c * 16]);
  }
  for (int c = threadIdx.x; c < O::kPieces; c += T) {
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
    unsigned char* sc = g.scale + g.scale_bytes(layer, s.page, kvh);
    if (threadIdx.x < 2 * kPageSlots) {
      const int sl = threadIdx.x & 15, i = threadIdx.x < kPageSlots ? key_scale8(sl) : val_scale8(sl);
      if (sl >= s.lo && sl < s.hi) sc[i] = s_sc[i];
    }
  }
}
