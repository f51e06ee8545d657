// Logits of a step's rows under their requests' constraints, the greedy token of each
// row, and the token counts that the penalties read (gfx950).
//
// Row i of a request follows its counted text, the pending token and the drafts on the
// way to row i; n(v) is how often token v occurs there and s(v) whether it does, or in
// the prompt.  A logit z of token v becomes
//   z += the bias entries of v;  s(v): z = z > 0 ? z / r : z r;  z -= f n(v);
//   n(v) > 0: z -= p;  -inf where the row's mask excludes v
// in fp32, each operation rounded by itself (no fused multiply-adds), so that any order
// of rows, chunks and batches gives the same bits.
//
// Memory bounds it: a logit is read and written once, its count (16 bits) once a
// request.  A workgroup takes 2048 ids of a request's rows: counts and biases stay
// in registers, the few tokens of the rows themselves are added where they fall into the
// chunk (a uniform test), and the next row's logits are in flight while a row is done.
// It leaves the best id of every 128 (as the LM head does without constraints), from
// which the greedy token, the acceptance and the sampler start.
// 192 rows of 151,936 ids under everything (255 MB): 46 us, 5.5 TB/s, and 4.6 for the
// greedy tokens.  The divisions as such, and each row looking through the biases, took 76.
#include "kernels.h"

#pragma clang fp contract(off)

namespace {

constexpr int kThreads = 256, kUnits = 2, kIds = kThreads * 4 * kUnits;  // ids a workgroup
constexpr int kNodes = 64;      // rows of a request
constexpr int kMaxBias = 1024;  // its bias entries
constexpr int kNone = 0x7fffffff;

typedef float f32x4_t __attribute__((ext_vector_type(4)));

// A request's penalties.  z / r is the quotient from the reciprocal with one residual step
// (Markstein 1990: correctly rounded where nothing over- or underflows, which the ranges
// here exclude), a third of a division's instructions.
struct Penalty {
  float r, rinv, f, p;
  bool plain;  // r in [2^-40, 2^40]
  __device__ void set(const ConstrainArgs& a, int seq) {
    r = a.repetition ? a.repetition[seq] : 1.f;
    f = a.frequency ? a.frequency[seq] : 0.f;
    p = a.presence ? a.presence[seq] : 0.f;
    rinv = 1.f / r;
    plain = r >= 0x1p-40f && r <= 0x1p40f;
  }
  // c: twice the occurrences, plus one for the prompt; not 0
  __device__ float operator()(float v, int c) const {
    const float q = v * rinv;
    float d = fmaf(fmaf(-q, r, v), rinv, q);
    if (!(plain && v >= 0x1p-60f && v <= 0x1p60f)) d = v > 0.f ? v / r : v * r;
    d -= f * (float)(c >> 1);
    return c > 1 ? d - p : d;
  }
};

template <bool VEC>
WAR_DEV f32x4_t load4(const float* z, int col, int V) {
  if constexpr (VEC) return col < V ? *reinterpret_cast<const f32x4_t*>(z + col) : f32x4_t{0.f, 0.f, 0.f, 0.f};
  f32x4_t x;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = col + e < V ? z[col + e] : 0.f;
  return x;
}

template <bool VEC>
__global__ void __launch_bounds__(kThreads) k_constrain(ConstrainArgs a) {
  __shared__ int s_tok[kNodes], s_mask[kNodes];
  __shared__ unsigned long long s_path[kNodes];
  __shared__ int s_hits, s_entry[kMaxBias], s_at[kMaxBias];
  __shared__ float s_sum[kMaxBias];
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int c0 = blockIdx.x * kIds, c1 = min(a.V, c0 + kIds);
  const int kp1 = a.k_max + 1;
  const int n = a.ntok ? a.ntok[b] : a.draft_lens ? min(max(a.draft_lens[b], 0), a.k_max) + 1 : kp1;
  const int seq = a.seq_ids[b];
  const int64_t row0 = (int64_t)b * kp1;
  const int nblk = (a.V + 127) / 128, words = (a.V + 31) / 32;
  const int step = gridDim.z;  // this workgroup's rows: blockIdx.z, + step, ...
  int i = blockIdx.z;
  if (i >= n) return;
  if (seq < 0 || seq >= a.n_seqs) {  // no such request: no token in any row
    if (a.best_v)
      for (; i < n; i += step)
        for (int q = c0 / 128 + tid; q < (c1 + 127) / 128; q += kThreads) {
          a.best_v[(row0 + i) * nblk + q] = -INFINITY;
          a.best_i[(row0 + i) * nblk + q] = kNone;
        }
    return;
  }
  if (tid == 0) s_hits = 0;
  __syncthreads();
  // everything that hangs on nothing else is requested first: the first row's logits, the
  // counts, the penalties
  int col[kUnits], cnt[kUnits][4];
  f32x4_t bias[kUnits], z[kUnits];
  const uint16_t* crow = a.counts ? a.counts + (int64_t)seq * a.V : nullptr;
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    col[u] = c0 + (u * kThreads + tid) * 4;
    bias[u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    z[u] = load4<VEC>(a.logits + (row0 + i) * a.stride, col[u], a.V);
  }
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
#pragma unroll
    for (int e = 0; e < 4; ++e) cnt[u][e] = 0;
    if (crow) {
      if constexpr (VEC) {
        if (col[u] < a.V) {
          const uint2 c = *reinterpret_cast<const uint2*>(crow + col[u]);
          cnt[u][0] = c.x & 0xffff;
          cnt[u][1] = c.x >> 16;
          cnt[u][2] = c.y & 0xffff;
          cnt[u][3] = c.y >> 16;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (col[u] + e < a.V) cnt[u][e] = crow[col[u] + e];
      }
    }
  }
  Penalty pen;
  pen.set(a, seq);
  // the rows' tokens (row j's own and its ancestors' are its text) and masks
  if (tid < n) {
    s_tok[tid] = tid == 0 ? a.last_tokens[b] : a.draft_tokens[(int64_t)b * a.k_max + tid - 1];
    int m = -1;  // (a mask that is not there allows nothing: -2)
    if (a.masks) {
      m = a.mask_index ? a.mask_index[row0 + tid] : (int)(row0 + tid);
      m = m >= a.n_masks ? -2 : max(m, -1);
    }
    s_mask[tid] = m;
    unsigned long long path = a.parents ? 1ull << tid : ~0ull >> (63 - tid);
    if (a.parents)
      for (int j = tid; j > 0;) {
        int q = a.parents[(int64_t)b * a.k_max + j - 1];
        if (q < 0 || q >= j) q = j - 1;  // as the step reads it
        path |= 1ull << q;
        j = q;
      }
    s_path[tid] = path;
  }
  // the bias entries of this chunk, in any order (few of them: the same id twice is looked
  // for among them alone)
  const int32_t* bid = a.bias_ids + (int64_t)seq * a.n_bias;
  const float* bval = a.bias_values + (int64_t)seq * a.n_bias;
  for (int e = tid; e < a.n_bias; e += kThreads) {
    const int id = bid[e];
    if (id >= c0 && id < c1) {
      const int at = atomicAdd(&s_hits, 1);
      s_entry[at] = e;
      s_at[at] = id - c0;
    }
  }
  __syncthreads();
  const int hits = s_hits;
  if (hits) {
    // an id's first entry adds up all of them, in list order
    for (int h = tid; h < hits; h += kThreads) {
      const int e = s_entry[h], id = s_at[h];
      bool first = true, more = false;
      for (int q = 0; q < hits; ++q)
        if (s_at[q] == id) {
          first = first && s_entry[q] >= e;
          more = more || s_entry[q] > e;
        }
      float sum = first ? bval[e] : 0.f;
      if (first && more)
        for (int q = e + 1; q < a.n_bias; ++q)
          if (bid[q] == c0 + id) sum += bval[q];
      s_sum[h] = sum;
    }
    __syncthreads();
    for (int h = 0; h < hits; ++h) {
      const int d = s_at[h];
      if (((d >> 2) & (kThreads - 1)) == tid) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (d == (u * kThreads + tid) * 4 + e) bias[u][e] += s_sum[h];
      }
    }
  }
  // the rows' tokens that lie in this chunk (n <= 64: lane j looks at token j)
  const unsigned long long here = __ballot(lane < n && s_tok[min(lane, n - 1)] >= c0 && s_tok[min(lane, n - 1)] < c1);
  auto mask_words = [&](int j, uint32_t (&w)[kUnits]) {
    const int m = __builtin_amdgcn_readfirstlane(s_mask[j]);
    const uint32_t* mrow = a.masks + (int64_t)max(m, 0) * words;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) w[u] = m == -2 ? 0u : m >= 0 && col[u] < a.V ? mrow[col[u] >> 5] : ~0u;
  };
  uint32_t word[kUnits];
  mask_words(i, word);
#pragma unroll
  for (int u = 0; u < kUnits; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      cnt[u][e] = (cnt[u][e] & 0x7fff) * 2 + (cnt[u][e] >> 15);  // prompt bit last
    }

  for (; i < n; i += step) {
    const int64_t row = row0 + i;
    f32x4_t next[kUnits];
    uint32_t next_word[kUnits];
    if (i + step < n) {
#pragma unroll
      for (int u = 0; u < kUnits; ++u) next[u] = load4<VEC>(a.logits + (row + step) * a.stride, col[u], a.V);
      mask_words(i + step, next_word);
    }
    const unsigned long long add = here & s_path[i];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      int c[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = cnt[u][e];
      for (unsigned long long q = add; q; q &= q - 1) {
        const int d = s_tok[__ffsll((long long)q) - 1] - col[u];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (d == e) c[e] += 2;
      }
      f32x4_t x = z[u];
      uint32_t allow = word[u] >> (col[u] & 31);
      if constexpr (VEC)
        allow = col[u] < a.V ? allow : 0u;
      else
        allow &= col[u] + 4 <= a.V ? 15u : col[u] < a.V ? (1u << (a.V - col[u])) - 1u : 0u;
      float best = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float v = x[e];
        v += bias[u][e];
        if (c[e]) v = pen(v, c[e]);
        // excluded: -inf, by a mask of the id's bit
        const uint32_t keep = (uint32_t)((int)(allow << (31 - e)) >> 31);
        x[e] = __uint_as_float((__float_as_uint(v) & keep) | (0xff800000u & ~keep));
        best = fmaxf(best, x[e]);  // (drops NaN)
      }
      if (a.out) {
        float* o = a.out + row * a.out_stride;
        if constexpr (VEC) {
          if (col[u] < a.V) *reinterpret_cast<f32x4_t*>(o + col[u]) = x;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col[u] + e < a.V) o[col[u] + e] = x[e];
        }
      }
      if (a.best_v) {
        // 128 ids are the 32 lanes of half a wave, ascending: the lowest lane that holds
        // the maximum has its lowest id; a maximum of -inf counts where an id is allowed
        float mx = best;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
        int at = kNone;
#pragma unroll
        for (int e = 3; e >= 0; --e)
          if (x[e] == mx && (mx > -INFINITY || ((allow >> e) & 1u))) at = col[u] + e;
        const unsigned long long half = lane < 32 ? 0xffffffffull : 0xffffffffull << 32;
        const unsigned long long eq = __ballot(at != kNone) & half;
        bool nan = false;
        if (a.nan_max) nan = (__ballot(x[0] != x[0] || x[1] != x[1] || x[2] != x[2] || x[3] != x[3]) & half) != 0;
        const int q = (c0 + u * kThreads * 4 + (tid & ~31) * 4) / 128;
        if (q < nblk && (eq ? __ffsll((long long)eq) - 1 == lane : (lane & 31) == 0)) {
          a.best_v[row * nblk + q] = nan ? __builtin_nanf("") : mx;
          a.best_i[row * nblk + q] = at;
        }
      }
      z[u] = next[u];
      word[u] = next_word[u];
    }
  }
}

// Greedy token of each row from the best of its 128-id blocks: the lowest id among the
// largest, -1 where no block has one (`finite`: or only -inf).  A workgroup a row; a
// thread's blocks ascend, so that the first of equals has the lowest id.
__global__ void __launch_bounds__(256) k_greedy(ConstrainArgs a, int32_t* greedy, bool finite) {
  __shared__ float s_v[4];
  __shared__ int s_i[4];
  const int kp1 = a.k_max + 1, nblk = (a.V + 127) / 128, lane = threadIdx.x & 63;
  const int r = blockIdx.x, b = r / kp1;
  const int n = a.ntok ? a.ntok[b] : a.draft_lens ? min(max(a.draft_lens[b], 0), a.k_max) + 1 : kp1;
  if (r % kp1 >= n) return;
  float v = -INFINITY;
  int idx = kNone;
  auto better = [&](float ov, int oi) {
    if (oi != kNone && (idx == kNone || ov > v || (ov == v && oi < idx))) {
      v = ov;
      idx = oi;
    }
  };
  for (int c0 = threadIdx.x; c0 < nblk; c0 += 256 * 8) {
    float bv[8];
    int bi[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int c = c0 + 256 * u;
      bv[u] = c < nblk ? a.best_v[(int64_t)r * nblk + c] : 0.f;
      bi[u] = c < nblk ? a.best_i[(int64_t)r * nblk + c] : kNone;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) better(bv[u], bi[u]);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) better(__shfl_xor(v, o, 64), __shfl_xor(idx, o, 64));
  if (lane == 0) {
    s_v[threadIdx.x >> 6] = v;
    s_i[threadIdx.x >> 6] = idx;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < 4; ++w) better(s_v[w], s_i[w]);
  greedy[r] = idx == kNone || (finite && v == -INFINITY) ? -1 : idx;
}

// A request's row of the counts begins: bit 15 for each token of its prompt, no
// occurrences.  A workgroup takes 16384 ids: the prompt's tokens among them as bits in
// LDS, then the row's numbers, written once.  Every workgroup of a request reads its whole
// prompt (from L2): 64 prompts of 8192 tokens into 151,936 ids 8.1 us, of which the 19 MB
// written are 4.
constexpr int kSlice = 16384;
template <bool VEC>
__global__ void __launch_bounds__(256) k_counts_begin(uint16_t* counts, int V, int n_seqs, const int32_t* seq_ids,
                                                      const int32_t* tokens, int n_tokens, const int32_t* offsets) {
  __shared__ uint32_t s_bits[kSlice / 32];
  const int b = blockIdx.y, c0 = blockIdx.x * kSlice, c1 = min(V, c0 + kSlice);
  const int seq = seq_ids[b];
  if (seq < 0 || seq >= n_seqs) return;
  for (int i = threadIdx.x; i < kSlice / 32; i += 256) s_bits[i] = 0;
  __syncthreads();
  const int t1 = min(offsets[b + 1], n_tokens);
  for (int64_t i0 = max(offsets[b], 0) + (int64_t)threadIdx.x; i0 < t1; i0 += 256 * 16) {
    int t[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) t[u] = i0 + 256 * u < t1 ? tokens[i0 + 256 * u] : -1;
#pragma unroll
    for (int u = 0; u < 16; ++u)
      if (t[u] >= c0 && t[u] < c1) atomicOr(&s_bits[(t[u] - c0) >> 5], 1u << ((t[u] - c0) & 31));
  }
  __syncthreads();
  uint16_t* row = counts + (int64_t)seq * V;
  if constexpr (VEC) {
    for (int c = c0 + threadIdx.x * 8; c < c1; c += 256 * 8) {
      const uint32_t w = s_bits[(c - c0) >> 5] >> ((c - c0) & 31);
      auto two = [w](int e) { return ((w >> e) & 1u) << 15 | ((w >> (e + 1)) & 1u) << 31; };
      *reinterpret_cast<uint4*>(row + c) = make_uint4(two(0), two(2), two(4), two(6));
    }
  } else {
    for (int c = c0 + threadIdx.x; c < c1; c += 256) row[c] = (s_bits[(c - c0) >> 5] >> ((c - c0) & 31) & 1u) << 15;
  }
}

// A request's tokens are counted: the first occurrence of a token among them adds all of
// its occurrences, so that no two threads touch one number and nothing hangs on their
// order.
__global__ void __launch_bounds__(256) k_counts_add(uint16_t* counts, int V, int n_seqs, const int32_t* seq_ids,
                                                    const int32_t* first, const int32_t* tokens, int n_max,
                                                    const int32_t* path, const int32_t* lens) {
  extern __shared__ int s_tok[];
  const int b = blockIdx.x;
  const int seq = seq_ids[b], len = lens ? min(lens[b], n_max) : n_max;
  if (seq < 0 || seq >= n_seqs || len < 0) return;
  const int f = first ? 1 : 0, n = len + f;
  for (int i = threadIdx.x; i < n; i += 256) {
    int j = i - f;
    if (j >= 0 && path) j = path[(int64_t)b * n_max + j] - 1;
    s_tok[i] = i < f ? first[b] : j >= 0 && j < n_max ? tokens[(int64_t)b * n_max + j] : -1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 256) {
    const int t = s_tok[i];
    if (t < 0 || t >= V) continue;
    int times = 1;
    bool mine = true;
    for (int q = 0; q < n; ++q) {
      if (q < i && s_tok[q] == t) mine = false;
      if (q > i && s_tok[q] == t) ++times;
    }
    if (!mine) continue;
    uint16_t* at = counts + (int64_t)seq * V + t;
    *at = (uint16_t)((*at & 0x8000) | min((*at & 0x7fff) + times, 0x7fff));
  }
}

}  // namespace

void launch_constrain(const ConstrainArgs& a, hipStream_t st) {
  // a workgroup takes all of a request's rows where that fills the chip (its counts are read
  // once), fewer otherwise
  const int chunks = cdiv_i(a.V, kIds), most = std::min(a.k_max + 1, 65535);
  int rows = std::max(1, std::min(most, cdiv_i(2048, chunks * a.B)));
  const dim3 grid(chunks, a.B, rows);
  auto quad = [](const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; };
  // 16-byte accesses where every row of every array allows them (192 rows of 151,936 ids 46
  // us, of 151,937 ids 66)
  const bool vec = a.V % 4 == 0 && a.stride % 4 == 0 && quad(a.logits, 16) && quad(a.counts, 8) &&
                   (!a.out || (a.out_stride % 4 == 0 && quad(a.out, 16)));
  if (vec) k_constrain<true><<<grid, kThreads, 0, st>>>(a);
  else k_constrain<false><<<grid, kThreads, 0, st>>>(a);
}
void launch_greedy(const ConstrainArgs& a, int32_t* greedy, bool finite, hipStream_t st) {
  k_greedy<<<a.B * (a.k_max + 1), 256, 0, st>>>(a, greedy, finite);
}
void launch_counts_begin(uint16_t* counts, int V, int n_seqs, int B, const int32_t* seq_ids, const int32_t* tokens,
                         int n_tokens, const int32_t* offsets, hipStream_t st) {
  const dim3 grid(cdiv_i(V, kSlice), B);
  if (V % 8 == 0 && (reinterpret_cast<uintptr_t>(counts) & 15) == 0)
    k_counts_begin<true><<<grid, 256, 0, st>>>(counts, V, n_seqs, seq_ids, tokens, n_tokens, offsets);
  else
    k_counts_begin<false><<<grid, 256, 0, st>>>(counts, V, n_seqs, seq_ids, tokens, n_tokens, offsets);
}
void launch_counts_add(uint16_t* counts, int V, int n_seqs, int B, const int32_t* seq_ids, const int32_t* first,
                       const int32_t* tokens, int n_max, const int32_t* path, const int32_t* lens, hipStream_t st) {
  k_counts_add<<<B, 256, (n_max + 1) * 4, st>>>(counts, V, n_seqs, seq_ids, first, tokens, n_max, path, lens);
}
