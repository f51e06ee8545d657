// C-ABI runtime of a decoder layer's other operators: rows into microscaled codes, the
// products with 4-bit weights, rotary positions into the cache.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "../../include/war_debug.h"
#include "api.h"
#include "mx.h"

struct war_linear {
  int N, K;
  uint8_t* mem;  // codes | scale words | bias
  const uint32_t* scales() const { return reinterpret_cast<const uint32_t*>(mem + mx_code_bytes(N, K)); }
  const bf16_t* bias() const { return reinterpret_cast<const bf16_t*>(scales() + mx_scale_words(N, K)); }
};

namespace {

#define CHECK(cond, msg)                              \
  do {                                                \
    if (!(cond)) return api_fail(WAR_ERR_INVALID_ARG, msg); \
  } while (0)
#define HIPCHK(x)                                                              \
  do {                                                                         \
    hipError_t e_ = (x);                                                       \
    if (e_ != hipSuccess) return api_fail(WAR_ERR_HIP, hipGetErrorString(e_)); \
  } while (0)
#define WARCHK(x)                      \
  do {                                 \
    const war_status s_ = (x);         \
    if (s_ != WAR_OK) return s_;       \
  } while (0)

bool aligned(const void* p, int n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

war_status check_size(int64_t rows, int64_t cols) {
  CHECK(rows >= 0 && rows <= 1 << 20, "rows out of range [0, 2^20]");
  CHECK(cols >= 32 && cols <= 65536 && cols % 32 == 0, "cols must be a multiple of 32 in [32, 65536]");
  CHECK(rows * cols <= (int64_t)1 << 34, "more than 2^34 numbers");
  return WAR_OK;
}
// any_place: codes and scales need no alignment (a matrix that is only repacked)
war_status check_mx(const war_mx* m, bool any_place = false) {
  CHECK(m, "null matrix");
  CHECK(m->format == WAR_MX_E4M3 || m->format == WAR_MX_E2M1, "unknown format");
  WARCHK(check_size(m->rows, m->cols));
  if (m->rows == 0) return WAR_OK;
  CHECK(m->codes && m->scales, "null codes or scales");
  CHECK(m->code_stride >= (m->format == WAR_MX_E4M3 ? m->cols : m->cols / 2) && m->scale_stride >= m->cols / 32,
        "strides must hold a row");
  CHECK(any_place || (aligned(m->codes, 16) && m->code_stride % 16 == 0), "codes must lie at multiples of 16 bytes");
  CHECK(any_place || (aligned(m->scales, 4) && m->scale_stride % 4 == 0), "scales must lie at multiples of 4 bytes");
  return WAR_OK;
}
war_status check_rows(const void* p, int64_t stride, int64_t cols) {
  CHECK(p && aligned(p, 16), "rows must be 16-byte aligned");
  CHECK(stride >= cols && stride % 8 == 0, "strides must hold a row and be multiples of 8");
  return WAR_OK;
}
bool is_type(int t) { return t == WAR_BF16 || t == WAR_F32; }
MxRef ref(const war_mx& m) { return {static_cast<uint8_t*>(m.codes), m.scales, m.code_stride, m.scale_stride}; }
int fmt(const war_mx& m) { return m.format - WAR_MX_E4M3; }

}  // namespace

extern "C" {

war_status war_residual_norm(int32_t rows, int32_t cols, const void* x, int64_t x_stride, void* h, int64_t h_stride,
                             int32_t h_type, const void* gain, float eps, const war_mx* mx, void* y, int64_t y_stride,
                             void* stream) {
  WARCHK(check_size(rows, cols));
  CHECK(is_type(h_type), "h_type must be WAR_BF16 or WAR_F32");
  CHECK(eps >= 0.f && std::isfinite(eps), "eps must be finite and not negative");
  CHECK((mx != nullptr) != (y != nullptr) || (rows == 0 && !mx), "one of mx and y is wanted");  // (no rows have no address)
  if (mx) {
    WARCHK(check_mx(mx));
    CHECK(mx->rows == rows && mx->cols == cols, "mx has another size");
  }
  if (rows == 0) return WAR_OK;
  if (x) WARCHK(check_rows(x, x_stride, cols));
  WARCHK(check_rows(h, h_stride, cols));
  if (y) WARCHK(check_rows(y, y_stride, cols));
  CHECK(!x || x != y || x_stride == y_stride, "in place, the strides must be the same");
  CHECK(gain && aligned(gain, 16), "gain must be 16-byte aligned");
  NormArgs a{};
  a.rows = rows;
  a.cols = cols;
  a.x = static_cast<const bf16_t*>(x);
  a.h = h;
  a.gain = static_cast<const bf16_t*>(gain);
  a.y = static_cast<bf16_t*>(y);
  if (mx) a.mx = ref(*mx);
  a.x_stride = x_stride;
  a.h_stride = h_stride;
  a.y_stride = y_stride;
  a.eps = eps;
  launch_residual_norm_mx(a, h_type == WAR_F32, mx ? fmt(*mx) : -1, static_cast<hipStream_t>(stream));
  HIPCHK(hipGetLastError());
  return WAR_OK;
}

war_status war_quantize(const war_mx* mx, const void* x, int64_t x_stride, const void* gate, int64_t gate_stride,
                        int32_t type, void* stream) {
  WARCHK(check_mx(mx));
  CHECK(is_type(type), "type must be WAR_BF16 or WAR_F32");
  if (mx->rows == 0) return WAR_OK;
  WARCHK(check_rows(x, x_stride, mx->cols));
  if (gate) WARCHK(check_rows(gate, gate_stride, mx->cols));
  const QuantArgs a{mx->rows, mx->cols, x, gate, x_stride, gate_stride, ref(*mx)};
  launch_quantize(a, type == WAR_F32, fmt(*mx), static_cast<hipStream_t>(stream));
  HIPCHK(hipGetLastError());
  return WAR_OK;
}

war_status war_dequantize(const war_mx* mx, void* y, int64_t y_stride, int32_t type, void* stream) {
  WARCHK(check_mx(mx));
  CHECK(is_type(type), "type must be WAR_BF16 or WAR_F32");
  if (mx->rows == 0) return WAR_OK;
  WARCHK(check_rows(y, y_stride, mx->cols));
  const DequantArgs a{mx->rows, mx->cols, ref(*mx), y, y_stride};
  launch_dequantize(a, type == WAR_F32, fmt(*mx), static_cast<hipStream_t>(stream));
  HIPCHK(hipGetLastError());
  return WAR_OK;
}

war_status war_linear_create(const war_mx* w, const void* bias, void* stream, war_linear** out) {
  CHECK(out, "null out");
  *out = nullptr;
  WARCHK(check_mx(w, true));
  CHECK(w->rows >= 1, "no rows");
  if (w->format != WAR_MX_E2M1) return api_fail(WAR_ERR_UNSUPPORTED, "weights must be WAR_MX_E2M1");
  CHECK(!bias || aligned(bias, 2), "bias must be 2-byte aligned");
  hipStream_t st = static_cast<hipStream_t>(stream);
  war_linear* l = new (std::nothrow) war_linear{w->rows, w->cols, nullptr};
  if (!l) return api_fail(WAR_ERR_HIP, "out of host memory");
  const int64_t n_bias = (int64_t)mx_tiles(l->N) * 32;
  hipError_t e = hipMalloc(reinterpret_cast<void**>(&l->mem),
                           mx_code_bytes(l->N, l->K) + 4 * mx_scale_words(l->N, l->K) + 2 * n_bias);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    delete l;
    return api_fail(WAR_ERR_HIP, "weight allocation failed");
  }
  launch_mx_pack(ref(*w), l->N, l->K, l->mem, const_cast<uint32_t*>(l->scales()), st);
  e = hipGetLastError();
  bf16_t* b = const_cast<bf16_t*>(l->bias());
  if (e == hipSuccess) e = hipMemsetAsync(b, 0, 2 * n_bias, st);
  if (e == hipSuccess && bias) e = hipMemcpyAsync(b, bias, 2 * (int64_t)l->N, hipMemcpyDeviceToDevice, st);
  const hipError_t es = hipStreamSynchronize(st);
  if (e == hipSuccess) e = es;
  if (e != hipSuccess) {
    war_linear_destroy(l);
    return api_fail(WAR_ERR_HIP, hipGetErrorString(e));
  }
  *out = l;
  return WAR_OK;
}

void war_linear_destroy(war_linear* l) {
  if (!l) return;
  (void)hipFree(l->mem);
  delete l;
}

static war_status run_linear(const war_linear* l, const war_mx* x, void* y, int64_t y_stride, int32_t y_type, int shape,
                             void* stream) {
  CHECK(l, "null linear");
  WARCHK(check_mx(x));
  CHECK(x->cols == l->K, "x has another number of columns than the weights");
  CHECK(is_type(y_type), "y_type must be WAR_BF16 or WAR_F32");
  if (x->rows == 0) return WAR_OK;
  const int size = y_type == WAR_F32 ? 4 : 2;
  CHECK(y && aligned(y, size), "y is null or not aligned to its type");
  CHECK(y_stride >= l->N, "y_stride must hold a row");
  CHECK(x->code_stride <= 1 << 22 && x->scale_stride <= 1 << 22, "strides of x beyond 2^22");  // (32-bit offsets in a tile)
  MxGemmArgs a{};
  a.M = x->rows;
  a.N = l->N;
  a.K = l->K;
  a.x = ref(*x);
  a.w = l->mem;
  a.ws = l->scales();
  a.bias = l->bias();
  a.y = y;
  a.y_stride = y_stride;
  a.scale16 = x->cols % 512 == 0 && x->scale_stride % 16 == 0 && aligned(x->scales, 16);
  if (!launch_mx_gemm(a, fmt(*x), y_type == WAR_F32, shape, static_cast<hipStream_t>(stream)))
    return api_fail(WAR_ERR_UNSUPPORTED, "more workgroups than a launch holds");
  HIPCHK(hipGetLastError());
  return WAR_OK;
}

war_status war_linear_run(const war_linear* l, const war_mx* x, void* y, int64_t y_stride, int32_t y_type, void* stream) {
  return run_linear(l, x, y, y_stride, y_type, -1, stream);
}

war_status war_debug_linear(const war_linear* l, const war_mx* x, void* y, int64_t y_stride, int32_t y_type, int32_t shape,
                            void* stream) {
  CHECK(shape >= 0 && shape < kMxShapes, "shape out of range");
  return run_linear(l, x, y, y_stride, y_type, shape, stream);
}

int32_t war_debug_linear_shape(int32_t M, int32_t N, int32_t K, int32_t x_format, int32_t y_type) {
  return plan_mx_gemm(M, N, K, x_format - WAR_MX_E4M3, y_type == WAR_F32);
}

war_status war_rope_write(war_kv_pool* p, int32_t layer, const war_rope* rope, int32_t B, const int32_t* seq_ids,
                          const int32_t* pos0, int32_t n_max, const int32_t* n_lens, const int32_t* positions,
                          const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k,
                          int64_t k_stride, const void* v, int64_t v_stride, void* stream) {
  CHECK(p, "null pool");
  CHECK(rope && rope->freqs, "null rope or freqs");
  const PoolView pv = pool_view(p);
  const int hd = pv.cfg.head_dim;
  CHECK(layer >= 0 && layer < pv.cfg.n_layers, "layer out of range");
  CHECK(rope->rotary_dim >= 8 && rope->rotary_dim <= hd && rope->rotary_dim % 8 == 0,
        "rotary_dim must be a multiple of 8 in [8, head_dim]");
  CHECK(rope->adjacent == 0 || rope->adjacent == 1, "adjacent must be 0 or 1");
  CHECK(rope->n_axes >= 1 && rope->n_axes <= 4, "n_axes out of range [1, 4]");
  CHECK(B >= 1 && B <= 1024, "B out of range [1, 1024]");
  CHECK(n_max >= 0 && (int64_t)B * n_max <= 1 << 26, "n_max negative, or more than 2^26 rows");
  RopeArgs a{};
  for (int j = 0; j < rope->rotary_dim / 2; ++j) {
    a.axis[j] = rope->axes ? rope->axes[j] : 0;
    CHECK(a.axis[j] < rope->n_axes, "an axis beyond n_axes");
    CHECK(std::fabs(rope->freqs[j]) <= 6.3, "a frequency is not finite, or more than a turn");
    a.turns[j] = rope->freqs[j] / 6.283185307179586476925;
  }
  CHECK(seq_ids && pos0, "null array");
  if (n_max == 0) return WAR_OK;
  const int64_t qrow = (int64_t)pv.cfg.n_q_heads * hd, row = (int64_t)pv.cfg.n_kv_heads * hd;
  WARCHK(check_rows(q, q_stride, qrow));
  WARCHK(check_rows(q_out, q_out_stride, qrow));
  WARCHK(check_rows(k, k_stride, row));
  WARCHK(check_rows(v, v_stride, row));
  CHECK(q != q_out || q_stride == q_out_stride, "in place, the strides must be the same");
  a.p = pv.dev;
  a.g = pv.geom;
  a.layer = layer;
  a.B = B;
  a.n_max = n_max;
  a.pages = (n_max + 15 + 15) / 16;
  a.group = pv.cfg.n_q_heads / pv.cfg.n_kv_heads;
  a.seq = seq_ids;
  a.pos0 = pos0;
  a.n = n_lens;
  a.positions = positions;
  a.q = static_cast<const bf16_t*>(q);
  a.k = static_cast<const bf16_t*>(k);
  a.v = static_cast<const bf16_t*>(v);
  a.qo = static_cast<bf16_t*>(q_out);
  a.q_stride = q_stride;
  a.qo_stride = q_out_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.rotary = rope->rotary_dim;
  a.adjacent = rope->adjacent;
  launch_rope_write(a, static_cast<hipStream_t>(stream));
  HIPCHK(hipGetLastError());
  return WAR_OK;
}

}  // extern "C"
