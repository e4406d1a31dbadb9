// C ABI of the attention sublayer's operators: checks of the arguments, workspaces, launches (zgr.h).  Nothing here touches the device before every check has passed.
#include "sublayer.h"

#include <cmath>

using namespace zgr;

namespace {

#define ZGR_LAUNCH(expr)                                                                              \
  do {                                                                                                \
    const hipError_t e__ = (expr);                                                                    \
    if (e__ != hipSuccess) return refuse(ZGR_ERR_DEVICE, "%s: %s", #expr, hipGetErrorString(e__));    \
  } while (0)

size_t up256(size_t x) { return (x + 255) / 256 * 256; }
int bytes_of(int dtype) { return dtype == ZGR_BF16 ? 2 : 4; }
bool off(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) != 0; }
constexpr int64_t kMostThreads = (int64_t)1 << 32;      // of one launch

// A view whose rows are read in pieces of 16 bytes, [tokens, heads, dim] in `batches`.  Strides of dimensions of one entry may be anything.
zgr_status check_heads(const zgr_heads* x, const char* name, int dtype, int64_t batches, int64_t tokens, int64_t heads) {
  if (!x || !x->data) return refuse(ZGR_ERR_NULL, "%s is NULL", name);
  const int64_t per = 16 / bytes_of(dtype);
  if (off(x->data, 16)) return refuse(ZGR_ERR_SHAPE, "%s must lie on 16 bytes", name);
  if ((batches > 1 && x->batch % per) || (tokens > 1 && x->token % per) || (heads > 1 && x->head % per))
    return refuse(ZGR_ERR_SHAPE, "%s: strides must be multiples of %d entries", name, (int)per);
  return ZGR_OK;
}
#define ZGR_CHECK(expr) do { const zgr_status st__ = (expr); if (st__ != ZGR_OK) return st__; } while (0)

zgr_status check_workspace(const void* workspace, size_t bytes, size_t needed) {
  if (!needed) return ZGR_OK;
  if (!workspace) return refuse(ZGR_ERR_NULL, "workspace is NULL");
  if (off(workspace, 256)) return refuse(ZGR_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (bytes < needed) return refuse(ZGR_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", bytes, needed);
  return ZGR_OK;
}

// ---- norms and rotation
zgr_status check_rotation(const zgr_rotation* h) {
  if (!h) return refuse(ZGR_ERR_NULL, "the description is NULL");
  if (h->dtype != ZGR_F32 && h->dtype != ZGR_BF16) return refuse(ZGR_ERR_DTYPE, "unknown dtype %d", h->dtype);
  if (h->rows < 0 || h->q_heads < 0 || h->k_heads < 0 || h->q_heads > 65536 || h->k_heads > 65536 || h->q_heads + h->k_heads < 1) return refuse(ZGR_ERR_SHAPE, "rows >= 0, and 1 to 65536 heads");
  if (h->head_dim < 8 || h->head_dim > 256 || h->head_dim % 8) return refuse(ZGR_ERR_SHAPE, "head_dim %d: a multiple of 8 up to 256", h->head_dim);
  if (h->rot_dim < 0 || h->rot_dim > h->head_dim || h->rot_dim % 8) return refuse(ZGR_ERR_SHAPE, "rot_dim %d: a multiple of 8 up to head_dim", h->rot_dim);
  if (!(h->eps >= 0.f) || std::isinf(h->eps)) return refuse(ZGR_ERR_CONFIG, "eps must be finite and not negative");
  if (h->interleaved != 0 && h->interleaved != 1) return refuse(ZGR_ERR_CONFIG, "interleaved must be 0 or 1");
  if (h->rot_dim && h->n_positions < 1) return refuse(ZGR_ERR_SHAPE, "the table has no rows");
  if ((int64_t)h->rows * (h->q_heads + h->k_heads) > ((int64_t)1 << 34) / h->head_dim * 8 || ((int64_t)h->rows * ((h->q_heads + h->k_heads + 3) / 4) + 4) * 64 >= kMostThreads)
    return refuse(ZGR_ERR_SHAPE, "too many rows for one launch");
  return ZGR_OK;
}
zgr_status check_rotation_pointers(const zgr_rotation* h) {
  if (h->rot_dim && (!h->table || !h->positions)) return refuse(ZGR_ERR_NULL, "table or positions is NULL");
  if (h->rot_dim && (off(h->table, 4) || off(h->positions, 4))) return refuse(ZGR_ERR_SHAPE, "table and positions must lie on 4 bytes");
  if (off(h->q_gain, bytes_of(h->dtype)) || off(h->k_gain, bytes_of(h->dtype))) return refuse(ZGR_ERR_SHAPE, "a gain is not aligned");
  return ZGR_OK;
}

// ---- dropout
zgr_status check_dropout(int32_t rows, int32_t cols, int32_t x_dtype, int32_t stream_dtype, double p, uint64_t step, uint32_t* threshold, float* scale) {
  if ((x_dtype != ZGR_F32 && x_dtype != ZGR_BF16) || (stream_dtype != ZGR_F32 && stream_dtype != ZGR_BF16)) return refuse(ZGR_ERR_DTYPE, "unknown dtype");
  if (rows < 0 || cols < 1) return refuse(ZGR_ERR_SHAPE, "rows >= 0 and cols >= 1");
  if (step >> 32) return refuse(ZGR_ERR_CONFIG, "step must be below 2^32");
  const double words = std::nearbyint(p * 4294967296.0);
  if (!(p >= 0.0) || !(words < 4294967296.0)) return refuse(ZGR_ERR_CONFIG, "p must be in [0, 1)");
  if ((((int64_t)cols + 7) / 8) * rows + 256 >= kMostThreads) return refuse(ZGR_ERR_SHAPE, "too many entries for one launch");
  *threshold = (uint32_t)words;
  *scale = (float)(1.0 / (1.0 - p));
  return ZGR_OK;
}
zgr_status check_rows(const void* x, const char* name, int dtype) {
  if (!x) return refuse(ZGR_ERR_NULL, "%s is NULL", name);
  if (off(x, bytes_of(dtype))) return refuse(ZGR_ERR_SHAPE, "%s is not aligned to its entries", name);
  return ZGR_OK;
}

// ---- attention
zgr_status check_attention(const zgr_attention* h) {
  if (!h) return refuse(ZGR_ERR_NULL, "the description is NULL");
  if (h->dtype != ZGR_F32 && h->dtype != ZGR_BF16) return refuse(ZGR_ERR_DTYPE, "unknown dtype %d", h->dtype);
  if (h->batch < 0 || h->n_q < 0 || h->n_k < 0 || h->n_q > 1 << 26 || h->n_k > 1 << 26 || h->batch > 1 << 20) return refuse(ZGR_ERR_SHAPE, "batch up to 2^20, n_q and n_k up to 2^26");
  if (h->n_head < 1 || h->n_head > 65536 || h->n_kv_head < 1 || h->n_head % h->n_kv_head) return refuse(ZGR_ERR_SHAPE, "n_head %d must be a multiple of n_kv_head %d", h->n_head, h->n_kv_head);
  if (h->head_dim < 8 || h->head_dim > 128 || h->head_dim % 8) return refuse(ZGR_ERR_SHAPE, "head_dim %d: a multiple of 8 up to 128", h->head_dim);
  if (h->causal != 0 && h->causal != 1) return refuse(ZGR_ERR_CONFIG, "causal must be 0 or 1");
  if (!(h->scale > 0.f) || std::isinf(h->scale)) return refuse(ZGR_ERR_CONFIG, "scale must be finite and positive");
  if (h->bias) {
    if (!h->bias_map) return refuse(ZGR_ERR_NULL, "bias_map is NULL");
    if (h->bias_buckets < 1 || h->bias_reach < 0 || h->bias_reach > ZGR_MAX_REACH) return refuse(ZGR_ERR_SHAPE, "bias_buckets >= 1 and bias_reach in [0, %d]", ZGR_MAX_REACH);
    if (off(h->bias, bytes_of(h->dtype)) || off(h->bias_map, 4)) return refuse(ZGR_ERR_SHAPE, "bias or bias_map is not aligned");
  }
  if (off(h->q_lengths, 4) || off(h->k_lengths, 4) || off(h->q_start, 4)) return refuse(ZGR_ERR_SHAPE, "lengths and starts must lie on 4 bytes");
  const int64_t blocks = (int64_t)(((h->n_q > h->n_k ? h->n_q : h->n_k) + 32) / 32) * h->n_head;
  if (h->batch && blocks > (kMostThreads >> 9) / h->batch) return refuse(ZGR_ERR_SHAPE, "too many blocks for one launch");
  return ZGR_OK;
}
bool nothing(const zgr_attention* h) { return h->batch == 0 || h->n_q == 0; }
zgr_attention plain_of(const zgr_attention* h) {
  zgr_attention p = *h;
  if (!p.bias) { p.bias_map = nullptr; p.bias_buckets = p.bias_reach = 0; }
  return p;
}

}  // namespace

extern "C" {

zgr_status zgr_norm_rotate(const zgr_rotation* how, const zgr_heads* q, const zgr_heads* k, const zgr_heads* q_out, const zgr_heads* k_out, void* hip_stream) {
  ZGR_CHECK(check_rotation(how));
  if (how->rows == 0) return ZGR_OK;
  ZGR_CHECK(check_rotation_pointers(how));
  RotateArgs a{};
  a.how = *how;
  if (how->q_heads) {
    ZGR_CHECK(check_heads(q, "q", how->dtype, 1, how->rows, how->q_heads));
    ZGR_CHECK(check_heads(q_out, "q_out", how->dtype, 1, how->rows, how->q_heads));
    a.q = *q, a.q_out = *q_out;
  }
  if (how->k_heads) {
    ZGR_CHECK(check_heads(k, "k", how->dtype, 1, how->rows, how->k_heads));
    ZGR_CHECK(check_heads(k_out, "k_out", how->dtype, 1, how->rows, how->k_heads));
    a.k = *k, a.k_out = *k_out;
  }
  ZGR_LAUNCH(launch_norm_rotate(a, reinterpret_cast<hipStream_t>(hip_stream)));
  return ZGR_OK;
}

size_t zgr_norm_rotate_backward_workspace(const zgr_rotation* how) {
  if (check_rotation(how) != ZGR_OK) return 0;
  return up256(how->rows ? (size_t)rotate_parts(*how) * 2 * how->head_dim * 4 : 0) + 256;
}

zgr_status zgr_norm_rotate_backward(const zgr_rotation* how, const zgr_heads* dq_out, const zgr_heads* dk_out, const zgr_heads* q, const zgr_heads* k, const zgr_heads* dq, const zgr_heads* dk,
                                    float* dgains, void* workspace, size_t workspace_bytes, void* hip_stream) {
  ZGR_CHECK(check_rotation(how));
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  RotateArgs a{};
  a.how = *how;
  if (off(dgains, 4)) return refuse(ZGR_ERR_SHAPE, "dgains must lie on 4 bytes");
  if (how->rows) {
    ZGR_CHECK(check_rotation_pointers(how));
    if (how->q_heads) {
      ZGR_CHECK(check_heads(dq_out, "dq_out", how->dtype, 1, how->rows, how->q_heads));
      ZGR_CHECK(check_heads(q, "q", how->dtype, 1, how->rows, how->q_heads));
      ZGR_CHECK(check_heads(dq, "dq", how->dtype, 1, how->rows, how->q_heads));
      a.q_out = *dq_out, a.q = *q, a.dq = *dq;
    }
    if (how->k_heads) {
      ZGR_CHECK(check_heads(dk_out, "dk_out", how->dtype, 1, how->rows, how->k_heads));
      ZGR_CHECK(check_heads(k, "k", how->dtype, 1, how->rows, how->k_heads));
      ZGR_CHECK(check_heads(dk, "dk", how->dtype, 1, how->rows, how->k_heads));
      a.k_out = *dk_out, a.k = *k, a.dk = *dk;
    }
    if (dgains) {
      ZGR_CHECK(check_workspace(workspace, workspace_bytes, zgr_norm_rotate_backward_workspace(how)));
      a.part = reinterpret_cast<float*>(workspace);
    }
    ZGR_LAUNCH(launch_norm_rotate_backward(a, s));
  }
  if (dgains) ZGR_LAUNCH(launch_part_sums(a.part, how->rows ? rotate_parts(*how) : 0, 2 * how->head_dim, dgains, s));
  return ZGR_OK;
}

zgr_status zgr_relative_buckets(int32_t buckets, int32_t reach, int32_t causal, int32_t* map) {
  if (!map) return refuse(ZGR_ERR_NULL, "map is NULL");
  if (causal != 0 && causal != 1) return refuse(ZGR_ERR_CONFIG, "causal must be 0 or 1");
  if (buckets < (causal ? 1 : 2) || reach < 0 || reach > ZGR_MAX_REACH) return refuse(ZGR_ERR_SHAPE, "buckets >= %d and reach in [0, %d]", causal ? 1 : 2, ZGR_MAX_REACH);
  const int n = causal ? buckets : buckets / 2, exact = n / 2 > 1 ? n / 2 : 1;
  for (int d = -reach; d <= reach; ++d) {
    const int distance = causal ? (d < 0 ? -d : 0) : (d < 0 ? -d : d);
    int bucket = distance;
    if (distance >= exact && reach > exact) {      // exact + the whole part of (n - exact) log(distance / exact) / log(reach / exact); a distance that is a power in question is on its upper side
      const double at = (n - exact) * std::log((double)distance / exact) / std::log((double)reach / exact);
      bucket = exact + (int)std::floor(at + 1e-9);
    }
    map[d + reach] = (bucket < n - 1 ? bucket : n - 1) + (!causal && d > 0 ? n : 0);
  }
  return ZGR_OK;
}

size_t zgr_attention_workspace(const zgr_attention* how) { return check_attention(how) == ZGR_OK ? attention_workspace(plain_of(how)) : 0; }

zgr_status zgr_attention_forward(const zgr_attention* how, const zgr_heads* q, const zgr_heads* k, const zgr_heads* v, const zgr_heads* out, float* lse, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  ZGR_CHECK(check_attention(how));
  if (nothing(how)) return ZGR_OK;
  AttentionArgs a{};
  a.how = plain_of(how);
  ZGR_CHECK(check_heads(q, "q", how->dtype, how->batch, how->n_q, how->n_head));
  ZGR_CHECK(check_heads(out, "out", how->dtype, how->batch, how->n_q, how->n_head));
  a.q = *q, a.out = *out;
  if (how->n_k) {
    ZGR_CHECK(check_heads(k, "k", how->dtype, how->batch, how->n_k, how->n_kv_head));
    ZGR_CHECK(check_heads(v, "v", how->dtype, how->batch, how->n_k, how->n_kv_head));
    a.k = *k, a.v = *v;
  }
  if (!lse) return refuse(ZGR_ERR_NULL, "lse is NULL");
  if (off(lse, 4)) return refuse(ZGR_ERR_SHAPE, "lse must lie on 4 bytes");
  a.lse = lse;
  ZGR_CHECK(check_workspace(workspace, workspace_bytes, attention_workspace(a.how)));
  a.workspace = reinterpret_cast<unsigned char*>(workspace);
  ZGR_LAUNCH(launch_heads_forward(a, reinterpret_cast<hipStream_t>(hip_stream)));
  return ZGR_OK;
}

size_t zgr_attention_backward_workspace(const zgr_attention* how) { return check_attention(how) == ZGR_OK ? attention_backward_workspace(plain_of(how)) + 256 : 0; }

zgr_status zgr_attention_backward(const zgr_attention* how, const zgr_heads* dout, const zgr_heads* q, const zgr_heads* k, const zgr_heads* v, const zgr_heads* out, const float* lse,
                                  const zgr_heads* dq, const zgr_heads* dk, const zgr_heads* dv, void* dbias, void* workspace, size_t workspace_bytes, void* hip_stream) {
  ZGR_CHECK(check_attention(how));
  AttentionArgs a{};
  a.how = plain_of(how);
  if (how->n_q && how->batch) {
    ZGR_CHECK(check_heads(dout, "dout", how->dtype, how->batch, how->n_q, how->n_head));
    ZGR_CHECK(check_heads(q, "q", how->dtype, how->batch, how->n_q, how->n_head));
    ZGR_CHECK(check_heads(out, "out", how->dtype, how->batch, how->n_q, how->n_head));
    ZGR_CHECK(check_heads(dq, "dq", how->dtype, how->batch, how->n_q, how->n_head));
    a.dout = *dout, a.q = *q, a.out = *out, a.dq = *dq;
    if (!lse) return refuse(ZGR_ERR_NULL, "lse is NULL");
    if (off(lse, 4)) return refuse(ZGR_ERR_SHAPE, "lse must lie on 4 bytes");
    a.lse = const_cast<float*>(lse);
  }
  if (how->n_k && how->batch) {
    ZGR_CHECK(check_heads(k, "k", how->dtype, how->batch, how->n_k, how->n_kv_head));
    ZGR_CHECK(check_heads(v, "v", how->dtype, how->batch, how->n_k, how->n_kv_head));
    ZGR_CHECK(check_heads(dk, "dk", how->dtype, how->batch, how->n_k, how->n_kv_head));
    ZGR_CHECK(check_heads(dv, "dv", how->dtype, how->batch, how->n_k, how->n_kv_head));
    a.k = *k, a.v = *v, a.dk = *dk, a.dv = *dv;
  }
  if (off(dbias, bytes_of(how->dtype))) return refuse(ZGR_ERR_SHAPE, "dbias is not aligned");
  a.dbias = how->bias ? dbias : nullptr;
  ZGR_CHECK(check_workspace(workspace, workspace_bytes, attention_backward_workspace(a.how) + 256));
  a.workspace = reinterpret_cast<unsigned char*>(workspace);
  ZGR_LAUNCH(launch_heads_backward(a, reinterpret_cast<hipStream_t>(hip_stream)));
  return ZGR_OK;
}

zgr_status zgr_dropout_add(int32_t rows, int32_t cols, int32_t x_dtype, const void* x, int64_t x_row, const void* bias, int32_t stream_dtype, const void* residual, int64_t residual_row, void* out,
                           int64_t out_row, double p, uint64_t seed, uint64_t step, uint32_t site, uint64_t first_row, void* hip_stream) {
  DropoutArgs a{};
  ZGR_CHECK(check_dropout(rows, cols, x_dtype, stream_dtype, p, step, &a.threshold, &a.scale));
  if (first_row >> 32) return refuse(ZGR_ERR_CONFIG, "first_row must be below 2^32");
  if (rows == 0) return ZGR_OK;
  ZGR_CHECK(check_rows(x, "x", x_dtype));
  ZGR_CHECK(check_rows(out, "out", stream_dtype));
  if (off(bias, bytes_of(x_dtype)) || off(residual, bytes_of(stream_dtype))) return refuse(ZGR_ERR_SHAPE, "bias or residual is not aligned to its entries");
  a.rows = rows, a.cols = cols, a.x_dtype = x_dtype, a.stream_dtype = stream_dtype;
  a.x_row = x_row, a.residual_row = residual_row, a.out_row = out_row;
  a.x = const_cast<void*>(x), a.bias = bias, a.residual = residual, a.out = out;
  a.site = site, a.step = (uint32_t)step, a.k0 = (uint32_t)seed, a.k1 = (uint32_t)(seed >> 32), a.first_row = first_row;
  ZGR_LAUNCH(launch_dropout_add(a, reinterpret_cast<hipStream_t>(hip_stream)));
  return ZGR_OK;
}

size_t zgr_dropout_add_backward_workspace(int32_t rows, int32_t cols) {
  if (rows < 0 || cols < 1) return 0;
  return up256(rows ? (size_t)dropout_parts(rows, cols) * cols * 4 : 0) + 256;
}

zgr_status zgr_dropout_add_backward(int32_t rows, int32_t cols, int32_t stream_dtype, const void* dout, int64_t dout_row, int32_t x_dtype, void* dx, int64_t dx_row, float* dbias, double p,
                                    uint64_t seed, uint64_t step, uint32_t site, uint64_t first_row, void* workspace, size_t workspace_bytes, void* hip_stream) {
  DropoutArgs a{};
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  ZGR_CHECK(check_dropout(rows, cols, x_dtype, stream_dtype, p, step, &a.threshold, &a.scale));
  if (first_row >> 32) return refuse(ZGR_ERR_CONFIG, "first_row must be below 2^32");
  if (off(dbias, 4)) return refuse(ZGR_ERR_SHAPE, "dbias must lie on 4 bytes");
  if (rows) {
    ZGR_CHECK(check_rows(dout, "dout", stream_dtype));
    ZGR_CHECK(check_rows(dx, "dx", x_dtype));
    a.rows = rows, a.cols = cols, a.x_dtype = x_dtype, a.stream_dtype = stream_dtype;
    a.x_row = dx_row, a.out_row = dout_row;
    a.x = dx, a.out = const_cast<void*>(dout);
    a.site = site, a.step = (uint32_t)step, a.k0 = (uint32_t)seed, a.k1 = (uint32_t)(seed >> 32), a.first_row = first_row;
    if (dbias) {
      ZGR_CHECK(check_workspace(workspace, workspace_bytes, zgr_dropout_add_backward_workspace(rows, cols)));
      a.part = reinterpret_cast<float*>(workspace);
    }
    ZGR_LAUNCH(launch_dropout_add_backward(a, s));
  }
  if (dbias) ZGR_LAUNCH(launch_part_sums(a.part, rows ? dropout_parts(rows, cols) : 0, cols, dbias, s));
  return ZGR_OK;
}

}  // extern "C"
