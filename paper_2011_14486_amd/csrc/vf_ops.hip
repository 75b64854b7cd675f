// C entry points of the sequence operators: argument checks.
#include <math.h>

#include "vf_internal.h"

namespace {

bool is_type(int32_t t) { return t == VF_FP32 || t == VF_BF16; }
bool is_mx(int32_t t) { return t == VF_E4M3 || t == VF_E2M1; }
bool is_kv(int32_t t) { return is_type(t) || t == VF_E4M3; }
bool aligned(const void *p, int n) { return (uintptr_t)p % (uintptr_t)n == 0; }
int bytes_of(int32_t type) { return type == VF_BF16 ? 2 : 4; }

constexpr int64_t MAX_ROWS = (int64_t)1 << 31, MAX_COLS = 1 << 24, MAX_LD = (int64_t)1 << 31;

// A matrix of a type as an argument: `rows` rows of `width`, `ld` apart.  Without rows nothing is looked at.
bool matrix_ok(const void *p, int64_t ld, int64_t rows, int64_t width, int32_t type) {
  return rows == 0 || (p && aligned(p, bytes_of(type)) && ld >= width && ld <= MAX_LD);
}
bool mx_ok(const void *codes, const void *scales, int64_t rows) { return rows == 0 || (codes && scales && aligned(codes, 16)); }

bool layer_ok(const vf_ssm *l) {
  if (l->heads < 1 || l->heads > 65536 || l->head_dim < 1 || l->head_dim > 256 || l->n_state < 1 || l->n_state > 256) return false;
  if (l->groups < 1 || l->heads % l->groups != 0 || l->taps < 1 || l->taps > 8) return false;
  if (!l->conv_w_dev || !l->a_dev) return false;
  const void *f[] = {l->conv_w_dev, l->conv_b_dev, l->a_dev, l->d_dev, l->dt_bias_dev};
  for (const void *p : f)
    if (!aligned(p, 4)) return false;
  return true;
}

// state buffers of one direction: both or none; a slot list or at least n_seq slots
bool state_ok(const vf_ssm *l, const vf_ssm_io *io, const void *conv, const float *ssm, const int32_t *slots, int32_t n) {
  if (!ssm) return !conv && !slots;
  if (l->taps > 1 && n > 0 && !conv) return false;
  if (n < 0 || !aligned(ssm, 4) || !aligned(conv, bytes_of(io->type)) || !aligned(slots, 4)) return false;
  return slots || n >= io->n_seq;
}

int ssm(vf_ctx *c, const vf_ssm *l, const vf_ssm_io *io, bool one) {
  if (!c || !l || !io || !layer_ok(l) || !is_type(io->type)) return VF_EINVAL;
  if (io->n_seq < 0 || io->tokens < 0 || io->tokens >= ((int64_t)1 << 31) || io->longest < 0) return VF_EINVAL;
  if (one && (io->offsets_dev || io->tokens != io->n_seq)) return VF_EINVAL;
  if (!io->offsets_dev && (io->n_seq == 0 ? io->tokens != 0 : io->tokens % io->n_seq != 0)) return VF_EINVAL;
  if (!aligned(io->offsets_dev, 4)) return VF_EINVAL;
  const int64_t HP = (int64_t)l->heads * l->head_dim, C = HP + 2 * (int64_t)l->groups * l->n_state;
  if (!matrix_ok(io->xbc_dev, io->ld_xbc, io->tokens, C, io->type) || !matrix_ok(io->dt_dev, io->ld_dt, io->tokens, l->heads, io->type) ||
      !matrix_ok(io->out_dev, io->ld_out, io->tokens, HP, io->type))
    return VF_EINVAL;
  if (io->z_dev && !matrix_ok(io->z_dev, io->ld_z, io->tokens, HP, io->type)) return VF_EINVAL;
  if (!state_ok(l, io, io->conv_in_dev, io->ssm_in_dev, io->slots_in_dev, io->n_slots_in) ||
      !state_ok(l, io, io->conv_out_dev, io->ssm_out_dev, io->slots_out_dev, io->n_slots_out))
    return VF_EINVAL;
  DeviceGuard g(c->device);
  return vfk_ssm(c, l, io, one);
}

bool kv_ok(const vf_kv *kv, int32_t type) {
  if (kv->format != type && kv->format != VF_E4M3) return false;
  if (kv->kv_heads < 1 || kv->kv_heads > 65536 || kv->head_dim < 1 || kv->head_dim > 256 || kv->pages < 1) return false;
  if (kv->page < 16 || kv->page > 1024 || (kv->page & (kv->page - 1)) != 0) return false;
  if (!kv->k_dev || !kv->v_dev || !aligned(kv->k_dev, 16) || !aligned(kv->v_dev, 16)) return false;
  return (kv->format == VF_E4M3) == (kv->k_scales_dev != nullptr) && (kv->format == VF_E4M3) == (kv->v_scales_dev != nullptr);
}

// the sequences, whose rows are looked at by the caller
bool seqs_ok(const vf_kv_seqs *s, const vf_kv *kv) {
  if (s->n_seq < 0 || s->tokens < 0 || s->tokens >= ((int64_t)1 << 31) || s->longest < 0) return false;
  if (!s->offsets_dev && (s->n_seq == 0 ? s->tokens != 0 : s->tokens % s->n_seq != 0)) return false;
  if (s->max_pages < 0 || (int64_t)s->max_pages * kv->page > ((int64_t)1 << 30) || s->ld_table < s->max_pages || s->ld_table > MAX_LD) return false;
  if (!aligned(s->offsets_dev, 4) || !aligned(s->lengths_dev, 4) || !aligned(s->table_dev, 4)) return false;
  return s->n_seq == 0 || (s->lengths_dev && (s->table_dev || s->max_pages == 0));
}

}  // namespace

void *vfk_ops_scratch(vf_ctx *c, size_t bytes) {
  if (bytes <= c->ops_bytes) return c->ops_scratch[c->ops_blocks - 1];
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(c->stream, &st) != hipSuccess || st != hipStreamCaptureStatusNone) {
    (void)hipGetLastError();
    return nullptr;
  }
  if (c->ops_blocks == 48) return nullptr;
  // at least twice the last block, so that what stays behind is less than what is held (no call asks for more than 260 MiB, so all
  // blocks together stay below 1 GiB)
  const size_t want = bytes < 2 * c->ops_bytes ? 2 * c->ops_bytes : bytes;
  void *p = nullptr;
  if (hipMalloc(&p, want) != hipSuccess) {
    (void)hipGetLastError();
    return nullptr;
  }
  c->ops_scratch[c->ops_blocks++] = p;
  c->ops_bytes = want;
  return p;
}

extern "C" {

int vf_rms_norm(vf_ctx *c, int32_t type, const void *x, int64_t ld_x, const void *res, int64_t ld_res, const float *gain,
                float eps, int64_t rows, int64_t width, void *sum, int64_t ld_sum, int32_t out_type, void *out, int64_t ld_out,
                uint8_t *scales) {
  if (!c || !is_type(type) || !(is_type(out_type) || is_mx(out_type))) return VF_EINVAL;
  if (rows < 0 || rows > MAX_ROWS || width < 1 || width > 32768 || !(eps >= 0.0f) || !isfinite(eps)) return VF_EINVAL;
  if (!matrix_ok(x, ld_x, rows, width, type) || !aligned(gain, 4)) return VF_EINVAL;
  if ((res && !matrix_ok(res, ld_res, rows, width, type)) || (sum && !matrix_ok(sum, ld_sum, rows, width, type))) return VF_EINVAL;
  if (sum && ((sum == x && ld_sum != ld_x) || (sum == res && ld_sum != ld_res))) return VF_EINVAL;
  if (is_mx(out_type) ? !mx_ok(out, scales, rows) : scales || !matrix_ok(out, ld_out, rows, width, out_type)) return VF_EINVAL;
  DeviceGuard g(c->device);
  return vfk_rms_norm(c, type, x, ld_x, res, ld_res, gain, eps, rows, (int)width, sum, ld_sum, out_type, out, ld_out, scales);
}

int vf_mx_quantize(vf_ctx *c, int32_t type, const void *x, int64_t ld_x, int64_t rows, int64_t cols, int32_t format, uint8_t *codes,
                   uint8_t *scales) {
  if (!c || !is_type(type) || !is_mx(format) || rows < 0 || rows > MAX_ROWS || cols < 1 || cols > MAX_COLS) return VF_EINVAL;
  if (!matrix_ok(x, ld_x, rows, cols, type) || !mx_ok(codes, scales, rows)) return VF_EINVAL;
  DeviceGuard g(c->device);
  return vfk_mx_quantize(c, type, x, ld_x, rows, (int)cols, format, codes, scales);
}

int vf_mx_dequantize(vf_ctx *c, int32_t format, const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols, int32_t type,
                     void *out, int64_t ld_out) {
  if (!c || !is_type(type) || !is_mx(format) || rows < 0 || rows > MAX_ROWS || cols < 1 || cols > MAX_COLS) return VF_EINVAL;
  if (!matrix_ok(out, ld_out, rows, cols, type) || !mx_ok(codes, scales, rows)) return VF_EINVAL;
  DeviceGuard g(c->device);
  return vfk_mx_dequantize(c, format, codes, scales, rows, (int)cols, type, out, ld_out);
}

int vf_mx_matmul(vf_ctx *c, int32_t a_format, const uint8_t *a, const uint8_t *as, const uint8_t *w, const uint8_t *ws, int64_t M,
                 int64_t N, int64_t K, const float *bias, int32_t out_type, void *out, int64_t ld_out) {
  if (!c || !is_mx(a_format) || !is_type(out_type)) return VF_EINVAL;
  if (M < 0 || M > MAX_ROWS || N < 0 || N > MAX_COLS || K < 1 || K > MAX_COLS || !aligned(bias, 4)) return VF_EINVAL;
  if (M == 0 || N == 0) return VF_OK;
  if (!mx_ok(a, as, M) || !mx_ok(w, ws, N) || !matrix_ok(out, ld_out, M, N, out_type)) return VF_EINVAL;
  DeviceGuard g(c->device);
  return vfk_mx_matmul(c, a_format, a, as, w, ws, M, (int)N, (int)K, bias, out_type, out, ld_out);
}

int vf_ssm_scan(vf_ctx *c, const vf_ssm *layer, const vf_ssm_io *io) { return ssm(c, layer, io, false); }
int vf_ssm_step(vf_ctx *c, const vf_ssm *layer, const vf_ssm_io *io) { return ssm(c, layer, io, true); }

int vf_kv_append(vf_ctx *c, const vf_kv *kv, const vf_kv_seqs *seqs, const vf_rope *rope, int32_t type, const void *k, int64_t ld_k,
                 const void *v, int64_t ld_v, int32_t heads, const void *q, int64_t ld_q, void *q_out, int64_t ld_q_out) {
  if (!c || !kv || !seqs || !is_type(type) || !kv_ok(kv, type) || !seqs_ok(seqs, kv)) return VF_EINVAL;
  const int64_t n = seqs->tokens;
  if (heads < 0 || heads > 65536 || (n > 0 && ((heads > 0) != (q != nullptr) || (heads > 0) != (q_out != nullptr)))) return VF_EINVAL;
  const int64_t each = (int64_t)kv->kv_heads * kv->head_dim, HD = (int64_t)heads * kv->head_dim;
  if (!matrix_ok(k, ld_k, n, each, type) || !matrix_ok(v, ld_v, n, each, type)) return VF_EINVAL;
  if (q && (!matrix_ok(q, ld_q, n, HD, type) || !matrix_ok(q_out, ld_q_out, n, HD, type) || (q_out == q && ld_q_out != ld_q))) return VF_EINVAL;
  if (rope && (rope->rotary < 0 || rope->rotary > kv->head_dim || rope->rotary % 2 != 0 || !aligned(rope->freq_dev, 8) ||
               (rope->rotary > 0 && !rope->freq_dev) || !isfinite(rope->magnitude)))
    return VF_EINVAL;
  DeviceGuard g(c->device);
  return vfk_kv_append(c, vf_kv_call{kv, seqs, type}, rope, k, ld_k, v, ld_v, heads, q, ld_q, q_out, ld_q_out);
}

int vf_kv_read(vf_ctx *c, const vf_kv *kv, const vf_kv_seqs *seqs, int32_t type, void *k, int64_t ld_k, void *v, int64_t ld_v) {
  if (!c || !kv || !seqs || !is_type(type) || !kv_ok(kv, kv->format == VF_E4M3 ? type : kv->format) || !is_kv(kv->format) || !seqs_ok(seqs, kv))
    return VF_EINVAL;
  const int64_t n = seqs->tokens, each = (int64_t)kv->kv_heads * kv->head_dim;
  if ((k && !matrix_ok(k, ld_k, n, each, type)) || (v && !matrix_ok(v, ld_v, n, each, type))) return VF_EINVAL;
  DeviceGuard g(c->device);
  return vfk_kv_read(c, vf_kv_call{kv, seqs, type}, k, ld_k, v, ld_v);
}

int vf_kv_attend(vf_ctx *c, const vf_kv *kv, const vf_kv_seqs *seqs, int32_t type, int32_t heads, const void *q, int64_t ld_q, int32_t causal,
                 int32_t window, float scale, int64_t longest_kv, void *out, int64_t ld_out) {
  if (!c || !kv || !seqs || !is_type(type) || !kv_ok(kv, type) || !seqs_ok(seqs, kv)) return VF_EINVAL;
  if (heads < 1 || heads > 65536 || heads % kv->kv_heads != 0) return VF_EINVAL;
  // (scores are powers of two inside: the scale times log2(e) has to be a number too)
  if (causal < 0 || causal > 1 || window < 0 || (window > 0 && !causal) || !(scale >= 0.0f) || !isfinite(scale * 1.5f) || longest_kv < 0) return VF_EINVAL;
  // (rows of one head of the cache are counted in 32 bits)
  if (seqs->tokens * (int64_t)(heads / kv->kv_heads) >= ((int64_t)1 << 31)) return VF_EINVAL;
  const int64_t HD = (int64_t)heads * kv->head_dim;
  if (!matrix_ok(q, ld_q, seqs->tokens, HD, type) || !matrix_ok(out, ld_out, seqs->tokens, HD, type)) return VF_EINVAL;
  if (out == q && ld_out != ld_q && seqs->tokens > 1) return VF_EINVAL;
  DeviceGuard g(c->device);
  return vfk_kv_attend(c, vf_kv_call{kv, seqs, type}, heads, q, ld_q, causal != 0, window, scale, longest_kv, out, ld_out);
}

}  // extern "C"
