// vf_ssm_scan and vf_ssm_step: short causal convolution, selective state space scan and gate.
//
//   S_t = e^(step a) S_(t-1) + step x B^T (head_dim x n_state), y = S C + d x
//
// Token by token a state of P x N numbers is read and written once per sequence, five operations a number and
// token; in chunks (below) the same sums are products of matrices.
#include "vf_internal.h"
#include "vf_ops_dev.h"

namespace {

using namespace vfo;

struct SsmArgs {
  const float *conv_w, *conv_b, *a, *d, *dt_bias;
  const int32_t *offsets, *slots_in, *slots_out;
  const void *xbc, *dt, *z;
  void *out;
  int64_t ld_xbc, ld_dt, ld_z, ld_out, tokens;
  const void *conv_in;
  const float *ssm_in;
  void *conv_out;
  float *ssm_out;
  int n_seq, n_in, n_out;
  int H, P, G, N, W, C;
  int has_in, has_out;
  int conv_later;  // the convolution's state is written by a launch of its own: its buffers overlap
};

// Rows first .. first + count - 1 of sequence s; a range that does not lie in the tokens is empty.
struct Span { int64_t first; int count; };
__device__ __forceinline__ Span span_of(const SsmArgs &p, int s) {
  if (!p.offsets) {
    const int64_t len = p.tokens / p.n_seq;
    return {s * len, (int)len};
  }
  const int64_t b = p.offsets[s], e = p.offsets[s + 1];
  if (b < 0 || e < b || e > p.tokens) return {0, 0};
  return {b, (int)(e - b)};
}
// -1: no state, -2: a slot that is not there (reads as NaN, nothing is written)
__device__ __forceinline__ int slot_of(const int32_t *slots, int has, int n_slots, int s) {
  if (!has) return -1;
  const int k = slots ? slots[s] : s;
  return k < -1 || k >= n_slots ? -2 : k;
}

// Input of channel c at position t of a sequence, t < 0: from the convolution's state (of `slot`)
template <typename T>
__device__ __forceinline__ float conv_input(const SsmArgs &p, const Span &sp, int slot, int c, int t) {
  if (t >= 0) return load1(reinterpret_cast<const T *>(p.xbc) + (sp.first + t) * p.ld_xbc + c);
  if (slot == -1) return 0.0f;
  if (slot == -2) return __uint_as_float(0x7fc00000u);
  return load1(reinterpret_cast<const T *>(p.conv_in) + ((int64_t)slot * p.C + c) * (p.W - 1) + (p.W - 1 + t));
}
// The last W - 1 inputs of channel c into the state; the old ones are read before any is written.
template <typename T>
__device__ __forceinline__ void conv_state(const SsmArgs &p, const Span &sp, int slot, int slot_to, int c) {
  float keep[7];
#pragma unroll
  for (int k = 0; k < 7; ++k)
    if (k < p.W - 1) keep[k] = conv_input<T>(p, sp, slot, c, sp.count - (p.W - 1) + k);
  T *to = reinterpret_cast<T *>(p.conv_out) + ((int64_t)slot_to * p.C + c) * (p.W - 1);
#pragma unroll
  for (int k = 0; k < 7; ++k)
    if (k < p.W - 1) store1(to + k, keep[k]);
}

// A wave's lanes 16 p + i hold p, n = 4 (16 k + i) .. + 3 of the state: 16 lanes read 256 bytes of a row of it.
constexpr int SEQ_TOKENS = 8;  // tokens convolved at a time

// Token by token: a workgroup holds 16 PI rows p of one head's state in registers, NK groups of 64 n.
template <typename T, int PI, int NK>
__global__ void __launch_bounds__(256) k_ssm_tokens(const SsmArgs p) {
  extern __shared__ float lds[];
  const int tid = threadIdx.x, i16 = tid & 15, prow = tid >> 4;
  const int slices = (p.P + 16 * PI - 1) / (16 * PI);
  const int h = (int)blockIdx.x / slices, p0 = ((int)blockIdx.x % slices) * 16 * PI;
  const int g = h / (p.H / p.G);
  const int np = p.P - p0 < 16 * PI ? p.P - p0 : 16 * PI;
  const int Nr = (p.N + 3) & ~3;                       // row of B and C in the LDS, zeros behind N
  float *uB = lds, *uC = uB + SEQ_TOKENS * Nr, *ux = uC + SEQ_TOKENS * Nr, *uy = ux + SEQ_TOKENS * 16 * PI;
  float *udt = uy + SEQ_TOKENS * 16 * PI, *uda = udt + SEQ_TOKENS;
  const int nch = np + 2 * p.N;
  const float A = p.a[h], D = p.d ? p.d[h] : 0.0f, bias_dt = p.dt_bias ? p.dt_bias[h] : 0.0f;
  const bool owns_bc = h == g * (p.H / p.G) && p0 == 0;  // writes the convolution's state of its group's B and C

  for (int s = blockIdx.y; s < p.n_seq; s += gridDim.y) {
    const Span sp = span_of(p, s);
    const int slot = slot_of(p.slots_in, p.has_in, p.n_in, s), slot_to = slot_of(p.slots_out, p.has_out, p.n_out, s);
    float S[PI][NK][4];
#pragma unroll
    for (int k = 0; k < PI; ++k) {
      const int pr = 16 * k + prow;
#pragma unroll
      for (int q = 0; q < NK; ++q) {
        const int n = 4 * (16 * q + i16);
#pragma unroll
        for (int j = 0; j < 4; ++j) S[k][q][j] = slot == -2 ? __uint_as_float(0x7fc00000u) : 0.0f;
        if (slot >= 0 && pr < np && n < p.N) {
          const float *from = p.ssm_in + (((int64_t)slot * p.H + h) * p.P + p0 + pr) * p.N + n;
          if (n + 4 <= p.N) {
            const f32v4 v = *reinterpret_cast<const f32v4 *>(from);
#pragma unroll
            for (int j = 0; j < 4; ++j) S[k][q][j] = v.v[j];
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (n + j < p.N) S[k][q][j] = from[j];
          }
        }
      }
    }
    for (int t0 = 0; t0 < sp.count; t0 += SEQ_TOKENS) {
      const int nt = sp.count - t0 < SEQ_TOKENS ? sp.count - t0 : SEQ_TOKENS;
      // convolution of this workgroup's x, and of B and C
      for (int e = tid; e < nt * nch; e += 256) {
        const int t = e / nch, k = e - t * nch;
        const int c = k < np ? h * p.P + p0 + k : k < np + p.N ? p.H * p.P + g * p.N + (k - np)
                                                               : p.H * p.P + p.G * p.N + g * p.N + (k - np - p.N);
        float v = p.conv_b ? p.conv_b[c] : 0.0f;
        for (int w = 0; w < p.W; ++w) v = fmaf(p.conv_w[c * p.W + w], conv_input<T>(p, sp, slot, c, t0 + t - p.W + 1 + w), v);
        v = silu(v);
        if (k < np) ux[t * 16 * PI + k] = v;
        else if (k < np + p.N) uB[t * Nr + (k - np)] = v;
        else uC[t * Nr + (k - np - p.N)] = v;
      }
      for (int e = tid; e < nt * (Nr - p.N); e += 256) {
        const int t = e / (Nr - p.N), k = p.N + e % (Nr - p.N);
        uB[t * Nr + k] = uC[t * Nr + k] = 0.0f;
      }
      if (tid < nt) {
        const float dt = softplus(load1(reinterpret_cast<const T *>(p.dt) + (sp.first + t0 + tid) * p.ld_dt + h) + bias_dt);
        udt[tid] = dt;
        uda[tid] = __expf(dt * A);
      }
      __syncthreads();
      for (int t = 0; t < nt; ++t) {
        const float dt = udt[t], da = uda[t];
        float y[PI];
#pragma unroll
        for (int k = 0; k < PI; ++k) y[k] = 0.0f;
#pragma unroll
        for (int q = 0; q < NK; ++q) {
          const int n = 4 * (16 * q + i16);
          if (n >= p.N) continue;
          const f32x4 B = *reinterpret_cast<const f32x4 *>(uB + t * Nr + n), Cv = *reinterpret_cast<const f32x4 *>(uC + t * Nr + n);
#pragma unroll
          for (int k = 0; k < PI; ++k) {
            const float dx = 16 * k + prow < np ? dt * ux[t * 16 * PI + 16 * k + prow] : 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              S[k][q][j] = fmaf(S[k][q][j], da, dx * B[j]);
              y[k] = fmaf(S[k][q][j], Cv[j], y[k]);
            }
          }
        }
#pragma unroll
        for (int k = 0; k < PI; ++k) {
#pragma unroll
          for (int m = 1; m < 16; m <<= 1) y[k] += __shfl_xor(y[k], m);
          if (i16 == 0) uy[t * 16 * PI + 16 * k + prow] = y[k];
        }
      }
      __syncthreads();
      for (int e = tid; e < nt * np; e += 256) {
        const int t = e / np, k = e - t * np;
        const int64_t row = sp.first + t0 + t;
        float y = fmaf(D, ux[t * 16 * PI + k], uy[t * 16 * PI + k]);
        if (p.z) y *= silu(load1(reinterpret_cast<const T *>(p.z) + row * p.ld_z + h * p.P + p0 + k));
        store1(reinterpret_cast<T *>(p.out) + row * p.ld_out + h * p.P + p0 + k, y);
      }
      __syncthreads();
    }
    if (slot_to < 0) continue;
#pragma unroll
    for (int k = 0; k < PI; ++k) {
      const int pr = 16 * k + prow;
#pragma unroll
      for (int q = 0; q < NK; ++q) {
        const int n = 4 * (16 * q + i16);
        if (pr >= np || n >= p.N) continue;
        float *to = p.ssm_out + (((int64_t)slot_to * p.H + h) * p.P + p0 + pr) * p.N + n;
        if (n + 4 <= p.N) {
          f32v4 v;
#pragma unroll
          for (int j = 0; j < 4; ++j) v.v[j] = S[k][q][j];
          *reinterpret_cast<f32v4 *>(to) = v;
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (n + j < p.N) to[j] = S[k][q][j];
        }
      }
    }
    if (p.conv_later || p.W == 1) continue;
    for (int k = tid; k < (owns_bc ? nch : np); k += 256)
      conv_state<T>(p, sp, slot, slot_to, k < np ? h * p.P + p0 + k : k < np + p.N ? p.H * p.P + g * p.N + (k - np)
                                                                                   : p.H * p.P + p.G * p.N + g * p.N + (k - np - p.N));
  }
}

// The convolution's state in place: behind the scan, since all its workgroups read the old one.
template <typename T>
__global__ void __launch_bounds__(256) k_ssm_conv_state(const SsmArgs p) {
  const int64_t total = (int64_t)p.n_seq * p.C;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int s = (int)(i / p.C), c = (int)(i - (int64_t)s * p.C);
    const int slot_to = slot_of(p.slots_out, p.has_out, p.n_out, s);
    if (slot_to >= 0) conv_state<T>(p, span_of(p, s), slot_of(p.slots_in, p.has_in, p.n_in, s), slot_to, c);
  }
}

template <typename T, int PI, int NK>
int launch_tokens(vf_ctx *c, const SsmArgs &p) {
  const int slices = (p.P + 16 * PI - 1) / (16 * PI), Nr = (p.N + 3) & ~3;
  const size_t smem = sizeof(float) * SEQ_TOKENS * (2 * Nr + 2 * 16 * PI + 2);
  const dim3 grid(p.H * slices, p.n_seq < 32768 ? p.n_seq : 32768);
  k_ssm_tokens<T, PI, NK><<<grid, 256, smem, c->stream>>>(p);
  VF_HIP(c, hipGetLastError());
  return VF_OK;
}
template <typename T>
int tokens(vf_ctx *c, const SsmArgs &p) {
  const int nk = (p.N + 63) / 64;
  // one slice of 64 rows unless there are too few workgroups for the compute units
  const bool wide = p.P > 16 && (int64_t)p.n_seq * p.H >= 512;
  int rc;
  if (wide) rc = nk <= 1 ? launch_tokens<T, 4, 1>(c, p) : nk <= 2 ? launch_tokens<T, 4, 2>(c, p) : launch_tokens<T, 4, 4>(c, p);
  else rc = nk <= 1 ? launch_tokens<T, 1, 1>(c, p) : nk <= 2 ? launch_tokens<T, 1, 2>(c, p) : launch_tokens<T, 1, 4>(c, p);
  if (rc != VF_OK || !p.conv_later) return rc;
  const int64_t blocks = ((int64_t)p.n_seq * p.C + 255) / 256;
  k_ssm_conv_state<T><<<(int)(blocks < (1 << 20) ? blocks : (1 << 20)), 256, 0, c->stream>>>(p);
  VF_HIP(c, hipGetLastError());
  return VF_OK;
}

bool overlap(const void *a, size_t na, const void *b, size_t nb) {
  const char *x = static_cast<const char *>(a), *y = static_cast<const char *>(b);
  return x && y && x < y + nb && y < x + na;
}

}  // namespace

int vfk_ssm(vf_ctx *c, const vf_ssm *l, const vf_ssm_io *io) {
  if (io->n_seq == 0) return VF_OK;
  SsmArgs p;
  p.conv_w = l->conv_w_dev; p.conv_b = l->conv_b_dev; p.a = l->a_dev; p.d = l->d_dev; p.dt_bias = l->dt_bias_dev;
  p.offsets = io->offsets_dev; p.slots_in = io->slots_in_dev; p.slots_out = io->slots_out_dev;
  p.xbc = io->xbc_dev; p.dt = io->dt_dev; p.z = io->z_dev; p.out = io->out_dev;
  p.ld_xbc = io->ld_xbc; p.ld_dt = io->ld_dt; p.ld_z = io->ld_z; p.ld_out = io->ld_out; p.tokens = io->tokens;
  p.conv_in = io->conv_in_dev; p.ssm_in = io->ssm_in_dev; p.conv_out = io->conv_out_dev; p.ssm_out = io->ssm_out_dev;
  p.n_seq = io->n_seq; p.n_in = io->n_slots_in; p.n_out = io->n_slots_out;
  p.H = l->heads; p.P = l->head_dim; p.G = l->groups; p.N = l->n_state; p.W = l->taps;
  p.C = l->heads * l->head_dim + 2 * l->groups * l->n_state;
  p.has_in = io->ssm_in_dev != nullptr; p.has_out = io->ssm_out_dev != nullptr;
  const size_t slot = (size_t)p.C * (p.W - 1) * (io->type == VF_BF16 ? 2 : 4);
  p.conv_later = overlap(p.conv_in, slot * p.n_in, p.conv_out, slot * p.n_out);
  return io->type == VF_BF16 ? tokens<uint16_t>(c, p) : tokens<float>(c, p);
}
