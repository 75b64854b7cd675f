// vf_rms_norm: residual's addition, root-mean-square norm and the rounding of its output in one pass.
//
// s = x + r; y = s / sqrt(mean(s^2) + eps) * gain.  Every element is read once and held in registers while
// the row's sum of squares is taken, so the kernel moves x, r, sum and out once each: it is bound by the memory's
// rate, and for a single row by the latency of a launch.  MI355X: 32768 x 2048 in bf16 with residual, 537 MB, 102 us = 5.26 TB/s, as
// a copy reaches (123 us with a workgroup for every row, which reads the gains again); one row of 1024 2.4 us.
#include "vf_internal.h"
#include "vf_ops_dev.h"

namespace {

using namespace vfo;

struct NormArgs {
  const void *x, *res;
  const float *gain;
  void *sum, *out;
  uint8_t *scales;
  int64_t ld_x, ld_res, ld_sum, ld_out, rows;
  int width, kb, tpr;  // columns, blocks of 32 columns, threads per row
  float eps;
};

template <int OUT> struct out_elem { typedef uint8_t type; };
template <> struct out_elem<VF_FP32> { typedef float type; };
template <> struct out_elem<VF_BF16> { typedef uint16_t type; };

// NCH chunks of eight columns per thread, chunk k of a thread at columns 8 (k tpr + t).  The threads of a row are a
// power of two of them, whole waves; a workgroup holds blockDim / tpr rows at a time and takes several, one after the other: its
// threads keep their gains, and the next row is on its way while this one is summed.
template <typename T, int OUT, int NCH>
__global__ void __launch_bounds__(1024) k_rms_norm(const NormArgs a) {
  __shared__ float part[2][16];
  const int t = (int)threadIdx.x & (a.tpr - 1), rpw = (int)blockDim.x / a.tpr, r0 = (int)threadIdx.x / a.tpr;
  const int waves = a.tpr >> 6, wave = (int)threadIdx.x >> 6;
  const int nchunk = OUT >= VF_E4M3 ? 4 * a.kb : (a.width + 7) >> 3;
  constexpr bool AHEAD = NCH < 4;  // (rows of more than 16,384 leave no registers for it)
  auto gain_of = [&](int k, float (&v)[8]) {
    const int c = k * a.tpr + t, n = a.width - 8 * c;
    raw8<float> g;
#pragma unroll
    for (int i = 0; i < 8; ++i) g.w[i] = __float_as_uint(1.0f);
    if (a.gain && n > 0) fetch8(a.gain + 8 * c, n, g);
    unpack8(g, v);
  };
  float gain[AHEAD ? NCH : 1][8];
  if constexpr (AHEAD) {
#pragma unroll
    for (int k = 0; k < NCH; ++k) gain_of(k, gain[k]);
  }
  raw8<T> x[NCH], res[NCH];
  auto ask = [&](int64_t row) {
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = k * a.tpr + t, n = row < a.rows ? a.width - 8 * c : 0;
      if (n <= 0) continue;
      fetch8(reinterpret_cast<const T *>(a.x) + row * a.ld_x + 8 * c, n, x[k]);
      if (a.res) fetch8(reinterpret_cast<const T *>(a.res) + row * a.ld_res + 8 * c, n, res[k]);
    }
  };
  int64_t base = (int64_t)blockIdx.x * rpw;
  if (AHEAD) ask(base + r0);
  for (int turn = 0; base < a.rows; ++turn) {
    const int64_t row = base + r0;
    const bool live = row < a.rows;
    if (!AHEAD) ask(row);
    float v[NCH][8];
    float ss = 0.0f;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = k * a.tpr + t, n = live ? a.width - 8 * c : 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[k][i] = 0.0f;
      if (n > 0) {
        unpack8(x[k], v[k]);
        if (a.res) {
          float r[8];
          unpack8(res[k], r);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[k][i] += r[i];
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(v[k][i], v[k][i], ss);
    }
    base += (int64_t)gridDim.x * rpw;
    if (AHEAD) ask(base + r0);
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = k * a.tpr + t, n = live ? a.width - 8 * c : 0;
      if (a.sum && n > 0) store_upto8(reinterpret_cast<T *>(a.sum) + row * a.ld_sum + 8 * c, n, v[k]);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) ss += __shfl_xor(ss, m);
    if (waves > 1) {  // (uniform over the launch; two arrays: one barrier a row)
      float *sums = part[turn & 1];
      if ((threadIdx.x & 63) == 0) sums[wave] = ss;
      __syncthreads();
      ss = 0.0f;
      for (int w = 0; w < waves; ++w) ss += sums[r0 * waves + w];
    }
    const float f = 1.0f / sqrtf(ss / (float)a.width + a.eps);
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
      const int c = k * a.tpr + t, n = a.width - 8 * c;
      float y[8];
      if constexpr (!AHEAD) gain_of(k, gain[0]);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = i < n ? v[k][i] * f * gain[AHEAD ? k : 0][i] : 0.0f;
      const bool on = live && c < nchunk;
      if constexpr (OUT >= VF_E4M3) {
        quantize_chunk<OUT>(y, c, on, reinterpret_cast<uint8_t *>(a.out) + row * a.kb * mx<OUT>::bytes32, a.scales + row * a.kb);
      } else {
        if (on) store_upto8(reinterpret_cast<typename out_elem<OUT>::type *>(a.out) + row * a.ld_out + 8 * c, n, y);
      }
    }
  }
}

template <typename T, int OUT>
void launch(hipStream_t st, const NormArgs &a, int nch, int grid, int block) {
  if (nch == 1) k_rms_norm<T, OUT, 1><<<grid, block, 0, st>>>(a);
  else if (nch == 2) k_rms_norm<T, OUT, 2><<<grid, block, 0, st>>>(a);
  else k_rms_norm<T, OUT, 4><<<grid, block, 0, st>>>(a);
}

template <typename T>
void launch_out(hipStream_t st, const NormArgs &a, int out_type, int nch, int grid, int block) {
  switch (out_type) {
    case VF_FP32: launch<T, VF_FP32>(st, a, nch, grid, block); break;
    case VF_BF16: launch<T, VF_BF16>(st, a, nch, grid, block); break;
    case VF_E4M3: launch<T, VF_E4M3>(st, a, nch, grid, block); break;
    default: launch<T, VF_E2M1>(st, a, nch, grid, block); break;
  }
}

}  // namespace

int vfk_rms_norm(vf_ctx *c, int type, const void *x, int64_t ld_x, const void *res, int64_t ld_res, const float *gain,
                 float eps, int64_t rows, int width, void *sum, int64_t ld_sum, int out_type, void *out, int64_t ld_out,
                 uint8_t *scales) {
  if (rows == 0) return VF_OK;
  NormArgs a;
  a.x = x; a.res = res; a.gain = gain; a.sum = sum; a.out = out; a.scales = scales;
  a.ld_x = ld_x; a.ld_res = ld_res; a.ld_sum = ld_sum; a.ld_out = ld_out; a.rows = rows;
  a.width = width; a.kb = (width + 31) / 32; a.eps = eps;
  const int nchunk = out_type >= VF_E4M3 ? 4 * a.kb : (width + 7) / 8;
  // a thread takes one chunk up to 256 threads a row, then two, then four with 1024 threads
  int tpr = 64;
  while (tpr < nchunk && tpr < 256) tpr *= 2;
  while (2 * tpr < nchunk && tpr < 1024) tpr *= 2;
  int nch = 1;
  while (nch * tpr < nchunk) nch *= 2;
  a.tpr = tpr;
  const int block = tpr < 256 ? 256 : tpr, rpw = block / tpr;
  const int64_t groups = (rows + rpw - 1) / rpw;
  // as many workgroups as run at a time (2048 threads on each of 256 compute units)
  const int64_t at_once = 256 * 2048 / block;
  const int grid = (int)(groups < at_once ? groups : at_once);
  if (type == VF_BF16) launch_out<uint16_t>(c->stream, a, out_type, nch, grid, block);
  else launch_out<float>(c->stream, a, out_type, nch, grid, block);
  VF_HIP(c, hipGetLastError());
  return VF_OK;
}
