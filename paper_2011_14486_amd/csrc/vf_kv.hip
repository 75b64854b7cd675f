// vf_kv_append and vf_kv_read: rows of keys and values into a paged cache and out of it, rotary positions on the way.
//
// Both move every number once and are bound by the memory's rate, or for few rows by the latency of a launch.  A workgroup takes up to 8 (16) rows of a
// sequence with all their heads: rows are contiguous in the call's matrices and a page's rows of a head in the cache, so that both sides move
// in whole lines, and what a row needs once (page, angles) is there once.
// MI355X: prompt of 16384 tokens, 32 + 2 x 8 heads of 128 in bf16, 403 MB, 86 us = 4.7 TB/s (104 with one head at a time); 64 prefixes of up to
// 4096 tokens, 8 heads of 128, from 8 bits to bf16, 823 MB, 174 us = 4.7 TB/s (252); a copy reaches 5.2.  One token: 4.2 and 3.8 us.
#include "vf_internal.h"
#include "vf_kv_dev.h"

namespace {

using namespace vfkv;

constexpr int THREADS = 256, TB = 16;   // TB: most rows of a workgroup at a time

// eight elements of the cache's row, whose places are aligned to eight of them
__device__ __forceinline__ void fetch_whole(const uint8_t *p, raw8<uint8_t> &r) {
  const uint2 w = *reinterpret_cast<const uint2 *>(p);
  r.w[0] = w.x;
  r.w[1] = w.y;
}
template <typename E> __device__ __forceinline__ void fetch_whole(const E *p, raw8<E> &r) { fetch8(p, 8, r); }

struct AppendArgs {
  Cache c;
  Seqs s;
  const double *freq;
  const void *q, *k, *v;
  void *q_out;
  int64_t ld_q, ld_k, ld_v, ld_q_out;
  float magnitude;
  int heads, half, interleaved;  // heads of q; half: pairs of a head that turn
  int lanes, chunks_q, tb;       // lanes of a head (a power of two), chunks of eight numbers in a head of q; rows of a workgroup
  int blocks;                    // workgroups' worth of rows in the longest sequence
  Divisor total;                 // heads of a row: of q, keys and values
};

// cos and sin of a in 64 bits, to about 1e-16 of 1: a minus the nearest multiple n of pi / 2, which is taken off in two parts of 53 bits
// (fma rounds once, so what is left has the error of the second part, n 2^-107), then the series in r, |r| <= pi / 4, whose first terms
// left out are r^17 / 17! and r^18 / 18!, below 1e-16.
__device__ __forceinline__ void cos_sin(double a, double &c, double &s) {
  const double n = __builtin_rint(a * 0.6366197723675814);
  double r = __builtin_fma(-n, 1.5707963267948966, a);
  r = __builtin_fma(-n, 6.123233995736766e-17, r);
  const double z = r * r;
  double p = -1.0 / 1307674368000.0;
  p = __builtin_fma(p, z, 1.0 / 6227020800.0);
  p = __builtin_fma(p, z, -1.0 / 39916800.0);
  p = __builtin_fma(p, z, 1.0 / 362880.0);
  p = __builtin_fma(p, z, -1.0 / 5040.0);
  p = __builtin_fma(p, z, 1.0 / 120.0);
  p = __builtin_fma(p, z, -1.0 / 6.0);
  const double sr = __builtin_fma(r * z, p, r);
  double w = 1.0 / 20922789888000.0;
  w = __builtin_fma(w, z, -1.0 / 87178291200.0);
  w = __builtin_fma(w, z, 1.0 / 479001600.0);
  w = __builtin_fma(w, z, -1.0 / 3628800.0);
  w = __builtin_fma(w, z, 1.0 / 40320.0);
  w = __builtin_fma(w, z, -1.0 / 720.0);
  w = __builtin_fma(w, z, 1.0 / 24.0);
  w = __builtin_fma(w, z, -0.5);
  const double cr = __builtin_fma(z, w, 1.0);
  const double q4 = n - 4.0 * __builtin_floor(n * 0.25);  // 0, 1, 2, 3
  const bool swap = q4 == 1.0 || q4 == 3.0;
  c = swap ? sr : cr;
  s = swap ? cr : sr;
  if (q4 == 1.0 || q4 == 2.0) c = -c;
  if (q4 == 2.0 || q4 == 3.0) s = -s;
}

// A thread takes eight neighbouring numbers of a head at a time, and the eight that they are paired with, of several heads at once, so that
// their loads are on their way together.  The rows' cosines and sines are worked out once, for all heads, into the LDS.
// ODD: halves of pairs that do not end between eights.
template <typename T, int FMT, bool ODD>
__global__ void __launch_bounds__(THREADS) k_kv_append(const AppendArgs a) {
  extern __shared__ float2 turn[];  // [tb][half]
  __shared__ int pages[TB];         // of the rows; -1: nowhere
  constexpr int U = sizeof(T) == 2 ? 4 : 2;
  const int lane = (int)threadIdx.x & (a.lanes - 1), D = a.c.dim, d0 = 8 * lane, n = D - d0, step = THREADS / a.lanes;
  const bool first = d0 < a.half, turns = d0 < 2 * a.half;
  const int64_t units = (int64_t)a.s.n * a.blocks;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int seq = a.blocks > 1 ? (int)(unit / a.blocks) : (int)unit;
    const Span sp = span_of(a.s, a.c.shift, seq);
    for (int64_t i0 = (unit - (int64_t)seq * a.blocks) * a.tb; i0 < sp.rows; i0 += (int64_t)a.blocks * a.tb) {
      const int rows = sp.rows - i0 < a.tb ? (int)(sp.rows - i0) : a.tb, pos0 = sp.length - sp.rows + (int)i0;
      __syncthreads();
      for (int i = threadIdx.x; i < rows * a.half; i += THREADS) {
        const int row = i / a.half;
        double c, s;
        cos_sin((double)(pos0 + row) * a.freq[i - row * a.half], c, s);
        turn[i] = make_float2((float)(c * (double)a.magnitude), (float)(s * (double)a.magnitude));
      }
      if ((int)threadIdx.x < rows) {
        const int pos = pos0 + (int)threadIdx.x, e = pos >= 0 ? entry_of(a.s, a.c.shift, seq, pos) : -1;
        pages[threadIdx.x] = (unsigned)e < (unsigned)a.c.pages ? e : -1;
      }
      __syncthreads();
      const int slots = rows * a.total.by;
      // (a head's lanes are in one wave, so that all of them have read it before any of them writes: q_out may be q)
      for (int slot0 = 0; slot0 < slots; slot0 += U * step) {
        raw8<T> own[U], other[U];
        int row[U], head[U];   // head: of q, then of keys, then of values
        const T *src[U];
        float each[ODD ? U : 1][8];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int slot = slot0 + u * step + (int)threadIdx.x / a.lanes;
          row[u] = slot < slots ? over(a.total, slot) : -1;
          head[u] = slot - row[u] * a.total.by;
          if (row[u] < 0) head[u] = a.total.by;
          const int64_t r = sp.first + i0 + row[u];
          const int hk = head[u] - a.heads, hv = hk - a.c.heads;
          src[u] = hk < 0 ? reinterpret_cast<const T *>(a.q) + r * a.ld_q + (int64_t)head[u] * D
                          : hv < 0 ? reinterpret_cast<const T *>(a.k) + r * a.ld_k + (int64_t)hk * D : reinterpret_cast<const T *>(a.v) + r * a.ld_v + (int64_t)hv * D;
          own[u] = {};
          if (row[u] >= 0 && n > 0) fetch8(src[u] + d0, n, own[u]);
          if (row[u] >= 0 && hv < 0 && turns && !a.interleaved) {
            if constexpr (!ODD) {
              fetch8(src[u] + (first ? d0 + a.half : d0 - a.half), 8, other[u]);
            } else {
              // (eight loads, all on their way together)
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const int d = d0 + i;
                each[ODD ? u : 0][i] = load1(src[u] + (d < a.half ? d + a.half : d < 2 * a.half ? d - a.half : 0));
              }
            }
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int hk = head[u] - a.heads, hv = hk - a.c.heads;
          float v[8];
          unpack8(own[u], v);
          if (row[u] >= 0 && hv < 0 && turns) {
            const float2 *cs = turn + row[u] * a.half;
            if (a.interleaved) {
#pragma unroll
              for (int i = 0; i < 8; i += 2) {
                if (d0 + i < 2 * a.half) {
                  const float2 w = cs[(d0 + i) >> 1];
                  const float x = v[i], y = v[i + 1];
                  v[i] = x * w.x - y * w.y;
                  v[i + 1] = y * w.x + x * w.y;
                }
              }
            } else if constexpr (!ODD) {
              float o[8];
              unpack8(other[u], o);
              cs += first ? d0 : d0 - a.half;
#pragma unroll
              for (int i = 0; i < 8; ++i) v[i] = first ? v[i] * cs[i].x - o[i] * cs[i].y : v[i] * cs[i].x + o[i] * cs[i].y;
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const int d = d0 + i;
                const bool low = d < a.half;
                const float2 w = cs[low ? d : d < 2 * a.half ? d - a.half : 0];
                const float o = each[ODD ? u : 0][i];
                const float x = low ? v[i] * w.x - o * w.y : v[i] * w.x + o * w.y;
                v[i] = d < 2 * a.half ? x : v[i];
              }
            }
          }
          asm volatile("" ::: "memory");
          __builtin_amdgcn_wave_barrier();
          if (hk < 0) {
            if (n > 0) store_upto8(reinterpret_cast<T *>(a.q_out) + (sp.first + i0 + row[u]) * a.ld_q_out + (int64_t)head[u] * D + d0, n, v);
          } else {
            // (exchanges between the lanes of a head, all of which come here)
            const int page = row[u] >= 0 ? pages[row[u]] : -1;
            const bool there = page >= 0 && d0 < a.c.width;
            const int64_t at = row_of(a.c, page < 0 ? 0 : page, hv < 0 ? hk : hv, pos0 + row[u]);
            if constexpr (FMT == VF_E4M3) {
              quantize_chunk<VF_E4M3>(v, lane, there, reinterpret_cast<uint8_t *>(hv < 0 ? a.c.k : a.c.v) + at * a.c.width, (hv < 0 ? a.c.ks : a.c.vs) + at * a.c.kb);
            } else {
              if (there) store8(reinterpret_cast<T *>(hv < 0 ? a.c.k : a.c.v) + at * a.c.width + d0, v);
            }
          }
        }
      }
    }
  }
}

struct ReadArgs {
  Cache c;
  Seqs s;
  void *k, *v;
  int64_t ld_k, ld_v;
  int lanes, tb, blocks;
  Divisor total;  // heads of a row that are read
};

template <typename T, int FMT>
__global__ void __launch_bounds__(THREADS) k_kv_read(const ReadArgs a) {
  __shared__ int entries[TB];  // of the rows' pages
  constexpr int U = 4;
  typedef typename kv_elem<FMT>::type E;
  const int lane = (int)threadIdx.x & (a.lanes - 1), d0 = 8 * lane, n = a.c.dim - d0, step = THREADS / a.lanes;
  const int64_t units = (int64_t)a.s.n * a.blocks;
  for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
    const int seq = a.blocks > 1 ? (int)(unit / a.blocks) : (int)unit;
    const Span sp = span_of(a.s, a.c.shift, seq);
    for (int64_t i0 = (unit - (int64_t)seq * a.blocks) * a.tb; i0 < sp.rows; i0 += (int64_t)a.blocks * a.tb) {
      const int rows = sp.rows - i0 < a.tb ? (int)(sp.rows - i0) : a.tb, pos0 = sp.length - sp.rows + (int)i0, slots = rows * a.total.by;
      __syncthreads();
      if ((int)threadIdx.x < rows) {
        const int pos = pos0 + (int)threadIdx.x;
        entries[threadIdx.x] = pos >= 0 ? entry_of(a.s, a.c.shift, seq, pos) : -1;
      }
      __syncthreads();
      if (n <= 0) continue;
      for (int slot0 = (int)threadIdx.x / a.lanes; slot0 < slots; slot0 += U * step) {
        raw8<E> raw[U];
        uint32_t scale[U];
        int row[U], head[U], entry[U];  // head: of keys, then of values
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int slot = slot0 + u * step;
          row[u] = slot < slots ? over(a.total, slot) : -1;
          head[u] = slot - row[u] * a.total.by + (a.k ? 0 : a.c.heads);
          entry[u] = row[u] >= 0 ? entries[row[u]] : -1;
          if ((unsigned)entry[u] < (unsigned)a.c.pages) {
            const bool is_k = head[u] < a.c.heads;
            const int64_t at = row_of(a.c, entry[u], is_k ? head[u] : head[u] - a.c.heads, pos0 + row[u]);
            fetch_whole(reinterpret_cast<const E *>(is_k ? a.c.k : a.c.v) + at * a.c.width + d0, raw[u]);
            if (FMT == VF_E4M3) scale[u] = (is_k ? a.c.ks : a.c.vs)[at * a.c.kb + (d0 >> 5)];
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (row[u] < 0) continue;
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = entry[u] == -1 ? 0.0f : __builtin_nanf("");
          if ((unsigned)entry[u] < (unsigned)a.c.pages) {
            if constexpr (FMT == VF_E4M3) {
              // (a scale's byte is the exponent field of 2^(byte - 127); the conversion takes 0 as 2^-127 and 255 as NaN)
              const float sc = __uint_as_float(scale[u] << 23);
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(raw[u].w[x], sc, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(raw[u].w[x], sc, true);
                v[4 * x] = lo[0]; v[4 * x + 1] = lo[1]; v[4 * x + 2] = hi[0]; v[4 * x + 3] = hi[1];
              }
            } else {
              unpack8(raw[u], v);
            }
          }
          const bool is_k = head[u] < a.c.heads;
          T *to = reinterpret_cast<T *>(is_k ? a.k : a.v) + (sp.first + i0 + row[u]) * (is_k ? a.ld_k : a.ld_v) +
                  (int64_t)(is_k ? head[u] : head[u] - a.c.heads) * a.c.dim + d0;
          store_upto8(to, n, v);
        }
      }
    }
  }
}

// lanes of a head: a power of two, one for every eight numbers of a row
int lanes_of(int width) {
  int n = 1;
  while (8 * n < width) n *= 2;
  return n;
}
// Rows of a workgroup where sequences are that long; the grid stays below what may be launched.
int rows_at_once(int64_t longest, int most) { return longest < most ? (longest < 1 ? 1 : (int)longest) : most; }
unsigned grid_of(int64_t units) { return (unsigned)(units < (1 << 20) ? units : 1 << 20); }

template <bool ODD>
void launch_append(const AppendArgs &a, int type, int format, unsigned grid, unsigned lds, hipStream_t st) {
  if (format == VF_E4M3) {
    if (type == VF_BF16) k_kv_append<uint16_t, VF_E4M3, ODD><<<grid, THREADS, lds, st>>>(a);
    else k_kv_append<float, VF_E4M3, ODD><<<grid, THREADS, lds, st>>>(a);
  } else if (type == VF_BF16) {
    k_kv_append<uint16_t, VF_BF16, ODD><<<grid, THREADS, lds, st>>>(a);
  } else {
    k_kv_append<float, VF_FP32, ODD><<<grid, THREADS, lds, st>>>(a);
  }
}

}  // namespace

int vfk_kv_append(vf_ctx *c, const vf_kv_call &call, const vf_rope *rope, const void *k, int64_t ld_k, const void *v, int64_t ld_v, int heads,
                  const void *q, int64_t ld_q, void *q_out, int64_t ld_q_out) {
  if (call.seqs->n_seq == 0 || call.seqs->tokens == 0) return VF_OK;
  AppendArgs a;
  a.c = cache_of(call.kv);
  a.s = seqs_of(call.seqs);
  a.freq = rope ? rope->freq_dev : nullptr;
  a.magnitude = rope ? rope->magnitude : 1.0f;
  a.half = rope ? rope->rotary / 2 : 0;
  a.interleaved = rope ? rope->interleaved : 0;
  a.q = q; a.k = k; a.v = v; a.q_out = q_out;
  a.ld_q = ld_q; a.ld_k = ld_k; a.ld_v = ld_v; a.ld_q_out = ld_q_out;
  a.heads = q ? heads : 0;
  a.lanes = lanes_of(a.c.width);
  const int64_t longest = longest_of(call.seqs);
  a.tb = rows_at_once(longest, 8);
  a.total = divisor_of(a.heads + 2 * a.c.heads);
  a.blocks = (int)((longest + a.tb - 1) / a.tb);
  if (a.blocks < 1) a.blocks = 1;
  const unsigned grid = grid_of((int64_t)a.s.n * a.blocks), lds = (unsigned)(a.tb * a.half * sizeof(float2));
  if (a.half % 8 != 0 && !a.interleaved) launch_append<true>(a, call.type, call.kv->format, grid, lds, c->stream);
  else launch_append<false>(a, call.type, call.kv->format, grid, lds, c->stream);
  VF_HIP(c, hipGetLastError());
  return VF_OK;
}

template <typename T>
static void launch_read(const ReadArgs &a, int format, unsigned grid, hipStream_t st) {
  if (format == VF_E4M3) k_kv_read<T, VF_E4M3><<<grid, THREADS, 0, st>>>(a);
  else if (format == VF_BF16) k_kv_read<T, VF_BF16><<<grid, THREADS, 0, st>>>(a);
  else k_kv_read<T, VF_FP32><<<grid, THREADS, 0, st>>>(a);
}

int vfk_kv_read(vf_ctx *c, const vf_kv_call &call, void *k, int64_t ld_k, void *v, int64_t ld_v) {
  if (call.seqs->n_seq == 0 || call.seqs->tokens == 0 || (!k && !v)) return VF_OK;
  ReadArgs a;
  a.c = cache_of(call.kv);
  a.s = seqs_of(call.seqs);
  a.k = k; a.v = v; a.ld_k = ld_k; a.ld_v = ld_v;
  a.lanes = lanes_of(a.c.width);
  const int64_t longest = longest_of(call.seqs);
  a.tb = rows_at_once(longest, TB);
  a.total = divisor_of(a.c.heads * ((k != nullptr) + (v != nullptr)));
  a.blocks = (int)((longest + a.tb - 1) / a.tb);
  if (a.blocks < 1) a.blocks = 1;
  const unsigned grid = grid_of((int64_t)a.s.n * a.blocks);
  if (call.type == VF_BF16) launch_read<uint16_t>(a, call.kv->format, grid, c->stream);
  else launch_read<float>(a, call.kv->format, grid, c->stream);
  VF_HIP(c, hipGetLastError());
  return VF_OK;
}
