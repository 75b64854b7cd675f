// vf_ssm_scan and vf_ssm_step: short causal convolution, selective state space scan and gate.
//
//   S_t = e^(step a) S_(t-1) + step x B^T (head_dim x n_state), y = S C + d x
//
// Token by token a state of P x N numbers is read and written once per sequence, five operations a number and
// token; in chunks (below) the same sums are products of matrices.
#include <algorithm>

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
  // Sequences in nseg segments of seg_len tokens (the last one runs to the end): seg_state [n_seq][nseg][H][P][N] holds what
  // a segment makes of nothing (behind the launch with `local`), then the state before it (behind k_ssm_join);
  // seg_log [n_seq][nseg][H] the logarithm of its decay.  nseg = 1: no segments.
  int nseg, seg_len, local;
  float *seg_state, *seg_log;
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
// Tokens [begin, end) of segment `seg`, and whether the sequence ends in it
struct Part { int begin, end; bool last; };
__device__ __forceinline__ Part part_of(const SsmArgs &p, int count, int seg) {
  if (p.nseg == 1) return {0, count, true};
  // (a segment begins at most 2^31 - 1 tokens in: seg_len nseg may be more)
  const int64_t b = (int64_t)seg * p.seg_len, e = b + p.seg_len;
  const int begin = b < count ? (int)b : count, end = seg == p.nseg - 1 || e > count ? count : (int)e;
  return {begin, end, end == count && (begin < count || seg == 0)};
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

// Sums of COUNT numbers over LANES neighbouring lanes (i: which of them this one is): in each step a lane keeps half of the numbers
// and gives the other half away, so that COUNT - 1 numbers are exchanged, not COUNT log2 LANES.
// A lane is left with kept_of numbers, from first_kept on; where lanes share a number, all of them have it.
template <int LANES, int COUNT> constexpr int kept_of() { return COUNT > LANES ? COUNT / LANES : 1; }
template <int LANES, int COUNT> __device__ __forceinline__ int first_kept(int i) {
  return COUNT >= LANES ? i * (COUNT / LANES) : i / (LANES / COUNT);
}
template <int LANES, int COUNT>
__device__ __forceinline__ void sum_lanes(float (&y)[COUNT], int i) {
  if constexpr (LANES > 1) {
    constexpr int m = LANES / 2;
    if constexpr (COUNT > 1) {
      constexpr int half = COUNT / 2;
      float rest[half];
      const bool up = i & m;
#pragma unroll
      for (int k = 0; k < half; ++k) {
        const float give = up ? y[k] : y[half + k];
        rest[k] = (up ? y[half + k] : y[k]) + __shfl_xor(give, m);
      }
      sum_lanes<m, half>(rest, i);
#pragma unroll
      for (int k = 0; k < half; ++k) y[k] = rest[k];
    } else {
      y[0] += __shfl_xor(y[0], m);
      sum_lanes<m, 1>(y, i);
    }
  }
}
// four numbers of a row of the state, `left` of which are there; zeros behind them
__device__ __forceinline__ f32x4 load_n(const float *at, int left) {
  if (left >= 4) {
    const f32v4 v = *reinterpret_cast<const f32v4 *>(at);
    return f32x4{v.v[0], v.v[1], v.v[2], v.v[3]};
  }
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (j < left) v[j] = at[j];
  return v;
}
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void store_n(float *at, int left, const f32x4 &v) {
  if (left >= 4) {
    __builtin_nontemporal_store(v, reinterpret_cast<f32x4_any *>(at));
    return;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (j < left) at[j] = v[j];
}
template <typename T> __device__ __forceinline__ float as_f32(T v) { return load1(&v); }
template <typename T> __device__ __forceinline__ T nan_of() { return sizeof(T) == 2 ? (T)0x7fc0 : (T)__uint_as_float(0x7fc00000u); }

// A workgroup's channels: R of x, then those of B and of C, `span` places each.  Channel of place k, or -1; `own`: this
// workgroup is the one that writes its convolution's state.
__device__ __forceinline__ int channel_of(const SsmArgs &p, int k, int R, int span, int h, int g, int p0, int np) {
  if (k < R) return k < np ? h * p.P + p0 + k : -1;
  k -= R;
  if (k >= 2 * span) return -1;
  const int n = k < span ? k : k - span;
  return n < p.N ? p.H * p.P + (k < span ? 0 : p.G * p.N) + g * p.N + n : -1;
}

// Token by token, fp32: a workgroup holds 256 / L PI rows p of one head's state in registers, L lanes a row, four numbers n
// each.  Eight tokens are convolved at a time, a thread a channel; their inputs were fetched while
// the eight before were worked on, and the outputs of the eight are summed over the lanes together.  What bounds it is the
// chain of a sequence's tokens, so long sequences are split (below).  MI355X: 37 sequences of up to 300 tokens, 5 heads of 40 x 24 in
// fp32, 64 us (240 with inputs asked for when they are needed and every token's outputs summed by themselves).
template <typename T, int L, int PI, int TW>
__global__ void __launch_bounds__(256, 2) k_ssm_tokens(const SsmArgs p) {
  constexpr int R = 256 / L * PI, SPAN = 4 * L, PLACES = R + 2 * SPAN, NC = (PLACES + 255) / 256, TB = 8;
  constexpr int COUNT = TB * PI, KEPT = kept_of<L, COUNT>();
  __shared__ float ux[2][TB][R];
  __shared__ __align__(16) float ubc[2][TB][2 * SPAN];
  __shared__ float udt[2][TB], uda[2][TB];
  const int tid = threadIdx.x, i = tid & (L - 1), prow = tid / L, n = 4 * i;
  const int slices = (p.P + R - 1) / R;
  const int h = (int)blockIdx.x / slices, p0 = ((int)blockIdx.x % slices) * R;
  const int g = h / (p.H / p.G);
  const int np = p.P - p0 < R ? p.P - p0 : R;
  const float A = p.a[h], D = p.d ? p.d[h] : 0.0f, bias_dt = p.dt_bias ? p.dt_bias[h] : 0.0f;
  const bool owns_bc = h == g * (p.H / p.G) && p0 == 0;  // writes the convolution's state of its group's B and C
  int chan[NC];
  float taps[NC][TW], bias[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    chan[j] = channel_of(p, j * 256 + tid, R, SPAN, h, g, p0, np);
    bias[j] = chan[j] >= 0 && p.conv_b ? p.conv_b[chan[j]] : 0.0f;
#pragma unroll
    for (int k = 0; k < TW; ++k) taps[j][k] = chan[j] >= 0 && k >= TW - p.W ? p.conv_w[(int64_t)chan[j] * p.W + k - (TW - p.W)] : 0.0f;
  }
  // the outputs that are left to this lane: number v is token v / PI, row PI prow + v % PI
  const int v0 = first_kept<L, COUNT>(i);
  const bool stores = !p.local && i % (COUNT < L ? L / COUNT : 1) == 0;

  const int64_t parts = (int64_t)p.n_seq * p.nseg, size = (int64_t)p.P * p.N;
  for (int64_t sx = blockIdx.y; sx < parts; sx += gridDim.y) {
    const int s = (int)(sx / p.nseg), seg = (int)(sx - (int64_t)s * p.nseg);
    if (p.local && seg == p.nseg - 1) continue;
    const Span sp = span_of(p, s);
    const Part pt = part_of(p, sp.count, seg);
    if (!p.local && seg > 0 && pt.begin >= pt.end) continue;
    const int slot = slot_of(p.slots_in, p.has_in, p.n_in, s), slot_to = slot_of(p.slots_out, p.has_out, p.n_out, s);
    // where the state before this part is, and where it goes
    float *const mine = p.nseg > 1 ? p.seg_state + (sx * p.H + h) * size + (int64_t)p0 * p.N : nullptr;
    const float *first = p.nseg > 1 ? mine : slot >= 0 ? p.ssm_in + ((int64_t)slot * p.H + h) * size + (int64_t)p0 * p.N : nullptr;
    float *left = p.local ? mine : pt.last && slot_to >= 0 ? p.ssm_out + ((int64_t)slot_to * p.H + h) * size + (int64_t)p0 * p.N : nullptr;
    if (p.local) first = nullptr;
    f32x4 S[PI];
    float log_decay = 0.0f;
    const float fill = slot == -2 && p.nseg == 1 ? __uint_as_float(0x7fc00000u) : 0.0f;
#pragma unroll
    for (int k = 0; k < PI; ++k) {
      const int pr = prow * PI + k;
      S[k] = f32x4{fill, fill, fill, fill};
      if (first && pr < np && n < p.N) S[k] = load_n(first + (int64_t)pr * p.N + n, p.N - n);
    }
    float past[NC][TW - 1];
    T raw[NC][TB], raw_z[KEPT], raw_dt = 0;
    // (tokens behind the end: the last one again, taken as zeros)
    auto row_of = [&](int t) { return sp.first + (t < pt.end ? t : pt.end - 1); };
    auto ask = [&](int t0) {
#pragma unroll
      for (int j = 0; j < NC; ++j)
        if (chan[j] >= 0) {
#pragma unroll
          for (int t = 0; t < TB; ++t) raw[j][t] = reinterpret_cast<const T *>(p.xbc)[row_of(t0 + t) * p.ld_xbc + chan[j]];
        }
      if (tid < TB) raw_dt = reinterpret_cast<const T *>(p.dt)[row_of(t0 + tid) * p.ld_dt + h];
    };
    if (pt.begin < pt.end) {
#pragma unroll
      for (int j = 0; j < NC; ++j)
#pragma unroll
        for (int k = 0; k < TW - 1; ++k)
          past[j][k] = chan[j] >= 0 && k >= TW - p.W ? conv_input<T>(p, sp, slot, chan[j], pt.begin - (TW - 1) + k) : 0.0f;
      ask(pt.begin);
    }
    for (int t0 = pt.begin; t0 < pt.end; t0 += TB) {
      const int nt = pt.end - t0 < TB ? pt.end - t0 : TB, buf = (t0 - pt.begin) / TB & 1;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int k = j * 256 + tid;
        if (k >= PLACES) continue;
        float in[TW - 1 + TB];
#pragma unroll
        for (int e = 0; e < TW - 1; ++e) in[e] = past[j][e];
#pragma unroll
        for (int t = 0; t < TB; ++t) in[TW - 1 + t] = chan[j] >= 0 ? as_f32<T>(raw[j][t]) : 0.0f;
#pragma unroll
        for (int t = 0; t < TB; ++t) {
          float v = bias[j];
#pragma unroll
          for (int e = 0; e < TW; ++e) v = e >= TW - p.W ? fmaf(taps[j][e], in[t + e], v) : v;
          v = chan[j] >= 0 && t < nt ? silu(v) : 0.0f;
          if (k < R) ux[buf][t][k] = v;
          else ubc[buf][t][k - R] = v;
        }
#pragma unroll
        for (int e = 0; e < TW - 1; ++e) past[j][e] = in[TB + e];
      }
      if (tid < TB) {
        const float dt = tid < nt ? softplus(as_f32<T>(raw_dt) + bias_dt) : 0.0f;
        udt[buf][tid] = dt;
        uda[buf][tid] = __expf(dt * A);
      }
      if (p.z && stores) {
#pragma unroll
        for (int e = 0; e < KEPT; ++e) {
          const int t = (v0 + e) / PI, pr = prow * PI + (v0 + e) % PI;
          if (t < nt && pr < np) raw_z[e] = reinterpret_cast<const T *>(p.z)[(sp.first + t0 + t) * p.ld_z + h * p.P + p0 + pr];
        }
      }
      if (t0 + TB < pt.end) ask(t0 + TB);
      __syncthreads();  // (two buffers: nobody writes the one that is read before all have passed the next barrier)
      float y[COUNT];
#pragma unroll
      for (int k = 0; k < COUNT; ++k) y[k] = 0.0f;
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        if ((t == 2 || t == 4) && nt <= t) break;  // (short sequences; a line at every token would cost the long ones 8 %)
        const float dt = udt[buf][t], da = uda[buf][t];
        log_decay = fmaf(dt, A, log_decay);
        const f32x4 B = *reinterpret_cast<const f32x4 *>(&ubc[buf][t][n]);
#pragma unroll
        for (int k = 0; k < PI; ++k) {
          const float dx = dt * ux[buf][t][prow * PI + k];
#pragma unroll
          for (int j = 0; j < 4; ++j) S[k][j] = fmaf(S[k][j], da, dx * B[j]);
        }
        if (p.local) continue;
        const f32x4 Cv = *reinterpret_cast<const f32x4 *>(&ubc[buf][t][SPAN + n]);
#pragma unroll
        for (int k = 0; k < PI; ++k) {
#pragma unroll
          for (int j = 0; j < 4; ++j) y[t * PI + k] = fmaf(S[k][j], Cv[j], y[t * PI + k]);
        }
        // (these sums are made here: moved behind the last token they would keep eight tokens' states in registers)
#pragma unroll
        for (int k = 0; k < PI; ++k) asm volatile("" : "+v"(y[t * PI + k]));
      }
      if (p.local) continue;
      sum_lanes<L, COUNT>(y, i);
      if (stores) {
#pragma unroll
        for (int e = 0; e < KEPT; ++e) {
          const int t = (v0 + e) / PI, pr = prow * PI + (v0 + e) % PI;
          if (t >= nt || pr >= np) continue;
          float v = fmaf(D, ux[buf][t][pr], y[e]);
          if (p.z) v *= silu(as_f32<T>(raw_z[e]));
          store1(reinterpret_cast<T *>(p.out) + (sp.first + t0 + t) * p.ld_out + h * p.P + p0 + pr, v);
        }
      }
    }
    __syncthreads();  // (the next part begins with the first buffer again)
    if (p.local && tid == 0 && p0 == 0) p.seg_log[sx * p.H + h] = log_decay;
    if (!left) continue;
#pragma unroll
    for (int k = 0; k < PI; ++k) {
      const int pr = prow * PI + k;
      if (pr < np && n < p.N) store_n(left + (int64_t)pr * p.N + n, p.N - n, S[k]);
    }
    if (p.local || p.conv_later || p.W == 1) continue;
#pragma unroll
    for (int j = 0; j < NC; ++j)
      if (chan[j] >= 0 && (owns_bc || j * 256 + tid < R)) conv_state<T>(p, sp, slot, slot_to, chan[j]);
  }
}

// One token: L lanes hold a row p of the state, four numbers n each; a thread has PI rows of it.  A workgroup takes the same rows p of one
// head for `each` sequences one after the other: the layer's weights stay in registers, and the next sequence's state and
// inputs are on their way while this one's are worked on.  Every state is read and written once, past the caches on the
// way out: the memory's rate bounds it.  Workgroups of one head run next to each other, so that the states of
// parents that many rows continue come from the second-level cache.  MI355X: 1024 rows of 32 heads of 64 x 128 behind 64 parents, 1.17 GB,
// 225 us = 5.2 TB/s (554 by k_ssm_tokens as it was, where a token's loads wait for each other); one row 5.5 us.
template <typename T, int PI, int NC, int TW>
struct StepIn {
  f32x4 S[PI];
  T window[NC][TW], dt, z;
};
template <typename T, int L, int PI, int TW>
__global__ void __launch_bounds__(256) k_ssm_step(const SsmArgs p, int slices, int each, int turns) {
  constexpr int RP = 256 / L, R = RP * PI, SPAN = 4 * L, PLACES = R + 2 * SPAN, NC = (PLACES + 255) / 256;
  __shared__ __align__(16) float u[2][PLACES];
  const int tid = threadIdx.x, i = tid & (L - 1), prow = tid / L, n = 4 * i;
  uint32_t id = blockIdx.x;
  const uint32_t chunk8 = gridDim.x / 8;
  if (id < chunk8 * 8) id = (id & 7) * chunk8 + (id >> 3);
  const int unit = (int)(id / (uint32_t)turns), s0 = (int)(id - (uint32_t)unit * turns) * each;
  const int s1 = p.n_seq - s0 < each ? p.n_seq : s0 + each;
  const int h = unit / slices, p0 = (unit - h * slices) * R, g = h / (p.H / p.G);
  const int np = p.P - p0 < R ? p.P - p0 : R;
  const float A = p.a[h], D = p.d ? p.d[h] : 0.0f, bias_dt = p.dt_bias ? p.dt_bias[h] : 0.0f;
  const bool owns_bc = h == g * (p.H / p.G) && p0 == 0;
  const int64_t size = (int64_t)p.P * p.N;
  int chan[NC];
  float taps[NC][TW], bias[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    chan[j] = channel_of(p, j * 256 + tid, R, SPAN, h, g, p0, np);
    bias[j] = chan[j] >= 0 && p.conv_b ? p.conv_b[chan[j]] : 0.0f;
#pragma unroll
    for (int k = 0; k < TW; ++k) taps[j][k] = chan[j] >= 0 && k >= TW - p.W ? p.conv_w[(int64_t)chan[j] * p.W + k - (TW - p.W)] : 0.0f;
  }
  const int p_own = prow * PI + first_kept<L, PI>(i);
  const bool stores = i % (L / PI) == 0 && p_own < np;

  auto ask = [&](int s, int slot, StepIn<T, PI, NC, TW> &in) {
#pragma unroll
    for (int k = 0; k < PI; ++k) {
      const int pr = prow * PI + k;
      const float fill = slot == -2 ? __uint_as_float(0x7fc00000u) : 0.0f;
      in.S[k] = f32x4{fill, fill, fill, fill};
      if (slot >= 0 && pr < np && n < p.N) in.S[k] = load_n(p.ssm_in + ((int64_t)slot * p.H + h) * size + (int64_t)(p0 + pr) * p.N + n, p.N - n);
    }
#pragma unroll
    for (int j = 0; j < NC; ++j) {
#pragma unroll
      for (int k = 0; k < TW - 1; ++k) in.window[j][k] = slot == -2 ? nan_of<T>() : (T)0;
      if (chan[j] < 0) continue;
      if (slot >= 0) {
        const T *at = reinterpret_cast<const T *>(p.conv_in) + ((int64_t)slot * p.C + chan[j]) * (p.W - 1);
#pragma unroll
        for (int k = 0; k < TW - 1; ++k)
          if (k >= TW - p.W) in.window[j][k] = at[k - (TW - p.W)];
      }
      in.window[j][TW - 1] = reinterpret_cast<const T *>(p.xbc)[s * p.ld_xbc + chan[j]];
    }
    in.dt = reinterpret_cast<const T *>(p.dt)[s * p.ld_dt + h];
    if (p.z && stores) in.z = reinterpret_cast<const T *>(p.z)[s * p.ld_z + h * p.P + p0 + p_own];
  };
  StepIn<T, PI, NC, TW> next;
  if (s0 < s1) ask(s0, slot_of(p.slots_in, p.has_in, p.n_in, s0), next);
  int slot_next = s0 + 1 < s1 ? slot_of(p.slots_in, p.has_in, p.n_in, s0 + 1) : -1;
  for (int s = s0; s < s1; ++s) {
    StepIn<T, PI, NC, TW> in = next;
    const int slot_to = slot_of(p.slots_out, p.has_out, p.n_out, s);
    if (s + 1 < s1) ask(s + 1, slot_next, next);
    if (s + 2 < s1) slot_next = slot_of(p.slots_in, p.has_in, p.n_in, s + 2);
    float *now = u[(s - s0) & 1];  // (two buffers: one barrier a sequence)
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int k = j * 256 + tid;
      if (k >= PLACES) continue;
      float v = bias[j];
#pragma unroll
      for (int e = 0; e < TW; ++e) v = e >= TW - p.W ? fmaf(taps[j][e], as_f32<T>(in.window[j][e]), v) : v;
      now[k] = chan[j] >= 0 ? silu(v) : 0.0f;
      if (chan[j] < 0 || slot_to < 0 || p.conv_later || !(owns_bc || k < R)) continue;
      T *to = reinterpret_cast<T *>(p.conv_out) + ((int64_t)slot_to * p.C + chan[j]) * (p.W - 1);
#pragma unroll
      for (int e = 1; e < TW; ++e)
        if (e > TW - p.W) to[e - 1 - (TW - p.W)] = in.window[j][e];
    }
    const float dt = softplus(as_f32<T>(in.dt) + bias_dt), da = __expf(dt * A);
    __syncthreads();
    const f32x4 B = *reinterpret_cast<const f32x4 *>(now + R + n), Cv = *reinterpret_cast<const f32x4 *>(now + R + SPAN + n);
    float y[PI];
#pragma unroll
    for (int k = 0; k < PI; ++k) {
      const float dx = dt * now[prow * PI + k];
      y[k] = 0.0f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        in.S[k][j] = fmaf(in.S[k][j], da, dx * B[j]);
        y[k] = fmaf(in.S[k][j], Cv[j], y[k]);
      }
      const int pr = prow * PI + k;
      if (slot_to >= 0 && pr < np && n < p.N)
        store_n(p.ssm_out + ((int64_t)slot_to * p.H + h) * size + (int64_t)(p0 + pr) * p.N + n, p.N - n, in.S[k]);
    }
    sum_lanes<L, PI>(y, i);
    if (!stores) continue;
    float v = fmaf(D, now[p_own], y[0]);
    if (p.z) v *= silu(as_f32<T>(in.z));
    store1(reinterpret_cast<T *>(p.out) + s * p.ld_out + h * p.P + p0 + p_own, v);
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

// The states before the segments of a sequence, one after the other: four neighbouring numbers a thread.
__global__ void __launch_bounds__(256) k_ssm_join(const SsmArgs p) {
  const int64_t size = (int64_t)p.H * p.P * p.N, total = p.n_seq * size;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int s = (int)(i / size);
    const int64_t e = i - s * size;
    const int h = (int)(e / ((int64_t)p.P * p.N));
    const int slot = slot_of(p.slots_in, p.has_in, p.n_in, s);
    float S = slot == -2 ? __uint_as_float(0x7fc00000u) : slot >= 0 ? p.ssm_in[slot * size + e] : 0.0f;
    float *at = p.seg_state + (int64_t)s * p.nseg * size + e;
    const float *lg = p.seg_log + (int64_t)s * p.nseg * p.H + h;
    int seg = 0;
    for (; seg + 8 < p.nseg; seg += 8) {
      float own[8], d[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        own[k] = at[(seg + k) * size];
        d[k] = lg[(seg + k) * p.H];
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        at[(seg + k) * size] = S;
        S = fmaf(__expf(d[k]), S, own[k]);
      }
    }
    for (; seg < p.nseg - 1; ++seg) {
      const float own = at[seg * size];
      at[seg * size] = S;
      S = fmaf(__expf(lg[seg * p.H]), S, own);
    }
    at[seg * size] = S;
  }
}

inline int blocks_for(int64_t threads) {
  const int64_t b = (threads + 255) / 256;
  return (int)(b < (1 << 20) ? b : (1 << 20));
}

// How a call is split: into segments of at least `least` tokens that fill one to four rounds of the `want` workgroups that run at a
// time, `each` for one segment of all sequences, if the rounds' tokens get fewer by it: a token of a split sequence is
// worked on twice, at about 1.6 of its cost.  Without the scratch for it (captured stream, no memory) the sequences stay whole.
void split(vf_ctx *c, SsmArgs &p, int64_t longest, int64_t each, int64_t want, int unit, int64_t least) {
  p.nseg = 1;
  p.seg_len = 0;
  if (each <= 0 || each >= want || longest < 2 * least) return;
  int64_t n = 1, cost = longest * 10;  // (one round)
  for (int64_t rounds = 1; rounds <= 4; ++rounds) {
    int64_t k = rounds * want / each;
    if (k > longest / least) k = longest / least;
    const int64_t with = (each * k + want - 1) / want * ((longest + k - 1) / k) * 16;
    if (k > 1 && with < cost) {
      n = k;
      cost = with;
    }
  }
  int64_t len = ((longest + n - 1) / n + unit - 1) / unit * unit;
  n = (longest + len - 1) / len;
  if (n < 2) return;
  // (at most 256 MiB of states: 8192 numbers for each wave of four rounds, which are eight waves on each of 256 compute units)
  const int64_t states = (int64_t)p.n_seq * n * p.H * p.P * p.N, logs = (int64_t)p.n_seq * n * p.H;
  float *at = static_cast<float *>(vfk_ops_scratch(c, (size_t)(states + logs) * sizeof(float)));
  if (!at) return;
  p.nseg = (int)n;
  p.seg_len = (int)len;
  p.seg_state = at;
  p.seg_log = at + states;
}

// Runs `launch` for whole sequences, or for segments: what each makes of nothing, the states before them, the rest.
template <typename F>
int run_parts(vf_ctx *c, SsmArgs &p, F launch) {
  if (p.nseg > 1) {
    p.local = 1;
    int rc = launch();
    if (rc != VF_OK) return rc;
    p.local = 0;
    k_ssm_join<<<blocks_for((int64_t)p.n_seq * p.H * p.P * p.N), 256, 0, c->stream>>>(p);
    VF_HIP(c, hipGetLastError());
  }
  return launch();
}

constexpr int SEQ_TOKENS = 8;  // tokens that k_ssm_tokens takes at a time

template <typename T, int L, int PI>
int launch_tokens(vf_ctx *c, SsmArgs &p, int64_t longest) {
  constexpr int R = 256 / L * PI;
  const int slices = (p.P + R - 1) / R;
  split(c, p, longest, (int64_t)p.n_seq * p.H * slices, 1024, SEQ_TOKENS, 64);
  const int64_t parts = (int64_t)p.n_seq * p.nseg;
  // Many parts: a workgroup takes several one after the other, up to 16, and keeps the layer's weights for them; there are four times as
  // many workgroups as run at a time (five of four waves on a compute unit), for the sake of unequal parts.
  const int64_t x = (int64_t)p.H * slices, most = std::max((int64_t)4 * 1280 / x, (parts + 15) / 16);
  const dim3 grid((unsigned)x, (unsigned)std::min(std::min(parts, std::max(most, (int64_t)1)), (int64_t)32768));
  return run_parts(c, p, [&] {
    if (p.W <= 4) k_ssm_tokens<T, L, PI, 4><<<grid, 256, 0, c->stream>>>(p);
    else k_ssm_tokens<T, L, PI, 8><<<grid, 256, 0, c->stream>>>(p);
    VF_HIP(c, hipGetLastError());
    return VF_OK;
  });
}
template <typename T>
int tokens(vf_ctx *c, SsmArgs &p, int64_t longest) {
  // 64 rows p a workgroup (32 of more than 128 numbers n), or a thread's one row where there are too few rows, or too few workgroups
  // for the compute units
  const bool wide = p.P > 16 && ((int64_t)p.n_seq * p.H * ((p.P + 63) / 64) >= 512 || longest >= 256);
  if (p.N <= 16) return launch_tokens<T, 4, 1>(c, p, longest);
  if (p.N <= 32) return wide ? launch_tokens<T, 8, 2>(c, p, longest) : launch_tokens<T, 8, 1>(c, p, longest);
  if (p.N <= 64) return wide ? launch_tokens<T, 16, 4>(c, p, longest) : launch_tokens<T, 16, 1>(c, p, longest);
  if (p.N <= 128) return wide ? launch_tokens<T, 32, 8>(c, p, longest) : launch_tokens<T, 32, 1>(c, p, longest);
  return wide ? launch_tokens<T, 64, 8>(c, p, longest) : launch_tokens<T, 64, 1>(c, p, longest);
}

template <typename T, int L, int PI>
int launch_step(vf_ctx *c, const SsmArgs &p) {
  constexpr int R = 256 / L * PI;
  const int slices = (p.P + R - 1) / R;
  const int64_t units = (int64_t)p.H * slices, total = units * p.n_seq;
  // sequences a workgroup: four rounds of the workgroups that run at a time, for the sake of an even end; and at most 2^22 workgroups
  int64_t each = total / 4096;
  each = each < 1 ? 1 : each > 16 ? 16 : each;
  if (each < (total >> 22) + 1) each = (total >> 22) + 1;
  if (each > p.n_seq) each = p.n_seq;
  const int turns = (int)((p.n_seq + each - 1) / each);
  const unsigned blocks = (unsigned)(units * turns);
  if (p.W <= 4) k_ssm_step<T, L, PI, 4><<<blocks, 256, 0, c->stream>>>(p, slices, (int)each, turns);
  else k_ssm_step<T, L, PI, 8><<<blocks, 256, 0, c->stream>>>(p, slices, (int)each, turns);
  VF_HIP(c, hipGetLastError());
  return VF_OK;
}
template <typename T>
int step(vf_ctx *c, const SsmArgs &p) {
  // 64 rows p a workgroup (32 of more than 128 numbers n), or 16 (8) where there are too few rows, or too few workgroups for the compute
  // units
  const bool wide = p.P > 16 && (int64_t)p.n_seq * p.H * ((p.P + 63) / 64) >= 512;
  if (p.N <= 16) return launch_step<T, 4, 1>(c, p);
  if (p.N <= 32) return wide ? launch_step<T, 8, 2>(c, p) : launch_step<T, 8, 1>(c, p);
  if (p.N <= 64) return wide ? launch_step<T, 16, 4>(c, p) : launch_step<T, 16, 1>(c, p);
  if (p.N <= 128) return wide ? launch_step<T, 32, 8>(c, p) : launch_step<T, 32, 2>(c, p);
  return wide ? launch_step<T, 64, 8>(c, p) : launch_step<T, 64, 2>(c, p);
}

// ---- in chunks of 32 tokens on the matrix cores ----
//
// With c_t = sum of step a over the chunk's tokens up to t, and the state S before the chunk:
//   y_t = e^(c_t) S C_t + sum_(s <= t) (C_t . B_s) e^(c_t - c_s) step_s x_s + d x_t
//   S'  = e^(c_31) S + sum_s step_s e^(c_31 - c_s) x_s B_s^T
// A wave holds 16 PT rows p of one head's state as the accumulators of the second sum, transposed (rows n, columns p): in that
// form a lane's numbers are, rounded to bf16, its part of an operand of the first sum's product with C, with the n of
// a k-step in another order, which the operand read from the LDS then takes too; the same holds for the 32 x 32 matrix
// (C_t . B_s) ... and its product with x.  So nothing but the convolved inputs passes through the LDS.
// Rounding: the outputs are bf16.  As operands S and C (for S C_t), the 32 x 32 matrix with d on its diagonal, and x are in two parts of
// bf16; B and C (for C_t . B_s) are rounded to one, which is less than 2 % of an output's own rounding over 300 tokens (error to the
// outputs' size in root mean square 1.68e-3, of exact outputs rounded 1.66e-3; with S and C in one part behind a state of the
// outputs' size 2.8e-3, and 3 - 15 % less time).  The state is fp32: what it takes up,
// x step e^(...) and B, is in two parts of fp16 each, 22 bits together, scaled by powers of two to fp16's range (the products with
// x by their row's largest, B by its row's), which the sum takes back.
//
// The waves of a workgroup take neighbouring heads of one group and convolve its B and C together.  All bytes of x, z, out
// pass once; what bounds the kernel is the vector work on them: convolution, silu (two quarter-rate
// functions a number) and the operands' parts, among it 220 to 340 scalar registers that do not fit and are kept in lanes of vector
// registers.  MI355X: 16,384 sequences of 50 tokens, 4 heads of 64 x 64, 670 us = 2.2 TB/s; a prompt of 16,384 tokens, 32 heads of 64 x 128, 268 us
// (under the profiler local states 90, join 13, outputs 185).  More than 128 numbers n: 268 bytes a lane are in memory.

constexpr int Q = 32;            // tokens of a chunk
constexpr int XS = Q + 4;        // row of x in the LDS, floats
// place of row n of the transposed B, in fp16 numbers: 80 bytes a row and 16 more after eight, so that the eight-token pieces that
// neighbouring lanes write (channels four apart) lie in different banks
__device__ __forceinline__ int bt_row(int n) { return n * (Q + 8) + (n >> 3) * 8; }
__host__ __device__ constexpr int bt_size(int np) { return np * (Q + 8) + (np >> 3) * 8; }

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ uint32_t pack_h(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}
// what is left of two numbers behind their parts in fp16 / bf16
__device__ __forceinline__ uint32_t rest_h(float a, float b, uint32_t hi) {
  const f16x2 h = __builtin_bit_cast(f16x2, hi);
  return pack_h(a - (float)h[0], b - (float)h[1]);
}
__device__ __forceinline__ uint32_t rest_b(float a, float b, uint32_t hi) {
  return pack2(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
}
__device__ __forceinline__ bool is_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }
// 2^k that brings a magnitude below 2^15, and its reciprocal; k is cut where either would leave the normal numbers
__device__ __forceinline__ float scale_to_f16(float top) {
  const int e = (int)(__float_as_uint(top) >> 23);
  return __uint_as_float((uint32_t)min(max(268 - e, 1), 253) << 23);
}
__device__ __forceinline__ float power_reciprocal(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

// Rows of a chunk as the memory instructions with a range check see them: a row before the sequence or behind the part
// reads as zeros and is not written.  `at`: row `base` of the matrix; rows base .. end - 1 are there.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
struct Rows { __amdgpu_buffer_rsrc_t rsrc; uint32_t ld2; int base; };
__device__ __forceinline__ Rows rows_of(const void *matrix, int64_t first, int64_t ld, int base, int end) {
  const char *at = static_cast<const char *>(matrix) + 2 * ((first + base) * ld);
  const int n = end > base ? end - base : 0;
  return {__builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(at), 0, (int)(n * (uint32_t)(2 * ld)), 0x00027000), (uint32_t)(2 * ld), base};
}
__device__ __forceinline__ uint2 load4(const Rows &m, int t, uint32_t byte) {
  const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(m.rsrc, (int)((uint32_t)(t - m.base) * m.ld2 + byte), 0, 0);
  return make_uint2(v[0], v[1]);
}
__device__ __forceinline__ void store4(const Rows &m, int t, uint32_t byte, const uint2 &v) {
  const u32x2 u = {v.x, v.y};
  __builtin_amdgcn_raw_buffer_store_b64(u, m.rsrc, (int)((uint32_t)(t - m.base) * m.ld2 + byte), 0, 0);
}

// Inputs of four channels for tokens t0 - 3 .. t0 - 4 + NR, byte `byte` of their rows
template <int NR>
__device__ __forceinline__ void fetch(const Rows &m, int t0, uint32_t byte, bool on, uint2 (&raw)[NR]) {
  const uint32_t at = on ? (uint32_t)(t0 - 3 - m.base) * m.ld2 + byte : 0x80000000u;  // (past the end of any chunk)
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const u32x2 v = __builtin_amdgcn_raw_buffer_load_b64(m.rsrc, (int)(at + r * m.ld2), 0, 0);
    raw[r] = make_uint2(v[0], v[1]);
  }
}
// Rows -3, -2, -1 of channels c0 .. c0 + 3 from the convolution's state, [channel][W - 1]
template <int NR>
__device__ __forceinline__ void fetch_state(const SsmArgs &p, int slot, int c0, uint2 (&raw)[NR]) {
  if (slot == -1) return;
  const int w1 = p.W - 1;
  const uint16_t *st = reinterpret_cast<const uint16_t *>(p.conv_in) + ((int64_t)slot * p.C + c0) * w1 - (3 - w1);
#pragma unroll
  for (int r = 0; r < 3; ++r) {
    if (slot == -2) raw[r] = make_uint2(0x7fc07fc0u, 0x7fc07fc0u);
    else if (r >= 3 - w1) raw[r] = make_uint2(st[r] | (uint32_t)st[w1 + r] << 16, st[2 * w1 + r] | (uint32_t)st[3 * w1 + r] << 16);
  }
}
// silu of the convolution for channel k of the four, divided by -ln 2: with weights and bias times -log2(e) the sum s is the exponent
// of silu's exponential, and s / (1 + 2^s) the result.  The constant is taken back where the results meet steps and decays.
// Weights in the LDS: four taps a channel, and the biases.  Of fewer taps (FOUR false) the first 4 - W are not there: an input that is not
// finite is not to reach tokens that do not see it by way of a zero.
// Tokens that are not there give silu(bias); their steps are zero and their outputs are not written.
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
template <int TB, bool FOUR>
__device__ __forceinline__ void convolve(const uint2 (&raw)[TB + 3], int k, int W, const float *w, const float *b, float (&v)[TB]) {
  const f32x4 tap = *reinterpret_cast<const f32x4 *>(w + 4 * k);
  const float bias = b[k];
#pragma unroll
  for (int t = 0; t < TB; ++t) {
    float s = bias;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = k < 2 ? raw[t + i].x : raw[t + i].y;
      const float with = fmaf(tap[i], __uint_as_float(k & 1 ? u & 0xffff0000u : u << 16), s);
      s = FOUR || i >= 4 - W ? with : s;
    }
    v[t] = s * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(s));
  }
}
// The largest magnitude, as bits, of TB numbers in each of 32 / TB neighbouring lanes (magnitudes compare as integers); NaN if one is.
__device__ __forceinline__ uint32_t max_abs(uint32_t a, float b, float c) {
  asm("v_maximum3_f32 %0, %1, |%2|, |%3|" : "=v"(a) : "v"(a), "v"(b), "v"(c));
  return a;
}
template <int CTRL>
__device__ __forceinline__ uint32_t max_lanes(uint32_t m) {
  return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, CTRL, 0xf, 0xf, true));
}
// over the lanes r, 16 + r, 32 + r, 48 + r
__device__ __forceinline__ uint32_t max_rows(uint32_t m) {
  const auto a = __builtin_amdgcn_permlane16_swap(m, m, false, false);
  m = max((uint32_t)a[0], (uint32_t)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  return max((uint32_t)b[0], (uint32_t)b[1]);
}
template <int TB>
__device__ __forceinline__ float top_of_32(const float (&v)[TB]) {
  uint32_t m = 0;
#pragma unroll
  for (int t = 0; t < TB; t += 2) m = max_abs(m, v[t], v[t + 1]);
  m = max_lanes<0xB1>(m);               // lanes 1 0 3 2
  m = max_lanes<0x4E>(m);               // lanes 2 3 0 1
  if (TB == 4) m = max_lanes<0x141>(m); // lanes 7 .. 0 of eight
  return __uint_as_float(m);
}
// the value N lanes before, or behind, in the same 16, zero where there is none
template <int N>
__device__ __forceinline__ float lanes_before(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x110 + N, 0xf, 0xf, true));
}
template <int N>
__device__ __forceinline__ float lanes_behind(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x100 + N, 0xf, 0xf, true));
}
// sums over the 16 lanes up to a lane, and from a lane on
__device__ __forceinline__ float sum_up_to(float v) {
  v += lanes_before<1>(v);
  v += lanes_before<2>(v);
  v += lanes_before<4>(v);
  return v + lanes_before<8>(v);
}
__device__ __forceinline__ float sum_from(float v) {
  v += lanes_behind<1>(v);
  v += lanes_behind<2>(v);
  v += lanes_behind<4>(v);
  return v + lanes_behind<8>(v);
}

__device__ __forceinline__ bf16x8 frag16(const uint16_t *at) { return *reinterpret_cast<const bf16x8 *>(at); }
// k = 8 q + i of the operand is number 4 q + i, i < 4, and 16 + 4 q + i - 4 of the row: how accumulators lie
__device__ __forceinline__ uint4 frag_acc(const uint16_t *row, int q) {
  const uint2 a = *reinterpret_cast<const uint2 *>(row + 4 * q), b = *reinterpret_cast<const uint2 *>(row + 16 + 4 * q);
  return make_uint4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ bf16x8 as_b(const uint4 &v) { return __builtin_bit_cast(bf16x8, v); }
__device__ __forceinline__ f16x8 as_h(const uint4 &v) { return __builtin_bit_cast(f16x8, v); }
__device__ __forceinline__ uint4 frag_of(const f32x4 &a, const f32x4 &b) {
  return make_uint4(pack2(a[0], a[1]), pack2(a[2], a[3]), pack2(b[0], b[1]), pack2(b[2], b[3]));
}
__device__ __forceinline__ uint4 rest_of(const f32x4 &a, const f32x4 &b, const uint4 &h) {
  return make_uint4(rest_b(a[0], a[1], h.x), rest_b(a[2], a[3], h.y), rest_b(b[0], b[1], h.z), rest_b(b[2], b[3], h.w));
}
#define VF_MFMA_B(a, b, c) __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0)
#define VF_MFMA_H(a, b, c) __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0)

// LDS: B and C by tokens, C's second part, B by n in two parts and its scales; per wave x by p and its rows' largest, weights of the convolution of all of
// these channels; per wave five numbers for each of the chunk's tokens.
constexpr int ROWS = 256;  // most rows p of a workgroup: PT tiles of 16 a wave
// `rows` of them, in `nw` waves
template <int NT> __host__ __device__ constexpr size_t chunk_lds(int rows, int nw) {
  return sizeof(uint16_t) * (3 * Q * (16 * NT + 8) + 2 * bt_size(16 * NT)) +
         sizeof(float) * (16 * NT + rows * (XS + 1) + 6 * (32 * NT + rows) + nw * 5 * Q);
}

template <int NT, int PT, bool LOCAL, bool FOUR>
__global__ void __launch_bounds__(1024 / PT, 2) k_ssm_chunks(const SsmArgs p) {
  extern __shared__ __align__(16) char smem[];
  constexpr int NP = 16 * NT, NS = NP + 8, KN = NT / 2, PS = 16 * PT;
  // Tokens of B and C that a thread takes at a time, so that there is one piece of x and one of B and C for a thread, or one of either
  constexpr int TB = PT == 4 ? 4 : 8;
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, q = lane >> 4, nthr = blockDim.x, nw = nthr >> 6;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // (what goes by the wave is held once, not per lane)
  uint16_t *Bs = reinterpret_cast<uint16_t *>(smem), *Cs = Bs + Q * NS, *CsL = Cs + Q * NS, *BtH = CsL + Q * NS, *BtL = BtH + bt_size(NP);
  float *bscale = reinterpret_cast<float *>(BtL + bt_size(NP));
  float *Xall = bscale + NP, *xsall = Xall + nw * PS * XS, *wl = xsall + nw * PS, *bl = wl + 4 * (2 * NP + nw * PS);
  int *chans = reinterpret_cast<int *>(bl + 2 * NP + nw * PS);
  // per token: exponent of its decay; their sums over the tokens of its 16 up to it, and behind it; factors of its product with B
  float *dec = bl + 2 * (2 * NP + nw * PS) + wave * 5 * Q, *upto = dec + Q, *rest = upto + Q, *stp = rest + Q, *wgt = stp + Q;
  float *X = Xall + wave * PS * XS, *xs = xsall + wave * PS;

  const int slices = (p.P + PS - 1) / PS, jobs = p.H / p.G * slices, per = (jobs + nw - 1) / nw, each = per * p.G;
  // Workgroups of one part share B and C: they get neighbouring places on one of the eight dies, to which the hardware
  // deals workgroups in turn.  A workgroup takes the same heads of every `stride`-th part.
  const int parts = p.n_seq * p.nseg, stride = (int)(gridDim.x / (unsigned)each);
  uint32_t id = blockIdx.x;
  const uint32_t chunk8 = gridDim.x / 8;
  if (id < chunk8 * 8) id = (id & 7) * chunk8 + (id >> 3);
  const int sx0 = (int)(id / (uint32_t)each), wg = (int)(id - (uint32_t)sx0 * each), g = wg / per, job = (wg - g * per) * nw + wave;
  const bool on = job < jobs;
  const int h = g * (p.H / p.G) + (on ? job / slices : 0), p0 = on ? (job % slices) * PS : 0, np = p.P - p0 < PS ? p.P - p0 : PS;
  const int size = p.P * p.N;
  const float A = p.a[h], D = p.d ? p.d[h] : 0.0f, bias_dt = p.dt_bias ? p.dt_bias[h] : 0.0f;

  // Channels of the convolution as the LDS has them: B, C (NP each, zeros behind N), x of the waves (PS each, zeros behind P): their
  // weights, and the channel of xbc, -1 where there is none.
  if (p.N != NP || p.P % PS != 0 || jobs % nw != 0)
    for (int e = tid; e < (int)(chunk_lds<NT>(nw * PS, nw) / 4); e += nthr) reinterpret_cast<uint32_t *>(smem)[e] = 0;
  __syncthreads();
  auto weights = [&](int k, int c) {
    chans[k] = c;
    if (c < 0) return;
    for (int i = 0; i < p.W; ++i) wl[4 * k + 4 - p.W + i] = p.conv_w[(int64_t)c * p.W + i] * -LOG2E;
    bl[k] = p.conv_b ? p.conv_b[c] * -LOG2E : 0.0f;
  };
  for (int k = tid; k < 2 * NP; k += nthr) {
    const int n = k < NP ? k : k - NP;
    weights(k, n < p.N ? p.H * p.P + (k < NP ? 0 : p.G * p.N) + g * p.N + n : -1);
  }
  if (lane < PS) weights(2 * NP + wave * PS + lane, on && lane < np ? h * p.P + p0 + lane : -1);
  __syncthreads();
  // A thread's work per chunk: pieces of four channels, TB tokens of B or C or eight tokens of x.
  constexpr int NB = (LOCAL ? NP : 2 * NP) / 4 * (Q / TB);
  const int NX = nw * PS;
  auto put_bc = [&](int item, const uint2 (&raw)[TB + 3]) {
    const int k0 = 4 * (item / (Q / TB)), tg = item % (Q / TB), isC = k0 >= NP, n0 = isC ? k0 - NP : k0;
    float back[4];
    // (two channels at a time, one pair after the other: all four would take too many registers)
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
      __builtin_amdgcn_sched_barrier(0);
      float v[2][TB];
      convolve<TB, FOUR>(raw, k, p.W, wl + 4 * k0, bl + k0, v[0]);
      convolve<TB, FOUR>(raw, k + 1, p.W, wl + 4 * k0, bl + k0, v[1]);
      if (!LOCAL) {
        uint16_t *to = (isC ? Cs : Bs) + TB * tg * NS + n0 + k;
#pragma unroll
        for (int t = 0; t < TB; ++t) {
          const uint32_t hi = pack2(v[0][t], v[1][t]);
          *reinterpret_cast<uint32_t *>(to + t * NS) = hi;
          if (isC) *reinterpret_cast<uint32_t *>(to + Q * NS + t * NS) = rest_b(v[0][t], v[1][t], hi);
        }
      }
      if (isC) continue;
#pragma unroll
      for (int o = 0; o < 2; ++o) {
        const float f = scale_to_f16(top_of_32<TB>(v[o]));
        back[k + o] = power_reciprocal(f);
        uint32_t hi[TB / 2], lo[TB / 2];
#pragma unroll
        for (int t = 0; t < TB / 2; ++t) {
          const float a = v[o][2 * t] * f, b = v[o][2 * t + 1] * f;
          hi[t] = pack_h(a, b);
          lo[t] = rest_h(a, b, hi[t]);
        }
        uint16_t *th = BtH + bt_row(n0) + (k + o) * (Q + 8) + TB * tg, *tl = th + bt_size(NP);
        if constexpr (TB == 8) {
          *reinterpret_cast<uint4 *>(th) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4 *>(tl) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        } else {
          *reinterpret_cast<uint2 *>(th) = make_uint2(hi[0], hi[1]);
          *reinterpret_cast<uint2 *>(tl) = make_uint2(lo[0], lo[1]);
        }
      }
    }
    if (!isC && tg == 0) *reinterpret_cast<f32x4 *>(bscale + n0) = f32x4{back[0], back[1], back[2], back[3]};
  };
  auto put_x = [&](int item, const uint2 (&raw)[11]) {
    const int x0 = 4 * (item >> 2), tg = item & 3;
    float top[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k % 2 == 0) __builtin_amdgcn_sched_barrier(0);
      float v[8];
      convolve<8, FOUR>(raw, k, p.W, wl + 4 * (2 * NP + x0), bl + 2 * NP + x0, v);
      float *to = Xall + (x0 + k) * XS + 8 * tg;
      *reinterpret_cast<f32x4 *>(to) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4 *>(to + 4) = f32x4{v[4], v[5], v[6], v[7]};
      if (!LOCAL) top[k] = top_of_32<8>(v);
    }
    if (!LOCAL && tg == 0) *reinterpret_cast<f32x4 *>(xsall + x0) = f32x4{top[0], top[1], top[2], top[3]};
  };
  // The piece whose inputs are fetched a chunk ahead.  PT = 4: a piece of x for every thread, those of B and C are asked for at the
  // chunk's begin and taken behind x.  PT = 2: pieces of x from the last thread down, of B and C from the first one up.
  const int xitem = PT == 4 ? tid : tid - (nthr - NX < 0 ? 0 : nthr - NX);
  const bool is_x = xitem >= 0 && xitem < NX;
  const int bitem = PT == 4 || !is_x ? tid : NB;  // (with more pieces than threads the rest is taken in turns)
  const int chan = is_x ? chans[2 * NP + 4 * (xitem >> 2)] : PT == 2 && bitem < NB ? chans[4 * (bitem / (Q / TB))] : -1;
  const int chan_bc = PT == 4 && bitem < NB ? chans[4 * (bitem / (Q / TB))] : -1, tgx = is_x ? xitem & 3 : bitem % (Q / TB);
  const int more0 = PT == 4 ? tid + nthr : nthr - NX > 0 ? tid + nthr - NX : tid;  // first of the other pieces of B and C, and their distance

  // Inputs are fetched a chunk ahead, also from a part to the next one: the thread's first piece, and a wave's steps.
  struct Where { Span sp; Part part; bool live; };
  auto where = [&](int sx) {
    Where w = {{0, 0}, {0, 0, false}, false};
    if (sx >= parts) return w;
    const int s = sx / p.nseg, seg = sx - s * p.nseg;
    w.sp = span_of(p, s);
    w.part = part_of(p, w.sp.count, seg);
    w.live = LOCAL ? seg < p.nseg - 1 : seg == 0 || w.part.begin < w.part.end;
    return w;
  };
  uint2 raw[11];
  uint16_t dt_raw;
  // (one place that loads, without branches: the loads are to be under way while the chunk before is worked on)
  auto ahead = [&](const Where &w, int t0) {
    const int end = w.live ? (w.part.end - t0 < Q ? w.part.end : t0 + Q) : 0;
    fetch(rows_of(p.xbc, w.sp.first, p.ld_xbc, t0 >= 3 ? t0 - 3 : 0, end), t0 + 8 * tgx, 2 * chan, chan >= 0, raw);
    const Rows dm = rows_of(p.dt, w.sp.first, p.ld_dt, t0, end);
    dt_raw = __builtin_amdgcn_raw_buffer_load_b16(dm.rsrc, (int)((uint32_t)(lane & (Q - 1)) * dm.ld2 + 2 * h), 0, 0);
  };
  Where next = where(sx0);
  ahead(next, next.part.begin);

  for (int sx = sx0; sx < parts; sx += stride) {
  const Where here = next;
  next = where(sx + stride);
  if (!here.live || here.part.begin >= here.part.end) {
    ahead(next, next.part.begin);
    if (!here.live) continue;
  }
  const int s = sx / p.nseg;
  const Span sp = here.sp;
  const Part part = here.part;
  const int slot = slot_of(p.slots_in, p.has_in, p.n_in, s), slot_to = slot_of(p.slots_out, p.has_out, p.n_out, s);
  auto rows_in = [&](int t0) { return rows_of(p.xbc, sp.first, p.ld_xbc, t0 >= 3 ? t0 - 3 : 0, part.end - t0 < Q ? part.end : t0 + Q); };

  // a lane's numbers: n = 16 i + 4 q .. + 3 of row p0 + 16 j + r
  f32x4 S[NT][PT];
  float *const mine = p.nseg > 1 ? p.seg_state + ((int64_t)sx * p.H + h) * size + p0 * p.N : nullptr;
  float *const left = LOCAL ? mine : part.last && slot_to >= 0 ? p.ssm_out + ((int64_t)slot_to * p.H + h) * size + p0 * p.N : nullptr;
  const float *first = LOCAL ? nullptr : p.nseg > 1 ? mine : slot >= 0 ? p.ssm_in + ((int64_t)slot * p.H + h) * size + p0 * p.N : nullptr;
  const bool lost = !LOCAL && p.nseg == 1 && slot == -2;
  {
    const float fill = lost ? __uint_as_float(0x7fc00000u) : 0.0f;
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < PT; ++j) {
        S[i][j] = f32x4{fill, fill, fill, fill};
        if (first && on && 16 * j + r < np && 16 * i + 4 * q < p.N) {
          const f32v4 v = *reinterpret_cast<const f32v4 *>(first + (16 * j + r) * p.N + 16 * i + 4 * q);
          S[i][j] = f32x4{v.v[0], v.v[1], v.v[2], v.v[3]};
        }
      }
  }
  float log_decay = 0.0f;

  for (int t0 = part.begin; t0 < part.end; t0 += Q) {
    const int end = part.end - t0 < Q ? part.end : t0 + Q;
    uint2 raw_bc[TB + 3];
    if constexpr (PT == 4) fetch(rows_in(t0), t0 + TB * (bitem % (Q / TB)), 2 * chan_bc, chan_bc >= 0, raw_bc);
    __syncthreads();  // (the arrays are still read for the chunk before)
    if (chan >= 0) {
      if (t0 == 0 && tgx == 0) {
        int c = chan;
        asm volatile("" : "+v"(c));  // (addresses of a path taken once are not to be kept in registers)
        fetch_state(p, slot, c, raw);
      }
      if (is_x) {
        put_x(xitem, raw);
      } else {
        if constexpr (PT == 2) put_bc(bitem, raw);
      }
    }
    if constexpr (PT == 4) {
      if (chan_bc >= 0) {
        if (t0 == 0 && bitem % (Q / TB) == 0) {
          int c = chan_bc;
          asm volatile("" : "+v"(c));
          fetch_state(p, slot, c, raw_bc);
        }
        put_bc(bitem, raw_bc);
      }
    }
    int more = more0;
    asm volatile("" : "+v"(more));
    for (int item = more; item < NB; item += nthr) {
      const int c = chans[4 * (item / (Q / TB))];
      if (c < 0) continue;
      uint2 now[TB + 3];
      fetch(rows_in(t0), t0 + TB * (item % (Q / TB)), 2 * c, true, now);
      if (t0 == 0 && item % (Q / TB) == 0) fetch_state(p, slot, c, now);
      put_bc(item, now);
    }
    // (behind the convolution, whose inputs are waited for together with whatever was asked for before)
    uint2 zr[2][PT];
    if (!LOCAL && p.z && on) {
      const Rows zm = rows_of(p.z, sp.first, p.ld_z, t0, end);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < PT; ++j) zr[t][j] = load4(zm, t0 + 16 * t + r, 16 * j < np ? 2 * (h * p.P + p0 + 16 * j + 4 * q) : 0);
    }
    float last = 0.0f;
    if (on) {
      const int t = lane & (Q - 1);
      const float dt = t0 + t < end ? softplus(bf16_f32(dt_raw) + bias_dt) : 0.0f;
      // Decays over some tokens have these tokens' exponents summed, never a difference of longer sums: behind a large step that
      // would be all rounding.
      const float v = dt * A, up = sum_up_to(v), behind = sum_from(lanes_behind<1>(v));
      const float half = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(up), Q - 1));
      last = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(up), Q / 2 - 1)) + half;
      const float w = dt * __expf(t < Q / 2 ? behind + half : behind) * (LN2 * LN2);
      if (lane < Q) {
        dec[t] = v;
        upto[t] = up;
        rest[t] = behind;
        stp[t] = dt * -(LN2 * LN2 * LN2);  // (x, B and C are each to be multiplied by -ln 2)
        wgt[t] = w;
      }
      log_decay += last;
    }
    {
      const bool more = t0 + Q < part.end;
      const Where w = {{more ? sp.first : next.sp.first, 0}, {0, more ? part.end : next.part.end, false}, more || next.live};
      ahead(w, more ? t0 + Q : next.part.begin);
    }
    __syncthreads();
    if (!on) continue;
    // (from here on addresses are made again for every chunk: kept in registers over the loop they would displace the state)
    int own_lane = tid & 63;
    asm volatile("" : "+v"(own_lane));
    const int lane = own_lane, r = lane & 15, q = lane >> 4;

    // A number of x that is not finite would, times the zeros of the matrix of tokens, reach the outputs before its own.  It is taken as
    // zero here; behind the outputs those of its row, from its token on, are set to NaN, and it is put back for the state.
    const bool odd = !LOCAL && __any(lane < PS && !is_finite(xs[lane & (PS - 1)]));
    if (odd && lane < PS && !is_finite(xs[lane])) {
      int from = Q;
#pragma unroll 1
      for (int t = Q - 1; t >= 0; --t)
        if (!is_finite(X[lane * XS + t])) {
          X[lane * XS + t] = 0.0f;
          from = t;
        }
      xs[lane] = __uint_as_float(0x7fc00000u | (uint32_t)from);
    }
    if constexpr (!LOCAL) {
      f32x4 G[3];  // rows s, columns t: (0, 0), (0, 1), (1, 1)
#pragma unroll
      for (int k = 0; k < 3; ++k) G[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < KN; ++k) {
        const bf16x8 b0 = frag16(Bs + r * NS + 32 * k + 8 * q), b1 = frag16(Bs + (16 + r) * NS + 32 * k + 8 * q);
        const bf16x8 c0 = frag16(Cs + r * NS + 32 * k + 8 * q), c1 = frag16(Cs + (16 + r) * NS + 32 * k + 8 * q);
        G[0] = VF_MFMA_B(b0, c0, G[0]);
        G[1] = VF_MFMA_B(b0, c1, G[1]);
        G[2] = VF_MFMA_B(b1, c1, G[2]);
      }
      const f32x4 st0 = *reinterpret_cast<const f32x4 *>(stp + 4 * q), st1 = *reinterpret_cast<const f32x4 *>(stp + 16 + 4 * q);
      // the exponents behind token 4 q + i up to token r, of either half: of the lane's own four tokens those that lie there, and
      // the sum from token 4 q + 4 to r; zero for later tokens
      auto between = [&](const float *of, float (&e)[4]) {
        const f32x4 own = *reinterpret_cast<const f32x4 *>(of + 4 * q);
        e[3] = sum_up_to(r >= 4 * q + 4 ? of[r] : 0.0f);
#pragma unroll
        for (int i = 2; i >= 0; --i) e[i] = e[i + 1] + (4 * q + i + 1 <= r ? own[i + 1] : 0.0f);
      };
      float e00[4], e11[4];
      between(dec, e00);
      between(dec + 16, e11);
      const f32x4 rs = *reinterpret_cast<const f32x4 *>(rest + 4 * q);
      const float up0 = upto[r], up1 = upto[16 + r];
      const bool behind = t0 > part.begin || first || lost;  // (otherwise the state is zero)
      const float e0 = __expf(up0) * -LN2, e1 = __expf(upto[15] + up1) * -LN2;
      f32x4 m00, m01, m11;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = 4 * q + i;
        m00[i] = at <= r ? fmaf(G[0][i], __expf(e00[i]) * st0[i], at == r ? D * -LN2 : 0.0f) : 0.0f;
        m11[i] = at <= r ? fmaf(G[2][i], __expf(e11[i]) * st1[i], at == r ? D * -LN2 : 0.0f) : 0.0f;
        m01[i] = G[1][i] * __expf(rs[i] + up1) * st0[i];
      }
      const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
      const uint4 f0 = frag_of(m00, zero), f1 = frag_of(m01, m11), g0 = rest_of(m00, zero, f0), g1 = rest_of(m01, m11, f1);
      const Rows om = rows_of(p.out, sp.first, p.ld_out, t0, end);
      // 16 rows p after the other, so that only theirs are in registers
#pragma unroll
      for (int j = 0; j < PT; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        f32x4 y[2] = {zero, zero};  // rows p, columns t
        if (behind) {
#pragma unroll
          for (int k = 0; k < KN; ++k) {
            const bf16x8 c0 = as_b(frag_acc(Cs + r * NS + 32 * k, q)), c1 = as_b(frag_acc(Cs + (16 + r) * NS + 32 * k, q));
            const bf16x8 l0 = as_b(frag_acc(CsL + r * NS + 32 * k, q)), l1 = as_b(frag_acc(CsL + (16 + r) * NS + 32 * k, q));
            const uint4 f = frag_of(S[2 * k][j], S[2 * k + 1][j]), fl = rest_of(S[2 * k][j], S[2 * k + 1][j], f);
            y[0] = VF_MFMA_B(as_b(f), l0, y[0]);
            y[1] = VF_MFMA_B(as_b(f), l1, y[1]);
            y[0] = VF_MFMA_B(as_b(fl), c0, y[0]);
            y[1] = VF_MFMA_B(as_b(fl), c1, y[1]);
            y[0] = VF_MFMA_B(as_b(f), c0, y[0]);
            y[1] = VF_MFMA_B(as_b(f), c1, y[1]);
          }
          y[0] *= e0;
          y[1] *= e1;
        }
        const f32x4 xa = *reinterpret_cast<const f32x4 *>(X + (16 * j + r) * XS + 4 * q), xb = *reinterpret_cast<const f32x4 *>(X + (16 * j + r) * XS + 16 + 4 * q);
        const uint4 xh = frag_of(xa, xb), xl = rest_of(xa, xb, xh);
        y[0] = VF_MFMA_B(as_b(xl), as_b(f0), y[0]);
        y[1] = VF_MFMA_B(as_b(xl), as_b(f1), y[1]);
        y[0] = VF_MFMA_B(as_b(xh), as_b(g0), y[0]);
        y[1] = VF_MFMA_B(as_b(xh), as_b(g1), y[1]);
        y[0] = VF_MFMA_B(as_b(xh), as_b(f0), y[0]);
        y[1] = VF_MFMA_B(as_b(xh), as_b(f1), y[1]);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          f32x4 v = y[t];
          if (p.z) {
            const uint32_t z4[2] = {zr[t][j].x, zr[t][j].y};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] *= silu(__uint_as_float(i & 1 ? z4[i >> 1] & 0xffff0000u : z4[i >> 1] << 16));
          }
          if (16 * j < np) store4(om, t0 + 16 * t + r, 2 * (h * p.P + p0 + 16 * j + 4 * q), make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3])));
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }

    if (odd && lane < PS && !is_finite(xs[lane])) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      const int from = (int)(__float_as_uint(xs[lane]) & 63);
#pragma unroll 1
      for (int t = from; t < Q && t0 + t < end; ++t)
        reinterpret_cast<uint16_t *>(p.out)[(sp.first + t0 + t) * p.ld_out + h * p.P + p0 + lane] = 0x7fc0;
      if (from < Q) X[lane * XS + from] = __uint_as_float(0x7fc00000u);
    }

    // the state behind the chunk
    if (!LOCAL && t0 + Q >= part.end && !left) continue;
    uint4 vh[PT], vl[PT];
    float back[PT];
    const f32x4 w0 = *reinterpret_cast<const f32x4 *>(wgt + 4 * q), w1 = *reinterpret_cast<const f32x4 *>(wgt + 16 + 4 * q);
#pragma unroll
    for (int j = 0; j < PT; ++j) {
      // (The scale goes by the products, not by the largest x and weight: where a large step meets zeros these are far from all products.
      // Up to 2^126 where a row is zero, it comes last: times a weight it may be infinite.)
      f32x4 a = *reinterpret_cast<const f32x4 *>(X + (16 * j + r) * XS + 4 * q) * w0;
      f32x4 b = *reinterpret_cast<const f32x4 *>(X + (16 * j + r) * XS + 16 + 4 * q) * w1;
      const float f = scale_to_f16(__uint_as_float(max_rows(max_abs(max_abs(max_abs(max_abs(0, a[0], a[1]), a[2], a[3]), b[0], b[1]), b[2], b[3]))));
      back[j] = power_reciprocal(f);
      a *= f;
      b *= f;
      vh[j] = make_uint4(pack_h(a[0], a[1]), pack_h(a[2], a[3]), pack_h(b[0], b[1]), pack_h(b[2], b[3]));
      vl[j] = make_uint4(rest_h(a[0], a[1], vh[j].x), rest_h(a[2], a[3], vh[j].y), rest_h(b[0], b[1], vh[j].z), rest_h(b[2], b[3], vh[j].w));
    }
    const float el = __expf(last);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const f16x8 bh = as_h(frag_acc(BtH + bt_row(16 * i + r), q)), bl2 = as_h(frag_acc(BtL + bt_row(16 * i + r), q));
      const f32x4 sc = *reinterpret_cast<const f32x4 *>(bscale + 16 * i + 4 * q);
#pragma unroll
      for (int j = 0; j < PT; ++j) {
        f32x4 u = {0.0f, 0.0f, 0.0f, 0.0f};
        u = VF_MFMA_H(bl2, as_h(vh[j]), u);
        u = VF_MFMA_H(bh, as_h(vl[j]), u);
        u = VF_MFMA_H(bh, as_h(vh[j]), u);
#pragma unroll
        for (int k = 0; k < 4; ++k) S[i][j][k] = fmaf(S[i][j][k], el, u[k] * (sc[k] * back[j]));
      }
    }
  }

  if (left && on) {
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int j = 0; j < PT; ++j)
        if (16 * j + r < np && 16 * i + 4 * q < p.N) {
          f32v4 v;
#pragma unroll
          for (int k = 0; k < 4; ++k) v.v[k] = S[i][j][k];
          *reinterpret_cast<f32v4 *>(left + (16 * j + r) * p.N + 16 * i + 4 * q) = v;
        }
  }
  if (LOCAL) {
    if (on && lane == 0 && p0 == 0) p.seg_log[(int64_t)sx * p.H + h] = log_decay;
    continue;
  }
  if (!part.last || slot_to < 0 || p.conv_later || p.W == 1) continue;
  if (on)
    for (int k = lane; k < np; k += 64) conv_state<uint16_t>(p, sp, slot, slot_to, h * p.P + p0 + k);
  if (wg == g * per)
    for (int k = tid; k < 2 * p.N; k += nthr)
      conv_state<uint16_t>(p, sp, slot, slot_to, p.H * p.P + (k < p.N ? g * p.N + k : p.G * p.N + g * p.N + k - p.N));
  }
}

// (byte offsets within a chunk are 32 bits wide, and a launch takes less than 2^32 threads)
bool chunks_fit(const SsmArgs &p) {
  constexpr int64_t most = 1 << 24;
  if ((int64_t)p.H * ((p.P + 31) / 32) > (1 << 22)) return false;
  return p.P % 16 == 0 && p.N % 16 == 0 && p.W <= 4 && p.ld_xbc < most && p.ld_dt < most && p.ld_out < most && (!p.z || p.ld_z < most);
}

template <int NT, int PT, bool FOUR>
int launch_chunks_of(vf_ctx *c, SsmArgs &p, int64_t longest) {
  constexpr int PS = 16 * PT, NW = ROWS / PS;
  // workgroups of a group's heads, each with the same number of waves but for the last
  const int jobs = p.H / p.G * ((p.P + PS - 1) / PS), per = (jobs + NW - 1) / NW, nw = (jobs + per - 1) / per;
  const int64_t each = (int64_t)p.n_seq * per * p.G;
  const size_t smem = chunk_lds<NT>(nw * PS, nw);
  // workgroups that run at a time: two waves on a SIMD, and what the LDS holds
  const int64_t by_waves = 8 / nw, by_lds = (int64_t)(160 * 1024 / smem), at_once = 256 * (by_waves < by_lds ? by_waves : by_lds);
  // a segment costs its state's way to memory and back, about 256 tokens' time
  split(c, p, longest, each, at_once, Q, 256);
  if (smem > 65536) {
    VF_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void *>(k_ssm_chunks<NT, PT, false, FOUR>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    VF_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void *>(k_ssm_chunks<NT, PT, true, FOUR>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  }
  // many short parts: a workgroup takes several, so that its weights are fetched once for them, but there are eight times as many
  // workgroups as run at a time, for the sake of unequal parts
  const int64_t wgs = (int64_t)per * p.G, parts = (int64_t)p.n_seq * p.nseg, most = 8 * at_once / wgs > 1 ? 8 * at_once / wgs : 1;
  const unsigned blocks = (unsigned)((parts < most ? parts : most) * wgs);
  return run_parts(c, p, [&] {
    if (p.local) k_ssm_chunks<NT, PT, true, FOUR><<<blocks, 64 * nw, smem, c->stream>>>(p);
    else k_ssm_chunks<NT, PT, false, FOUR><<<blocks, 64 * nw, smem, c->stream>>>(p);
    VF_HIP(c, hipGetLastError());
    return VF_OK;
  });
}
template <int NT, int PT>
int launch_chunks(vf_ctx *c, SsmArgs &p, int64_t longest) {
  return p.W == 4 ? launch_chunks_of<NT, PT, true>(c, p, longest) : launch_chunks_of<NT, PT, false>(c, p, longest);
}
int chunks(vf_ctx *c, SsmArgs &p, int64_t longest) {
  // Four waves of 64 rows, two workgroups on a compute unit, where the state leaves registers for it; else eight waves of 32 rows.
  if (p.P > 32 && p.N <= 64) return p.N <= 32 ? launch_chunks<2, 4>(c, p, longest) : launch_chunks<4, 4>(c, p, longest);
  return p.N <= 32 ? launch_chunks<2, 2>(c, p, longest) : p.N <= 64 ? launch_chunks<4, 2>(c, p, longest)
       : p.N <= 128 ? launch_chunks<8, 2>(c, p, longest) : launch_chunks<16, 2>(c, p, longest);
}

bool overlap(const void *a, size_t na, const void *b, size_t nb) {
  const char *x = static_cast<const char *>(a), *y = static_cast<const char *>(b);
  return x && y && x < y + nb && y < x + na;
}

}  // namespace

int vfk_ssm(vf_ctx *c, const vf_ssm *l, const vf_ssm_io *io, bool one) {
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
  p.nseg = 1; p.seg_len = 0; p.local = 0; p.seg_state = p.seg_log = nullptr;
  const int64_t longest = io->offsets_dev ? (io->longest < io->tokens ? io->longest : io->tokens) : io->tokens / io->n_seq;
  int rc;
  if (one || (!io->offsets_dev && io->tokens == io->n_seq)) rc = io->type == VF_BF16 ? step<uint16_t>(c, p) : step<float>(c, p);
  else if (io->type == VF_BF16 && chunks_fit(p) && longest > 8) rc = chunks(c, p, longest);
  else rc = io->type == VF_BF16 ? tokens<uint16_t>(c, p, longest) : tokens<float>(c, p, longest);
  if (rc != VF_OK || !p.has_out || !p.conv_later || p.W == 1) return rc;
  const int grid = blocks_for((int64_t)p.n_seq * p.C);
  if (io->type == VF_BF16) k_ssm_conv_state<uint16_t><<<grid, 256, 0, c->stream>>>(p);
  else k_ssm_conv_state<float><<<grid, 256, 0, c->stream>>>(p);
  VF_HIP(c, hipGetLastError());
  return VF_OK;
}
