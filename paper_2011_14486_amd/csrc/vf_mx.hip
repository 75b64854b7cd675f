// Microscaled matrices: quantization, the values of the codes, and the product of 8- or 4-bit rows with 4-bit
// weights on the scaled matrix instructions.
#include "vf_internal.h"
#include "vf_ops_dev.h"

namespace {

using namespace vfo;

// ---- quantization: a thread holds eight columns, four neighbouring threads a block of 32 ----
// Every value is read once and every code written once: the memory's rate bounds it.
template <typename T, int FMT>
__global__ void __launch_bounds__(256) k_mx_quantize(const T *x, int64_t ld, int64_t rows, int cols, int kb, uint8_t *codes,
                                                     uint8_t *scales) {
  const int nchunk = 4 * kb;
  const int64_t total = rows * nchunk;  // a multiple of four: a block's four threads are all in or all out
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / nchunk;
    const int c = (int)(i - row * nchunk), n = cols - 8 * c;
    float v[8];
    if (n > 0) {
      load_upto8(x + row * ld + 8 * c, n, v);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 0.0f;
    }
    quantize_chunk<FMT>(v, c, true, codes + row * kb * mx<FMT>::bytes32, scales + row * kb);
  }
}

template <int FMT>
__device__ __forceinline__ void decode8(const uint8_t *codes_row, int c, float (&v)[8]) {
  if constexpr (FMT == VF_E4M3) {
    const uint2 q = reinterpret_cast<const uint2 *>(codes_row)[c];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int w = (int)(i ? q.y : q.x);
      const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
      v[4 * i] = a[0]; v[4 * i + 1] = a[1]; v[4 * i + 2] = b[0]; v[4 * i + 3] = b[1];
    }
  } else {
    const uint32_t q = reinterpret_cast<const uint32_t *>(codes_row)[c];
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1);
    const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1]; v[4] = d[0]; v[5] = d[1]; v[6] = e[0]; v[7] = e[1];
  }
}

template <int FMT, typename T>
__global__ void __launch_bounds__(256) k_mx_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int cols, int kb,
                                                       T *out, int64_t ld) {
  const int nchunk = (cols + 7) >> 3;
  const int64_t total = rows * nchunk;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / nchunk;
    const int c = (int)(i - row * nchunk);
    float v[8];
    decode8<FMT>(codes + row * kb * mx<FMT>::bytes32, c, v);
    const int b = scales[row * kb + (c >> 2)];
    // 2^(b - 127): byte 0 is the subnormal number 2^-127, byte 255 a NaN
    const float s = b == 0 ? __uint_as_float(0x00400000u) : b == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)b << 23);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= s;
    store_upto8(out + row * ld + 8 * c, cols - 8 * c, v);
  }
}

// ---- the product ----
// The scaled matrix instruction 16x16x128 takes, per lane (r = lane % 16, g = lane / 16): of a 4-bit operand the
// block of 32 k at 32 g of row r (16 bytes); of an 8-bit operand the 16 k at 16 g and the 16 at 64 + 16 g of row r;
// of either operand's scales the byte of row r, block g.  The weights are the first operand and the rows of
// a the second: a lane then holds four neighbouring columns of out.

struct MatmulArgs {
  const uint8_t *a, *as, *w, *ws;
  const float *bias;
  void *out;
  int64_t M, ld_out;
  int N, kb;
  int out_bf16;
};

// the 16 or 32 bytes of a row for k-step `s` (four blocks), zeros where blocks are missing
template <int FMT>
__device__ __forceinline__ i32x8 fragment(const uint8_t *row, int s, int g, int kb) {
  i32x8 f = {0, 0, 0, 0, 0, 0, 0, 0};
  if constexpr (FMT == VF_E2M1) {
    const int b = 4 * s + g;
    if (b < kb) {
      const uint4 q = *reinterpret_cast<const uint4 *>(row + 16 * (int64_t)b);
      f[0] = (int)q.x; f[1] = (int)q.y; f[2] = (int)q.z; f[3] = (int)q.w;
    }
  } else {
    const int b0 = 4 * s + (g >> 1), b1 = b0 + 2;
    if (b0 < kb) {
      const uint4 q = *reinterpret_cast<const uint4 *>(row + 32 * (int64_t)b0 + 16 * (g & 1));
      f[0] = (int)q.x; f[1] = (int)q.y; f[2] = (int)q.z; f[3] = (int)q.w;
    }
    if (b1 < kb) {
      const uint4 q = *reinterpret_cast<const uint4 *>(row + 32 * (int64_t)b1 + 16 * (g & 1));
      f[4] = (int)q.x; f[5] = (int)q.y; f[6] = (int)q.z; f[7] = (int)q.w;
    }
  }
  return f;
}

// The instruction adds the terms of eight neighbouring k with what lies more than 13 binary places below the largest
// of them cut off, and everything else in fp32 (found by feeding it pairs of powers of two).  4-bit by 4-bit terms
// span 8 places and lose nothing.  Terms of 8-bit rows span 22: with outputs in bf16 the cut, 2^-13 of the largest of
// eight terms at most (1e-4 of an output on normal data), is far below the output's own rounding and stays; with
// outputs in fp32 (EXACT) the row is taken in two parts, the numbers of 2 and more and those below: the
// terms' last place is then 2^-3 under a largest of 2^10, and 2^-10 under a largest of 2^2: nothing is cut.
// (Format codes of the instruction: 0 for E4M3, 4 for E2M1.)
template <int AF, bool EXACT>
__device__ __forceinline__ f32x4 mfma128(const i32x8 &w, const i32x8 &a, f32x4 c, int ws, int as) {
  if constexpr (AF == VF_E4M3 && EXACT) {
    i32x8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // numbers of 2 and more have the highest exponent bit
      const uint32_t m = (((uint32_t)a[i] >> 6) & 0x01010101u) * 255u;
      hi[i] = (int)((uint32_t)a[i] & m);
      lo[i] = (int)((uint32_t)a[i] & ~m);
    }
    c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, lo, c, 4, 0, 0, ws, 0, as);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, hi, c, 4, 0, 0, ws, 0, as);
  } else {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, a, c, 4, AF == VF_E4M3 ? 0 : 4, 0, ws, 0, as);
  }
}

__device__ __forceinline__ void store4(const MatmulArgs &p, int64_t m, int n, const f32x4 &v) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = v[i] + (p.bias && n + i < p.N ? p.bias[n + i] : 0.0f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (n + i >= p.N) break;
    if (p.out_bf16) reinterpret_cast<uint16_t *>(p.out)[m * p.ld_out + n + i] = round_bf16(y[i]);
    else reinterpret_cast<float *>(p.out)[m * p.ld_out + n + i] = y[i];
  }
}

// Few rows: a workgroup makes 16 columns of 16 MT rows, its four waves take the k-steps in turn and join their sums
// in the LDS.  The operands come straight from memory, each weight once.
template <int AF, bool EXACT, int MT>
__global__ void __launch_bounds__(256) k_mx_rows(const MatmulArgs p) {
  __shared__ f32x4 join[3][MT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int n0 = (int)blockIdx.x * 16;
  const int64_t m0 = (int64_t)blockIdx.y * (16 * MT);
  const int nr = n0 + r < p.N ? n0 + r : p.N - 1;
  const uint8_t *wrow = p.w + (int64_t)nr * p.kb * 16, *wsrow = p.ws + (int64_t)nr * p.kb;
  f32x4 acc[MT];
  const uint8_t *arow[MT], *asrow[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t m = m0 + 16 * t + r < p.M ? m0 + 16 * t + r : p.M - 1;
    arow[t] = p.a + m * p.kb * mx<AF>::bytes32;
    asrow[t] = p.as + m * p.kb;
  }
  const int steps = (p.kb + 3) >> 2;
  for (int s = wave; s < steps; s += 4) {
    const int b = 4 * s + g;
    const i32x8 w = fragment<VF_E2M1>(wrow, s, g, p.kb);
    const int wsc = b < p.kb ? wsrow[b] : 127;
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const i32x8 a = fragment<AF>(arow[t], s, g, p.kb);
      const int asc = b < p.kb ? asrow[t][b] : 127;
      acc[t] = mfma128<AF, EXACT>(w, a, acc[t], wsc, asc);
    }
  }
  // (the compiler may move this instruction into a branch, where lanes that are off would not set its operands)
#pragma unroll
  for (int t = 0; t < MT; ++t) asm volatile("" : "+v"(acc[t]));
  if (wave > 0) {
#pragma unroll
    for (int t = 0; t < MT; ++t) join[wave - 1][t][lane] = acc[t];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int t = 0; t < MT; ++t) {
#pragma unroll
    for (int w = 0; w < 3; ++w) acc[t] += join[w][t][lane];
    const int64_t m = m0 + 16 * t + r;
    if (m < p.M) store4(p, m, n0 + 4 * g, acc[t]);
  }
}

// Many rows: tiles of 64 MI rows by 256 columns in the LDS, eight waves of 16 MI rows by 128 columns of accumulators.
//
// A stage of the k loop is 128 k.  Its bytes go from memory straight to the LDS, in pieces of 16 bytes; where a piece lies is
// chosen by which lane fetches it: piece c of row m at place c ^ (m % 8) of eight, or c ^ (m / 4 % 4) of four, so that the 16 rows that
// lanes read at a time meet all banks.  The weights are the first operand, with the columns dealt to the operand's 16
// rows in such an order that a lane ends up with 32 neighbouring columns of a row of the output.
//
// The weights' operands are read two tiles ahead, across the end of a stage too.  The only barrier is in a stage's middle: behind it
// the next stage's bytes are there for everybody, and nobody reads the stage before any more, whose place the
// newest fetch takes.  Of the two waves of a SIMD one has priority, so that they do not reach the reads of a's operands, at a
// stage's begin, together.
template <int AF> constexpr int a_bytes() { return AF == VF_E4M3 ? 128 : 64; }   // of a row, in a stage
template <int AF> constexpr int stages() { return AF == VF_E4M3 ? 3 : 4; }       // that the LDS holds
// (S4: scales four to a word; else each in a word of its own)
template <int AF, int MI, bool S4> constexpr int stage_bytes() { return 64 * MI * a_bytes<AF>() + 256 * 64 + (64 * MI + 256) * (S4 ? 4 : 16); }

// 64 lanes fetch 16 bytes (or one byte, into a word) each from addresses of their own to consecutive places of the LDS from `to` on.
// The compiler does not know of these loads: they are waited for by wait_loads.
__device__ __forceinline__ void to_lds16(const uint8_t *from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}
__device__ __forceinline__ void to_lds1(const uint8_t *from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, off" ::"s"(to), "v"(from) : "memory");
}
__device__ __forceinline__ void to_lds4(const uint8_t *from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "memory");
}
// (accesses of the LDS are not moved across it)
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

template <int AF, bool EXACT, int MI, bool S4>
__global__ void __launch_bounds__(512, 2) k_mx_tile(const MatmulArgs p, int tiles_n, int tiles) {
  extern __shared__ __align__(16) uint8_t lds[];
  constexpr int BM = 64 * MI, AB = a_bytes<AF>(), NT = 8, NST = stages<AF>(), SB = stage_bytes<AF, MI, S4>();
  constexpr int WAT = BM * AB, SAT = WAT + 256 * 64;  // the weights and the scales in a stage
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4, wm = wave & 3, wn = wave >> 2;
  // Workgroups are dealt to the eight dies in turn: each die gets neighbouring tiles, in blocks of eight rows of tiles that pass over
  // the columns, so that its cache keeps what they share.
  int id = blockIdx.x;
  const int chunk8 = tiles / 8;
  if (id < chunk8 * 8) id = (id & 7) * chunk8 + (id >> 3);
  const int tiles_m = tiles / tiles_n, band = id / (8 * tiles_n), in_band = id - band * 8 * tiles_n;
  const int high = tiles_m - 8 * band < 8 ? tiles_m - 8 * band : 8, mt = 8 * band + in_band % high;
  const int64_t m0 = (int64_t)mt * BM;
  const int n0 = in_band / high * 256;
  const int steps = (p.kb + 3) >> 2;

  // Pieces that this thread fetches in every stage: their sources at block 0 of the row, and their block within the stage
  constexpr int PA = BM * (AB / 16) / 512, PW = 2, PS = ((BM + 256) * (S4 ? 1 : 4) + 511) / 512;
  const uint8_t *src_a[PA], *src_w[PW], *src_s[PS];
  int blk_a[PA], blk_w[PW], blk_s[PS];
  auto row_a = [&](int row) { return m0 + row < p.M ? m0 + row : p.M - 1; };
  // row 16 j + x of a wave's 128 rows of weights is its column 32 (x / 4) + 4 j + x % 4
  auto col_w = [&](int row) {
    const int col = n0 + (row & 128) + 32 * ((row & 15) >> 2) + 4 * ((row & 127) >> 4) + (row & 3);
    return col < p.N ? col : p.N - 1;
  };
#pragma unroll
  for (int i = 0; i < PA; ++i) {
    const int e = i * 512 + tid, row = e / (AB / 16), c = AB == 128 ? (e & 7) ^ (row & 7) : (e & 3) ^ ((row >> 2) & 3);
    src_a[i] = p.a + row_a(row) * p.kb * mx<AF>::bytes32 + (AF == VF_E4M3 ? 16 * (c & 1) : 0);
    blk_a[i] = AF == VF_E4M3 ? c >> 1 : c;
  }
#pragma unroll
  for (int i = 0; i < PW; ++i) {
    const int e = i * 512 + tid, row = e >> 2;
    src_w[i] = p.w + (int64_t)col_w(row) * p.kb * 16;
    blk_w[i] = (e & 3) ^ ((row >> 2) & 3);
  }
#pragma unroll
  for (int i = 0; i < PS; ++i) {
    const int e = i * 512 + tid, row = S4 ? e : e >> 2;
    blk_s[i] = S4 ? 0 : e & 3;
    src_s[i] = row < BM ? p.as + row_a(row) * p.kb : p.ws + (int64_t)col_w(row - BM) * p.kb;
  }
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
  const uint32_t wave_at = __builtin_amdgcn_readfirstlane(wave);
  // (blocks behind the row's end: the row's last block, which is there; its k of a are then cleared)
  auto fetch = [&](int st) {
    const uint32_t at = base + (uint32_t)(st % NST) * SB;
    const int b0 = 4 * (st < steps ? st : steps - 1);
    const bool whole = b0 + 4 <= p.kb;
    auto block = [&](int b) { return whole || b0 + b < p.kb ? b0 + b : p.kb - 1; };
#pragma unroll
    for (int i = 0; i < PA; ++i) to_lds16(src_a[i] + (int64_t)block(blk_a[i]) * mx<AF>::bytes32, at + (i * 512 + wave_at * 64) * 16);
#pragma unroll
    for (int i = 0; i < PW; ++i) to_lds16(src_w[i] + (int64_t)block(blk_w[i]) * 16, at + WAT + (i * 512 + wave_at * 64) * 16);
#pragma unroll
    for (int i = 0; i < PS; ++i) {
      const uint32_t to = at + SAT + (i * 512 + wave_at * 64) * 4;
      if (S4) to_lds4(src_s[i] + b0, to);  // (rows of scales are whole words then)
      else to_lds1(src_s[i] + block(blk_s[i]), to);
    }
  };
  constexpr int LOADS = PA + PW + PS;

  f32x4 acc[NT][MI];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MI; ++i) acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  uint4 ar[MI][AB / 64], wq[4];
  int as[MI], ws[4];
  // places of this lane's pieces in a stage: of row 16 i + r they lie a constant further for every i
  constexpr int SW = S4 ? 4 : 16;  // a row's scales
  const int sw_a = AB == 128 ? r & 7 : (r >> 2) & 3;
  const int la0 = (wm * 16 * MI + r) * AB + 16 * (g ^ sw_a), la1 = (wm * 16 * MI + r) * AB + 16 * ((4 + g) ^ sw_a);
  const int lw = WAT + (wn * 128 + r) * 64 + 16 * (g ^ ((r >> 2) & 3));
  const int lsa = SAT + (wm * 16 * MI + r) * SW + g * (SW / 4), lsw = SAT + (BM + wn * 128 + r) * SW + g * (SW / 4);
  auto read_a = [&](int st) {
    // (16 k at 16 g and, of 8-bit rows, 16 at 64 + 16 g)
    const uint8_t *at = lds + (st % NST) * SB;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      ar[i][0] = *reinterpret_cast<const uint4 *>(at + la0 + i * 16 * AB);
      if (AF == VF_E4M3) ar[i][AB / 64 - 1] = *reinterpret_cast<const uint4 *>(at + la1 + i * 16 * AB);
      as[i] = at[lsa + i * 16 * SW];
    }
  };
  auto read_w = [&](int st, int j) {
    const uint8_t *at = lds + (st % NST) * SB;
    wq[j & 3] = *reinterpret_cast<const uint4 *>(at + lw + j * 16 * 64);
    ws[j & 3] = at[lsw + j * 16 * SW];
  };
  auto products = [&](int j) {
    __builtin_amdgcn_sched_barrier(0);
    const uint4 q = wq[j & 3];
    const i32x8 fw = {(int)q.x, (int)q.y, (int)q.z, (int)q.w, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const uint4 u = ar[i][0], v = ar[i][AB / 64 - 1];
      const i32x8 fa = AF == VF_E4M3 ? i32x8{(int)u.x, (int)u.y, (int)u.z, (int)u.w, (int)v.x, (int)v.y, (int)v.z, (int)v.w}
                                     : i32x8{(int)u.x, (int)u.y, (int)u.z, (int)u.w, 0, 0, 0, 0};
      acc[j][i] = mfma128<AF, EXACT>(fw, fa, acc[j][i], ws[j & 3], as[i]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
#pragma unroll
  for (int st = 0; st < NST - 1; ++st) fetch(st);
  wait_loads<0>();
  meet();
  if (wave < 4) __builtin_amdgcn_s_setprio(1);
  read_w(0, 0);
  read_w(0, 1);
  // (no branches in this loop: the compiler would move the products past them, behind all reads.  Stages behind the last
  // one are the last one's bytes again, in places that nobody reads.)
  for (int st = 0; st < steps - 1; ++st) {
    read_a(st);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      if (j == NT / 2) {
        wait_loads<NST == 3 ? 0 : LOADS>();  // (of four stages the newest may still be under way)
        meet();
        fetch(st + NST - 1);
      }
      if (j + 2 < NT) read_w(st, j + 2);
      else read_w(st + 1, j + 2 - NT);
      products(j);
    }
  }
  read_a(steps - 1);
  if (p.kb % 4 != 0) {  // k behind the row's end
    const int b0 = 4 * (steps - 1);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      if (b0 + (AF == VF_E4M3 ? g >> 1 : g) >= p.kb) ar[i][0] = make_uint4(0, 0, 0, 0);
      if (AF == VF_E4M3 && b0 + 2 + (g >> 1) >= p.kb) ar[i][AB / 64 - 1] = make_uint4(0, 0, 0, 0);
    }
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    if (j + 2 < NT) read_w(steps - 1, j + 2);
    products(j);
  }
  __builtin_amdgcn_s_setprio(0);
  wait_loads<0>();
  // a lane has columns n .. n + 31 of rows r, 16 + r, ...
  const int n = n0 + wn * 128 + 32 * g;
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int i = 0; i < MI; ++i) asm volatile("" : "+v"(acc[j][i]));
#pragma unroll
  for (int j = 0; j < NT; j += 2) {
    float b[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) b[k] = p.bias && n + 4 * j + k < p.N ? p.bias[n + 4 * j + k] : 0.0f;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const int64_t m = m0 + wm * 16 * MI + 16 * i + r;
      if (m >= p.M || n + 4 * j >= p.N) continue;
      float y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = acc[j + (k >> 2)][i][k & 3] + b[k];
      if (p.out_bf16) store_upto8(reinterpret_cast<uint16_t *>(p.out) + m * p.ld_out + n + 4 * j, p.N - n - 4 * j, y);
      else store_upto8(reinterpret_cast<float *>(p.out) + m * p.ld_out + n + 4 * j, p.N - n - 4 * j, y);
    }
  }
}

inline int blocks_for(int64_t threads) {
  const int64_t g = (threads + 255) / 256;
  return (int)(g < (1 << 20) ? g : (1 << 20));
}

template <int AF, bool EXACT, int MI, bool S4>
int launch_tile(vf_ctx *c, const MatmulArgs &p) {
  constexpr int smem = stages<AF>() * stage_bytes<AF, MI, S4>(), BM = 64 * MI;
  const int tiles_n = (p.N + 255) / 256;
  // (less than 2^22 workgroups in a launch; the rows are taken in several)
  const int64_t most = ((int64_t)1 << 22) / tiles_n, per = (most > 1 ? most : 1) * BM;
  VF_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void *>(k_mx_tile<AF, EXACT, MI, S4>), hipFuncAttributeMaxDynamicSharedMemorySize, smem));
  for (int64_t m = 0; m < p.M; m += per) {
    MatmulArgs q = p;
    q.a += m * p.kb * mx<AF>::bytes32;
    q.as += m * p.kb;
    q.M = p.M - m < per ? p.M - m : per;
    q.out = static_cast<char *>(p.out) + m * p.ld_out * (p.out_bf16 ? 2 : 4);
    const int tiles = (int)((q.M + BM - 1) / BM) * tiles_n;
    k_mx_tile<AF, EXACT, MI, S4><<<tiles, 512, smem, c->stream>>>(q, tiles_n, tiles);
    VF_HIP(c, hipGetLastError());
  }
  return VF_OK;
}

bool aligned4(const void *p) { return (uintptr_t)p % 4 == 0; }

template <int AF, bool EXACT>
int matmul(vf_ctx *c, const MatmulArgs &p) {
  const int64_t big = ((p.M + 255) / 256) * ((p.N + 255) / 256);
  if (p.M > 64 && big >= 64) {
    // (rows of scales that begin at whole words travel four at a time)
    if (p.kb % 4 == 0 && aligned4(p.as) && aligned4(p.ws)) return launch_tile<AF, EXACT, 4, true>(c, p);
    return launch_tile<AF, EXACT, 2, false>(c, p);
  }
  const int nb = (p.N + 15) / 16;
  const int MT = p.M <= 16 ? 1 : p.M <= 32 ? 2 : 4;
  // rows beyond the grid's second dimension are taken in further launches
  const int64_t per = (int64_t)65535 * 16 * MT;
  for (int64_t m = 0; m < p.M; m += per) {
    MatmulArgs q = p;
    q.a += m * p.kb * mx<AF>::bytes32;
    q.as += m * p.kb;
    q.M = p.M - m < per ? p.M - m : per;
    q.out = static_cast<char *>(p.out) + m * p.ld_out * (p.out_bf16 ? 2 : 4);
    const dim3 grid(nb, (unsigned)((q.M + 16 * MT - 1) / (16 * MT)));
    if (MT == 1) k_mx_rows<AF, EXACT, 1><<<grid, 256, 0, c->stream>>>(q);
    else if (MT == 2) k_mx_rows<AF, EXACT, 2><<<grid, 256, 0, c->stream>>>(q);
    else k_mx_rows<AF, EXACT, 4><<<grid, 256, 0, c->stream>>>(q);
    VF_HIP(c, hipGetLastError());
  }
  return VF_OK;
}

}  // namespace

int vfk_mx_quantize(vf_ctx *c, int type, const void *x, int64_t ld, int64_t rows, int cols, int format, uint8_t *codes,
                    uint8_t *scales) {
  if (rows == 0) return VF_OK;
  const int kb = (cols + 31) / 32, grid = blocks_for(rows * 4 * kb);
  const uint16_t *h = static_cast<const uint16_t *>(x);
  const float *f = static_cast<const float *>(x);
  if (type == VF_BF16 && format == VF_E4M3) k_mx_quantize<uint16_t, VF_E4M3><<<grid, 256, 0, c->stream>>>(h, ld, rows, cols, kb, codes, scales);
  else if (type == VF_BF16) k_mx_quantize<uint16_t, VF_E2M1><<<grid, 256, 0, c->stream>>>(h, ld, rows, cols, kb, codes, scales);
  else if (format == VF_E4M3) k_mx_quantize<float, VF_E4M3><<<grid, 256, 0, c->stream>>>(f, ld, rows, cols, kb, codes, scales);
  else k_mx_quantize<float, VF_E2M1><<<grid, 256, 0, c->stream>>>(f, ld, rows, cols, kb, codes, scales);
  VF_HIP(c, hipGetLastError());
  return VF_OK;
}

int vfk_mx_dequantize(vf_ctx *c, int format, const uint8_t *codes, const uint8_t *scales, int64_t rows, int cols, int type,
                      void *out, int64_t ld) {
  if (rows == 0) return VF_OK;
  const int kb = (cols + 31) / 32, grid = blocks_for(rows * ((cols + 7) / 8));
  uint16_t *h = static_cast<uint16_t *>(out);
  float *f = static_cast<float *>(out);
  if (type == VF_BF16 && format == VF_E4M3) k_mx_dequantize<VF_E4M3, uint16_t><<<grid, 256, 0, c->stream>>>(codes, scales, rows, cols, kb, h, ld);
  else if (type == VF_BF16) k_mx_dequantize<VF_E2M1, uint16_t><<<grid, 256, 0, c->stream>>>(codes, scales, rows, cols, kb, h, ld);
  else if (format == VF_E4M3) k_mx_dequantize<VF_E4M3, float><<<grid, 256, 0, c->stream>>>(codes, scales, rows, cols, kb, f, ld);
  else k_mx_dequantize<VF_E2M1, float><<<grid, 256, 0, c->stream>>>(codes, scales, rows, cols, kb, f, ld);
  VF_HIP(c, hipGetLastError());
  return VF_OK;
}

int vfk_mx_matmul(vf_ctx *c, int a_format, const uint8_t *a, const uint8_t *as, const uint8_t *w, const uint8_t *ws, int64_t M,
                  int N, int K, const float *bias, int out_type, void *out, int64_t ld_out) {
  if (M == 0 || N == 0) return VF_OK;
  MatmulArgs p;
  p.a = a; p.as = as; p.w = w; p.ws = ws; p.bias = bias; p.out = out;
  p.M = M; p.ld_out = ld_out; p.N = N; p.kb = (K + 31) / 32; p.out_bf16 = out_type == VF_BF16;
  if (a_format == VF_E2M1) return matmul<VF_E2M1, false>(c, p);
  return p.out_bf16 ? matmul<VF_E4M3, false>(c, p) : matmul<VF_E4M3, true>(c, p);
}
