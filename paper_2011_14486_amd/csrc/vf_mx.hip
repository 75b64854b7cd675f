// Microscaled matrices: quantization, the values of the codes, and the product of 8- or 4-bit rows with 4-bit
// weights on the scaled matrix instructions.
#include "vf_internal.h"
#include "vf_ops_dev.h"

namespace {

using namespace vfo;

// ---- quantization: a thread holds eight columns, four neighbouring threads a block of 32 ----
// Every value is read once and every code written once: the memory's rate bounds it.  MI355X: 8192 x 4096 from bf16 to 4 bits 19 us, 85 MB
// (4.5 TB/s), back 15 us.
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
// in the LDS.  The operands come straight from memory, each weight once.  MI355X: 4 x 4384 x 1024 4.2 us, which is the latency of
// four waves' passes over k; 20 x 8192 x 4096 13.8 us (1.3 TB/s of weights).
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

// Many rows: tiles of 256 rows by 256 columns in the LDS, eight waves of 64 rows by 128 columns of accumulators; where these would leave
// compute units idle, tiles of 128 by 128, four waves of 64 by 64, two workgroups on a compute unit.
//
// A stage of the k loop is 128 k.  Its bytes go from memory straight to the LDS, in pieces of 16 bytes; where a piece lies is
// chosen by which lane fetches it: piece c of row m at place c ^ (m % 8) of eight, or c ^ (m / 4 % 4) of four, so that the 16 rows that
// lanes read at a time meet all banks.  The weights are the first operand, with the columns dealt to the operand's 16
// rows in such an order that of a row of the output a lane ends up with eight neighbouring columns of every 32, and four
// lanes together with all 32 of them: a store instruction writes 64 bytes of 16 rows.
//
// The weights' operands are read two tiles ahead, across the end of a stage too.  The only barrier is in a stage's middle: behind it
// the next stage's bytes are there for everybody, and nobody reads the stage before any more, whose place the
// newest fetch takes.  Of the two waves of a SIMD one has priority, so that they do not reach the reads of a's operands, at a
// stage's begin, together.
//
// What bounds it besides the matrix cores is the number of requests to the second-level cache.  So scales, four bytes a row and
// stage, are taken 16 bytes at a time, four stages' worth, through a register: a request per row and stage for them would be half of all
// requests.  A workgroup goes on to its next tile by itself: that tile's first stages are on their way while the results of
// the last one are stored.
// MI355X: 16384 x 8192 x 4096 with 8-bit rows 455 us = 2.4 PFLOP/s (the vendor library's product of 8-bit by 8-bit numbers 2.65 at 8192^3;
// 0.74 ms with a barrier at a stage's end and scales fetched every stage), 5000 x 4384 x 4096 in 4 bits 78 - 87 us.
// The matrix cores are busy 53 % of the cycles there, and 26 % in 4 bits, where an instruction takes half the time.
template <int AF> constexpr int a_bytes() { return AF == VF_E4M3 ? 128 : 64; }   // of a row, in a stage
template <int AF> constexpr int stages() { return AF == VF_E4M3 ? 3 : 4; }       // that the LDS holds
// WM by WN waves of 64 rows by 16 NT columns: a thread for every row and column of the tile
template <int WM_, int WN_, int NT_> struct Tile {
  static constexpr int WM = WM_, WN = WN_, NT = NT_, M = 64 * WM, N = 16 * NT * WN, THREADS = 64 * WM * WN;
  static constexpr int SCALES = THREADS * 16;  // bytes of four stages' scales; the LDS holds them twice
  static_assert(M + N == THREADS, "");
};
typedef Tile<4, 2, 8> Large;
typedef Tile<2, 2, 4> Small;
template <int AF, class TL> constexpr int stage_bytes() { return TL::M * a_bytes<AF>() + TL::N * 64; }

// A part of memory as the instructions with a range check see it: what lies behind its end reads as zeros.
typedef int i32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ i32x4 part_of(const uint8_t *at, int64_t bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)at;
  const int64_t n = bytes < 0xfffffff0ll ? bytes : 0xfffffff0ll;
  return i32x4{__builtin_amdgcn_readfirstlane((int)a), __builtin_amdgcn_readfirstlane((int)(a >> 32) & 0xffff),
               __builtin_amdgcn_readfirstlane((int)(uint32_t)n), 0x00027000};
}
// 64 lanes fetch 16 bytes each, `lane_at` + `at` into the part, to consecutive places of the LDS from `to` on.
// The compiler does not know of these loads: they are waited for by wait_loads.
__device__ __forceinline__ void to_lds16(const i32x4 &part, uint32_t lane_at, uint32_t at, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(lane_at), "s"(part), "s"(at) : "memory");
}
// (accesses of the LDS are not moved across it)
__device__ __forceinline__ void meet() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

template <int N> struct phase_is { static constexpr int value = N; };

template <int AF, bool EXACT, class TL>
__global__ void __launch_bounds__(TL::THREADS, 2) k_mx_tile(const MatmulArgs p, int tiles_n, int tiles) {
  extern __shared__ __align__(16) uint8_t lds[];
  constexpr int AB = a_bytes<AF>(), MI = 4, NT = TL::NT, NST = stages<AF>(), SB = stage_bytes<AF, TL>(), WAT = TL::M * AB, SAT = NST * SB;
  constexpr int TM = TL::M, TN = TL::N, THREADS = TL::THREADS, SCALES = TL::SCALES;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, g = lane >> 4, wm = wave % TL::WM, wn = wave / TL::WM;
  const int steps = (p.kb + 3) >> 2;

  // Pieces that this thread fetches in every stage, from the tile's first row and column on;
  // and the row of a (the first TM threads) or of the weights whose scales it takes
  constexpr int PA = TM * AB / 16 / THREADS, PW = TN * 4 / THREADS, LOADS = PA + PW;
  const uint32_t row_bytes = (uint32_t)p.kb * mx<AF>::bytes32, col_bytes = (uint32_t)p.kb * 16;
  // row 16 j + x of a wave's rows of weights is its column 32 (j / 2) + 8 (x / 4) + 4 (j % 2) + x % 4
  auto column = [](int row) { return (row & 0xe0) + 8 * ((row & 15) >> 2) + 4 * ((row >> 4) & 1) + (row & 3); };
  uint32_t lane_a[PA], lane_w[PW];
#pragma unroll
  for (int i = 0; i < PA; ++i) {
    const int e = i * THREADS + tid, row = e / (AB / 16), c = AB == 128 ? (e & 7) ^ (row & 7) : (e & 3) ^ ((row >> 2) & 3);
    lane_a[i] = (uint32_t)row * row_bytes + 16 * c;
  }
#pragma unroll
  for (int i = 0; i < PW; ++i) {
    const int e = i * THREADS + tid, row = e >> 2, c = (e & 3) ^ ((row >> 2) & 3);
    lane_w[i] = (uint32_t)column(row) * col_bytes + 16 * c;
  }
  int64_t m0;
  int n0;
  i32x4 part_a, part_w;
  const uint8_t *src_s;
  auto place = [&](int k) {  // the workgroup's k-th tile; false behind the last
    // Workgroups are dealt to the eight dies in turn: each die gets neighbouring tiles, in blocks of eight rows of tiles that
    // pass over the columns, so that its cache keeps what they share.
    const int turn = k * (int)gridDim.x + (int)blockIdx.x;
    if (turn >= tiles) return false;
    const int chunk8 = tiles / 8, id = turn < chunk8 * 8 ? (turn & 7) * chunk8 + (turn >> 3) : turn;
    const int tiles_m = tiles / tiles_n, band = id / (8 * tiles_n), in_band = id - band * 8 * tiles_n;
    const int high = tiles_m - 8 * band < 8 ? tiles_m - 8 * band : 8;
    m0 = (int64_t)(8 * band + in_band % high) * TM;
    n0 = in_band / high * TN;
    part_a = part_of(p.a + m0 * row_bytes, (p.M - m0) * row_bytes);
    part_w = part_of(p.w + (int64_t)n0 * col_bytes, (int64_t)(p.N - n0) * col_bytes);
    // (rows that are not there take the last one's scales)
    const int64_t row = tid < TM ? (m0 + tid < p.M ? m0 + tid : p.M - 1) : (n0 + column(tid - TM) < p.N ? n0 + column(tid - TM) : p.N - 1);
    src_s = (tid < TM ? p.as : p.ws) + row * p.kb;
    return true;
  };
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
  const uint32_t wave_at = __builtin_amdgcn_readfirstlane(wave);
  // (behind a row's end lies the next row: those k of a are cleared before they are used)
  auto fetch = [&](int st) {
    const uint32_t at = base + (uint32_t)(st % NST) * SB + wave_at * 1024, k = st < steps ? st : steps - 1;
#pragma unroll
    for (int i = 0; i < PA; ++i) to_lds16(part_a, lane_a[i], k * AB, at + i * THREADS * 16);
#pragma unroll
    for (int i = 0; i < PW; ++i) to_lds16(part_w, lane_w[i], k * 64, at + WAT + i * THREADS * 16);
  };
  uint4 sq;  // scales on their way: of stages 4 k .. 4 k + 3
  // 16 bytes at any address, where the row ends before: its last 16, moved down, and scales of one behind them
  auto ask_scales = [&](int st) {
    const int b0 = 4 * st, from = b0 + 16 <= p.kb ? b0 : p.kb - 16, sh = b0 - from < 15 ? 8 * (b0 - from) : 120;
    const u16x8 v = *reinterpret_cast<const u16x8 *>(src_s + from);
    const uint64_t one = 0x7f7f7f7f7f7f7f7full, lo = v[0] | (uint64_t)v[1] << 32, hi = v[2] | (uint64_t)v[3] << 32;
    const uint64_t in = sh & 63 ? ~0ull : 0;  // (a shift by 64 is none)
    const uint64_t lo1 = sh < 64 ? lo : hi, hi1 = sh < 64 ? hi : one;
    const uint64_t a = lo1 >> (sh & 63) | (hi1 << (64 - (sh & 63) & 63) & in), b = hi1 >> (sh & 63) | (one << (64 - (sh & 63) & 63) & in);
    sq = make_uint4((uint32_t)a, (uint32_t)(a >> 32), (uint32_t)(sh < 64 ? b : one), (uint32_t)((sh < 64 ? b : one) >> 32));
  };
  auto first_scales = [&]() {
    if (p.kb >= 16) {
      ask_scales(0);
      return;
    }
    uint32_t w[4] = {0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu};
#pragma unroll
    for (int i = 0; i < 15; ++i)
      if (i < p.kb) w[i >> 2] = (w[i >> 2] & ~(255u << (8 * (i & 3)))) | (uint32_t)src_s[i] << (8 * (i & 3));
    sq = make_uint4(w[0], w[1], w[2], w[3]);
  };
  auto put_scales = [&](int st) { *reinterpret_cast<uint4 *>(lds + SAT + ((st >> 2) & 1) * SCALES + tid * 16) = sq; };

  f32x4 acc[NT][MI];
  uint4 ar[MI][AB / 64], wq[4];
  int as[MI], ws[4];
  // places of this lane's pieces in a stage: of row 16 i + r they lie a constant further for every i
  const int sw_a = AB == 128 ? r & 7 : (r >> 2) & 3;
  const int la0 = (wm * 64 + r) * AB + 16 * (g ^ sw_a), la1 = (wm * 64 + r) * AB + 16 * ((4 + g) ^ sw_a);
  const int lw = WAT + (wn * 16 * NT + r) * 64 + 16 * (g ^ ((r >> 2) & 3));
  const int lsa = SAT + (wm * 64 + r) * 16 + g, lsw = SAT + (TM + wn * 16 * NT + r) * 16 + g;
  auto read_a = [&](int st) {
    // (16 k at 16 g and, of 8-bit rows, 16 at 64 + 16 g)
    const uint8_t *at = lds + (st % NST) * SB, *sc = lds + lsa + ((st >> 2) & 1) * SCALES + 4 * (st & 3);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      ar[i][0] = *reinterpret_cast<const uint4 *>(at + la0 + i * 16 * AB);
      if (AF == VF_E4M3) ar[i][AB / 64 - 1] = *reinterpret_cast<const uint4 *>(at + la1 + i * 16 * AB);
      as[i] = sc[i * 256];
    }
  };
  auto read_w = [&](int st, int j) {
    wq[j & 3] = *reinterpret_cast<const uint4 *>(lds + (st % NST) * SB + lw + j * 16 * 64);
    ws[j & 3] = lds[lsw + ((st >> 2) & 1) * SCALES + 4 * (st & 3) + j * 256];
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
  // phase: st % 4, or -1: found at run time
  auto stage = [&](int st, auto phase) {
    const int ph = decltype(phase)::value >= 0 ? decltype(phase)::value : st & 3;
    read_a(st);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      if (j == NT / 2) {
        if (ph == 3) {
          put_scales(st + 1);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
        wait_loads<NST == 3 ? 0 : LOADS>();  // (of four stages the newest may still be under way)
        meet();
        fetch(st + NST - 1);
        if (ph == 1 && (decltype(phase)::value >= 0 || st + 3 < steps)) ask_scales(st + 3);
      }
      if (j + 2 < NT) read_w(st, j + 2);
      else read_w(st + 1, j + 2 - NT);
      products(j);
    }
  };

  bool there = place(0);
  if (there) {
    first_scales();
#pragma unroll
    for (int st = 0; st < NST - 1; ++st) fetch(st);
  }
  if (THREADS == 512 && wave < 4) __builtin_amdgcn_s_setprio(1);
  for (int k = 1; there; ++k) {
    const int64_t m_at = m0;
    const int n_at = n0;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MI; ++i) acc[j][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    put_scales(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wait_loads<0>();
    meet();
    read_w(0, 0);
    read_w(0, 1);
    // (Four stages without branches: past a branch the compiler would move the products, behind all reads.  Stages behind the last
    // one are the last one's bytes again, in places that nobody reads.)
    int st = 0;
    for (; st + 4 < steps; st += 4) {
      stage(st, phase_is<0>());
      stage(st + 1, phase_is<1>());
      stage(st + 2, phase_is<2>());
      stage(st + 3, phase_is<3>());
    }
    for (; st + 1 < steps; ++st) stage(st, phase_is<-1>());
    read_a(st);
    if (p.kb % 4 != 0) {  // k behind the row's end
      const int b0 = 4 * st;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        if (b0 + (AF == VF_E4M3 ? g >> 1 : g) >= p.kb) ar[i][0] = make_uint4(0, 0, 0, 0);
        if (AF == VF_E4M3 && b0 + 2 + (g >> 1) >= p.kb) ar[i][AB / 64 - 1] = make_uint4(0, 0, 0, 0);
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      if (j + 2 < NT) read_w(st, j + 2);
      products(j);
    }
    // the next tile's first stages, into places that the last stages no longer need
    wait_loads<0>();
    meet();
    there = place(k);
    if (there) {
      first_scales();
#pragma unroll
      for (int s = 0; s < NST - 1; ++s) fetch(s);
    }
    // a lane has columns n + 32 j / 2 .. + 7 of rows r, 16 + r, ...
    const int n = n_at + wn * 16 * NT + 8 * g;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < MI; ++i) asm volatile("" : "+v"(acc[j][i]));
#pragma unroll
    for (int j = 0; j < NT; j += 2) {
      const int c0 = n + 16 * j;
      float b[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) b[c] = p.bias && c0 + c < p.N ? p.bias[c0 + c] : 0.0f;
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        const int64_t m = m_at + wm * 64 + 16 * i + r;
        if (m >= p.M || c0 >= p.N) continue;
        float y[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) y[c] = acc[j + (c >> 2)][i][c & 3] + b[c];
        if (p.out_bf16) store_upto8(reinterpret_cast<uint16_t *>(p.out) + m * p.ld_out + c0, p.N - c0, y);
        else store_upto8(reinterpret_cast<float *>(p.out) + m * p.ld_out + c0, p.N - c0, y);
      }
    }
  }
  wait_loads<0>();
}

inline int blocks_for(int64_t threads) {
  const int64_t g = (threads + 255) / 256;
  return (int)(g < (1 << 20) ? g : (1 << 20));
}

template <int AF, bool EXACT, class TL>
int launch_tile(vf_ctx *c, const MatmulArgs &p) {
  constexpr int smem = stages<AF>() * stage_bytes<AF, TL>() + 2 * TL::SCALES, at_once = 256 * 512 / TL::THREADS;
  const int tiles_n = (p.N + TL::N - 1) / TL::N;
  // (tiles are counted in 32 bits; the rows are taken in several launches)
  const int64_t most = ((int64_t)1 << 28) / tiles_n, per = (most > 1 ? most : 1) * TL::M;
  const auto kernel = k_mx_tile<AF, EXACT, TL>;
  VF_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, smem));
  for (int64_t m = 0; m < p.M; m += per) {
    MatmulArgs q = p;
    q.a += m * p.kb * mx<AF>::bytes32;
    q.as += m * p.kb;
    q.M = p.M - m < per ? p.M - m : per;
    q.out = static_cast<char *>(p.out) + m * p.ld_out * (p.out_bf16 ? 2 : 4);
    const int tiles = (int)((q.M + TL::M - 1) / TL::M) * tiles_n;
    kernel<<<tiles < at_once ? tiles : at_once, TL::THREADS, smem, c->stream>>>(q, tiles_n, tiles);
    VF_HIP(c, hipGetLastError());
  }
  return VF_OK;
}

template <int AF, bool EXACT>
int matmul(vf_ctx *c, const MatmulArgs &p) {
  const int nb = (p.N + 15) / 16;
  // Tiles from 33 rows on, where the workgroups of k_mx_rows are more than the compute units (8-bit rows, K 4096, us: 64 rows, 4384
  // columns 27.8 in rows, 21.8 in tiles; 200 rows, 1024 columns 15.9 and 21.5; 1000 rows, 4384 columns 219 and 33).
  // (Offsets within 256 rows are 32 bits wide.)
  if (p.M > 32 && nb * ((p.M + 63) / 64) > 256 && p.kb <= (1 << 18)) {
    // By rounds of tiles: one of 256 large tiles takes 50 us, one of 512 small ones 34, of up to 256 small ones 22 (K 4096): 300 rows, 4384
    // columns 48 large, 22 small; 1400 rows 52 and 35; 3000 rows 55 and 68.  With rows taken in two parts the large ones' operands
    // do not fit the registers: 16384 rows 762 large, 540 small.
    const int64_t large = (((p.M + 255) / 256) * ((p.N + 255) / 256) + 255) / 256, small = ((p.M + 127) / 128) * ((p.N + 127) / 128);
    const int64_t rest = small % 512, small_cost = small / 512 * 34 + (rest == 0 ? 0 : rest <= 256 ? 22 : 34);
    if constexpr (!EXACT) {
      if (50 * large <= small_cost) return launch_tile<AF, EXACT, Large>(c, p);
    }
    return launch_tile<AF, EXACT, Small>(c, p);
  }
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
