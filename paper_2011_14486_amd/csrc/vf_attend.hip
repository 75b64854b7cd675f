// vf_kv_attend: attention of sequences' new tokens over their keys in a paged cache.
//
// One pass over the keys with a running maximum m and sum l per row: for every block of keys, S = scale q k^T, p = exp(S - m),
// l += sum p, out += p v; where a row's maximum grows, out and l shrink by exp(m_old - m_new) first, and at the end out / l is the result.
// Exponentials are powers of two, log2(e) is part of the scale.  m follows the maximum only when that has grown by more than MARGIN powers of two:
// p then goes up to 2^MARGIN, which no sum minds, and in nearly all blocks no lane has to ask the others.
//
// All heads that share a head of the cache are rows of one product (row r of a sequence: token r / group, head r % group), so its
// keys and values are fetched once for them.  Products are made as S^T = K Q^T and out^T = V^T P^T: a lane then holds scores of one row only, and the
// scores come out in the lanes and registers in which the second product takes them, up to the order of the keys in it, which is free as
// long as the values follow it.
//
// In bf16 the second product takes the weights as bf16.  Few rows, whose time is the memory's, have them as two numbers of bf16 each, right to 2^-15: one token
// behind 1001 keys 11.2 us for 11.0 with one number, 64 rows behind 2001 keys 104.4 for 104.4, 4 rows behind 131,072 keys in 8 bits 199.0 for 198.2, 1024 rows of 64 prefixes
// 52.7 for 51.4.  Many rows, whose time is the products', have one, rounded by 2^-8 of it at most, as outputs are: with two a prompt of 8192 tokens takes 797 us
// for 569, chunks from 8 bits 461 for 340, short whole sequences 356 for 338.  Their error to the outputs' size in root mean square is 1.8 - 2.3e-3, of exact outputs rounded 1.7e-3.
//
// Which kernel takes a call goes by what the host knows: rows of the longest sequence times heads that share one of the cache's, and the longest length.
// Up to 16 such rows: k_attend_rows; more: k_attend_tile in bf16, k_attend_wide or k_attend_rows in fp32.  Where there would be fewer workgroups than run at a
// time, several share the keys of a row block and k_attend_join joins them.
#include <math.h>

#include "vf_internal.h"
#include "vf_kv_dev.h"

namespace {

using namespace vfkv;

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float MARGIN = 8.0f;
constexpr float LOG2E = 1.44269504088896340736f;

struct AttendArgs {
  Cache c;
  Seqs s;
  const void *q;
  void *out;
  float *part;      // of workgroups that share a row block: [unit][rows][DP] sums, then [unit][rows] maxima, then [unit][rows] sums of weights
  int64_t ld_q, ld_out;
  float scale2;     // scale log2(e)
  Divisor group;
  int causal, window, longest;
  int blocks, splits;  // row blocks of the longest sequence; workgroups that share one along the keys
  bool by_length;      // sequences with most keys first
  const int2 *order;     // GROUP: sequences and their lengths, by first pages,
  const int32_t *items;  // and where groups that go together begin
};

// A workgroup's place: x = head of the cache + heads (share of the keys + splits row block), y: sequence.  (The launch has at most MAX_Y
// sequences side by side; workgroups go on to further ones.)
constexpr int MAX_Y = 32768;
struct Place { int head, split, block; };
__device__ __forceinline__ Place place_of(const AttendArgs &a) {
  Place p;
  const unsigned x = blockIdx.x, rest = x / (unsigned)a.c.heads;
  p.head = (int)(x - rest * (unsigned)a.c.heads);
  p.block = a.splits > 1 ? (int)(rest / (unsigned)a.splits) : (int)rest;
  p.split = a.splits > 1 ? (int)rest - p.block * a.splits : 0;
  return p;
}
// A number that is the same in all of a launch, as one that the compiler has to take anew: what it derives from it (which of an
// unrolled loop's numbers are there) is not kept over loops in registers that are then missing inside them.
__device__ __forceinline__ int anew(int v) {
  asm volatile("" : "+s"(v));
  return v;
}

// The keys that row i of a sequence sees: [lo, hi).
__device__ __forceinline__ void seen_by(const AttendArgs &a, const Span &sp, int i, int &lo, int &hi) {
  const int pos = sp.length - sp.rows + i;
  lo = a.window && pos >= a.window ? pos - a.window + 1 : 0;
  hi = !a.causal ? sp.length : pos < 0 ? 0 : pos + 1;
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// The maximum that weights are taken against: a row that has seen nothing yet has none.
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }

// A row's maxima and sums where parts of it are joined.
__device__ __forceinline__ float weight_of(float m, float top) { return exp2_(m - base_of(top)); }

// ---- few rows: keys and values straight from memory into the operands ----
//
// A wave holds 16 RB rows; its operands' other side are 32 keys (16 in fp32) at a time.  The four waves of a workgroup share the
// rows and take turns at the keys, or have rows of their own, or sequences.
//
// Rows of a search that go on from the same prefix have the same pages in front.  GROUP takes single tokens of up to 16 / group sequences that begin
// with the same page as the rows of one product: keys and values of blocks whose pages are the same are fetched once for all of them, others for one sequence at a
// time, with the other sequences' rows not seeing them.
//
// What bounds it is the memory, with few workgroups its latency: keys, values and pages of a step are asked for one step before.  Values lie with their numbers side by
// side, and the product wants keys side by side: the numbers of eight keys, eight of each, are turned around in registers, halves by halves, 32 instructions
// for 8 products, which memory's time hides.
// MI355X: 4 rows of 32 heads of 128 behind 131,072 keys of 8 heads in 8 bits, 1.1 GB, 199 us = 5.6 TB/s (503 with a step's loads behind the step before, 235 with pages
// by vector loads); 64 rows behind 2001 keys in bf16 105 us = 5.0 TB/s, in 8 bits 45; 1024 rows behind 501 keys of 64 prefixes, 16 over 4 heads of 64, 42 us and 10 for the groups (57
// apart); one row behind 1001 keys 11 us, of which 5 are there without keys.
enum { SHARE, ROWWISE, SEQWISE, GROUP, SHARE8 };   // SHARE8: eight waves, where there are few workgroups

template <typename T, int FMT, int DP> struct Shape;
// K operand: the lane of key n and quarter g takes elements; V operand: lane c takes VW neighbouring numbers of a value, NH times
template <int FMT, int DP> struct Shape<uint16_t, FMT, DP> {
  static constexpr int STEP = 32, VW = DP >= 128 ? 8 : DP / 16, NH = DP / (16 * VW), NK = DP / 32;
};
template <int FMT, int DP> struct Shape<float, FMT, DP> {
  static constexpr int STEP = 16, VW = DP >= 64 ? 4 : DP / 16, NH = DP / (16 * VW), NK = DP / 16;
};

__device__ __forceinline__ bf16x8 as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d});
}
__device__ __forceinline__ uint32_t cvt2(uint32_t codes, float scale, bool high) {
  const bf16x2 v = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float scale_of(uint8_t byte) { return __uint_as_float((uint32_t)byte << 23); }
// whether a half of a pair of bf16 is infinite or NaN, and the pair without such halves, and 1 in their places
__device__ __forceinline__ bool not_finite(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ uint32_t finite_of(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0 : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0 : w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t marks_of(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0x3f80u : 0) | ((w & 0x7f800000u) == 0x7f800000u ? 0x3f800000u : 0);
}

// Two weights as pairs of bf16 whose sums they are to 2^-15: their upper halves, and what is left of them, which is never negative.  (The rest
// of a weight that is not zero is not zero either, so that an infinite value stays infinite in both products.)
__device__ __forceinline__ void two_parts(float a, float b, uint32_t &upper, uint32_t &rest) {
  const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
  upper = __builtin_amdgcn_perm(y, x, 0x07060302u);
  rest = pack2(fmaxf(a - __uint_as_float(x & 0xffff0000u), a * 0x1p-24f), fmaxf(b - __uint_as_float(y & 0xffff0000u), b * 0x1p-24f));
}

// First of the eight numbers (four in fp32) of k-step ks that a lane of quarter g holds: whole pieces of 16 bytes of a row.
template <typename T, int FMT, int DP>
__device__ __forceinline__ int k_at(int ks, int g) {
  if constexpr (sizeof(T) == 4) return 16 * ks + 4 * g;
  else if constexpr (FMT == VF_E4M3 && DP >= 64) return ((ks >> 1) * 4 + g) * 16 + (ks & 1) * 8;
  else return 32 * ks + 8 * g;
}

template <typename T, int FMT, int DP, int RB, int MODE>
__global__ void __launch_bounds__(MODE == SHARE8 ? 512 : 256, MODE == GROUP && DP <= 64 ? 3 : DP <= 128 ? 2 : MODE == SHARE8 ? 2 : 1) k_attend_rows(const AttendArgs a) {
  typedef Shape<T, FMT, DP> S;
  constexpr bool ALONG = MODE == ROWWISE || MODE == SEQWISE, G = MODE == GROUP;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int STEP = S::STEP, VW = S::VW, NH = S::NH, NK = S::NK, ROWS = 16 * RB * (MODE == ROWWISE ? 4 : 1), NA = NH * VW;
  constexpr int KB = STEP / 16;  // blocks of 16 keys in a step
  constexpr int WAVES = MODE == SHARE8 ? 8 : 4;
  __shared__ f32x4 join[ALONG ? 1 : WAVES / 2][ALONG ? 1 : RB * NA][64];
  __shared__ float join_m[ALONG ? 1 : WAVES][16 * RB], join_l[ALONG ? 1 : WAVES][16 * RB];
  const int lane = (int)threadIdx.x & 63, n = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const Cache &c = a.c;
  const Place place = place_of(a);
  const int head = place.head, split = place.split;
  constexpr int SEQS = MODE == SEQWISE ? 4 : 1;
  for (int turn = (int)blockIdx.y * SEQS + (MODE == SEQWISE ? wave : 0); turn < a.s.n; turn += (int)gridDim.y * SEQS) {
    // (a group: its first place in the order, its sequences)
    const int begin = G ? a.items[turn] : 0, members = G ? a.items[turn + 1] - begin : 1;
    if (members == 0) break;
    const int seq = G ? 0 : turn;
    const Span sp = G ? Span{0, 1, 0} : span_of(a.s, c.shift, seq);
    const int all = G ? members * a.group.by : sp.rows * a.group.by;
    for (int block = place.block; (int64_t)block * ROWS < all; block += a.blocks) {
      // (row blocks that the plan did not count on are not shared)
      const bool shared = a.splits > 1 && block < a.blocks;
      if (block >= a.blocks && split > 0) break;
      const int dim = anew(c.dim), width = anew(c.width);
      const int r0 = block * ROWS + (MODE == ROWWISE ? wave * 16 * RB : 0), r1 = all - r0 > 16 * RB ? r0 + 16 * RB : all;
      // what the wave's rows see: all of [lo_in, hi_in), nothing outside [lo, hi)
      int lo = 0, hi = 0, lo_in = 0, hi_in = 0;
      if (!G && r0 < r1) {
        seen_by(a, sp, over(a.group, r0), lo, hi_in);
        seen_by(a, sp, over(a.group, r1 - 1), lo_in, hi);
      }
      int row_lo[RB], row_hi[RB], row_seq[RB];
      const T *q_row[RB];
      int64_t out_row[RB];
      const int member = G ? over(a.group, n) : 0;   // of a group: the lane's row's sequence
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const int r = r0 + 16 * b + n;
        row_lo[b] = row_hi[b] = 0;
        row_seq[b] = seq;
        q_row[b] = nullptr;
        out_row[b] = -1;
        if (r < r1) {
          const int x = over(a.group, r), h = head * a.group.by + r - x * a.group.by;
          Span own = sp;
          if constexpr (G) {   // (a row a sequence, without offsets)
            const int2 of = a.order[begin + x];
            row_seq[b] = of.x;
            own = Span{of.x, 1, of.y};
          }
          const int i = G ? 0 : x;
          seen_by(a, own, i, row_lo[b], row_hi[b]);
          q_row[b] = reinterpret_cast<const T *>(a.q) + (own.first + i) * a.ld_q + (int64_t)h * dim;
          out_row[b] = (own.first + i) * a.ld_out + (int64_t)h * dim;
        }
      }
      if constexpr (G) {
        lo = lo_in = row_lo[0];
        hi = hi_in = row_hi[0];
        if (n >= r1) {   // (no row: it bounds nothing)
          lo = hi_in = 0x7fffffff;
          hi = lo_in = 0;
        }
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) {
          int o = __shfl_xor(lo, x);
          lo = o < lo ? o : lo;
          o = __shfl_xor(hi_in, x);
          hi_in = o < hi_in ? o : hi_in;
          o = __shfl_xor(hi, x);
          hi = o > hi ? o : hi;
          o = __shfl_xor(lo_in, x);
          lo_in = o > lo_in ? o : lo_in;
        }
        lo = __builtin_amdgcn_readfirstlane(lo);
        hi = __builtin_amdgcn_readfirstlane(hi);
        lo_in = __builtin_amdgcn_readfirstlane(lo_in);
        hi_in = __builtin_amdgcn_readfirstlane(hi_in);
      }
      // queries as operands
      uint4 q16[F32 ? 1 : RB][F32 ? 1 : NK];
      f32x4 q32[F32 ? RB : 1][F32 ? NK : 1];
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int ks = 0; ks < NK; ++ks) {
          const int d = k_at<T, FMT, DP>(ks, g), left = q_row[b] ? dim - d : 0;
          if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) q32[b][ks][i] = i < left ? q_row[b][d + i] : 0.0f;
          } else {
            raw8<uint16_t> w = {};
            if (left > 0) fetch8(q_row[b] + d, left, w);
            q16[b][ks] = make_uint4(w.w[0], w.w[1], w.w[2], w.w[3]);
          }
        }
      f32x4 acc[RB][NA];
      float m[RB], l[RB];
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        m[b] = -INFINITY;
        l[b] = 0.0f;
#pragma unroll
        for (int i = 0; i < NA; ++i) acc[b][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
      // the steps of this workgroup, and of this wave among them
      const int from = lo & ~(STEP - 1);
      int steps = hi > from ? (hi - from + STEP - 1) / STEP : 0, s0 = 0;
      if (shared) {
        const int each = (steps + a.splits - 1) / a.splits;
        s0 = (int)((int64_t)each * split < steps ? each * split : steps);
        steps = steps - s0 < each ? steps : s0 + each;
      }
      // A step's keys and values on their way: as they are in memory.  A step's are sent for when the registers of the step before are free, keys behind
      // the scores, values behind the outputs; pages one step earlier.
      constexpr int STRIDE = ALONG ? 1 : WAVES;
      constexpr int VD = F32 ? VW : (VW + 1) / 2;                    // registers of VW values
      constexpr int KL = F32 ? NK : FMT == VF_E4M3 && DP >= 64 ? NK / 2 : NK;   // pieces of a key
      typedef uint32_t kv4 __attribute__((ext_vector_type(FMT == VF_E4M3 ? (F32 ? 1 : DP >= 64 ? 4 : 2) : 4)));
      kv4 kraw[KB][KL];
      uint32_t vraw[KB][4][NH][FMT == VF_E4M3 ? (VW + 3) / 4 : VD];
      uint8_t kscale[KB][FMT == VF_E4M3 ? KL : 1], vscale[KB][4][FMT == VF_E4M3 ? NH : 1];
      // what a turn of the loop takes: a step's blocks of 16 keys in these pages, for all rows (who -1) or for those of one member of a group, which sees
      // [lo, hi)
      struct Pages { int st, who, lo, hi, entry[KB]; };
      auto pages_at = [&](int st) {
        Pages p;
        p.st = st;
        p.who = -1;
        p.lo = lo;
        p.hi = hi;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) p.entry[kb] = st < steps ? entry_of(a.s, c.shift, seq, from + st * STEP + 16 * kb) : -1;
        return p;
      };
      // a group's: lane x asks for block x % KB of member x / KB
      const int asker = lane / KB, asked_block = lane % KB;
      int ask_seq = 0, ask_lo = 0, ask_hi = 0;
      if (G && asker < members) {
        const int2 of = a.order[begin + asker];
        ask_seq = of.x;
        seen_by(a, Span{of.x, 1, of.y}, 0, ask_lo, ask_hi);
      }
      auto entries_at = [&](int st) {
        const int t = from + st * STEP + 16 * asked_block;
        return asker < members && st < steps && t < ask_hi ? entry_of(a.s, c.shift, ask_seq, t) : -1;
      };
      // the pages of step st from member `who` on; who = members if none is left
      auto pages_of_group = [&](int st, int entries, int who) {
        Pages p;
        p.st = st;
        p.who = -1;
        p.lo = lo;
        p.hi = hi;
        const int t = from + st * STEP + 16 * asked_block;
        const bool on = asker < members && t < ask_hi && t + 16 > ask_lo;
        bool same = true;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const unsigned long long those = __ballot(on && asked_block == kb);
          p.entry[kb] = those ? __builtin_amdgcn_readlane(entries, (int)__ffsll(those) - 1) : -1;
          same = same && !__ballot(on && asked_block == kb && entries != p.entry[kb]);
        }
        if (same) {
          if (who > 0) p.who = members;
          return p;
        }
        const unsigned long long those = __ballot(on && asker >= who);
        p.who = those ? ((int)__ffsll(those) - 1) / KB : members;
        if (!those) return p;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const bool sees = __ballot(on) >> (p.who * KB + kb) & 1;
          p.entry[kb] = sees ? __builtin_amdgcn_readlane(entries, p.who * KB + kb) : -1;
        }
        p.lo = __builtin_amdgcn_readlane(ask_lo, p.who * KB);
        p.hi = __builtin_amdgcn_readlane(ask_hi, p.who * KB);
        return p;
      };
      // (what is fetched of an entry that is no page, and behind a row's end, is not used)
      auto page_of = [&](const Pages &p, int kb) { return (unsigned)p.entry[kb] < (unsigned)c.pages ? p.entry[kb] : 0; };
      auto ask_keys = [&](const Pages &p) {
        const int st = p.st;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const int64_t row = row_of(c, page_of(p, kb), head, from + st * STEP + 16 * kb + n);
          const typename kv_elem<FMT>::type *k = reinterpret_cast<const typename kv_elem<FMT>::type *>(c.k) + row * width;
#pragma unroll
          for (int x = 0; x < KL; ++x) {
            int d = k_at<T, FMT, DP>(x * (NK / KL), g);
            d = d < width ? d : 0;
            kraw[kb][x] = *reinterpret_cast<const kv4 *>(k + d);
            if constexpr (FMT == VF_E4M3) kscale[kb][x] = c.ks[row * c.kb + (d >> 5)];
          }
        }
      };
      auto ask_values = [&](const Pages &p) {
        const int st = p.st;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const int64_t row = row_of(c, page_of(p, kb), head, from + st * STEP + 16 * kb + 4 * g);
          const typename kv_elem<FMT>::type *v = reinterpret_cast<const typename kv_elem<FMT>::type *>(c.v) + row * width;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < NH; ++h) {
              int d = h * 16 * VW + n * VW;
              d = d < width ? d : 0;
              const auto *at = v + (int64_t)i * width + d;
              if constexpr (FMT == VF_E4M3) {
                if constexpr (VW == 8) {
                  const uint2 w = *reinterpret_cast<const uint2 *>(at);
                  vraw[kb][i][h][0] = w.x;
                  vraw[kb][i][h][(VW + 3) / 4 - 1] = w.y;
                } else if constexpr (VW == 4) {
                  vraw[kb][i][h][0] = *reinterpret_cast<const uint32_t *>(at);
                } else {
                  vraw[kb][i][h][0] = *reinterpret_cast<const uint16_t *>(at);
                }
                vscale[kb][i][h] = c.vs[(row + i) * c.kb + (d >> 5)];
              } else if constexpr (VD == 1) {
                vraw[kb][i][h][0] = *reinterpret_cast<const uint32_t *>(at);
              } else {
                typedef uint32_t uv __attribute__((ext_vector_type(VD)));
                const uv w = *reinterpret_cast<const uv *>(at);
#pragma unroll
                for (int x = 0; x < VD; ++x) vraw[kb][i][h][x] = w[x];
              }
            }
        }
      };
      const int first = s0 + (ALONG ? 0 : wave);
      Pages now, next;
      int entries = 0, entries_after = 0;   // of a group: of now's step, and of the one behind it
      if constexpr (G) {
        entries = entries_at(first);
        now = pages_of_group(first, entries, 0);
        entries_after = entries_at(first + STRIDE);
      } else {
        now = pages_at(first);
        next = pages_at(first + STRIDE);
      }
      if (first < steps) {
        ask_keys(now);
        ask_values(now);
      }
      while (now.st < steps) {
        const int t0 = from + now.st * STEP, who = now.who;
        Pages after = now;
        if constexpr (G) {
          next = now;
          next.who = members;
          if (who >= 0) next = pages_of_group(now.st, entries, who + 1);
          if (next.who == members) {
            entries = entries_after;
            next = pages_of_group(now.st + STRIDE, entries, 0);
            entries_after = entries_at(now.st + 2 * STRIDE);
          }
        }
        bool fine = true;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) fine = fine && (unsigned)now.entry[kb] < (unsigned)c.pages;
        const bool edge = !fine || t0 < lo_in || t0 + STEP > hi_in || (G && who >= 0);
        const int(&entry)[KB] = now.entry;
        f32x4 sc[RB][KB];
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) sc[b][kb] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int x = 0; x < KL; ++x) {
            const bool in = k_at<T, FMT, DP>(x * (NK / KL), g) < width;
            kv4 w = kraw[kb][x];
            if constexpr (F32) {
              f32x4 key;
              if constexpr (FMT == VF_E4M3) {
                const float s = scale_of(kscale[kb][x]);
                const f32x2 lo2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], s, false), hi2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], s, true);
                key = f32x4{lo2[0], lo2[1], hi2[0], hi2[1]};
              } else {
                key = __builtin_bit_cast(f32x4, w);
              }
#pragma unroll
              for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int b = 0; b < RB; ++b) sc[b][kb] = __builtin_amdgcn_mfma_f32_16x16x4f32(in ? key[e] : 0.0f, q32[b][x][e], sc[b][kb], 0, 0, 0);
            } else if constexpr (FMT == VF_E4M3) {
              const float s = scale_of(kscale[kb][x]);
#pragma unroll
              for (int half = 0; half < NK / KL; ++half) {
                const uint32_t w0 = in ? w[2 * half] : 0, w1 = in ? w[2 * half + 1] : 0;
                const bf16x8 key = as_bf16x8(cvt2(w0, in ? s : 1.0f, false), cvt2(w0, in ? s : 1.0f, true), cvt2(w1, in ? s : 1.0f, false), cvt2(w1, in ? s : 1.0f, true));
#pragma unroll
                for (int b = 0; b < RB; ++b)
                  sc[b][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, __builtin_bit_cast(bf16x8, q16[b][x * (NK / KL) + half]), sc[b][kb], 0, 0, 0);
              }
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) w[e] = in ? w[e] : 0;
#pragma unroll
              for (int b = 0; b < RB; ++b)
                sc[b][kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, q16[b][x]), sc[b][kb], 0, 0, 0);
            }
          }
        if (next.st < steps) ask_keys(next);
        if constexpr (!G) after = pages_at(now.st + 2 * STRIDE);
        // values as numbers: of key 4 g + i of each block of 16 the VW numbers at c VW of each part
        uint32_t val[KB][4][NH][VD];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < NH; ++h) {
              if constexpr (FMT != VF_E4M3) {
#pragma unroll
                for (int x = 0; x < VD; ++x) val[kb][i][h][x] = vraw[kb][i][h][x];
              } else {
                const float s = scale_of(vscale[kb][i][h]);
#pragma unroll
                for (int x = 0; x < (VW + 1) / 2; ++x) {
                  const uint32_t w = vraw[kb][i][h][x >> 1];
                  if constexpr (F32) {
                    const f32x2 v = x & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, true) : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, false);
                    val[kb][i][h][2 * x] = __float_as_uint(v[0]);
                    val[kb][i][h][2 * x + 1] = __float_as_uint(v[1]);
                  } else {
                    val[kb][i][h][x] = cvt2(w, s, x & 1);
                  }
                }
              }
            }
        bool odd = false;  // whether some value that only some rows see is not finite
        if (edge) {
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int t = t0 + 16 * kb + 4 * g + i;
              const bool there = (unsigned)entry[kb] < (unsigned)c.pages;
#pragma unroll
              for (int b = 0; b < RB; ++b) {
                const bool seen = t >= row_lo[b] && t < row_hi[b] && entry[kb] != -1 && (!G || who < 0 || member == who);
                sc[b][kb][i] = !seen ? -INFINITY : there ? sc[b][kb][i] : __builtin_nanf("");
              }
              const bool any = t >= now.lo && t < now.hi && there;
#pragma unroll
              for (int h = 0; h < NH; ++h)
#pragma unroll
                for (int x = 0; x < VD; ++x) {
                  if (!any || h * 16 * VW + n * VW >= width) val[kb][i][h][x] = 0;
                  odd = odd || (F32 ? (val[kb][i][h][x] & 0x7f800000u) == 0x7f800000u : not_finite(val[kb][i][h][x]));
                }
            }
        }
        // maxima: followed where one has grown by much
        float top[RB];
        bool grown = false;
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          top[b] = sc[b][0][0];
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) top[b] = fmaxf(top[b], sc[b][kb][i]);
          top[b] *= a.scale2;
          grown = grown || top[b] > m[b] + MARGIN;
        }
        if (__any(grown)) {
#pragma unroll
          for (int b = 0; b < RB; ++b) {
            float t = fmaxf(top[b], m[b]);
            t = fmaxf(t, __shfl_xor(t, 16));
            t = fmaxf(t, __shfl_xor(t, 32));
            const float f = exp2_(m[b] - base_of(t));
            m[b] = t;
            l[b] *= f;
#pragma unroll
            for (int i = 0; i < NA; ++i) acc[b][i] *= f;
          }
        }
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          const float base = base_of(m[b]);
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              sc[b][kb][i] = exp2_(fmaf(sc[b][kb][i], a.scale2, -base));
              l[b] += sc[b][kb][i];
            }
        }
        // values that are not finite reach the rows that see them only: they are left out of the products, and of a product of
        // ones in their places with ones in the places of what is seen, whatever is not zero makes NaN
        auto seen_mark = [&](int b, int kb, int i) {
          const int t = t0 + 16 * kb + 4 * g + i;
          return t >= row_lo[b] && t < row_hi[b] && entry[kb] != -1 && (!G || who < 0 || member == who);
        };
        const bool odd_step = edge && __any(odd);
        if constexpr (F32) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < NH; ++h)
#pragma unroll
              for (int x = 0; x < VW; ++x) {
                float v = __uint_as_float(val[0][i][h][x]);
                if (odd_step) {
                  const bool bad = (val[0][i][h][x] & 0x7f800000u) == 0x7f800000u;
#pragma unroll
                  for (int b = 0; b < RB; ++b) {
                    f32x4 hit = {0.0f, 0.0f, 0.0f, 0.0f};
                    hit = __builtin_amdgcn_mfma_f32_16x16x4f32(bad ? 1.0f : 0.0f, seen_mark(b, 0, i) ? 1.0f : 0.0f, hit, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                      if (hit[e] != 0.0f) acc[b][h * VW + x][e] = __builtin_nanf("");
                  }
                  v = bad ? 0.0f : v;
                }
#pragma unroll
                for (int b = 0; b < RB; ++b) acc[b][h * VW + x] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, sc[b][0][i], acc[b][h * VW + x], 0, 0, 0);
              }
        } else {
          bf16x8 p[RB], rest[RB];
#pragma unroll
          for (int b = 0; b < RB; ++b) {
            uint32_t w[4], r[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) two_parts(sc[b][e >> 1][2 * (e & 1)], sc[b][e >> 1][2 * (e & 1) + 1], w[e], r[e]);
            p[b] = as_bf16x8(w[0], w[1], w[2], w[3]);
            rest[b] = as_bf16x8(r[0], r[1], r[2], r[3]);
          }
#pragma unroll
          for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int x = 0; x < VW; ++x) {
              // (halves x % 2 of registers x / 2 of neighbouring keys)
              const uint32_t pick = x & 1 ? 0x07060302u : 0x05040100u;
              uint32_t w[4];
#pragma unroll
              for (int e = 0; e < 4; ++e)
                w[e] = __builtin_amdgcn_perm(val[e >> 1][2 * (e & 1) + 1][h][x >> 1], val[e >> 1][2 * (e & 1)][h][x >> 1], pick);
              if (odd_step) {
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                  f32x4 hit = {0.0f, 0.0f, 0.0f, 0.0f};
                  uint32_t see[4];
#pragma unroll
                  for (int e = 0; e < 4; ++e)
                    see[e] = (seen_mark(b, e >> 1, 2 * (e & 1)) ? 0x3f80u : 0) | (seen_mark(b, e >> 1, 2 * (e & 1) + 1) ? 0x3f800000u : 0);
                  hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(marks_of(w[0]), marks_of(w[1]), marks_of(w[2]), marks_of(w[3])),
                                                               as_bf16x8(see[0], see[1], see[2], see[3]), hit, 0, 0, 0);
#pragma unroll
                  for (int e = 0; e < 4; ++e)
                    if (hit[e] != 0.0f) acc[b][h * VW + x][e] = __builtin_nanf("");
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = finite_of(w[e]);
              }
#pragma unroll
              for (int b = 0; b < RB; ++b)
                acc[b][h * VW + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w[0], w[1], w[2], w[3]), p[b], acc[b][h * VW + x], 0, 0, 0);
#pragma unroll
              for (int b = 0; b < RB; ++b)
                acc[b][h * VW + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w[0], w[1], w[2], w[3]), rest[b], acc[b][h * VW + x], 0, 0, 0);
            }
        }
        if (next.st < steps) ask_values(next);
        now = next;
        if constexpr (!G) next = after;
      }
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        l[b] += __shfl_xor(l[b], 16);
        l[b] += __shfl_xor(l[b], 32);
      }
      // the waves' shares of the keys: the upper half of the waves gives theirs to the lower, until one has all
      if constexpr (!ALONG) {
        __syncthreads();
        if (g == 0) {
#pragma unroll
          for (int b = 0; b < RB; ++b) {
            join_m[wave][16 * b + n] = m[b];
            join_l[wave][16 * b + n] = l[b];
          }
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          float t = join_m[0][16 * b + n];
#pragma unroll
          for (int w = 1; w < WAVES; ++w) t = fmaxf(t, join_m[w][16 * b + n]);
          l[b] = 0.0f;
#pragma unroll
          for (int w = 0; w < WAVES; ++w) l[b] += join_l[w][16 * b + n] * weight_of(join_m[w][16 * b + n], t);
          const float f = weight_of(m[b], t);
          m[b] = t;
#pragma unroll
          for (int i = 0; i < NA; ++i) acc[b][i] *= f;
        }
#pragma unroll
        for (int half = WAVES / 2; half >= 1; half >>= 1) {
          if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
              for (int i = 0; i < NA; ++i) join[wave - half][b * NA + i][lane] = acc[b][i];
          }
          __syncthreads();
          if (wave < half) {
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
              for (int i = 0; i < NA; ++i) acc[b][i] += join[wave][b * NA + i][lane];
          }
          __syncthreads();
        }
        if (wave > 0) continue;
      }
      // numbers h 16 VW + (4 g + e) VW + x of row n are in acc[h VW + x][e]
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        if (shared) {
          const int64_t at = ((int64_t)row_seq[b] * gridDim.x + blockIdx.x) * ROWS + (G ? n - member * a.group.by : (MODE == ROWWISE ? wave * 16 * RB : 0) + 16 * b + n);
          if (G && n >= r1) continue;
          float *o = a.part + at * DP;
#pragma unroll
          for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int x = 0; x < VW; ++x) o[h * 16 * VW + (4 * g + e) * VW + x] = acc[b][h * VW + x][e];
          if (g == 0) {
            const int64_t parts = (int64_t)a.s.n * gridDim.x * ROWS;
            float *stat = a.part + parts * DP;
            stat[at] = m[b];
            stat[parts + at] = l[b];
          }
        } else if (out_row[b] >= 0) {
          const float inv = l[b] == 0.0f ? 0.0f : 1.0f / l[b];
          T *o = reinterpret_cast<T *>(a.out) + out_row[b];
#pragma unroll
          for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int d = h * 16 * VW + (4 * g + e) * VW;
              float v[8];
#pragma unroll
              for (int x = 0; x < 8; ++x) v[x] = x < VW ? acc[b][h * VW + x % VW][e] * inv : 0.0f;
              const int left = dim - d < VW ? dim - d : VW;
              if (left > 0) store_upto8(o + d, left, v);
            }
        }
      }
    }
  }
}

// ---- many rows in fp32: 32 rows a wave, keys and values straight from memory ----
//
// Products of 32 by 32 numbers, two of the sum at a time, take so long that one wave a SIMD keeps the matrix cores busy as long as its operands are
// there: a step's keys are sent for behind the scores of the step before, its values behind the outputs.  Lane n of half g holds key n, and takes the
// numbers d = 8 x + 4 g + e for product (x, e); of value 8 (i / 4) + 4 g + i % 4, whose weight is in register i, it takes the VW numbers at VW n, one for each of VW products.
// MI355X: a prompt of 2048 tokens, 32 heads of 128 over 8 of the cache, 400 us = 86 TFLOP/s, of the 154 that the vendor library's product reaches: matrix cores busy
// 54 % of the cycles, the rest is weights and moves beside them, which nothing else hides with one wave a SIMD.
template <int FMT, int DP>
__global__ void __launch_bounds__(256, DP <= 64 ? 2 : 1) k_attend_wide(const AttendArgs a) {
  constexpr int ROWS = 128, STEP = 32, NX = DP / 8, VW = DP / 32;
  constexpr bool MX8 = FMT == VF_E4M3;
  typedef typename kv_elem<FMT>::type E;
  typedef uint32_t k4 __attribute__((ext_vector_type(MX8 ? 1 : 4)));
  constexpr int VR = MX8 ? 1 : VW;   // registers of VW numbers
  const int lane = (int)threadIdx.x & 63, n = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const Cache &c = a.c;
  const Place place = place_of(a);
  const int head = place.head, split = place.split;
  for (int seq = blockIdx.y; seq < a.s.n; seq += gridDim.y) {
    const Span sp = span_of(a.s, c.shift, seq);
    const int all = sp.rows * a.group.by;
    // (row blocks that see the most keys come first)
    for (int block = a.blocks - 1 - place.block; (int64_t)block * ROWS < all; block += a.blocks) {
      const bool shared = a.splits > 1 && block < a.blocks;
      if (block >= a.blocks && split > 0) break;
      const int dim = anew(c.dim), width = anew(c.width);
      const int r0 = block * ROWS + 32 * wave, r1 = all - r0 > 32 ? r0 + 32 : all;
      int lo = 0, hi = 0, lo_in = 0, hi_in = 0, row_lo = 0, row_hi = 0;
      if (r0 < r1) {
        seen_by(a, sp, over(a.group, r0), lo, hi_in);
        seen_by(a, sp, over(a.group, r1 - 1), lo_in, hi);
      }
      const float *q_row = nullptr;
      int64_t out_row = -1;
      const int r = r0 + n;
      if (r < r1) {
        const int i = over(a.group, r), h = head * a.group.by + r - i * a.group.by;
        seen_by(a, sp, i, row_lo, row_hi);
        q_row = reinterpret_cast<const float *>(a.q) + (sp.first + i) * a.ld_q + (int64_t)h * dim;
        out_row = (sp.first + i) * a.ld_out + (int64_t)h * dim;
      }
      f32x4 q[NX];
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const int d = 8 * x + 4 * g, left = q_row ? dim - d : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) q[x][e] = e < left ? q_row[d + e] : 0.0f;
      }
      f32x16 acc[VW];
#pragma unroll
      for (int x = 0; x < VW; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[x][i] = 0.0f;
      float m = -INFINITY, l = 0.0f;
      const int from = lo & ~(STEP - 1);
      int steps = hi > from ? (hi - from + STEP - 1) / STEP : 0, s0 = 0;
      if (shared) {
        const int each = (steps + a.splits - 1) / a.splits;
        s0 = (int)((int64_t)each * split < steps ? each * split : steps);
        steps = steps - s0 < each ? steps : s0 + each;
      }
      k4 kraw[NX];
      uint32_t vraw[16][VR];
      uint8_t kscale[MX8 ? VW : 1], vscale[MX8 ? 16 : 1];
      struct Pages { int entry[2]; };
      auto pages_at = [&](int st) {
        Pages p;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) p.entry[kb] = st < steps ? entry_of(a.s, c.shift, seq, from + st * STEP + 16 * kb) : -1;
        return p;
      };
      // (what is fetched of an entry that is no page, and behind a row's end, is not used)
      auto page_of = [&](const Pages &p, int kb) { return (unsigned)p.entry[kb] < (unsigned)c.pages ? p.entry[kb] : 0; };
      // A lane's numbers of a value, which end with the row: three are no part of a row of 80 or 88, and the lane whose three would go past its end
      // takes the last three of the row and leaves the first `skip` of them out.  MI355X, a prompt of 2048 with 32 heads of 80 over 8: 316 us, in the instance for 128 388.
      const int own_d = VW * n >= width ? 0 : VW * n + VW <= width ? VW * n : width - VW, skip = VW == 3 && VW * n < width ? VW * n - own_d : 0;
      auto ask_keys = [&](int st, const Pages &p) {
        const int64_t row = row_of(c, n < 16 ? page_of(p, 0) : page_of(p, 1), head, from + st * STEP + n);
        const E *k = reinterpret_cast<const E *>(c.k) + row * width;
#pragma unroll
        for (int x = 0; x < NX; ++x) {
          const int d = 8 * x + 4 * g;
          kraw[x] = *reinterpret_cast<const k4 *>(k + (d < width ? d : 0));
        }
        if constexpr (MX8) {
#pragma unroll
          for (int b = 0; b < VW; ++b) kscale[b] = c.ks[row * c.kb + (b < c.kb ? b : 0)];
        }
      };
      auto ask_values = [&](int st, const Pages &p) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int64_t row = row_of(c, page_of(p, i >> 3), head, from + st * STEP + 8 * (i >> 2) + 4 * g + (i & 3));
          const E *v = reinterpret_cast<const E *>(c.v) + row * width + own_d;
          if constexpr (!MX8) {
            typedef uint32_t uv __attribute__((ext_vector_type(VW), aligned(4)));
            const uv w = *reinterpret_cast<const uv *>(v);
#pragma unroll
            for (int x = 0; x < VW; ++x) vraw[i][x] = w[x];
          } else {
            if constexpr (VW == 4) vraw[i][0] = *reinterpret_cast<const uint32_t *>(v);
            else if constexpr (VW == 2) vraw[i][0] = *reinterpret_cast<const uint16_t *>(v);
            else vraw[i][0] = *v;
            vscale[i] = c.vs[row * c.kb + (own_d >> 5)];
          }
        }
      };
      Pages now = pages_at(s0), next = pages_at(s0 + 1);
      if (s0 < steps) {
        ask_keys(s0, now);
        ask_values(s0, now);
      }
      for (int st = s0; st < steps; ++st) {
        const int t0 = from + st * STEP;
        const bool there0 = (unsigned)now.entry[0] < (unsigned)c.pages, there1 = (unsigned)now.entry[1] < (unsigned)c.pages;
        const bool edge = !there0 || !there1 || t0 < lo_in || t0 + STEP > hi_in;
        f32x16 sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
#pragma unroll
        for (int x = 0; x < NX; ++x) {
          f32x4 k;
          if constexpr (MX8) {
            const float s = scale_of(kscale[x >> 2]);
            const f32x2 k0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(kraw[x][0], s, false), k1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(kraw[x][0], s, true);
            k = f32x4{k0[0], k0[1], k1[0], k1[1]};
          } else {
            k = __builtin_bit_cast(f32x4, kraw[x]);
          }
          const bool in = 8 * x + 4 * g < width;
#pragma unroll
          for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_32x32x2f32(in ? k[e] : 0.0f, q[x][e], sc, 0, 0, 0);
        }
        if (st + 1 < steps) ask_keys(st + 1, next);
        const Pages after = pages_at(st + 2);
        float val[16][VW];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if constexpr (MX8) {
            const float s = scale_of(vscale[i]);
            const f32x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(vraw[i][0], s, false), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(vraw[i][0], s, true);
#pragma unroll
            for (int x = 0; x < VW; ++x) val[i][x] = x < 2 ? v0[x & 1] : v1[x & 1];
          } else {
#pragma unroll
            for (int x = 0; x < VW; ++x) val[i][x] = __uint_as_float(vraw[i][x]);
          }
        }
        if constexpr (VW == 3) {
          if (width % 3 != 0) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              val[i][0] = skip == 0 ? val[i][0] : skip == 1 ? val[i][1] : val[i][2];
              val[i][1] = skip == 0 ? val[i][1] : skip == 1 ? val[i][2] : 0.0f;
              val[i][2] = skip == 0 ? val[i][2] : 0.0f;
            }
          }
        }
        auto key_of = [&](int i) { return t0 + 8 * (i >> 2) + 4 * g + (i & 3); };
        auto sees = [&](int i) { return key_of(i) >= row_lo && key_of(i) < row_hi && now.entry[i >> 3] != -1; };
        bool odd = false;
        if (edge) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const bool there = i < 8 ? there0 : there1;
            sc[i] = !sees(i) ? -INFINITY : there ? sc[i] : __builtin_nanf("");
            const bool any = key_of(i) >= lo && key_of(i) < hi && there && VW * n < width;
#pragma unroll
            for (int x = 0; x < VW; ++x) {
              val[i][x] = any ? val[i][x] : 0.0f;
              odd = odd || !(fabsf(val[i][x]) < INFINITY);
            }
          }
        }
        float top = sc[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, sc[i]);
        top *= a.scale2;
        if (__any(top > m + MARGIN)) {
          float t = fmaxf(top, m);
          t = fmaxf(t, __shfl_xor(t, 32));
          const float f = exp2_(m - base_of(t));
          m = t;
          l *= f;
#pragma unroll
          for (int x = 0; x < VW; ++x) acc[x] *= f;
        }
        const float mb = base_of(m);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sc[i] = exp2_(fmaf(sc[i], a.scale2, -mb));
          l += sc[i];
        }
        if (edge && __any(odd)) {
          // (as in k_attend_rows: values that are not finite make NaN in the rows that see them, and are left out of the products)
#pragma unroll
          for (int x = 0; x < VW; ++x) {
            f32x16 hit;
#pragma unroll
            for (int i = 0; i < 16; ++i) hit[i] = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const bool bad = !(fabsf(val[i][x]) < INFINITY);
              hit = __builtin_amdgcn_mfma_f32_32x32x2f32(bad ? 1.0f : 0.0f, sees(i) ? 1.0f : 0.0f, hit, 0, 0, 0);
              val[i][x] = bad ? 0.0f : val[i][x];
            }
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (hit[i] != 0.0f) acc[x][i] = __builtin_nanf("");
          }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int x = 0; x < VW; ++x) acc[x] = __builtin_amdgcn_mfma_f32_32x32x2f32(val[i][x], sc[i], acc[x], 0, 0, 0);
        if (st + 1 < steps) ask_values(st + 1, next);
        now = next;
        next = after;
      }
      l += __shfl_xor(l, 32);
      // numbers VW (8 (i / 4) + 4 g + i % 4) + x of row n are in acc[x][i]
      if (shared) {
        const int64_t at = ((int64_t)seq * gridDim.x + blockIdx.x) * ROWS + 32 * wave + n, parts = (int64_t)a.s.n * gridDim.x * ROWS;
        float *o = a.part + at * DP;
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int x = 0; x < VW; ++x) o[VW * (8 * (i >> 2) + 4 * g + (i & 3)) + x] = acc[x][i];
        if (g == 0) {
          float *stat = a.part + parts * DP;
          stat[at] = m;
          stat[parts + at] = l;
        }
      } else if (out_row >= 0) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        float *o = reinterpret_cast<float *>(a.out) + out_row;
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
          for (int x = 0; x < VW; ++x) {
            const int d = VW * (8 * (i >> 2) + 4 * g + (i & 3)) + x;
            if (d < dim) o[d] = acc[x][i] * inv;
          }
      }
    }
  }
}

// ---- many rows: keys and values through the LDS ----
//
// A wave holds 32 rows, a workgroup four waves; a tile is 64 keys, keys and values of two tiles are in the LDS.  Pieces of 16 bytes go there straight from
// memory (numbers in 8 bits through registers, where they become bf16); which lane fetches a piece says where it lies: piece x of key t at place x ^ key_turn(t), so
// that the 16 keys whose pieces lanes read at a time meet all banks, and values in pairs of pieces at pair ^ value_turn(t).  S^T is made by products of
// 32 keys by 32 rows; values are read with the reads that turn a 4 by 16 block around, so that a lane gets four keys' numbers of one column.
//
// Two workgroups a compute unit: while waves of one are at their weights, those of the other may be at their products.  MI355X: prompt of 8192 tokens, 32 over 8 heads of
// 128, 570 - 620 us from card to card = 890 - 965 TFLOP/s (the vendor library's product of 8192^3 reaches 1280); without weights and maxima, in a copy that leaves them out, 538 of then 604 us,
// without loads too 462: products, their reads and one barrier a tile are three quarters of it.  Matrix cores are busy 40 % of the cycles, the vector unit 38 %.  Tried and slower:
// scores of the next tile beside this one's weights (spills), 64 rows a wave with one wave a SIMD (790 us), a higher priority at products (614), operands' reads ordered
// by hand (610).  16384 sequences of 50 tokens, 4 over 2 heads of 64: 340 us, 3.7 TB/s; a workgroup is one tile there, and its chain of loads (length, pages, keys) is
// what three workgroups a unit overlap.
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int TK = 64;  // keys of a tile
template <int DP> constexpr int tile_bytes() { return TK * DP * 2; }   // of keys, or of values
template <int DP> __device__ __forceinline__ int key_turn(int t) { return DP == 64 ? (t >> 1) & 7 : t & 15; }
template <int DP> __device__ __forceinline__ int value_turn(int t) { return DP == 64 ? (t >> 1) & 3 : t & 7; }
// place of a row's pair of pieces, before it is turned, and the other way round: of 32 lanes that read four rows' neighbouring pairs at a time, the second 16
// are half of the banks away from the first
template <int DP> __device__ __forceinline__ int place_of_pair(int x) {
  return DP == 64 ? (x >> 1 & 1) | (x & 1) << 1 : (x & 8) | (x >> 1 & 3) | (x & 1) << 2;
}
template <int DP> __device__ __forceinline__ int pair_at(int x) { return DP == 64 ? (x >> 1 & 1) | (x & 1) << 1 : (x & 8) | (x & 3) << 1 | (x >> 2 & 1); }

// A part of memory as the instructions with a range check see it: what lies behind its end reads as zeros.
__device__ __forceinline__ i32x4 part_of(const void *at, int bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)at;
  return i32x4{__builtin_amdgcn_readfirstlane((int)a), __builtin_amdgcn_readfirstlane((int)(a >> 32) & 0xffff), __builtin_amdgcn_readfirstlane(bytes), 0x00027000};
}
// 64 lanes fetch 16 bytes each, `lane_at` into the part, to consecutive places of the LDS from `to` on.  The compiler does not know
// of these loads: they are waited for by wait_loads.
__device__ __forceinline__ void to_lds16(const i32x4 &part, uint32_t lane_at, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(lane_at), "s"(part) : "memory");
}
template <int N> __device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// The sequence that comes k-th if those with most keys come first, which make the longest workgroups, of at most 64: every lane takes one of them
// and counts those before it.
__device__ __forceinline__ int kth_by_length(const AttendArgs &a, int k) {
  const int lane = (int)threadIdx.x & 63;
  float w = -1.0f;
  if (lane < a.s.n) {
    const Span sp = span_of(a.s, a.c.shift, lane);
    w = sp.rows > 0 ? (float)sp.length : 0.0f;
  }
  int before = 0;
  for (int j = 0; j < a.s.n; ++j) {
    const float o = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), j));
    before += o > w || (o == w && j < lane);
  }
  return __ffsll((unsigned long long)__ballot(lane < a.s.n && before == k)) - 1;
}

template <int FMT, int DP>
__global__ void __launch_bounds__(256, DP <= 64 ? 3 : DP <= 128 ? 2 : 1) k_attend_tile(const AttendArgs a) {
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ int odd_any[2];   // by tiles in turn: whether a value that only some rows see is not finite
  constexpr int TB = tile_bytes<DP>(), RB = DP * 2, ROWS = 128, NK = DP / 16, ND = DP / 32;
  constexpr int PIECES = DP / 8, TURNS = TK * PIECES / 256;  // pieces of 16 bytes in a row; of a tile, for every thread
  const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, g = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Cache &c = a.c;
  const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;

  // a thread's pieces: of the keys 16 wave .. 16 wave + 15 of a tile, whose page is one
  int from_k[TURNS], from_v[TURNS], zero = 0;
#pragma unroll
  for (int i = 0; i < TURNS; ++i) {
    const int e = i * 64 + lane, t = 16 * wave + e / PIECES, x = e % PIECES, last = (c.width >> 3) - 1;
    const int xk = x ^ key_turn<DP>(t), xv = pair_at<DP>(x >> 1 ^ value_turn<DP>(t)) << 1 | (x & 1);
    // (pieces behind a row's end are zeros: they lie behind what the loads see, or are fetched again and not used)
    if constexpr (FMT == VF_E4M3) {
      from_k[i] = e / PIECES * c.width + 8 * (xk < last ? xk : last);
      from_v[i] = e / PIECES * c.width + 8 * (xv < last ? xv : last);
      zero |= (xk > last) << i;
    } else {
      from_k[i] = xk > last ? 1 << 28 : e / PIECES * c.width + 8 * xk;
      from_v[i] = xv > last ? 1 << 28 : e / PIECES * c.width + 8 * xv;
    }
  }
  // places that a lane reads: of keys n (and 32 + n, a constant further), of values 4 g .. 4 g + 3 (and further ones)
  int at_k[NK], at_v[ND];
#pragma unroll
  for (int ks = 0; ks < NK; ++ks) at_k[ks] = n * RB + 16 * ((2 * ks + g) ^ key_turn<DP>(n));
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    const int t = 4 * g + ((lane & 15) >> 2), pair = 2 * d + ((lane >> 4) & 1);
    at_v[d] = TB + t * RB + 32 * (place_of_pair<DP>(pair) ^ value_turn<DP>(t)) + 8 * (lane & 3);
  }

  const Place place = place_of(a);
  const int head = place.head, split = place.split;
  for (int y = blockIdx.y; y < a.s.n; y += gridDim.y) {
    const int seq = a.by_length ? kth_by_length(a, y) : y;
    const Span sp = span_of(a.s, c.shift, seq);
    const int all = sp.rows * a.group.by;
    // (row blocks that see the most keys come first)
    for (int block = a.blocks - 1 - place.block; (int64_t)block * ROWS < all; block += a.blocks) {
      // (row blocks that the plan did not count on are not shared)
      const bool shared = a.splits > 1 && block < a.blocks;
      if (block >= a.blocks && split > 0) break;
      const int dim = anew(c.dim);
      const int w0 = block * ROWS, w1 = all - w0 > ROWS ? w0 + ROWS : all, r0 = w0 + 32 * wave, r1 = w1 - r0 > 32 ? r0 + 32 : w1;
      // what the workgroup's rows, and the wave's, see: all of [.., in), nothing outside
      int lo, hi, lo_in, hi_in, wlo = 0, whi = 0, wlo_in = 0, whi_in = 0;
      seen_by(a, sp, over(a.group, w0), lo, hi_in);
      seen_by(a, sp, over(a.group, w1 - 1), lo_in, hi);
      if (r0 < r1) {
        seen_by(a, sp, over(a.group, r0), wlo, whi_in);
        seen_by(a, sp, over(a.group, r1 - 1), wlo_in, whi);
      }
      int row_lo = 0, row_hi = 0;
      const uint16_t *q_row = nullptr;
      int64_t out_row = -1;
      const int r = r0 + n;
      if (r < r1) {
        const int i = over(a.group, r), h = head * a.group.by + r - i * a.group.by;
        seen_by(a, sp, i, row_lo, row_hi);
        q_row = reinterpret_cast<const uint16_t *>(a.q) + (sp.first + i) * a.ld_q + (int64_t)h * dim;
        out_row = (sp.first + i) * a.ld_out + (int64_t)h * dim;
      }
      const int from = lo & ~(TK - 1);
      int tiles = hi > from ? (hi - from + TK - 1) / TK : 0, s0 = 0;
      if (shared) {
        const int each = (tiles + a.splits - 1) / a.splits;
        s0 = (int)((int64_t)each * split < tiles ? each * split : tiles);
        tiles = tiles - s0 < each ? tiles : s0 + each;
      }
      // The wave's share of a tile on its way: straight to the LDS, or 8-bit codes and scales in registers.
      uint2 raw_k[FMT == VF_E4M3 ? TURNS : 1], raw_v[FMT == VF_E4M3 ? TURNS : 1];
      uint32_t sc_k[FMT == VF_E4M3 ? TURNS : 1], sc_v[FMT == VF_E4M3 ? TURNS : 1];
      // Pages of a tile's blocks of 16 keys, asked for two tiles ahead: the wave's own block's, and bits of those that are there, and of
      // entries that are no page and not -1.
      constexpr int ALL = (1 << (TK / 16)) - 1;
      int asked[TK / 16];
      auto ask_pages = [&](int st) {
#pragma unroll
        for (int x = 0; x < TK / 16; ++x) asked[x] = st < tiles ? entry_of(a.s, c.shift, seq, from + st * TK + 16 * x) : -1;
      };
      struct Bits { int own, there, wrong; };
      auto bits_of = [&]() {
        Bits b = {-1, 0, 0};
#pragma unroll
        for (int x = 0; x < TK / 16; ++x) {
          const int e = __builtin_amdgcn_readfirstlane(asked[x]);
          b.there |= ((unsigned)e < (unsigned)c.pages) << x;
          b.wrong |= ((unsigned)e >= (unsigned)c.pages && e != -1) << x;
          b.own = x == wave ? e : b.own;
        }
        return b;
      };
      auto fetch = [&](int st, int entry) {
        const int page = (unsigned)entry < (unsigned)c.pages ? entry : 0;  // (what is fetched there is not used)
        const int64_t row = row_of(c, page, head, from + st * TK + 16 * wave);
        if constexpr (FMT == VF_E4M3) {
          const uint8_t *k = reinterpret_cast<const uint8_t *>(c.k) + row * c.width, *v = reinterpret_cast<const uint8_t *>(c.v) + row * c.width;
          const uint8_t *ks = c.ks + row * c.kb, *vs = c.vs + row * c.kb;
#pragma unroll
          for (int i = 0; i < TURNS; ++i) {
            raw_k[i] = *reinterpret_cast<const uint2 *>(k + from_k[i]);
            raw_v[i] = *reinterpret_cast<const uint2 *>(v + from_v[i]);
            sc_k[i] = ks[from_k[i] >> 5];   // (a row's scales are a 32nd of its width)
            sc_v[i] = vs[from_v[i] >> 5];
          }
        } else {
          const i32x4 pk = part_of(reinterpret_cast<const uint16_t *>(c.k) + row * c.width, 32 * c.width);
          const i32x4 pv = part_of(reinterpret_cast<const uint16_t *>(c.v) + row * c.width, 32 * c.width);
          const uint32_t to = base + (uint32_t)((st & 1) * 2 * TB) + (uint32_t)wave * (16 * RB);
#pragma unroll
          for (int i = 0; i < TURNS; ++i) to_lds16(pk, 2 * (uint32_t)from_k[i], to + i * 1024);
#pragma unroll
          for (int i = 0; i < TURNS; ++i) to_lds16(pv, 2 * (uint32_t)from_v[i], to + TB + i * 1024);
        }
      };
      auto put = [&](int st) {  // 8 bits: what has arrived becomes bf16 in the LDS
        if constexpr (FMT == VF_E4M3) {
          uint8_t *to = lds + (st & 1) * 2 * TB + wave * (16 * RB) + lane * 16;
#pragma unroll
          for (int i = 0; i < TURNS; ++i) {
            if (zero >> i & 1) {
              raw_k[i] = make_uint2(0, 0);
              sc_k[i] = 127;
            }
            const float fk = scale_of((uint8_t)sc_k[i]), fv = scale_of((uint8_t)sc_v[i]);
            *reinterpret_cast<uint4 *>(to + i * 1024) = make_uint4(cvt2(raw_k[i].x, fk, false), cvt2(raw_k[i].x, fk, true), cvt2(raw_k[i].y, fk, false), cvt2(raw_k[i].y, fk, true));
            *reinterpret_cast<uint4 *>(to + TB + i * 1024) = make_uint4(cvt2(raw_v[i].x, fv, false), cvt2(raw_v[i].x, fv, true), cvt2(raw_v[i].y, fv, false), cvt2(raw_v[i].y, fv, true));
          }
        }
      };
      ask_pages(s0);
      Bits now = bits_of();
      __syncthreads();  // (the row block before is done with the LDS)
      if (tid < 2) odd_any[tid] = 0;
      if (s0 < tiles) fetch(s0, now.own);
      ask_pages(s0 + 1);

      // queries as operands
      uint4 q16[NK];
#pragma unroll
      for (int ks = 0; ks < NK; ++ks) {
        const int d = 16 * ks + 8 * g, left = q_row ? dim - d : 0;
        raw8<uint16_t> w = {};
        if (left > 0) fetch8(q_row + d, left, w);
        q16[ks] = make_uint4(w.w[0], w.w[1], w.w[2], w.w[3]);
      }
      f32x16 acc[ND];
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[d][i] = 0.0f;
      float m = -INFINITY, l = 0.0f;

      for (int st = s0; st < tiles; ++st) {
        const int t0 = from + st * TK;
        if constexpr (FMT == VF_E4M3) put(st);
        else wait_loads<0>();
        __syncthreads();  // the tile is there, and nobody reads the one before any more
        const int there = now.there, wrong = now.wrong;
        if (st + 1 < tiles) {
          now = bits_of();
          fetch(st + 1, now.own);
          ask_pages(st + 2);
        }
        uint8_t *tile = lds + (st & 1) * 2 * TB;
        if (tid == 0) odd_any[~st & 1] = 0;
        if (t0 < lo_in || t0 + TK > hi_in || there != ALL) {
          // Values that no row sees become zeros.  Of others that are not finite the rows that see them get NaN; then they are zeros too, so that
          // they reach no other row.
          bool bad = false;
#pragma unroll 1
          for (int e = tid; e < TK * PIECES; e += 256) {
            const int t = t0 + e / PIECES;
            uint4 *at = reinterpret_cast<uint4 *>(tile + TB) + e;
            if (t < lo || t >= hi || !(there >> (e / PIECES / 16) & 1)) *at = make_uint4(0, 0, 0, 0);
            else bad = bad || not_finite(at->x) || not_finite(at->y) || not_finite(at->z) || not_finite(at->w);
          }
          if (bad) odd_any[st & 1] = 1;
          __syncthreads();
          if (odd_any[st & 1]) {
#pragma unroll 1
            for (int t = 0; t < TK; ++t) {
              if (t0 + t < row_lo || t0 + t >= row_hi) continue;
#pragma unroll
              for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                  const int piece = 4 * d + (i >> 2);
                  const uint2 w = *reinterpret_cast<const uint2 *>(tile + TB + t * RB + 32 * (place_of_pair<DP>(piece >> 1) ^ value_turn<DP>(t)) + 16 * (piece & 1) + 8 * g);
                  if ((w.x & 0x7f80u) == 0x7f80u) acc[d][i] = __builtin_nanf("");
                  if ((w.x & 0x7f800000u) == 0x7f800000u) acc[d][i + 1] = __builtin_nanf("");
                  if ((w.y & 0x7f80u) == 0x7f80u) acc[d][i + 2] = __builtin_nanf("");
                  if ((w.y & 0x7f800000u) == 0x7f800000u) acc[d][i + 3] = __builtin_nanf("");
                }
            }
            __syncthreads();
#pragma unroll 1
            for (int e = tid; e < TK * PIECES; e += 256) {
              uint4 *at = reinterpret_cast<uint4 *>(tile + TB) + e;
              *at = make_uint4(finite_of(at->x), finite_of(at->y), finite_of(at->z), finite_of(at->w));
            }
            __syncthreads();
          }
        }
        if (t0 >= whi || t0 + TK <= wlo) continue;  // (nothing for this wave's rows)

        f32x16 sc[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[b][i] = 0.0f;
#pragma unroll
        for (int ks = 0; ks < NK; ++ks)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const uint4 k = *reinterpret_cast<const uint4 *>(tile + at_k[ks] + b * 32 * RB);
            sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q16[ks]), sc[b], 0, 0, 0);
          }
        if (there != ALL) {
#pragma unroll
          for (int x = 0; x < TK / 16; ++x) {
            if (there >> x & 1) continue;
            const float no = wrong >> x & 1 ? __builtin_nanf("") : -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) sc[x >> 1][8 * (x & 1) + i] = no;
          }
        }
        if (t0 < wlo_in || t0 + TK > whi_in) {
          const int rel = t0 + 4 * g - row_lo, len = row_hi - row_lo;  // (key 32 b + 8 (i / 4) + 4 g + i % 4 is in register i of block b)
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[b][i] = (unsigned)(rel + 32 * b + 8 * (i >> 2) + (i & 3)) < (unsigned)len ? sc[b][i] : -INFINITY;
        }
        float top = sc[0][0];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[b][i]);
        top *= a.scale2;
        if (__any(top > m + MARGIN)) {
          float t = fmaxf(top, m);
          t = fmaxf(t, __shfl_xor(t, 32));
          const float f = exp2_(m - base_of(t));
          m = t;
          l *= f;
#pragma unroll
          for (int d = 0; d < ND; ++d) acc[d] *= f;
        }
        const float mb = base_of(m);
        bf16x8 p[4];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            sc[b][i] = exp2_(fmaf(sc[b][i], a.scale2, -mb));
            l += sc[b][i];
          }
#pragma unroll
          for (int x = 0; x < 2; ++x)
            p[2 * b + x] = as_bf16x8(pack2(sc[b][8 * x], sc[b][8 * x + 1]), pack2(sc[b][8 * x + 2], sc[b][8 * x + 3]), pack2(sc[b][8 * x + 4], sc[b][8 * x + 5]),
                                     pack2(sc[b][8 * x + 6], sc[b][8 * x + 7]));
        }
        auto values = [&](int d, int x) {  // of keys 16 x + 4 g .. + 3 and 16 x + 8 + 4 g .. + 3, column 32 d + n
          const uint8_t *at = tile + at_v[d] + x * 16 * RB;
          const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at));
          const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + 8 * RB));
          const uint2 w0 = __builtin_bit_cast(uint2, v0), w1 = __builtin_bit_cast(uint2, v1);
          return make_uint4(w0.x, w0.y, w1.x, w1.y);
        };
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int d = 0; d < ND; ++d) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, values(d, x)), p[x], acc[d], 0, 0, 0);
      }
      l += __shfl_xor(l, 32);
      // numbers 32 d + 8 (i / 4) + 4 g + i % 4 of row n are in acc[d][i]
      if (shared) {
        const int64_t at = ((int64_t)seq * gridDim.x + blockIdx.x) * ROWS + 32 * wave + n, parts = (int64_t)a.s.n * gridDim.x * ROWS;
        float *o = a.part + at * DP;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<f32x4 *>(o + 32 * d + 2 * i + 4 * g) = f32x4{acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]};
        if (g == 0) {
          float *stat = a.part + parts * DP;
          stat[at] = m;
          stat[parts + at] = l;
        }
      } else if (out_row >= 0) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        uint16_t *o = reinterpret_cast<uint16_t *>(a.out) + out_row;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const int at = 32 * d + 2 * i + 4 * g, left = dim - at;
            float v[8] = {};
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[d][i + e] * inv;
            if (left >= 4) {
              typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));
              *reinterpret_cast<u32x2 *>(o + at) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
            } else if (left > 0) {
              store_upto8(o + at, left, v);
            }
          }
      }
    }
  }
}

// Sorts sequences by their first page and cuts them into groups of up to `most` that have the same: order[n] = (sequence, its length), items[n + 1] = first
// places of the groups (behind the last one n).  A sequence without keys is a group of its own.  One workgroup, a bitonic network of 64-bit keys (page,
// sequence), key 1024 r + t in register r of thread t: neighbours up to 32 apart are exchanged between lanes, up to 512 through the LDS.
// MI355X: 1024 sequences 10 us.
constexpr int MAX_GROUPED = 4096;
template <int PER>
__global__ void __launch_bounds__(1024) k_attend_group(const AttendArgs a, int2 *order, int32_t *items, int most) {
  __shared__ uint64_t key[1024 * PER];
  __shared__ int total[16];
  const int n = a.s.n, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint64_t mine[PER];
#pragma unroll
  for (int r = 0; r < PER; ++r) {
    const int i = 1024 * r + tid;
    mine[r] = ~0ull;
    if (i < n) {
      const Span sp = span_of(a.s, a.c.shift, i);
      const int e = sp.length > 0 ? entry_of(a.s, a.c.shift, i, 0) : -1;
      mine[r] = (uint64_t)((unsigned)e < (unsigned)a.c.pages ? (uint32_t)e : 0x80000000u + (uint32_t)i) << 32 | (uint32_t)i;
    }
  }
  // exchanges key i with key i + d, or i - d: the one with bit d clear keeps the smaller where the run of `width` that both are in ascends
  auto keep = [&](uint64_t &v, uint64_t o, int i, int d, int width) {
    const bool smaller = ((i & d) == 0) == ((i & width) == 0);
    if ((o < v) == smaller) v = o;
  };
#pragma unroll
  for (int width = 2; width <= 1024 * PER; width *= 2) {
#pragma unroll
    for (int d = 1024 * PER / 2; d > 0; d /= 2) {
      if (d >= width) continue;
      if (d >= 1024) {
#pragma unroll
        for (int r = 0; r < PER; ++r)
          if ((r & (d / 1024)) == 0) {
            const uint64_t u = mine[r], v = mine[r | (d / 1024)];
            keep(mine[r], v, 1024 * r + tid, d, width);
            keep(mine[r | (d / 1024)], u, 1024 * (r | (d / 1024)) + tid, d, width);
          }
      } else if (d >= 64) {
        __syncthreads();
#pragma unroll
        for (int r = 0; r < PER; ++r) key[1024 * r + tid] = mine[r];
        __syncthreads();
#pragma unroll
        for (int r = 0; r < PER; ++r) keep(mine[r], key[1024 * r + (tid ^ d)], 1024 * r + tid, d, width);
      } else {
#pragma unroll
        for (int r = 0; r < PER; ++r) {
          const uint32_t lo = (uint32_t)__shfl_xor((int)(uint32_t)mine[r], d), hi = (uint32_t)__shfl_xor((int)(uint32_t)(mine[r] >> 32), d);
          keep(mine[r], (uint64_t)hi << 32 | lo, 1024 * r + tid, d, width);
        }
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < PER; ++r) key[1024 * r + tid] = mine[r];
  __syncthreads();
  // places in order, 1024 at a time: where its run of equal pages begins is the largest beginning up to a place, and a group begins every
  // `most` places of a run
  int run_before = 0, items_before = 0;
#pragma unroll
  for (int r = 0; r < PER; ++r) {
    const int i = 1024 * r + tid;
    int run = i == 0 || (uint32_t)(mine[r] >> 32) != (uint32_t)(key[i > 0 ? i - 1 : 0] >> 32) ? i : -1;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int o = __shfl_up(run, x);
      run = lane >= x && o > run ? o : run;
    }
    if (lane == 63) total[wave] = run;
    __syncthreads();
    for (int w = 0; w < 16; ++w) {
      const int o = total[w];
      if (w < wave) run = o > run ? o : run;
    }
    run = run_before > run ? run_before : run;
    __syncthreads();
    const bool begins = i < n && (i - run) % most == 0;
    const unsigned long long those = __ballot(begins);
    if (lane == 63) total[wave] = __popcll(those);
    if (tid == 1023) key[0] = (uint64_t)run;   // (its first place has been looked at)
    __syncthreads();
    int at = items_before + __popcll(those & ((1ull << lane) - 1));
    for (int w = 0; w < 16; ++w) {
      const int o = total[w];
      at += w < wave ? o : 0;
      items_before += o;
    }
    run_before = (int)key[0];
    if (begins) items[at] = i;
    if (i < n) {
      const int s = (int)(uint32_t)mine[r];
      order[i] = make_int2(s, span_of(a.s, a.c.shift, s).length);
    }
    __syncthreads();
  }
  for (int i = items_before + tid; i <= n; i += 1024) items[i] = n;
}

// Joins the parts of row blocks that several workgroups have shared: a wave a row.
template <typename T, int DP>
__global__ void __launch_bounds__(256) k_attend_join(const AttendArgs a, int rows, bool last_first) {
  const int lane = (int)threadIdx.x & 63;
  const Cache &c = a.c;
  const int64_t blocks = (int64_t)a.s.n * a.blocks * c.heads, items = blocks * rows, parts = items * a.splits;
  for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items; item += (int64_t)gridDim.x * 4) {
    const int ub = (int)(item / rows);   // (sequence, row block, head of the cache), heads fastest
    const int row = (int)(item - (int64_t)ub * rows), sb = ub / c.heads, head = ub - sb * c.heads;
    const int seq = sb / a.blocks, place = sb - seq * a.blocks, block = last_first ? a.blocks - 1 - place : place;
    const Span sp = span_of(a.s, c.shift, seq);
    const int r = block * rows + row;
    if (r >= sp.rows * a.group.by) continue;
    const float *stat = a.part + parts * DP;
    auto at_of = [&](int k) { return ((int64_t)(sb * a.splits + k) * c.heads + head) * rows + row; };
    float top = -INFINITY;
    for (int k = lane; k < a.splits; k += 64) top = fmaxf(top, stat[at_of(k)]);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x));
    float l = 0.0f, o[(DP + 63) / 64] = {};
    for (int k = 0; k < a.splits; ++k) {
      const int64_t at = at_of(k);
      const float f = weight_of(stat[at], top);
      l += f * stat[parts + at];
#pragma unroll
      for (int x = 0; x < (DP + 63) / 64; ++x)
        if (64 * x + lane < DP) o[x] += f * a.part[at * DP + 64 * x + lane];
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int i = over(a.group, r), h = head * a.group.by + r - i * a.group.by;
    T *to = reinterpret_cast<T *>(a.out) + (sp.first + i) * a.ld_out + (int64_t)h * c.dim;
#pragma unroll
    for (int x = 0; x < (DP + 63) / 64; ++x)
      if (64 * x + lane < c.dim) store1(to + 64 * x + lane, o[x] * inv);
  }
}

// Row blocks that a launch counts on: those of the longest sequence, as long as the grid stays below 2^22 workgroups a sequence.
int blocks_of(int64_t longest, int rows, int heads) {
  const int64_t n = (longest + rows - 1) / rows, most = ((1 << 22) + heads - 1) / heads;
  return (int)(n < 1 ? 1 : n < most ? n : most);
}

// (about 70 us at the memory's rate; below, the 10 us that finding the groups takes are more than what sharing saves)
// Whether rows do share pages the host does not know.  MI355X, us, in groups / each by itself: 1024 rows of 64 prefixes of 501 keys, 16 over 4 heads of 64, 52 / 57; 256 of 16 prefixes of
// 2001, 32 over 8 heads of 128, 106 / 150.  What the rule costs where nothing is shared: 1000 rows of 501 keys 133 / 99, 256 of 2001 373 / 362, 64 of 4001, 8 heads of 128, 193 / 182, 4000 of
// 101, 16 over 8 heads of 64, 364 / 174; and where there are few groups, whose keys no more workgroups share than before, 64 rows of one prefix of 4001 113 / 80; or short
// prefixes, 4000 of 250 prefixes of 101 184 / 117.
constexpr int64_t GROUP_BYTES = 384 << 20;

template <typename T, int FMT, int DP>
int launch_rows(vf_ctx *c, AttendArgs &a, int64_t longest_kv) {
  constexpr int STEP = Shape<T, FMT, DP>::STEP;
  const int64_t longest = (int64_t)a.longest * a.group.by;
  // (bf16 comes here with up to 16 rows only)
  // (and fp32 with more, see launch)
  const bool along = sizeof(T) == 4 && longest > 16;
  const int rows = along ? 64 : 16;
  a.blocks = blocks_of(longest, rows, a.c.heads);
  // Workgroups share the keys of a row block where there would be fewer than run at a time, as long as every wave keeps some steps.
  const int64_t units = (int64_t)a.s.n * a.blocks * a.c.heads, steps = (longest_kv + STEP - 1) / STEP, most = along ? steps / 8 : (steps + 31) / 32;
  int64_t splits = (512 + units - 1) / units;
  if (splits > most) splits = most;
  if (splits > 512) splits = 512;
  if (splits < 1) splits = 1;
  // Single tokens whose keys and values take the memory longer than it takes to find out which sequences share pages
  const int most_members = 16 / a.group.by;
  const int64_t bytes = (int64_t)a.s.n * longest_kv * a.c.heads * a.c.width * 2 * (int64_t)sizeof(typename kv_elem<FMT>::type);
  bool grouped = !a.s.offsets && a.s.each == 1 && most_members > 1 && a.s.n >= 16 && a.s.n <= MAX_GROUPED && bytes >= GROUP_BYTES;
  const size_t part_bytes = splits > 1 ? (size_t)(units * splits * rows) * (DP + 2) * sizeof(float) : 0;
  const size_t group_bytes = grouped ? (size_t)a.s.n * sizeof(int2) + ((size_t)a.s.n + 1) * sizeof(int32_t) : 0;
  if (part_bytes + group_bytes > 0) {
    uint8_t *scratch = reinterpret_cast<uint8_t *>(vfk_ops_scratch(c, part_bytes + group_bytes));
    if (!scratch) {
      splits = 1;
      grouped = false;
    }
    a.part = reinterpret_cast<float *>(scratch);
    a.order = reinterpret_cast<int2 *>(scratch + part_bytes);
    a.items = reinterpret_cast<const int32_t *>(a.order + a.s.n);
  }
  a.splits = (int)splits;
  const dim3 grid((unsigned)(a.blocks * a.c.heads * a.splits), (unsigned)(a.s.n < MAX_Y ? a.s.n : MAX_Y));
  if constexpr (sizeof(T) == 4) {
    if (along) k_attend_rows<T, FMT, DP, 1, ROWWISE><<<grid, 256, 0, c->stream>>>(a);
  }
  if (grouped) {
    int2 *order = const_cast<int2 *>(a.order);
    int32_t *items = const_cast<int32_t *>(a.items);
    if (a.s.n <= 1024) k_attend_group<1><<<1, 1024, 0, c->stream>>>(a, order, items, most_members);
    else k_attend_group<4><<<1, 1024, 0, c->stream>>>(a, order, items, most_members);
    VF_HIP(c, hipGetLastError());
    k_attend_rows<T, FMT, DP, 1, GROUP><<<grid, 256, 0, c->stream>>>(a);
  } else if (!along) {
    if (units >= 2048 && a.s.n >= 4) {
      const int by_four = (a.s.n + 3) / 4;
      k_attend_rows<T, FMT, DP, 1, SEQWISE><<<dim3(grid.x, by_four < MAX_Y ? by_four : MAX_Y), 256, 0, c->stream>>>(a);
    } else {
      // (with one workgroup a compute unit there are registers for eight waves, up to 128 numbers a head)
      constexpr int FEW = DP <= 128 ? SHARE8 : SHARE;
      if (DP <= 128 && units * splits <= 256 && steps > 4) k_attend_rows<T, FMT, DP, 1, FEW><<<grid, 512, 0, c->stream>>>(a);
      else k_attend_rows<T, FMT, DP, 1, SHARE><<<grid, 256, 0, c->stream>>>(a);
    }
  }
  VF_HIP(c, hipGetLastError());
  if (splits > 1) {
    const int64_t items = (units * rows + 3) / 4;
    k_attend_join<T, DP><<<(unsigned)(items < 4096 ? items : 4096), 256, 0, c->stream>>>(a, rows, false);
    VF_HIP(c, hipGetLastError());
  }
  return VF_OK;
}

template <int FMT, int DP>
int launch_tile(vf_ctx *c, AttendArgs &a, int64_t longest_kv) {
  constexpr int ROWS = 128, LDS = 4 * tile_bytes<DP>(), AT_ONCE = DP <= 128 ? 512 : 256;
  const int64_t longest = (int64_t)a.longest * a.group.by;
  a.blocks = blocks_of(longest, ROWS, a.c.heads);
  const int64_t units = (int64_t)a.s.n * a.blocks * a.c.heads, most = (longest_kv + TK - 1) / TK / 4;
  int64_t splits = (AT_ONCE + units - 1) / units;
  if (splits > most) splits = most;
  if (splits < 1) splits = 1;
  if (splits > 1) {
    a.part = reinterpret_cast<float *>(vfk_ops_scratch(c, (size_t)(units * splits * ROWS) * (DP + 2) * sizeof(float)));
    if (!a.part) splits = 1;
  }
  a.splits = (int)splits;
  // (where workgroups come in several rounds, long ones that come last would be waited for; with many sequences they are a small part)
  a.by_length = a.s.n > 1 && a.s.n <= 64 && units * splits > AT_ONCE;
  const dim3 grid((unsigned)(a.blocks * a.c.heads * a.splits), (unsigned)(a.s.n < MAX_Y ? a.s.n : MAX_Y));
  VF_HIP(c, hipFuncSetAttribute(reinterpret_cast<const void *>(&k_attend_tile<FMT, DP>), hipFuncAttributeMaxDynamicSharedMemorySize, LDS));
  k_attend_tile<FMT, DP><<<grid, 256, LDS, c->stream>>>(a);
  VF_HIP(c, hipGetLastError());
  if (splits > 1) {
    const int64_t items = (units * ROWS + 3) / 4;
    k_attend_join<uint16_t, DP><<<(unsigned)(items < 4096 ? items : 4096), 256, 0, c->stream>>>(a, ROWS, true);
    VF_HIP(c, hipGetLastError());
  }
  return VF_OK;
}

// Rows of a workgroup are four waves' of 32.
template <int FMT, int DP>
int launch_wide(vf_ctx *c, AttendArgs &a, int64_t longest_kv) {
  constexpr int ROWS = 128, AT_ONCE = DP <= 64 ? 512 : 256;
  const int64_t longest = (int64_t)a.longest * a.group.by;
  a.blocks = blocks_of(longest, ROWS, a.c.heads);
  const int64_t units = (int64_t)a.s.n * a.blocks * a.c.heads, most = (longest_kv + 31) / 32 / 8;
  int64_t splits = (AT_ONCE + units - 1) / units;
  if (splits > most) splits = most;
  if (splits < 1) splits = 1;
  if (splits > 1) {
    a.part = reinterpret_cast<float *>(vfk_ops_scratch(c, (size_t)(units * splits * ROWS) * (DP + 2) * sizeof(float)));
    if (!a.part) splits = 1;
  }
  a.splits = (int)splits;
  const dim3 grid((unsigned)(a.blocks * a.c.heads * a.splits), (unsigned)(a.s.n < MAX_Y ? a.s.n : MAX_Y));
  k_attend_wide<FMT, DP><<<grid, 256, 0, c->stream>>>(a);
  VF_HIP(c, hipGetLastError());
  if (splits > 1) {
    const int64_t items = (units * ROWS + 3) / 4;
    k_attend_join<float, DP><<<(unsigned)(items < 4096 ? items : 4096), 256, 0, c->stream>>>(a, ROWS, true);
    VF_HIP(c, hipGetLastError());
  }
  return VF_OK;
}

template <typename T, int FMT>
int launch(vf_ctx *c, AttendArgs &a, int64_t longest_kv) {
  if constexpr (sizeof(T) == 2) {
    if ((int64_t)a.longest * a.group.by > 16) {
      if (a.c.dim <= 64) return launch_tile<FMT, 64>(c, a, longest_kv);
      if (a.c.dim <= 128) return launch_tile<FMT, 128>(c, a, longest_kv);
      return launch_tile<FMT, 256>(c, a, longest_kv);
    }
  }
  if constexpr (sizeof(T) == 4) {
    // Rows of 32 a wave fetch half as much as rows of 16, but see more keys that are not all theirs, and there are fewer waves.  MI355X, us, 16 / 32:
    // 37 sequences of up to 300 rows with a window of 100, heads of 40, 46 / 64; 312 of 87 behind 48, heads of 32, 129 / 135; a prompt of 2048, 32 heads of 128, 576 /
    // 390, of 64 295 / 253.
    if ((int64_t)a.longest * a.group.by > 16 && a.c.dim <= 128 && longest_kv >= 512) {
      if (a.c.dim <= 32) return launch_wide<FMT, 32>(c, a, longest_kv);
      if (a.c.dim <= 64) return launch_wide<FMT, 64>(c, a, longest_kv);
      if (FMT == VF_FP32 && a.c.dim <= 96) return launch_wide<FMT, FMT == VF_FP32 ? 96 : 128>(c, a, longest_kv);
      return launch_wide<FMT, 128>(c, a, longest_kv);
    }
  }
  if (a.c.dim <= 32) return launch_rows<T, FMT, 32>(c, a, longest_kv);
  if (a.c.dim <= 64) return launch_rows<T, FMT, 64>(c, a, longest_kv);
  if (a.c.dim <= 128) return launch_rows<T, FMT, 128>(c, a, longest_kv);
  return launch_rows<T, FMT, 256>(c, a, longest_kv);
}

}  // namespace

int vfk_kv_attend(vf_ctx *c, const vf_kv_call &call, int heads, const void *q, int64_t ld_q, bool causal, int window, float scale, int64_t longest_kv,
                  void *out, int64_t ld_out) {
  if (call.seqs->n_seq == 0 || call.seqs->tokens == 0) return VF_OK;
  AttendArgs a = {};
  a.c = cache_of(call.kv);
  a.s = seqs_of(call.seqs);
  a.q = q; a.out = out; a.ld_q = ld_q; a.ld_out = ld_out;
  // (scores that a row does not see are -inf and have to stay it: the smallest number there is does for 0, as it takes every finite score below 1e-6)
  a.scale2 = scale * LOG2E > 0.0f ? scale * LOG2E : 1.4e-45f;
  a.group = divisor_of(heads / call.kv->kv_heads);
  a.causal = causal; a.window = window;
  a.longest = (int)longest_of(call.seqs);
  const int64_t most = (int64_t)call.seqs->max_pages * call.kv->page;
  if (longest_kv > most) longest_kv = most;
  if (window > 0 && longest_kv > (int64_t)window + a.longest) longest_kv = (int64_t)window + a.longest;   // (what a sequence's rows see)
  if (call.type == VF_BF16) return call.kv->format == VF_E4M3 ? launch<uint16_t, VF_E4M3>(c, a, longest_kv) : launch<uint16_t, VF_BF16>(c, a, longest_kv);
  return call.kv->format == VF_E4M3 ? launch<float, VF_E4M3>(c, a, longest_kv) : launch<float, VF_FP32>(c, a, longest_kv);
}
