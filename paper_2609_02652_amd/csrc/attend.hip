// Attention of new tokens over the paged key/value cache for gfx950.
//
// Both products run transposed on the matrix cores: Sᵀ = K Qᵀ, then Oᵀ = Vᵀ Pᵀ,
// in 16×16×32 products.  A lane then holds, for one query (its column), the
// scores of the tokens whose values it feeds to the second product, so weights
// go from one product to the next in the lane's own registers; the maximum and
// the sum of a query are two exchanges across the wave's four quarters; and the
// rescaling of Oᵀ is by one factor a lane.  Keys are rows as they lie (sixteen
// bytes a lane); row m of the u-th key tile is token I·(m / 4) + 4u + m % 4 of
// the step, so that quarter g of the wave ends up with the scores of tokens
// I·g .. I·g + I − 1, the run of tokens that sixteen bytes of the value pages
// hold.  Both operands come from memory straight into the registers that the
// products read.
//
// One pass.  A query keeps a base (of two's powers), the sum l of its weights
// 2^(s − base) and O; the base follows the largest score seen, but only once that
// is far enough above it, and l and O are scaled to it.  The second product takes
// weights rounded to its type: with a second number for what that leaves off, out is as
// good as f32 weights make it (64 sequences of up to 8000 bf16 keys: off by 0.17%, 0.23%
// with one), but a 4096-token prompt takes 235 us (178), 4 x 999 tokens over int8 1052
// (819), 16 x 5 28.7 (27.3), and rows would depend on the kernel that takes them if only
// stream_kernel, which mostly waits for memory, did it.  In f16 the base stays 2^11 to 2^15 under the
// largest score: the large weights fill f16's range from the top, so that the many
// small ones of a long context are numbers too.  Rows are (new token, query head of
// the group) of one sequence and cache head, so a group's heads share every key read.
//
// 8-bit codes become f16, which holds all of them; a key's scale multiplies its
// scores, a value's its weight in the second product.  The base is then that of
// weight times scale, log2 of the largest scale higher, so that the products'
// f16 weights stay in range whatever the scales are; the scale of a weight in l
// is the same, so out = O / l as before.  bf16 queries over 8-bit codes become
// f16 times a power of two a row.

#include "kv_device.h"

#include <algorithm>
#include <cmath>

namespace leech {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.69314718055994531f;

struct AttendArgs {
  CacheShape c;
  const uint8_t *ck, *cv;
  const float *sk, *sv;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  int64_t q_token, q_head, o_token, o_head, table_stride;
  const int32_t *q_start, *kv_len, *table;
  int64_t T, pages;
  int32_t type, q_heads, group, B, table_pages, max_new, causal, window;
  float scale;                // times log2 e, its magnitude; never 0 (2^-126 stands for it)
  uint32_t flip;              // sign bits that a negative scale puts on the queries
  // how the work is cut (see the plan)
  int32_t block_rows, log_step, min_steps, whole_few, whole_many, units, split;
  int32_t over, upto;         // sequences of over < rows <= upto are this launch's
  int32_t slices;             // workgroups that join a tile's rows
  int32_t direct;             // unit b is sequence b, of one tile and part
  float target;
  float *part_o, *part_ml;    // [head][unit][row][dim], [head][unit][row][2]
};

// ------------------------------------------------------------------- the plan
// A sequence's rows are cut in tiles of block_rows, its keys in steps of
// 2^log_step tokens, and the steps that a sequence's rows see in equal parts, so
// many that all parts of all sequences together come to about `target`
// workgroups of equal work (never less than min_steps a part).  What a second
// launch does not pay for stays whole: whole_few steps, or whole_many where there
// are a quarter of `target` workgroups already.  A unit is a part
// of a tile; units are numbered sequence by sequence, tile by tile.  Every wave
// works the numbering out for itself, a lane a sequence.
struct Sequence {
  int64_t first;              // row of q of its first new token
  int32_t n, rows, tiles, len, steps, parts;
  int32_t at;                 // what was looked for, counted from the sequence's first
};

__device__ __forceinline__ int64_t start_of(const AttendArgs& a, int b) {
  const int64_t s = a.q_start ? a.q_start[b] : b;
  return s < 0 ? 0 : s > a.T ? a.T : s;
}

__device__ __forceinline__ Sequence sequence(const AttendArgs& a, int b) {
  Sequence s = {0, 0, 0, 0, 0, 0, 1, 0};
  if (b >= a.B) return s;
  s.first = start_of(a, b);
  const int64_t n = start_of(a, b + 1) - s.first;
  s.n = n < 0 ? 0 : (int32_t)n;
  s.rows = (s.n < a.max_new ? s.n : a.max_new) * a.group;
  if (s.rows <= a.over || s.rows > a.upto) return s;
  s.tiles = (s.rows + a.block_rows - 1) / a.block_rows;
  const int64_t room = (int64_t)a.table_pages << a.c.log_page;
  const int32_t len = a.kv_len[b];
  s.len = len < 0 ? 0 : len > room ? (int32_t)room : len;
  int64_t lo = a.window ? (int64_t)s.len - s.n - a.window + 1 : 0;
  if (lo < 0) lo = 0;
  s.steps = ((s.len + (1 << a.log_step) - 1) >> a.log_step) - (int32_t)(lo >> a.log_step);
  if (s.steps < 1) s.steps = 1;
  return s;
}

// A lane's value from the lane that a data-parallel-primitive control names; rows
// and banks without one keep `old`.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int old, int v) {
  return __builtin_amdgcn_update_dpp(old, v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int wave_scan(int v) {       // inclusive sums
  v += moved<0x111, 0xF>(0, v);                         // row_shr 1, 2, 4, 8
  v += moved<0x112, 0xF>(0, v);
  v += moved<0x114, 0xF>(0, v);
  v += moved<0x118, 0xF>(0, v);
  v += moved<0x142, 0xA>(0, v);                         // row 0's last to row 1, row 2's to row 3
  v += moved<0x143, 0xC>(0, v);                         // lane 31 to rows 2 and 3
  return v;
}
__device__ __forceinline__ float wave_total(float v) {
  const auto add = [](float a, int b) { return a + __builtin_bit_cast(float, b); };
  v = add(v, moved<0x111, 0xF>(0, __builtin_bit_cast(int, v)));
  v = add(v, moved<0x112, 0xF>(0, __builtin_bit_cast(int, v)));
  v = add(v, moved<0x114, 0xF>(0, __builtin_bit_cast(int, v)));
  v = add(v, moved<0x118, 0xF>(0, __builtin_bit_cast(int, v)));
  v = add(v, moved<0x142, 0xA>(0, __builtin_bit_cast(int, v)));
  v = add(v, moved<0x143, 0xC>(0, __builtin_bit_cast(int, v)));
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// The sequence, and the number of its first unit, of a unit or of a tile (numbered
// alike, parts left out); false if there is none.
enum Number { kUnitNumber, kTileNumber };
__device__ __forceinline__ bool find(const AttendArgs& a, Number what, int number, Sequence* out,
                                     int* seq, int* first_unit) {
  if (a.direct) {
    *out = sequence(a, number);
    *seq = *first_unit = number;
    return out->tiles > 0;
  }
  const int lane = threadIdx.x & 63;
  const Sequence head = sequence(a, lane);
  int steps = 0x7fffffff, whole = 0x7fffffff;           // of a part, of one that stays whole
  if (a.split) {
    float total = 0.0f, tiles = 0.0f;
    for (int b = 0; b < a.B; b += 64) {
      const Sequence s = b ? sequence(a, b + lane) : head;
      total += wave_total((float)s.tiles * (float)s.steps);
      tiles += wave_total((float)s.tiles);
    }
    const float share = ceilf(total * (float)a.c.heads / a.target);
    steps = share > 1e9f ? 1000000000 : share > (float)a.min_steps ? (int)share : a.min_steps;
    whole = tiles * (float)a.c.heads * 4.0f >= a.target ? a.whole_many : a.whole_few;
  }
  int before = 0, units_before = 0;
  for (int b = 0; b < a.B; b += 64) {
    Sequence s = b ? sequence(a, b + lane) : head;
    s.parts = s.steps > whole ? (s.steps + steps - 1) / steps : 1;
    const int units = s.tiles * s.parts, own = what == kUnitNumber ? units : s.tiles;
    const int upto = before + wave_scan(own);
    const uint64_t mask = __ballot(number >= upto - own && number < upto);
    const int units_upto = what == kUnitNumber ? upto : units_before + wave_scan(units);
    if (mask) {
      const int at = __ffsll((unsigned long long)mask) - 1;
      out->first = (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)s.first, at);
      out->n = __builtin_amdgcn_readlane(s.n, at);
      out->rows = __builtin_amdgcn_readlane(s.rows, at);
      out->tiles = __builtin_amdgcn_readlane(s.tiles, at);
      out->len = __builtin_amdgcn_readlane(s.len, at);
      out->steps = __builtin_amdgcn_readlane(s.steps, at);
      out->parts = __builtin_amdgcn_readlane(s.parts, at);
      out->at = number - __builtin_amdgcn_readlane(upto - own, at);
      *seq = b + at;
      *first_unit = __builtin_amdgcn_readlane(units_upto - units, at);
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
    units_before = __builtin_amdgcn_readlane(units_upto, 63);
  }
  return false;
}

// The keys [lo, hi) that row r of a sequence sees.
__device__ __forceinline__ void row_range(const AttendArgs& a, const Sequence& s, int r, int& lo,
                                          int& hi) {
  const int64_t p = (int64_t)s.len - s.n + r / a.group;
  hi = a.causal && p + 1 < s.len ? (p + 1 < 0 ? 0 : (int)(p + 1)) : s.len;
  const int64_t l = a.window ? p - a.window + 1 : 0;
  lo = l < 0 ? 0 : l > hi ? hi : (int)l;
}

// ------------------------------------------------------------------ the waves
enum { kF16 = 0, kBf16 = 1, kInt8 = 2, kE4m3 = 3 };       // what the cache holds
template <int CT>
constexpr int kBytes = CT < 2 ? 2 : 1;
template <int CT>
constexpr int kRun = 16 / kBytes<CT>;                     // tokens a run
template <int CT>
constexpr int kStep = 4 * kRun<CT>;                       // tokens a wave takes at once

template <int CT>
__device__ __forceinline__ f32x4 mfma16(kv_u32x4 a, kv_u32x4 b, f32x4 c) {
  if constexpr (CT == kBf16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Two f32 to a pair of the type that the products take, to nearest.
template <int CT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (CT == kBf16) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, b2{(__bf16)a, (__bf16)b});
  } else {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, h2{(_Float16)a, (_Float16)b});
  }
}

// Four codes (a word) to two pairs of f16.
template <int CT>
__device__ __forceinline__ void widen(uint32_t w, uint32_t& lo, uint32_t& hi) {
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  if constexpr (CT == kInt8) {
    // code + 128 as the low byte of a half of 1024 is 1152 + code
    w ^= 0x80808080u;
    const h2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
    lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) - off);
    hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) - off);
  } else {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, true));
  }
}
// The h-th operand of eight elements that sixteen bytes hold.
template <int CT>
__device__ __forceinline__ kv_u32x4 operand(kv_u32x4 w, int h) {
  if constexpr (kBytes<CT> == 2) return w;
  uint32_t o[4];
  widen<CT>(h ? w.z : w.x, o[0], o[1]);
  widen<CT>(h ? w.w : w.y, o[2], o[3]);
  return kv_u32x4{o[0], o[1], o[2], o[3]};
}

// v of the wave's quarters 0, 0, 2, 2 and 1, 1, 3, 3 (across: 32), or of its
// halves (64).  The exchange swaps two registers in place: given one value
// twice, the compiler names one register twice, so the copy is made opaque.
struct Pair {
  float a, b;
};
template <int ACROSS>
__device__ __forceinline__ Pair swapped(float v) {
  uint32_t x = __builtin_bit_cast(uint32_t, v), y = x;
  asm("" : "+v"(y));
  if constexpr (ACROSS == 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    return {__builtin_bit_cast(float, (uint32_t)p[0]), __builtin_bit_cast(float, (uint32_t)p[1])};
  } else {
    const auto p = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    return {__builtin_bit_cast(float, (uint32_t)p[0]), __builtin_bit_cast(float, (uint32_t)p[1])};
  }
}
// Largest, and sum, over the wave's four quarters (lanes l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float quarters_max(float v) {
  Pair p = swapped<32>(v);
  p = swapped<64>(fmaxf(p.a, p.b));
  return fmaxf(p.a, p.b);
}
__device__ __forceinline__ float quarters_sum(float v) {
  Pair p = swapped<32>(v);
  p = swapped<64>(p.a + p.b);
  return p.a + p.b;
}

// Bit e of the result: element e of the run w holds is not finite; those become 0.
template <int CT>
__device__ __forceinline__ uint32_t drop_non_finite(kv_u32x4& w) {
  uint32_t bad = 0;
  if constexpr (kBytes<CT> == 2) {
    constexpr uint32_t ones = CT == kF16 ? 0x7C00u : 0x7F80u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t h = w[e >> 1] >> (16 * (e & 1));
      if ((h & ones) == ones) {
        bad |= 1u << e;
        w[e >> 1] &= e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
      }
    }
  } else if constexpr (CT == kE4m3) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if ((w[e >> 2] >> (8 * (e & 3)) & 0x7Fu) == 0x7Fu) {
        bad |= 1u << e;
        w[e >> 2] &= ~(0xFFu << (8 * (e & 3)));
      }
  }
  return bad;
}

// A query's bf16 operands (its lanes: those that differ by WIDTH / 2, and by 32) to
// f16, the row's largest just below 2^15: what falls under f16's range there is
// under 2^-39 of the largest.  Returns scale times the power of two taken out.
template <int KM, int WIDTH>
__device__ __forceinline__ float to_f16(kv_u32x4* q, float scale) {
  float big = 0.0f;
#pragma unroll
  for (int m = 0; m < KM; ++m)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      big = fmaxf(big, __builtin_fabsf(bf16_value(q[m][e >> 1] >> (16 * (e & 1)) & 0xFFFFu)));
  if constexpr (WIDTH == 32) {
    big = quarters_max(big);
  } else {
    const Pair p = swapped<64>(big);
    big = fmaxf(p.a, p.b);
  }
  int ex = (int)(__builtin_bit_cast(uint32_t, big) >> 23 & 0xFF) - 127 - 14;
  ex = big > 0.0f && big < __builtin_inff() ? ex : 0;
#pragma unroll
  for (int m = 0; m < KM; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t w = q[m][e];
      q[m][e] = pack2<kF16>(ldexpf(bf16_value(w & 0xFFFFu), -ex), ldexpf(bf16_value(w >> 16), -ex));
    }
  return fminf(fmaxf(ldexpf(scale, ex), 0x1p-126f), __FLT_MAX__);
}

// How far the largest score seen lies above a row's base: with products in f16 up to
// 2^11 .. 2^15 of weight, so that f16, which rounds what is under 2^-25 to nothing,
// keeps weights down to 2^-36 of the largest (32845 light keys of a thousandth of the
// mass beside one heavy one: with the largest weight between 1 and 2^8 their part of
// out was off by 60%, now by 7e-4; a 4096-token prompt takes 176 us, 172.5 then).
// bf16 has f32's range.
template <int CT>
constexpr float kLift = CT == kBf16 ? 0.0f : 11.0f;
template <int CT>
constexpr float kMost = CT == kBf16 ? 8.0f : 15.0f;

// log2 of a step's largest value scale.  Scales under 2^-81 count as that: weights
// then stay under 2^96, and l in range.
template <int CT>
__device__ __forceinline__ float scale_lift(float big) {
  if constexpr (CT < 2) return 0.0f;
  return __builtin_amdgcn_logf(fmaxf(big, 0x1p-81f));
}
// The base that a row whose largest score (not yet scaled) is top moves to, if that
// asks for more than the most above its base; else its own.  The distance is one fma,
// so it is right however large the scores are.
template <int CT>
__device__ __forceinline__ bool outgrown(float base, float top, float qs, float lift) {
  return fmaf(top, qs, -base) + lift > kMost<CT>;
}
template <int CT>
__device__ __forceinline__ float moved_base(float base, float top, float qs, float lift) {
  return outgrown<CT>(base, top, qs, lift) ? fmaf(top, qs, lift - kLift<CT>) : base;
}

// Largest of three, numbers before NaN: one instruction, and the compiler keeps the
// wait behind a matrix product (it does not for an instruction in inline assembly).
__device__ __forceinline__ float max3(float a, float b, float c) {
  return fmaxf(fmaxf(a, b), c);
}

// Waves of a workgroup: stream_kernel's eight, or four where a wave needs the
// registers of two (at dim > 128, and for 32 rows of 128 over codes, eight waves
// spilled 100 to 300 bytes a lane: 16 sequences of 3000 int8 keys at 256 took 119 us,
// now 48; 16 x 5 tokens of 4000 at 128 62.8, now 47), and the others' four.
constexpr int stream_waves(bool codes, int dim, int rows) {
  return dim > 128 || (codes && dim > 64 && rows > 16) ? 4 : 8;
}
constexpr int kWaves = 4;

// A workgroup is a unit of up to 16·NT rows; its waves take the unit's steps in
// turn and join at the end.  DT: the head's dimension, or the next of 64, 128,
// 256 above it.  What bounds it is the cache's bytes: a step's keys and values
// are 32 registers a lane each at DT = 128, the next step's keys loading while
// this one's weights and values are worked on and the other way round.
template <int CT, int DT, int NT>
__global__ __launch_bounds__(64 * stream_waves(kBytes<CT> == 1, DT, 16 * NT),
                             stream_waves(kBytes<CT> == 1, DT, 16 * NT) / 4) void stream_kernel(AttendArgs a) {
  constexpr int W = stream_waves(kBytes<CT> == 1, DT, 16 * NT);
  constexpr int R = kRun<CT>, TOK = kStep<CT>, NU = R / 4;
  constexpr int KC = DT * kBytes<CT> / 64;       // sixteen-byte loads of a key row's lane
  constexpr int KM = DT / 32;                    // products along a head
  constexpr int VM = DT / 16;                    // tiles of coordinates
  constexpr int H = kBytes<CT> == 2 ? 1 : 2;     // operands in sixteen bytes
  // coordinates joined at once: a thread four of a row
  constexpr int COLS = 4 * (64 * W) / (16 * NT) < DT ? 4 * (64 * W) / (16 * NT) : DT;
  __shared__ float joined[W][16 * NT][COLS + 4];
  __shared__ kv_f32x2 stats[16 * NT][W];
  __shared__ float inverse[16 * NT];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int h = blockIdx.x % a.c.heads, unit = blockIdx.x / a.c.heads;
  Sequence s;
  int b, u0;
  if (!find(a, kUnitNumber, unit, &s, &b, &u0)) return;
  const int tile = s.at / s.parts, part = s.at % s.parts;
  const int row0 = tile * a.block_rows;
  const int rows = s.rows - row0 < 16 * NT ? s.rows - row0 : 16 * NT;
  const int col = lane & 15, g = lane >> 4;

  // the tile's keys, and those that every one of its rows sees
  int lo_first, hi_first, lo_last, hi_last;
  row_range(a, s, row0, lo_first, hi_first);
  row_range(a, s, row0 + rows - 1, lo_last, hi_last);
  int step0 = lo_first / TOK, step1 = (hi_last + TOK - 1) / TOK;
  if (step1 < step0) step1 = step0;
  // parts of whole rounds of the waves
  const int share = ((step1 - step0 + s.parts - 1) / s.parts + W - 1) / W *
                    W;
  const int64_t from_step = step0 + (int64_t)part * share;
  step1 = from_step + share < step1 ? (int)(from_step + share) : step1;
  step0 = from_step < step1 ? (int)from_step : step1;

  int lo[NT], hi[NT];
  kv_u32x4 qf[NT][KM];
  float qs[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = row0 + 16 * t + col;
    const bool in = 16 * t + col < rows;
    lo[t] = hi[t] = 0;
    if (in) row_range(a, s, r, lo[t], hi[t]);
    const uint16_t* q = a.q + (s.first + r / a.group) * a.q_token +
                        ((int64_t)h * a.group + r % a.group) * a.q_head;
#pragma unroll
    for (int m = 0; m < KM; ++m) {
      // the coordinates that sixteen bytes of a key hold, in their order
      const int d = H == 1 ? 32 * m + 8 * g : 64 * (m / 2) + 16 * g + 8 * (m % 2);
      qf[t][m] = in && d < a.c.dim ? *(const kv_u32x4*)(q + d) : kv_u32x4{0, 0, 0, 0};
    }
  }

  f32x4 o[NT][VM];
  float base[NT], l[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    base[t] = -__builtin_inff();
    l[t] = 0.0f;
#pragma unroll
    for (int v = 0; v < VM; ++v) o[t][v] = f32x4{0, 0, 0, 0};
  }

  // A key lane reads run col / 4 of the step, a value lane run g.
  const int row_bytes = a.c.dim * kBytes<CT>;
  const int page_mask = (1 << a.c.log_page) - 1;
  const int32_t* table = a.table + b * a.table_stride;
  const int first_run = lo_first & ~(R - 1), last_run = (hi_last - 1) & ~(R - 1);
  const auto run_at = [&](int step, int run) {
    const int j = step * TOK + R * run;
    return j < first_run ? first_run : j > last_run ? last_run : j;
  };
  const auto page_of = [&](int j) { return table[j >> a.c.log_page]; };
  const auto place = [&](int page, int j) {          // slot, in units of slots of one head
    const int p = page < 0 || page >= a.pages ? 0 : page;
    return (((int64_t)p * a.c.heads + h) << a.c.log_page) + (j & page_mask);
  };
  kv_u32x4 kw[NU][KC], vw[VM];
  float ks[R], vs[R];
  const auto load_keys = [&](int page, int j) {
    const uint8_t* row = a.ck + (place(page, j) + (col & 3)) * row_bytes;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const int at = 64 * c + 16 * g;
        kw[u][c] = *(const kv_u32x4*)(row + 4 * u * row_bytes + (at < row_bytes ? at : 0));
      }
  };
  const auto load_values = [&](int page, int j) {
    const int64_t at = place(page, j);
    const uint8_t* run = a.cv + at * row_bytes + 16 * col;
    if constexpr (H == 2) {
#pragma unroll
      for (int e = 0; e < R; e += 4) {
        const f32x4 x = *(const f32x4*)(a.sv + at + e);
#pragma unroll
        for (int r = 0; r < 4; ++r) vs[e + r] = x[r];
      }
    }
#pragma unroll
    for (int v = 0; v < VM; ++v)
      if (16 * v < a.c.dim) vw[v] = *(const kv_u32x4*)(run + 256 * v);
  };
  const auto load_scales = [&](int page, int j) {
    if constexpr (H == 2) {
      const int64_t at = place(page, j);
#pragma unroll
      for (int e = 0; e < R; e += 4) {
        const f32x4 x = *(const f32x4*)(a.sk + at + e);
#pragma unroll
        for (int r = 0; r < 4; ++r) ks[e + r] = x[r];
      }
    }
  };

  int step = step0 + wave;
  if (step < step1) {
    int jk = run_at(step, col >> 2), jv = run_at(step, g);
    int pk = page_of(jk), pv = page_of(jv);
    load_keys(pk, jk);
    load_scales(pv, jv);
    load_values(pv, jv);
    // (the queries have arrived with the pages; their signs and types wait for nothing)
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      qs[x] = a.scale;
#pragma unroll
      for (int k = 0; k < KM; ++k) qf[x][k] ^= a.flip;
      if (H == 2 && a.type == LEECH_BF16) qs[x] = to_f16<KM, 32>(qf[x], a.scale);
    }
    // the pages of a step are asked for a step ahead of its keys: loads come back in
    // their order, so what waits for a page must not have asked for more before it
    const auto after = [&](int st, int n) {
      return st + n * W < step1 ? st + n * W : st;
    };
    jk = run_at(after(step, 1), col >> 2);
    jv = run_at(after(step, 1), g);
    int pk2 = page_of(jk), pv2 = page_of(jv);
    for (;; step += W) {
      const bool lost = pv < 0 || pv >= a.pages;       // this lane's run has no page
      f32x4 sc[NT][NU];
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int t = 0; t < NT; ++t) sc[t][u] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int k = 0; k < KM; ++k) {
          const kv_u32x4 x = operand<CT>(kw[u][k / H], k % H);
#pragma unroll
          for (int t = 0; t < NT; ++t) sc[t][u] = mfma16<CT>(x, qf[t][k], sc[t][u]);
        }
      const bool more = step + W < step1;
      int jk3 = jk, jv3 = jv, pk3 = pk2, pv3 = pv2;
      if (more) {
        jk3 = run_at(after(step + W, 1), col >> 2);
        jv3 = run_at(after(step + W, 1), g);
        pk3 = page_of(jk3);
        pv3 = page_of(jv3);
        load_keys(pk2, jk);
      }

      // what a row does not see, and what is not a number behind its mask
      const int t0 = step * TOK;
      const bool edge = t0 + TOK > hi_first || t0 < lo_last || __any(lost);
      uint32_t bad = 0;
      if (edge) {
#pragma unroll
        for (int v = 0; v < VM; ++v)
          if (16 * v < a.c.dim) bad |= drop_non_finite<CT>(vw[v]);
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) bad |= __shfl_xor(bad, d, 64);
        if (lost) bad = 0xFFFFu;
      }
      float all_big = 0.0f;
      if constexpr (H == 2) {
#pragma unroll
        for (int e = 0; e < R; ++e) all_big = fmaxf(all_big, vs[e]);
        all_big = quarters_max(all_big);
      }
      kv_u32x4 pw[NT][H];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float x[R];
#pragma unroll
        for (int e = 0; e < R; ++e) {
          x[e] = sc[t][e >> 2][e & 3];
          if constexpr (H == 2) x[e] *= ks[e];
        }
        float big = all_big;
        if (edge) {
          big = 0.0f;
#pragma unroll
          for (int e = 0; e < R; ++e) {
            const int j = t0 + R * g + e;
            const bool sees = j < hi[t] && j >= lo[t];
            x[e] = sees ? (bad >> e & 1 ? __builtin_nanf("") : x[e]) : -__builtin_inff();
            if constexpr (H == 2) big = fmaxf(big, sees ? vs[e] : 0.0f);
          }
          if constexpr (H == 2) big = quarters_max(big);
        }
        float top = -__builtin_inff();
#pragma unroll
        for (int e = 0; e < R; e += 2) top = max3(top, x[e], x[e + 1]);
        top = quarters_max(top);
        const float lift = scale_lift<CT>(big);
        if (__any(outgrown<CT>(base[t], top, qs[t], lift))) {
          // (each row by its own scores alone, whatever its neighbours do)
          const float to = moved_base<CT>(base[t], top, qs[t], lift);
          const float f = to > base[t] ? __builtin_amdgcn_exp2f(base[t] - to) : 1.0f;
          l[t] *= f;
#pragma unroll
          for (int v = 0; v < VM; ++v) o[t][v] *= f;
          base[t] = to;
        }
        const float from = base[t] == -__builtin_inff() ? 0.0f : base[t];
        float w[R], sum = 0.0f;          // (of the step's: see tile_kernel's)
#pragma unroll
        for (int e = 0; e < R; ++e) {
          w[e] = __builtin_amdgcn_exp2f(fmaf(x[e], qs[t], -from));
          sum += w[e];
          // (what a row does not see may have any scale)
          if constexpr (H == 2) w[e] = x[e] == -__builtin_inff() ? 0.0f : w[e] * vs[e];
        }
        l[t] += sum;
#pragma unroll
        for (int i = 0; i < H; ++i)
          pw[t][i] = kv_u32x4{pack2<CT>(w[8 * i], w[8 * i + 1]), pack2<CT>(w[8 * i + 2], w[8 * i + 3]),
                              pack2<CT>(w[8 * i + 4], w[8 * i + 5]),
                              pack2<CT>(w[8 * i + 6], w[8 * i + 7])};
      }
      if (more) load_scales(pv2, jv);
#pragma unroll
      for (int v = 0; v < VM; ++v)
        if (16 * v < a.c.dim)
#pragma unroll
          for (int i = 0; i < H; ++i) {
            const kv_u32x4 x = operand<CT>(vw[v], i);
#pragma unroll
            for (int t = 0; t < NT; ++t) o[t][v] = mfma16<CT>(x, pw[t][i], o[t][v]);
          }
      if (!more) break;
      load_values(pv2, jv);
      pv = pv2;
      jk = jk3;
      jv = jv3;
      pk2 = pk3;
      pv2 = pv3;
    }
  }

  // the waves join: each scales its part to the largest base of a row
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    l[t] = quarters_sum(l[t]);
    if (g == 0) stats[16 * t + col][wave] = kv_f32x2{base[t], l[t]};
  }
  __syncthreads();
  const bool whole = s.parts == 1;
  const int64_t part_row = ((int64_t)h * a.units + unit) * a.block_rows;
  float f[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    kv_f32x2 y[W];
    float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      y[w] = stats[16 * t + col][w];
      top = fmaxf(top, y[w][0]);
    }
    const float to = top == -__builtin_inff() ? 0.0f : top;
    f[t] = __builtin_amdgcn_exp2f(base[t] - to);
    if (wave == t && g == 0 && 16 * t + col < rows) {
#pragma unroll
      for (int w = 0; w < W; ++w) sum += y[w][1] * __builtin_amdgcn_exp2f(y[w][0] - to);
      const int r = 16 * t + col;
      inverse[r] = whole ? (sum != 0.0f ? 1.0f / sum : 0.0f) : 1.0f;     // a NaN sum stays one
      if (!whole)
        *(kv_f32x2*)(a.part_ml + 2 * (part_row + r)) = kv_f32x2{top, sum};
      else if (a.lse)
        a.lse[(s.first + (row0 + r) / a.group) * a.q_heads + h * a.group + (row0 + r) % a.group] =
            sum != 0.0f ? (top + log2f(sum)) * kLn2 : -__builtin_inff();
    }
  }
#pragma unroll
  for (int c0 = 0; c0 < DT; c0 += COLS) {
    if (c0 >= a.c.dim) break;
    if (c0) __syncthreads();
#pragma unroll
    for (int v = c0 / 16; v < (c0 + COLS) / 16; ++v)
#pragma unroll
      for (int t = 0; t < NT; ++t)
        *(f32x4*)&joined[wave][16 * t + col][16 * v - c0 + 4 * g] = o[t][v] * f[t];
    __syncthreads();
    const int r = threadIdx.x / (COLS / 4), c = 4 * (threadIdx.x % (COLS / 4));
    if (r >= rows || c0 + c >= a.c.dim) continue;
    f32x4 x = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < W; ++w) x += *(const f32x4*)&joined[w][r][c];
    x *= inverse[r];
    if (!whole) {
      *(f32x4*)(a.part_o + (part_row + r) * a.c.dim + c0 + c) = x;
      continue;
    }
    const int64_t t = s.first + (row0 + r) / a.group;
    const int qh = h * a.group + (row0 + r) % a.group;
    *(kv_u32x2*)(a.out + t * a.o_token + qh * a.o_head + c0 + c) =
        a.type == LEECH_F16 ? kv_u32x2{pack2<kF16>(x[0], x[1]), pack2<kF16>(x[2], x[3])}
                            : kv_u32x2{pack2<kBf16>(x[0], x[1]), pack2<kBf16>(x[2], x[3])};
  }
}

// ------------------------------------------------------------- many rows at once
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int CT>
__device__ __forceinline__ f32x16 mfma32(kv_u32x4 a, kv_u32x4 b, f32x16 c) {
  if constexpr (CT == kBf16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

constexpr int kTileRows = 32 * kWaves;
template <int DT>
constexpr int kTileTokens = DT > 128 ? 32 : 64;

// LDS of the tile kernel: two buffers of keys and values (as the products take
// them, two bytes an element), of their scales and the largest value scale; for
// three tiles which tokens have no number for a value, or no page; for eight where
// the tokens lie.
template <int CT, int DT>
struct TileLds {
  static constexpr int TOK = kTileTokens<DT>;
  kv_u32x4 k[2][TOK * (DT / 8 + 1)];
  kv_u32x4 v[2][TOK * DT / 8];
  float ks[2][TOK], vs[2][TOK], big[2];
  uint32_t bad[3][TOK / 8];
  int64_t where[8][TOK / 16], slot[8][TOK / 16];    // byte, and slot, of each sixteen tokens
  uint32_t lost[8][TOK / 16];                       // set where there is no such page
};

// A workgroup is a unit of up to 128 rows, a wave 32 of them; all share the keys
// and values, which go through LDS a tile of 64 (32 at DT = 256) tokens at a time:
// the next tile's sixteen-byte loads are under way while this one is worked on,
// widened to 16 bits on their way if they are codes.  Products are 32×32×16,
// transposed as in stream_kernel: row m of a 32-token key tile is token 16·(m / 16)
// + 8·(m / 4 % 2) + 4·(m / 8 % 2) + m % 4, so that a lane's scores are of whole
// runs of eight tokens, those whose values it multiplies next.  Keys lie in LDS
// row by row with sixteen bytes between, which puts the chunks of eight rows that a
// read takes at once in different banks.
template <int CT, int DT>
__global__ __launch_bounds__(64 * kWaves, DT > 128 ? 1 : 2) void tile_kernel(AttendArgs a) {
  constexpr int TOK = kTileTokens<DT>, S = kBytes<CT>, R = kRun<CT>;
  constexpr int NK = TOK / 32;                 // key tiles of 32
  constexpr int KM = DT / 16;                  // products along a head
  constexpr int VM = DT / 32;                  // tiles of coordinates
  constexpr int CH = DT / 8 + 1;               // LDS chunks of a key row, one of them empty
  constexpr int LC = DT * S / 16;              // sixteen-byte loads of a key row
  constexpr int NL = TOK * LC / (64 * kWaves); // of a thread, for keys; as many for values
  constexpr bool CODES = S == 1;
  constexpr int A = CODES && DT == 128 ? 2 : 3;   // LDS reads ahead of a product (more spill)
  extern __shared__ __attribute__((aligned(16))) uint8_t raw[];
  TileLds<CT, DT>& lds = *reinterpret_cast<TileLds<CT, DT>*>(raw);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.x % a.c.heads, unit = blockIdx.x / a.c.heads;
  Sequence s;
  int b, u0;
  if (!find(a, kUnitNumber, unit, &s, &b, &u0)) return;
  // (starts that do not ascend can number units that the workspace does not hold)
  if (s.parts > 1 && u0 + s.tiles * s.parts > a.units) return;
  // the tiles that see most keys first: they run longest
  const int tile = s.tiles - 1 - s.at / s.parts, part = s.at % s.parts;
  const int row0 = tile * kTileRows;
  const int rows = s.rows - row0 < kTileRows ? s.rows - row0 : kTileRows;
  const int col = lane & 31, half = lane >> 5;

  int lo_first, hi_first, lo_last, hi_last;
  row_range(a, s, row0, lo_first, hi_first);
  row_range(a, s, row0 + rows - 1, lo_last, hi_last);
  int step0 = lo_first / TOK, step1 = (hi_last + TOK - 1) / TOK;
  if (step1 < step0) step1 = step0;
  const int64_t span = step1 - step0;
  step1 = step0 + (int)(span * (part + 1) / s.parts);
  step0 = step0 + (int)(span * part / s.parts);

  // this wave's rows, and the keys that they see
  const int wrow = 32 * wave, r = row0 + wrow + col;
  const bool in = wrow + col < rows, live = wrow < rows;
  int lo = 0, hi = 0, wlo = 0, whi = 0, wlo_last = 0, whi_first = 0;
  if (live) {
    const int last = rows - wrow < 32 ? rows - 1 : wrow + 31;
    row_range(a, s, row0 + wrow, wlo, whi_first);
    row_range(a, s, row0 + last, wlo_last, whi);
  }
  if (in) row_range(a, s, r, lo, hi);
  kv_u32x4 qf[KM];
  const uint16_t* q = a.q + (s.first + r / a.group) * a.q_token +
                      ((int64_t)h * a.group + r % a.group) * a.q_head;
#pragma unroll
  for (int m = 0; m < KM; ++m) {
    const int d = 16 * m + 8 * half;
    qf[m] = in && d < a.c.dim ? *(const kv_u32x4*)(q + d) ^ a.flip : kv_u32x4{0, 0, 0, 0};
  }
  float qs = a.scale;
  if (CODES && a.type == LEECH_BF16) qs = to_f16<KM, 64>(qf, a.scale);

  f32x16 o[VM];
#pragma unroll
  for (int v = 0; v < VM; ++v)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[v][e] = 0.0f;
  float base = -__builtin_inff(), l = 0.0f;

  const int row_bytes = a.c.dim * S;
  const int32_t* table = a.table + b * a.table_stride;
  const int first16 = lo_first & ~15, last16 = (hi_last - 1) & ~15;
  // Where sixteen tokens lie (clamped to those that are seen), four tiles at a time, a
  // thread sixteen tokens.  Pages are asked for ahead of a tile's own loads and
  // looked at behind them.
  constexpr int G = TOK / 16;
  int page = 0, spot = 0;
  const auto look_up = [&](int step) {
    spot = step * TOK + 16 * tid;
    spot = spot < first16 ? first16 : spot > last16 ? last16 : spot;
    page = table[spot >> a.c.log_page];
  };
  const auto note = [&](int step) {
    const bool lost = page < 0 || page >= a.pages;
    const int64_t slot = (((int64_t)(lost ? 0 : page) * a.c.heads + h) << a.c.log_page) +
                         (spot & ((1 << a.c.log_page) - 1));
    const int to = (step + tid / G) & 7;
    lds.where[to][tid % G] = slot * row_bytes;
    if (CODES) lds.slot[to][tid % G] = slot;
    lds.lost[to][tid % G] = lost ? 0xFFu : 0u;
  };
  // Tokens of no page count as without numbers.
  const auto clear = [&](int step) {
    lds.bad[step % 3][tid] = lds.lost[step & 7][tid >> 1];
  };
  // A tile's loads and LDS writes come in 2·NL pieces, keys first, to be spread among
  // the products: eight waves that ask for all of theirs at once wait for each other.
  // Columns past the head's dimension read others again: those of the queries are 0,
  // those of out are not kept.
  kv_u32x4 kw[NL], vw[NL];
  float sc = 0.0f;
  const auto load = [&](int step, int piece) {
    const int64_t* where = lds.where[step & 7];
    const int i = piece % NL, at = i * 64 * kWaves + tid;
    if (piece < NL) {
      const int t = at / LC, c = at % LC;
      kw[i] = *(const kv_u32x4*)(a.ck + where[t >> 4] + (t & 15) * row_bytes +
                                 (16 * c < row_bytes ? 16 * c : 0));
    } else {
      const int run = at / DT, d = at % DT;
      vw[i] = *(const kv_u32x4*)(a.cv + where[run * R >> 4] + (run * R & 15) * row_bytes +
                                 16 * (d < a.c.dim ? d : 0));
    }
    if (CODES && piece == 2 * NL - 1) {
      const int t = tid & (TOK - 1);
      sc = ((tid & TOK) ? a.sv : a.sk)[lds.slot[step & 7][t >> 4] + (t & 15)];
    }
  };
  const auto keep = [&](int step, int piece) {
    const int buf = step & 1, i = piece % NL, at = i * 64 * kWaves + tid;
    if (piece < NL) {
      const int t = at / LC, c = at % LC;
      if constexpr (CODES) {
        lds.k[buf][t * CH + 2 * c] = operand<CT>(kw[i], 0);
        lds.k[buf][t * CH + 2 * c + 1] = operand<CT>(kw[i], 1);
      } else {
        lds.k[buf][t * CH + c] = kw[i];
      }
      return;
    }
    const int run = at / DT, d = at % DT;
    // values behind some row's mask must be numbers; a token that has none counts
    // as NaN for the rows that see it
    if (CT != kInt8 && (step * TOK + TOK > hi_first || step * TOK < lo_last)) {
      const uint32_t bad = drop_non_finite<CT>(vw[i]);
      if (bad) {
        atomicOr(&lds.bad[step % 3][run * R / 8], bad & 0xFFu);
        if (CODES) atomicOr(&lds.bad[step % 3][run * R / 8 + 1], bad >> 8);
      }
    }
    if constexpr (CODES) {
      lds.v[buf][2 * run * DT + d] = operand<CT>(vw[i], 0);
      lds.v[buf][(2 * run + 1) * DT + d] = operand<CT>(vw[i], 1);
    } else {
      lds.v[buf][run * DT + d] = vw[i];
    }
    if (CODES && piece == 2 * NL - 1) {
      // a value scale that is no number counts as its value not being one
      if (tid >= TOK && tid < 2 * TOK && !(__builtin_fabsf(sc) < __builtin_inff())) {
        atomicOr(&lds.bad[step % 3][(tid & (TOK - 1)) >> 3], 1u << (tid & 7));
        sc = 0.0f;
      }
      if (tid < 2 * TOK) (tid < TOK ? lds.ks : lds.vs)[buf][tid & (TOK - 1)] = sc;
      float big = sc;                   // every TOK threads hold a whole tile's scales
#pragma unroll
      for (int x = 1; x < TOK; x <<= 1) big = fmaxf(big, __shfl_xor(big, x, 64));
      if (tid == TOK) lds.big[buf] = big;
    }
  };
  // The pieces that belong to the k-th of n products.
  const auto share = [](int k, int n, auto piece) {
#pragma unroll
    for (int i = 0; i < 2 * NL; ++i)
      if (i * n / (2 * NL) == k) piece(i);
  };

  if (step0 < step1) {
    if (tid < 8 * G) {
      look_up(step0);
      note(step0);
    }
    __syncthreads();
    if (tid < TOK / 8) {
      clear(step0);
      clear(step0 + 1);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2 * NL; ++i) load(step0, i);
#pragma unroll
    for (int i = 0; i < 2 * NL; ++i) keep(step0, i);
    __syncthreads();
  }
  // (the last turn fetches its own tile again: every place is clamped to those seen)
  for (int step = step0; step < step1; ++step) {
    const int buf = step & 1, t0 = step * TOK;
    const bool turn = ((step - step0) & 3) == 0 && step != step0;
    if (turn && tid < 4 * G) look_up(step + 4);
    if (live && t0 < whi && t0 + TOK > wlo) {
      // score e of the n-th 32 tokens: token 16 (e / 8) + 8 half + e % 8 of them.  Reads
      // run A products ahead.
      f32x16 x[NK];
      {
        const int t = 16 * (col >> 4) + 8 * (col >> 2 & 1) + 4 * (col >> 3 & 1) + (col & 3);
        const kv_u32x4* row = &lds.k[buf][t * CH + half];
        kv_u32x4 kf[A + 1];
#pragma unroll
        for (int k = 0; k < A; ++k) kf[k] = row[2 * k];
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) x[n][e] = 0.0f;
#pragma unroll
        for (int k = 0; k < NK * KM; ++k) {
          if (k + A < NK * KM) kf[(k + A) % (A + 1)] = row[(k + A) / KM * 32 * CH + 2 * ((k + A) % KM)];
          x[k / KM] = mfma32<CT>(kf[k % (A + 1)], qf[k % KM], x[k / KM]);
          share(k, NK * KM, [&](int i) { load(step + 1, i); });
          if constexpr (!CODES) __builtin_amdgcn_sched_barrier(0);
        }
      }
      if constexpr (CODES)
#pragma unroll
        for (int n = 0; n < 4 * NK; ++n) {
          const f32x4 y = *(const f32x4*)&lds.ks[buf][16 * (n >> 1) + 8 * half + 4 * (n & 1)];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[n >> 2][4 * (n & 3) + e] *= y[e];
        }
      uint32_t bad = 0;
#pragma unroll
      for (int n = 0; n < 2 * NK; ++n) bad |= lds.bad[step % 3][2 * n + half] << (8 * n);
      const bool edge = t0 + TOK > whi_first || t0 < wlo_last || __any(bad != 0);
      float big = CODES ? lds.big[buf] : 0.0f;
      if (edge) {
        big = 0.0f;
#pragma unroll
        for (int n = 0; n < 4 * NK; ++n) {
          const int j0 = 16 * (n >> 1) + 8 * half + 4 * (n & 1);
          f32x4 y = {0, 0, 0, 0};
          if constexpr (CODES) y = *(const f32x4*)&lds.vs[buf][j0];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = t0 + j0 + e;
            const bool sees = j < hi && j >= lo;
            const float z = bad >> (4 * n + e) & 1 ? __builtin_nanf("") : x[n >> 2][4 * (n & 3) + e];
            x[n >> 2][4 * (n & 3) + e] = sees ? z : -__builtin_inff();
            if constexpr (CODES) big = fmaxf(big, sees ? y[e] : 0.0f);
          }
        }
        if constexpr (CODES) {
          const Pair p = swapped<64>(big);
          big = fmaxf(p.a, p.b);
        }
      }
      float top = -__builtin_inff();
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int e = 0; e < 16; e += 2) top = max3(top, x[n][e], x[n][e + 1]);
      const Pair p = swapped<64>(top);
      top = fmaxf(p.a, p.b);
      const float lift = scale_lift<CT>(big);
      if (__any(outgrown<CT>(base, top, qs, lift))) {
        // (each row by its own scores alone, whatever its neighbours do)
        const float to = moved_base<CT>(base, top, qs, lift);
        const float f = to > base ? __builtin_amdgcn_exp2f(base - to) : 1.0f;
        l *= f;
#pragma unroll
        for (int v = 0; v < VM; ++v) o[v] *= f;
        base = to;
      }
      const float from = base == -__builtin_inff() ? 0.0f : base;
      // Weights of four tokens, as a half of the second product's operand.
      // A tile's weights are summed before l takes them: one by one, what lies under 2^-24
      // of l would be lost (32845 light keys of a thousandth of the mass beside a heavy
      // one: l was off by 3e-4, now by 2e-5).
      float sum = 0.0f;
      kv_u32x4 pw[2 * NK];
      const auto weights = [&](int n) {
        f32x4 y = {1, 1, 1, 1};
        if constexpr (CODES) y = *(const f32x4*)&lds.vs[buf][16 * (n >> 1) + 8 * half + 4 * (n & 1)];
        float w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] = __builtin_amdgcn_exp2f(fmaf(x[n >> 2][4 * (n & 3) + e], qs, -from));
          sum += w[e];
          if constexpr (CODES) w[e] *= y[e];
        }
        pw[n >> 1][2 * (n & 1)] = pack2<CT>(w[0], w[1]);
        pw[n >> 1][2 * (n & 1) + 1] = pack2<CT>(w[2], w[3]);
      };
      // The first sixteen tokens' weights, then each sixteen's products with the next
      // ones' weights and the next tile's LDS writes among them.
      constexpr int N = 2 * NK * VM;
      const kv_u32x4* values = &lds.v[buf][half * DT + col];
      const auto value = [&](int i) { return values[2 * (i / VM) * DT + 32 * (i % VM)]; };
      kv_u32x4 vf[A + 1];
#pragma unroll
      for (int i = 0; i < A; ++i) vf[i] = value(i);
      weights(0);
      weights(1);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (i + A < N) vf[(i + A) % (A + 1)] = value(i + A);
        o[i % VM] = mfma32<CT>(vf[i % (A + 1)], pw[i / VM], o[i % VM]);
        if (i / VM + 1 < 2 * NK && i % VM % (VM / 2) == 0)
          weights(2 * (i / VM + 1) + i % VM / (VM / 2));
        if (i >= N / 2) share(i - N / 2, N / 2, [&](int x) { keep(step + 1, x); });
        if constexpr (!CODES) __builtin_amdgcn_sched_barrier(0);
      }
      l += sum;
    } else {
#pragma unroll
      for (int i = 0; i < 2 * NL; ++i) load(step + 1, i);
#pragma unroll
      for (int i = 0; i < 2 * NL; ++i) keep(step + 1, i);
    }
    if (turn && tid < 4 * G) note(step + 4);
    if (tid < TOK / 8) clear(step + 2);
    __syncthreads();
  }

  Pair p = swapped<64>(l);
  l = p.a + p.b;
  if (!in) return;
  if (s.parts > 1) {
    const int64_t at = ((int64_t)h * a.units + u0 + tile * s.parts + part) * kTileRows + wrow + col;
#pragma unroll
    for (int v = 0; v < VM; ++v)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d = 32 * v + 8 * i + 4 * half;
        if (d < a.c.dim)
          *(f32x4*)(a.part_o + at * a.c.dim + d) =
              f32x4{o[v][4 * i], o[v][4 * i + 1], o[v][4 * i + 2], o[v][4 * i + 3]};
      }
    if (half == 0) {
      a.part_ml[2 * at] = base;
      a.part_ml[2 * at + 1] = l;
    }
    return;
  }
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;          // a NaN sum stays one
  const int64_t t = s.first + r / a.group;
  const int qh = h * a.group + r % a.group;
  uint16_t* out = a.out + t * a.o_token + qh * a.o_head;
#pragma unroll
  for (int v = 0; v < VM; ++v)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 32 * v + 8 * i + 4 * half;
      if (d >= a.c.dim) continue;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = o[v][4 * i + e] * inv;
      *(kv_u32x2*)(out + d) = a.type == LEECH_F16
                                  ? kv_u32x2{pack2<kF16>(x[0], x[1]), pack2<kF16>(x[2], x[3])}
                                  : kv_u32x2{pack2<kBf16>(x[0], x[1]), pack2<kBf16>(x[2], x[3])};
    }
  if (a.lse && half == 0)
    a.lse[t * a.q_heads + qh] = l != 0.0f ? (base + log2f(l)) * kLn2 : -__builtin_inff();
}

// Joins the parts of a tile's rows: a wave a row, or, where there are more parts
// than its eight loads at once take, a workgroup a row.  A wave weighs all parts,
// a lane a part, then sums its share of them, a lane four coordinates.
__global__ __launch_bounds__(64 * kWaves) void join_kernel(AttendArgs a) {
  __shared__ f32x4 quarter[kWaves][kMaxHeadDim / 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int h = blockIdx.x % a.c.heads;
  const int slice = blockIdx.x / a.c.heads % a.slices, at_tile = blockIdx.x / a.c.heads / a.slices;
  Sequence s;
  int b, u0;
  if (!find(a, kTileNumber, at_tile, &s, &b, &u0) || s.parts == 1) return;
  const int tile = s.at;
  // (starts that do not ascend can number units that the workspace does not hold)
  if (u0 + s.tiles * s.parts > a.units) return;
  const int row0 = tile * a.block_rows;
  const int rows = s.rows - row0 < a.block_rows ? s.rows - row0 : a.block_rows;
  const int64_t first = ((int64_t)h * a.units + u0 + tile * s.parts) * a.block_rows;
  const int each = a.c.dim <= 64 ? 4 : a.c.dim <= 128 ? 2 : 1;      // parts a wave reads at once
  const int sub = lane / (64 / each), c = 4 * (lane % (64 / each));
  const bool in = c < a.c.dim;
  constexpr int U = 8;
  const int team = s.parts > U * each ? kWaves : 1, member = wave % team;     // waves of a row
  for (int r = (slice * kWaves + wave) / team; r < rows; r += a.slices * (kWaves / team)) {
    const int64_t at = first + r;
    const auto ml = [&](int p) {
      return *(const kv_f32x2*)(a.part_ml + 2 * (at + (int64_t)p * a.block_rows));
    };
    float top = -__builtin_inff();
    for (int p = lane; p < s.parts; p += 64) top = fmaxf(top, ml(p)[0]);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float base = top == -__builtin_inff() ? 0.0f : top;
    float sum = 0.0f;
    f32x4 x = {0, 0, 0, 0};
    for (int p0 = 0; p0 < s.parts; p0 += 64) {
      float f = 0.0f;
      if (p0 + lane < s.parts) {
        const kv_f32x2 y = ml(p0 + lane);
        f = __builtin_amdgcn_exp2f(y[0] - base);
        sum += f * y[1];
      }
      const int n = s.parts - p0 < 64 ? s.parts - p0 : 64;
      for (int p = member * each; p < n; p += U * team * each) {
        f32x4 y[U];
        float w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = p + u * team * each + sub, k = i < n ? i : n - 1;
          y[u] = *(const f32x4*)(a.part_o + (at + (int64_t)(p0 + k) * a.block_rows) * a.c.dim +
                                 (in ? c : 0));
          w[u] = __shfl(f, k, 64);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          // (a weight of 0 too: what is no number in a part reaches the row)
          if (p + u * team * each + sub < n) x += y[u] * w[u];
      }
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
    for (int d = 64 / each; d < 64; d <<= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], d, 64);
    if (team > 1) {
      __syncthreads();
      if (in && sub == 0) quarter[wave][c / 4] = x;
      __syncthreads();
      if (wave == 0 && in)
#pragma unroll
        for (int w = 1; w < kWaves; ++w) x += quarter[w][c / 4];
    }
    if (member || !in || sub) continue;
    const int64_t t = s.first + (row0 + r) / a.group;
    const int qh = h * a.group + (row0 + r) % a.group;
    x *= sum != 0.0f ? 1.0f / sum : 0.0f;              // a NaN sum stays one
    *(kv_u32x2*)(a.out + t * a.o_token + qh * a.o_head + c) =
        a.type == LEECH_F16 ? kv_u32x2{pack2<kF16>(x[0], x[1]), pack2<kF16>(x[2], x[3])}
                            : kv_u32x2{pack2<kBf16>(x[0], x[1]), pack2<kBf16>(x[2], x[3])};
    if (a.lse && lane == 0)
      a.lse[t * a.q_heads + qh] = sum != 0.0f ? (top + log2f(sum)) * kLn2 : -__builtin_inff();
  }
}

// ------------------------------------------------------------------ host side
constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1;
constexpr int kFewRows = 32;           // rows of a sequence that stream_kernel takes
constexpr int kTargetFew = 512, kTargetMany = 512;    // workgroups that split sequences come to
constexpr int kMinTokens = 256;        // keys of a part of many rows, at least

// One launch's share of a call: a function of sizes alone.
struct Cut {
  int waves, block_rows, log_step, min_steps, whole_few, whole_many, split, direct, over, upto,
      target;
  int64_t tiles, units;
  size_t bytes;
};
struct Cuts {
  Cut few, many;                       // units = 0: not launched
};

int cut(const leech_attend_args* g, const CacheShape& c, bool many, Cut* k) {
  const int64_t group = g->q_heads / c.heads, T = g->T * group;
  const int64_t keys = (int64_t)g->table_pages << c.log_page;
  k->target = many ? kTargetMany : kTargetFew;
  k->log_step = many ? (c.dim > 128 ? 5 : 6) : type_bytes(c.type) == 2 ? 5 : 6;
  k->waves = many ? kWaves : stream_waves(type_bytes(c.type) == 1, c.dim, k->block_rows);
  k->min_steps = many ? kMinTokens >> k->log_step : k->waves;
  const int64_t least = (T + k->block_rows - 1) / k->block_rows;
  // A round of the waves takes about 2 us, the join 3.5: three rounds stay whole
  // (one sequence of 700 f16 keys: 12.8 us whole, 13.0 split; of 2000 24.2 and 13.2);
  // with the card half full already eight do (16 of 2000: 26.8 and 34.4), four where a
  // step has twice the products (16 x 5 of 4000 int8 keys: eight 74.8, split 62.7).
  // Many rows: up to 1024 keys.
  k->whole_few = many ? 1024 >> k->log_step : 3 * k->waves;
  k->whole_many = many ? k->whole_few : (k->block_rows > 16 ? 4 : 8) * k->waves;
  k->split = keys > ((int64_t)k->whole_few << k->log_step) && least * c.heads < k->target;
  // Few rows are a tile a sequence, however few they are.  Where those fill the card
  // eight times over (4096 workgroups) they stay whole: every wave would number all of
  // them (f16, 8 heads and as many of the queries, dim 128: 1000 sequences of 300 keys
  // 820 us split, 311 whole, one of them of 30000 keys 850 and 371; 512 sequences 301
  // and 165, 310 and 351; 256 sequences 122 and 84, 134 and 345: split).
  if (!many && std::min<int64_t>(g->B, g->T) * c.heads >= 8 * k->target) k->split = 0;
  // (two more for the roundings of the plan's f32 total)
  k->tiles = T / k->block_rows + std::min<int64_t>(g->B, g->T);
  // Few rows are one tile a sequence: unsplit, nothing has to be looked for
  // (1024 sequences of 300 f16 keys: 603 us when every workgroup numbers them, 326).
  k->direct = !many && !k->split;
  k->units = k->direct ? g->B
             : k->tiles + (k->split ? (k->target + c.heads - 1) / c.heads + 2 : 0);
  if (k->units * c.heads * 64 * k->waves > kMaxThreads)
    return set_error(LEECH_E_SHAPE, "too many rows for a launch");
  k->bytes = k->split ? (size_t)(c.heads * k->units * k->block_rows) * (c.dim + 2) * sizeof(float)
                      : 0;
  return LEECH_OK;
}

// Sequences of up to kFewRows rows are stream_kernel's (16 at dim > 128, where two
// tiles of them do not fit the registers); tile_kernel takes longer ones, and all
// of them where B sequences are 256 rows long on average: few can be short then,
// and a second launch, for most calls without work, costs 10 us.
int cut_all(const leech_attend_args* g, const CacheShape& c, Cuts* k) {
  const int64_t group = g->q_heads / c.heads;
  const int64_t rows = std::min<int64_t>(g->max_new, g->T) * group;
  *k = {};
  int rc = LEECH_OK;
  const int few_rows = c.dim > 128 ? 16 : kFewRows;
  const bool many = rows > few_rows;
  const bool few = !many || g->T * group < (int64_t)g->B * 256;
  if (few) {
    k->few.block_rows = std::min<int64_t>(rows, few_rows) > 16 ? 32 : 16;
    k->few.over = 0;
    k->few.upto = few_rows;
    rc = cut(g, c, false, &k->few);
  }
  if (many && !rc) {
    k->many.block_rows = kTileRows;
    k->many.over = few ? few_rows : 0;
    k->many.upto = 0x7fffffff;
    rc = cut(g, c, true, &k->many);
  }
  return rc;
}

// Sizes alone: what the workspace goes by.
int check_sizes(const leech_kv_cache* cache, const leech_attend_args* g, CacheShape* shape,
                Cuts* k) {
  const int rc = check_cache(cache, shape);
  if (rc) return rc;
  if (!g) return set_error(LEECH_E_ARG, "the arguments are NULL");
  if (g->type != LEECH_F16 && g->type != LEECH_BF16)
    return set_error(LEECH_E_ARG, "queries must be f16 or bf16");
  if (type_bytes(cache->type) == 2 && cache->type != g->type)
    return set_error(LEECH_E_ARG, "a 16-bit cache must have the queries' type");
  if (g->q_heads <= 0 || g->q_heads > 65535 || g->q_heads % cache->heads)
    return set_error(LEECH_E_SHAPE, "query heads must be a multiple of the cache's, up to 65535");
  if (g->T < 0 || g->B < 0 || g->max_new < 0 || g->T > 0x7fffffff / g->q_heads)
    return set_error(LEECH_E_SHAPE, "B and max_new must not be negative, T · q_heads 0 to 2^31 - 1");
  if (g->table_pages < 0 || ((int64_t)g->table_pages << shape->log_page) > 0x7fffff00)
    return set_error(LEECH_E_SHAPE, "a row of the page table holds fewer than 2^31 - 256 tokens");
  if (!g->q_start && g->T != g->B)
    return set_error(LEECH_E_SHAPE, "without q_start there is one new token a sequence");
  return cut_all(g, *shape, k);
}

int check_strides(const char* name, const void* p, int64_t token, int64_t head) {
  if (!p) return set_error(LEECH_E_ARG, std::string(name) + " is NULL");
  if (((uintptr_t)p & 15) || token % 8 || head % 8)
    return set_error(LEECH_E_ARG, std::string(name) +
                                      ": needs 16-byte alignment and strides of 8 elements");
  return LEECH_OK;
}

typedef void (*AttendFn)(AttendArgs);
struct Launch {
  AttendFn fn;
  size_t lds;
};
template <int CT, int DT>
Launch pick_dim(int block_rows) {
  if (block_rows == 16) return {stream_kernel<CT, DT, 1>, 0};
  if constexpr (DT <= 128)
    if (block_rows == 32) return {stream_kernel<CT, DT, 2>, 0};
  return {tile_kernel<CT, DT>, sizeof(TileLds<CT, DT>)};
}
template <int CT>
Launch pick(int dim, int block_rows) {
  return dim <= 64    ? pick_dim<CT, 64>(block_rows)
         : dim <= 128 ? pick_dim<CT, 128>(block_rows)
                      : pick_dim<CT, 256>(block_rows);
}

int launch(AttendArgs a, const Cut& k, float* workspace, hipStream_t stream) {
  a.block_rows = k.block_rows;
  a.log_step = k.log_step;
  a.min_steps = k.min_steps;
  a.whole_few = k.whole_few;
  a.whole_many = k.whole_many;
  a.units = (int32_t)k.units;
  a.split = k.split;
  a.over = k.over;
  a.upto = k.upto;
  a.target = (float)k.target;
  a.direct = k.direct;
  // a row a wave, unless that makes more workgroups than the card takes at once
  a.slices = (int32_t)std::max<int64_t>(
      1, std::min<int64_t>(k.block_rows / kWaves, 4096 / (k.tiles * a.c.heads)));
  a.part_o = workspace;
  a.part_ml = workspace + (int64_t)a.c.heads * k.units * k.block_rows * a.c.dim;
  const Launch f = a.c.type == LEECH_F16    ? pick<kF16>(a.c.dim, k.block_rows)
                   : a.c.type == LEECH_BF16 ? pick<kBf16>(a.c.dim, k.block_rows)
                   : a.c.type == LEECH_INT8 ? pick<kInt8>(a.c.dim, k.block_rows)
                                            : pick<kE4m3>(a.c.dim, k.block_rows);
  hipError_t e;
  if (f.lds > 64 * 1024) {
    e = hipFuncSetAttribute((const void*)f.fn, hipFuncAttributeMaxDynamicSharedMemorySize,
                            (int)f.lds);
    if (e != hipSuccess) return hip_fail("hipFuncSetAttribute", e);
  }
  hipLaunchKernelGGL(f.fn, dim3((unsigned)(a.c.heads * k.units)), dim3(64 * k.waves), f.lds,
                     stream, a);
  e = hipGetLastError();
  if (e != hipSuccess) return hip_fail("attend launch", e);
  if (!k.split) return LEECH_OK;
  hipLaunchKernelGGL(join_kernel, dim3((unsigned)(k.tiles * a.c.heads * a.slices)),
                     dim3(64 * kWaves), 0, stream, a);
  e = hipGetLastError();
  return e == hipSuccess ? LEECH_OK : hip_fail("attend join launch", e);
}

}  // namespace
}  // namespace leech

using namespace leech;

extern "C" int leech_attend_workspace(const leech_kv_cache* cache, const leech_attend_args* args,
                                      size_t* bytes) {
  clear_error();
  CacheShape shape;
  Cuts k;
  const int rc = check_sizes(cache, args, &shape, &k);
  if (rc) return rc;
  if (!bytes) return set_error(LEECH_E_ARG, "bytes is NULL");
  *bytes = k.few.bytes + k.many.bytes;
  return LEECH_OK;
}

extern "C" int leech_attend(const leech_kv_cache* cache, const leech_attend_args* g,
                            void* stream) {
  clear_error();
  AttendArgs a = {};
  Cuts k;
  int rc = check_sizes(cache, g, &a.c, &k);
  if (rc) return rc;
  if ((g->causal != 0 && g->causal != 1) || g->window < 0)
    return set_error(LEECH_E_ARG, "causal must be 0 or 1 and window not negative");
  if (!(__builtin_fabsf(g->scale) < __builtin_inff()))
    return set_error(LEECH_E_ARG, "the scale must be finite");
  if (g->T == 0 || g->B == 0 || g->max_new == 0) return LEECH_OK;
  if ((rc = check_strides("q", g->q, g->q_token_stride, g->q_head_stride)) ||
      (rc = check_strides("out", g->out, g->out_token_stride, g->out_head_stride)))
    return rc;
  if (!rows_apart(g->out_token_stride, g->out_head_stride, g->T, g->q_heads, cache->dim))
    return set_error(LEECH_E_SHAPE, "out: rows overlap (strides too small)");
  if (!g->kv_len || (!g->page_table && g->table_pages))
    return set_error(LEECH_E_ARG, "kv_len or the page table is NULL");
  if (((uintptr_t)g->q_start & 3) || ((uintptr_t)g->kv_len & 3) || ((uintptr_t)g->page_table & 3) ||
      ((uintptr_t)g->lse & 3))
    return set_error(LEECH_E_ARG, "misaligned device pointer");
  const size_t bytes = k.few.bytes + k.many.bytes;
  if (bytes && (!g->workspace || g->workspace_bytes < bytes || ((uintptr_t)g->workspace & 15)))
    return set_error(LEECH_E_ARG, "the workspace is NULL, misaligned or smaller than "
                                  "leech_attend_workspace says");
  a.ck = (const uint8_t*)cache->k;
  a.cv = (const uint8_t*)cache->v;
  a.sk = cache->k_scale;
  a.sv = cache->v_scale;
  a.q = (const uint16_t*)g->q;
  a.out = (uint16_t*)g->out;
  a.lse = g->lse;
  a.q_token = g->q_token_stride;
  a.q_head = g->q_head_stride;
  a.o_token = g->out_token_stride;
  a.o_head = g->out_head_stride;
  a.table_stride = g->table_stride;
  a.q_start = g->q_start;
  a.kv_len = g->kv_len;
  a.table = g->page_table;
  a.T = g->T;
  a.pages = cache->pages;
  a.type = g->type;
  a.q_heads = g->q_heads;
  a.group = g->q_heads / cache->heads;
  a.B = g->B;
  a.table_pages = g->table_pages;
  a.max_new = g->max_new;
  a.causal = g->causal;
  a.window = g->window;
  // (an infinite one would make NaN of a product that is 0)
  a.scale = std::min(std::max(std::fabs(g->scale) * kLog2e, 0x1p-126f), __FLT_MAX__);
  a.flip = g->scale < 0.0f ? 0x80008000u : 0u;
  float* room = (float*)g->workspace;
  if (k.few.units && (rc = launch(a, k.few, room, (hipStream_t)stream))) return rc;
  if (k.many.units &&
      (rc = launch(a, k.many, room + k.few.bytes / sizeof(float), (hipStream_t)stream)))
    return rc;
  return LEECH_OK;
}
