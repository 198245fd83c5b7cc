// Rotary positions and the paged key/value cache's writes and reads for gfx950.
//
// Rotation.  Token t at position p_t turns pair i of a head by the angle
// p_t · f_i, with f_i the caller's f64 frequencies.  The angle is formed and
// reduced to a turn in f64 (at position 2^20 an f32 product would be off by
// 2^-4 of a radian), its sine and cosine are f32, and so is the rotation; the
// result is rounded once, to the type it is kept in.
//
// Cache.  16-bit caches keep the rounded numbers.  8-bit caches keep, per token
// and head, scale = largest / 127 (int8) or / 448 (e4m3) in f32 and the codes
// x / scale rounded to nearest even.  Keys lie token by token.  Values lie in
// runs: sixteen bytes hold value_run consecutive tokens' values of one
// coordinate, which is what a lane of the attention's second matrix product
// takes, so that it reads them from memory as they are.
//
// Geometry.  Teams of sixteen lanes own a key or query row (one head of one token),
// a lane eight coordinates at a time: four pairs where the rotation reaches.  A
// team keeps its token and walks over heads, four rows loading at once, so a sine
// is computed once for several of them.  A wave owns the values of a few
// consecutive tokens and one head.  Where tokens fill a run of slots it takes the
// run whole: half of the wave half of the run's tokens, a lane four coordinates of
// each, so that the run's sixteen bytes a coordinate are put together (or taken
// apart) in the lane's registers.  Elsewhere it goes token by token.

#include "kv_device.h"

#include <type_traits>

namespace leech {
namespace {

constexpr int kThreads = 256;
constexpr int kTeam = 16;                 // lanes of a row
constexpr int kTeams = kThreads / kTeam;
constexpr int kWaves = kThreads / 64;
constexpr int kAtOnce = 4;                // rows a team has on their way

struct Rows {
  void* data;
  int64_t token, head;                    // strides in elements
  int32_t type, wide;                     // wide: four elements load and store as one
};

struct Turn {
  const double* freq;
  float cosine, sine;                     // factors of each: the magnitude, and its sign for
                                          // the opposite angle
  int32_t width, interleaved;
};

struct WriteArgs {
  CacheShape c;
  Rows q, qo, k, v;
  uint8_t *ck, *cv;
  float *sk, *sv;
  const int64_t *slots, *positions;
  Turn turn;
  int64_t T, token_blocks, turn_blocks;   // blocks that turn, before those of the values
  int32_t q_heads, k_heads;               // rows of q, then of k, that a token turns
  int32_t by_token;                       // teams of a block: as many tokens, or heads of one
  int32_t slice, slices;                  // heads of a block; blocks of a token's heads
  int32_t tokens;                         // of a wave's values
};

struct ReadArgs {
  CacheShape c;
  const uint8_t *ck, *cv;
  const float *sk, *sv;
  const int64_t* slots;
  Rows k, v;
  int64_t T, key_blocks;
  int32_t tokens;
};

// Four elements as they lie: an f32 each, or two 16-bit ones a word.
template <int SRC>
using Four = typename std::conditional<SRC == LEECH_F32, kv_u32x4, kv_u32x2>::type;
template <int SRC>
__device__ __forceinline__ Four<SRC> load4(const Rows& r, int64_t at) {
  Four<SRC> w;
  if constexpr (SRC == LEECH_F32) {
    const uint32_t* p = (const uint32_t*)r.data + at;
    if (r.wide)
      w = *(const kv_u32x4*)p;
    else
#pragma unroll
      for (int t = 0; t < 4; ++t) w[t] = p[t];
  } else {
    const uint16_t* p = (const uint16_t*)r.data + at;
    if (r.wide)
      w = *(const kv_u32x2*)p;
    else
#pragma unroll
      for (int t = 0; t < 2; ++t) w[t] = p[2 * t] | (uint32_t)p[2 * t + 1] << 16;
  }
  return w;
}
template <int SRC>
__device__ __forceinline__ void values4(const Four<SRC>& w, float v[4]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if constexpr (SRC == LEECH_F32)
      v[t] = __builtin_bit_cast(float, (uint32_t)w[t]);
    else if constexpr (SRC == LEECH_F16)
      v[t] = half_value(w[t >> 1] >> (16 * (t & 1)));
    else
      v[t] = bf16_value(w[t >> 1] >> (16 * (t & 1)) & 0xFFFFu);
  }
}

__device__ __forceinline__ uint32_t bits16(int type, float v) {
  return type == LEECH_F16 ? half_bits(v) : bf16_bits(v);
}

__device__ __forceinline__ void store4(const Rows& r, int64_t at, const float v[4]) {
  if (r.type == LEECH_F32) {
    float* p = (float*)r.data + at;
    if (r.wide) {
      *(kv_f32x4*)p = kv_f32x4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) p[t] = v[t];
    }
    return;
  }
  uint16_t* p = (uint16_t*)r.data + at;
  uint32_t h[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) h[t] = bits16(r.type, v[t]);
  if (r.wide) {
    *(kv_u32x2*)p = kv_u32x2{h[0] | h[1] << 16, h[2] | h[3] << 16};
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t) p[t] = (uint16_t)h[t];
  }
}

// An eight's two fours of coordinates: pairs (a, b) of a half-split rotation lie
// width / 2 apart, everything else is consecutive.
__device__ __forceinline__ void item_coords(const Turn& t, int item, int& lo, int& hi) {
  const bool split = !t.interleaved && 8 * item < t.width;
  lo = split ? 4 * item : 8 * item;
  hi = split ? t.width / 2 + 4 * item : 8 * item + 4;
}

// Sines and cosines of an eight's four pairs (of turn.width / 2).
__device__ __forceinline__ void angles(const Turn& t, int64_t position, int item, float c[4],
                                       float s[4]) {
  const double p = (double)position;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    // in turns; 1 / 2π
    double a = p * t.freq[4 * item + j] * 0.15915494309189533577;
    a -= __builtin_rint(a);
    float sn, cs;
    sincospif(2.0f * (float)a, &sn, &cs);
    c[j] = cs * t.cosine;
    s[j] = sn * t.sine;
  }
}

__device__ __forceinline__ void rotate8(const Turn& t, float lo[4], float hi[4], const float c[4],
                                        const float s[4]) {
  if (t.interleaved) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float* v = (j < 2 ? lo : hi) + 2 * (j & 1);
      const float a = v[0], b = v[1];
      v[0] = a * c[j] - b * s[j];
      v[1] = a * s[j] + b * c[j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = lo[j], b = hi[j];
      lo[j] = a * c[j] - b * s[j];
      hi[j] = a * s[j] + b * c[j];
    }
  }
}

// Largest magnitude over groups of N lanes, NaN if any value is not finite.
template <int N>
__device__ __forceinline__ float group_largest(float v) {
#pragma unroll
  for (int m = 1; m < N; m <<= 1) {
    const float o = __shfl_xor(v, m, 64);
    v = o > v || o != o ? o : v;
  }
  return v;
}
__device__ __forceinline__ float larger(float m, float v) {
  const float a = __builtin_fabsf(v);
  return a > m || !(a < __builtin_inff()) ? (a < __builtin_inff() ? a : __builtin_nanf("")) : m;
}

__device__ __forceinline__ float code_scale(int type, float largest) {
  return largest / (type == LEECH_INT8 ? 127.0f : 448.0f);
}
// The code of v: v / scale to the nearest, ties to even; 0 where the scale is 0
// (a row of zeros, or of numbers below the scale's smallest) or not a number.
__device__ __forceinline__ uint32_t code_of(int type, float v, float scale) {
  const float q = scale > 0.0f ? v / scale : 0.0f;
  if (type == LEECH_INT8) {
    const float r = __builtin_rintf(__builtin_fminf(__builtin_fmaxf(q, -127.0f), 127.0f));
    return (uint32_t)(int)r & 0xFFu;
  }
  const float r = __builtin_fminf(__builtin_fmaxf(q, -448.0f), 448.0f);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(r, r, 0, false) & 0xFFu;
}
__device__ __forceinline__ uint32_t codes4(int type, const float v[4], float scale) {
  uint32_t w = 0;
#pragma unroll
  for (int t = 0; t < 4; ++t) w |= code_of(type, v[t], scale) << (8 * t);
  return w;
}
// The number that a code stands for: an f32 product, whatever it is rounded to next.
// (It is made opaque: the compiler otherwise makes one instruction, and one rounding, of
// some of the products and their f16 results, and a key differs from a value of the same
// code and scale.)
__device__ __forceinline__ float code_value(int type, uint32_t code, float scale) {
  float v = scale * (type == LEECH_INT8 ? (float)(int8_t)code
                                        : __builtin_amdgcn_cvt_f32_fp8((int)code, 0));
  asm("" : "+v"(v));
  return v;
}

// ------------------------------------------------------------------- writing
// A key row into its slot; a lane holds eights lane and lane + 16 (ITEMS = 2).
template <int ITEMS>
__device__ __forceinline__ void keep_key(const WriteArgs& a, int64_t slot, int h, int lane,
                                         float lo[ITEMS][4], float hi[ITEMS][4]) {
  const int n_items = a.c.dim / 8;
  const int64_t base = key_at(a.c, slot, h);
  float scale = 0.0f;
  if (type_bytes(a.c.type) == 1) {
    float m = 0.0f;
#pragma unroll
    for (int g = 0; g < ITEMS; ++g)
      if (lane + g * kTeam < n_items)
#pragma unroll
        for (int t = 0; t < 4; ++t) m = larger(larger(m, lo[g][t]), hi[g][t]);
    scale = code_scale(a.c.type, group_largest<kTeam>(m));
    if (lane == 0) a.sk[scale_at(a.c, slot, h)] = scale;
  }
#pragma unroll
  for (int g = 0; g < ITEMS; ++g) {
    const int item = lane + g * kTeam;
    if (item >= n_items) break;
    int d0, d1;
    item_coords(a.turn, item, d0, d1);
    if (type_bytes(a.c.type) == 1) {
      *(uint32_t*)(a.ck + base + d0) = codes4(a.c.type, lo[g], scale);
      *(uint32_t*)(a.ck + base + d1) = codes4(a.c.type, hi[g], scale);
    } else {
      const Rows to = {a.ck, 0, 0, a.c.type, 1};
      store4(to, base + d0, lo[g]);
      store4(to, base + d1, hi[g]);
    }
  }
}

template <int SRC, int ITEMS>
__device__ __forceinline__ void turn_block(const WriteArgs& a, int64_t block) {
  const int team = threadIdx.x / kTeam, lane = threadIdx.x % kTeam;
  const int n_items = a.c.dim / 8;
  const int64_t part = block % a.slices, tokens = block / a.slices;
  const int64_t t = a.by_token ? tokens * kTeams + team : tokens;
  if (t >= a.T) return;
  const int step = a.by_token ? 1 : kTeams;
  const int first = (int)part * a.slice + (a.by_token ? 0 : team);
  const int all = a.q_heads + a.k_heads;
  const int last = (int)part * a.slice + a.slice < all ? (int)part * a.slice + a.slice : all;
  int64_t slot = -1;
  if (a.k_heads) slot = a.slots[t];
  const bool kept = slot >= 0 && slot < a.c.slots;
  int d0[ITEMS], d1[ITEMS];
#pragma unroll
  for (int g = 0; g < ITEMS; ++g) {
    const int item = lane + g * kTeam;
    item_coords(a.turn, item < n_items ? item : 0, d0[g], d1[g]);
  }
  float c[ITEMS][4], s[ITEMS][4];
  for (int h0 = first; h0 < last; h0 += kAtOnce * step) {
    Four<SRC> lo[kAtOnce][ITEMS], hi[kAtOnce][ITEMS];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int h = h0 + u * step;
      if (h >= last) break;
      const bool key = h >= a.q_heads;
      const Rows& from = key ? a.k : a.q;
      const int64_t at = t * from.token + (key ? h - a.q_heads : h) * from.head;
#pragma unroll
      for (int g = 0; g < ITEMS; ++g) {
        lo[u][g] = load4<SRC>(from, at + d0[g]);
        hi[u][g] = load4<SRC>(from, at + d1[g]);
      }
    }
    if (h0 == first)                     // while the first rows are on their way
#pragma unroll
      for (int g = 0; g < ITEMS; ++g)
        if (8 * (lane + g * kTeam) < a.turn.width)
          angles(a.turn, a.positions[t], lane + g * kTeam, c[g], s[g]);
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int h = h0 + u * step;
      if (h >= last) break;
      float vl[ITEMS][4], vh[ITEMS][4];
#pragma unroll
      for (int g = 0; g < ITEMS; ++g) {
        values4<SRC>(lo[u][g], vl[g]);
        values4<SRC>(hi[u][g], vh[g]);
        if (8 * (lane + g * kTeam) < a.turn.width) rotate8(a.turn, vl[g], vh[g], c[g], s[g]);
      }
      if (h >= a.q_heads) {
        if (kept) keep_key<ITEMS>(a, slot, h - a.q_heads, lane, vl, vh);
        continue;
      }
      const int64_t to = t * a.qo.token + h * a.qo.head;
#pragma unroll
      for (int g = 0; g < ITEMS; ++g)
        if (lane + g * kTeam < n_items) {
          store4(a.qo, to + d0[g], vl[g]);
          store4(a.qo, to + d1[g], vh[g]);
        }
    }
  }
}

// The slots around a wave's tokens: lane L has that of token t0 − 16 + L (−1 past
// either end).  Bit L of `joins`: lane L's slot follows lane L − 1's in its run;
// of `heads`: it is the first place of a run.
struct Neighbours {
  int64_t slot;
  uint64_t joins, heads;
};
__device__ __forceinline__ Neighbours neighbours(const int64_t* slots, int64_t T, int64_t all,
                                                 int64_t t0, int run) {
  const int lane = threadIdx.x & 63;
  const int64_t t = t0 - 16 + lane;
  int64_t slot = t >= 0 && t < T ? slots[t] : -1;
  if (slot >= all) slot = -1;
  const int64_t before = __shfl_up(slot, 1, 64);
  const bool inner = slot >= 0 && (slot & (run - 1)) != 0;
  return {slot, __ballot(inner && lane > 0 && slot == before + 1),
          __ballot(slot >= 0 && (slot & (run - 1)) == 0)};
}
// Whether a whole run starts at lane `at`.
__device__ __forceinline__ bool whole_run(const Neighbours& n, int at, int run) {
  const uint64_t rest = ((1ull << (run - 1)) - 1) << (at + 1);
  return (n.heads >> at & 1) && (n.joins & rest) == rest;
}
__device__ __forceinline__ int64_t lane_slot(const Neighbours& n, int at) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(n.slot >> 32), at) << 32 |
                   (uint32_t)__builtin_amdgcn_readlane((int)n.slot, at));
}

// Values of `tokens` tokens and one head, a wave.  A whole run belongs to the wave
// of its first token; a token of no whole run to its own.
template <int SRC, int ITEMS>
__device__ __forceinline__ void value_wave(const WriteArgs& a, int64_t group) {
  const int lane = threadIdx.x & 63, size = type_bytes(a.c.type), run = value_run(a.c.type);
  const int h = (int)(group % a.c.heads);
  const int64_t t0 = group / a.c.heads * a.tokens;
  if (t0 >= a.T) return;
  const Neighbours n = neighbours(a.slots, a.T, a.c.slots, t0, run);
  const int end = 16 + (int)(a.T - t0 < a.tokens ? a.T - t0 : a.tokens);
  for (int at = 16; at < end; ++at) {
    const int64_t slot = lane_slot(n, at);
    if (slot < 0) continue;
    const int64_t t = t0 + at - 16;
    const int place = (int)(slot & (run - 1));
    if (place && at >= place && whole_run(n, at - place, run)) continue;    // another's
    if (place == 0 && whole_run(n, at, run)) {
      const int half = lane >> 5, d = 4 * (lane & 31), mine = run / 2;
      const int64_t base = value_at(a.c, slot, h) * size + 8 * half;
      constexpr int J = 8;
      Four<SRC> w[J][ITEMS];
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int g = 0; g < ITEMS; ++g) {
          const int dd = d + 128 * g;
          if (j < mine)
            w[j][g] = load4<SRC>(a.v, (t + half * mine + j) * a.v.token + h * a.v.head +
                                          (dd < a.c.dim ? dd : 0));
        }
      if (size == 1) {
        float scale[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
          float m = 0.0f;
#pragma unroll
          for (int g = 0; g < ITEMS; ++g) {
            float v[4];
            values4<SRC>(w[j][g], v);
            if (d + 128 * g < a.c.dim)
#pragma unroll
              for (int e = 0; e < 4; ++e) m = larger(m, v[e]);
          }
          scale[j] = code_scale(a.c.type, group_largest<32>(m));
        }
        if ((lane & 31) == 0) {
          float* to = a.sv + scale_at(a.c, slot, h) + 8 * half;
          *(kv_f32x4*)to = kv_f32x4{scale[0], scale[1], scale[2], scale[3]};
          *(kv_f32x4*)(to + 4) = kv_f32x4{scale[4], scale[5], scale[6], scale[7]};
        }
#pragma unroll
        for (int g = 0; g < ITEMS; ++g) {
          if (d + 128 * g >= a.c.dim) break;
          kv_u32x2 o[4] = {{0, 0}, {0, 0}, {0, 0}, {0, 0}};
#pragma unroll
          for (int j = 0; j < J; ++j) {
            float v[4];
            values4<SRC>(w[j][g], v);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e][j >> 2] |= code_of(a.c.type, v[e], scale[j]) << (8 * (j & 3));
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) *(kv_u32x2*)(a.cv + base + 16 * (d + 128 * g + e)) = o[e];
        }
      } else {
#pragma unroll
        for (int g = 0; g < ITEMS; ++g) {
          if (d + 128 * g >= a.c.dim) break;
          kv_u32x2 o[4] = {{0, 0}, {0, 0}, {0, 0}, {0, 0}};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float v[4];
            values4<SRC>(w[j][g], v);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e][j >> 1] |= bits16(a.c.type, v[e]) << (16 * (j & 1));
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) *(kv_u32x2*)(a.cv + base + 16 * (d + 128 * g + e)) = o[e];
        }
      }
      continue;
    }
    // one token: a lane four coordinates
    const int d = 4 * lane;
    float v[4];
    values4<SRC>(load4<SRC>(a.v, t * a.v.token + h * a.v.head + (d < a.c.dim ? d : 0)), v);
    float scale = 0.0f;
    if (size == 1) {
      float m = 0.0f;
      if (d < a.c.dim)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = larger(m, v[e]);
      scale = code_scale(a.c.type, group_largest<64>(m));
      if (lane == 0) a.sv[scale_at(a.c, slot, h)] = scale;
    }
    if (d >= a.c.dim) continue;
    const int64_t base = value_at(a.c, slot, h) + (int64_t)d * run;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (size == 1)
        a.cv[base + e * run] = (uint8_t)code_of(a.c.type, v[e], scale);
      else
        ((uint16_t*)a.cv)[base + e * run] = (uint16_t)bits16(a.c.type, v[e]);
    }
  }
}

// CACHE: the cache's type, LEECH_F32 where there is none (rows only turned).  As an
// argument it cost registers and instructions (4096 bf16 tokens 35.5 us, 32.9 now).
template <int SRC, int ITEMS, int CACHE>
__global__ __launch_bounds__(kThreads) void write_kernel(WriteArgs a) {
  a.c.type = CACHE;
  if constexpr (CACHE == LEECH_F32) a.k_heads = 0;
  if ((int64_t)blockIdx.x < a.turn_blocks)
    turn_block<SRC, ITEMS>(a, blockIdx.x);
  else if constexpr (CACHE != LEECH_F32)
    value_wave<SRC, ITEMS>(a, (blockIdx.x - a.turn_blocks) * kWaves + threadIdx.x / 64);
}

// ------------------------------------------------------------------- reading
// Eight keys' numbers.
__device__ __forceinline__ void values8(int type, const kv_u32x4& w, float scale, float v[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (type_bytes(type) == 1) {
      v[e] = code_value(type, w[e >> 2] >> (8 * (e & 3)) & 0xFFu, scale);
    } else {
      const uint32_t h = w[e >> 1] >> (16 * (e & 1)) & 0xFFFFu;
      v[e] = type == LEECH_F16 ? half_value(h) : bf16_value(h);
    }
  }
}

__device__ __forceinline__ void read_keys(const ReadArgs& a, int64_t block) {
  const int team = threadIdx.x / kTeam, lane = threadIdx.x % kTeam;
  const int size = type_bytes(a.c.type);
  const int64_t rows = a.T * a.c.heads, first = block * kTeams * kAtOnce + team;
  int64_t slot[kAtOnce];
#pragma unroll
  for (int u = 0; u < kAtOnce; ++u) {
    const int64_t row = first + u * kTeams;
    slot[u] = a.slots[(row < rows ? row : first < rows ? first : 0) / a.c.heads];
    if (slot[u] >= a.c.slots) slot[u] = -1;
  }
  for (int item = lane; item < a.c.dim / 8; item += kTeam) {
    kv_u32x4 w[kAtOnce];
    float scale[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int64_t row = first + u * kTeams;
      const int h = (int)(row % a.c.heads);
      const int64_t at = scale_at(a.c, slot[u] < 0 ? 0 : slot[u], h);
      const uint8_t* p = a.ck + (at * a.c.dim + 8 * item) * size;
      w[u] = kv_u32x4{0, 0, 0, 0};
      scale[u] = 1.0f;
      if (size == 1) {
        const kv_u32x2 x = *(const kv_u32x2*)p;
        w[u] = kv_u32x4{x[0], x[1], 0, 0};
        scale[u] = a.sk[at];
      } else {
        w[u] = *(const kv_u32x4*)p;
      }
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int64_t row = first + u * kTeams;
      if (row >= rows) break;
      float v[8];
      values8(a.c.type, w[u], scale[u], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = slot[u] < 0 ? 0.0f : v[e];
      const int64_t to = row / a.c.heads * a.k.token + row % a.c.heads * a.k.head + 8 * item;
      store4(a.k, to, v);
      store4(a.k, to + 4, v + 4);
    }
  }
}

// Values of `tokens` tokens (up to 32) and one head, a wave: run by run, as far as
// consecutive tokens lie in one; half the wave each half of the run's sixteen bytes.
__device__ __forceinline__ void read_values(const ReadArgs& a, int64_t group) {
  const int lane = threadIdx.x & 63, size = type_bytes(a.c.type), run = value_run(a.c.type);
  const int h = (int)(group % a.c.heads);
  const int64_t t0 = group / a.c.heads * a.tokens;
  if (t0 >= a.T) return;
  const Neighbours n = neighbours(a.slots, a.T, a.c.slots, t0, run);
  const int end = 16 + (int)(a.T - t0 < a.tokens ? a.T - t0 : a.tokens);
  const int half = lane >> 5;
  for (int at = 16; at < end;) {
    const int64_t slot = lane_slot(n, at);
    int count = 1;
    if (slot >= 0)
      while (at + count < end && (n.joins >> (at + count) & 1)) ++count;
    const int place = slot < 0 ? half * (run / 2) : (int)(slot & (run - 1));
    const int64_t row = t0 + at - 16;
    at += count;
    const int64_t first = slot < 0 ? 0 : slot - place;
    float scale[8] = {1, 1, 1, 1, 1, 1, 1, 1};
    if (size == 1) {
      const float* p = a.sv + scale_at(a.c, first, h) + 8 * half;
      const kv_f32x4 x = *(const kv_f32x4*)p, y = *(const kv_f32x4*)(p + 4);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        scale[e] = x[e];
        scale[4 + e] = y[e];
      }
    }
    const uint8_t* base = a.cv + value_at(a.c, first, h) * size + 8 * half;
    for (int d = 4 * (lane & 31); d < a.c.dim; d += 128) {
      kv_u32x2 w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = *(const kv_u32x2*)(base + 16 * (d + e));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e0 = half * (run / 2) + j - place;       // the token's, counted from the first
        if (j >= run / 2 || e0 < 0 || e0 >= count) continue;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (size == 1) {
            v[e] = code_value(a.c.type, w[e][j >> 2] >> (8 * (j & 3)) & 0xFFu, scale[j]);
          } else {
            const uint32_t x = w[e][(j >> 1) & 1] >> (16 * (j & 1)) & 0xFFFFu;
            v[e] = a.c.type == LEECH_F16 ? half_value(x) : bf16_value(x);
          }
          if (slot < 0) v[e] = 0.0f;
        }
        store4(a.v, (row + e0) * a.v.token + h * a.v.head + d, v);
      }
    }
  }
}

// The types are the template's: with them read from the arguments a value took 23
// vector instructions, and 30000 int8 tokens of 8 heads 60 us (47 now).
template <int CACHE, int OUT>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a) {
  a.c.type = CACHE;
  a.k.type = a.v.type = OUT;
  if ((int64_t)blockIdx.x < a.key_blocks)
    read_keys(a, blockIdx.x);
  else
    read_values(a, (blockIdx.x - a.key_blocks) * kWaves + threadIdx.x / 64);
}

// ------------------------------------------------------------------ host side
constexpr int64_t kMaxBlocks = ((int64_t)1 << 32) / kThreads - 1;   // a launch's 2^32 threads

bool model_type(int type) { return type == LEECH_F32 || type == LEECH_F16 || type == LEECH_BF16; }

int rows_of(const char* name, const leech_rows* r, int64_t T, int heads, int dim, Rows* out) {
  if (!r || !r->data) return set_error(LEECH_E_ARG, std::string(name) + " is NULL");
  if (!model_type(r->type))
    return set_error(LEECH_E_ARG, std::string(name) + ": type must be f32, f16 or bf16");
  const int size = type_bytes(r->type);
  if ((uintptr_t)r->data % size)
    return set_error(LEECH_E_ARG, std::string(name) + ": misaligned device pointer");
  *out = {r->data, r->token_stride, r->head_stride, r->type,
          (uintptr_t)r->data % (4 * size) == 0 && r->token_stride % 4 == 0 &&
              r->head_stride % 4 == 0};
  return LEECH_OK;
}
int own_rows(const char* name, const Rows& r, int64_t T, int heads, int dim) {
  return rows_apart(r.token, r.head, T, heads, dim)
             ? LEECH_OK
             : set_error(LEECH_E_SHAPE, std::string(name) + ": rows overlap (strides too small)");
}

int turn_of(const leech_rotary* r, int dim, bool transpose, Turn* out) {
  *out = {nullptr, 1.0f, 1.0f, 0, 0};
  if (!r) return LEECH_OK;
  if (!r->freq) return set_error(LEECH_E_ARG, "the rotary's frequencies are NULL");
  if ((uintptr_t)r->freq & 7) return set_error(LEECH_E_ARG, "misaligned frequencies");
  if (r->width <= 0 || r->width % 8 || r->width > dim)
    return set_error(LEECH_E_SHAPE, "the rotated width must be a multiple of 8 up to the head's");
  if (r->interleaved != 0 && r->interleaved != 1)
    return set_error(LEECH_E_ARG, "interleaved must be 0 or 1");
  if (!(r->magnitude > 0.0f) || !(r->magnitude < __builtin_inff()))
    return set_error(LEECH_E_ARG, "the rotary's magnitude must be positive and finite");
  *out = {r->freq, r->magnitude, transpose ? -r->magnitude : r->magnitude, r->width,
          r->interleaved};
  return LEECH_OK;
}

// Teams of a block take as many tokens, or, while tokens are few, heads of one.
void share_out(WriteArgs* a) {
  const int heads = a->q_heads + a->k_heads;
  a->by_token = a->T >= 256;
  a->slice = a->by_token ? 8 : kTeams;
  a->slices = (heads + a->slice - 1) / a->slice;
  a->token_blocks = a->by_token ? (a->T + kTeams - 1) / kTeams : a->T;
  a->turn_blocks = heads ? a->token_blocks * a->slices : 0;
}

typedef void (*ReadFn)(ReadArgs);
template <int CACHE>
ReadFn pick_read(int out) {
  return out == LEECH_F32   ? read_kernel<CACHE, LEECH_F32>
         : out == LEECH_F16 ? read_kernel<CACHE, LEECH_F16>
                            : read_kernel<CACHE, LEECH_BF16>;
}

typedef void (*WriteFn)(WriteArgs);
template <int SRC, int ITEMS>
WriteFn pick_write(int cache) {
  return cache == LEECH_F16    ? write_kernel<SRC, ITEMS, LEECH_F16>
         : cache == LEECH_BF16 ? write_kernel<SRC, ITEMS, LEECH_BF16>
         : cache == LEECH_INT8 ? write_kernel<SRC, ITEMS, LEECH_INT8>
         : cache == LEECH_E4M3 ? write_kernel<SRC, ITEMS, LEECH_E4M3>
                               : write_kernel<SRC, ITEMS, LEECH_F32>;
}
int launch_write(const WriteArgs& a, int src, int64_t blocks, const char* what, void* stream) {
  const bool one = a.c.dim <= 8 * kTeam;
  const WriteFn fn = src == LEECH_F32   ? (one ? pick_write<LEECH_F32, 1>(a.c.type)
                                               : pick_write<LEECH_F32, 2>(a.c.type))
                     : src == LEECH_F16 ? (one ? pick_write<LEECH_F16, 1>(a.c.type)
                                               : pick_write<LEECH_F16, 2>(a.c.type))
                                        : (one ? pick_write<LEECH_BF16, 1>(a.c.type)
                                               : pick_write<LEECH_BF16, 2>(a.c.type));
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LEECH_OK : hip_fail(what, e);
}

}  // namespace

bool rows_apart(int64_t token, int64_t head, int64_t T, int heads, int dim) {
  const int64_t ts = token < 0 ? -token : token, hs = head < 0 ? -head : head;
  return (heads == 1 || hs >= dim) && (T == 1 || ts >= dim) &&
         (heads == 1 || T == 1 || ts >= (heads - 1) * hs + dim || hs >= (T - 1) * ts + dim);
}

int check_cache(const leech_kv_cache* c, CacheShape* shape) {
  if (!c || !c->k || !c->v) return set_error(LEECH_E_ARG, "the cache or a part of it is NULL");
  if (c->type != LEECH_F16 && c->type != LEECH_BF16 && c->type != LEECH_INT8 &&
      c->type != LEECH_E4M3)
    return set_error(LEECH_E_ARG, "a cache's type must be f16, bf16, int8 or e4m3");
  if (type_bytes(c->type) == 1 && (!c->k_scale || !c->v_scale))
    return set_error(LEECH_E_ARG, "an 8-bit cache needs its scales");
  if (c->heads <= 0 || c->heads > 65535)
    return set_error(LEECH_E_SHAPE, "a cache needs 1 to 65535 heads");
  if (c->dim <= 0 || c->dim % 16 || c->dim > kMaxHeadDim)
    return set_error(LEECH_E_SHAPE, "a cache's head dimension must be a multiple of 16 up to 256");
  if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1)))
    return set_error(LEECH_E_SHAPE, "a page must hold a power of two of tokens, 16 to 65536");
  if (c->pages <= 0 || c->pages > 0x7fffffff)
    return set_error(LEECH_E_SHAPE, "a cache needs 1 to 2^31 - 1 pages");
  if (((uintptr_t)c->k & 15) || ((uintptr_t)c->v & 15) || ((uintptr_t)c->k_scale & 15) ||
      ((uintptr_t)c->v_scale & 15))
    return set_error(LEECH_E_ARG, "a cache's pointers must be 16-byte aligned");
  int log_page = 4;
  while (1 << log_page < c->page_size) ++log_page;
  *shape = {c->pages * c->page_size, c->heads, c->dim, log_page, c->type};
  return LEECH_OK;
}

}  // namespace leech

using namespace leech;

extern "C" int leech_rope(int64_t T, int32_t heads, int32_t dim, const leech_rows* x,
                          const int64_t* d_positions, const leech_rotary* rotary, int transpose,
                          const leech_rows* out, void* stream) {
  clear_error();
  if (T < 0 || heads <= 0 || heads > 65535)
    return set_error(LEECH_E_SHAPE, "need T >= 0 and 1 to 65535 heads");
  if (dim <= 0 || dim % 8 || dim > kMaxHeadDim)
    return set_error(LEECH_E_SHAPE, "the head dimension must be a multiple of 8 up to 256");
  if (!rotary) return set_error(LEECH_E_ARG, "the rotary is NULL");
  if (transpose != 0 && transpose != 1) return set_error(LEECH_E_ARG, "transpose must be 0 or 1");
  WriteArgs a = {};
  int rc = turn_of(rotary, dim, transpose != 0, &a.turn);
  if (rc) return rc;
  if (T == 0) return LEECH_OK;
  if (!d_positions || ((uintptr_t)d_positions & 7))
    return set_error(LEECH_E_ARG, "positions are NULL or misaligned");
  if ((rc = rows_of("x", x, T, heads, dim, &a.q)) || (rc = rows_of("out", out, T, heads, dim, &a.qo)) ||
      (rc = own_rows("out", a.qo, T, heads, dim)))
    return rc;
  a.c.dim = dim;
  a.c.type = LEECH_F32;
  a.positions = d_positions;
  a.T = T;
  a.q_heads = heads;
  share_out(&a);
  if (a.turn_blocks > kMaxBlocks) return set_error(LEECH_E_SHAPE, "too many rows for a launch");
  return launch_write(a, a.q.type, a.turn_blocks, "rope launch", stream);
}

extern "C" int leech_cache_write(const leech_kv_cache* cache, int64_t T, const leech_rows* k,
                                 const leech_rows* v, const int64_t* d_slots,
                                 const int64_t* d_positions, const leech_rotary* rotary,
                                 int32_t q_heads, const leech_rows* q, const leech_rows* q_out,
                                 void* stream) {
  clear_error();
  WriteArgs a = {};
  int rc = check_cache(cache, &a.c);
  if (rc || (rc = turn_of(rotary, cache->dim, false, &a.turn))) return rc;
  if (T < 0 || q_heads < 0 || q_heads > 65535)
    return set_error(LEECH_E_SHAPE, "need T >= 0 and 0 to 65535 query heads");
  if (q_heads > 0 && !rotary)
    return set_error(LEECH_E_ARG, "queries are only turned: they need a rotary");
  if (T == 0) return LEECH_OK;
  if (!d_slots || ((uintptr_t)d_slots & 7))
    return set_error(LEECH_E_ARG, "slots are NULL or misaligned");
  if (rotary && (!d_positions || ((uintptr_t)d_positions & 7)))
    return set_error(LEECH_E_ARG, "positions are NULL or misaligned");
  const int heads = cache->heads, dim = cache->dim;
  if ((rc = rows_of("k", k, T, heads, dim, &a.k)) || (rc = rows_of("v", v, T, heads, dim, &a.v)))
    return rc;
  if (q_heads > 0 &&
      ((rc = rows_of("q", q, T, q_heads, dim, &a.q)) ||
       (rc = rows_of("q_out", q_out, T, q_heads, dim, &a.qo)) ||
       (rc = own_rows("q_out", a.qo, T, q_heads, dim))))
    return rc;
  if (a.k.type != a.v.type || (q_heads > 0 && a.q.type != a.k.type))
    return set_error(LEECH_E_ARG, "k, v and q must be of one type");
  a.ck = (uint8_t*)cache->k;
  a.cv = (uint8_t*)cache->v;
  a.sk = cache->k_scale;
  a.sv = cache->v_scale;
  a.slots = d_slots;
  a.positions = d_positions;
  a.T = T;
  a.q_heads = q_heads;
  a.k_heads = heads;
  // a token a wave while waves are few; eight (a run of 16-bit values) make a whole
  // run likely to be one wave's
  a.tokens = T < 512 ? 1 : 8;
  share_out(&a);
  const int64_t blocks = a.turn_blocks + ((T + a.tokens - 1) / a.tokens * heads + kWaves - 1) / kWaves;
  if (T > kMaxBlocks || blocks > kMaxBlocks)
    return set_error(LEECH_E_SHAPE, "too many rows for a launch");
  return launch_write(a, a.k.type, blocks, "cache write launch", stream);
}

extern "C" int leech_cache_read(const leech_kv_cache* cache, int64_t T, const int64_t* d_slots,
                                const leech_rows* k_out, const leech_rows* v_out, void* stream) {
  clear_error();
  ReadArgs a = {};
  int rc = check_cache(cache, &a.c);
  if (rc) return rc;
  if (T < 0) return set_error(LEECH_E_SHAPE, "need T >= 0");
  if (T == 0) return LEECH_OK;
  if (!d_slots || ((uintptr_t)d_slots & 7))
    return set_error(LEECH_E_ARG, "slots are NULL or misaligned");
  const int heads = cache->heads, dim = cache->dim;
  if ((rc = rows_of("k_out", k_out, T, heads, dim, &a.k)) ||
      (rc = rows_of("v_out", v_out, T, heads, dim, &a.v)) ||
      (rc = own_rows("k_out", a.k, T, heads, dim)) || (rc = own_rows("v_out", a.v, T, heads, dim)))
    return rc;
  if (a.k.type != a.v.type) return set_error(LEECH_E_ARG, "k_out and v_out must be of one type");
  a.ck = (const uint8_t*)cache->k;
  a.cv = (const uint8_t*)cache->v;
  a.sk = cache->k_scale;
  a.sv = cache->v_scale;
  a.slots = d_slots;
  a.T = T;
  a.tokens = T < 512 ? 1 : 16;
  a.key_blocks = (T * heads + kTeams * kAtOnce - 1) / (kTeams * kAtOnce);
  const int64_t blocks = a.key_blocks + ((T + a.tokens - 1) / a.tokens * heads + kWaves - 1) / kWaves;
  if (T > kMaxBlocks || blocks > kMaxBlocks)
    return set_error(LEECH_E_SHAPE, "too many rows for a launch");
  const ReadFn fn = cache->type == LEECH_F16    ? pick_read<LEECH_F16>(a.k.type)
                    : cache->type == LEECH_BF16 ? pick_read<LEECH_BF16>(a.k.type)
                    : cache->type == LEECH_INT8 ? pick_read<LEECH_INT8>(a.k.type)
                                                : pick_read<LEECH_E4M3>(a.k.type);
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(kThreads), 0, (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LEECH_OK : hip_fail("cache read launch", e);
}
