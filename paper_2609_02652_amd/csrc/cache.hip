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
// Geometry.  Teams of sixteen lanes own a row (one head of one token), a lane
// eight coordinates at a time: four pairs where the rotation reaches.  A team
// keeps its token and walks over heads, so a sine is computed once for several
// of them.  Value rows go through LDS, tile by tile of consecutive tokens: where
// value_run tokens fill a run of slots the tile writes sixteen bytes at once,
// anywhere else element by element.

#include "kv_device.h"

namespace leech {
namespace {

constexpr int kThreads = 256;
constexpr int kTeam = 16;                 // lanes of a row
constexpr int kTeams = kThreads / kTeam;
constexpr int kItems = kMaxHeadDim / 8 / kTeam;   // eights of coordinates a lane owns
constexpr int kSpare = 15;                // tokens a tile reads past its own

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
  int32_t tile;                           // tokens of a value tile
};

struct ReadArgs {
  CacheShape c;
  const uint8_t *ck, *cv;
  const float *sk, *sv;
  const int64_t* slots;
  Rows k, v;
  int64_t T, key_blocks;
  int32_t tile;
};

__device__ __forceinline__ void load4(const Rows& r, int64_t at, float v[4]) {
  if (r.type == LEECH_F32) {
    const float* p = (const float*)r.data + at;
    if (r.wide) {
      const kv_f32x4 w = *(const kv_f32x4*)p;
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = w[t];
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) v[t] = p[t];
    }
    return;
  }
  const uint16_t* p = (const uint16_t*)r.data + at;
  uint32_t h[4];
  if (r.wide) {
    const kv_u32x2 w = *(const kv_u32x2*)p;
#pragma unroll
    for (int t = 0; t < 4; ++t) h[t] = w[t >> 1] >> (16 * (t & 1)) & 0xFFFFu;
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t) h[t] = p[t];
  }
  const bool half = r.type == LEECH_F16;
#pragma unroll
  for (int t = 0; t < 4; ++t) v[t] = half ? half_value(h[t]) : bf16_value(h[t]);
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

// Largest magnitude over a team's lanes, NaN if any value is not finite.
__device__ __forceinline__ float team_largest(float v) {
#pragma unroll
  for (int m = 1; m < kTeam; m <<= 1) {
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
__device__ __forceinline__ float code_value(int type, uint32_t code) {
  if (type == LEECH_INT8) return (float)(int8_t)code;
  return __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}

// ------------------------------------------------------------------- writing
// A key row into its slot.
__device__ __forceinline__ void keep_key(const WriteArgs& a, int64_t slot, int h, int n_items,
                                         int lane, float lo[kItems][4], float hi[kItems][4]) {
  const int64_t base = key_at(a.c, slot, h);
  float scale = 0.0f;
  if (type_bytes(a.c.type) == 1) {
    float m = 0.0f;
#pragma unroll
    for (int g = 0; g < kItems; ++g)
      if (lane + g * kTeam < n_items)
#pragma unroll
        for (int t = 0; t < 4; ++t) m = larger(larger(m, lo[g][t]), hi[g][t]);
    scale = code_scale(a.c.type, team_largest(m));
    if (lane == 0) a.sk[scale_at(a.c, slot, h)] = scale;
  }
#pragma unroll
  for (int g = 0; g < kItems; ++g) {
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
  float c[kItems][4], s[kItems][4];
#pragma unroll
  for (int g = 0; g < kItems; ++g)
    if (8 * (lane + g * kTeam) < a.turn.width)
      angles(a.turn, a.positions[t], lane + g * kTeam, c[g], s[g]);
  int64_t slot = -1;
  if (a.k_heads) slot = a.slots[t];
  for (int h = first; h < last; h += step) {
    const bool key = h >= a.q_heads;
    if (key && (slot < 0 || slot >= a.c.slots)) continue;
    const Rows& from = key ? a.k : a.q;
    const int64_t at = t * from.token + (key ? h - a.q_heads : h) * from.head;
    float lo[kItems][4], hi[kItems][4];
#pragma unroll
    for (int g = 0; g < kItems; ++g) {
      const int item = lane + g * kTeam;
      if (item >= n_items) continue;
      int d0, d1;
      item_coords(a.turn, item, d0, d1);
      load4(from, at + d0, lo[g]);
      load4(from, at + d1, hi[g]);
    }
#pragma unroll
    for (int g = 0; g < kItems; ++g)
      if (8 * (lane + g * kTeam) < a.turn.width) rotate8(a.turn, lo[g], hi[g], c[g], s[g]);
    if (key) {
      keep_key(a, slot, h - a.q_heads, n_items, lane, lo, hi);
      continue;
    }
    const int64_t to = t * a.qo.token + h * a.qo.head;
#pragma unroll
    for (int g = 0; g < kItems; ++g) {
      const int item = lane + g * kTeam;
      if (item >= n_items) continue;
      int d0, d1;
      item_coords(a.turn, item, d0, d1);
      store4(a.qo, to + d0, lo[g]);
      store4(a.qo, to + d1, hi[g]);
    }
  }
}

// Whether tokens t .. t + run - 1 exist and fill a run of slots that starts at
// slot (of token t), itself the first place of a run.
__device__ __forceinline__ bool fills_run(const int64_t* slots, int64_t T, int64_t all, int64_t t,
                                          int run) {
  if (t < 0 || t + run > T) return false;
  const int64_t s = slots[t];
  if (s < 0 || s + run > all || (s & (run - 1))) return false;
  for (int j = 1; j < run; ++j)
    if (slots[t + j] != s + j) return false;
  return true;
}

// Value rows of a tile of tokens and one head.  A tile writes the runs that
// start at its own tokens (it reads up to run - 1 tokens past them for that)
// and those of its tokens that lie in no filled run.
__device__ __forceinline__ void value_block(const WriteArgs& a, int64_t block, uint8_t* tile) {
  const int team = threadIdx.x / kTeam, lane = threadIdx.x % kTeam;
  const int size = type_bytes(a.c.type), run = value_run(a.c.type);
  const int dim = a.c.dim, n_items = dim / 8, pitch = dim * size + 4;
  const int h = (int)(block % a.c.heads);
  const int64_t t0 = block / a.c.heads * a.tile;
  const int own = (int)(a.T - t0 < a.tile ? a.T - t0 : a.tile);
  const int held = (int)(a.T - t0 < own + run - 1 ? a.T - t0 : own + run - 1);
  // per token: whether it starts a run that its tile writes whole (1), or is
  // written by itself (2), or lies in such a run (0)
  uint8_t* how = tile + (a.tile + kSpare) * pitch;
  for (int i = threadIdx.x; i < own; i += kThreads) {
    const int64_t t = t0 + i, slot = a.slots[t];
    const int place = (int)(slot & (run - 1));
    uint8_t w = 0;
    if (slot >= 0 && slot < a.c.slots) {
      if (!fills_run(a.slots, a.T, a.c.slots, t - place, run))
        w = 2;
      else if (place == 0)
        w = 1;
    }
    how[i] = w;
  }
  for (int i = team; i < held; i += kTeams) {
    const int64_t t = t0 + i, slot = a.slots[t];
    if (slot < 0 || slot >= a.c.slots) continue;
    const int64_t at = t * a.v.token + h * a.v.head;
    float v[kItems][8];
    float m = 0.0f;
#pragma unroll
    for (int g = 0; g < kItems; ++g) {
      const int item = lane + g * kTeam;
      if (item >= n_items) continue;
      load4(a.v, at + 8 * item, v[g]);
      load4(a.v, at + 8 * item + 4, v[g] + 4);
#pragma unroll
      for (int e = 0; e < 8; ++e) m = larger(m, v[g][e]);
    }
    float scale = 0.0f;
    if (size == 1) {
      scale = code_scale(a.c.type, team_largest(m));
      if (lane == 0 && i < own) a.sv[scale_at(a.c, slot, h)] = scale;
    }
#pragma unroll
    for (int g = 0; g < kItems; ++g) {
      const int item = lane + g * kTeam;
      if (item >= n_items) continue;
      uint32_t* to = (uint32_t*)(tile + i * pitch + 8 * item * size);
      if (size == 1) {
        to[0] = codes4(a.c.type, v[g], scale);
        to[1] = codes4(a.c.type, v[g] + 4, scale);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          to[e] = bits16(a.c.type, v[g][2 * e]) | bits16(a.c.type, v[g][2 * e + 1]) << 16;
      }
    }
  }
  __syncthreads();
  const int wave = threadIdx.x / 64, l = threadIdx.x % 64;
  for (int i = wave; i < own; i += kThreads / 64) {
    const int w = how[i];
    if (w == 0) continue;
    const int64_t base = value_at(a.c, a.slots[t0 + i], h);
    for (int d = l; d < dim; d += 64) {
      const uint8_t* from = tile + i * pitch + d * size;
      if (w == 2) {
        if (size == 1)
          a.cv[base + (int64_t)d * run] = *from;
        else
          *(uint16_t*)(a.cv + 2 * (base + (int64_t)d * run)) = *(const uint16_t*)from;
        continue;
      }
      kv_u32x4 o;
      if (size == 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t x = 0;
#pragma unroll
          for (int b = 0; b < 4; ++b) x |= (uint32_t)from[(4 * e + b) * pitch] << (8 * b);
          o[e] = x;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          o[e] = (uint32_t) * (const uint16_t*)(from + 2 * e * pitch) |
                 (uint32_t) * (const uint16_t*)(from + (2 * e + 1) * pitch) << 16;
      }
      *(kv_u32x4*)(a.cv + size * (base + (int64_t)d * run)) = o;
    }
  }
}

__global__ __launch_bounds__(kThreads) void write_kernel(WriteArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t tile[];
  if ((int64_t)blockIdx.x < a.turn_blocks)
    turn_block(a, blockIdx.x);
  else
    value_block(a, blockIdx.x - a.turn_blocks, tile);
}

// ------------------------------------------------------------------- reading
__device__ __forceinline__ void values8(int type, const uint8_t* p, float v[8]) {
  if (type_bytes(type) == 1) {
    const kv_u32x2 w = *(const kv_u32x2*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = code_value(type, w[e >> 2] >> (8 * (e & 3)) & 0xFFu);
  } else {
    const kv_u32x4 w = *(const kv_u32x4*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t h = w[e >> 1] >> (16 * (e & 1)) & 0xFFFFu;
      v[e] = type == LEECH_F16 ? half_value(h) : bf16_value(h);
    }
  }
}

__device__ __forceinline__ void put_row(const ReadArgs& a, const Rows& to, int64_t t, int h,
                                        bool valid, const uint8_t* row, float scale, int lane) {
  const int size = type_bytes(a.c.type);
  const int64_t at = t * to.token + h * to.head;
  for (int item = lane; item < a.c.dim / 8; item += kTeam) {
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (valid) {
      values8(a.c.type, row + 8 * item * size, v);
      if (size == 1)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= scale;
    }
    store4(to, at + 8 * item, v);
    store4(to, at + 8 * item + 4, v + 4);
  }
}

__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t tile[];
  const int team = threadIdx.x / kTeam, lane = threadIdx.x % kTeam;
  const int size = type_bytes(a.c.type), run = value_run(a.c.type), dim = a.c.dim;
  if ((int64_t)blockIdx.x < a.key_blocks) {
    const int64_t row = (int64_t)blockIdx.x * kTeams + team;
    if (row >= a.T * a.c.heads) return;
    const int64_t t = row / a.c.heads;
    const int h = (int)(row % a.c.heads);
    const int64_t slot = a.slots[t];
    const bool valid = slot >= 0 && slot < a.c.slots;
    put_row(a, a.k, t, h, valid, valid ? a.ck + size * key_at(a.c, slot, h) : nullptr,
            valid && size == 1 ? a.sk[scale_at(a.c, slot, h)] : 0.0f, lane);
    return;
  }
  const int64_t block = blockIdx.x - a.key_blocks;
  const int h = (int)(block % a.c.heads);
  const int64_t t0 = block / a.c.heads * a.tile;
  const int own = (int)(a.T - t0 < a.tile ? a.T - t0 : a.tile);
  const int pitch = dim * size + 16;
  // A token leads if it does not lie behind its predecessor in one run; the
  // leader reads the run's sixteen bytes for those that follow it there.
  const int wave = threadIdx.x / 64, l = threadIdx.x % 64;
  for (int i = wave; i < own; i += kThreads / 64) {
    const int64_t slot = a.slots[t0 + i];
    if (slot < 0 || slot >= a.c.slots) continue;
    const int place = (int)(slot & (run - 1));
    if (i > 0 && place > 0 && a.slots[t0 + i - 1] == slot - 1) continue;
    int n = 1;
    while (place + n < run && i + n < own && a.slots[t0 + i + n] == slot + n) ++n;
    const int64_t base = value_at(a.c, slot - place, h);
    for (int d = l; d < dim; d += 64) {
      const kv_u32x4 w = *(const kv_u32x4*)(a.cv + size * (base + (int64_t)d * run));
      for (int j = 0; j < n; ++j) {
        const int e = place + j;
        uint8_t* to = tile + (i + j) * pitch + d * size;
        const uint32_t x = e * size < 4 ? w[0] : e * size < 8 ? w[1] : e * size < 12 ? w[2] : w[3];
        if (size == 1)
          *to = (uint8_t)(x >> (8 * (e & 3)));
        else
          *(uint16_t*)to = (uint16_t)(x >> (16 * (e & 1)));
      }
    }
  }
  __syncthreads();
  for (int i = team; i < own; i += kTeams) {
    const int64_t t = t0 + i, slot = a.slots[t];
    const bool valid = slot >= 0 && slot < a.c.slots;
    put_row(a, a.v, t, h, valid, tile + i * pitch,
            valid && size == 1 ? a.sv[scale_at(a.c, slot, h)] : 0.0f, lane);
  }
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
  a.positions = d_positions;
  a.T = T;
  a.q_heads = heads;
  share_out(&a);
  if (a.turn_blocks > kMaxBlocks) return set_error(LEECH_E_SHAPE, "too many rows for a launch");
  hipLaunchKernelGGL(write_kernel, dim3((unsigned)a.turn_blocks), dim3(kThreads), 0,
                     (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LEECH_OK : hip_fail("rope launch", e);
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
  a.ck = (uint8_t*)cache->k;
  a.cv = (uint8_t*)cache->v;
  a.sk = cache->k_scale;
  a.sv = cache->v_scale;
  a.slots = d_slots;
  a.positions = d_positions;
  a.T = T;
  a.q_heads = q_heads;
  a.k_heads = heads;
  a.tile = T < 256 ? 16 : 64;
  share_out(&a);
  const int64_t blocks = a.turn_blocks + (T + a.tile - 1) / a.tile * heads;
  if (blocks > kMaxBlocks) return set_error(LEECH_E_SHAPE, "too many rows for a launch");
  const size_t lds = (size_t)(a.tile + kSpare) * (dim * type_bytes(a.c.type) + 4) + a.tile;
  hipLaunchKernelGGL(write_kernel, dim3((unsigned)blocks), dim3(kThreads), lds,
                     (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LEECH_OK : hip_fail("cache write launch", e);
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
  a.ck = (const uint8_t*)cache->k;
  a.cv = (const uint8_t*)cache->v;
  a.sk = cache->k_scale;
  a.sv = cache->v_scale;
  a.slots = d_slots;
  a.T = T;
  a.tile = T < 256 ? 16 : 64;
  a.key_blocks = (T * heads + kTeams - 1) / kTeams;
  const int64_t blocks = a.key_blocks + (T + a.tile - 1) / a.tile * heads;
  if (T > kMaxBlocks || blocks > kMaxBlocks)
    return set_error(LEECH_E_SHAPE, "too many rows for a launch");
  const size_t lds = (size_t)a.tile * (dim * type_bytes(a.c.type) + 16);
  hipLaunchKernelGGL(read_kernel, dim3((unsigned)blocks), dim3(kThreads), lds,
                     (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LEECH_OK : hip_fail("cache read launch", e);
}
