// Attention of new tokens over the paged key/value cache for gfx950.
//
// A wave owns one query row (a token's query head) and walks the keys it sees
// in blocks of 64, a lane a key: scores, their running maximum and sum (one
// pass: what is summed so far is scaled down when the maximum grows), then the
// weighted values, a lane a coordinate.

#include "kv_device.h"

namespace leech {
namespace {

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
  float scale;
};

__device__ __forceinline__ int64_t start_of(const AttendArgs& a, int b) {
  const int64_t s = a.q_start ? a.q_start[b] : b;
  return s < 0 ? 0 : s > a.T ? a.T : s;
}

__device__ __forceinline__ float element(const uint8_t* p, int type, int64_t at) {
  if (type == LEECH_INT8) return (float)((const int8_t*)p)[at];
  if (type == LEECH_E4M3) return __builtin_amdgcn_cvt_f32_fp8((int)p[at], 0);
  const uint32_t h = ((const uint16_t*)p)[at];
  return type == LEECH_F16 ? half_value(h) : bf16_value(h);
}

__global__ __launch_bounds__(64) void attend_kernel(AttendArgs a) {
  __shared__ float qs[kMaxHeadDim];
  __shared__ float ws[64];
  __shared__ int64_t where[64];
  const int lane = threadIdx.x, h = blockIdx.y, d0 = a.c.dim;
  const int64_t t = blockIdx.x;
  int lo = 0, hi = a.B;                     // the last sequence that starts at or before t
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (start_of(a, mid + 1) <= t)
      lo = mid + 1;
    else
      hi = mid;
  }
  if (lo >= a.B || start_of(a, lo) > t) return;
  const int64_t first = start_of(a, lo), n = start_of(a, lo + 1) - first, i = t - first;
  if (i >= a.max_new) return;
  int64_t len = a.kv_len[lo];
  const int64_t room = (int64_t)a.table_pages << a.c.log_page;
  len = len < 0 ? 0 : len > room ? room : len;
  const int64_t p = len - n + i;
  const int64_t to = a.causal && p + 1 < len ? p + 1 : len;
  int64_t from = a.window ? p - a.window + 1 : 0;
  if (from < 0) from = 0;
  const int type = a.c.type;
  for (int d = lane; d < d0; d += 64) {
    const uint32_t x = a.q[t * a.q_token + h * a.q_head + d];
    qs[d] = a.type == LEECH_F16 ? half_value(x) : bf16_value(x);
  }
  __syncthreads();
  float m = -__builtin_inff(), l = 0.0f, o[4] = {0, 0, 0, 0};
  const int kh = h / a.group;
  for (int64_t j0 = from; j0 < to; j0 += 64) {
    const int64_t j = j0 + lane;
    float s = -__builtin_inff();
    int64_t slot = -1;
    if (j < to) {
      const int64_t page = a.table[lo * a.table_stride + (j >> a.c.log_page)];
      if (page < 0 || page >= a.pages) {
        s = __builtin_nanf("");
      } else {
        slot = (page << a.c.log_page) + (j & ((1 << a.c.log_page) - 1));
        const int64_t at = key_at(a.c, slot, kh);
        s = 0.0f;
        for (int d = 0; d < d0; ++d) s += qs[d] * element(a.ck, type, at + d);
        s *= a.scale;
        if (type_bytes(type) == 1) s *= a.sk[scale_at(a.c, slot, kh)];
      }
    }
    float top = s;
    for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    const float mn = fmaxf(m, top);
    const float base = mn == -__builtin_inff() ? 0.0f : mn;
    const float w = j < to ? expf(s - base) : 0.0f, old = expf(m - base);
    float sum = w;
    for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x, 64);
    l = l * old + sum;
    m = mn;
    __syncthreads();
    ws[lane] = slot >= 0 && type_bytes(type) == 1 ? w * a.sv[scale_at(a.c, slot, kh)] : w;
    where[lane] = slot;
    __syncthreads();
    for (int e = 0; e < 4; ++e) {
      const int d = lane + 64 * e;
      if (d >= d0) break;
      float x = o[e] * old;
      for (int k = 0; k < 64 && j0 + k < to; ++k)
        x += where[k] < 0 ? ws[k]
                          : ws[k] * element(a.cv, type,
                                            value_at(a.c, where[k], kh) + d * value_run(type));
      o[e] = x;
    }
  }
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;     // a NaN sum stays one
  for (int e = 0; e < 4; ++e) {
    const int d = lane + 64 * e;
    if (d < d0)
      a.out[t * a.o_token + h * a.o_head + d] =
          (uint16_t)(a.type == LEECH_F16 ? half_bits(o[e] * inv) : bf16_bits(o[e] * inv));
  }
  if (a.lse && lane == 0) a.lse[t * a.q_heads + h] = l != 0.0f ? m + logf(l) : -__builtin_inff();
}

// ------------------------------------------------------------------ host side
// Sizes alone: what the workspace goes by.
int check_sizes(const leech_kv_cache* cache, const leech_attend_args* g, CacheShape* shape) {
  const int rc = check_cache(cache, shape);
  if (rc) return rc;
  if (!g) return set_error(LEECH_E_ARG, "the arguments are NULL");
  if (g->type != LEECH_F16 && g->type != LEECH_BF16)
    return set_error(LEECH_E_ARG, "queries must be f16 or bf16");
  if (type_bytes(cache->type) == 2 && cache->type != g->type)
    return set_error(LEECH_E_ARG, "a 16-bit cache must have the queries' type");
  if (g->q_heads <= 0 || g->q_heads > 65535 || g->q_heads % cache->heads)
    return set_error(LEECH_E_SHAPE, "query heads must be a multiple of the cache's, up to 65535");
  if (g->T < 0 || g->T > 0x7fffffff || g->B < 0 || g->max_new < 0)
    return set_error(LEECH_E_SHAPE, "T, B and max_new must be 0 to 2^31 - 1");
  if (g->table_pages < 0 || ((int64_t)g->table_pages << shape->log_page) > 0x7fffffff)
    return set_error(LEECH_E_SHAPE, "a row of the page table holds at most 2^31 - 1 tokens");
  if (!g->q_start && g->T != g->B)
    return set_error(LEECH_E_SHAPE, "without q_start there is one new token a sequence");
  return LEECH_OK;
}

int check_strides(const char* name, const void* p, int64_t token, int64_t head) {
  if (!p) return set_error(LEECH_E_ARG, std::string(name) + " is NULL");
  if (((uintptr_t)p & 15) || token % 8 || head % 8)
    return set_error(LEECH_E_ARG, std::string(name) +
                                      ": needs 16-byte alignment and strides of 8 elements");
  return LEECH_OK;
}

}  // namespace
}  // namespace leech

using namespace leech;

extern "C" int leech_attend_workspace(const leech_kv_cache* cache, const leech_attend_args* args,
                                      size_t* bytes) {
  clear_error();
  CacheShape shape;
  const int rc = check_sizes(cache, args, &shape);
  if (rc) return rc;
  if (!bytes) return set_error(LEECH_E_ARG, "bytes is NULL");
  *bytes = 0;
  return LEECH_OK;
}

extern "C" int leech_attend(const leech_kv_cache* cache, const leech_attend_args* g,
                            void* stream) {
  clear_error();
  AttendArgs a = {};
  int rc = check_sizes(cache, g, &a.c);
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
  a.scale = g->scale;
  hipLaunchKernelGGL(attend_kernel, dim3((unsigned)a.T, (unsigned)a.q_heads), dim3(64), 0,
                     (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? LEECH_OK : hip_fail("attend launch", e);
}
