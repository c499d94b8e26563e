// Host side of the head norms and position rotation, and of the appends that apply them:
// argument validation and launches (see abi.cpp for the conventions).
#include <algorithm>
#include <cmath>
#include <cstring>

#include "abi_host.h"

using namespace aoh;

namespace {

constexpr int64_t kMaxRopeRows = 1 << 27;

aoh_status check_norm(const aoh_tensor* w, const char* name, int dtype, int64_t D) {
  if (!w) return AOH_OK;
  aoh_status st;
  if ((st = check_tensor(w, name, 1, dtype, AOH_F32))) return st;
  if (w->shape[0] != D) return fail(AOH_ERR_INVALID_ARG, "%s must have D=%lld weights", name, (long long)D);
  return AOH_OK;
}

// Norms, rotation and positions of rows of width D.
aoh_status fill_rope(const aoh_tensor* q_norm, const aoh_tensor* k_norm, float eps, const aoh_rope* rope,
                     const int32_t* positions, int64_t tokens, int dtype, int64_t D, RopeArgs* a) {
  aoh_status st;
  if (D != 64 && D != 128) return fail(AOH_ERR_UNSUPPORTED, "D=%lld; supported: 64, 128", (long long)D);
  if ((st = check_norm(q_norm, "q_norm", dtype, D))) return st;
  if ((st = check_norm(k_norm, "k_norm", dtype, D))) return st;
  if (q_norm && k_norm && q_norm->dtype != k_norm->dtype)
    return fail(AOH_ERR_INVALID_ARG, "q_norm and k_norm have different dtypes");
  if (!(eps >= 0.f) || std::isinf(eps)) return fail(AOH_ERR_INVALID_ARG, "eps=%g must be >= 0 and finite", (double)eps);
  if (q_norm) a->q_norm = q_norm->data;
  if (k_norm) a->k_norm = k_norm->data;
  a->norm_f32 = (q_norm ? q_norm->dtype : k_norm ? k_norm->dtype : AOH_F32) == AOH_F32;
  a->eps = eps;
  if (!rope) {
    if (positions) return fail(AOH_ERR_INVALID_ARG, "positions without a rotation");
    return AOH_OK;
  }
  if (!rope->inv_freq) return fail(AOH_ERR_INVALID_ARG, "rope.inv_freq: null pointer");
  if (rope->n_pairs < 1 || rope->n_pairs > D / 2)
    return fail(AOH_ERR_INVALID_ARG, "rope.n_pairs=%d outside [1, %lld]", rope->n_pairs, (long long)D / 2);
  if (rope->n_axes < 1 || rope->n_axes > 4) return fail(AOH_ERR_UNSUPPORTED, "rope.n_axes=%d outside [1, 4]", rope->n_axes);
  if (rope->interleaved != 0 && rope->interleaved != 1)
    return fail(AOH_ERR_INVALID_ARG, "rope.interleaved=%d; must be 0 or 1", rope->interleaved);
  if (!std::isfinite(rope->scale)) return fail(AOH_ERR_INVALID_ARG, "rope.scale must be finite");
  if (rope->axis)
    for (int i = 0; i < rope->n_pairs; ++i) {
      if (rope->axis[i] >= rope->n_axes)
        return fail(AOH_ERR_INVALID_ARG, "rope.axis[%d]=%d; there are %d axes", i, (int)rope->axis[i], rope->n_axes);
      a->axis[i] = rope->axis[i];
    }
  if (!positions && rope->n_axes > 1) return fail(AOH_ERR_INVALID_ARG, "positions: null pointer, for %d axes", rope->n_axes);
  if (reinterpret_cast<uintptr_t>(rope->inv_freq) % 4 || reinterpret_cast<uintptr_t>(positions) % 4)
    return fail(AOH_ERR_INVALID_ARG, "rope.inv_freq and positions must be 4-byte aligned");
  a->inv_freq = rope->inv_freq;
  a->n_pairs = rope->n_pairs;
  a->interleaved = rope->interleaved;
  a->scale = rope->scale;
  a->positions = positions;
  a->pos_stride = tokens;
  return AOH_OK;
}

// An output of the input's shape and dtype; in place only as the very same view.
aoh_status check_out(const aoh_tensor* in, const aoh_tensor* out, const char* name) {
  aoh_status st;
  if ((st = check_tensor(out, name, in->ndim, in->dtype, in->dtype))) return st;
  for (int i = 0; i < in->ndim; ++i)
    if (out->shape[i] != in->shape[i]) return fail(AOH_ERR_INVALID_ARG, "%s must have its input's shape", name);
  if (out->data == in->data)
    for (int i = 0; i < in->ndim; ++i)
      if (out->stride[i] != in->stride[i] && in->shape[i] > 1)
        return fail(AOH_ERR_INVALID_ARG, "%s: in place, but with other strides than its input", name);
  return AOH_OK;
}

// Strides of [B][T][H][D], or of packed [total][H][D] (batch stride 0).
void strides(const aoh_tensor* t, int64_t* sb, int64_t* st, int64_t* sh) {
  const int i = t->ndim - 3;
  *sb = i ? t->stride[0] : 0;
  *st = t->stride[i];
  *sh = t->stride[i + 1];
}

aoh_status append_impl(const aoh_tensor* q, const aoh_tensor* k_new, const aoh_tensor* v_new, bool packed,
                       const int32_t* cu_seqlens, int32_t batch, int32_t max_new, const aoh_tensor* q_norm,
                       const aoh_tensor* k_norm, float eps, const aoh_rope* rope, const int32_t* positions,
                       const uint8_t* head_is_streaming, const int32_t* start_pos, const aoh_paged_cache* kv_full,
                       const aoh_ring_cache* kv_ring, int32_t n_sink, int32_t window, aoh_tensor* q_out, void* stream) {
  aoh_status st;
  const int nd = packed ? 3 : 4;
  if ((st = check_tensor(k_new, "k_new", nd, AOH_BF16, AOH_F32))) return st;
  const int dt = k_new->dtype;
  if ((st = check_tensor(v_new, "v_new", nd, dt, dt))) return st;
  for (int i = 0; i < nd; ++i)
    if (v_new->shape[i] != k_new->shape[i]) return fail(AOH_ERR_INVALID_ARG, "k_new and v_new shapes differ");
  if (!q != !q_out) return fail(AOH_ERR_INVALID_ARG, "q and q_out: one of them is null");
  if (!q && q_norm) return fail(AOH_ERR_INVALID_ARG, "q_norm without q");
  const int64_t D = k_new->shape[nd - 1], Hkv = k_new->shape[nd - 2];
  RopeArgs a;
  std::memset(&a, 0, sizeof(a));
  if (q) {
    if ((st = check_tensor(q, "q", nd, dt, dt))) return st;
    for (int i = 0; i < nd; ++i)
      if (i != nd - 2 && q->shape[i] != k_new->shape[i]) return fail(AOH_ERR_INVALID_ARG, "q and k_new have different tokens or width");
    if ((st = check_out(q, q_out, "q_out"))) return st;
    if (q->shape[nd - 2] > (1 << 20)) return fail(AOH_ERR_UNSUPPORTED, "too many query heads");
    a.q = q->data; a.q_out = q_out->data;
    strides(q, &a.q_sb, &a.q_st, &a.q_sh);
    strides(q_out, &a.qo_sb, &a.qo_st, &a.qo_sh);
    a.Hq = (int)q->shape[nd - 2];
  }
  int64_t B = k_new->shape[0], n_new = k_new->shape[1];
  const int64_t tokens = packed ? k_new->shape[0] : B * n_new;
  if (tokens > (1ll << 31) - 1) return fail(AOH_ERR_UNSUPPORTED, "too many tokens");
  if (packed) {
    if (!cu_seqlens) return fail(AOH_ERR_INVALID_ARG, "cu_seqlens: null pointer");
    if (batch < 1) return fail(AOH_ERR_INVALID_ARG, "batch=%d must be >= 1", batch);
    if (max_new < 1) return fail(AOH_ERR_INVALID_ARG, "max_new=%d must be >= 1", max_new);
    B = batch;
    n_new = std::min<int64_t>(max_new, tokens);
    a.cu_seqlens = cu_seqlens;
    a.total = (int)tokens;
  }
  if (n_new > kMaxTokens) return fail(AOH_ERR_UNSUPPORTED, "%lld tokens a sequence are too many", (long long)n_new);
  if ((st = fill_rope(q_norm, k_norm, eps, rope, positions, tokens, dt, D, &a))) return st;
  if ((st = check_mask_params(n_sink, window))) return st;
  HeadSchedule hs;
  if ((st = schedule_heads(head_is_streaming, (int)std::min<int64_t>(Hkv, kMaxKvHeads + 1), &hs))) return st;
  if ((st = check_paged(kv_full, hs.n_ret, B))) return st;
  if ((st = check_ring(kv_ring, hs.n_str, n_sink, window, B))) return st;
  a.k = k_new->data; a.v = v_new->data;
  strides(k_new, &a.k_sb, &a.k_st, &a.k_sh);
  strides(v_new, &a.v_sb, &a.v_st, &a.v_sh);
  a.start_pos = start_pos;
  a.B = (int)B; a.T = (int)n_new; a.Hkv = (int)Hkv;
  if (hs.n_ret) {
    a.pk = kv_full->k; a.pv = kv_full->v; a.block_table = kv_full->block_table;
    a.max_pages = kv_full->max_pages_per_seq; a.num_pages = (int)kv_full->num_pages; a.n_ret = hs.n_ret;
    a.v_token_major = kv_full->v_token_major;
  }
  if (hs.n_str) {
    a.rk = kv_ring->k; a.rv = kv_ring->v; a.n_str = hs.n_str;
    a.ring_blocks = (int)ceil_div(kv_ring->capacity, kPageTokens);
  }
  a.n_sink = n_sink; a.window = window;
  a.streaming_mask = hs.streaming_mask;
  std::memcpy(a.rank, hs.rank, sizeof(a.rank));
  hipError_t e = launch_rope(a, dt, (int)D, true, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(AOH_ERR_HIP, "append launch: %s", hipGetErrorString(e));
  return ok();
}

}  // namespace

extern "C" {

aoh_status aoh_qk_rope(const aoh_tensor* q, const aoh_tensor* k, const aoh_tensor* q_norm, const aoh_tensor* k_norm,
                       float eps, const aoh_rope* rope, const int32_t* positions, const int32_t* start_pos,
                       aoh_tensor* q_out, aoh_tensor* k_out, void* stream) {
  aoh_status st;
  if (!q && !k) return fail(AOH_ERR_INVALID_ARG, "q and k are both null");
  if (!q != !q_out) return fail(AOH_ERR_INVALID_ARG, "q and q_out: one of them is null");
  if (!k != !k_out) return fail(AOH_ERR_INVALID_ARG, "k and k_out: one of them is null");
  if ((q_norm && !q) || (k_norm && !k)) return fail(AOH_ERR_INVALID_ARG, "a norm without its rows");
  if (!rope && !q_norm && !k_norm) return fail(AOH_ERR_INVALID_ARG, "neither a rotation nor a norm");
  const aoh_tensor* one = q ? q : k;
  RopeArgs a;
  std::memset(&a, 0, sizeof(a));
  if (q) {
    if ((st = check_tensor(q, "q", 4, AOH_BF16, AOH_F32))) return st;
    if ((st = check_out(q, q_out, "q_out"))) return st;
    a.q = q->data; a.q_out = q_out->data;
    strides(q, &a.q_sb, &a.q_st, &a.q_sh);
    strides(q_out, &a.qo_sb, &a.qo_st, &a.qo_sh);
    a.Hq = (int)q->shape[2];
  }
  if (k) {
    if ((st = check_tensor(k, "k", 4, q ? q->dtype : AOH_BF16, q ? q->dtype : AOH_F32))) return st;
    if ((st = check_out(k, k_out, "k_out"))) return st;
    a.k = k->data; a.k_out = k_out->data;
    strides(k, &a.k_sb, &a.k_st, &a.k_sh);
    strides(k_out, &a.ko_sb, &a.ko_st, &a.ko_sh);
    a.Hkv = (int)k->shape[2];
  }
  if (q && k && (q->shape[0] != k->shape[0] || q->shape[1] != k->shape[1] || q->shape[3] != k->shape[3]))
    return fail(AOH_ERR_INVALID_ARG, "q and k have different tokens or width");
  for (const aoh_tensor* t : {q, k})
    if (t && t->shape[2] > (1 << 20)) return fail(AOH_ERR_UNSUPPORTED, "too many heads");
  const int64_t B = one->shape[0], T = one->shape[1];
  if (B > kMaxRopeRows || T > kMaxRopeRows || B * T > kMaxRopeRows) return fail(AOH_ERR_UNSUPPORTED, "too many tokens");
  if ((st = fill_rope(q_norm, k_norm, eps, rope, positions, B * T, one->dtype, one->shape[3], &a))) return st;
  a.start_pos = start_pos;
  a.B = (int)B; a.T = (int)T;
  hipError_t e = launch_rope(a, one->dtype, (int)one->shape[3], false, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(AOH_ERR_HIP, "rotation launch: %s", hipGetErrorString(e));
  return ok();
}

aoh_status aoh_kv_append_rope(const aoh_tensor* q, const aoh_tensor* k_new, const aoh_tensor* v_new,
                              const aoh_tensor* q_norm, const aoh_tensor* k_norm, float eps, const aoh_rope* rope,
                              const int32_t* positions, const uint8_t* head_is_streaming, const int32_t* start_pos,
                              const aoh_paged_cache* kv_full, const aoh_ring_cache* kv_ring, int32_t n_sink,
                              int32_t window, aoh_tensor* q_out, void* stream) {
  return append_impl(q, k_new, v_new, false, nullptr, 0, 0, q_norm, k_norm, eps, rope, positions, head_is_streaming,
                     start_pos, kv_full, kv_ring, n_sink, window, q_out, stream);
}

aoh_status aoh_kv_append_rope_varlen(const aoh_tensor* q, const aoh_tensor* k_new, const aoh_tensor* v_new,
                                     const int32_t* cu_seqlens, int32_t batch, int32_t max_new, const aoh_tensor* q_norm,
                                     const aoh_tensor* k_norm, float eps, const aoh_rope* rope, const int32_t* positions,
                                     const uint8_t* head_is_streaming, const int32_t* start_pos,
                                     const aoh_paged_cache* kv_full, const aoh_ring_cache* kv_ring, int32_t n_sink,
                                     int32_t window, aoh_tensor* q_out, void* stream) {
  return append_impl(q, k_new, v_new, true, cu_seqlens, batch, max_new, q_norm, k_norm, eps, rope, positions,
                     head_is_streaming, start_pos, kv_full, kv_ring, n_sink, window, q_out, stream);
}

}  // extern "C"
