// Host side of the attention of new tokens over the caches: argument validation and
// launches (see abi.cpp for the conventions).
#include <algorithm>
#include <cmath>
#include <cstring>

#include "abi_host.h"

using namespace aoh;

namespace {

aoh_status extend_impl(const aoh_tensor* q, const aoh_tensor* k_new, const aoh_tensor* v_new, bool packed,
                       const int32_t* cu_seqlens, int32_t batch, int32_t max_new, const uint8_t* head_is_streaming,
                       const int32_t* start_pos, const aoh_paged_cache* kv_full, const aoh_ring_cache* kv_ring,
                       int32_t n_sink, int32_t window, int32_t evict, int32_t append, aoh_tensor* out, void* workspace,
                       size_t workspace_bytes, void* stream) {
  aoh_status st;
  const int nd = packed ? 3 : 4;
  if ((st = check_tensor(q, "q", nd, AOH_BF16, AOH_F32))) return st;
  const int dt = q->dtype;
  if ((st = check_tensor(k_new, "k_new", nd, dt, dt))) return st;
  if ((st = check_tensor(v_new, "v_new", nd, dt, dt))) return st;
  if ((st = check_tensor(out, "out", nd, dt, AOH_F32))) return st;
  const int64_t Hq = q->shape[nd - 2], Hkv = k_new->shape[nd - 2], D = q->shape[nd - 1];
  for (int i = 0; i < nd; ++i) {
    if (v_new->shape[i] != k_new->shape[i]) return fail(AOH_ERR_INVALID_ARG, "k_new and v_new shapes differ");
    if (i != nd - 2 && k_new->shape[i] != q->shape[i])
      return fail(AOH_ERR_INVALID_ARG, "q and k_new have different tokens or width");
    if (out->shape[i] != q->shape[i]) return fail(AOH_ERR_INVALID_ARG, "out must have the shape of q");
  }
  if (D != 64 && D != 128) return fail(AOH_ERR_UNSUPPORTED, "D=%lld; supported: 64, 128", (long long)D);
  if (Hq % Hkv) return fail(AOH_ERR_UNSUPPORTED, "Hq=%lld is not a multiple of Hkv=%lld", (long long)Hq, (long long)Hkv);
  if (Hq / Hkv > 16) return fail(AOH_ERR_UNSUPPORTED, "Hq/Hkv=%lld > 16", (long long)(Hq / Hkv));
  if (evict != 0 && evict != 1) return fail(AOH_ERR_INVALID_ARG, "evict=%d; must be 0 or 1", evict);
  if (append != 0 && append != 1) return fail(AOH_ERR_INVALID_ARG, "append=%d; must be 0 or 1", append);
  int64_t B = q->shape[0], T = q->shape[1];
  const int64_t tokens = packed ? q->shape[0] : B * T;
  if (B > (1ll << 31) - 1 || T > (1ll << 31) - 1 || tokens > (1ll << 31) - 1) return fail(AOH_ERR_UNSUPPORTED, "too many tokens");
  if (packed) {
    if (!cu_seqlens) return fail(AOH_ERR_INVALID_ARG, "cu_seqlens: null pointer");
    if (batch < 1) return fail(AOH_ERR_INVALID_ARG, "batch=%d must be >= 1", batch);
    if (max_new < 1) return fail(AOH_ERR_INVALID_ARG, "max_new=%d must be >= 1", max_new);
    B = batch;
    T = std::min<int64_t>(max_new, tokens);
  }
  if (T > kMaxTokens) return fail(AOH_ERR_UNSUPPORTED, "%lld tokens a sequence are too many", (long long)T);
  if ((st = check_mask_params(n_sink, window))) return st;
  HeadSchedule hs;
  if ((st = schedule_heads(head_is_streaming, (int)std::min<int64_t>(Hkv, kMaxKvHeads + 1), &hs))) return st;
  if ((st = check_paged(kv_full, hs.n_ret, B))) return st;
  if (hs.n_ret && kv_full->v_token_major)
    return fail(AOH_ERR_UNSUPPORTED, "aoh_extend needs dimension-major V pages (kv_full.v_token_major=0)");
  if ((st = check_ring(kv_ring, hs.n_str, n_sink, window, B))) return st;

  const int cus = std::min(compute_units(), kWsMaxWgs / 2);
  if (dt == AOH_BF16) {
    const size_t need = extend_workspace(B, packed ? std::min(tokens, B * T) : tokens, (int)Hq, (int)Hkv, (int)D, kWsMaxWgs / 2);
    if (!workspace) return fail(AOH_ERR_WORKSPACE, "workspace is null; %zu bytes needed", need);
    if (workspace_bytes < need) return fail(AOH_ERR_WORKSPACE, "workspace has %zu bytes; %zu needed", workspace_bytes, need);
    if (reinterpret_cast<uintptr_t>(workspace) % 16) return fail(AOH_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  }

  // Rows are stored while others still read Q, K and V (of a range taken again, its own Q too).
  const aoh_tensor* inputs[] = {q, k_new, v_new};
  const char* names[] = {"q", "k_new", "v_new"};
  for (int j = 0; j < 3; ++j)
    if (out->data == inputs[j]->data) return fail(AOH_ERR_INVALID_ARG, "out in place of %s; it must overlap no input", names[j]);

  ExtendArgs a;
  std::memset(&a, 0, sizeof(a));
  const int i = nd - 3;  // the token axis
  a.q = q->data; a.k = k_new->data; a.v = v_new->data; a.out = out->data;
  a.q_sb = i ? q->stride[0] : 0; a.q_st = q->stride[i]; a.q_sh = q->stride[i + 1];
  a.k_sb = i ? k_new->stride[0] : 0; a.k_st = k_new->stride[i]; a.k_sh = k_new->stride[i + 1];
  a.v_sb = i ? v_new->stride[0] : 0; a.v_st = v_new->stride[i]; a.v_sh = v_new->stride[i + 1];
  a.o_sb = i ? out->stride[0] : 0; a.o_st = out->stride[i]; a.o_sh = out->stride[i + 1];
  a.start_pos = start_pos;
  if (packed) {
    a.cu_seqlens = cu_seqlens;
    a.total = (int)tokens;
  }
  a.B = (int)B; a.T = (int)T; a.Hq = (int)Hq; a.gs = (int)(Hq / Hkv);
  a.n_sink = n_sink; a.window = window; a.ring_cap = n_sink + window;
  a.evict = evict;
  a.out_f32 = out->dtype == AOH_F32;
  a.scale = (float)(1.0 / std::sqrt((double)D));
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)D));
  if (hs.n_ret) {
    a.pk = kv_full->k; a.pv = kv_full->v; a.block_table = kv_full->block_table;
    a.max_pages = kv_full->max_pages_per_seq; a.num_pages = (int)kv_full->num_pages; a.n_ret = hs.n_ret;
  }
  if (hs.n_str) {
    a.rk = kv_ring->k; a.rv = kv_ring->v; a.n_str = hs.n_str;
    a.ring_blocks = (int)ceil_div(kv_ring->capacity, kPageTokens);
  }
  a.streaming_mask = hs.streaming_mask;
  std::memcpy(a.rank, hs.rank, sizeof(a.rank));
  std::memcpy(a.kv_heads, hs.ret, hs.n_ret);
  std::memcpy(a.kv_heads + hs.n_ret, hs.str, hs.n_str);
  a.gs_mul = ((1ull << 36) + a.gs - 1) / a.gs;
  a.workspace = workspace;
  a.cus = cus;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  hipError_t e = launch_extend(a, dt, (int)D, s);
  if (e != hipSuccess) return fail(AOH_ERR_HIP, "extend launch: %s", hipGetErrorString(e));
  if (append) {
    RopeArgs r;  // no norm and no rotation: a copy
    std::memset(&r, 0, sizeof(r));
    r.k = a.k; r.k_sb = a.k_sb; r.k_st = a.k_st; r.k_sh = a.k_sh;
    r.v = a.v; r.v_sb = a.v_sb; r.v_st = a.v_st; r.v_sh = a.v_sh;
    r.start_pos = start_pos; r.cu_seqlens = a.cu_seqlens; r.total = a.total;
    r.B = a.B; r.T = a.T; r.Hkv = (int)Hkv;
    if (hs.n_ret) {
      r.pk = kv_full->k; r.pv = kv_full->v; r.block_table = a.block_table;
      r.max_pages = a.max_pages; r.num_pages = a.num_pages; r.n_ret = a.n_ret;
    }
    if (hs.n_str) {
      r.rk = kv_ring->k; r.rv = kv_ring->v; r.n_str = a.n_str; r.ring_blocks = a.ring_blocks;
    }
    r.n_sink = n_sink; r.window = window;
    r.streaming_mask = hs.streaming_mask;
    std::memcpy(r.rank, hs.rank, sizeof(r.rank));
    e = launch_rope(r, dt, (int)D, true, s);
    if (e != hipSuccess) return fail(AOH_ERR_HIP, "append launch: %s", hipGetErrorString(e));
  }
  return ok();
}

}  // namespace

extern "C" {

size_t aoh_extend_workspace_bytes(int32_t batch, int64_t n_tokens, int32_t n_q_heads, int32_t n_kv_heads, int32_t d_head) {
  if (batch < 1 || n_tokens < 1 || n_tokens > (1ll << 31) - 1 || n_kv_heads < 1 || n_q_heads < n_kv_heads || n_q_heads % n_kv_heads ||
      n_q_heads / n_kv_heads > 16 || (d_head != 64 && d_head != 128))
    return 0;
  return extend_workspace(batch, n_tokens, n_q_heads, n_kv_heads, d_head, kWsMaxWgs / 2);
}

aoh_status aoh_extend(const aoh_tensor* q, const aoh_tensor* k_new, const aoh_tensor* v_new,
                      const uint8_t* head_is_streaming, const int32_t* start_pos, const aoh_paged_cache* kv_full,
                      const aoh_ring_cache* kv_ring, int32_t n_sink, int32_t window, int32_t evict, int32_t append,
                      aoh_tensor* out, void* workspace, size_t workspace_bytes, void* stream) {
  return extend_impl(q, k_new, v_new, false, nullptr, 0, 0, head_is_streaming, start_pos, kv_full, kv_ring, n_sink,
                     window, evict, append, out, workspace, workspace_bytes, stream);
}

aoh_status aoh_extend_varlen(const aoh_tensor* q, const aoh_tensor* k_new, const aoh_tensor* v_new,
                             const int32_t* cu_seqlens, int32_t batch, int32_t max_new,
                             const uint8_t* head_is_streaming, const int32_t* start_pos, const aoh_paged_cache* kv_full,
                             const aoh_ring_cache* kv_ring, int32_t n_sink, int32_t window, int32_t evict, int32_t append,
                             aoh_tensor* out, void* workspace, size_t workspace_bytes, void* stream) {
  return extend_impl(q, k_new, v_new, true, cu_seqlens, batch, max_new, head_is_streaming, start_pos, kv_full, kv_ring,
                     n_sink, window, evict, append, out, workspace, workspace_bytes, stream);
}

}  // extern "C"
