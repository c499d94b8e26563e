// Host side of the 8-bit caches' entry points: argument validation and launch
// plans (see abi.cpp for the conventions).
#include <algorithm>
#include <cmath>
#include <cstring>

#include "abi_host.h"

using namespace aoh;

namespace {

size_t align16(size_t x) { return (x + 15) & ~(size_t)15; }

aoh_status check_caches(const aoh_paged_cache_q8* full, const aoh_ring_cache_q8* ring, const HeadSchedule& hs,
                        int n_sink, int window, int64_t B, int* format) {
  aoh_status st;
  if (full) {
    const aoh_paged_cache c = {full->k, full->v, full->block_table, full->num_pages, full->max_pages_per_seq,
                               full->n_heads, full->n_seqs, 0};
    if ((st = check_paged(&c, hs.n_ret, B))) return st;
  } else if ((st = check_paged(nullptr, hs.n_ret, B))) {
    return st;
  }
  if (ring) {
    const aoh_ring_cache c = {ring->k, ring->v, ring->n_heads, ring->capacity, ring->batch};
    if ((st = check_ring(&c, hs.n_str, n_sink, window, B))) return st;
  } else if ((st = check_ring(nullptr, hs.n_str, n_sink, window, B))) {
    return st;
  }
  *format = -1;
  struct Use { bool on; const void* scales; int32_t format; const char* name; };
  const Use uses[2] = {{hs.n_ret > 0, full ? full->scales : nullptr, full ? full->format : 0, "kv_full"},
                       {hs.n_str > 0, ring ? ring->scales : nullptr, ring ? ring->format : 0, "kv_ring"}};
  for (const Use& u : uses) {
    if (!u.on) continue;
    if (!u.scales) return fail(AOH_ERR_INVALID_ARG, "%s: null pointer", u.name);
    if (reinterpret_cast<uintptr_t>(u.scales) % 16)
      return fail(AOH_ERR_INVALID_ARG, "%s: cache pointers must be 16-byte aligned", u.name);
    if (u.format != AOH_E4M3 && u.format != AOH_I8)
      return fail(AOH_ERR_UNSUPPORTED, "%s: format %d is not an 8-bit one", u.name, u.format);
    if (*format >= 0 && *format != u.format)
      return fail(AOH_ERR_INVALID_ARG, "kv_full and kv_ring have different formats");
    *format = u.format;
  }
  return AOH_OK;
}

// The caches, heads and mask of a write or read of n tokens a sequence.
aoh_status fill_args(const aoh_paged_cache_q8* full, const aoh_ring_cache_q8* ring, const uint8_t* head_is_streaming,
                     int n_sink, int window, int64_t B, int64_t n, int64_t Hkv, int64_t D, Q8Args* a, int* format) {
  aoh_status st;
  if (D != 64 && D != 128) return fail(AOH_ERR_UNSUPPORTED, "D=%lld; supported: 64, 128", (long long)D);
  if (n > kMaxTokens) return fail(AOH_ERR_UNSUPPORTED, "%lld tokens a sequence are too many", (long long)n);
  if (B > (1ll << 31) - 1) return fail(AOH_ERR_UNSUPPORTED, "batch too large");
  if ((st = check_mask_params(n_sink, window))) return st;
  HeadSchedule hs;
  if ((st = schedule_heads(head_is_streaming, (int)std::min<int64_t>(Hkv, kMaxKvHeads + 1), &hs))) return st;
  if ((st = check_caches(full, ring, hs, n_sink, window, B, format))) return st;
  a->B = (int)B; a->n = (int)n;
  if (hs.n_ret) {
    a->pk = static_cast<uint8_t*>(full->k); a->pv = static_cast<uint8_t*>(full->v); a->ps = full->scales;
    a->block_table = full->block_table;
    a->max_pages = full->max_pages_per_seq; a->num_pages = (int)full->num_pages; a->n_ret = hs.n_ret;
  }
  if (hs.n_str) {
    a->rk = static_cast<uint8_t*>(ring->k); a->rv = static_cast<uint8_t*>(ring->v); a->rs = ring->scales;
    a->n_str = hs.n_str;
    a->ring_blocks = (int)ceil_div(ring->capacity, kPageTokens);
  }
  a->n_sink = n_sink; a->window = window;
  std::memcpy(a->ret, hs.ret, hs.n_ret);
  std::memcpy(a->str, hs.str, hs.n_str);
  return AOH_OK;
}

// k and v as [B][n][Hkv][D], or packed [total][Hkv][D].
void fill_tensors(const aoh_tensor* k, const aoh_tensor* v, Q8Args* a) {
  a->k = k->data; a->v = v->data;
  const int t = k->ndim - 3;  // the token axis
  a->k_sb = t ? k->stride[0] : 0; a->k_st = k->stride[t]; a->k_sh = k->stride[t + 1];
  a->v_sb = t ? v->stride[0] : 0; a->v_st = v->stride[t]; a->v_sh = v->stride[t + 1];
}

// Number of split partials (rows of gs heads) and of int32 places that the two
// split passes use; see DecodeArgs.
size_t ws_bytes(int64_t rows, int64_t ints, int64_t d) {
  return align16((size_t)rows * (d + 2) * sizeof(float)) + (size_t)ints * sizeof(int32_t);
}

size_t decode_need(int64_t batch, int64_t hq, int64_t d) {
  const int64_t gs = std::min<int64_t>(hq, 16), few = std::min<int64_t>(batch, kWsMaxBatch);
  return std::max(ws_bytes(kWsMaxWgs * gs + few * hq, 2 * few * hq, d), ws_bytes(2 * kWsMaxWgs * gs, 4 * kWsMaxWgs, d));
}

// Whether a step is split by the pass for many items (decode_split.h), which starts
// later (its tables) and merges the workgroups of an item one after the other, but
// holds whole items, so it saves partials (of all query heads) at every item.  us a
// step, work-space pass / many, half of the heads streaming, window 512, 300-6000 tokens
// a sequence, then 2000-30000.  Width 128, 64 items of four heads 16.8 / 23.1, 33.3 / 40.9,
// 128 of four 25.2 / 24.4, 58.1 / 58.3, of seven 29.9 / 25.5, 62.9 / 60.1, 256 of one
// 31.8 / 33.2, 97.5 / 98.3, of two 35.2 / 33.2, 101.0 / 98.4, 32 of sixteen 18.4 / 27.4,
// 27.7 / 58.4.  Width 64, 128 of four 16.9 / 17.8, 33.3 / 34.9, 256 of one 20.7 / 22.4,
// 54.2 / 53.8, of four 25.3 / 22.8, 58.4 / 54.2, of two 22.2 / 22.3, 55.9 / 54.8.
// In caches of 32 blocks and fewer no item is in many workgroups (200-400 tokens,
// window 256).  Width 128, 64 items of four heads 12.1 / 13.0, of seven 14.6 / 13.3, 60 of
// eight 15.3 / 13.2, 32 of sixteen 15.5 / 16.4, 128 of four 17.7 / 13.5; width 64, 64 of
// seven 11.3 / 11.9, 60 of sixteen 14.6 / 12.1, 128 of four 12.2 / 11.3.
// The host knows the capacity only, not the lengths: short sequences in wide block
// tables are judged as long ones (64 of 100-1000 tokens, two KV heads of width 64, 32
// query heads: 22.7 here, 15.2 with many), and one long sequence among short ones, whose
// many partials the other pass merges one after the other, loses where few KV heads
// share it (64 sequences, one of 100000 tokens and 63 of 100-1000, two KV heads of
// width 128, 32 query heads: 46.8 / 114.2; eight KV heads: 78.0 / 67.9).
bool takes_many(int64_t B, int64_t Hkv, int gs, int D, int64_t blocks) {
  if (B > kWsMaxBatch) return true;
  const int64_t items = B * Hkv;
  if (blocks <= 32) return items >= 48 && items * gs >= 448;
  return items >= (D == 128 ? 128 : 256) && items * gs >= 512;
}

aoh_status decode_impl(const aoh_tensor* q, const aoh_tensor* k_new, const aoh_tensor* v_new, bool step,
                       const aoh_paged_cache_q8* full, const aoh_ring_cache_q8* ring, const uint8_t* head_is_streaming,
                       const int32_t* lens, int32_t n_sink, int32_t window, aoh_tensor* out, void* workspace,
                       size_t workspace_bytes, void* stream) {
  aoh_status st;
  if ((st = check_tensor(q, "q", 3, AOH_BF16, AOH_BF16))) return st;
  if ((st = check_tensor(out, "out", 3, AOH_BF16, AOH_F32))) return st;
  const int64_t B = q->shape[0], Hq = q->shape[1], D = q->shape[2];
  if (out->shape[0] != B || out->shape[1] != Hq || out->shape[2] != D)
    return fail(AOH_ERR_INVALID_ARG, "out must have the shape of q");
  if (D != 64 && D != 128) return fail(AOH_ERR_UNSUPPORTED, "D=%lld; supported: 64, 128", (long long)D);
  if (B > (1ll << 31) - 1) return fail(AOH_ERR_UNSUPPORTED, "batch too large");
  if (!lens) return fail(AOH_ERR_INVALID_ARG, "lens: null pointer");
  if ((st = check_mask_params(n_sink, window))) return st;
  const int64_t Hkv = (int64_t)(full ? full->n_heads : 0) + (ring ? ring->n_heads : 0);
  if (Hkv < 1) return fail(AOH_ERR_INVALID_ARG, "no cache given");
  if (Hq % Hkv) return fail(AOH_ERR_UNSUPPORTED, "Hq=%lld is not a multiple of Hkv=%lld", (long long)Hq, (long long)Hkv);
  HeadSchedule hs;
  if ((st = schedule_heads(head_is_streaming, (int)std::min<int64_t>(Hkv, kMaxKvHeads + 1), &hs))) return st;
  int format;
  if ((st = check_caches(full, ring, hs, n_sink, window, B, &format))) return st;
  const int gs = (int)(Hq / Hkv);
  if (gs > 16) return fail(AOH_ERR_UNSUPPORTED, "Hq/Hkv=%d > 16", gs);
  if (step) {
    if ((st = check_tensor(k_new, "k_new", 3, AOH_BF16, AOH_BF16))) return st;
    if ((st = check_tensor(v_new, "v_new", 3, AOH_BF16, AOH_BF16))) return st;
    for (const aoh_tensor* t : {k_new, v_new})
      if (t->shape[0] != B || t->shape[1] != Hkv || t->shape[2] != D)
        return fail(AOH_ERR_INVALID_ARG, "k_new / v_new must be [B=%lld][Hkv=%lld][D=%lld]", (long long)B,
                    (long long)Hkv, (long long)D);
  }
  const size_t need = decode_need(B, Hq, D);
  if (!workspace) return fail(AOH_ERR_WORKSPACE, "workspace is null; %zu bytes needed", need);
  if (workspace_bytes < need) return fail(AOH_ERR_WORKSPACE, "workspace has %zu bytes; %zu needed", workspace_bytes, need);
  if (reinterpret_cast<uintptr_t>(workspace) % 16) return fail(AOH_ERR_INVALID_ARG, "workspace must be 16-byte aligned");

  const int ring_cap = n_sink + window;
  const int ring_blocks = (int)ceil_div(ring_cap, kPageTokens);
  const int64_t blocks = std::max<int64_t>(hs.n_ret ? full->max_pages_per_seq : 0, hs.n_str ? ring_blocks : 0);
  // places of a launch's work space stay below 2^29: larger batches go in parts
  const int64_t part = std::min<int64_t>(kManyMaxBatch, ((1ll << 29) - 1) / (Hkv * (blocks + 16)));
  if (part < 1) return fail(AOH_ERR_UNSUPPORTED, "%lld KV heads of %lld blocks are too many", (long long)Hkv, (long long)blocks);

  const int cu = std::min(compute_units(), kWsMaxWgs / 2);
  const int out_es = out->dtype == AOH_F32 ? 4 : 2;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  for (int64_t b0 = 0; b0 < B; b0 += part) {
    const int64_t nb = std::min(part, B - b0);
    DecodeArgs a;
    std::memset(&a, 0, sizeof(a));
    a.q = static_cast<const char*>(q->data) + b0 * q->stride[0] * 2; a.q_sb = q->stride[0]; a.q_sh = q->stride[1];
    a.lens = lens + b0;
    a.B = (int)nb; a.Hq = (int)Hq; a.gs = gs;
    a.ring_cap = ring_cap;
    a.empty = 0.f;
    a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)D));
    a.out = static_cast<char*>(out->data) + b0 * out->stride[0] * out_es; a.o_sb = out->stride[0]; a.o_sh = out->stride[1];
    a.out_f32 = out->dtype == AOH_F32;
    if (hs.n_ret) {
      CacheView& c = a.full;
      c.k = full->k; c.v = full->v; c.scales = full->scales;
      c.block_table = full->block_table + b0 * full->max_pages_per_seq;
      c.max_pages = full->max_pages_per_seq; c.num_pages = (int)full->num_pages;
      c.n_kv = hs.n_ret;
      std::memcpy(c.kv_heads, hs.ret, hs.n_ret);
    }
    if (hs.n_str) {
      CacheView& c = a.ring;
      const int64_t units = b0 * hs.n_str * ring_blocks;
      c.k = static_cast<const uint8_t*>(ring->k) + units * kPageTokens * D;
      c.v = static_cast<const uint8_t*>(ring->v) + units * kPageTokens * D;
      c.scales = ring->scales + units * 2 * kPageTokens;
      c.ring_blocks = ring_blocks;
      c.n_kv = hs.n_str;
      std::memcpy(c.kv_heads, hs.str, hs.n_str);
    }
    if (step) {
      a.k_new = static_cast<const char*>(k_new->data) + b0 * k_new->stride[0] * 2;
      a.v_new = static_cast<const char*>(v_new->data) + b0 * v_new->stride[0] * 2;
      a.kn_sb = k_new->stride[0]; a.kn_sh = k_new->stride[1];
      a.vn_sb = v_new->stride[0]; a.vn_sh = v_new->stride[1];
      a.n_sink = n_sink; a.window = window;
    }
    a.ws_cu = cu;
    int64_t rows = (2 * cu + nb * Hkv) * gs;
    if (takes_many(nb, Hkv, gs, (int)D, blocks)) {
      a.many_wgs = 2 * cu;
      rows = (int64_t)4 * cu * gs;
    }
    a.part_acc = static_cast<float*>(workspace);
    a.part_ml = a.part_acc + rows * D;
    a.ws_items = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + ws_bytes(rows, 0, D));
    hipError_t e = launch_decode_q8_split(a, (int)D, format, s);
    if (e != hipSuccess) return fail(AOH_ERR_HIP, "decode split launch: %s", hipGetErrorString(e));
    MergeArgs m;
    std::memset(&m, 0, sizeof(m));
    m.part_acc = a.part_acc; m.part_ml = a.part_ml; m.lens = a.lens;
    m.out = a.out; m.o_sb = a.o_sb; m.o_sh = a.o_sh;
    m.B = (int)nb; m.Hq = (int)Hq; m.gs = gs;
    m.max_len = hs.n_ret ? full->max_pages_per_seq * kPageTokens : 0;
    m.ring_cap = ring_cap;
    m.empty = a.empty;
    m.many_wgs = a.many_wgs;
    m.ws_cu = a.ws_cu; m.ws_n_ret = hs.n_ret; m.ws_n_str = hs.n_str; m.ws_items = a.ws_items;
    m.streaming_mask = hs.streaming_mask;
    e = launch_decode_merge(m, AOH_BF16, a.out_f32, (int)D, s);
    if (e != hipSuccess) return fail(AOH_ERR_HIP, "decode merge launch: %s", hipGetErrorString(e));
  }
  return ok();
}

}  // namespace

extern "C" {

aoh_status aoh_kv_append_q8(const aoh_tensor* k_new, const aoh_tensor* v_new, const uint8_t* head_is_streaming,
                            const int32_t* start_pos, const aoh_paged_cache_q8* kv_full,
                            const aoh_ring_cache_q8* kv_ring, int32_t n_sink, int32_t window, void* stream) {
  aoh_status st;
  if ((st = check_tensor(k_new, "k_new", 4, AOH_BF16, AOH_F32))) return st;
  if ((st = check_tensor(v_new, "v_new", 4, k_new->dtype, k_new->dtype))) return st;
  for (int i = 0; i < 4; ++i)
    if (v_new->shape[i] != k_new->shape[i]) return fail(AOH_ERR_INVALID_ARG, "k_new and v_new shapes differ");
  Q8Args a;
  std::memset(&a, 0, sizeof(a));
  int format;
  if ((st = fill_args(kv_full, kv_ring, head_is_streaming, n_sink, window, k_new->shape[0], k_new->shape[1],
                      k_new->shape[2], k_new->shape[3], &a, &format)))
    return st;
  fill_tensors(k_new, v_new, &a);
  a.start_pos = start_pos;
  hipError_t e = launch_q8(a, k_new->dtype, format, (int)k_new->shape[3], true, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(AOH_ERR_HIP, "append launch: %s", hipGetErrorString(e));
  return ok();
}

aoh_status aoh_kv_append_q8_varlen(const aoh_tensor* k_new, const aoh_tensor* v_new, const int32_t* cu_seqlens,
                                   int32_t batch, int32_t max_new, const uint8_t* head_is_streaming,
                                   const int32_t* start_pos, const aoh_paged_cache_q8* kv_full,
                                   const aoh_ring_cache_q8* kv_ring, int32_t n_sink, int32_t window, void* stream) {
  aoh_status st;
  if ((st = check_tensor(k_new, "k_new", 3, AOH_BF16, AOH_F32))) return st;
  if ((st = check_tensor(v_new, "v_new", 3, k_new->dtype, k_new->dtype))) return st;
  for (int i = 0; i < 3; ++i)
    if (v_new->shape[i] != k_new->shape[i]) return fail(AOH_ERR_INVALID_ARG, "k_new and v_new shapes differ");
  if (!cu_seqlens) return fail(AOH_ERR_INVALID_ARG, "cu_seqlens: null pointer");
  if (batch < 1) return fail(AOH_ERR_INVALID_ARG, "batch=%d must be >= 1", batch);
  if (max_new < 1) return fail(AOH_ERR_INVALID_ARG, "max_new=%d must be >= 1", max_new);
  const int64_t total = k_new->shape[0];
  if (total > (1ll << 31) - 1) return fail(AOH_ERR_UNSUPPORTED, "too many packed tokens");
  Q8Args a;
  std::memset(&a, 0, sizeof(a));
  int format;
  if ((st = fill_args(kv_full, kv_ring, head_is_streaming, n_sink, window, batch, std::min<int64_t>(max_new, total),
                      k_new->shape[1], k_new->shape[2], &a, &format)))
    return st;
  fill_tensors(k_new, v_new, &a);
  a.start_pos = start_pos; a.cu_seqlens = cu_seqlens; a.total = (int)total;
  hipError_t e = launch_q8(a, k_new->dtype, format, (int)k_new->shape[2], true, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(AOH_ERR_HIP, "append launch: %s", hipGetErrorString(e));
  return ok();
}

aoh_status aoh_kv_read_q8(const aoh_paged_cache_q8* kv_full, const aoh_ring_cache_q8* kv_ring,
                          const uint8_t* head_is_streaming, const int32_t* start_pos, const int32_t* lens,
                          int32_t n_sink, int32_t window, aoh_tensor* k_out, aoh_tensor* v_out, void* stream) {
  aoh_status st;
  if ((st = check_tensor(k_out, "k_out", 4, AOH_BF16, AOH_F32))) return st;
  if ((st = check_tensor(v_out, "v_out", 4, k_out->dtype, k_out->dtype))) return st;
  for (int i = 0; i < 4; ++i)
    if (v_out->shape[i] != k_out->shape[i]) return fail(AOH_ERR_INVALID_ARG, "k_out and v_out shapes differ");
  if (!lens) return fail(AOH_ERR_INVALID_ARG, "lens: null pointer");
  Q8Args a;
  std::memset(&a, 0, sizeof(a));
  int format;
  if ((st = fill_args(kv_full, kv_ring, head_is_streaming, n_sink, window, k_out->shape[0], k_out->shape[1],
                      k_out->shape[2], k_out->shape[3], &a, &format)))
    return st;
  fill_tensors(k_out, v_out, &a);
  a.start_pos = start_pos; a.lens = lens;
  hipError_t e = launch_q8(a, k_out->dtype, format, (int)k_out->shape[3], false, reinterpret_cast<hipStream_t>(stream));
  if (e != hipSuccess) return fail(AOH_ERR_HIP, "read launch: %s", hipGetErrorString(e));
  return ok();
}

size_t aoh_decode_q8_workspace_bytes(int32_t batch, int32_t n_q_heads, int32_t d_head) {
  if (batch < 1 || n_q_heads < 1 || (d_head != 64 && d_head != 128)) return 0;
  return decode_need(batch, n_q_heads, d_head);
}

aoh_status aoh_decode_q8(const aoh_tensor* q, const aoh_paged_cache_q8* kv_full, const aoh_ring_cache_q8* kv_ring,
                         const uint8_t* head_is_streaming, const int32_t* lens, int32_t n_sink, int32_t window,
                         aoh_tensor* out, void* workspace, size_t workspace_bytes, void* stream) {
  return decode_impl(q, nullptr, nullptr, false, kv_full, kv_ring, head_is_streaming, lens, n_sink, window, out,
                     workspace, workspace_bytes, stream);
}

aoh_status aoh_decode_step_q8(const aoh_tensor* q, const aoh_tensor* k_new, const aoh_tensor* v_new,
                              const aoh_paged_cache_q8* kv_full, const aoh_ring_cache_q8* kv_ring,
                              const uint8_t* head_is_streaming, const int32_t* lens, int32_t n_sink, int32_t window,
                              aoh_tensor* out, void* workspace, size_t workspace_bytes, void* stream) {
  return decode_impl(q, k_new, v_new, true, kv_full, kv_ring, head_is_streaming, lens, n_sink, window, out, workspace,
                     workspace_bytes, stream);
}

}  // extern "C"
