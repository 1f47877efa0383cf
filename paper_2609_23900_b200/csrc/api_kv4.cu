// extern "C" entry points around the paged 4-bit cache: argument checking and launch orchestration.
#include <cuda_runtime.h>

#include <climits>
#include <cstring>

#include "api_common.h"

using namespace lumo;

namespace {

// Last of the checks of every call: all that is wrong with the arguments is said on a host-only context too.
int launchable(lumo_ctx* ctx) { return ctx->device < 0 ? fail(ctx, LUMO_ERR_UNSUPPORTED, "host-only context cannot launch") : (int)LUMO_OK; }

// Common checks of the calls on the 4-bit cache; fills the shape shared by all layers.  desc is null for the calls that list tokens.
int prepare_kv4(lumo_ctx* ctx, const lumo_tree_desc* desc, bool tree, const lumo_kv4_args* layers, int n_layers, Kv4Shape* s) {
  if (!ctx || (tree && !desc) || !layers) return fail(ctx, LUMO_ERR_ARG, "null ctx, desc or layers");
  if (tree && desc->ctx != ctx) return fail(ctx, LUMO_ERR_ARG, "descriptor belongs to another context");
  if (n_layers < 1 || n_layers > kMaxAttnLayers)
    return fail(ctx, LUMO_ERR_ARG, "n_layers must be in [1, " + std::to_string(kMaxAttnLayers) + "]");
  if (tree && desc->Ns > kMaxAttnSlots) return fail(ctx, LUMO_ERR_UNSUPPORTED, "the attention calls take at most 256 physical slots");
  if (tree && desc->B > 65535) return fail(ctx, LUMO_ERR_UNSUPPORTED, "at most 65535 sequences per call");
  const lumo_kv4_args& a0 = layers[0];
  if (a0.dh != 128) return fail(ctx, LUMO_ERR_UNSUPPORTED, "dh must be 128");
  if (a0.Hq < 1 || a0.Hkv < 1 || a0.Hq % a0.Hkv != 0) return fail(ctx, LUMO_ERR_UNSUPPORTED, "Hq must be a positive multiple of Hkv");
  if (a0.Hkv > 32767 || a0.Hq > (1 << 20)) return fail(ctx, LUMO_ERR_UNSUPPORTED, "at most 32767 KV heads and 2^20 query heads");
  int log2 = 4;
  while (log2 < 8 && (1 << log2) != a0.page_size) ++log2;
  if (log2 == 8) return fail(ctx, LUMO_ERR_UNSUPPORTED, "page_size must be 16, 32, 64 or 128");
  if (a0.n_rows < 1 || a0.n_pages < 1 || a0.max_pages < 1 || (long long)a0.max_pages * a0.page_size > (1 << 30))
    return fail(ctx, LUMO_ERR_ARG, "need n_rows, n_pages, max_pages >= 1 and at most 2^30 positions a row");
  if (tree && (long long)a0.max_pages * a0.page_size < desc->Ns) return fail(ctx, LUMO_ERR_ARG, "a row must hold n_slots positions");
  if (a0.k_exp < -24 || a0.k_exp > 24 || a0.v_exp < -24 || a0.v_exp > 24) return fail(ctx, LUMO_ERR_ARG, "k_exp and v_exp must be in [-24, 24]");
  if (!a0.table) return fail(ctx, LUMO_ERR_ARG, "table is required");
  if (tree && (!a0.ctx_len || !a0.cache_row)) return fail(ctx, LUMO_ERR_ARG, "ctx_len and cache_row are required");
  const long long kv_stride = a0.kv_stride ? a0.kv_stride : (long long)a0.Hkv * 128, q_stride = a0.q_stride ? a0.q_stride : (long long)a0.Hq * 128;
  if (kv_stride < (long long)a0.Hkv * 128 || kv_stride % 8 || q_stride < (long long)a0.Hq * 128 || q_stride % 8)
    return fail(ctx, LUMO_ERR_ARG, "strides must be multiples of 8 elements and at least heads * dh");
  for (int l = 0; l < n_layers; ++l) {
    const lumo_kv4_args& a = layers[l];
    auto bad = [&](const char* msg) { return fail(ctx, LUMO_ERR_ARG, msg + (" (layer " + std::to_string(l) + ")")); };
    if (l && (a.Hq != a0.Hq || a.Hkv != a0.Hkv || a.dh != a0.dh || a.scale != a0.scale || a.n_rows != a0.n_rows || a.max_pages != a0.max_pages ||
        a.n_pages != a0.n_pages || a.page_size != a0.page_size || a.k_exp != a0.k_exp || a.v_exp != a0.v_exp || a.table != a0.table ||
        a.refs != a0.refs || a.ctx_len != a0.ctx_len || a.cache_row != a0.cache_row || a.q_stride != a0.q_stride || a.kv_stride != a0.kv_stride ||
        a.out_dtype != a0.out_dtype || a.n_splits != a0.n_splits))
      return bad("all layers must share shapes, options, table, refs, ctx_len and cache_row");
    if (!a.pages) return bad("pages is required");
    for (const void* p : {(const void*)a.pages, a.q, a.k_new, a.v_new, (const void*)a.out, (const void*)a.work})
      if (!aligned16(p)) return bad("tensor pointers must be 16-byte aligned");
  }
  std::memset(s, 0, sizeof(*s));
  if (tree) { s->B = desc->B; s->N = desc->N; s->Ns = desc->Ns; s->parent = desc->d_parent; s->slot = desc->d_slot; }
  s->Hq = a0.Hq; s->Hkv = a0.Hkv; s->n_rows = a0.n_rows; s->max_pages = a0.max_pages; s->n_pages = a0.n_pages;
  s->page = a0.page_size; s->page_log2 = log2; s->k_exp = a0.k_exp; s->v_exp = a0.v_exp;
  s->table = a0.table; s->refs = a0.refs; s->ctx_len = a0.ctx_len; s->cache_row = a0.cache_row;
  s->kv_stride = kv_stride;
  return LUMO_OK;
}

Kv4Layers kv4_views(const lumo_kv4_args* layers, int n_layers) {
  Kv4Layers L;
  std::memset(&L, 0, sizeof(L));
  for (int l = 0; l < n_layers; ++l) {
    L.pages[l] = layers[l].pages; L.kn[l] = layers[l].k_new; L.vn[l] = layers[l].v_new; L.status[l] = layers[l].status;
  }
  return L;
}

int check_new(lumo_ctx* ctx, const lumo_kv4_args* layers, int n_layers) {
  for (int l = 0; l < n_layers; ++l)
    if (!layers[l].k_new || !layers[l].v_new) return fail(ctx, LUMO_ERR_ARG, "k_new and v_new are required");
  return LUMO_OK;
}

int check_tokens(lumo_ctx* ctx, const Kv4Shape& s, int T, const int32_t* row, const int32_t* pos) {
  if (T < 1 || (long long)T * s.Hkv >= (1 << 30)) return fail(ctx, LUMO_ERR_ARG, "T must be positive and T * Hkv below 2^30");
  if (!row || !pos) return fail(ctx, LUMO_ERR_ARG, "tok_row and tok_pos are required");
  return LUMO_OK;
}

int prepare_pages(lumo_ctx* ctx, const lumo_page_table* t, PageTableDev* d, PagePools* pools) {
  if (!ctx || !t) return fail(ctx, LUMO_ERR_ARG, "null ctx or table");
  if (t->n_rows < 1 || t->max_pages < 1 || t->max_pages > kMaxPages || t->n_pages < 1 || t->n_pages > kMaxPages || t->page_size < 1 || t->page_size > 4096)
    return fail(ctx, LUMO_ERR_ARG, "need n_rows >= 1, max_pages and n_pages in [1, 262144], page_size in [1, 4096]");
  if (!t->table || !t->row_pages || !t->refs || !t->free_list || !t->free_count || !t->work)
    return fail(ctx, LUMO_ERR_ARG, "table, row_pages, refs, free_list, free_count and work are required");
  if (t->n_pools < 0 || t->n_pools > kMaxPools || (t->n_pools && !t->pools)) return fail(ctx, LUMO_ERR_ARG, "n_pools must be in [0, 64]");
  if (t->n_pools && (t->page_bytes < 16 || t->page_bytes % 16 || t->page_bytes > (1LL << 32)))
    return fail(ctx, LUMO_ERR_ARG, "page_bytes must be a multiple of 16, at most 2^32");
  std::memset(pools, 0, sizeof(*pools));
  pools->n = t->n_pools;
  for (int i = 0; i < t->n_pools; ++i) {
    if (!t->pools[i] || !aligned16(t->pools[i])) return fail(ctx, LUMO_ERR_ARG, "pools must be 16-byte aligned device pointers");
    pools->p[i] = reinterpret_cast<unsigned char*>(t->pools[i]);
    pools->bytes[i] = t->page_bytes;
  }
  d->n_rows = t->n_rows; d->max_pages = t->max_pages; d->n_pages = t->n_pages; d->page = t->page_size;
  d->table = t->table; d->row_pages = t->row_pages; d->refs = t->refs; d->free_list = t->free_list; d->free_count = t->free_count; d->work = t->work;
  return LUMO_OK;
}

int check_listed(lumo_ctx* ctx, int n) {
  if (n < 1 || n > kMaxPageRows) return fail(ctx, LUMO_ERR_ARG, "a call lists 1 to 1024 rows");
  return LUMO_OK;
}

}  // namespace

extern "C" {

int lumo_qk_norm_rope(lumo_ctx* ctx, const lumo_tree_desc* desc, const lumo_qk_args* x, void* stream) {
  if (!ctx || !x) return fail(ctx, LUMO_ERR_ARG, "null ctx or args");
  if (desc && desc->ctx != ctx) return fail(ctx, LUMO_ERR_ARG, "descriptor belongs to another context");
  if (x->dh != 64 && x->dh != 128 && x->dh != 256) return fail(ctx, LUMO_ERR_UNSUPPORTED, "dh must be 64, 128 or 256");
  if (x->dtype != LUMO_F32 && x->dtype != LUMO_BF16) return fail(ctx, LUMO_ERR_UNSUPPORTED, "dtype must be f32 or bf16");
  if (x->T < 1 || x->Hq < 1 || x->Hkv < 0 || x->Hq > 32767 || x->Hkv > 32767) return fail(ctx, LUMO_ERR_ARG, "need T >= 1, Hq in [1, 32767], Hkv in [0, 32767]");
  if (x->rot < 0 || x->rot > x->dh || x->rot % 16) return fail(ctx, LUMO_ERR_UNSUPPORTED, "rot must be a multiple of 16 in [0, dh]");
  if (x->style != 0 && x->style != 1) return fail(ctx, LUMO_ERR_ARG, "style must be 0 (halves) or 1 (pairs)");
  if (x->axes != 1 && x->axes != 3) return fail(ctx, LUMO_ERR_ARG, "axes must be 1 or 3");
  if (x->normalise && !(x->eps >= 0.f)) return fail(ctx, LUMO_ERR_ARG, "eps must not be negative");
  if (!x->q || !x->q_out || (x->Hkv && (!x->k || !x->k_out))) return fail(ctx, LUMO_ERR_ARG, "q, k, q_out and k_out are required");
  if (x->rot && !x->inv_freq) return fail(ctx, LUMO_ERR_ARG, "inv_freq is required");
  if (x->axes == 3) {
    if (!x->pos) return fail(ctx, LUMO_ERR_ARG, "three axes need pos");
    const int n = x->rot / 2;
    for (int i = 0; i < 3; ++i)
      if (x->section[i] < 0 || x->section[i] > n) return fail(ctx, LUMO_ERR_ARG, "sections must be in [0, rot / 2]");
    if (x->section[0] + x->section[1] + x->section[2] != n) return fail(ctx, LUMO_ERR_ARG, "sections must add up to rot / 2");
    if (x->turns)
      for (int i = 1; i < 3; ++i)
        if (x->section[i] && i + 3 * (x->section[i] - 1) >= n) return fail(ctx, LUMO_ERR_ARG, "a section does not fit by turns");
  }
  if (!x->pos && x->rot) {
    if (!desc || !x->ctx_len) return fail(ctx, LUMO_ERR_ARG, "without pos, desc and ctx_len are required");
    if ((long long)desc->B * desc->N != x->T) return fail(ctx, LUMO_ERR_ARG, "without pos, T must be batch * nodes");
  }
  RopeArgs a = {};
  const int esize = x->dtype == LUMO_BF16 ? 2 : 4;
  const long long qd = (long long)x->Hq * x->dh, kd = (long long)x->Hkv * x->dh;
  a.q_stride = x->q_stride ? x->q_stride : qd; a.q_out_stride = x->q_out_stride ? x->q_out_stride : qd;
  a.k_stride = x->k_stride ? x->k_stride : kd; a.k_out_stride = x->k_out_stride ? x->k_out_stride : kd;
  for (long long st : {a.q_stride, a.q_out_stride})
    if (st < qd || st * esize % 16) return fail(ctx, LUMO_ERR_ARG, "strides must be at least heads * dh and multiples of 16 bytes");
  for (long long st : {a.k_stride, a.k_out_stride})
    if (st < kd || st * esize % 16) return fail(ctx, LUMO_ERR_ARG, "strides must be at least heads * dh and multiples of 16 bytes");
  for (const void* p : {x->q, x->k, (const void*)x->q_out, (const void*)x->k_out, x->q_weight, x->k_weight})
    if (!aligned16(p)) return fail(ctx, LUMO_ERR_ARG, "tensor pointers must be 16-byte aligned");
  if ((x->q == x->q_out && a.q_stride != a.q_out_stride) || (x->Hkv && x->k == x->k_out && a.k_stride != a.k_out_stride))
    return fail(ctx, LUMO_ERR_ARG, "an output that is its input must have the same stride");
  a.q = x->q; a.k = x->k; a.q_out = x->q_out; a.k_out = x->k_out;
  a.T = x->T; a.Hq = x->Hq; a.Hkv = x->Hkv; a.dh = x->dh; a.rot = x->rot; a.style = x->style; a.norm = x->normalise != 0;
  a.axes = x->axes; a.turns = x->turns != 0;
  for (int i = 0; i < 3; ++i) a.section[i] = x->section[i];
  a.inv_freq = x->inv_freq; a.pos = x->pos; a.ctx_len = x->ctx_len;
  a.depth = desc ? desc->d_depth : nullptr; a.N = desc ? desc->N : 1;
  a.q_weight = x->q_weight; a.k_weight = x->k_weight;
  a.eps = x->eps; a.weight_offset = x->weight_offset; a.mscale = x->mscale;
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  ctx->order.begin(ctx->device, stream);
  cudaError_t e = timed(ctx, LUMO_K_ROPE, st, [&] { return launch_rope(a, x->dtype, ctx->sm_count, ctx->overlap, st); });
  return launched(ctx, e, CallOrder::kOther, "norm and rotation launch");
}

int lumo_kv4_write_tree(lumo_ctx* ctx, const lumo_tree_desc* desc, const lumo_kv4_args* layers, int n_layers, void* stream) {
  Kv4Shape s;
  int rc = prepare_kv4(ctx, desc, true, layers, n_layers, &s);
  if (rc == LUMO_OK) rc = check_new(ctx, layers, n_layers);
  if (rc != LUMO_OK) return rc;
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  const Kv4Layers L = kv4_views(layers, n_layers);
  ctx->order.begin(ctx->device, stream);
  cudaError_t e = timed(ctx, LUMO_K_KV4_WRITE, st, [&] { return launch_kv4_write(L, s, n_layers, ctx->overlap, st); });
  return launched(ctx, e, CallOrder::kOther, "4-bit write launch");
}

int lumo_kv4_append(lumo_ctx* ctx, const lumo_kv4_args* layers, int n_layers, int T, const int32_t* tok_row, const int32_t* tok_pos,
                    int32_t* status, void* stream) {
  Kv4Shape s;
  int rc = prepare_kv4(ctx, nullptr, false, layers, n_layers, &s);
  if (rc == LUMO_OK) rc = check_new(ctx, layers, n_layers);
  if (rc == LUMO_OK) rc = check_tokens(ctx, s, T, tok_row, tok_pos);
  if (rc != LUMO_OK) return rc;
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  const Kv4Layers L = kv4_views(layers, n_layers);
  const Kv4Tokens t = {T, tok_row, tok_pos, status};
  ctx->order.begin(ctx->device, stream);
  cudaError_t e = timed(ctx, LUMO_K_KV4_WRITE, st, [&] { return launch_kv4_append(L, s, n_layers, t, ctx->sm_count, ctx->overlap, st); });
  return launched(ctx, e, CallOrder::kOther, "4-bit append launch");
}

int lumo_kv4_read(lumo_ctx* ctx, const lumo_kv4_args* layer, int T, const int32_t* tok_row, const int32_t* tok_pos, void* k_out, void* v_out,
                  int32_t* status, void* stream) {
  Kv4Shape s;
  int rc = prepare_kv4(ctx, nullptr, false, layer, 1, &s);
  if (rc == LUMO_OK) rc = check_tokens(ctx, s, T, tok_row, tok_pos);
  if (rc != LUMO_OK) return rc;
  if (!k_out || !v_out || !aligned16(k_out) || !aligned16(v_out)) return fail(ctx, LUMO_ERR_ARG, "k_out and v_out are required, 16-byte aligned");
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  const Kv4Tokens t = {T, tok_row, tok_pos, status};
  ctx->order.begin(ctx->device, stream);
  cudaError_t e = timed(ctx, LUMO_K_KV4_READ, st, [&] {
    return launch_kv4_read(layer->pages, s, t, k_out, v_out, ctx->sm_count, ctx->overlap, st);
  });
  return launched(ctx, e, CallOrder::kOther, "4-bit read launch");
}

int64_t lumo_kv4_work_bytes(const lumo_ctx* ctx, const lumo_tree_desc* desc, int Hq, int Hkv, int n_splits) {
  if (!ctx || !desc || ctx->device < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv || n_splits < 0 || n_splits > 32) return 0;
  return (int64_t)kv4_work_bytes(desc->B, desc->N, Hq, Hkv, n_splits, ctx->sm_count);
}

int lumo_kv4_attention(lumo_ctx* ctx, const lumo_tree_desc* desc, const lumo_kv4_args* layers, int n_layers, void* stream) {
  Kv4Shape s;
  const int rc = prepare_kv4(ctx, desc, true, layers, n_layers, &s);
  if (rc != LUMO_OK) return rc;
  const lumo_kv4_args& a0 = layers[0];
  if (!(a0.scale > 0.f)) return fail(ctx, LUMO_ERR_ARG, "scale must be positive");
  if (a0.out_dtype != LUMO_F32 && a0.out_dtype != LUMO_BF16) return fail(ctx, LUMO_ERR_UNSUPPORTED, "out_dtype must be f32 or bf16");
  if (a0.n_splits < 0 || a0.n_splits > 32) return fail(ctx, LUMO_ERR_ARG, "n_splits must be 0 (automatic) or in [1, 32]");
  // The kernels number the key tiles of all (sequence, KV head, row tile) units in 32 bits (and add a CTA's share to a position: hence not
  // quite 2^31), and so they do the slots, 32 to a unit at most.
  if (kv4_line(s) > 2000000000LL || kv4_units(s.B, s.N, s.Hq, s.Hkv) * 32 > INT_MAX)
    return fail(ctx, LUMO_ERR_UNSUPPORTED, "batch x KV heads x positions too large for one call");
  const size_t need = kv4_work_bytes(s.B, s.N, s.Hq, s.Hkv, a0.n_splits, ctx->sm_count);
  for (int l = 0; l < n_layers; ++l) {
    if (!layers[l].q || !layers[l].out) return fail(ctx, LUMO_ERR_ARG, "q and out are required");
    if (!layers[l].work || layers[l].work_bytes < 0 || (size_t)layers[l].work_bytes < need)
      return fail(ctx, LUMO_ERR_ARG, "work must hold " + std::to_string(need) + " bytes (lumo_kv4_work_bytes)");
  }
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  ctx->order.begin(ctx->device, stream);
  for (int l = 0; l < n_layers; ++l) {
    const lumo_kv4_args& a = layers[l];
    const Kv4AttnPtrs p = {a.pages, a.q, a.out, a.lse, a.status};
    Kv4Plan plan;
    kv4_plan(s, p, desc->d_vis, desc->d_slot_used, a.scale, a.q_stride ? a.q_stride : (long long)a.Hq * 128, a.out_dtype == LUMO_BF16, a.n_splits, a.work,
             ctx->sm_count, ctx->timeout_drill, &plan);
    cudaError_t e = timed(ctx, LUMO_K_KV4_ATTN, st, [&] { return launch_kv4_attn(plan, ctx->overlap, st); });
    if (e != cudaSuccess) return cuda_fail(ctx, e, "4-bit attention launch");
    e = timed(ctx, LUMO_K_KV4_MERGE, st, [&] { return launch_kv4_merge(plan, ctx->overlap, st); });
    if (e != cudaSuccess) return cuda_fail(ctx, e, "4-bit attention merge launch");
  }
  ctx->order.done(CallOrder::kOther);
  return LUMO_OK;
}

int lumo_kv4_publish(lumo_ctx* ctx, const lumo_tree_desc* desc, const lumo_kv4_args* layers, int n_layers, const int32_t* accepted_dev,
                     const int32_t* len_dev, int lmax, int32_t* ctx_len_out, void* stream) {
  if (ctx && (lmax < 1 || lmax > kMaxNodes))
    return fail(ctx, LUMO_ERR_ARG, "lmax must be in [1, " + std::to_string(kMaxNodes) + "] (a path holds each node at most once)");
  Kv4Shape s;
  const int rc = prepare_kv4(ctx, desc, true, layers, n_layers, &s);
  if (rc != LUMO_OK) return rc;
  if (!accepted_dev || !len_dev) return fail(ctx, LUMO_ERR_ARG, "accepted_dev and len_dev are required");
  if (ctx_len_out == s.ctx_len) return fail(ctx, LUMO_ERR_ARG, "ctx_len_out must not alias ctx_len");
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  const Kv4Layers L = kv4_views(layers, n_layers);
  ctx->order.begin(ctx->device, stream);
  cudaError_t e = timed(ctx, LUMO_K_KV4_PUBLISH, st, [&] {
    return launch_kv4_publish(L, s, n_layers, accepted_dev, len_dev, lmax, ctx_len_out, ctx->overlap, st);
  });
  return launched(ctx, e, CallOrder::kOther, "4-bit publish launch");
}

int64_t lumo_pages_work_ints(int n_rows, int n_pages) {
  return n_rows < 1 || n_pages < 1 ? 0 : (int64_t)n_rows + 4 * (int64_t)n_pages + 8;
}

int lumo_pages_init(lumo_ctx* ctx, const lumo_page_table* t, void* stream) {
  PageTableDev d;
  PagePools pools;
  const int rc = prepare_pages(ctx, t, &d, &pools);
  if (rc != LUMO_OK) return rc;
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  ctx->order.begin(ctx->device, stream);
  cudaError_t e = timed(ctx, LUMO_K_PAGES, st, [&] { return launch_pages_init(d, ctx->sm_count, ctx->overlap, st); });
  return launched(ctx, e, CallOrder::kOther, "page table set-up launch");
}

int lumo_pages_fork(lumo_ctx* ctx, const lumo_page_table* t, const int32_t* src, const int32_t* dst, int n, int32_t* status, void* stream) {
  PageTableDev d;
  PagePools pools;
  int rc = prepare_pages(ctx, t, &d, &pools);
  if (rc == LUMO_OK) rc = check_listed(ctx, n);
  if (rc != LUMO_OK) return rc;
  if (!src || !dst) return fail(ctx, LUMO_ERR_ARG, "src and dst are required");
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  ctx->order.begin(ctx->device, stream);
  cudaError_t e = timed(ctx, LUMO_K_PAGES, st, [&] { return launch_pages_fork(d, src, dst, n, status, ctx->overlap, st); });
  return launched(ctx, e, CallOrder::kOther, "page fork launch");
}

// (A pool may be anything the caller pages, recurrent states among it: what follows a call that copies pages or rows reads nothing early.)
int lumo_pages_reserve(lumo_ctx* ctx, const lumo_page_table* t, const int32_t* rows, const int32_t* start, const int32_t* end, int add, int n,
                       int32_t* status, void* stream) {
  PageTableDev d;
  PagePools pools;
  int rc = prepare_pages(ctx, t, &d, &pools);
  if (rc == LUMO_OK) rc = check_listed(ctx, n);
  if (rc != LUMO_OK) return rc;
  if (!rows || !start) return fail(ctx, LUMO_ERR_ARG, "rows and start are required");
  if (!end && add < 0) return fail(ctx, LUMO_ERR_ARG, "add must not be negative");
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  ctx->order.begin(ctx->device, stream);
  cudaError_t e = timed(ctx, LUMO_K_PAGES, st, [&] {
    return launch_pages_reserve(d, pools, rows, start, end, add, n, status, ctx->sm_count, ctx->overlap, st);
  });
  return launched(ctx, e, CallOrder::kNone, "page reserve launch");
}

int lumo_pages_free(lumo_ctx* ctx, const lumo_page_table* t, const int32_t* rows, const int32_t* keep, int n, int32_t* status, void* stream) {
  PageTableDev d;
  PagePools pools;
  int rc = prepare_pages(ctx, t, &d, &pools);
  if (rc == LUMO_OK) rc = check_listed(ctx, n);
  if (rc != LUMO_OK) return rc;
  if (!rows) return fail(ctx, LUMO_ERR_ARG, "rows is required");
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  ctx->order.begin(ctx->device, stream);
  cudaError_t e = timed(ctx, LUMO_K_PAGES, st, [&] { return launch_pages_free(d, rows, keep, n, status, ctx->overlap, st); });
  return launched(ctx, e, CallOrder::kOther, "page free launch");
}

int lumo_pages_compact(lumo_ctx* ctx, const lumo_page_table* t, void* stream) {
  PageTableDev d;
  PagePools pools;
  const int rc = prepare_pages(ctx, t, &d, &pools);
  if (rc != LUMO_OK) return rc;
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  ctx->order.begin(ctx->device, stream);
  cudaError_t e = timed(ctx, LUMO_K_PAGES, st, [&] { return launch_pages_compact(d, pools, ctx->sm_count, ctx->overlap, st); });
  return launched(ctx, e, CallOrder::kNone, "page compaction launch");
}

int lumo_rows_copy(lumo_ctx* ctx, void* const* blocks, const int64_t* row_bytes, int n_blocks, int n_rows, const int32_t* src, const int32_t* dst,
                   int n, int32_t* status, void* stream) {
  if (!ctx || !blocks || !row_bytes || !src || !dst) return fail(ctx, LUMO_ERR_ARG, "null argument");
  if (n_blocks < 1 || n_blocks > kMaxPools || n_rows < 1) return fail(ctx, LUMO_ERR_ARG, "need n_blocks in [1, 64] and n_rows >= 1");
  const int rc = check_listed(ctx, n);
  if (rc != LUMO_OK) return rc;
  PagePools b;
  std::memset(&b, 0, sizeof(b));
  b.n = n_blocks;
  for (int i = 0; i < n_blocks; ++i) {
    if (!blocks[i] || !aligned16(blocks[i]) || row_bytes[i] < 16 || row_bytes[i] % 16 || row_bytes[i] > (1LL << 32))
      return fail(ctx, LUMO_ERR_ARG, "blocks must be 16-byte aligned device pointers, row_bytes multiples of 16 up to 2^32");
    b.p[i] = reinterpret_cast<unsigned char*>(blocks[i]);
    b.bytes[i] = row_bytes[i];
  }
  if (const int host = launchable(ctx)) return host;
  DeviceGuard g(ctx->device);
  cudaStream_t st = (cudaStream_t)stream;
  ctx->order.begin(ctx->device, stream);
  cudaError_t e = timed(ctx, LUMO_K_ROWS_COPY, st, [&] { return launch_rows_copy(b, n_rows, src, dst, n, status, ctx->sm_count, ctx->overlap, st); });
  return launched(ctx, e, CallOrder::kNone, "row copy launch");
}

}  // extern "C"
