// Entry points of generation over a paged cache: argument checks on the host and the launches.
#include <climits>
#include <cmath>

#include "internal.h"

using namespace sp;

static bool al(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

#define SP_PG_CUDA(call, where)                                                                       \
  do {                                                                                                \
    const cudaError_t e__ = (call);                                                                   \
    if (e__ != cudaSuccess) return report(SP_ERR_CUDA, "%s: %s (%d)", where, cudaGetErrorString(e__), (int)e__); \
  } while (0)

// log2 of a page size, -1 where it is none
static int page_shift_of(int page_size) {
  for (int s = 4; s <= 10; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}

static sp_status check_heads(const char* who, int n_heads, int n_kv_heads, int head_dim) {
  if (head_dim != 64 && head_dim != 128) return report(SP_ERR_SHAPE, "%s: head_dim must be 64 or 128", who);
  if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0 || n_heads > 1024)
    return report(SP_ERR_SHAPE, "%s: n_kv_heads must divide n_heads (1..1024)", who);
  return SP_OK;
}

static sp_status check_pages(const char* who, const sp_paged_kv* c) {
  if (!c->kv || !c->table) return report(SP_ERR_INVALID_ARG, "%s: kv and table required", who);
  if (page_shift_of(c->page_size) < 0)
    return report(SP_ERR_SHAPE, "%s: page_size must be a power of two in 16..1024", who);
  if (c->n_pages < 1 || (long long)c->n_pages * c->page_size > (1ll << 30) || c->max_pages < 1 ||
      (long long)c->max_pages * c->page_size > (1ll << 30))
    return report(SP_ERR_SHAPE, "%s: n_pages and max_pages must be at least 1 and at most 2^30 positions", who);
  if (!al(c->kv, 16)) return report(SP_ERR_ALIGN, "%s: kv must be 16-byte aligned", who);
  return SP_OK;
}

extern "C" {

sp_status sp_paged_append(const sp_paged_append_io* io, sp_stream stream) {
  const char* who = "sp_paged_append";
  if (!io) return report(SP_ERR_INVALID_ARG, "%s: NULL io", who);
  sp_status s = check_heads(who, io->n_heads, io->n_kv_heads, io->head_dim);
  if (s != SP_OK) return s;
  s = check_pages(who, &io->cache);
  if (s != SP_OK) return s;
  const int qkvw = (io->n_heads + 2 * io->n_kv_heads) * io->head_dim;
  if (io->B < 1 || io->B > SP_MAX_BATCH || io->T_cap < 0 || (!io->cu_rows && io->T_cap != io->B))
    return report(SP_ERR_SHAPE, "%s: B must be in 1..SP_MAX_BATCH and T_cap >= 0 (= B without cu_rows)", who);
  if (io->T_cap == 0) return SP_OK;  // nothing to do
  if (!io->qkv) return report(SP_ERR_INVALID_ARG, "%s: qkv required", who);
  if (io->ld < qkvw || io->ld % 8 != 0 || (io->q_out && (io->ld_q < io->n_heads * io->head_dim || io->ld_q % 8 != 0)))
    return report(SP_ERR_SHAPE, "%s: row strides must be multiples of 8 and hold a row", who);
  if (!al(io->qkv, 16) || !al(io->q_out, 16) || !al(io->rope, 16) || !al(io->pos3, 16))
    return report(SP_ERR_ALIGN, "%s: qkv, q_out, rope, pos3 must be 16-byte aligned", who);
  const int* sec = io->mrope_section;
  if (io->rope) {
    if ((io->pos != nullptr) == (io->pos3 != nullptr))
      return report(SP_ERR_INVALID_ARG, "%s: a rotation takes either pos or pos3", who);
    if (io->max_pos < 1) return report(SP_ERR_SHAPE, "%s: max_pos must be at least 1", who);
    if (io->pos3 && (sec[0] < 0 || sec[1] < 0 || sec[2] < 0 || sec[0] % 2 || sec[1] % 2 || sec[2] % 2 ||
                     sec[0] + sec[1] + sec[2] != io->head_dim / 2))
      return report(SP_ERR_SHAPE, "%s: mrope_section must be even and sum to head_dim / 2", who);
  }
  PagedAppendArgs a;
  a.qkv = static_cast<const __nv_bfloat16*>(io->qkv);
  a.ld = io->ld;
  a.q_out = static_cast<__nv_bfloat16*>(io->q_out);
  a.ld_q = io->ld_q;
  a.kv = static_cast<__nv_bfloat16*>(io->cache.kv);
  a.n_pages = io->cache.n_pages;
  a.page_shift = page_shift_of(io->cache.page_size);
  a.table = io->cache.table;
  a.max_pages = io->cache.max_pages;
  a.lens = io->cache.lens;
  a.cu_rows = io->cu_rows;
  a.B = io->B;
  a.T_cap = io->T_cap;
  a.Hq = io->n_heads;
  a.Hkv = io->n_kv_heads;
  a.dh = io->head_dim;
  a.rope = reinterpret_cast<const float2*>(io->rope);
  a.max_pos = io->max_pos;
  a.pos = io->rope ? io->pos : nullptr;
  a.pos3 = io->rope ? io->pos3 : nullptr;
  a.sec1 = io->pos3 ? sec[0] : 0;
  a.sec2 = io->pos3 ? sec[0] + sec[1] : 0;
  a.err = io->err;
  SP_PG_CUDA(paged_append_launch(a, (cudaStream_t)stream), who);
  return SP_OK;
}

size_t sp_prefix_attention_workspace(int T_cap, int B, int n_groups, int n_heads, int n_kv_heads, int head_dim) {
  const char* who = "sp_prefix_attention_workspace";
  if (check_heads(who, n_heads, n_kv_heads, head_dim) != SP_OK) return 0;
  if (T_cap < 0 || B < 1 || B > SP_MAX_BATCH || n_groups < 0 || n_groups > SP_MAX_BATCH ||
      (long long)T_cap * n_heads > (1ll << 28)) {
    report(SP_ERR_SHAPE, "%s: B must be in 1..SP_MAX_BATCH, n_groups in 0..SP_MAX_BATCH, T_cap >= 0, T_cap * n_heads at most 2^28", who);
    return 0;
  }
  return prefix_attention_bytes(T_cap, B, n_groups, n_heads, n_kv_heads, head_dim) + 256;
}

sp_status sp_prefix_attention(const sp_prefix_attention_io* io, void* workspace, size_t workspace_bytes,
                              sp_stream stream) {
  const char* who = "sp_prefix_attention";
  if (!io) return report(SP_ERR_INVALID_ARG, "%s: NULL io", who);
  sp_status s = check_heads(who, io->n_heads, io->n_kv_heads, io->head_dim);
  if (s != SP_OK) return s;
  s = check_pages(who, &io->cache);
  if (s != SP_OK) return s;
  const int dq = io->n_heads * io->head_dim;
  if (io->B < 1 || io->B > SP_MAX_BATCH || io->T_cap < 0 || (!io->cu_rows && io->T_cap != io->B))
    return report(SP_ERR_SHAPE, "%s: B must be in 1..SP_MAX_BATCH and T_cap >= 0 (= B without cu_rows)", who);
  if (io->n_groups < 0 || io->n_groups > SP_MAX_BATCH ||
      (io->n_groups > 0 && (io->prefix_max_pages < 1 ||
                            (long long)io->prefix_max_pages * io->cache.page_size > (1ll << 30))))
    return report(SP_ERR_SHAPE, "%s: n_groups must be in 0..SP_MAX_BATCH, prefix_max_pages at least 1 with groups", who);
  if ((long long)io->T_cap * io->n_heads > (1ll << 28))
    return report(SP_ERR_SHAPE, "%s: T_cap * n_heads must be at most 2^28", who);
  if (io->T_cap == 0) return SP_OK;  // nothing to do
  if (!io->q || !io->out || !io->cache.lens)
    return report(SP_ERR_INVALID_ARG, "%s: q, out and cache.lens required", who);
  if (io->n_groups > 0 && (!io->group_cu || !io->prefix_table || !io->prefix_lens))
    return report(SP_ERR_INVALID_ARG, "%s: groups need group_cu, prefix_table and prefix_lens", who);
  if (io->ld_q < dq || io->ld_q % 8 != 0 || io->ld_out < dq || io->ld_out % 8 != 0)
    return report(SP_ERR_SHAPE, "%s: row strides must be multiples of 8 and hold a row", who);
  if (!al(io->q, 16) || !al(io->out, 16) || !al(io->lse, 4))
    return report(SP_ERR_ALIGN, "%s: q and out must be 16-byte aligned", who);
  if (!(io->scale >= 0.f) || !std::isfinite(io->scale))
    return report(SP_ERR_INVALID_ARG, "%s: scale must be finite and not negative", who);
  const size_t need =
      prefix_attention_bytes(io->T_cap, io->B, io->n_groups, io->n_heads, io->n_kv_heads, io->head_dim) + 256;
  if (!workspace || workspace_bytes < need)
    return report(SP_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, workspace_bytes, need);
  if (!al(workspace, 16)) return report(SP_ERR_ALIGN, "%s: workspace must be 16-byte aligned", who);
  PrefixAttention a;
  a.q = io->q;
  a.ld_q = io->ld_q;
  a.out = io->out;
  a.ld_out = io->ld_out;
  a.lse = io->lse;
  a.kv = io->cache.kv;
  a.n_pages = io->cache.n_pages;
  a.page_size = io->cache.page_size;
  a.table = io->cache.table;
  a.max_pages = io->cache.max_pages;
  a.lens = io->cache.lens;
  a.ptable = io->prefix_table;
  a.pmax_pages = io->n_groups > 0 ? io->prefix_max_pages : 0;
  a.plens = io->prefix_lens;
  a.group_cu = io->group_cu;
  a.n_groups = io->n_groups;
  a.cu_rows = io->cu_rows;
  a.B = io->B;
  a.T_cap = io->T_cap;
  a.Hq = io->n_heads;
  a.Hkv = io->n_kv_heads;
  a.dh = io->head_dim;
  a.scale = io->scale;
  a.err = io->err;
  void* base = reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~uintptr_t(255));
  SP_PG_CUDA(prefix_attention(a, base, (cudaStream_t)stream), who);
  return SP_OK;
}

static sp_status check_beams(const char* who, int B, int W, int V, int n_out) {
  if (B < 1 || B > SP_MAX_BATCH || W < 1 || W > SP_MAX_BEAMS)
    return report(SP_ERR_SHAPE, "%s: B must be in 1..SP_MAX_BATCH and W in 1..SP_MAX_BEAMS", who);
  if (V < 1 || V > (1 << 24)) return report(SP_ERR_SHAPE, "%s: V must be in 1..2^24", who);
  if (n_out < 1 || n_out > 2 * SP_MAX_BEAMS)
    return report(SP_ERR_SHAPE, "%s: n_out must be in 1..2 SP_MAX_BEAMS", who);
  return SP_OK;
}

size_t sp_beam_select_workspace(int B, int W, int V, int n_out) {
  if (check_beams("sp_beam_select_workspace", B, W, V, n_out) != SP_OK) return 0;
  return beam_select_bytes(B * W, V, n_out) + 256;
}

sp_status sp_beam_select(const sp_beam_select_io* io, void* workspace, size_t workspace_bytes, sp_stream stream) {
  const char* who = "sp_beam_select";
  if (!io) return report(SP_ERR_INVALID_ARG, "%s: NULL io", who);
  const sp_status s = check_beams(who, io->B, io->W, io->V, io->n_out);
  if (s != SP_OK) return s;
  if (!io->logits || !io->cum || !io->score || !io->parent || !io->token)
    return report(SP_ERR_INVALID_ARG, "%s: logits, cum, score, parent, token required", who);
  if (io->ld < io->V) return report(SP_ERR_SHAPE, "%s: row stride %lld < V %d", who, io->ld, io->V);
  if (io->done && (io->eos < 0 || io->eos >= io->V))
    return report(SP_ERR_INVALID_ARG, "%s: eos must be a token with done", who);
  if (!al(io->logits, io->logits_f32 ? 4 : 2))
    return report(SP_ERR_ALIGN, "%s: logits must be aligned to their type", who);
  const size_t need = beam_select_bytes(io->B * io->W, io->V, io->n_out) + 256;
  if (!workspace || workspace_bytes < need)
    return report(SP_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, workspace_bytes, need);
  void* base = reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~uintptr_t(255));
  SP_PG_CUDA(beam_select_launch(io->logits, io->logits_f32 != 0, io->ld, io->B, io->W, io->V, io->cum, io->done,
                                io->eos, io->n_out, base, io->score, io->parent, io->token, (cudaStream_t)stream),
             who);
  return SP_OK;
}

sp_status sp_beam_reorder(const sp_beam_reorder_io* io, sp_stream stream) {
  const char* who = "sp_beam_reorder";
  if (!io) return report(SP_ERR_INVALID_ARG, "%s: NULL io", who);
  if (io->B < 1 || io->B > SP_MAX_BATCH || io->W < 1 || io->W > SP_MAX_BEAMS || io->ld_parent < io->W)
    return report(SP_ERR_SHAPE, "%s: B must be in 1..SP_MAX_BATCH, W in 1..SP_MAX_BEAMS, ld_parent at least W", who);
  if (io->n_layers < 1 || io->n_layers > SP_MAX_LM_LAYERS)
    return report(SP_ERR_SHAPE, "%s: n_layers must be in 1..SP_MAX_LM_LAYERS", who);
  if (io->row_elems < 8 || io->row_elems % 8 != 0 || io->row_elems > (1 << 20))
    return report(SP_ERR_SHAPE, "%s: row_elems must be a multiple of 8 in 8..2^20", who);
  const int shift = page_shift_of(io->page_size);
  if (shift < 0) return report(SP_ERR_SHAPE, "%s: page_size must be a power of two in 16..1024", who);
  if (io->n_pages < 1 || (long long)io->n_pages * io->page_size > (1ll << 30) || io->max_pages < 1 ||
      (long long)io->max_pages * io->page_size > (1ll << 30))
    return report(SP_ERR_SHAPE, "%s: n_pages and max_pages must be at least 1 and at most 2^30 positions", who);
  if (!io->kv || !io->table || !io->own_table || !io->lens || !io->parent)
    return report(SP_ERR_INVALID_ARG, "%s: kv, table, own_table, lens, parent required", who);
  if (io->table == io->own_table) return report(SP_ERR_INVALID_ARG, "%s: table and own_table must be two arrays", who);
  if (!al(io->kv, 16)) return report(SP_ERR_ALIGN, "%s: kv must be 16-byte aligned", who);
  SP_PG_CUDA(beam_reorder_launch(io->kv, io->n_layers, io->n_pages, shift, io->row_elems * 2, io->table, io->own_table,
                                 io->max_pages, io->lens, io->parent, io->ld_parent, io->B, io->W, io->err,
                                 (cudaStream_t)stream),
             who);
  return SP_OK;
}

}  // extern "C"
