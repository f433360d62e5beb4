// Entry points of generation over a paged cache (attention, beams, drafted tokens, pages): argument checks on the host and the launches.
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

static sp_status check_drafts(const char* who, int T_cap, int B, int V) {
  if (B < 1 || B > SP_MAX_BATCH || V < 1 || V > (1 << 24))
    return report(SP_ERR_SHAPE, "%s: B must be in 1..SP_MAX_BATCH and V in 1..2^24", who);
  if (T_cap < 0 || T_cap > (1 << 24)) return report(SP_ERR_SHAPE, "%s: T_cap must be in 0..2^24", who);
  return SP_OK;
}

size_t sp_draft_verify_workspace(int T_cap, int B, int V) {
  if (check_drafts("sp_draft_verify_workspace", T_cap, B, V) != SP_OK) return 0;
  return verify_bytes(T_cap, B, V) + 256;
}

sp_status sp_draft_verify(const sp_draft_verify_io* io, void* workspace, size_t workspace_bytes, sp_stream stream) {
  const char* who = "sp_draft_verify";
  if (!io) return report(SP_ERR_INVALID_ARG, "%s: NULL io", who);
  const sp_status s = check_drafts(who, io->T_cap, io->B, io->V);
  if (s != SP_OK) return s;
  if (io->max_rows < 1 || io->max_rows > SP_MAX_DRAFT_ROWS || (!io->cu_rows && io->T_cap != io->B))
    return report(SP_ERR_SHAPE, "%s: max_rows must be in 1..SP_MAX_DRAFT_ROWS, T_cap = B without cu_rows", who);
  if (!io->n_accept || !io->token || (io->T_cap > 0 && !io->logits))
    return report(SP_ERR_INVALID_ARG, "%s: logits, n_accept, token required", who);
  const bool drafts = io->max_rows > 1 && io->T_cap > 0;
  if (drafts && (!io->draft || (io->noise && !io->u)))
    return report(SP_ERR_INVALID_ARG, "%s: rows behind drafts need draft, and u with noise", who);
  const bool with_q = drafts && io->noise && io->draft_logits;
  if (io->ld < io->V || (with_q && io->ld_draft < io->V) || (io->noise && io->ld_noise < io->V))
    return report(SP_ERR_SHAPE, "%s: row strides must be at least V", who);
  const size_t esz = io->logits_f32 ? 4 : 2;
  if (!al(io->logits, esz) || (with_q && !al(io->draft_logits, esz)) || !al(io->noise, 4))
    return report(SP_ERR_ALIGN, "%s: logits, draft_logits, noise must be aligned to their types", who);
  const size_t need = verify_bytes(io->T_cap, io->B, io->V) + 256;
  if (!workspace || workspace_bytes < need)
    return report(SP_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, workspace_bytes, need);
  VerifyArgs a;
  a.B = io->B;
  a.V = io->V;
  a.T_cap = io->T_cap;
  a.max_rows = io->max_rows;
  a.cu_rows = io->cu_rows;
  a.logits = io->logits;
  a.logits_f32 = io->logits_f32 != 0;
  a.ld = io->ld;
  a.draft = io->draft;
  a.draft_logits = with_q ? io->draft_logits : nullptr;
  a.ld_draft = io->ld_draft;
  a.u = io->u;
  a.noise = io->noise;
  a.ld_noise = io->ld_noise;
  a.temperature = io->temperature;
  a.n_accept = io->n_accept;
  a.token = io->token;
  a.logp = io->logp;
  a.err = io->err;
  a.clear_err = io->clear_err != 0;
  void* base = reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~uintptr_t(255));
  SP_PG_CUDA(verify_launch(a, base, (cudaStream_t)stream), who);
  return SP_OK;
}

static sp_status check_rows(const char* who, int S, int max_pages) {
  if (S < 1 || S > SP_MAX_TABLE_ROWS || max_pages < 1 || (long long)S * max_pages > (1ll << 30))
    return report(SP_ERR_SHAPE, "%s: S must be in 1..SP_MAX_TABLE_ROWS, S * max_pages in 1..2^30", who);
  return SP_OK;
}

// moves: the call moves positions, so it needs the pool
static sp_status page_args(const char* who, const sp_pages* p, bool moves, PagesArgs* a) {
  if (!p) return report(SP_ERR_INVALID_ARG, "%s: NULL pages", who);
  const sp_status s = check_rows(who, p->S, p->max_pages);
  if (s != SP_OK) return s;
  const int shift = page_shift_of(p->page_size);
  if (shift < 0) return report(SP_ERR_SHAPE, "%s: page_size must be a power of two in 16..1024", who);
  if (p->n_pages < 1 || (long long)p->n_pages * p->page_size > (1ll << 30) ||
      (long long)p->max_pages * p->page_size > (1ll << 30))
    return report(SP_ERR_SHAPE, "%s: n_pages must be at least 1, n_pages and max_pages at most 2^30 positions", who);
  if (!p->table || !p->lens || !p->refs || (moves && !p->kv))
    return report(SP_ERR_INVALID_ARG, "%s: %stable, lens, refs required", who, moves ? "kv, " : "");
  if (moves && (p->n_layers < 1 || p->n_layers > SP_MAX_LM_LAYERS))
    return report(SP_ERR_SHAPE, "%s: n_layers must be in 1..SP_MAX_LM_LAYERS", who);
  if (moves && (p->row_elems < 8 || p->row_elems % 8 != 0 || p->row_elems > (1 << 20)))
    return report(SP_ERR_SHAPE, "%s: row_elems must be a multiple of 8 in 8..2^20", who);
  if ((moves && !al(p->kv, 16)) || !al(p->refs, 16))
    return report(SP_ERR_ALIGN, "%s: %srefs must be 16-byte aligned", who, moves ? "kv and " : "");
  a->kv = static_cast<uint4*>(p->kv);
  a->planes = 2 * p->n_layers;
  a->n_pages = p->n_pages;
  a->page_shift = shift;
  a->row16 = p->row_elems / 8;
  a->S = p->S;
  a->table = p->table;
  a->max_pages = p->max_pages;
  a->lens = p->lens;
  a->refs = p->refs;
  a->err = p->err;
  return SP_OK;
}

sp_status sp_pages_trim(const sp_pages* p, sp_stream stream) {
  PagesArgs a;
  const sp_status s = page_args("sp_pages_trim", p, false, &a);
  if (s != SP_OK) return s;
  SP_PG_CUDA(pages_trim_launch(a, (cudaStream_t)stream), "sp_pages_trim");
  return SP_OK;
}

sp_status sp_pages_fork(const sp_pages* p, const int* parent, sp_stream stream) {
  PagesArgs a;
  const sp_status s = page_args("sp_pages_fork", p, false, &a);
  if (s != SP_OK) return s;
  if (!parent) return report(SP_ERR_INVALID_ARG, "sp_pages_fork: parent required");
  SP_PG_CUDA(pages_fork_launch(a, parent, (cudaStream_t)stream), "sp_pages_fork");
  return SP_OK;
}

size_t sp_pages_workspace(int S, int max_pages) {
  if (check_rows("sp_pages_workspace", S, max_pages) != SP_OK) return 0;
  return pages_bytes(S, max_pages) + 256;
}

static sp_status move_pages(const char* who, const PagesArgs& a, const int* add, const int* keep, long long ld_keep,
                            int keep_cap, void* workspace, size_t workspace_bytes, cudaStream_t stream) {
  const size_t need = pages_bytes(a.S, a.max_pages) + 256;
  if (!workspace || workspace_bytes < need)
    return report(SP_ERR_WORKSPACE, "%s: workspace %zu < %zu bytes", who, workspace_bytes, need);
  void* base = reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~uintptr_t(255));
  SP_PG_CUDA(pages_move_launch(a, add, keep, ld_keep, keep_cap, base, stream), who);
  return SP_OK;
}

sp_status sp_pages_reserve(const sp_pages* p, const int* add, void* workspace, size_t workspace_bytes, sp_stream stream) {
  const char* who = "sp_pages_reserve";
  PagesArgs a;
  const sp_status s = page_args(who, p, true, &a);
  if (s != SP_OK) return s;
  if (!add) return report(SP_ERR_INVALID_ARG, "%s: add required", who);
  return move_pages(who, a, add, nullptr, 0, 0, workspace, workspace_bytes, (cudaStream_t)stream);
}

sp_status sp_pages_compact(const sp_pages* p, const int* keep, long long ld_keep, int keep_cap, const int* count,
                           void* workspace, size_t workspace_bytes, sp_stream stream) {
  const char* who = "sp_pages_compact";
  PagesArgs a;
  const sp_status s = page_args(who, p, true, &a);
  if (s != SP_OK) return s;
  if (!keep || !count) return report(SP_ERR_INVALID_ARG, "%s: keep and count required", who);
  if (keep_cap < 1 || ld_keep < keep_cap || (long long)a.S * keep_cap > (1ll << 30))
    return report(SP_ERR_SHAPE, "%s: keep_cap must be at least 1 and at most ld_keep, S * keep_cap at most 2^30", who);
  return move_pages(who, a, count, keep, ld_keep, keep_cap, workspace, workspace_bytes, (cudaStream_t)stream);
}

}  // extern "C"
