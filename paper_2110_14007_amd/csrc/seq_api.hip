// Host side of the sequence operators: argument checks and launches.  Nothing
// here waits for the GPU or allocates, so the calls may be captured into a
// HIP graph.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include "seq.h"

namespace {

using tod::set_error;

constexpr int64_t kMaxCount = 0x7fffffffLL;
constexpr int32_t kPartKeys = 512;  // fewest keys of a split of a tile
constexpr int64_t kBeyond = 64;     // positions past a sequence's last that its last stages name

tod_status invalid(const char* msg) { return set_error(TOD_ERR_INVALID_ARG, msg); }
tod_status unsupported(const char* msg) { return set_error(TOD_ERR_UNSUPPORTED, msg); }

tod_status launched(hipError_t e, const char* where) {
  if (e == hipSuccess) return TOD_OK;
  char msg[256];
  snprintf(msg, sizeof(msg), "%s: %s", where, hipGetErrorString(e));
  return set_error(TOD_ERR_HIP, msg);
}

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

tod_status check_pages(int64_t n_pages, int32_t page_rows, int64_t kv_heads) {
  if (page_rows <= 0 || page_rows > 65536)
    return invalid("page_rows must be in [1, 65536]");
  if (n_pages <= 0) return invalid("the cache needs at least one page");
  if (n_pages > kMaxCount / page_rows / kv_heads)
    return unsupported("more than 2^31 - 1 rows of all heads in the cache");
  return TOD_OK;
}

tod_status check_half(int32_t precision) {
  if (precision == TOD_PREC_FP16 || precision == TOD_PREC_BF16) return TOD_OK;
  return precision == TOD_PREC_FP32 || precision == TOD_PREC_AUTO
             ? unsupported("sequence operators take fp16 or bf16 tensors")
             : invalid("unknown precision");
}

// Sizes, types and strides that all attention calls share.  rows: the row and
// head strides that *a leaves 0 become those of a contiguous [rows, heads, dim].
tod_status check_attn(const tod_attn* a, tod_attn* out) {
  if (!a) return invalid("null tod_attn");
  if (a->struct_size != sizeof(tod_attn))
    return invalid("tod_attn.struct_size does not match this library");
  *out = *a;
  const tod_status st = check_half(a->precision);
  if (st != TOD_OK) return st;
  if (a->heads <= 0 || a->kv_heads <= 0 || a->dim <= 0)
    return invalid("heads, kv_heads and dim must be positive");
  if (a->heads % a->kv_heads)
    return invalid("heads must be a multiple of kv_heads");
  if (a->dim % 8) return unsupported("dim must be a multiple of 8");
  if (a->dim > 256) return unsupported("dim > 256");
  if (a->heads > 65536) return unsupported("more than 65536 heads");
  if (a->causal != 0 && a->causal != 1) return invalid("causal must be 0 or 1");
  if (!(a->scale >= 0.0f) || isinf(a->scale))
    return invalid("scale must be finite and positive (0: 1 / sqrt(dim))");
  int64_t* const strides[6] = {&out->q_row, &out->q_head, &out->k_row,
                               &out->k_head, &out->v_row, &out->v_head};
  for (int i = 0; i < 6; ++i) {
    if (*strides[i] < 0) return invalid("strides must not be negative");
    if (*strides[i] % 8) return unsupported("strides must be multiples of 8 elements");
    if (*strides[i] == 0)
      *strides[i] = i % 2 ? a->dim : (int64_t)a->dim * (i == 0 ? a->heads : a->kv_heads);
  }
  if (out->scale == 0.0f) out->scale = 1.0f / sqrtf((float)a->dim);
  return TOD_OK;
}

tod_status check_rows(const tod_attn& a, int64_t tokens, int64_t n_seq) {
  if (tokens <= 0 || n_seq <= 0) return invalid("tokens and n_seq must be positive");
  if (n_seq > kMaxCount / 2) return unsupported("more than 2^30 - 1 sequences");
  const int64_t group = a.heads / a.kv_heads;
  // Rows and tile slots (tokens * group / 128 + n_seq + 1 a head) in 32 bits; make_plan() has the
  // launches.
  if (tokens > kMaxCount / 2 / group ||
      tokens * group / 128 + n_seq + 1 > kMaxCount / 32 / a.kv_heads)
    return unsupported("too many rows for one call");
  return TOD_OK;
}

void fill(const tod_attn& o, tod::AttnArgs* a) {
  memset(a, 0, sizeof(*a));
  a->q_row = o.q_row;
  a->q_head = o.q_head;
  a->k_row = o.k_row;
  a->k_head = o.k_head;
  a->v_row = o.v_row;
  a->v_head = o.v_head;
  a->heads = o.heads;
  a->kv_heads = o.kv_heads;
  a->dim = o.dim;
  a->group = tod::fast_div((uint32_t)(o.heads / o.kv_heads));
  a->heads_div = tod::fast_div((uint32_t)o.kv_heads);
  a->page = tod::fast_div(1);
  a->causal = o.causal;
  a->scale = o.scale * 1.44269504088896341f;
  a->unscale = 1.0f / a->scale;
}

// Workspace of a call, and how its work is split.
struct Plan {
  int32_t skip_rows, tile_parts;
  int64_t tile_slots;
  bool tile;  // some sequence may have more rows than the token kernel takes
  bool fits;  // every launch has fewer than 2^32 threads
  size_t line, token_stat, token_o, tile_stat, tile_o, tile_cut, total;
};

enum class Form { kPrompt, kPaged, kPaged4 };  // whole prompts; pages; pages of a 4-bit cache

// Over pages a call may hold sequences of few tokens for the token kernel.
Plan make_plan(const tod_attn& o, int64_t tokens, int64_t n_seq, int64_t max_fresh, Form form) {
  const bool paged = form != Form::kPrompt;
  Plan p;
  memset(&p, 0, sizeof(p));
  const int64_t group = o.heads / o.kv_heads;
  const int64_t most = max_fresh < tokens ? max_fresh * group : tokens * group;
  const int64_t dp = o.dim <= 64 ? 64 : o.dim <= 128 ? 128 : 256;
  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t here = at;
    at += (size_t)((bytes + 255) / 256 * 256);
    return here;
  };
  p.tile = !paged || most > tod::kTokenMaxRows;
  if (paged && group <= tod::kTokenMaxRows) {
    // Beside tiles the workers over a 4-bit cache keep one block of 16 rows where a token fits in;
    // sequences of more rows are tiles.  (4 chunks beside 44 times 4 new tokens, 64 / 8 heads: 167 us,
    // with blocks of 32 in a launch of their own 181.)
    const bool four = form == Form::kPaged4;
    const int64_t limit = four && p.tile && group <= 16 ? 16 : tod::kTokenMaxRows;
    p.skip_rows = (int32_t)(most < limit ? most : limit / group * group);
    const int64_t workers = !four   ? tod::token_workers(o.dim)
                            : p.tile && p.skip_rows <= 16 ? 4 * (int64_t)tod::tile4_workers(o.dim)
                                                          : tod::token4_workers(o.dim);
    const int64_t rows = 2 * workers * p.skip_rows;
    p.line = take((n_seq + 1) * 8);
    p.token_stat = take(rows * 8);
    p.token_o = take(rows * dp * 4);
  }
  p.tile_parts = 1;
  p.tile_slots = tokens * group / 128 + n_seq + 1;
  if (p.tile && form == Form::kPaged4) {
    // Two pieces of a tile for every worker.
    const int64_t workers = tod::tile4_workers(o.dim);
    p.tile_stat = take(workers * 2 * 128 * 8);
    p.tile_o = take(workers * 2 * 128 * dp * 4);
    p.tile_cut = take(workers * (int64_t)sizeof(tod::TileCut));
  } else if (p.tile) {
    // Two workgroups on every compute unit, from the rows that there are; slots beside them, one a
    // sequence and head, stay empty but count towards the 2,048 workgroups.  A prompt has no more
    // keys than tokens; a split has at least 512.  (512 tokens after 60,007, 2 heads of 128: 8 parts
    // 312 us, 4 415, 16 327, unsplit 1,380; 256 after 8,000, 8 heads: 8 parts 62, 4 73, 16 77,
    // unsplit 197; 64 after 30,000: 32 parts 63, 16 68.  Splitting only the longest tiles of a step
    // of mixed lengths cost more in partial results, 345 us, than it evened out, 280.)
    const int64_t tiles = (tokens * group + 127) / 128 * o.kv_heads;
    const int64_t slots = p.tile_slots * o.kv_heads;
    int64_t parts = 512 / tiles;
    if (!paged && parts > tokens / kPartKeys) parts = tokens / kPartKeys;
    while (parts > 1 && (parts > 64 || slots * parts > 2048)) --parts;
    p.tile_parts = (int32_t)(parts < 1 ? 1 : parts);
    if (p.tile_parts > 1) {
      p.tile_stat = take(slots * p.tile_parts * 128 * 8);
      p.tile_o = take(slots * p.tile_parts * 128 * dp * 4);
    }
  }
  // (Where tiles are split, their slots times splits are few, and so are the join's workgroups.
  // The tokens' join has a workgroup of a wave a row, at most 8, for every pair.)
  constexpr int64_t kThreads = 1LL << 32;
  const int64_t join = 64 * (p.skip_rows < 8 ? p.skip_rows : 8);
  const int64_t beside = form == Form::kPaged4 ? 2048 : 0;  // more than the tiles' workgroups
  p.fits = (!p.tile || (p.tile_slots * o.kv_heads * p.tile_parts + 1024) * 256 < kThreads) &&
           (n_seq * o.kv_heads + beside) * join < kThreads;
  p.total = at ? at : 256;
  return p;
}

tod_status run_attn(const tod_attn& o, tod::AttnArgs* a, const Plan& p, Form form, void* ws,
                    size_t ws_bytes, void* stream, const char* where) {
  if (!p.fits) return unsupported("too many rows for one call");
  if (!aligned(ws, 256)) return set_error(TOD_ERR_WORKSPACE, "workspace misaligned");
  if (ws_bytes < p.total)
    return set_error(TOD_ERR_WORKSPACE,
                     form == Form::kPaged4
                         ? "workspace smaller than tod_attn_paged4_workspace_size()"
                         : "workspace smaller than tod_attn_workspace_size()");
  char* const base = (char*)ws;
  a->skip_rows = p.skip_rows;
  a->token_tail = p.tile ? 0 : 1;
  a->token_line = (int64_t*)(base + p.line);
  a->token_stat = (float2*)(base + p.token_stat);
  a->token_o = (float*)(base + p.token_o);
  a->tile_slots = (int32_t)p.tile_slots;
  a->tile_parts = p.tile_parts;
  a->tile_groups = form == Form::kPaged4 ? (uint32_t)tod::tile4_workers(o.dim)
                                         : (uint32_t)(p.tile_slots * o.kv_heads * p.tile_parts);
  a->tile_cut = (tod::TileCut*)(base + p.tile_cut);
  a->parts_div = tod::fast_div((uint32_t)p.tile_parts);
  a->part_keys = kPartKeys;
  a->tile_stat = (float2*)(base + p.tile_stat);
  a->tile_o = (float*)(base + p.tile_o);
  const hipStream_t s = (hipStream_t)stream;
  const bool half = o.precision == TOD_PREC_FP16;
  hipError_t e = hipSuccess;
  const bool paged = form == Form::kPaged;
  if (form == Form::kPaged4) {
    a->ride = p.tile && p.skip_rows && p.skip_rows <= 16;
    if (p.tile)
      e = half ? tod::launch_attn_tile4_f16(*a, s) : tod::launch_attn_tile4_bf16(*a, s);
    if (e == hipSuccess && p.skip_rows && !a->ride)
      e = half ? tod::launch_attn_token4_f16(*a, s) : tod::launch_attn_token4_bf16(*a, s);
    return launched(e, where);
  }
  // The tile kernel's launch holds the token workers too.
  if (p.tile)
    e = half ? tod::launch_attn_tile_f16(*a, paged, s) : tod::launch_attn_tile_bf16(*a, paged, s);
  else
    e = half ? tod::launch_attn_token_f16(*a, s) : tod::launch_attn_token_bf16(*a, s);
  if (e == hipSuccess && p.skip_rows)
    e = half ? tod::launch_attn_token_join_f16(*a, s) : tod::launch_attn_token_join_bf16(*a, s);
  return launched(e, where);
}

// What attention over pages of either kind shares: the checks and the arguments beside the pages'.
tod_status over_pages(const tod_attn& o, const void* q, int64_t n_pages, int32_t page_rows,
                      const int32_t* table, int64_t table_cols, const int32_t* row_start,
                      const int32_t* cached, int64_t n_seq, int64_t tokens, int64_t max_fresh,
                      void* workspace, void* out, float* lse_out, tod::AttnArgs* a) {
  if (!q || !table || !row_start || !cached || !out || !workspace) return invalid("null pointer");
  if (!o.causal) return unsupported("attention over pages is causal");
  tod_status st = check_rows(o, tokens, n_seq);
  if (st != TOD_OK) return st;
  if ((st = check_pages(n_pages, page_rows, o.kv_heads)) != TOD_OK) return st;
  if (table_cols <= 0 || max_fresh <= 0)
    return invalid("table_cols and max_fresh must be positive");
  if (table_cols > (kMaxCount - kBeyond - tokens) / page_rows)
    return unsupported("positions that do not fit into 32 bits");
  if (!aligned(q, 16) || !aligned(out, 16)) return invalid("tensors must be 16-byte aligned");
  if (!aligned(table, 4) || !aligned(row_start, 4) || !aligned(cached, 4) || !aligned(lse_out, 4))
    return invalid("misaligned pointer");
  a->q = q;
  a->row_start = row_start;
  a->cached = cached;
  a->table = table;
  a->cols = table_cols;
  a->n_pages = (int32_t)n_pages;
  a->page = tod::fast_div((uint32_t)page_rows);
  a->n_seq = (int32_t)n_seq;
  a->tokens = (int32_t)tokens;
  a->out = out;
  a->lse = lse_out;
  return TOD_OK;
}

tod_status check_cache4(const tod_cache4* c) {
  if (!c) return invalid("null tod_cache4");
  if (c->struct_size != sizeof(tod_cache4))
    return invalid("tod_cache4.struct_size does not match this library");
  if (!c->k_codes || !c->k_scales || !c->v_codes || !c->v_scales) return invalid("null pointer");
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scales, 16) ||
      !aligned(c->v_scales, 16))
    return invalid("codes and scales must be 16-byte aligned");
  return TOD_OK;
}

// Whether the rows of x [tokens, heads, dim], by their strides, share memory with the contiguous out.
bool overlap(const void* x, int64_t row, int64_t head, int64_t tokens, int32_t heads, int32_t dim,
             const void* out, int64_t out_bytes) {
  typedef unsigned __int128 u128;  // (strides may be anything)
  const u128 a = (uintptr_t)x, b = (uintptr_t)out;
  const u128 n = 2 * ((u128)(tokens - 1) * (u128)row + (u128)(heads - 1) * (u128)head + (u128)dim);
  return a < b + (u128)out_bytes && b < a + n;
}

// Checks and arguments that both appends share.
tod_status check_append(const tod_append* o, const void* q, const void* k, const void* v,
                        int64_t tokens, const int32_t* pos, const float* rates,
                        const int64_t* slot, int64_t n_pages, int32_t page_rows, void* q_out,
                        tod::AppendArgs* a) {
  if (!o) return invalid("null tod_append");
  if (o->struct_size != sizeof(tod_append))
    return invalid("tod_append.struct_size does not match this library");
  tod_status st = check_half(o->precision);
  if (st != TOD_OK) return st;
  if (tokens <= 0 || o->heads <= 0 || o->kv_heads <= 0 || o->dim <= 0)
    return invalid("tokens, heads, kv_heads and dim must be positive");
  if (o->dim % 8) return unsupported("dim must be a multiple of 8");
  if (o->dim > 256) return unsupported("dim > 256");
  if (o->rotary < 0 || o->rotary > o->dim || o->rotary % 2)
    return invalid("rotary must be even and in [0, dim]");
  if (o->interleaved != 0 && o->interleaved != 1) return invalid("interleaved must be 0 or 1");
  if (!q || !k || !v || !pos || !slot || !q_out || (o->rotary && !rates))
    return invalid("null pointer");
  if ((st = check_pages(n_pages, page_rows, o->kv_heads)) != TOD_OK) return st;
  // A token's pieces count in 32 bits; strides as 64-bit products.
  if ((int64_t)o->heads + 2 * (int64_t)o->kv_heads > 65536 || tokens > kMaxCount)
    return unsupported("more than 65536 heads of queries, keys and values, or 2^31 - 1 tokens");
  memset(a, 0, sizeof(*a));
  const int64_t given[6] = {o->q_row, o->q_head, o->k_row, o->k_head, o->v_row, o->v_head};
  int64_t* const to[6] = {&a->q_row, &a->q_head, &a->k_row, &a->k_head, &a->v_row, &a->v_head};
  for (int i = 0; i < 6; ++i) {
    if (given[i] < 0) return invalid("strides must not be negative");
    if (given[i] % 8) return unsupported("strides must be multiples of 8 elements");
    *to[i] = given[i] ? given[i]
                      : i % 2 ? o->dim : (int64_t)o->dim * (i == 0 ? o->heads : o->kv_heads);
  }
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16))
    return invalid("tensors must be 16-byte aligned");
  if (!aligned(pos, 4) || !aligned(rates, 4) || !aligned(slot, 8))
    return invalid("misaligned pointer");
  const int64_t out_bytes = 2 * tokens * o->heads * o->dim;
  if (overlap(q, a->q_row, a->q_head, tokens, o->heads, o->dim, q_out, out_bytes) ||
      overlap(k, a->k_row, a->k_head, tokens, o->kv_heads, o->dim, q_out, out_bytes) ||
      overlap(v, a->v_row, a->v_head, tokens, o->kv_heads, o->dim, q_out, out_bytes))
    return invalid("q_out shares memory with an input");
  a->q = q;
  a->k = k;
  a->v = v;
  a->pos = pos;
  a->rates = rates;
  a->slot = slot;
  a->q_out = q_out;
  a->tokens = tokens;
  a->slots = n_pages * page_rows;
  a->page = tod::fast_div((uint32_t)page_rows);
  a->per_row = tod::fast_div((uint32_t)(o->dim / 8));
  a->heads = o->heads;
  a->kv_heads = o->kv_heads;
  a->rotary = o->rotary;
  a->interleaved = o->interleaved;
  return TOD_OK;
}

}  // namespace

extern "C" {

void tod_default_attn(tod_attn* a, int32_t heads, int32_t kv_heads, int32_t dim,
                      int32_t precision) {
  if (!a) return;
  memset(a, 0, sizeof(*a));
  a->struct_size = sizeof(*a);
  a->precision = precision;
  a->heads = heads;
  a->kv_heads = kv_heads;
  a->dim = dim;
  a->causal = 1;
}

tod_status tod_page_map(const int32_t* cached, const int32_t* fresh, int64_t n_seq,
                        const int32_t* free_pages, int64_t n_free, int32_t page_rows,
                        int32_t* table, int64_t table_cols, int64_t tokens, void* stream,
                        int32_t* row_start_out, int64_t* slot_out, int32_t* pos_out,
                        int64_t* used_out) {
  set_error(TOD_OK, "");
  if (!cached || !fresh || !table || !row_start_out || !slot_out)
    return invalid("null pointer");
  if (n_seq <= 0 || tokens <= 0 || table_cols <= 0)
    return invalid("n_seq, tokens and table_cols must be positive");
  if (n_free < 0 || (n_free > 0 && !free_pages)) return invalid("free_pages missing");
  if (page_rows <= 0 || page_rows > 65536) return invalid("page_rows must be in [1, 65536]");
  if (n_seq > kMaxCount || tokens > kMaxCount || table_cols > kMaxCount / page_rows)
    return unsupported("more than 2^31 - 1 sequences, tokens or positions");
  if (!aligned(cached, 4) || !aligned(fresh, 4) || !aligned(free_pages, 4) ||
      !aligned(table, 4) || !aligned(row_start_out, 4) || !aligned(pos_out, 4) ||
      !aligned(slot_out, 8) || !aligned(used_out, 8))
    return invalid("misaligned pointer");
  tod::PageMapArgs a;
  a.cached = cached;
  a.fresh = fresh;
  a.free_pages = free_pages;
  a.n_seq = n_seq;
  a.n_free = n_free;
  a.cols = table_cols;
  a.tokens = tokens;
  a.page = tod::fast_div((uint32_t)page_rows);
  a.table = table;
  a.row_start = row_start_out;
  a.pos = pos_out;
  a.slot = slot_out;
  a.used = used_out;
  return launched(tod::launch_page_map(a, (hipStream_t)stream), "tod_page_map");
}

tod_status tod_page_write(const void* k, const void* v, int64_t tokens, int32_t kv_heads,
                          int32_t dim, int64_t k_row, int64_t k_head, int64_t v_row,
                          int64_t v_head, const int64_t* slot, void* k_pages, void* v_pages,
                          int64_t n_pages, int32_t page_rows, void* stream) {
  set_error(TOD_OK, "");
  if (!k || !v || !slot || !k_pages || !v_pages) return invalid("null pointer");
  if (tokens <= 0 || kv_heads <= 0 || dim <= 0)
    return invalid("tokens, kv_heads and dim must be positive");
  if (dim % 8) return unsupported("dim must be a multiple of 8");
  if (k_row < 0 || k_head < 0 || v_row < 0 || v_head < 0)
    return invalid("strides must not be negative");
  if (k_row % 8 || k_head % 8 || v_row % 8 || v_head % 8)
    return unsupported("strides must be multiples of 8 elements");
  const tod_status st = check_pages(n_pages, page_rows, kv_heads);
  if (st != TOD_OK) return st;
  const int64_t per_row = dim / 8;
  if (per_row > kMaxCount / kv_heads || tokens > (kMaxCount - 256) / (per_row * kv_heads))
    return unsupported("more than 2^31 - 1 pieces of 16 bytes in one call");
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16))
    return invalid("tensors must be 16-byte aligned");
  if (!aligned(slot, 8)) return invalid("misaligned pointer");
  tod::PageWriteArgs a;
  a.k = k;
  a.v = v;
  a.k_head = k_head ? k_head : dim;
  a.v_head = v_head ? v_head : dim;
  a.k_row = k_row ? k_row : (int64_t)kv_heads * dim;
  a.v_row = v_row ? v_row : (int64_t)kv_heads * dim;
  a.slot = slot;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.tokens = tokens;
  a.slots = n_pages * page_rows;
  a.page = tod::fast_div((uint32_t)page_rows);
  a.per_token = tod::fast_div((uint32_t)(per_row * kv_heads));
  a.per_row = tod::fast_div((uint32_t)per_row);
  a.kv_heads = kv_heads;
  return launched(tod::launch_page_write(a, (hipStream_t)stream), "tod_page_write");
}

size_t tod_attn_workspace_size(const tod_attn* attn, int64_t tokens, int64_t n_seq,
                               int64_t max_fresh) {
  tod_attn o;
  if (check_attn(attn, &o) != TOD_OK || check_rows(o, tokens, n_seq) != TOD_OK || max_fresh <= 0)
    return 0;
  const Plan paged = make_plan(o, tokens, n_seq, max_fresh, Form::kPaged);
  const Plan prompt = make_plan(o, tokens, n_seq, max_fresh, Form::kPrompt);
  const size_t a = paged.fits ? paged.total : 0, b = prompt.fits ? prompt.total : 0;
  return a > b ? a : b;
}

tod_status tod_attn_prompt(const tod_attn* attn, const void* q, const void* k, const void* v,
                           int64_t tokens, const int32_t* row_start, int64_t n_seq,
                           void* workspace, size_t ws_bytes, void* stream, void* out,
                           float* lse_out) {
  set_error(TOD_OK, "");
  tod_attn o;
  tod_status st = check_attn(attn, &o);
  if (st != TOD_OK) return st;
  if (!q || !k || !v || !row_start || !out || !workspace) return invalid("null pointer");
  if ((st = check_rows(o, tokens, n_seq)) != TOD_OK) return st;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16))
    return invalid("tensors must be 16-byte aligned");
  if (!aligned(row_start, 4) || !aligned(lse_out, 4)) return invalid("misaligned pointer");
  tod::AttnArgs a;
  fill(o, &a);
  a.q = q;
  a.k = k;
  a.v = v;
  a.row_start = row_start;
  a.n_seq = (int32_t)n_seq;
  a.tokens = (int32_t)tokens;
  a.out = out;
  a.lse = lse_out;
  return run_attn(o, &a, make_plan(o, tokens, n_seq, tokens, Form::kPrompt), Form::kPrompt,
                  workspace, ws_bytes, stream, "tod_attn_prompt");
}

tod_status tod_attn_paged(const tod_attn* attn, const void* q, const void* k_pages,
                          const void* v_pages, int64_t n_pages, int32_t page_rows,
                          const int32_t* table, int64_t table_cols, const int32_t* row_start,
                          const int32_t* cached, int64_t n_seq, int64_t tokens,
                          int64_t max_fresh, void* workspace, size_t ws_bytes, void* stream,
                          void* out, float* lse_out) {
  set_error(TOD_OK, "");
  tod_attn o;
  tod_status st = check_attn(attn, &o);
  if (st != TOD_OK) return st;
  if (!k_pages || !v_pages) return invalid("null pointer");
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16))
    return invalid("tensors must be 16-byte aligned");
  tod::AttnArgs a;
  fill(o, &a);
  a.k = k_pages;
  a.v = v_pages;
  st = over_pages(o, q, n_pages, page_rows, table, table_cols, row_start, cached, n_seq, tokens,
                  max_fresh, workspace, out, lse_out, &a);
  if (st != TOD_OK) return st;
  return run_attn(o, &a, make_plan(o, tokens, n_seq, max_fresh, Form::kPaged), Form::kPaged,
                  workspace, ws_bytes, stream, "tod_attn_paged");
}

void tod_default_append(tod_append* a, int32_t heads, int32_t kv_heads, int32_t dim,
                        int32_t precision) {
  if (!a) return;
  memset(a, 0, sizeof(*a));
  a->struct_size = sizeof(*a);
  a->precision = precision;
  a->heads = heads;
  a->kv_heads = kv_heads;
  a->dim = dim;
  a->rotary = dim;
}

tod_status tod_page_append(const tod_append* append, const void* q, const void* k, const void* v,
                           int64_t tokens, const int32_t* pos, const float* rates,
                           const int64_t* slot, void* k_pages, void* v_pages, int64_t n_pages,
                           int32_t page_rows, void* stream, void* q_out) {
  set_error(TOD_OK, "");
  tod::AppendArgs a;
  const tod_status st = check_append(append, q, k, v, tokens, pos, rates, slot, n_pages, page_rows,
                                     q_out, &a);
  if (st != TOD_OK) return st;
  if (!k_pages || !v_pages) return invalid("null pointer");
  if (!aligned(k_pages, 16) || !aligned(v_pages, 16))
    return invalid("tensors must be 16-byte aligned");
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  return launched(tod::launch_append(a, append->precision == TOD_PREC_FP16, false,
                                     (hipStream_t)stream), "tod_page_append");
}

tod_status tod_page_append4(const tod_append* append, const void* q, const void* k, const void* v,
                            int64_t tokens, const int32_t* pos, const float* rates,
                            const int64_t* slot, const tod_cache4* cache, void* stream,
                            void* q_out) {
  set_error(TOD_OK, "");
  tod_status st = check_cache4(cache);
  if (st != TOD_OK) return st;
  tod::AppendArgs a;
  st = check_append(append, q, k, v, tokens, pos, rates, slot, cache->n_pages, cache->page_rows,
                    q_out, &a);
  if (st != TOD_OK) return st;
  if (append->dim % 32) return unsupported("dim must be a multiple of 32");
  a.k_pages = cache->k_codes;
  a.v_pages = cache->v_codes;
  a.k_scales = cache->k_scales;
  a.v_scales = cache->v_scales;
  return launched(tod::launch_append(a, append->precision == TOD_PREC_FP16, true,
                                     (hipStream_t)stream), "tod_page_append4");
}

tod_status tod_page_read4(const tod_cache4* cache, int32_t kv_heads, int32_t dim,
                          int32_t precision, const int64_t* slot, int64_t tokens, void* stream,
                          void* k_out, void* v_out) {
  set_error(TOD_OK, "");
  tod_status st = check_cache4(cache);
  if (st != TOD_OK) return st;
  if (!slot || !k_out || !v_out) return invalid("null pointer");
  if (tokens <= 0 || kv_heads <= 0 || dim <= 0)
    return invalid("tokens, kv_heads and dim must be positive");
  if ((st = check_half(precision)) != TOD_OK) return st;
  if (dim % 32) return unsupported("dim must be a multiple of 32");
  if (dim > 256) return unsupported("dim > 256");
  if ((st = check_pages(cache->n_pages, cache->page_rows, kv_heads)) != TOD_OK) return st;
  const int64_t per_token = (int64_t)(dim / 8) * kv_heads;
  if (per_token > kMaxCount || tokens > (kMaxCount - 256) / per_token)
    return unsupported("more than 2^31 - 1 pieces of 16 bytes in one call");
  if (!aligned(k_out, 16) || !aligned(v_out, 16))
    return invalid("tensors must be 16-byte aligned");
  if (!aligned(slot, 8)) return invalid("misaligned pointer");
  tod::Read4Args a;
  a.k_codes = cache->k_codes;
  a.v_codes = cache->v_codes;
  a.k_scales = cache->k_scales;
  a.v_scales = cache->v_scales;
  a.slot = slot;
  a.k_out = k_out;
  a.v_out = v_out;
  a.tokens = tokens;
  a.slots = cache->n_pages * cache->page_rows;
  a.page = tod::fast_div((uint32_t)cache->page_rows);
  a.per_token = tod::fast_div((uint32_t)per_token);
  a.per_row = tod::fast_div((uint32_t)(dim / 8));
  a.kv_heads = kv_heads;
  return launched(tod::launch_read4(a, precision == TOD_PREC_FP16, (hipStream_t)stream),
                  "tod_page_read4");
}

size_t tod_attn_paged4_workspace_size(const tod_attn* attn, int64_t tokens, int64_t n_seq,
                                      int64_t max_fresh) {
  tod_attn o;
  if (check_attn(attn, &o) != TOD_OK || check_rows(o, tokens, n_seq) != TOD_OK || max_fresh <= 0 ||
      o.dim % 32)
    return 0;
  const Plan p = make_plan(o, tokens, n_seq, max_fresh, Form::kPaged4);
  return p.fits ? p.total : 0;
}

tod_status tod_attn_paged4(const tod_attn* attn, const void* q, const tod_cache4* cache,
                           const int32_t* table, int64_t table_cols, const int32_t* row_start,
                           const int32_t* cached, int64_t n_seq, int64_t tokens,
                           int64_t max_fresh, void* workspace, size_t ws_bytes, void* stream,
                           void* out, float* lse_out) {
  set_error(TOD_OK, "");
  tod_attn o;
  tod_status st = check_attn(attn, &o);
  if (st != TOD_OK) return st;
  if (o.dim % 32) return unsupported("dim must be a multiple of 32");
  if ((st = check_cache4(cache)) != TOD_OK) return st;
  tod::AttnArgs a;
  fill(o, &a);
  a.k = cache->k_codes;
  a.v = cache->v_codes;
  a.k_scales = cache->k_scales;
  a.v_scales = cache->v_scales;
  st = over_pages(o, q, cache->n_pages, cache->page_rows, table, table_cols, row_start, cached,
                  n_seq, tokens, max_fresh, workspace, out, lse_out, &a);
  if (st != TOD_OK) return st;
  return run_attn(o, &a, make_plan(o, tokens, n_seq, max_fresh, Form::kPaged4), Form::kPaged4,
                  workspace, ws_bytes, stream, "tod_attn_paged4");
}

}  // extern "C"
