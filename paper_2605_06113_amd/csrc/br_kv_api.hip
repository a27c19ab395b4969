// C-ABI entry points of the worker's part (include/br_kv.h): argument checks, workspace layout, kernel launches.
// Host code only.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "br_kv.h"
#include "br_kv_device.h"

namespace {

uint64_t align_up(uint64_t x) { return (x + 255u) & ~(uint64_t)255u; }

int log2_of(int32_t x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

bool config_ok(const br_kv_config *c) {
  if (!c) return false;
  if (c->n_workers < 1 || c->n_workers > BR_KV_MAX_WORKERS) return false;  // (a block of 256 threads each: a launch has fewer than 2^32)
  if (c->rows < 1 || c->rows > BR_KV_MAX_ROWS || (int64_t)c->n_workers * c->rows >= 1 << 26) return false;
  if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64 && c->block_tokens != 128) return false;
  if (c->n_blocks < 1 || c->n_blocks > BR_KV_MAX_BLOCKS) return false;
  if (c->max_blocks < 1 || c->max_blocks > BR_KV_MAX_LEN / c->block_tokens) return false;
  if (c->n_kv_heads < 1 || c->n_q_heads < c->n_kv_heads || c->n_q_heads > BR_KV_MAX_HEADS || c->n_q_heads % c->n_kv_heads) return false;
  if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 192 && c->head_dim != 256) return false;
  return c->fmt == BR_KV_INT8 || c->fmt == BR_KV_E4M3;
}

struct Places {
  uint64_t lens, table, tail, used, runs, part, ml, arrived, total;
};

Places make_layout(const br_kv_config &c) {
  const uint64_t rows = (uint64_t)c.n_workers * c.rows;
  uint64_t off = 0;
  auto take = [&](uint64_t words) {
    const uint64_t at = off;
    off = align_up(off + words * 4u);
    return at;
  };
  Places l;
  l.lens = take(rows);
  l.table = take(rows * c.max_blocks);
  l.tail = take(rows);
  l.used = take((uint64_t)c.n_workers * ((c.n_blocks + 31) / 32));
  l.runs = take(2 * rows);
  // two pieces of a query tile's rows for each block of the attention's largest launch
  const uint64_t pieces = 2ull * BR_KV_SPLIT_WGS_OF(c.head_dim) * 128;
  l.part = take(pieces * c.head_dim);
  l.ml = take(pieces * 2);
  l.arrived = take(BR_KV_SPLIT_WGS);
  l.total = off;
  return l;
}

}  // namespace

struct br_kv_ctx {
  br_kv_config cfg;
  Places at;
  BrKvTables t;
  hipStream_t st;
  int32_t last_hip;
  int cus;
};

namespace {

template <class Fn>
int32_t enqueue(br_kv_ctx *ctx, Fn &&fn) {
  (void)hipGetLastError();  // an error left behind by an earlier, unrelated call is not this launch's
  fn();
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return BR_OK;
  ctx->last_hip = (int32_t)e;
  return BR_EHIP;
}

bool layer_ok(const br_kv_layer *l) {
  if (!l || !l->k || !l->v || !l->k_scale || !l->v_scale) return false;
  return (((uintptr_t)l->k | (uintptr_t)l->v | (uintptr_t)l->k_scale | (uintptr_t)l->v_scale) & 15u) == 0;
}

BrKvCache cache_of(const br_kv_ctx *ctx, const br_kv_layer *l) {
  BrKvCache c;
  c.k = l->k, c.v = l->v, c.ks = l->k_scale, c.vs = l->v_scale;
  c.shift = ctx->t.shift, c.n_blocks = ctx->cfg.n_blocks, c.heads = ctx->cfg.n_kv_heads, c.dim = ctx->cfg.head_dim;
  return c;
}

// (no token stride is looked at)
bool one_token(const br_kv_ctx *ctx, const br_kv_tokens *x) { return ctx->cfg.n_workers == 1 && x->n_tokens == 1; }

bool tokens_ok(const br_kv_ctx *ctx, const br_kv_tokens *x) {
  if (!x || x->n_tokens < 0 || x->dtype < BR_KV_F16 || x->dtype > BR_KV_F32) return false;
  if ((int64_t)ctx->cfg.n_workers * x->n_tokens > INT32_MAX - 256) return false;  // (the kernels look up to 192 places ahead)
  if (x->n_tokens == 0) return true;
  if (!x->k || !x->v || !x->slot) return false;
  if (!one_token(ctx, x) && (x->k_token < 0 || x->k_token >= BR_KV_MAX_STRIDE || x->v_token < 0 || x->v_token >= BR_KV_MAX_STRIDE))
    return false;  // (32-bit offsets within a block)
  const uintptr_t size = x->dtype == BR_KV_F32 ? 4 : 2;
  return (((uintptr_t)x->k | (uintptr_t)x->v) & (size - 1)) == 0 && ((uintptr_t)x->slot & 3u) == 0;
}

BrKvTokens tokens_of(const br_kv_ctx *ctx, const br_kv_tokens *x) {
  BrKvTokens t;
  t.k = x->k, t.v = x->v, t.slot = x->slot;
  t.k_token = x->k_token, t.k_head = x->k_head, t.v_token = x->v_token, t.v_head = x->v_head;
  if (one_token(ctx, x)) t.k_token = t.v_token = 0;
  t.n = x->n_tokens, t.W = ctx->cfg.n_workers, t.dtype = x->dtype;
  const int64_t strides = t.k_token | t.k_head | t.v_token | t.v_head;
  t.wide = (((uintptr_t)x->k | (uintptr_t)x->v) & 15u) == 0 && (strides & (x->dtype == BR_KV_F32 ? 3 : 7)) == 0;
  return t;
}

}  // namespace

extern "C" {

uint64_t br_kv_workspace_bytes(const br_kv_config *cfg) { return config_ok(cfg) ? make_layout(*cfg).total : 0; }

int32_t br_kv_init(const br_kv_config *cfg, const br_kv_state *init, br_kv_ctx **out) {
  if (!out || !config_ok(cfg) || !cfg->workspace || ((uintptr_t)cfg->workspace & 255u) != 0) return BR_EINVAL;
  if (init && (!init->lens || !init->table)) return BR_EINVAL;
  const Places at = make_layout(*cfg);
  if (cfg->workspace_bytes < at.total) return BR_ENOMEM;
  br_kv_ctx *ctx = new (std::nothrow) br_kv_ctx();
  if (!ctx) return BR_ENOMEM;
  ctx->cfg = *cfg;
  ctx->at = at;
  ctx->st = (hipStream_t)cfg->stream;
  ctx->last_hip = 0;
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&ctx->cus, hipDeviceAttributeMultiprocessorCount, device);
  if (e != hipSuccess || ctx->cus < 1) {
    delete ctx;
    return BR_EHIP;
  }
  char *base = (char *)cfg->workspace;
  BrKvTables &t = ctx->t;
  t.W = cfg->n_workers, t.B = cfg->rows, t.shift = log2_of(cfg->block_tokens);
  t.n_blocks = cfg->n_blocks, t.max_blocks = cfg->max_blocks, t.words = (cfg->n_blocks + 31) / 32;
  t.lens = (int *)(base + at.lens);
  t.table = (int *)(base + at.table);
  t.tail = (int *)(base + at.tail);
  t.used = (unsigned *)(base + at.used);
  t.arrived = (int *)(base + at.arrived);
  int32_t rc = enqueue(ctx, [&] { br_kv_launch_clear(t, ctx->st); });
  if (rc == BR_OK && init) rc = enqueue(ctx, [&] { br_kv_launch_load(t, init->lens, init->table, ctx->st); });
  if (rc != BR_OK) {
    delete ctx;
    return rc;
  }
  *out = ctx;
  return BR_OK;
}

int32_t br_kv_step(br_kv_ctx *ctx, const br_kv_lengths *in, const br_kv_step_out *out) {
  if (!ctx || !in || !in->keep || !in->add || !out || out->token_cap < 0) return BR_EINVAL;
  if ((int64_t)ctx->cfg.n_workers * out->token_cap > INT32_MAX - 2 * BR_KV_LIST) return BR_EINVAL;
  BrKvStep s;
  s.keep = in->keep, s.add = in->add;
  s.slot = out->slot, s.pos = out->pos, s.start = out->start, s.count = out->count, s.status = out->status;
  s.stats = (long long *)out->stats;
  s.runs = (int2 *)((char *)ctx->cfg.workspace + ctx->at.runs);
  s.cap = out->token_cap;
  s.wide = (((uintptr_t)s.slot | (uintptr_t)s.pos) & 15u) == 0;
  return enqueue(ctx, [&] { br_kv_launch_step(ctx->t, s, ctx->st); });
}

int32_t br_kv_append(br_kv_ctx *ctx, const br_kv_layer *layer, const br_kv_tokens *in) {
  if (!ctx || !layer_ok(layer) || !tokens_ok(ctx, in)) return BR_EINVAL;
  if (in->n_tokens == 0) return BR_OK;
  return enqueue(ctx, [&] { br_kv_launch_append(cache_of(ctx, layer), tokens_of(ctx, in), ctx->cfg.rows, ctx->cfg.fmt == BR_KV_E4M3, ctx->st); });
}

int32_t br_kv_read(br_kv_ctx *ctx, const br_kv_layer *layer, const br_kv_tokens *out) {
  if (!ctx || !layer_ok(layer) || !tokens_ok(ctx, out)) return BR_EINVAL;
  if (out->n_tokens == 0) return BR_OK;
  return enqueue(ctx, [&] { br_kv_launch_read(cache_of(ctx, layer), tokens_of(ctx, out), ctx->cfg.rows, ctx->cfg.fmt == BR_KV_E4M3, ctx->st); });
}

int32_t br_kv_attend(br_kv_ctx *ctx, const br_kv_layer *layer, const br_kv_attention *a) {
  if (!ctx || !layer_ok(layer) || !a || a->n_tokens < 0 || a->max_count < 1 || a->window < 0 || !std::isfinite(a->scale)) return BR_EINVAL;
  if (a->dtype != BR_KV_F16 && a->dtype != BR_KV_BF16) return BR_EINVAL;
  if ((a->start == nullptr) != (a->count == nullptr)) return BR_EINVAL;
  if (a->n_tokens == 0) return BR_OK;
  if (!a->q || !a->out || (((uintptr_t)a->q | (uintptr_t)a->out) & 1u) || ((uintptr_t)a->lse & 3u)) return BR_EINVAL;
  const br_kv_config &c = ctx->cfg;
  const int group = c.n_q_heads / c.n_kv_heads;
  if ((int64_t)a->n_tokens * group > INT32_MAX - 256) return BR_EINVAL;
  char *base = (char *)c.workspace;
  BrKvAttend p;
  p.q = (const unsigned short *)a->q;
  p.out = (unsigned short *)a->out;
  p.lse = a->lse;
  p.start = a->start, p.count = a->count;
  p.lens = a->lens ? a->lens : ctx->t.lens;
  p.table = a->table ? a->table : ctx->t.table;
  p.k = layer->k, p.v = layer->v, p.ks = layer->k_scale, p.vs = layer->v_scale;
  p.part = (float *)(base + ctx->at.part);
  p.ml = (float *)(base + ctx->at.ml);
  p.arrived = ctx->t.arrived;
  p.q_token = a->q_token, p.q_head = a->q_head, p.out_token = a->out_token, p.out_head = a->out_head;
  p.n_rows = c.n_workers * c.rows, p.rows = c.rows, p.n_tokens = a->n_tokens;
  p.window = a->window < c.max_blocks << ctx->t.shift ? a->window : 0;  // (a longer one hides nothing)
  p.group = group, p.kv_heads = c.n_kv_heads, p.shift = ctx->t.shift, p.n_blocks = c.n_blocks, p.max_blocks = c.max_blocks;
  p.group_shift = (unsigned)log2_of(group);
  p.group_mul = (unsigned)((((uint64_t)1 << 32) * (((uint64_t)1 << p.group_shift) - group)) / group + 1);
  p.bf16 = a->dtype == BR_KV_BF16;
  p.q_wide = ((uintptr_t)a->q & 15u) == 0 && ((a->q_token | a->q_head) & 7) == 0;
  p.out_wide = ((uintptr_t)a->out & 7u) == 0 && ((a->out_token | a->out_head) & 3) == 0;
  p.scale2 = a->scale * 1.4426950408889634f;
  // Rows of many queries share their block's token tiles, those of few have waves of their own: two launches where a call may have
  // both (two chunks of 512 tokens beside 46 single ones: 375 us in one launch).
  const int64_t rows = (int64_t)a->max_count * group;
  const bool fp8 = c.fmt == BR_KV_E4M3;
  auto launch = [&](int tile) {
    switch (c.head_dim) {
      case 64: br_kv_launch_attend_64(p, tile, fp8, ctx->cus, ctx->st); break;
      case 96: br_kv_launch_attend_96(p, tile, fp8, ctx->cus, ctx->st); break;
      case 128: br_kv_launch_attend_128(p, tile, fp8, ctx->cus, ctx->st); break;
      case 192: br_kv_launch_attend_192(p, tile, fp8, ctx->cus, ctx->st); break;
      default: br_kv_launch_attend_256(p, tile, fp8, ctx->cus, ctx->st); break;
    }
  };
  // One does where the tables span few tiles: 10 rows of up to 110 tokens and 6 key heads 13.4 us, in two launches 24; 30 rows of 470 and
  // 8 key heads, near the line, 27 to 33 us and 38.
  const int64_t tiles = (int64_t)p.n_rows * c.n_kv_heads * ((((int64_t)c.max_blocks << ctx->t.shift) + BR_KV_TILE - 1) / BR_KV_TILE);
  const bool both = rows > 64 && tiles > 8 * ctx->cus;
  const int few = both ? 16 / group : 0;  // query tokens up to which a row of a mixed call goes with the few
  p.least = 1, p.most = both ? few : INT32_MAX;
  if (rows <= 64 || few > 0) {
    const int64_t most = both ? 16 : rows;
    const int32_t rc = enqueue(ctx, [&] { launch(most <= 16 ? BR_KV_TILE_16 : most <= 32 ? BR_KV_TILE_32 : BR_KV_TILE_64); });
    if (rc != BR_OK || rows <= 64) return rc;
  }
  p.least = few + 1, p.most = INT32_MAX;
  return enqueue(ctx, [&] { launch(BR_KV_TILE_128); });
}

void br_kv_free(br_kv_ctx *ctx) { delete ctx; }

int32_t br_kv_last_hip_error(const br_kv_ctx *ctx) { return ctx ? ctx->last_hip : 0; }

int32_t br_kv_get_layout(const br_kv_ctx *ctx, br_kv_layout *out) {
  if (!ctx || !out) return BR_EINVAL;
  out->lens = ctx->at.lens;
  out->table = ctx->at.table;
  out->total_bytes = ctx->at.total;
  return BR_OK;
}

}  // extern "C"
