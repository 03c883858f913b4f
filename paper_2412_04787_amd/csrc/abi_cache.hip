// C ABI, second part: rotary positions, the 8-bit cache of keys and values, attention
// over it, its pages.  Every check runs before anything is enqueued; see
// include/dqt.h for the contract of each entry point.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include "abi_check.h"
#include "cache_launch.h"

namespace {

constexpr int64_t kMaxTokens = (int64_t(1) << 31) - 1;

dqt_status check_rope(const dqt_rope* r) {
  if (r == nullptr) return DQT_ERR_NULL;
  if (r->d < 16 || r->d > 1024 || r->d % 16 != 0 || r->rot < 16 || r->rot > r->d || r->rot % 16 != 0) return DQT_ERR_SHAPE;
  if (r->freq == nullptr) return DQT_ERR_NULL;
  if (!aligned8(r->freq)) return DQT_ERR_ALIGN;
  if ((r->pairs != 0 && r->pairs != 1) || r->reserved != 0 || !isfinite(r->amp)) return DQT_ERR_RANGE;
  return DQT_OK;
}

dqt_status rope(const dqt_rope* r, int32_t n, const dqt_rope_io* io, int32_t x_t, int64_t tokens, const int32_t* pos,
                void* stream, int back) {
  dqt_status st = check_rope(r);
  if (st != DQT_OK) return st;
  if (n < 1 || n > DQT_MAX_ROPE) return DQT_ERR_SHAPE;
  if (io == nullptr) return DQT_ERR_NULL;
  if (!is_float_type(x_t)) return DQT_ERR_DTYPE;
  if (tokens < 0 || tokens > kMaxTokens || tokens >= 4 * kMaxBlocks) return DQT_ERR_SHAPE;
  if (!aligned4(pos)) return DQT_ERR_ALIGN;
  dqt::RopeArgs a{};
  const int64_t size = x_t == DQT_BF16 ? 2 : 4;
  for (int t = 0; t < n; ++t) {
    if (io[t].heads < 1 || io[t].heads > 1024) return DQT_ERR_SHAPE;
    if (io[t].reserved != 0) return DQT_ERR_RANGE;
    if ((st = check_rows(&io[t].X, tokens, io[t].heads, r->d, false)) != DQT_OK) return st;
    if ((st = check_rows(&io[t].Y, tokens, io[t].heads, r->d, true)) != DQT_OK) return st;
    // (in place: the same rows)
    if (io[t].X.p == io[t].Y.p && ((tokens > 1 && io[t].X.token != io[t].Y.token) || (io[t].heads > 1 && io[t].X.head != io[t].Y.head)))
      return DQT_ERR_SHAPE;
    dqt::RopeIO& o = a.io[t];
    o.X = static_cast<const uint8_t*>(io[t].X.p);
    o.Y = static_cast<uint8_t*>(io[t].Y.p);
    o.x_tok = io[t].X.token * size;
    o.x_head = io[t].X.head * size;
    o.y_tok = io[t].Y.token * size;
    o.y_head = io[t].Y.head * size;
    o.heads = io[t].heads;
    a.all_heads += io[t].heads;
  }
  if (tokens == 0) return DQT_OK;
  a.freq = r->freq;
  a.pos = pos;
  a.tokens = tokens;
  a.amp = r->amp;
  a.n = n;
  a.d = r->d;
  a.rot = r->rot;
  a.pairs = r->pairs;
  a.back = back;
  return from_hip(dqt::launch_rope(x_t == DQT_BF16, a, static_cast<hipStream_t>(stream)));
}

dqt_status check_cache(const dqt_kv_cache* c) {
  if (c == nullptr) return DQT_ERR_NULL;
  if (c->pages < 0 || c->pages > kMaxTokens || c->kv_heads < 1 || c->kv_heads > 1024) return DQT_ERR_SHAPE;
  if (c->d != 64 && c->d != 128) return DQT_ERR_SHAPE;
  if (c->fmt != DQT_FP8E4M3 && c->fmt != DQT_I8) return DQT_ERR_DTYPE;
  if (c->reserved != 0) return DQT_ERR_RANGE;
  if (c->pages > 0 && (c->K == nullptr || c->V == nullptr || c->scales == nullptr)) return DQT_ERR_NULL;
  if (!aligned16(c->K) || !aligned16(c->V) || !aligned8(c->scales)) return DQT_ERR_ALIGN;
  return DQT_OK;
}

// Checks cache and batch and fills what the kernels take of both.
dqt_status check_batch(const dqt_kv_cache* c, const dqt_kv_batch* b, dqt::KvArgs* a) {
  dqt_status st = check_cache(c);
  if (st != DQT_OK) return st;
  if (b == nullptr) return DQT_ERR_NULL;
  if (b->n_seq < 0 || b->table_stride < 0 || b->q_tokens < 0 || b->q_tokens > kMaxTokens) return DQT_ERR_SHAPE;
  if (b->heads < 1 || b->heads > 1024 || b->heads % c->kv_heads != 0) return DQT_ERR_SHAPE;
  if (b->q_tokens * b->heads > kMaxTokens) return DQT_ERR_SHAPE;
  if (b->max_len < 0 || b->max_len > kMaxTokens - 1023 || b->max_len > (int64_t)DQT_KV_PAGE * b->table_stride) return DQT_ERR_SHAPE;
  if (b->q_start == nullptr && b->q_tokens != b->n_seq) return DQT_ERR_SHAPE;
  if (b->q_tokens > 0 && b->n_seq == 0) return DQT_ERR_SHAPE;
  if (b->n_seq > 0 && (b->kv_len == nullptr || (b->max_len > 0 && b->table == nullptr))) return DQT_ERR_NULL;
  if (!aligned4(b->table) || !aligned4(b->kv_len) || !aligned4(b->q_start)) return DQT_ERR_ALIGN;
  if (!(b->scale >= 0x1p-20f && b->scale <= 0x1p20f) || (b->causal != 0 && b->causal != 1) || b->reserved != 0) return DQT_ERR_RANGE;
  *a = dqt::KvArgs{};
  a->K = static_cast<uint8_t*>(c->K);
  a->V = static_cast<uint8_t*>(c->V);
  a->scales = c->scales;
  a->pages = c->pages;
  a->table = b->table;
  a->kv_len = b->kv_len;
  a->q_start = b->q_start;
  a->tq = (int)b->q_tokens;
  a->n_seq = b->n_seq;
  a->table_stride = b->table_stride;
  a->max_len = (int)b->max_len;
  a->heads = b->heads;
  a->kv_heads = c->kv_heads;
  a->group = b->heads / c->kv_heads;
  a->d = c->d;
  // the pages that tokens are written to, and the tiles of 16 rows, at most
  const int64_t pages = a->tq / dqt::kPage + 2 * (int64_t)a->n_seq, tiles = (int64_t)a->tq * a->group / 16 + a->n_seq;
  if (4 * pages * a->kv_heads >= kMaxBlocks || tiles * a->kv_heads >= kMaxBlocks) return DQT_ERR_SHAPE;
  return DQT_OK;
}

dqt_status attn_args(const dqt_kv_cache* c, const dqt_kv_batch* b, dqt::KvAttnArgs* a) {
  *a = dqt::KvAttnArgs{};
  const dqt_status st = check_batch(c, b, &a->c);
  if (st != DQT_OK) return st;
  group_division(a->c.group, &a->gmul, &a->gone, &a->gshift);
  a->scale = b->scale;
  a->causal = b->causal;
  dqt::kv_attn_plan(c->fmt == DQT_FP8E4M3, a);
  return DQT_OK;
}

size_t attn_bytes(const dqt::KvAttnArgs& a) {
  return a.splits == 1 ? 0 : (size_t)a.splits * a.c.tq * a.c.heads * (a.c.d + 1) * 4;
}

bool pool_ok(const dqt_kv_pool* p) { return p->pages >= 0 && p->n_free >= 0 && p->n_free <= p->pages; }

int64_t pages_of(int64_t len) { return (len + DQT_KV_PAGE - 1) / DQT_KV_PAGE; }

// A row of the page table that holds len tokens in pages that are in use.
dqt_status check_row(const dqt_kv_pool* p, const int32_t* row, int32_t row_pages, int64_t len) {
  if (p == nullptr || p->refs == nullptr || p->free_pages == nullptr) return DQT_ERR_NULL;
  if (row == nullptr && row_pages > 0) return DQT_ERR_NULL;
  if (row_pages < 0 || len < 0 || len > (int64_t)DQT_KV_PAGE * row_pages) return DQT_ERR_SHAPE;
  if (!pool_ok(p)) return DQT_ERR_RANGE;
  for (int64_t i = 0; i < pages_of(len); ++i)
    if (row[i] < 0 || row[i] >= p->pages || p->refs[row[i]] < 1) return DQT_ERR_RANGE;
  return DQT_OK;
}

}  // namespace

extern "C" {

dqt_status dqt_rope_freqs(int32_t rot, double base, double factor, double context, double slow, double fast, uint64_t* freq) {
  if (freq == nullptr) return DQT_ERR_NULL;
  if (rot < 16 || rot > 1024 || rot % 16 != 0) return DQT_ERR_SHAPE;
  if (!(isfinite(base) && base > 1.0 && isfinite(factor) && factor >= 1.0 && isfinite(context) && context >= 0.0 &&
        isfinite(fast) && slow >= 0.0 && slow <= fast))
    return DQT_ERR_RANGE;
  const long double turn = 8.0L * atanl(1.0L);
  for (int32_t i = 0; i < rot / 2; ++i) {
    long double f = powl((long double)base, -2.0L * i / rot) / turn;
    if (factor != 1.0) {
      long double k = slow < fast ? ((long double)context * f - slow) / ((long double)fast - slow) : 0.0L;
      k = k < 0.0L ? 0.0L : k > 1.0L ? 1.0L : k;
      f *= k + (1.0L - k) / (long double)factor;
    }
    freq[i] = (uint64_t)rintl(ldexpl(f, 64));
  }
  return DQT_OK;
}

dqt_status dqt_rope_fwd(const dqt_rope* r, int32_t n, const dqt_rope_io* io, int32_t x_t, int64_t tokens, const int32_t* pos,
                        void* stream) {
  return rope(r, n, io, x_t, tokens, pos, stream, 0);
}

dqt_status dqt_rope_bwd(const dqt_rope* r, int32_t n, const dqt_rope_io* io, int32_t x_t, int64_t tokens, const int32_t* pos,
                        void* stream) {
  return rope(r, n, io, x_t, tokens, pos, stream, 1);
}

dqt_status dqt_kv_append(const dqt_kv_cache* c, const dqt_kv_batch* b, const dqt_rows* K, const dqt_rows* V,
                         const dqt_rope* r, const dqt_rows* Q, const dqt_rows* Qr, void* stream) {
  dqt::KvAppendArgs a{};
  dqt_status st = check_batch(c, b, &a.c);
  if (st != DQT_OK) return st;
  if ((st = check_rows(K, a.c.tq, a.c.kv_heads, a.c.d, false)) != DQT_OK) return st;
  if ((st = check_rows(V, a.c.tq, a.c.kv_heads, a.c.d, false)) != DQT_OK) return st;
  if (r != nullptr) {
    if ((st = check_rope(r)) != DQT_OK) return st;
    if (r->d != a.c.d) return DQT_ERR_SHAPE;
  }
  if ((Q == nullptr) != (Qr == nullptr) || (Q != nullptr && r == nullptr)) return DQT_ERR_NULL;
  if (Q != nullptr) {
    if ((st = check_rows(Q, a.c.tq, a.c.heads, a.c.d, false)) != DQT_OK) return st;
    if ((st = check_rows(Qr, a.c.tq, a.c.heads, a.c.d, true)) != DQT_OK) return st;
    if (Q->p == Qr->p && ((a.c.tq > 1 && Q->token != Qr->token) || (a.c.heads > 1 && Q->head != Qr->head))) return DQT_ERR_SHAPE;
    a.q = static_cast<const uint8_t*>(Q->p); a.q_tok = Q->token * 2; a.q_head = Q->head * 2;
    a.qr = static_cast<uint8_t*>(Qr->p); a.qr_tok = Qr->token * 2; a.qr_head = Qr->head * 2;
  }
  if (a.c.tq == 0) return DQT_OK;
  a.k = static_cast<const uint8_t*>(K->p); a.k_tok = K->token * 2; a.k_head = K->head * 2;
  a.v = static_cast<const uint8_t*>(V->p); a.v_tok = V->token * 2; a.v_head = V->head * 2;
  if (r != nullptr) {
    a.freq = r->freq;
    a.amp = r->amp;
    a.rot = r->rot;
    a.pairs = r->pairs;
  }
  return from_hip(dqt::launch_kv_append(c->fmt == DQT_FP8E4M3, a, static_cast<hipStream_t>(stream)));
}

size_t dqt_kv_attn_workspace(const dqt_kv_cache* c, const dqt_kv_batch* b) {
  dqt::KvAttnArgs a;
  if (attn_args(c, b, &a) != DQT_OK || a.c.tq == 0) return 0;
  return attn_bytes(a);
}

dqt_status dqt_kv_attn(const dqt_kv_cache* c, const dqt_kv_batch* b, const dqt_rows* Q, const dqt_rows* O, float* lse,
                       void* ws, size_t ws_bytes, void* stream) {
  dqt::KvAttnArgs a;
  dqt_status st = attn_args(c, b, &a);
  if (st != DQT_OK) return st;
  if ((st = check_rows(Q, a.c.tq, a.c.heads, a.c.d, false)) != DQT_OK) return st;
  if ((st = check_rows(O, a.c.tq, a.c.heads, a.c.d, true)) != DQT_OK) return st;
  if (!aligned4(lse) || !aligned16(ws)) return DQT_ERR_ALIGN;
  if (a.c.tq == 0) return DQT_OK;
  const size_t need = attn_bytes(a);
  if (need > 0 && (ws == nullptr || ws_bytes < need)) return DQT_ERR_WORKSPACE;
  a.Q = static_cast<const uint8_t*>(Q->p); a.q_tok = Q->token * 2; a.q_head = Q->head * 2;
  a.O = static_cast<uint8_t*>(O->p); a.o_tok = O->token * 2; a.o_head = O->head * 2;
  a.lse = lse;
  a.part = static_cast<float*>(ws);
  a.part_lse = a.part + (need == 0 ? 0 : (size_t)a.splits * a.c.tq * a.c.heads * a.c.d);
  return from_hip(dqt::launch_kv_attn(c->fmt == DQT_FP8E4M3, a, static_cast<hipStream_t>(stream)));
}

dqt_status dqt_kv_copy(int32_t n_caches, const dqt_kv_cache* c, int32_t n, const int32_t* src, const int32_t* dst, void* stream) {
  if (n_caches < 0 || n < 0) return DQT_ERR_SHAPE;
  if ((n_caches > 0 && c == nullptr) || (n > 0 && (src == nullptr || dst == nullptr))) return DQT_ERR_NULL;
  for (int32_t i = 0; i < n_caches; ++i) {
    const dqt_status st = check_cache(&c[i]);
    if (st != DQT_OK) return st;
    if (c[i].pages != c[0].pages || c[i].kv_heads != c[0].kv_heads || c[i].d != c[0].d || c[i].fmt != c[0].fmt) return DQT_ERR_SHAPE;
  }
  if (n_caches == 0 || n == 0) return DQT_OK;
  // a bit for each page that is written
  constexpr int64_t kLocal = 1 << 16;
  uint8_t local[kLocal / 8], *bits = local;
  const int64_t pages = c[0].pages;
  if (pages > kLocal) {
    bits = static_cast<uint8_t*>(malloc((size_t)((pages + 7) / 8)));
    if (bits == nullptr) return DQT_ERR_UNSUPPORTED;
  }
  memset(bits, 0, (size_t)((pages + 7) / 8));
  dqt_status st = DQT_OK;
  for (int32_t i = 0; i < n && st == DQT_OK; ++i) {
    if (src[i] < 0 || src[i] >= pages || dst[i] < 0 || dst[i] >= pages) st = DQT_ERR_RANGE;
    else if (bits[dst[i] >> 3] & (1 << (dst[i] & 7))) st = DQT_ERR_RANGE;
    else bits[dst[i] >> 3] |= (uint8_t)(1 << (dst[i] & 7));
  }
  for (int32_t i = 0; i < n && st == DQT_OK; ++i)
    if (bits[src[i] >> 3] & (1 << (src[i] & 7))) st = DQT_ERR_RANGE;
  if (bits != local) free(bits);
  if (st != DQT_OK) return st;
  dqt::LaunchStatus ls;
  dqt::KvCopyArgs a{};
  a.kv_heads = c[0].kv_heads;
  a.page_bytes = (int64_t)c[0].kv_heads * DQT_KV_PAGE * c[0].d;
  for (int32_t c0 = 0; c0 < n_caches; c0 += dqt::kCopyCaches) {
    const int nc = n_caches - c0 < dqt::kCopyCaches ? n_caches - c0 : dqt::kCopyCaches;
    for (int i = 0; i < nc; ++i) a.c[i] = {static_cast<uint8_t*>(c[c0 + i].K), static_cast<uint8_t*>(c[c0 + i].V), c[c0 + i].scales};
    for (int32_t p0 = 0; p0 < n; p0 += dqt::kCopyPages) {
      const int np = n - p0 < dqt::kCopyPages ? n - p0 : dqt::kCopyPages;
      for (int i = 0; i < np; ++i) a.p[i] = {src[p0 + i], dst[p0 + i]};
      ls << dqt::launch_kv_copy(a, nc, np, static_cast<hipStream_t>(stream));
    }
  }
  return from_hip(ls.e);
}

dqt_status dqt_kv_pool_init(dqt_kv_pool* p, int32_t pages, int32_t* refs, int32_t* free_pages) {
  if (p == nullptr) return DQT_ERR_NULL;
  if (pages < 0) return DQT_ERR_SHAPE;
  if (pages > 0 && (refs == nullptr || free_pages == nullptr)) return DQT_ERR_NULL;
  *p = dqt_kv_pool{refs, free_pages, pages, pages};
  for (int32_t i = 0; i < pages; ++i) {
    refs[i] = 0;
    free_pages[i] = pages - 1 - i;
  }
  return DQT_OK;
}

dqt_status dqt_kv_pool_extend(dqt_kv_pool* p, int32_t* row, int32_t row_pages, int64_t len, int64_t new_len, int32_t* src,
                              int32_t* dst) {
  if (src == nullptr || dst == nullptr) return DQT_ERR_NULL;
  const dqt_status st = check_row(p, row, row_pages, len);
  if (st != DQT_OK) return st;
  if (new_len < len || new_len > (int64_t)DQT_KV_PAGE * row_pages) return DQT_ERR_SHAPE;
  const int64_t have = pages_of(len), need = pages_of(new_len);
  const bool split = new_len > len && len % DQT_KV_PAGE != 0 && p->refs[row[have - 1]] > 1;
  const int64_t take = need - have + (split ? 1 : 0);
  if (take > p->n_free) return DQT_ERR_WORKSPACE;
  for (int64_t i = 0; i < take; ++i) {
    const int32_t x = p->free_pages[p->n_free - 1 - i];
    if (x < 0 || x >= p->pages || p->refs[x] != 0) return DQT_ERR_RANGE;
  }
  *src = *dst = -1;
  if (split) {
    *src = row[have - 1];
    --p->refs[*src];
    *dst = row[have - 1] = p->free_pages[--p->n_free];
    p->refs[*dst] = 1;
  }
  for (int64_t i = have; i < need; ++i) {
    row[i] = p->free_pages[--p->n_free];
    p->refs[row[i]] = 1;
  }
  return DQT_OK;
}

dqt_status dqt_kv_pool_fork(dqt_kv_pool* p, const int32_t* row, int32_t row_pages, int64_t len, int32_t* to) {
  const dqt_status st = check_row(p, row, row_pages, len);
  if (st != DQT_OK) return st;
  if (to == nullptr && row_pages > 0) return DQT_ERR_NULL;
  if (to == row && row_pages > 0) return DQT_ERR_RANGE;
  for (int64_t i = 0; i < row_pages; ++i) {
    to[i] = i < pages_of(len) ? row[i] : -1;
    if (to[i] >= 0) ++p->refs[to[i]];
  }
  return DQT_OK;
}

dqt_status dqt_kv_pool_trim(dqt_kv_pool* p, int32_t* row, int32_t row_pages, int64_t len, int64_t new_len) {
  const dqt_status st = check_row(p, row, row_pages, len);
  if (st != DQT_OK) return st;
  if (new_len < 0 || new_len > len) return DQT_ERR_SHAPE;
  const int64_t have = pages_of(len), keep = pages_of(new_len);
  for (int64_t i = keep; i < have; ++i)
    if (--p->refs[row[i]] < 0) {                     // the row holds a page more often than it has holders
      for (; i >= keep; --i) ++p->refs[row[i]];
      return DQT_ERR_RANGE;
    }
  for (int64_t i = have; i-- > keep;)                // (the first of them is the first to be taken again)
    if (p->refs[row[i]] == 0 && p->n_free < p->pages) {
      p->free_pages[p->n_free++] = row[i];
      p->refs[row[i]] = -1;                          // (once, should the row hold it twice)
    }
  for (int64_t i = keep; i < have; ++i) {
    if (p->refs[row[i]] < 0) p->refs[row[i]] = 0;
    row[i] = -1;
  }
  return DQT_OK;
}

dqt_status dqt_kv_pool_compact(dqt_kv_pool* p, int32_t* table, int32_t n_seq, int32_t row_pages, int32_t* src, int32_t* dst,
                               int32_t* n) {
  if (p == nullptr || n == nullptr) return DQT_ERR_NULL;
  if (n_seq < 0 || row_pages < 0) return DQT_ERR_SHAPE;
  if (!pool_ok(p)) return DQT_ERR_RANGE;
  const int64_t entries = (int64_t)n_seq * row_pages;
  if ((entries > 0 && table == nullptr) || (p->pages > 0 && (p->refs == nullptr || p->free_pages == nullptr || src == nullptr || dst == nullptr)))
    return DQT_ERR_NULL;
  const int32_t used = p->pages - p->n_free;
  for (int32_t i = 0; i < p->pages; ++i) dst[i] = 0;
  for (int64_t i = 0; i < entries; ++i)
    if (table[i] >= p->pages) return DQT_ERR_RANGE;
    else if (table[i] >= 0) ++dst[table[i]];
  int32_t held = 0;
  for (int32_t i = 0; i < p->pages; ++i) {
    if (dst[i] != p->refs[i]) return DQT_ERR_RANGE;
    held += p->refs[i] > 0;
  }
  if (held != used) return DQT_ERR_RANGE;
  int32_t moves = 0, to = 0;
  for (int32_t i = used; i < p->pages; ++i) {
    if (p->refs[i] == 0) continue;
    while (p->refs[to] != 0) ++to;                   // (below `used` as many are free as there are moves)
    src[moves] = i;
    dst[moves++] = to++;
  }
  for (int64_t i = 0; i < entries; ++i) {
    if (table[i] < used) continue;
    int32_t lo = 0, hi = moves;                      // src ascends
    while (hi - lo > 1) {
      const int32_t mid = lo + (hi - lo) / 2;
      if (src[mid] <= table[i]) lo = mid;
      else hi = mid;
    }
    table[i] = dst[lo];
  }
  for (int32_t i = 0; i < moves; ++i) {
    p->refs[dst[i]] = p->refs[src[i]];
    p->refs[src[i]] = 0;
  }
  for (int32_t i = 0; i < p->n_free; ++i) p->free_pages[i] = p->pages - 1 - i;
  *n = moves;
  return DQT_OK;
}

}  // extern "C"
