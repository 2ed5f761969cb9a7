// Entry points of the block-scaled 8-bit cache: validation and launch set-up.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "rq_block.h"
#include "rq_internal.h"

namespace {

rq_status fail(rq_status code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return rq::set_error(code, buf);
}

rq_status ok() { return rq::set_error(RQ_OK, ""); }

rq_status launched(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(RQ_EDEVICE, "%s: %s", what, hipGetErrorString(e));
  return ok();
}

bool unaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 != 0; }

rq_status check_shape(const rq_block_cache* c) {
  if (!c) return fail(RQ_EINVAL, "cache descriptor is NULL");
  if (c->format != RQ_INT8 && c->format != RQ_E4M3)
    return fail(RQ_EINVAL, "unknown code format %d", c->format);
  if (c->dtype != RQ_F16 && c->dtype != RQ_BF16)
    return fail(RQ_EINVAL, "unknown dtype %d", c->dtype);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(RQ_EUNSUPPORTED, "head_dim %d (64 and 128 are supported)", c->head_dim);
  if (c->n_layers < 1 || c->batch < 1)
    return fail(RQ_EINVAL, "n_layers and batch must be >= 1");
  if (c->n_kv_heads < 1 || c->n_kv_heads > RQ_MAX_KV_HEADS)
    return fail(RQ_EINVAL, "n_kv_heads %d outside 1..%d", c->n_kv_heads, RQ_MAX_KV_HEADS);
  if ((int64_t)c->batch * c->n_kv_heads > 32767)
    return fail(RQ_EUNSUPPORTED, "batch * n_kv_heads = %lld exceeds 32767",
                (long long)c->batch * c->n_kv_heads);
  if (c->n_q_heads < c->n_kv_heads || c->n_q_heads % c->n_kv_heads)
    return fail(RQ_EINVAL, "n_q_heads %d is not a multiple of n_kv_heads %d", c->n_q_heads,
                c->n_kv_heads);
  if (c->n_q_heads / c->n_kv_heads > 16)
    return fail(RQ_EUNSUPPORTED, "more than 16 query heads per kv-head");
  if (c->capacity < rq::kBlockTokens || c->capacity % rq::kBlockTokens ||
      c->capacity > (1 << 24))
    return fail(RQ_EINVAL, "capacity %d must be a positive multiple of 32, at most 2^24",
                c->capacity);
  const double codes = 2.0 * c->n_layers * c->batch * c->n_kv_heads * c->capacity * c->head_dim;
  if (codes > 9.0e18) return fail(RQ_EINVAL, "cache too large");
  return RQ_OK;
}

rq_status check_buffers(const rq_block_cache* c, int32_t layer) {
  rq_status st = check_shape(c);
  if (st != RQ_OK) return st;
  if (layer < 0 || layer >= c->n_layers) return fail(RQ_EINVAL, "layer %d out of range", layer);
  if (!c->codes || !c->scales || !c->tail || !c->positions)
    return fail(RQ_EINVAL, "the cache has a NULL buffer");
  if (unaligned(c->codes) || unaligned(c->scales) || unaligned(c->tail) ||
      unaligned(c->positions) || unaligned(c->weights) ||
      reinterpret_cast<uintptr_t>(c->counters) % 4)
    return fail(RQ_EINVAL, "a cache buffer is not 16-byte aligned");
  return RQ_OK;
}

// Two arrays of n int32 (none overlaps NULL).
bool overlap(const int32_t* a, const int32_t* b, int32_t n) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && (x > y ? x - y : y - x) < n * sizeof(int32_t);
}

uint64_t units(const rq_block_cache* c) { return (uint64_t)c->batch * c->n_kv_heads; }

rq::BlockLayer layer_of(const rq_block_cache* c, int32_t layer) {
  const uint64_t u = units(c) * layer, cap = c->capacity, D = c->head_dim;
  rq::BlockLayer l{};
  l.codes = static_cast<uint8_t*>(c->codes) + u * 2 * cap * D;
  l.scales = c->scales + u * 2 * (cap / rq::kBlockTokens);
  l.tail = static_cast<uint16_t*>(c->tail) + u * 2 * rq::kBlockTokens * D;
  l.positions = c->positions + u * cap;
  l.weights = c->weights ? c->weights + u * cap : nullptr;
  l.counters = c->counters ? c->counters + u : nullptr;
  l.B = c->batch;
  l.H = c->n_kv_heads;
  l.by_H = rq::divider(c->n_kv_heads);
  l.cap = c->capacity;
  l.D = c->head_dim;
  l.fmt = c->format;
  l.is_bf16 = c->dtype == RQ_BF16;
  return l;
}

rq::BlockRows rows_of(const rq_block_rows* r) {
  return rq::BlockRows{r->data, r->stride_batch, r->stride_head, r->stride_token};
}

rq_status check_query(const rq_block_cache* c, const rq_block_query* a) {
  if (!a) return fail(RQ_EINVAL, "query is NULL");
  if (a->n_new < 1 || a->n_new > c->capacity)
    return fail(RQ_EINVAL, "n_new %d outside 1..%d", a->n_new, c->capacity);
  if (a->max_tokens < a->n_new || a->max_tokens > c->capacity)
    return fail(RQ_EINVAL, "max_tokens %d outside %d..%d", a->max_tokens, a->n_new, c->capacity);
  if (a->window < 0) return fail(RQ_EINVAL, "window %d must be >= 0", a->window);
  return RQ_OK;
}

// How an attention call is split, and what it needs of the workspace.
struct Plan {
  int prompt;                      // tiles of 128 rows (rq_block_prompt.hip)
  int row_tiles, splits, row_parts;
  uint64_t part, part_ml, stats, scores, queries, factors, sums;   // bytes
  uint64_t bytes() const { return part + part_ml + stats + scores + queries + factors + sums; }
};

// Up to 32 rows: one workgroup a CU over the units, at least four blocks
// (one a wave) each.  Four waves with a block in flight each keep a CU's share
// of the memory busy; more workgroups are set-ups and parts to merge, but even
// out sequences of unlike lengths where the scores are kept too.  us with one /
// two / three a CU: 128 full units of 8192 tokens 44.7 / 47 / 47, 32 of 32768 (8
// heads, capped) 43.7 / 48.5 / 50, 8 of 131072 46.8 / 48 / 49.4, 64 of 4000 15.6 /
// 17 / 18, 192 of 4000 31.3 / 39 / 36.5; uneven lengths: 128 units to 8192 35 /
// 33.8 / 34, with weights 42.5 / 37.8 / 39.  Two tiles of rows are more work a
// block, and units that leave a workgroup alone with a long one wait for it: 104
// units of 24 rows to 9029 even 60.1 / 54.5 / 57.7, uneven 54.2 / 39.3 / 39.3, but
// 64 units of 32 rows to 8192 31.2 / 33.1 / 40, 8 of 65536 30.5 / 34.5 / 39.
// More than two tiles of 16 rows: tiles of 128 rows, two workgroups a CU, at
// least four blocks each.  Where the new tokens are few beside the cached ones,
// sequences may differ in length and a round's workgroups with them: one split
// more (4 sequences, 8 kv-heads of 4 heads, 512 tokens over 8192: 426 us
// unsplit, 440 in two; lengths from 2048 to 8192: 322 and 254).  Up to eight blocks
// a split saves less than its merging launch takes (256 tiles of 143 tokens 15.3
// us, in two splits 24.6).
Plan plan_attention(const rq_block_cache* c, const rq_block_query* a) {
  Plan p{};
  const int64_t G = c->n_q_heads / c->n_kv_heads, u = (int64_t)units(c);
  p.row_tiles = (int)((a->n_new * G + 15) / 16);
  p.prompt = p.row_tiles > 2;
  int64_t blocks = (a->max_tokens + rq::kBlockTokens - 1) / rq::kBlockTokens;
  if (a->window) {
    const int64_t seen = ((int64_t)a->window + (p.prompt ? 128 / G + 1 : a->n_new)) / rq::kBlockTokens + 2;
    blocks = seen < blocks ? seen : blocks;
  }
  int64_t s;
  if (p.prompt) {
    s = 2 * (int64_t)rq::device_cus() / (u * ((a->n_new * G + 127) / 128));
    s = blocks > 8 ? std::min(s, (blocks + 3) / 4) : 1;
    if (s <= 1 && a->max_tokens >= 4 * (int64_t)a->n_new && blocks >= 128) s = 2;
  } else {
    const bool two = (a->accumulate && c->batch > 1) || (p.row_tiles > 1 && u > 64);
    s = (two ? 2 : 1) * (int64_t)rq::device_cus() / u;
    s = std::min(s, (blocks + 3) / 4);
  }
  p.splits = (int)std::max<int64_t>(s, 1);
  const uint64_t tiles = (uint64_t)u * p.row_tiles;
  if (p.splits > 1) {
    p.part = tiles * p.splits * 16 * c->head_dim * sizeof(float);
    p.part_ml = tiles * p.splits * 16 * 2 * sizeof(float);
  }
  if (a->accumulate) {
    p.stats = tiles * 16 * 2 * sizeof(float);
    // one or two tiles of rows: the scores are kept (4 bytes a row and token, out
    // and back) rather than computed again from the keys, which takes a prompt's
    // kernels.  us so / with those, 4, 8, 16 and 32 rows: 16 sequences to 8192
    // tokens 38, 42, 49, 70 / 128 to 131, to 1000 14, 15, 17, 24 / 30 to 32, two to
    // 8192 15, 16, 18, 27 / 30 to 33.
    const int64_t rows = a->n_new * G;
    if (!p.prompt) {
      p.scores = (uint64_t)u * ((a->max_tokens + rq::kBlockTokens - 1) / rq::kBlockTokens) * rows *
                 rq::kBlockTokens * sizeof(float);
      return p;
    }
    // else workgroups of 256 tokens, and parts of the rows to fill two rounds (two
    // a CU; windows leave some without rows: four), about 128 rows or more in
    // each.  us a call with four / two rounds: 32 units of 2000 tokens, 1000 rows
    // 125 / 118, 8 of 32000 and 400 rows 169 / 159, 2 of 8000 and 400 rows 42 / 41;
    // 32 of 8192 and 2036 rows, window of 2000: 324 / 428.
    // (A window needs no more workspace than none: the size counts its parts.)
    const int64_t round = 2 * (int64_t)rq::device_cus(), wgs = u * ((a->max_tokens + 255) / 256);
    const int64_t most = std::max<int64_t>(std::min(4 * round / wgs, (rows + 63) / 128), 1);
    p.row_parts = (int)(a->window ? most : std::max<int64_t>(std::min(2 * round / wgs, most), 1));
    p.queries = tiles * 16 * c->head_dim * sizeof(uint16_t);
    p.factors = tiles * 16 * sizeof(float);
    if (most > 1) p.sums = (uint64_t)most * u * a->max_tokens * sizeof(float);
  }
  return p;
}

// Calls of many rows form cap tanh(x) as cap - 2 cap / (1 + e^(2x)), which errs by
// 2^-22 of the cap (a probability by 2^-16 at this one), where the cap is small
// and the output has 16 bits; else by tanh_f, relative to the score, however
// large the cap is.  (Two prompts of 4096 tokens: 466 us so, 626 by tanh_f; 509
// tokens over 8192 with weights 455 and 709.)
constexpr float kSmallCap = 64.0f;

// How an eviction selects, and what it needs of the workspace (bytes).
struct EvictPlan {
  int part, parts;
  uint64_t slots, state, before, counts;
  uint64_t bytes() const { return slots + state + before + counts; }
};

EvictPlan plan_eviction(const rq_block_cache* src, int keep) {
  EvictPlan p{};
  const uint64_t u = units(src);
  p.slots = (u * keep * sizeof(int32_t) + 15) / 16 * 16;
  p.parts = 1;
  if (src->capacity <= rq::kSelectShort) return p;
  const int most = (src->capacity + rq::kSelectParts - 1) / rq::kSelectParts;
  p.part = (most + rq::kSelectPart - 1) / rq::kSelectPart * rq::kSelectPart;
  p.parts = (src->capacity + p.part - 1) / p.part;
  p.state = u * rq::kSelectState * sizeof(uint32_t);
  p.before = (u * p.parts * sizeof(uint32_t) + 15) / 16 * 16;
  p.counts = 3 * u * p.parts * 2048 * sizeof(uint32_t);
  return p;
}

}  // namespace

extern "C" {

rq_status rq_block_sizes(const rq_block_cache* c, uint64_t* codes_bytes, uint64_t* scales_bytes,
                         uint64_t* tail_bytes, uint64_t* positions_bytes,
                         uint64_t* weights_bytes, uint64_t* counters_bytes) {
  rq_status st = check_shape(c);
  if (st != RQ_OK) return st;
  const uint64_t u = units(c) * c->n_layers, cap = c->capacity, D = c->head_dim;
  if (codes_bytes) *codes_bytes = u * 2 * cap * D;
  if (scales_bytes) *scales_bytes = u * 2 * (cap / rq::kBlockTokens) * sizeof(float);
  if (tail_bytes) *tail_bytes = u * 2 * rq::kBlockTokens * D * sizeof(uint16_t);
  if (positions_bytes) *positions_bytes = u * cap * sizeof(int32_t);
  if (weights_bytes) *weights_bytes = u * cap * sizeof(float);
  if (counters_bytes) *counters_bytes = u * sizeof(uint32_t);
  return ok();
}

rq_status rq_block_append(const rq_block_cache* c, int32_t layer, const int32_t* past,
                          int32_t n_new, const int32_t* new_len, const rq_block_rows* k,
                          const rq_block_rows* v, rq_stream stream) {
  rq_status st = check_buffers(c, layer);
  if (st != RQ_OK) return st;
  if (n_new < 1 || n_new > c->capacity)
    return fail(RQ_EINVAL, "n_new %d outside 1..%d", n_new, c->capacity);
  if (!past || !k || !v || !k->data || !v->data) return fail(RQ_EINVAL, "NULL device pointer");
  rq::BlockAppendLaunch a{};
  a.c = layer_of(c, layer);
  a.past = past;
  a.new_len = new_len;
  a.k = rows_of(k);
  a.v = rows_of(v);
  a.n = n_new;
  return launched(rq::launch_block_append(a, reinterpret_cast<hipStream_t>(stream)),
                  "append launch");
}

rq_status rq_block_advance(const rq_block_cache* c, int32_t* lengths, int32_t n_new,
                           const int32_t* new_len, int32_t* past, int32_t* fitting,
                           int32_t* dropped, rq_stream stream) {
  rq_status st = check_shape(c);
  if (st != RQ_OK) return st;
  if (n_new < 1 || n_new > c->capacity)
    return fail(RQ_EINVAL, "n_new %d outside 1..%d", n_new, c->capacity);
  if (!lengths) return fail(RQ_EINVAL, "NULL device pointer");
  const int32_t* arrays[] = {lengths, new_len, past, fitting, dropped};
  for (int i = 0; i < 5; ++i)
    for (int j = 0; j < i; ++j)
      if (overlap(arrays[i], arrays[j], c->batch)) return fail(RQ_EINVAL, "two of the arrays overlap");
  const rq::BlockAdvanceLaunch a{lengths, new_len, past, fitting, dropped, c->batch, c->capacity, n_new};
  return launched(rq::launch_block_advance(a, reinterpret_cast<hipStream_t>(stream)),
                  "advance launch");
}

rq_status rq_block_attention_workspace(const rq_block_cache* c, const rq_block_query* a,
                                       uint64_t* bytes) {
  rq_status st = check_shape(c);
  if (st != RQ_OK) return st;
  st = check_query(c, a);
  if (st != RQ_OK) return st;
  if (!bytes) return fail(RQ_EINVAL, "bytes is NULL");
  *bytes = plan_attention(c, a).bytes();
  return ok();
}

rq_status rq_block_attention(const rq_block_cache* c, int32_t layer, const rq_block_query* q,
                             void* ws, uint64_t ws_bytes, rq_stream stream) {
  rq_status st = check_buffers(c, layer);
  if (st != RQ_OK) return st;
  st = check_query(c, q);
  if (st != RQ_OK) return st;
  if (!q->past || !q->q.data || !q->out.data) return fail(RQ_EINVAL, "NULL device pointer");
  if (q->out_dtype != RQ_F32 && q->out_dtype != RQ_F16 && q->out_dtype != RQ_BF16)
    return fail(RQ_EINVAL, "unknown output dtype %d", q->out_dtype);
  if (!std::isfinite(q->scale)) return fail(RQ_EINVAL, "scale is not finite");
  // (beyond, scores over the cap leave the normal numbers)
  if (!(q->cap >= 0.0f && q->cap <= 0x1p100f))
    return fail(RQ_EINVAL, "cap must be in 0..2^100 (0: none)");
  if (q->accumulate && !c->weights) return fail(RQ_EINVAL, "the cache keeps no weights");
  const float log2e = 1.4426950408889634f;
  const float qscale = q->cap > 0.0f ? q->scale / q->cap : q->scale * log2e;
  if (!std::isfinite(qscale))
    return fail(RQ_EINVAL, "scale %g and cap %g leave the fp32 range", q->scale, q->cap);
  const Plan p = plan_attention(c, q);
  if ((double)p.row_tiles * p.splits * units(c) > 2.0e9)
    return fail(RQ_EUNSUPPORTED, "more than 2e9 tiles of 16 query rows");
  if (ws_bytes < p.bytes())
    return fail(RQ_ESMALLWS, "workspace %llu bytes < %llu needed", (unsigned long long)ws_bytes,
                (unsigned long long)p.bytes());
  if (p.bytes() && (!ws || unaligned(ws)))
    return fail(RQ_EINVAL, "the workspace is NULL or not 16-byte aligned");
  rq::BlockAttendLaunch a{};
  a.c = layer_of(c, layer);
  a.past = q->past;
  a.new_len = q->new_len;
  a.q = rows_of(&q->q);
  a.out = rows_of(&q->out);
  a.out_dtype = q->out_dtype;
  a.G = c->n_q_heads / c->n_kv_heads;
  a.n = q->n_new;
  a.max_tokens = q->max_tokens;
  a.row_tiles = p.row_tiles;
  a.splits = p.splits;
  a.by_G = rq::divider(a.G);
  a.by_splits = rq::divider(p.splits);
  a.qscale = qscale;
  a.cap = q->cap * log2e;
  a.fine = q->cap > kSmallCap || (q->cap > 0.0f && q->out_dtype == RQ_F32);
  a.window = q->window;
  a.slopes = q->slopes;
  a.accumulate = q->accumulate != 0;
  uint8_t* w = static_cast<uint8_t*>(ws);
  auto take = [&w](uint64_t bytes) {
    uint8_t* p = bytes ? w : nullptr;
    w += bytes;
    return p;
  };
  a.part = reinterpret_cast<float*>(take(p.part));
  a.part_ml = reinterpret_cast<float*>(take(p.part_ml));
  a.stats = reinterpret_cast<float*>(take(p.stats));
  a.scores = reinterpret_cast<float*>(take(p.scores));
  a.queries = reinterpret_cast<uint16_t*>(take(p.queries));
  a.factors = reinterpret_cast<float*>(take(p.factors));
  a.sums = reinterpret_cast<float*>(take(p.sums));
  a.row_parts = p.row_parts;
  a.by_parts = rq::divider(std::max(p.row_parts, 1));
  // The last workgroup of a tile adds its splits where they are few: a launch
  // less, but one workgroup's loads.  us with / without, splits x rows: 8 x 4
  // 8.5 / 9.4, 8 x 8 44.2 / 45.4 (32 units of 32768 tokens), 2 x 4 15.4 / 16.5,
  // 32 x 4 10.8 / 9.3, 16 x 16 18.7 / 18.1, 32 x 8 15.0 / 12.5.
  a.tickets = !p.prompt && p.splits > 1 && p.splits <= rq::kTicketSplits &&
              p.splits * a.n * a.G <= 100 && a.c.counters && !a.accumulate;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  hipError_t e = p.prompt ? rq::launch_block_prompt(a, s) : rq::launch_block_attend(a, s);
  if (e == hipSuccess && p.prompt) e = rq::launch_block_merge(a, s);
  if (e == hipSuccess && a.accumulate && !a.scores) e = rq::launch_block_weigh(a, s);
  return launched(e, "attention launch");
}

rq_status rq_block_evict_workspace(const rq_block_cache* src, int32_t keep, uint64_t* bytes) {
  rq_status st = check_shape(src);
  if (st != RQ_OK) return st;
  if (keep < 1) return fail(RQ_EINVAL, "keep %d must be >= 1", keep);
  if (!bytes) return fail(RQ_EINVAL, "bytes is NULL");
  *bytes = plan_eviction(src, keep).bytes();
  return ok();
}

rq_status rq_block_evict(const rq_block_cache* src, const rq_block_cache* dst, int32_t layer,
                         const int32_t* lengths, int32_t keep, int32_t n_sink, int32_t n_recent,
                         int32_t* new_lengths, void* ws, uint64_t ws_bytes, rq_stream stream) {
  rq_status st = check_buffers(src, layer);
  if (st != RQ_OK) return st;
  st = check_buffers(dst, layer);
  if (st != RQ_OK) return st;
  if (src->format != dst->format || src->dtype != dst->dtype || src->n_layers != dst->n_layers ||
      src->batch != dst->batch || src->n_kv_heads != dst->n_kv_heads ||
      src->n_q_heads != dst->n_q_heads || src->head_dim != dst->head_dim)
    return fail(RQ_EINVAL, "the two caches differ in more than their capacity");
  if (src->codes == dst->codes || src->scales == dst->scales || src->tail == dst->tail ||
      src->positions == dst->positions || src->weights == dst->weights)
    return fail(RQ_EINVAL, "the two caches share a buffer, or the source keeps no weights");
  if (!src->weights) return fail(RQ_EINVAL, "the source keeps no weights");
  if (keep < 1 || keep > dst->capacity)
    return fail(RQ_EINVAL, "keep %d outside 1..%d", keep, dst->capacity);
  if (n_sink < 0 || n_recent < 1 || (int64_t)n_sink + n_recent > keep)
    return fail(RQ_EINVAL, "n_sink %d >= 0 and n_recent %d >= 1 must fit keep %d", n_sink,
                n_recent, keep);
  if (!lengths || !new_lengths) return fail(RQ_EINVAL, "NULL device pointer");
  const EvictPlan p = plan_eviction(src, keep);
  const uint64_t need = p.bytes();
  if (ws_bytes < need)
    return fail(RQ_ESMALLWS, "workspace %llu bytes < %llu needed", (unsigned long long)ws_bytes,
                (unsigned long long)need);
  if (!ws || unaligned(ws)) return fail(RQ_EINVAL, "the workspace is NULL or not 16-byte aligned");
  if (overlap(lengths, new_lengths, src->batch))
    return fail(RQ_EINVAL, "lengths and new_lengths overlap (the lengths are read to the end)");
  rq::BlockEvictLaunch a{};
  a.src = layer_of(src, layer);
  a.dst = layer_of(dst, layer);
  a.lengths = lengths;
  a.new_lengths = new_lengths;
  a.keep = keep;
  a.n_sink = n_sink;
  a.n_recent = n_recent;
  uint8_t* w = static_cast<uint8_t*>(ws);
  a.slots = reinterpret_cast<int32_t*>(w);
  a.part = p.part;
  a.parts = p.parts;
  a.state = reinterpret_cast<uint32_t*>(w + p.slots);
  a.before = reinterpret_cast<uint32_t*>(w + p.slots + p.state);
  a.counts = reinterpret_cast<uint32_t*>(w + p.slots + p.state + p.before);
  return launched(rq::launch_block_evict(a, reinterpret_cast<hipStream_t>(stream)),
                  "eviction launch");
}

}  // extern "C"
