// Entry points of trees of drafted tokens: validation and launch set-up.
#include <algorithm>
#include <cstdarg>
#include <cstdio>

#include "rq_internal.h"
#include "rq_tree.h"

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

rq_status check_nodes(int32_t batch, int32_t n_nodes) {
  if (batch < 1 || batch > 65535) return fail(RQ_EINVAL, "batch %d outside 1..65535", batch);
  if (n_nodes < 1 || n_nodes > RQ_MAX_NODES)
    return fail(RQ_EINVAL, "n_nodes %d outside 1..%d", n_nodes, RQ_MAX_NODES);
  return RQ_OK;
}

rq_status check_draft(const rq_tree_draft* d) {
  if (!d) return fail(RQ_EINVAL, "draft is NULL");
  rq_status st = check_nodes(d->batch, d->n_nodes);
  if (st != RQ_OK) return st;
  if (d->vocab < 1 || d->vocab > (1 << 24))
    return fail(RQ_EINVAL, "vocab %d outside 1..2^24", d->vocab);
  return RQ_OK;
}

// A row's parts, a workgroup each: as many steps of the kernel, at most kVerifyParts,
// and no more than leave every sequence's workgroups room on the chip together.
struct VerifyPlan {
  int part, parts;
  uint64_t slots, done;            // bytes
  uint64_t bytes() const { return slots + done; }
};

VerifyPlan plan_verify(const rq_tree_draft* d) {
  VerifyPlan p{};
  const int steps = (d->vocab + rq::kVerifyStep - 1) / rq::kVerifyStep;
  const int most = std::max(std::min({steps, rq::kVerifyParts, rq::device_cus() / d->batch}), 1);
  p.part = ((d->vocab + most - 1) / most + 15) / 16 * 16;
  p.parts = (d->vocab + p.part - 1) / p.part;
  const uint64_t b = d->batch;
  p.slots = b * rq::kVerifySums * p.parts * sizeof(uint64_t);
  p.done = b * sizeof(uint32_t);
  return p;
}

}  // namespace

extern "C" {

rq_status rq_tree_mask(int32_t batch, int32_t n_nodes, const int32_t* parents,
                       const int32_t* new_len, uint32_t* mask, int32_t* depth, rq_stream stream) {
  rq_status st = check_nodes(batch, n_nodes);
  if (st != RQ_OK) return st;
  if (!parents || !mask) return fail(RQ_EINVAL, "NULL device pointer");
  rq::TreeMaskLaunch a{parents, new_len, mask, depth, batch, n_nodes, (n_nodes + 31) / 32};
  const uint64_t nodes = (uint64_t)batch * n_nodes * 4;
  const struct {
    const void* p;
    uint64_t bytes;
  } arrays[] = {{mask, nodes * a.words}, {depth, nodes}, {parents, nodes}, {new_len, batch * 4ull}};
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < i && j < 2; ++j)       // (the first two are written)
      if (rq::overlap(arrays[i].p, arrays[i].bytes, arrays[j].p, arrays[j].bytes))
        return fail(RQ_EINVAL, "two of the arrays overlap");
  return launched(rq::launch_tree_mask(a, reinterpret_cast<hipStream_t>(stream)), "tree layout launch");
}

rq_status rq_tree_verify_workspace(const rq_tree_draft* d, uint64_t* bytes) {
  rq_status st = check_draft(d);
  if (st != RQ_OK) return st;
  if (!bytes) return fail(RQ_EINVAL, "bytes is NULL");
  *bytes = plan_verify(d).bytes();
  return ok();
}

rq_status rq_tree_verify(const rq_tree_draft* d, void* ws, uint64_t ws_bytes, rq_stream stream) {
  rq_status st = check_draft(d);
  if (st != RQ_OK) return st;
  if (d->dtype != RQ_F32 && d->dtype != RQ_F16 && d->dtype != RQ_BF16)
    return fail(RQ_EINVAL, "unknown dtype %d", d->dtype);
  if (d->n_path < 1 || d->n_path > d->n_nodes)
    return fail(RQ_EINVAL, "n_path %d outside 1..%d", d->n_path, d->n_nodes);
  if (!d->tokens || !d->parents || !d->target || !d->uniforms || !d->path || !d->count || !d->next)
    return fail(RQ_EINVAL, "NULL device pointer");
  const uint64_t b = d->batch, nodes = b * d->n_nodes * 4;
  const struct {
    const void* p;
    uint64_t bytes;
  } arrays[] = {{d->path, b * d->n_path * 4}, {d->count, b * 4}, {d->next, b * 4}, {d->tokens, nodes},
                {d->parents, nodes}, {d->uniforms, nodes}, {d->new_len, b * 4}};
  for (int i = 0; i < 7; ++i)
    for (int j = 0; j < i && j < 3; ++j)       // (the first three are written)
      if (rq::overlap(arrays[i].p, arrays[i].bytes, arrays[j].p, arrays[j].bytes))
        return fail(RQ_EINVAL, "two of the arrays overlap");
  const VerifyPlan p = plan_verify(d);
  if (ws_bytes < p.bytes())
    return fail(RQ_ESMALLWS, "workspace %llu bytes < %llu needed", (unsigned long long)ws_bytes,
                (unsigned long long)p.bytes());
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 16)
    return fail(RQ_EINVAL, "the workspace is NULL or not 16-byte aligned");
  rq::TreeVerifyLaunch a{};
  a.tokens = d->tokens;
  a.parents = d->parents;
  a.new_len = d->new_len;
  a.target = d->target;
  a.draft = d->draft;
  a.t_sb = d->target_stride_batch;
  a.t_sn = d->target_stride_node;
  a.d_sb = d->draft_stride_batch;
  a.d_sn = d->draft_stride_node;
  a.uniforms = d->uniforms;
  a.B = d->batch;
  a.n = d->n_nodes;
  a.vocab = d->vocab;
  a.dtype = d->dtype;
  a.n_path = d->n_path;
  a.path = d->path;
  a.count = d->count;
  a.next = d->next;
  a.part = p.part;
  a.parts = p.parts;
  uint8_t* w = static_cast<uint8_t*>(ws);
  a.slots = reinterpret_cast<uint64_t*>(w);
  a.done = reinterpret_cast<uint32_t*>(w + p.slots);
  while (a.spread < 6 && (2 << a.spread) * d->n_nodes <= RQ_MAX_NODES) ++a.spread;
  return launched(rq::launch_tree_verify(a, reinterpret_cast<hipStream_t>(stream)), "verification launch");
}

}  // extern "C"
