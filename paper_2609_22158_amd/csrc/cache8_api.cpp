// C ABI of the 8-bit cache (include/stepkv_cache8.h): argument validation,
// launch planning and workspace layout.
#include "stepkv_cache8.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>

#include "cache8.h"

using namespace stepkv;

namespace {

constexpr size_t kAlign = 256;

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int hip_status(hipError_t e) { return e == hipSuccess ? STEPKV_OK : STEPKV_EHIP; }

bool offsets(const int32_t* cu, int n) {
  if (cu[0] != 0) return false;
  for (int i = 0; i < n; ++i)
    if (cu[i + 1] < cu[i]) return false;
  return true;
}

int check_cache(const stepkv_cache8* c) {
  if (!c) return STEPKV_EINVAL;
  if (c->num_layers < 1 || c->num_kv_heads < 1 || c->num_seqs < 1 || c->head_dim < 1)
    return STEPKV_EINVAL;
  if (!c->cu_rows_host || !c->cu_rows || !c->lens || !c->seen) return STEPKV_EINVAL;
  if (!offsets(c->cu_rows_host, c->num_seqs)) return STEPKV_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128) return STEPKV_EUNSUPPORTED;
  if (c->cu_rows_host[c->num_seqs] > STEPKV_CACHE8_MAX_ROWS) return STEPKV_EUNSUPPORTED;
  if (c->cu_rows_host[c->num_seqs] > 0) {  // NULL buffers hold 0 rows
    if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return STEPKV_EINVAL;
    if (!c->weights != !c->positions) return STEPKV_EINVAL;
  }
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scales, 4) ||
      !aligned(c->v_scales, 4) || !aligned(c->weights, 4) || !aligned(c->positions, 4))
    return STEPKV_EINVAL;
  const int64_t lh = (int64_t)c->num_layers * c->num_kv_heads;
  if (lh * c->num_seqs > std::numeric_limits<int32_t>::max()) return STEPKV_EUNSUPPORTED;
  return STEPKV_OK;
}

int check_heads(const stepkv_cache8* c, int32_t num_q_heads) {
  if (num_q_heads < 1 || num_q_heads % c->num_kv_heads != 0) return STEPKV_EINVAL;
  if ((int64_t)c->num_layers * c->num_seqs * num_q_heads > std::numeric_limits<int32_t>::max())
    return STEPKV_EUNSUPPORTED;
  return STEPKV_OK;
}

// Whether the cache holds weights and positions (one without rows need not).
bool gathers(const stepkv_cache8* c) {
  return (c->weights && c->positions) || c->cu_rows_host[c->num_seqs] == 0;
}

Cache8View view(const stepkv_cache8* c) {
  Cache8View w;
  w.k_codes = static_cast<uint8_t*>(c->k_codes);
  w.v_codes = static_cast<uint8_t*>(c->v_codes);
  w.k_scales = c->k_scales;
  w.v_scales = c->v_scales;
  w.weights = c->weights;
  w.positions = c->positions;
  w.cu_rows = c->cu_rows;
  w.lens = c->lens;
  w.seen = c->seen;
  w.status = c->status;
  w.L = c->num_layers;
  w.H = c->num_kv_heads;
  w.S = c->num_seqs;
  w.d = c->head_dim;
  w.rows = c->cu_rows_host[c->num_seqs];
  w.nblk = w.rows / kBlock8 + w.S;
  return w;
}

Attend8Args attend_args(const stepkv_cache8* c, int32_t num_q_heads, int32_t gather) {
  Attend8Args a{};
  a.c = view(c);
  a.gather = gather != 0 && a.c.rows > 0;
  a.Hq = num_q_heads;
  a.G = num_q_heads / c->num_kv_heads;
  plan_attend8(a, c->cu_rows_host);
  return a;
}

// The workspace of a decode step: the splits' states and, to gather, the logits.
size_t partial_bytes(const Attend8Args& a) {
  return align_up(sizeof(float) * attend8_partial_floats(a));
}
size_t logits_bytes(const Attend8Args& a) {
  return align_up(sizeof(float) * attend8_logits(a));
}
size_t decode_bytes(const Attend8Args& a) {
  return partial_bytes(a) + (a.gather ? logits_bytes(a) : 0);
}

Evict8Args evict_args(const stepkv_cache8* c, int32_t keep, const int32_t* keeps) {
  Evict8Args a{};
  a.c = view(c);
  a.keep = keep;
  a.keeps = keeps;
  plan_evict8(a, c->cu_rows_host);
  return a;
}
size_t heads_bytes(const Evict8Args& a) {
  return align_up(sizeof(Evict8Head) * (size_t)a.c.L * a.c.H * a.c.S);
}
size_t evict_bytes(const Evict8Args& a) {
  return heads_bytes(a) + align_up(sizeof(int2) * (size_t)a.c.L * a.c.H * (a.c.rows / 2));
}

}  // namespace

extern "C" {

int stepkv_cache8_compact(const stepkv_problem* pb, const stepkv_cache8* c, const void* k,
                          const void* v, const int32_t* idx, int32_t shared_idx,
                          const int32_t* cu_retained, const float* weights, void* stream) {
  const int rc = check_cache(c);
  if (rc != STEPKV_OK) return rc;
  if (!pb || pb->num_layers != c->num_layers || pb->num_kv_heads != c->num_kv_heads ||
      pb->head_dim != c->head_dim || pb->num_seqs != c->num_seqs || !pb->cu_seqlens_host ||
      !pb->cu_seqlens || !offsets(pb->cu_seqlens_host, pb->num_seqs))
    return STEPKV_EINVAL;
  if (!cu_retained || !aligned(k, 16) || !aligned(v, 16) || !aligned(weights, 4))
    return STEPKV_EINVAL;
  if (weights && !gathers(c)) return STEPKV_EINVAL;
  if (pb->cu_seqlens_host[pb->num_seqs] > 0 && (!k || !v || !idx))
    return STEPKV_EINVAL;  // NULL sources hold 0 tokens
  Write8Args a;
  a.c = view(c);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.nsrc = pb->cu_seqlens_host[pb->num_seqs];
  a.k_row = a.v_row = c->head_dim;
  a.k_head = a.v_head = (int64_t)a.nsrc * c->head_dim;
  a.k_layer = a.v_layer = a.k_head * c->num_kv_heads;
  a.cu_src = pb->cu_seqlens;
  a.cu_retained = cu_retained;
  a.idx = idx;
  a.gathered = weights;
  a.shared_idx = shared_idx != 0;
  int64_t nb = 0;  // R_s is at most the sequence's source tokens
  for (int s = 0; s < c->num_seqs; ++s) {
    const int32_t room = c->cu_rows_host[s + 1] - c->cu_rows_host[s];
    const int32_t n = pb->cu_seqlens_host[s + 1] - pb->cu_seqlens_host[s];
    nb += ((int64_t)std::min(room, n) + kBlock8 - 1) / kBlock8;
  }
  a.nblocks = (int)nb;
  if (!write8_fits(a)) return STEPKV_EUNSUPPORTED;
  return hip_status(launch_write8(a, static_cast<hipStream_t>(stream)));
}

int stepkv_cache8_advance(const stepkv_cache8* c, const int32_t* cu_new, void* stream) {
  const int rc = check_cache(c);
  if (rc != STEPKV_OK) return rc;
  if (!cu_new) return STEPKV_EINVAL;
  return hip_status(launch_advance8(view(c), cu_new, static_cast<hipStream_t>(stream)));
}

int stepkv_cache8_append(const stepkv_cache8* c, const void* k_new, const int64_t* k_strides,
                         const void* v_new, const int64_t* v_strides, const int32_t* cu_new,
                         int32_t num_new, void* stream) {
  const int rc = check_cache(c);
  if (rc != STEPKV_OK) return rc;
  if (!cu_new || num_new < 0) return STEPKV_EINVAL;
  if (num_new > 0 && (!k_new || !v_new)) return STEPKV_EINVAL;  // NULL tensors hold 0 tokens
  if (!k_strides || !v_strides || !aligned(k_new, 16) || !aligned(v_new, 16))
    return STEPKV_EINVAL;
  for (int i = 0; i < 3; ++i)
    if (k_strides[i] % 8 != 0 || v_strides[i] % 8 != 0) return STEPKV_EINVAL;
  if (num_new == 0) return STEPKV_OK;
  Write8Args a;
  a.c = view(c);
  a.k = static_cast<const uint16_t*>(k_new);
  a.v = static_cast<const uint16_t*>(v_new);
  a.k_layer = k_strides[0];
  a.k_row = k_strides[1];
  a.k_head = k_strides[2];
  a.v_layer = v_strides[0];
  a.v_row = v_strides[1];
  a.v_head = v_strides[2];
  a.cu_src = cu_new;
  a.cu_retained = nullptr;
  a.idx = nullptr;
  a.gathered = nullptr;
  a.nsrc = num_new;
  a.shared_idx = 0;
  // n rows in order touch at most floor((n - 1) / 64) + 2 blocks, and at most n
  a.nblocks = (int)std::min<int64_t>(num_new, (int64_t)num_new / kBlock8 + 2 * (int64_t)c->num_seqs);
  if (!write8_fits(a)) return STEPKV_EUNSUPPORTED;
  return hip_status(launch_write8(a, static_cast<hipStream_t>(stream)));
}

int stepkv_cache8_read(const stepkv_cache8* c, const int32_t* cu_out, int32_t out_rows,
                       void* k_out, void* v_out, void* stream) {
  const int rc = check_cache(c);
  if (rc != STEPKV_OK) return rc;
  if (!cu_out || out_rows < 0 || (out_rows > 0 && !k_out && !v_out)) return STEPKV_EINVAL;
  if (!aligned(k_out, 16) || !aligned(v_out, 16)) return STEPKV_EINVAL;
  if (out_rows == 0) return STEPKV_OK;
  Read8Args a;
  a.c = view(c);
  a.cu_out = cu_out;
  a.k_out = static_cast<uint16_t*>(k_out);
  a.v_out = static_cast<uint16_t*>(v_out);
  a.out_rows = out_rows;
  if (out_rows > STEPKV_CACHE8_MAX_ROWS || !read8_fits(a)) return STEPKV_EUNSUPPORTED;
  return hip_status(launch_read8(a, static_cast<hipStream_t>(stream)));
}

size_t stepkv_cache8_decode_workspace_bytes(const stepkv_cache8* c, int32_t num_q_heads,
                                            int32_t gather) {
  if (check_cache(c) != STEPKV_OK || check_heads(c, num_q_heads) != STEPKV_OK) return 0;
  return std::max(decode_bytes(attend_args(c, num_q_heads, gather)), kAlign);
}

int stepkv_cache8_decode(const stepkv_cache8* c, int32_t num_q_heads, const void* q_dec,
                         float scale, int32_t gather, float* out, float* lse, void* workspace,
                         size_t ws_bytes, void* stream) {
  int rc = check_cache(c);
  if (rc == STEPKV_OK) rc = check_heads(c, num_q_heads);
  if (rc != STEPKV_OK) return rc;
  if (!q_dec || !out || !std::isfinite(scale) || !aligned(q_dec, 16)) return STEPKV_EINVAL;
  // the kernel scales logits by scale * log2(e): 0 times an infinity is NaN
  if (scale > 0.0f && !std::isfinite(scale * 1.44269504088896341f)) return STEPKV_EINVAL;
  if (gather && !gathers(c)) return STEPKV_EINVAL;
  Attend8Args a = attend_args(c, num_q_heads, gather);
  if (!attend8_fits(a)) return STEPKV_EUNSUPPORTED;
  const size_t need = decode_bytes(a);
  if (need > 0 && (!workspace || !aligned(workspace, kAlign) || ws_bytes < need))
    return STEPKV_EWORKSPACE;
  uint8_t* const ws = static_cast<uint8_t*>(workspace);
  a.q = static_cast<const uint16_t*>(q_dec);
  a.out = out;
  a.lse = lse;
  a.partial = reinterpret_cast<float*>(ws);
  if (a.gather) a.logits = reinterpret_cast<float*>(ws + partial_bytes(a));
  a.scale = scale > 0.0f ? scale : (float)(1.0 / std::sqrt((double)c->head_dim));
  return hip_status(launch_attend8(a, static_cast<hipStream_t>(stream)));
}

size_t stepkv_cache8_evict_workspace_bytes(const stepkv_cache8* c) {
  if (check_cache(c) != STEPKV_OK) return 0;
  return evict_bytes(evict_args(c, 1, nullptr));
}

int stepkv_cache8_evict(const stepkv_cache8* c, int32_t keep, const int32_t* keeps, int32_t first,
                        int32_t recent, void* workspace, size_t ws_bytes, void* stream) {
  const int rc = check_cache(c);
  if (rc != STEPKV_OK) return rc;
  if (!gathers(c) || first < 0 || recent < 0 || (!keeps && keep < 1)) return STEPKV_EINVAL;
  Evict8Args a = evict_args(c, keep, keeps);
  if (!evict8_fits(a)) return STEPKV_EUNSUPPORTED;
  if (!workspace || !aligned(workspace, kAlign) || ws_bytes < evict_bytes(a))
    return STEPKV_EWORKSPACE;
  a.first = first;
  a.recent = recent;
  a.heads = static_cast<Evict8Head*>(workspace);
  a.moves = reinterpret_cast<int2*>(static_cast<uint8_t*>(workspace) + heads_bytes(a));
  return hip_status(launch_evict8(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
