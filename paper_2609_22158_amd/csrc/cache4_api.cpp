// C ABI of the 4-bit cache (include/stepkv_cache4.h): argument validation,
// launch planning and workspace layout.
#include "stepkv_cache4.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>

#include "cache4.h"

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

int check_cache(const stepkv_cache4* c) {
  if (!c) return STEPKV_EINVAL;
  if (c->num_layers < 1 || c->num_kv_heads < 1 || c->num_seqs < 1 || c->head_dim < 1)
    return STEPKV_EINVAL;
  if (!c->cu_rows_host || !c->cu_rows || !c->lens) return STEPKV_EINVAL;
  if (!offsets(c->cu_rows_host, c->num_seqs)) return STEPKV_EINVAL;
  if (c->head_dim != 64 && c->head_dim != 128) return STEPKV_EUNSUPPORTED;
  if (c->cu_rows_host[c->num_seqs] > STEPKV_CACHE4_MAX_ROWS) return STEPKV_EUNSUPPORTED;
  if (c->cu_rows_host[c->num_seqs] > 0 &&
      (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales))
    return STEPKV_EINVAL;  // NULL buffers hold 0 rows
  const size_t ns = c->head_dim / kGroup4;
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_scales, ns) ||
      !aligned(c->v_scales, ns) || !aligned(c->k_bounds, 16))
    return STEPKV_EINVAL;
  const int64_t lh = (int64_t)c->num_layers * c->num_kv_heads;
  if (lh * c->num_seqs > std::numeric_limits<int32_t>::max()) return STEPKV_EUNSUPPORTED;
  return STEPKV_OK;
}

int check_heads(const stepkv_cache4* c, int32_t num_q_heads) {
  if (num_q_heads < 1 || num_q_heads % c->num_kv_heads != 0) return STEPKV_EINVAL;
  if ((int64_t)c->num_layers * c->num_seqs * num_q_heads > std::numeric_limits<int32_t>::max())
    return STEPKV_EUNSUPPORTED;
  return STEPKV_OK;
}

Cache4View view(const stepkv_cache4* c) {
  Cache4View w;
  w.k_codes = static_cast<uint8_t*>(c->k_codes);
  w.v_codes = static_cast<uint8_t*>(c->v_codes);
  w.k_scales = static_cast<uint8_t*>(c->k_scales);
  w.v_scales = static_cast<uint8_t*>(c->v_scales);
  w.k_bounds = static_cast<uint16_t*>(c->k_bounds);
  w.cu_rows = c->cu_rows;
  w.lens = c->lens;
  w.status = c->status;
  w.L = c->num_layers;
  w.H = c->num_kv_heads;
  w.S = c->num_seqs;
  w.d = c->head_dim;
  w.rows = c->cu_rows_host[c->num_seqs];
  w.nblk = w.rows / kBlock4 + w.S;
  return w;
}

Attend4Args attend_args(const stepkv_cache4* c, int32_t num_q_heads, int32_t num_blocks) {
  Attend4Args a{};
  a.c = view(c);
  a.Hq = num_q_heads;
  a.G = num_q_heads / c->num_kv_heads;
  a.nlist = num_blocks;
  plan_attend4(a, c->cu_rows_host);
  return a;
}

size_t keys_bytes(const stepkv_cache4* c) {
  const Cache4View w = view(c);
  return align_up(sizeof(uint64_t) * (size_t)w.L * w.H * w.nblk);
}

int check_attend(const stepkv_cache4* c, int32_t num_q_heads, const void* q_dec, float scale,
                 const float* out) {
  const int rc = check_heads(c, num_q_heads);
  if (rc != STEPKV_OK) return rc;
  if (!q_dec || !out || !std::isfinite(scale) || !aligned(q_dec, 16)) return STEPKV_EINVAL;
  // the kernel scales logits by scale * log2(e): 0 times an infinity is NaN
  if (scale > 0.0f && !std::isfinite(scale * 1.44269504088896341f)) return STEPKV_EINVAL;
  return STEPKV_OK;
}

int check_select(const stepkv_cache4* c, int32_t num_q_heads, const void* q_dec,
                 int32_t num_blocks, int32_t first_blocks, int32_t last_blocks,
                 const int32_t* blocks) {
  const int rc = check_heads(c, num_q_heads);
  if (rc != STEPKV_OK) return rc;
  if (!q_dec || !blocks || !c->k_bounds || !aligned(q_dec, 16)) return STEPKV_EINVAL;
  if (num_blocks < 1 || first_blocks < 0 || last_blocks < 0 ||
      (int64_t)first_blocks + last_blocks > num_blocks)
    return STEPKV_EINVAL;
  return STEPKV_OK;
}

size_t partial_bytes(const Attend4Args& a) {
  return align_up(sizeof(float) * attend4_partial_floats(a));
}

int run_attend(const stepkv_cache4* c, Attend4Args a, const void* q_dec, const int32_t* blocks,
               float scale, float* out, float* lse, void* workspace, hipStream_t st) {
  a.q = static_cast<const uint16_t*>(q_dec);
  a.blocks = blocks;
  a.out = out;
  a.lse = lse;
  a.partial = static_cast<float*>(workspace);
  a.scale = scale > 0.0f ? scale : (float)(1.0 / std::sqrt((double)c->head_dim));
  return hip_status(launch_attend4(a, st));
}

Select4Args select_args(const stepkv_cache4* c, int32_t num_q_heads, const void* q_dec,
                        int32_t num_blocks, int32_t first_blocks, int32_t last_blocks,
                        int32_t* blocks, void* workspace) {
  Select4Args a;
  a.c = view(c);
  a.q = static_cast<const uint16_t*>(q_dec);
  a.keys = static_cast<uint64_t*>(workspace);
  a.blocks = blocks;
  a.Hq = num_q_heads;
  a.G = num_q_heads / c->num_kv_heads;
  a.n = num_blocks;
  a.first = first_blocks;
  a.last = last_blocks;
  plan_select4(a, c->cu_rows_host);
  return a;
}

}  // namespace

extern "C" {

int stepkv_cache4_compact(const stepkv_problem* pb, const stepkv_cache4* c, const void* k,
                          const void* v, const int32_t* idx, int32_t shared_idx,
                          const int32_t* cu_retained, void* stream) {
  const int rc = check_cache(c);
  if (rc != STEPKV_OK) return rc;
  if (!pb || pb->num_layers != c->num_layers || pb->num_kv_heads != c->num_kv_heads ||
      pb->head_dim != c->head_dim || pb->num_seqs != c->num_seqs || !pb->cu_seqlens_host ||
      !pb->cu_seqlens || !offsets(pb->cu_seqlens_host, pb->num_seqs))
    return STEPKV_EINVAL;
  if (!cu_retained || !aligned(k, 16) || !aligned(v, 16)) return STEPKV_EINVAL;
  if (pb->cu_seqlens_host[pb->num_seqs] > 0 && (!k || !v || !idx))
    return STEPKV_EINVAL;  // NULL sources hold 0 tokens
  Write4Args a;
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
  a.shared_idx = shared_idx != 0;
  int64_t nb = 0;  // R_s is at most the sequence's source tokens
  for (int s = 0; s < c->num_seqs; ++s) {
    const int32_t room = c->cu_rows_host[s + 1] - c->cu_rows_host[s];
    const int32_t n = pb->cu_seqlens_host[s + 1] - pb->cu_seqlens_host[s];
    nb += ((int64_t)std::min(room, n) + kBlock4 - 1) / kBlock4;
  }
  a.nblocks = (int)nb;
  if (!write4_fits(a)) return STEPKV_EUNSUPPORTED;
  return hip_status(launch_write4(a, static_cast<hipStream_t>(stream)));
}

int stepkv_cache4_advance(const stepkv_cache4* c, const int32_t* cu_new, void* stream) {
  const int rc = check_cache(c);
  if (rc != STEPKV_OK) return rc;
  if (!cu_new) return STEPKV_EINVAL;
  return hip_status(launch_advance4(view(c), cu_new, static_cast<hipStream_t>(stream)));
}

int stepkv_cache4_append(const stepkv_cache4* c, const void* k_new, const int64_t* k_strides,
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
  Write4Args a;
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
  a.nsrc = num_new;
  a.shared_idx = 0;
  // n rows in order touch at most floor((n - 1) / 64) + 2 blocks, and at most n
  a.nblocks = (int)std::min<int64_t>(num_new, (int64_t)num_new / kBlock4 + 2 * (int64_t)c->num_seqs);
  if (!write4_fits(a)) return STEPKV_EUNSUPPORTED;
  return hip_status(launch_write4(a, static_cast<hipStream_t>(stream)));
}

int stepkv_cache4_read(const stepkv_cache4* c, const int32_t* cu_out, int32_t out_rows,
                       void* k_out, void* v_out, void* stream) {
  const int rc = check_cache(c);
  if (rc != STEPKV_OK) return rc;
  if (!cu_out || out_rows < 0 || (out_rows > 0 && !k_out && !v_out)) return STEPKV_EINVAL;
  if (!aligned(k_out, 16) || !aligned(v_out, 16)) return STEPKV_EINVAL;
  if (out_rows == 0) return STEPKV_OK;
  Read4Args a;
  a.c = view(c);
  a.cu_out = cu_out;
  a.k_out = static_cast<uint16_t*>(k_out);
  a.v_out = static_cast<uint16_t*>(v_out);
  a.out_rows = out_rows;
  if (out_rows > STEPKV_CACHE4_MAX_ROWS || !read4_fits(a)) return STEPKV_EUNSUPPORTED;
  return hip_status(launch_read4(a, static_cast<hipStream_t>(stream)));
}

size_t stepkv_cache4_decode_workspace_bytes(const stepkv_cache4* c, int32_t num_q_heads,
                                            int32_t num_blocks) {
  if (check_cache(c) != STEPKV_OK || check_heads(c, num_q_heads) != STEPKV_OK || num_blocks < 0)
    return 0;
  return std::max(partial_bytes(attend_args(c, num_q_heads, num_blocks)), kAlign);
}

int stepkv_cache4_decode(const stepkv_cache4* c, int32_t num_q_heads, const void* q_dec,
                         const int32_t* blocks, int32_t num_blocks, float scale, float* out,
                         float* lse, void* workspace, size_t ws_bytes, void* stream) {
  int rc = check_cache(c);
  if (rc == STEPKV_OK) rc = check_attend(c, num_q_heads, q_dec, scale, out);
  if (rc != STEPKV_OK) return rc;
  if (blocks ? num_blocks < 1 : num_blocks != 0) return STEPKV_EINVAL;
  const Attend4Args a = attend_args(c, num_q_heads, num_blocks);
  if (!attend4_fits(a)) return STEPKV_EUNSUPPORTED;
  const size_t need = partial_bytes(a);
  if (need > 0 && (!workspace || !aligned(workspace, kAlign) || ws_bytes < need))
    return STEPKV_EWORKSPACE;
  return run_attend(c, a, q_dec, blocks, scale, out, lse, workspace,
                    static_cast<hipStream_t>(stream));
}

size_t stepkv_cache4_select_workspace_bytes(const stepkv_cache4* c) {
  if (check_cache(c) != STEPKV_OK) return 0;
  return keys_bytes(c);
}

int stepkv_cache4_select_blocks(const stepkv_cache4* c, int32_t num_q_heads, const void* q_dec,
                                int32_t num_blocks, int32_t first_blocks, int32_t last_blocks,
                                int32_t* blocks, void* workspace, size_t ws_bytes, void* stream) {
  int rc = check_cache(c);
  if (rc == STEPKV_OK)
    rc = check_select(c, num_q_heads, q_dec, num_blocks, first_blocks, last_blocks, blocks);
  if (rc != STEPKV_OK) return rc;
  if (!workspace || !aligned(workspace, kAlign) || ws_bytes < keys_bytes(c))
    return STEPKV_EWORKSPACE;
  const Select4Args a = select_args(c, num_q_heads, q_dec, num_blocks, first_blocks, last_blocks,
                                    blocks, workspace);
  if (!select4_fits(a)) return STEPKV_EUNSUPPORTED;
  return hip_status(launch_select4(a, static_cast<hipStream_t>(stream)));
}

size_t stepkv_cache4_sparse_workspace_bytes(const stepkv_cache4* c, int32_t num_q_heads,
                                            int32_t num_blocks) {
  if (num_blocks < 1) return 0;
  const size_t part = stepkv_cache4_decode_workspace_bytes(c, num_q_heads, num_blocks);
  return part == 0 ? 0 : part + keys_bytes(c);
}

int stepkv_cache4_decode_sparse(const stepkv_cache4* c, int32_t num_q_heads, const void* q_dec,
                                int32_t num_blocks, int32_t first_blocks, int32_t last_blocks,
                                float scale, int32_t* blocks, float* out, float* lse,
                                void* workspace, size_t ws_bytes, void* stream) {
  // every argument of both steps is validated before anything is launched
  int rc = check_cache(c);
  if (rc == STEPKV_OK) rc = check_attend(c, num_q_heads, q_dec, scale, out);
  if (rc == STEPKV_OK)
    rc = check_select(c, num_q_heads, q_dec, num_blocks, first_blocks, last_blocks, blocks);
  if (rc != STEPKV_OK) return rc;
  const Attend4Args a = attend_args(c, num_q_heads, num_blocks);
  if (!attend4_fits(a)) return STEPKV_EUNSUPPORTED;
  const Select4Args b = select_args(c, num_q_heads, q_dec, num_blocks, first_blocks, last_blocks,
                                    blocks, workspace);
  if (!select4_fits(b)) return STEPKV_EUNSUPPORTED;
  const size_t keys = keys_bytes(c);
  if (!workspace || !aligned(workspace, kAlign) || ws_bytes < keys + partial_bytes(a))
    return STEPKV_EWORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  rc = hip_status(launch_select4(b, st));
  if (rc != STEPKV_OK) return rc;
  return run_attend(c, a, q_dec, blocks, scale, out, lse, static_cast<uint8_t*>(workspace) + keys,
                    st);
}

}  // extern "C"
