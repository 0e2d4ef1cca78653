// C ABI of libstc: argument validation and dispatch to the kernel launchers.
#include <math.h>

#include <algorithm>

#include "../../include/stc.h"
#include "stc_kernels.hpp"

namespace {

constexpr int kMaxGridY = 65535;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool shape_ok(const stc_shape_t* s) {
  if (s->B < 1 || s->Hq < 1 || s->Hkv < 1 || s->N < 1) return false;
  if (s->Hq % s->Hkv != 0 || s->Hq / s->Hkv > 16) return false;
  if (s->D != 64 && s->D != 128) return false;
  if (s->P != 16) return false;
  if (s->G < 1 || s->G > 16 || (s->G & (s->G - 1)) != 0) return false;
  if (s->D % s->G != 0 || s->D / s->G < 8) return false;
  if (s->v_cap_groups < 0) return false;
  if (s->N_cap != 0 && (s->N_cap < s->N || (long long)s->N_cap > (1ll << 30))) return false;
  if ((long long)s->B * s->Hkv > kMaxGridY) return false;
  if ((long long)s->N > (1ll << 30)) return false;
  // the packed store is addressed with 32-bit group offsets
  if ((long long)stc::token_cap(*s) * s->G >= (1ll << 32)) return false;
  return true;
}

int num_pages(const stc_shape_t* s) { return (s->N + s->P - 1) / s->P; }

size_t select_ws_bytes(const stc_shape_t* s, bool per_head = false) {
  return (size_t)s->B * (per_head ? s->Hq : s->Hkv) * num_pages(s) * sizeof(float);
}

bool rot_dim_ok(int rot_dim, int D) { return rot_dim >= 16 && rot_dim <= D && rot_dim % 16 == 0; }

// Whether rows of D elements lie apart: every dimension's stride passes all that the dimensions of smaller
// strides span.  (Strides that interleave without meeting would pass a closer look; no order of a tensor's
// dimensions and no slice of one has such.)
bool rows_apart(const int32_t* sizes, const int64_t* strides, int D) {
  int at[3] = {0, 1, 2};
  std::sort(at, at + 3, [&](int i, int j) { return strides[i] < strides[j]; });
  __int128 span = D;
  for (int i : at) {
    if (sizes[i] == 1) continue;
    if (strides[i] < span) return false;
    span += (__int128)(sizes[i] - 1) * strides[i];
  }
  return true;
}

// Strides of rows that are read in 16-byte pieces, in bf16 elements.
bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0; }

// Page scores at the front of the workspace of stc_decode_step, padded so that the attention
// partials behind them start on a 256-byte boundary.
size_t step_score_bytes(const stc_shape_t* s, int k_pages) {
  if (k_pages >= num_pages(s)) return 0;
  return (select_ws_bytes(s) + 255) & ~(size_t)255;
}

// Scratch memory of stc_decode_step_static: one copy per GPU, held until the process ends.
// In host code the array's name is only a handle; its address on the current device comes
// from hipGetSymbolAddress (static_scratch below) and is what the kernels are given.
static __device__ __align__(256) unsigned char scratch[STC_STATIC_SCRATCH_BYTES];

constexpr int kMaxDevices = 64;
std::atomic<void*> g_scratch_ptr[kMaxDevices];

// Device address of `scratch` on the current device, looked up once per device.
void* static_scratch() {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
  void* p = g_scratch_ptr[dev].load(std::memory_order_acquire);
  if (p) return p;
  if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) return nullptr;
  g_scratch_ptr[dev].store(p, std::memory_order_release);
  return p;
}

}  // namespace

extern "C" {

int stc_version(void) { return 2; }

const char* stc_status_string(int status) {
  switch (status) {
    case STC_OK: return "ok";
    case STC_ERR_NULL: return "a required pointer is NULL";
    case STC_ERR_SHAPE: return "shape or argument out of range";
    case STC_ERR_ALIGN: return "pointer is not 16-byte aligned";
    case STC_ERR_WORKSPACE: return "workspace missing or too small";
    case STC_ERR_LAUNCH: return "kernel launch failed";
    default: return "unknown status";
  }
}

size_t stc_workspace_bytes(const stc_shape_t* shape, int which_call, int k_pages) {
  if (!shape || !shape_ok(shape)) return 0;
  switch (which_call) {
    case STC_WS_ROUTE: return stc::route_ws_bytes(*shape);
    case STC_WS_SELECT: return k_pages >= num_pages(shape) ? 0 : select_ws_bytes(shape);
    case STC_WS_ATTENTION:
      if (k_pages < 1 || k_pages > num_pages(shape)) return 0;
      return stc::attention_ws_bytes(*shape, k_pages);
    case STC_WS_ATTENTION_TAIL:  // k_pages counts the tail's pages too
      if (k_pages < 1) return 0;
      return stc::attention_ws_bytes(*shape, k_pages);
    case STC_WS_SELECT_PER_HEAD:
      return k_pages >= num_pages(shape) ? 0 : select_ws_bytes(shape, true);
    case STC_WS_ATTENTION_PER_HEAD:
      if (k_pages < 1 || k_pages > num_pages(shape)) return 0;
      return stc::attention_ws_bytes(*shape, k_pages, true);
    case STC_WS_STEP:
      if (k_pages < 1 || k_pages > num_pages(shape)) return 0;
      return step_score_bytes(shape, k_pages) + stc::attention_ws_bytes(*shape, k_pages);
    case STC_WS_STEP_TAIL:  // k_pages counts the tail's pages too; scores always have room
      if (k_pages < 1) return 0;
      return step_score_bytes(shape, 0) + stc::attention_ws_bytes(*shape, k_pages);
    default: return 0;
  }
}

size_t stc_bounds_bytes(const stc_shape_t* shape) {
  if (!shape || !shape_ok(shape)) return 0;
  const size_t tiles = stc::bounds_tiles(stc::token_cap(*shape));
  return (size_t)shape->B * shape->Hkv * tiles * stc::kBoundsTilePages * shape->D * 4;
}

int stc_build_page_bounds(const stc_shape_t* shape, const void* K, void* bounds, void* stream) {
  if (!shape || !K || !bounds) return STC_ERR_NULL;
  if (!shape_ok(shape)) return STC_ERR_SHAPE;
  if (!aligned16(K) || !aligned16(bounds)) return STC_ERR_ALIGN;
  return stc::launch_bounds(*shape, K, bounds, (hipStream_t)stream) ? STC_ERR_LAUNCH : STC_OK;
}

int stc_route_and_pack_values(const stc_shape_t* shape, int mode, const void* V,
                              const float* logits, const uint8_t* kcount, int fixed_k,
                              const uint16_t* mask_in, uint16_t* mask, uint32_t* tok_off,
                              void* vpacked, int32_t* dev_status, void* ws, size_t ws_bytes,
                              void* stream) {
  if (!shape || !V || !mask || !tok_off || !vpacked) return STC_ERR_NULL;
  if (!shape_ok(shape)) return STC_ERR_SHAPE;
  const int base_mode = mode & ~STC_ROUTE_SHARED;
  if (base_mode == STC_ROUTE_TOPK) {
    if (!logits) return STC_ERR_NULL;
    if (!kcount && (fixed_k < 0 || fixed_k > shape->G)) return STC_ERR_SHAPE;
  } else if (base_mode == STC_ROUTE_GLOBAL) {
    if (!logits) return STC_ERR_NULL;
    if (fixed_k < 0 || fixed_k > shape->G) return STC_ERR_SHAPE;
  } else if (base_mode == STC_ROUTE_MASK) {
    if (!mask_in) return STC_ERR_NULL;
    if ((mode & STC_ROUTE_SHARED) && (const void*)mask_in == (const void*)mask) return STC_ERR_SHAPE;
  } else {
    return STC_ERR_SHAPE;
  }
  if (!aligned16(V) || !aligned16(vpacked) || !aligned16(mask) || !aligned16(tok_off) ||
      (logits && !aligned16(logits)) || (mask_in && !aligned16(mask_in)))
    return STC_ERR_ALIGN;
  if (!ws || ws_bytes < stc::route_ws_bytes(*shape) || !aligned16(ws)) return STC_ERR_WORKSPACE;
  return stc::launch_route_pack(*shape, mode, V, logits, kcount, fixed_k, mask_in, mask, tok_off,
                                vpacked, dev_status, ws, (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

namespace {

int select_pages_impl(const stc_shape_t* shape, const void* q, const void* bounds, int k_pages,
                      int32_t* page_idx, float* page_score, void* ws, size_t ws_bytes,
                      bool per_head, void* stream) {
  if (!shape || !page_idx) return STC_ERR_NULL;
  if (!shape_ok(shape) || k_pages < 1) return STC_ERR_SHAPE;
  if (!aligned16(page_idx)) return STC_ERR_ALIGN;
  float* score = page_score;
  if (k_pages < num_pages(shape)) {
    if (!q || !bounds) return STC_ERR_NULL;
    if (!aligned16(q) || !aligned16(bounds) || (page_score && !aligned16(page_score)))
      return STC_ERR_ALIGN;
    if (!score) {
      if (!ws || ws_bytes < select_ws_bytes(shape, per_head) || !aligned16(ws))
        return STC_ERR_WORKSPACE;
      score = (float*)ws;
    }
  }
  return stc::launch_select(*shape, q, bounds, k_pages, page_idx, score, per_head,
                            (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

}  // namespace

int stc_select_pages(const stc_shape_t* shape, const void* q, const void* bounds, int k_pages,
                     int32_t* page_idx, float* page_score, void* ws, size_t ws_bytes,
                     void* stream) {
  return select_pages_impl(shape, q, bounds, k_pages, page_idx, page_score, ws, ws_bytes, false,
                           stream);
}

int stc_select_pages_per_head(const stc_shape_t* shape, const void* q, const void* bounds,
                              int k_pages, int32_t* page_idx, float* page_score, void* ws,
                              size_t ws_bytes, void* stream) {
  return select_pages_impl(shape, q, bounds, k_pages, page_idx, page_score, ws, ws_bytes, true,
                           stream);
}

int stc_score_pages(const stc_shape_t* shape, const void* q, const void* bounds,
                    float* page_score, void* stream) {
  if (!shape || !q || !bounds || !page_score) return STC_ERR_NULL;
  if (!shape_ok(shape)) return STC_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(bounds) || !aligned16(page_score)) return STC_ERR_ALIGN;
  return stc::launch_score(*shape, q, bounds, page_score, false, (hipStream_t)stream) ? STC_ERR_LAUNCH
                                                                               : STC_OK;
}

namespace {

// Argument checks of the attention calls; launches nothing.
int decode_attention_check(const stc_shape_t* shape, const void* q, const void* K,
                           const void* vpacked, const uint16_t* mask, const uint32_t* tok_off,
                           const int32_t* page_idx, int k_pages, const void* K_tail,
                           const void* V_tail, int n_tail, int tail_cap, bool per_head,
                           const float* out, const void* ws, size_t ws_bytes) {
  if (!shape || !q || !K || !vpacked || !mask || !tok_off || !out) return STC_ERR_NULL;
  if (!shape_ok(shape) || k_pages < 1 || k_pages > num_pages(shape) || shape->v_cap_groups < 1)
    return STC_ERR_SHAPE;
  // the kernels address one stream's keys and packed values with 32-bit byte offsets
  if ((long long)stc::token_cap(*shape) * shape->D * 2 >= (1ll << 32) ||
      shape->v_cap_groups * (shape->D / shape->G) * 2 >= (1ll << 32))
    return STC_ERR_SHAPE;
  if (n_tail < 0 || tail_cap < 0 || n_tail > tail_cap ||
      (long long)tail_cap * shape->D * 2 >= (1ll << 32))
    return STC_ERR_SHAPE;
  if (n_tail > 0 && (!K_tail || !V_tail)) return STC_ERR_NULL;
  if (!aligned16(q) || !aligned16(K) || !aligned16(vpacked) || !aligned16(mask) ||
      !aligned16(tok_off) || (page_idx && !aligned16(page_idx)) || !aligned16(out) ||
      (n_tail > 0 && (!aligned16(K_tail) || !aligned16(V_tail))))
    return STC_ERR_ALIGN;
  const int slots = k_pages + (n_tail + shape->P - 1) / shape->P;
  if (per_head && (long long)shape->B * shape->Hq > kMaxGridY) return STC_ERR_SHAPE;
  const size_t need = stc::attention_ws_bytes(*shape, slots, per_head);
  if (need && (!ws || ws_bytes < need || !aligned16(ws))) return STC_ERR_WORKSPACE;
  return STC_OK;
}

int decode_attention_impl(const stc_shape_t* shape, const void* q, const void* K,
                          const void* vpacked, const uint16_t* mask, const uint32_t* tok_off,
                          const int32_t* page_idx, int k_pages, const void* K_tail,
                          const void* V_tail, int n_tail, int tail_cap, bool per_head,
                          const uint16_t* page_heads, float* out, void* ws, size_t ws_bytes,
                          void* stream) {
  const int rc = decode_attention_check(shape, q, K, vpacked, mask, tok_off, page_idx, k_pages,
                                        K_tail, V_tail, n_tail, tail_cap, per_head, out, ws,
                                        ws_bytes);
  if (rc) return rc;
  return stc::launch_attention(*shape, q, K, vpacked, mask, tok_off, page_idx, k_pages, K_tail,
                               V_tail, n_tail, tail_cap, per_head, page_heads, nullptr, nullptr,
                               out, ws, (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

}  // namespace

int stc_decode_attention(const stc_shape_t* shape, const void* q, const void* K,
                         const void* vpacked, const uint16_t* mask, const uint32_t* tok_off,
                         const int32_t* page_idx, int k_pages, float* out, void* ws,
                         size_t ws_bytes, void* stream) {
  return decode_attention_impl(shape, q, K, vpacked, mask, tok_off, page_idx, k_pages, nullptr,
                               nullptr, 0, 0, false, nullptr, out, ws, ws_bytes, stream);
}

int stc_decode_attention_per_head(const stc_shape_t* shape, const void* q, const void* K,
                                  const void* vpacked, const uint16_t* mask,
                                  const uint32_t* tok_off, const int32_t* page_idx, int k_pages,
                                  float* out, void* ws, size_t ws_bytes, void* stream) {
  return decode_attention_impl(shape, q, K, vpacked, mask, tok_off, page_idx, k_pages, nullptr,
                               nullptr, 0, 0, true, nullptr, out, ws, ws_bytes, stream);
}

int stc_decode_attention_tail(const stc_shape_t* shape, const void* q, const void* K,
                              const void* vpacked, const uint16_t* mask, const uint32_t* tok_off,
                              const int32_t* page_idx, int k_pages, const void* K_tail,
                              const void* V_tail, int n_tail, int tail_cap, float* out, void* ws,
                              size_t ws_bytes, void* stream) {
  return decode_attention_impl(shape, q, K, vpacked, mask, tok_off, page_idx, k_pages, K_tail,
                               V_tail, n_tail, tail_cap, false, nullptr, out, ws, ws_bytes, stream);
}

namespace {

// Selection followed by attention (with or without a tail) on one stream.  score_bytes =
// size of the score region at the front of the workspace.
int decode_step_impl(const stc_shape_t* shape, const void* q, const void* bounds, const void* K,
                     const void* vpacked, const uint16_t* mask, const uint32_t* tok_off,
                     int k_pages, const void* K_tail, const void* V_tail, int n_tail,
                     int tail_cap, int32_t* page_idx, float* out, void* ws, size_t ws_bytes,
                     size_t score_bytes, void* stream) {
  if (!shape || !q || !bounds || !page_idx) return STC_ERR_NULL;
  if (!shape_ok(shape) || k_pages < 1 || k_pages > num_pages(shape)) return STC_ERR_SHAPE;
  if (!aligned16(bounds) || !aligned16(page_idx)) return STC_ERR_ALIGN;
  const bool selecting = k_pages < num_pages(shape);
  if (selecting && (!ws || ws_bytes < score_bytes || !aligned16(ws))) return STC_ERR_WORKSPACE;
  char* attn_ws = ws ? (char*)ws + score_bytes : nullptr;
  const size_t attn_bytes = ws_bytes >= score_bytes ? ws_bytes - score_bytes : 0;
  const int rc = decode_attention_check(shape, q, K, vpacked, mask, tok_off, nullptr, k_pages,
                                        K_tail, V_tail, n_tail, tail_cap, false, out, attn_ws,
                                        attn_bytes);
  if (rc) return rc;
  const hipStream_t st = (hipStream_t)stream;
  const int tail_pages = (n_tail + shape->P - 1) / shape->P;
  if (!selecting) {  // every page: the attention kernel writes the list 0 .. NP-1 itself
    return stc::launch_attention(*shape, q, K, vpacked, mask, tok_off, nullptr, k_pages, K_tail,
                                 V_tail, n_tail, tail_cap, false, nullptr, nullptr, page_idx, out,
                                 attn_ws, st)
               ? STC_ERR_LAUNCH
               : STC_OK;
  }
  if (stc::step_is_one_kernel(*shape, k_pages, tail_pages))
    return stc::launch_step(*shape, q, bounds, K, vpacked, mask, tok_off, k_pages, K_tail, V_tail,
                            n_tail, tail_cap, (float*)ws, page_idx, out, st)
               ? STC_ERR_LAUNCH
               : STC_OK;
  if (!stc::attention_can_select(*shape, k_pages, tail_pages)) {
    if (stc::launch_select(*shape, q, bounds, k_pages, page_idx, (float*)ws, false, st) ||
        stc::launch_attention(*shape, q, K, vpacked, mask, tok_off,
                              selecting ? page_idx : nullptr, k_pages, K_tail, V_tail, n_tail,
                              tail_cap, false, nullptr, nullptr, nullptr, out, attn_ws, st))
      return STC_ERR_LAUNCH;
    return STC_OK;
  }
  if (stc::launch_score(*shape, q, bounds, (float*)ws, false, st) ||
      stc::launch_attention(*shape, q, K, vpacked, mask, tok_off, nullptr, k_pages, K_tail,
                            V_tail, n_tail, tail_cap, false, nullptr, (const float*)ws, page_idx,
                            out, attn_ws, st))
    return STC_ERR_LAUNCH;
  return STC_OK;
}

}  // namespace

int stc_decode_step(const stc_shape_t* shape, const void* q, const void* bounds, const void* K,
                    const void* vpacked, const uint16_t* mask, const uint32_t* tok_off,
                    int k_pages, int32_t* page_idx, float* out, void* ws, size_t ws_bytes,
                    void* stream) {
  if (!shape) return STC_ERR_NULL;
  if (!shape_ok(shape)) return STC_ERR_SHAPE;
  return decode_step_impl(shape, q, bounds, K, vpacked, mask, tok_off, k_pages, nullptr, nullptr,
                          0, 0, page_idx, out, ws, ws_bytes, step_score_bytes(shape, k_pages),
                          stream);
}

int stc_decode_step_tail(const stc_shape_t* shape, const void* q, const void* bounds,
                         const void* K, const void* vpacked, const uint16_t* mask,
                         const uint32_t* tok_off, int k_pages, const void* K_tail,
                         const void* V_tail, int n_tail, int tail_cap, int32_t* page_idx,
                         float* out, void* ws, size_t ws_bytes, void* stream) {
  if (!shape) return STC_ERR_NULL;
  if (!shape_ok(shape)) return STC_ERR_SHAPE;
  return decode_step_impl(shape, q, bounds, K, vpacked, mask, tok_off, k_pages, K_tail, V_tail,
                          n_tail, tail_cap, page_idx, out, ws, ws_bytes,
                          step_score_bytes(shape, 0), stream);
}

int stc_decode_step_static(const stc_shape_t* shape, const void* q, const void* bounds,
                           const void* K, const void* vpacked, const uint16_t* mask,
                           const uint32_t* tok_off, int k_pages, int32_t* page_idx, float* out,
                           void* stream) {
  if (!shape) return STC_ERR_NULL;
  if (!shape_ok(shape) || k_pages < 1 || k_pages > num_pages(shape)) return STC_ERR_SHAPE;
  const size_t score_bytes = step_score_bytes(shape, k_pages);
  const size_t need = score_bytes + stc::attention_ws_bytes(*shape, k_pages);
  if (need > (size_t)STC_STATIC_SCRATCH_BYTES) return STC_ERR_WORKSPACE;
  void* ws = static_scratch();
  if (!ws) return STC_ERR_LAUNCH;
  // every byte of the scratch region that a kernel of the step reads (page scores, split
  // partials) has been written earlier in the same step, so nothing needs clearing
  return decode_step_impl(shape, q, bounds, K, vpacked, mask, tok_off, k_pages, nullptr, nullptr,
                          0, 0, page_idx, out, ws, STC_STATIC_SCRATCH_BYTES, score_bytes, stream);
}

int stc_flush_tail(const stc_shape_t* shape, void* K_tail, void* V_tail, int n_flush, int n_tail,
                   int tail_cap, int mode, const float* logits, const uint8_t* kcount, int fixed_k,
                   const uint16_t* mask_in, void* K, void* bounds, uint16_t* mask,
                   uint32_t* tok_off, void* vpacked, int32_t* dev_status, void* stream) {
  if (!shape || !K_tail || !V_tail || !K || !bounds || !mask || !tok_off || !vpacked)
    return STC_ERR_NULL;
  if (!shape_ok(shape) || n_flush < 1 || n_flush > n_tail || n_tail > tail_cap ||
      (long long)shape->N + n_flush > stc::token_cap(*shape))
    return STC_ERR_SHAPE;
  if (mode == STC_ROUTE_TOPK) {
    if (!logits) return STC_ERR_NULL;
    if (!kcount && (fixed_k < 0 || fixed_k > shape->G)) return STC_ERR_SHAPE;
  } else if (mode == STC_ROUTE_MASK) {
    if (!mask_in) return STC_ERR_NULL;
  } else {
    return STC_ERR_SHAPE;  // a global budget is not incremental
  }
  if (!aligned16(K_tail) || !aligned16(V_tail) || !aligned16(K) || !aligned16(bounds) ||
      !aligned16(mask) || !aligned16(tok_off) || !aligned16(vpacked) ||
      (logits && !aligned16(logits)) || (mask_in && !aligned16(mask_in)))
    return STC_ERR_ALIGN;
  return stc::launch_flush_tail(*shape, K_tail, V_tail, n_flush, n_tail, tail_cap, mode, logits, kcount,
                                fixed_k, mask_in, K, bounds, mask, tok_off, vpacked, dev_status,
                                (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

int stc_union_pages(const stc_shape_t* shape, const int32_t* page_idx_per_head, int k_pages,
                    int32_t* union_idx, uint16_t* union_heads, int union_cap, void* stream) {
  if (!shape || !page_idx_per_head || !union_idx || !union_heads) return STC_ERR_NULL;
  if (!shape_ok(shape) || k_pages < 1 || k_pages > num_pages(shape)) return STC_ERR_SHAPE;
  const long long R = shape->Hq / shape->Hkv;
  // every selected page must fit; the lists are staged in 64 KiB of LDS
  const long long need = R * k_pages < num_pages(shape) ? R * k_pages : num_pages(shape);
  if (union_cap < need || R * k_pages * 4 > 65536) return STC_ERR_SHAPE;
  if (!aligned16(page_idx_per_head) || !aligned16(union_idx) || !aligned16(union_heads))
    return STC_ERR_ALIGN;
  return stc::launch_union_pages(*shape, page_idx_per_head, k_pages, union_idx, union_heads,
                                 union_cap, (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

int stc_decode_attention_union(const stc_shape_t* shape, const void* q, const void* K,
                               const void* vpacked, const uint16_t* mask, const uint32_t* tok_off,
                               const int32_t* union_idx, const uint16_t* union_heads,
                               int union_cap, float* out, void* ws, size_t ws_bytes,
                               void* stream) {
  if (!union_idx || !union_heads) return STC_ERR_NULL;
  if (!aligned16(union_heads)) return STC_ERR_ALIGN;
  return decode_attention_impl(shape, q, K, vpacked, mask, tok_off, union_idx, union_cap, nullptr,
                               nullptr, 0, 0, false, union_heads, out, ws, ws_bytes, stream);
}

int stc_append_tail(const stc_shape_t* shape, const void* k_new, const void* v_new, void* K_tail,
                    void* V_tail, int n_tail, int tail_cap, void* stream) {
  if (!shape || !k_new || !v_new || !K_tail || !V_tail) return STC_ERR_NULL;
  if (!shape_ok(shape) || n_tail < 0 || n_tail >= tail_cap) return STC_ERR_SHAPE;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(K_tail) || !aligned16(V_tail))
    return STC_ERR_ALIGN;
  return stc::launch_append_tail(*shape, k_new, v_new, K_tail, V_tail, n_tail, tail_cap,
                                 (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

int stc_router_logits(int32_t B, int32_t Hkv, int32_t N, int32_t d_model, int32_t G,
                      const void* h, const void* W, const float* bias, int32_t bias_per_batch,
                      float* logits, void* stream) {
  if (!h || !W || !logits) return STC_ERR_NULL;
  if (bias_per_batch != 0 && bias_per_batch != 1) return STC_ERR_SHAPE;
  if (B < 1 || Hkv < 1 || N < 1 || d_model < 128 || d_model % 128 != 0 || B > kMaxGridY ||
      !(G == 1 || G == 2 || G == 4 || G == 8 || G == 16))
    return STC_ERR_SHAPE;
  if (!aligned16(h) || !aligned16(W) || !aligned16(logits) || (bias && ((uintptr_t)bias & 3)))
    return STC_ERR_ALIGN;
  return stc::launch_router_logits(h, W, bias, bias_per_batch ? G : 0, logits, B, Hkv, N, d_model,
                                   G, (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

namespace {
bool shared_ok(const stc_shape_t* s, int k_pages, int tail_cap) {
  return shape_ok(s) && k_pages >= 1 && k_pages <= num_pages(s) && tail_cap >= 0 &&
         tail_cap <= (1 << 30) && s->v_cap_groups >= 1;
}
}  // namespace

size_t stc_shared_workspace_bytes(const stc_shape_t* shape, int k_pages, int tail_cap) {
  if (!shape || !shared_ok(shape, k_pages, tail_cap)) return 0;
  return stc::shared_ws_bytes(*shape, k_pages, tail_cap);
}

int stc_decode_attention_shared(const stc_shape_t* shape, const void* q, const void* K,
                                const void* vpacked, const uint16_t* mask, const uint32_t* tok_off,
                                const int32_t* page_idx, int k_pages, const void* K_tail,
                                const void* V_tail, const int32_t* n_tail, int tail_cap, int out_type,
                                void* out, void* ws, size_t ws_bytes, void* stream) {
  if (!shape || !q || !K || !vpacked || !mask || !tok_off || !out) return STC_ERR_NULL;
  if (!shared_ok(shape, k_pages, tail_cap) || (out_type != STC_OUT_F32 && out_type != STC_OUT_BF16))
    return STC_ERR_SHAPE;
  if (tail_cap > 0 && (!K_tail || !V_tail || !n_tail)) return STC_ERR_NULL;
  if (!aligned16(q) || !aligned16(K) || !aligned16(vpacked) || !aligned16(mask) ||
      !aligned16(tok_off) || (page_idx && !aligned16(page_idx)) || !aligned16(out) ||
      ((uintptr_t)n_tail & 3) || (tail_cap > 0 && (!aligned16(K_tail) || !aligned16(V_tail))))
    return STC_ERR_ALIGN;
  const size_t need = stc::shared_ws_bytes(*shape, k_pages, tail_cap);
  if (need && (!ws || ws_bytes < need || !aligned16(ws))) return STC_ERR_WORKSPACE;
  return stc::launch_shared(*shape, q, K, vpacked, mask, tok_off, page_idx, k_pages, K_tail, V_tail,
                            n_tail, tail_cap, out_type == STC_OUT_BF16, out, ws, (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

int stc_rotary_turns(int32_t rot_dim, const stc_rotary_scaling_t* scaling, double* turns) {
  if (!scaling || !turns) return STC_ERR_NULL;
  const stc_rotary_scaling_t& s = *scaling;
  if (!rot_dim_ok(rot_dim, 128) || !(s.base > 1) || !isfinite(s.base)) return STC_ERR_SHAPE;
  if (s.kind < STC_ROTARY_SCALE_NONE || s.kind > STC_ROTARY_SCALE_WAVELENGTHS) return STC_ERR_SHAPE;
  if (s.kind != STC_ROTARY_SCALE_NONE && (!(s.factor > 0) || !isfinite(s.factor)))
    return STC_ERR_SHAPE;
  if (s.kind >= STC_ROTARY_SCALE_CHANNELS &&
      (s.original_len < 1 || !(s.slow > 0) || !(s.fast > s.slow) || !isfinite(s.fast)))
    return STC_ERR_SHAPE;
  double all[64];
  stc::rotary_turns(rot_dim, s, all);
  // base and factor are finite, but their powers and quotients need not be, nor what the farthest position
  // makes of them
  for (int j = 0; j < rot_dim / 2; ++j)
    if (!isfinite(all[j] * 0x1p31)) return STC_ERR_SHAPE;
  std::copy(all, all + rot_dim / 2, turns);
  return STC_OK;
}

int stc_rotary(int32_t B, int32_t H, int32_t N, int32_t D, int32_t rot_dim, int32_t layout,
               const double* turns, float amplitude, const int32_t* pos, int32_t pos0, const void* x,
               const int64_t* x_stride, void* y, const int64_t* y_stride, void* stream) {
  if (!turns || !x || !x_stride || !y || !y_stride) return STC_ERR_NULL;
  if (B < 1 || B > kMaxGridY || H < 1 || N < 1 || (D != 64 && D != 128) || !rot_dim_ok(rot_dim, D) ||
      !isfinite(amplitude))
    return STC_ERR_SHAPE;
  // a thread for 16 channels, and a launch counts fewer than 2^32 threads, in workgroups of 256
  if ((long long)N * H > ((1ll << 32) - 256) / (D / 16)) return STC_ERR_SHAPE;
  if ((layout & ~STC_ROTARY_INVERSE) != STC_ROTARY_HALVES &&
      (layout & ~STC_ROTARY_INVERSE) != STC_ROTARY_INTERLEAVED)
    return STC_ERR_SHAPE;
  if (!pos && (long long)pos0 + N - 1 > INT32_MAX) return STC_ERR_SHAPE;
  if (!aligned16(turns) || !aligned16(x) || !aligned16(y) || (pos && ((uintptr_t)pos & 3)))
    return STC_ERR_ALIGN;
  const int32_t sizes[3] = {B, H, N};
  for (int i = 0; i < 3; ++i)
    if (!stride_ok(x_stride[i]) || !stride_ok(y_stride[i])) return STC_ERR_ALIGN;
  if (!rows_apart(sizes, y_stride, D)) return STC_ERR_SHAPE;
  // in place only where every row stays where it is: others would be overwritten before they are read
  if (x == y)
    for (int i = 0; i < 3; ++i)
      if (sizes[i] > 1 && x_stride[i] != y_stride[i]) return STC_ERR_SHAPE;
  return stc::launch_rotary(B, H, N, D, rot_dim, layout, turns, amplitude, pos, pos0, x, x_stride, y,
                            y_stride, (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

int stc_rotary_append(const stc_shape_t* shape, const void* q, int64_t q_stride, const void* k_new,
                      int64_t k_stride, const void* v_new, int64_t v_stride, void* q_out,
                      void* K_tail, void* V_tail, const int32_t* n_tail, int32_t* n_out,
                      int tail_cap, int rot_dim, int layout, const double* turns, float amplitude,
                      const int32_t* pos, int32_t pos0, int32_t* dev_status, void* stream) {
  if (!shape || !q || !k_new || !v_new || !q_out || !K_tail || !V_tail || !n_tail)
    return STC_ERR_NULL;
  if (rot_dim != 0 && !turns) return STC_ERR_NULL;
  if (!shape_ok(shape) || tail_cap < 1 || (rot_dim != 0 && !rot_dim_ok(rot_dim, shape->D)) ||
      (layout != STC_ROTARY_HALVES && layout != STC_ROTARY_INTERLEAVED) || !isfinite(amplitude))
    return STC_ERR_SHAPE;
  if (!pos && (long long)pos0 + tail_cap - 1 > INT32_MAX) return STC_ERR_SHAPE;
  // in place only where the rows of a sequence stay where they are
  if (q_out == q && shape->B > 1 && q_stride != (int64_t)shape->Hq * shape->D) return STC_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(q_out) ||
      !aligned16(K_tail) || !aligned16(V_tail) || (turns && !aligned16(turns)) ||
      ((uintptr_t)n_tail & 3) || ((uintptr_t)n_out & 3) || ((uintptr_t)pos & 3) ||
      !stride_ok(q_stride) || !stride_ok(k_stride) || !stride_ok(v_stride))
    return STC_ERR_ALIGN;
  return stc::launch_rotary_append(*shape, q, q_stride, k_new, k_stride, v_new, v_stride, q_out,
                                   K_tail, V_tail, n_tail, n_out, tail_cap, rot_dim, layout, turns,
                                   amplitude, pos, pos0, dev_status, (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

namespace {
constexpr int kMostNodes = 64, kMostLayers = 1024;

bool tree_ok(const stc_shape_t* s, int T, int n_prefix, int k_pages, int tail_cap) {
  return shared_ok(s, k_pages, tail_cap) && tail_cap >= 1 && T >= 1 && T <= kMostNodes &&
         (n_prefix == 1 || n_prefix == s->B);
}

// Sorts the places of n arrays of so many bytes; whether no two of them overlap.
bool apart(uintptr_t* at, int n, size_t bytes) {
  std::sort(at, at + n);
  for (int i = 1; i < n; ++i)
    if (at[i] - at[i - 1] < bytes) return false;
  return true;
}

// Whether an array of so many bytes overlaps one of the n sorted ones, of `each` bytes, other than `own`, which it may be
// itself.
bool overlaps(const void* p, size_t bytes, const uintptr_t* at, int n, size_t each, const void* own = nullptr) {
  const uintptr_t x = (uintptr_t)p;
  for (const uintptr_t* w = std::lower_bound(at, at + n, x < each ? 0 : x - each + 1);
       w != at + n && *w < x + bytes; ++w)
    if (*w != (uintptr_t)own || *w != x) return true;
  return false;
}

// The tails of all layers and their lengths: all there and aligned, and what is written apart from what else is
// read or written.  `also`, `also2`: two more arrays that are read, of B numbers of so many bytes, or NULL.
int layers_status(const stc_shape_t* s, int n_layers, void* const* K, void* const* V, const int32_t* const* n,
                  int32_t* const* out, int tail_cap, const void* also, size_t also_bytes, const void* also2) {
  uintptr_t tails[2 * kMostLayers], written[kMostLayers];
  for (int i = 0; i < n_layers; ++i) {
    if (!K[i] || !V[i] || !n[i] || !out[i]) return STC_ERR_NULL;
    if (!aligned16(K[i]) || !aligned16(V[i]) || ((uintptr_t)n[i] & 3) || ((uintptr_t)out[i] & 3))
      return STC_ERR_ALIGN;
    tails[2 * i] = (uintptr_t)K[i], tails[2 * i + 1] = (uintptr_t)V[i], written[i] = (uintptr_t)out[i];
  }
  const size_t lengths = (size_t)s->B * 4;
  if (!apart(tails, 2 * n_layers, (size_t)s->B * s->Hkv * tail_cap * s->D * 2) ||
      !apart(written, n_layers, lengths))
    return STC_ERR_SHAPE;
  for (int i = 0; i < n_layers; ++i)
    if (overlaps(n[i], lengths, written, n_layers, lengths, out[i])) return STC_ERR_SHAPE;
  if ((also && overlaps(also, s->B * also_bytes, written, n_layers, lengths)) ||
      (also2 && overlaps(also2, lengths, written, n_layers, lengths)))
    return STC_ERR_SHAPE;
  return STC_OK;
}
}  // namespace

int stc_rotary_append_drafts(const stc_shape_t* shape, int T, const void* q, const int64_t* q_stride,
                             const void* k_new, const int64_t* k_stride, const void* v_new,
                             const int64_t* v_stride, void* q_out, void* K_tail, void* V_tail,
                             const int32_t* n_tail, const int32_t* n_draft, int tail_cap, const uint64_t* tree,
                             int tree_per_batch, int rot_dim, int layout, const double* turns, float amplitude,
                             const int32_t* pos, int32_t pos0, int32_t* n_have, int32_t* dev_status,
                             void* stream) {
  if (!shape || !q || !q_stride || !k_new || !k_stride || !v_new || !v_stride || !q_out || !K_tail || !V_tail ||
      !n_tail)
    return STC_ERR_NULL;
  if (rot_dim != 0 && !turns) return STC_ERR_NULL;
  if (!shape_ok(shape) || T < 1 || T > kMostNodes || tail_cap < 1 || tail_cap > (1 << 30) ||
      (tree_per_batch != 0 && tree_per_batch != 1) || (rot_dim != 0 && !rot_dim_ok(rot_dim, shape->D)) ||
      (layout != STC_ROTARY_HALVES && layout != STC_ROTARY_INTERLEAVED) || !isfinite(amplitude))
    return STC_ERR_SHAPE;
  if ((long long)T * (shape->Hq + 2ll * shape->Hkv) * (shape->D / 16) > INT32_MAX - 256) return STC_ERR_SHAPE;
  if (!pos && (long long)pos0 + tail_cap - 1 > INT32_MAX) return STC_ERR_SHAPE;
  // in place only where every row stays where it is
  const int64_t row = (int64_t)shape->Hq * shape->D;
  if (q_out == q && ((shape->B > 1 && q_stride[0] != T * row) || (T > 1 && q_stride[1] != row))) return STC_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || !aligned16(q_out) || !aligned16(K_tail) ||
      !aligned16(V_tail) || (turns && !aligned16(turns)) || ((uintptr_t)n_tail & 3) || ((uintptr_t)n_draft & 3) ||
      ((uintptr_t)pos & 3) || ((uintptr_t)tree & 7) || ((uintptr_t)n_have & 3) ||
      ((uintptr_t)dev_status & 3))
    return STC_ERR_ALIGN;
  const uintptr_t have = (uintptr_t)n_have;  // read by others while it is written
  const size_t counts = (size_t)shape->B * 4;
  if (n_have && (overlaps(n_tail, counts, &have, 1, counts) || (n_draft && overlaps(n_draft, counts, &have, 1, counts))))
    return STC_ERR_SHAPE;
  for (int i = 0; i < 2; ++i)
    if (!stride_ok(q_stride[i]) || !stride_ok(k_stride[i]) || !stride_ok(v_stride[i])) return STC_ERR_ALIGN;
  return stc::launch_rotary_append_tree(*shape, T, q, q_stride, k_new, k_stride, v_new, v_stride, q_out, K_tail,
                                        V_tail, n_tail, n_draft, tail_cap, tree, tree_per_batch != 0, rot_dim,
                                        layout, turns, amplitude, pos, pos0, n_have, dev_status,
                                        (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

int stc_rotary_append_tree(const stc_shape_t* shape, int T, const void* q, const int64_t* q_stride,
                           const void* k_new, const int64_t* k_stride, const void* v_new,
                           const int64_t* v_stride, void* q_out, void* K_tail, void* V_tail,
                           const int32_t* n_tail, const int32_t* n_draft, int tail_cap, const uint64_t* tree,
                           int tree_per_batch, int rot_dim, int layout, const double* turns, float amplitude,
                           const int32_t* pos, int32_t pos0, int32_t* dev_status, void* stream) {
  return stc_rotary_append_drafts(shape, T, q, q_stride, k_new, k_stride, v_new, v_stride, q_out, K_tail, V_tail, n_tail,
                                  n_draft, tail_cap, tree, tree_per_batch, rot_dim, layout, turns, amplitude, pos, pos0,
                                  nullptr, dev_status, stream);
}

size_t stc_tree_workspace_bytes(const stc_shape_t* shape, int T, int n_prefix, int k_pages, int tail_cap) {
  if (!shape || !tree_ok(shape, T, n_prefix, k_pages, tail_cap)) return 0;
  return stc::tree_ws_bytes(*shape, T, n_prefix, k_pages, tail_cap);
}

int stc_decode_attention_tree(const stc_shape_t* shape, int T, int n_prefix, const void* q, const void* K,
                              const void* vpacked, const uint16_t* mask, const uint32_t* tok_off,
                              const int32_t* page_idx, int k_pages, const void* K_tail, const void* V_tail,
                              const int32_t* n_tail, const int32_t* n_draft, int tail_cap, const uint64_t* tree,
                              int tree_per_batch, int out_type, void* out, void* ws, size_t ws_bytes,
                              void* stream) {
  if (!shape || !q || !K || !vpacked || !mask || !tok_off || !K_tail || !V_tail || !n_tail || !out)
    return STC_ERR_NULL;
  if (!tree_ok(shape, T, n_prefix, k_pages, tail_cap) || (tree_per_batch != 0 && tree_per_batch != 1) ||
      (out_type != STC_OUT_F32 && out_type != STC_OUT_BF16))
    return STC_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(K) || !aligned16(vpacked) || !aligned16(mask) || !aligned16(tok_off) ||
      (page_idx && !aligned16(page_idx)) || !aligned16(K_tail) || !aligned16(V_tail) || !aligned16(out) ||
      ((uintptr_t)n_tail & 3) || ((uintptr_t)n_draft & 3) || ((uintptr_t)tree & 7))
    return STC_ERR_ALIGN;
  const size_t need = stc::tree_ws_bytes(*shape, T, n_prefix, k_pages, tail_cap);
  if (!ws || ws_bytes < need || !aligned16(ws)) return STC_ERR_WORKSPACE;
  return stc::launch_tree(*shape, T, n_prefix, q, K, vpacked, mask, tok_off, page_idx, k_pages, K_tail, V_tail,
                          n_tail, n_draft, tail_cap, tree, tree_per_batch != 0, out_type == STC_OUT_BF16, out, ws,
                          (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

int stc_accept_drafts(const stc_shape_t* shape, int T, int n_layers, void* const* K_tail, void* const* V_tail,
                      const int32_t* const* n_tail, int32_t* const* n_out, int tail_cap, const uint64_t* keep,
                      const int32_t* n_draft, void* stream) {
  if (!shape || !K_tail || !V_tail || !n_tail || !n_out || !keep) return STC_ERR_NULL;
  if (!shape_ok(shape) || T < 1 || T > kMostNodes || n_layers < 1 || n_layers > kMostLayers || tail_cap < 1 ||
      tail_cap > (1 << 30))
    return STC_ERR_SHAPE;
  if (((uintptr_t)keep & 7) || ((uintptr_t)n_draft & 3)) return STC_ERR_ALIGN;
  const int status = layers_status(shape, n_layers, K_tail, V_tail, n_tail, n_out, tail_cap, keep, 8, n_draft);
  if (status != STC_OK) return status;
  return stc::launch_accept_tail(*shape, T, n_layers, K_tail, V_tail, n_tail, n_out, tail_cap, keep, n_draft,
                                 (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

int stc_accept_tail(const stc_shape_t* shape, int T, int n_layers, void* const* K_tail, void* const* V_tail,
                    const int32_t* const* n_tail, int32_t* const* n_out, int tail_cap, const uint64_t* keep,
                    void* stream) {
  return stc_accept_drafts(shape, T, n_layers, K_tail, V_tail, n_tail, n_out, tail_cap, keep, nullptr, stream);
}

int stc_fork_tail(const stc_shape_t* shape, int n_layers, void* const* K_tail, void* const* V_tail,
                  const int32_t* const* n_tail, int32_t* const* n_out, int tail_cap, const int32_t* src,
                  const int32_t* n_keep, int32_t* dev_status, void* stream) {
  if (!shape || !K_tail || !V_tail || !n_tail || !n_out || !src) return STC_ERR_NULL;
  if (!shape_ok(shape) || shape->B > stc::kForkMost || n_layers < 1 || n_layers > kMostLayers || tail_cap < 1 ||
      tail_cap > (1 << 30))
    return STC_ERR_SHAPE;
  if (((uintptr_t)src & 3) || ((uintptr_t)n_keep & 3) || ((uintptr_t)dev_status & 3)) return STC_ERR_ALIGN;
  const int status = layers_status(shape, n_layers, K_tail, V_tail, n_tail, n_out, tail_cap, src, 4, n_keep);
  if (status != STC_OK) return status;
  return stc::launch_fork_tail(*shape, n_layers, K_tail, V_tail, n_tail, n_out, tail_cap, src, n_keep, dev_status,
                               (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

int stc_compact_tokens(const void* src, const int32_t* token_idx, void* dst, int32_t B,
                       int32_t Hkv, int32_t N_src, int32_t n_keep, int32_t D,
                       int32_t* dev_status, void* stream) {
  if (!src || !token_idx || !dst) return STC_ERR_NULL;
  if (B < 1 || Hkv < 1 || N_src < 1 || n_keep < 1 || (D != 64 && D != 128)) return STC_ERR_SHAPE;
  if ((long long)B * Hkv > kMaxGridY) return STC_ERR_SHAPE;
  if (!aligned16(src) || !aligned16(dst) || !aligned16(token_idx)) return STC_ERR_ALIGN;
  return stc::launch_compact(src, token_idx, dst, B, Hkv, N_src, n_keep, D, dev_status,
                             (hipStream_t)stream)
             ? STC_ERR_LAUNCH
             : STC_OK;
}

}  // extern "C"
