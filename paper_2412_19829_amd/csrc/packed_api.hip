// C ABI of packed attention and the paged cache: argument validation and dispatch (include/gformer.h).
#include "../../include/gformer.h"

#include <math.h>
#include <string.h>

#include "packed.hpp"
#include "paged.hpp"

namespace gformer {
namespace {

constexpr int64_t kMaxTokenStride = 1 << 20;   // elements
constexpr int64_t kMaxCached = 1 << 30;        // tokens of one sequence, or rows of a packed tensor

// Scales that stay finite as factors of base-2 exponents.
bool scale_fits(float scale) { return fabsf(scale) <= 0x1p127f; }
bool misaligned(uintptr_t all, unsigned bytes) { return (all & (bytes - 1)) != 0; }
template <typename... P> uintptr_t bits(P... p) { return (0 | ... | (uintptr_t)p); }

// (row, head) strides of [rows, heads, d]
gf_status strides2(const int64_t* in, int64_t* out, int heads, int d) {
  if (in[0] == 0 && in[1] == 0) {
    out[0] = (int64_t)heads * d;
    out[1] = d;
    return out[0] > kMaxTokenStride ? GF_ERR_UNSUPPORTED : GF_OK;
  }
  for (int i = 0; i < 2; ++i) {
    if (in[i] < 0 || in[i] % 8 != 0) return GF_ERR_INVALID_ARG;
    out[i] = in[i];
  }
  if (in[0] < d || (heads > 1 && in[1] < d)) return GF_ERR_INVALID_ARG;   // rows would overlap
  return in[0] > kMaxTokenStride ? GF_ERR_UNSUPPORTED : GF_OK;
}

// (page, head, token) strides of [pages, heads, page, d]
gf_status strides3(const int64_t* in, int64_t* out, int heads, int page, int d) {
  if (in[0] == 0 && in[1] == 0 && in[2] == 0) {
    out[0] = (int64_t)heads * page * d;
    out[1] = (int64_t)page * d;
    out[2] = d;
    return GF_OK;
  }
  for (int i = 0; i < 3; ++i) {
    if (in[i] < 0 || in[i] % 8 != 0) return GF_ERR_INVALID_ARG;
    out[i] = in[i];
  }
  if (in[0] < d || in[2] < d || (heads > 1 && in[1] < d)) return GF_ERR_INVALID_ARG;
  return in[2] > kMaxTokenStride ? GF_ERR_UNSUPPORTED : GF_OK;
}

gf_status check_device(void* stream) {
  int dev = 0;
  return call_device(reinterpret_cast<hipStream_t>(stream), &dev) == hipSuccess ? GF_OK : GF_ERR_DEVICE;
}

gf_status check_heads(int dtype, int H, int Hkv, int d) {
  if (dtype != GF_F32 && dtype != GF_BF16) return GF_ERR_INVALID_ARG;
  if (H < 1 || Hkv < 1 || d < 1 || H % Hkv != 0) return GF_ERR_INVALID_ARG;
  return d == 64 || d == 128 ? GF_OK : GF_ERR_UNSUPPORTED;
}

gf_status check_packed(bool backward, int n_seqs, int total_q, int total_k, int H, int Hkv, int d, const gformer_packed_params* p,
                       PackedArgs* a) {
  if (!p || p->struct_size != sizeof(gformer_packed_params)) return GF_ERR_INVALID_ARG;
  if (n_seqs < 0 || total_q < 0 || total_k < 0 || !scale_fits(p->softmax_scale) || (p->zero_tail != 0 && p->zero_tail != 1))
    return GF_ERR_INVALID_ARG;
  gf_status st = check_heads(p->dtype, H, Hkv, d);
  if (st != GF_OK) return st;
  memset(a, 0, sizeof(*a));
  if ((st = strides2(p->q_stride, a->qs, H, d)) != GF_OK || (st = strides2(p->k_stride, a->ks, Hkv, d)) != GF_OK ||
      (st = strides2(p->v_stride, a->vs, Hkv, d)) != GF_OK || (st = strides2(p->o_stride, a->os, H, d)) != GF_OK ||
      (st = strides2(p->do_stride, a->gs, H, d)) != GF_OK || (st = strides2(p->dq_stride, a->dqs, H, d)) != GF_OK ||
      (st = strides2(p->dk_stride, a->dks, Hkv, d)) != GF_OK || (st = strides2(p->dv_stride, a->dvs, Hkv, d)) != GF_OK)
    return st;
  if (total_q > kMaxCached || total_k > kMaxCached || n_seqs > kMaxCached) return GF_ERR_UNSUPPORTED;
  const bool fp32 = p->dtype == GF_F32;
  if (!packed_queries_fit(fp32, d, total_q, H, n_seqs) || (backward && total_k > 0 && !packed_keys_fit(fp32, d, total_k, H, Hkv, n_seqs)))
    return GF_ERR_UNSUPPORTED;
  a->n_seqs = n_seqs;
  a->total_q = total_q;
  a->total_k = total_k;
  a->H = H;
  a->Hkv = Hkv;
  a->d = d;
  a->zero_tail = p->zero_tail;
  a->scale = p->softmax_scale;
  return GF_OK;
}

gf_status check_paged(int Hkv, int d, int n_pages, const gformer_paged_params* p, int* shift, int64_t* kps, int64_t* vps) {
  if (!p || p->struct_size != sizeof(gformer_paged_params)) return GF_ERR_INVALID_ARG;
  gf_status st = check_heads(p->dtype, Hkv, Hkv, d);
  if (st != GF_OK) return st;
  if (n_pages < 0 || p->page_size < 1) return GF_ERR_INVALID_ARG;
  if (p->page_size < 8 || p->page_size > 65536 || (p->page_size & (p->page_size - 1))) return GF_ERR_UNSUPPORTED;
  for (*shift = 3; (1 << *shift) < p->page_size;) ++*shift;
  if ((st = strides3(p->kpage_stride, kps, Hkv, p->page_size, d)) != GF_OK) return st;
  return strides3(p->vpage_stride, vps, Hkv, p->page_size, d);
}

// Whether the table's sequences can be numbered, and how many keys one may have.
gf_status check_table(int width, int shift, int max_len, int* room) {
  if (width < 0 || max_len < 0) return GF_ERR_INVALID_ARG;
  const int64_t held = (int64_t)width << shift;
  if (held > kMaxCached) return GF_ERR_UNSUPPORTED;
  *room = (int)(max_len > 0 && max_len < held ? max_len : held);
  return GF_OK;
}

size_t decode_bytes(int B, int H, int Hkv, int d, int room) {
  const PagedSplit s = paged_split(B, H, Hkv, room);
  if (s.splits == 1) return 0;
  return ((size_t)B * H * s.splits * (d + 2) * sizeof(float) + 255) / 256 * 256;
}

gf_status status(hipError_t e) { return e == hipSuccess ? GF_OK : GF_ERR_DEVICE; }

}  // namespace
}  // namespace gformer

using namespace gformer;

extern "C" {

void gformer_packed_params_init(gformer_packed_params* p) {
  if (!p) return;
  memset(p, 0, sizeof(*p));
  p->struct_size = sizeof(*p);
  p->dtype = GF_BF16;
  p->softmax_scale = 1.f;
}

void gformer_paged_params_init(gformer_paged_params* p) {
  if (!p) return;
  memset(p, 0, sizeof(*p));
  p->struct_size = sizeof(*p);
  p->dtype = GF_BF16;
  p->page_size = 64;
  p->softmax_scale = 1.f;
}

gf_status gformer_packed_attn_fwd(const void* q, const void* k, const void* v, void* out, void* out_rest, float* lse,
                                  const int32_t* cu_q, const int32_t* cu_k, int n_seqs, int total_q, int total_k, int H, int Hkv, int d,
                                  const gformer_packed_params* p, void* hip_stream) {
  PackedArgs a;
  gf_status st = check_packed(false, n_seqs, total_q, total_k, H, Hkv, d, p, &a);
  if (st != GF_OK) return st;
  if (total_q == 0) return GF_OK;
  if (!q || !out || !cu_q || (total_k > 0 && (!k || !v))) return GF_ERR_INVALID_ARG;
  if (!cu_k && total_q != total_k) return GF_ERR_INVALID_ARG;
  if (misaligned(bits(q, k, v, out, out_rest), 16) || misaligned(bits(lse, cu_q, cu_k), 4)) return GF_ERR_INVALID_ARG;
  for (const void* x : {q, k, v})
    if (out == x || (out_rest && out_rest == x)) return GF_ERR_INVALID_ARG;
  if (out_rest == out || (out_rest && p->dtype == GF_F32)) return GF_ERR_INVALID_ARG;
  if ((st = check_device(hip_stream)) != GF_OK) return st;
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = out;
  a.rest = out_rest;
  a.lse = lse;
  a.cu_q = cu_q;
  a.cu_k = cu_k ? cu_k : cu_q;
  return status(launch_packed_fwd(a, p->dtype == GF_BF16, reinterpret_cast<hipStream_t>(hip_stream)));
}

size_t gformer_packed_attn_bwd_workspace_bytes(int total_q, int total_k, int n_seqs, int H, int Hkv, int d,
                                               const gformer_packed_params* p) {
  PackedArgs a;
  if (check_packed(true, n_seqs, total_q, total_k, H, Hkv, d, p, &a) != GF_OK) return 0;
  return packed_stats_bytes(total_q, H) + packed_sums_bytes(total_k, H, Hkv, d);
}

gf_status gformer_packed_attn_bwd(const void* q, const void* k, const void* v, const void* out, const void* out_rest,
                                  const float* lse, const void* dout, void* dq, void* dk, void* dv, const int32_t* cu_q, const int32_t* cu_k, int n_seqs, int total_q,
                                  int total_k, int H, int Hkv, int d, const gformer_packed_params* p, void* workspace,
                                  size_t workspace_bytes, void* hip_stream) {
  PackedArgs a;
  gf_status st = check_packed(true, n_seqs, total_q, total_k, H, Hkv, d, p, &a);
  if (st != GF_OK) return st;
  if (total_q == 0 && total_k == 0) return GF_OK;
  if (!cu_q || (total_q > 0 && (!q || !out || !lse || !dout || !dq)) || (total_k > 0 && (!k || !v || !dk || !dv))) return GF_ERR_INVALID_ARG;
  if (!cu_k && total_q != total_k) return GF_ERR_INVALID_ARG;
  if (out_rest && p->dtype == GF_F32) return GF_ERR_INVALID_ARG;
  if (misaligned(bits(q, k, v, out, out_rest, dout, dq, dk, dv), 16) || misaligned(bits(lse, cu_q, cu_k), 4)) return GF_ERR_INVALID_ARG;
  const void* in[] = {q, k, v, out, out_rest, dout, lse};
  void* grads[] = {dq, dk, dv};
  for (int i = 0; i < 3; ++i) {
    for (const void* x : in)
      if (grads[i] && grads[i] == x) return GF_ERR_INVALID_ARG;
    if (grads[i] && grads[i] == grads[(i + 1) % 3]) return GF_ERR_INVALID_ARG;
  }
  const size_t need = gformer_packed_attn_bwd_workspace_bytes(total_q, total_k, n_seqs, H, Hkv, d, p);
  if (need > 0 && (!workspace || workspace_bytes < need)) return GF_ERR_WORKSPACE;
  if (misaligned(bits(workspace), 256)) return GF_ERR_INVALID_ARG;
  if ((st = check_device(hip_stream)) != GF_OK) return st;
  a.q = q;
  a.k = k;
  a.v = v;
  a.dout = dout;
  a.out = const_cast<void*>(out);   // read by this pass, and so are the rest of it and lse
  a.rest = const_cast<void*>(out_rest);
  a.lse = const_cast<float*>(lse);
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.stats = static_cast<float*>(workspace);
  a.sums = a.stats + packed_stats_bytes(total_q, H) / sizeof(float);
  a.cu_q = cu_q;
  a.cu_k = cu_k ? cu_k : cu_q;
  return status(launch_packed_bwd(a, p->dtype == GF_BF16, reinterpret_cast<hipStream_t>(hip_stream)));
}

size_t gformer_paged_decode_workspace_bytes(int B, int H, int Hkv, int d, int table_width, int max_len,
                                            const gformer_paged_params* p) {
  int shift, room;
  int64_t kps[3], vps[3];
  if (!p || B < 1 || check_heads(p->dtype, H, Hkv, d) != GF_OK || check_paged(Hkv, d, 1, p, &shift, kps, vps) != GF_OK ||
      check_table(table_width, shift, max_len, &room) != GF_OK)
    return 0;
  return decode_bytes(B, H, Hkv, d, room);
}

gf_status gformer_paged_decode(const void* q, const void* k, const void* v, void* out, void* kpages, void* vpages,
                               const int32_t* table, const int32_t* lens, int B, int H, int Hkv, int d, int n_pages,
                               int table_width, int max_len, const gformer_paged_params* p, void* workspace,
                               size_t workspace_bytes, void* hip_stream) {
  PagedDecodeArgs a;
  memset(&a, 0, sizeof(a));
  if (!p) return GF_ERR_INVALID_ARG;
  gf_status st = check_paged(Hkv, d, n_pages, p, &a.shift, a.kps, a.vps);
  if (st != GF_OK) return st;
  if ((st = check_heads(p->dtype, H, Hkv, d)) != GF_OK) return st;
  if (B < 0 || !scale_fits(p->softmax_scale)) return GF_ERR_INVALID_ARG;
  if ((st = check_table(table_width, a.shift, max_len, &a.room)) != GF_OK) return st;
  if ((st = strides2(p->q_stride, a.qs, H, d)) != GF_OK || (st = strides2(p->k_stride, a.ks, Hkv, d)) != GF_OK ||
      (st = strides2(p->v_stride, a.vs, Hkv, d)) != GF_OK || (st = strides2(p->o_stride, a.os, H, d)) != GF_OK)
    return st;
  if (B == 0) return GF_OK;
  const PagedSplit s = paged_split(B, H, Hkv, a.room);
  if (!paged_decode_fits(B, H, Hkv, s)) return GF_ERR_UNSUPPORTED;
  if (n_pages < 1) return GF_ERR_INVALID_ARG;
  if (!q || !out || !kpages || !vpages || (!table && table_width > 0) || !lens || !k != !v) return GF_ERR_INVALID_ARG;
  if (misaligned(bits(q, k, v, out, kpages, vpages), 16) || misaligned(bits(table, lens), 4)) return GF_ERR_INVALID_ARG;
  if (out == q || out == k || out == v || out == kpages || out == vpages || kpages == vpages) return GF_ERR_INVALID_ARG;
  const size_t need = decode_bytes(B, H, Hkv, d, a.room);
  if (need > 0 && (!workspace || workspace_bytes < need)) return GF_ERR_WORKSPACE;
  if (need > 0 && misaligned(bits(workspace), 256)) return GF_ERR_INVALID_ARG;
  if ((st = check_device(hip_stream)) != GF_OK) return st;
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = out;
  a.kpages = kpages;
  a.vpages = vpages;
  a.table = table;
  a.lens = lens;
  a.B = B;
  a.H = H;
  a.Hkv = Hkv;
  a.d = d;
  a.n_pages = n_pages;
  a.width = table_width;
  a.chunk = s.chunk;
  a.splits = s.splits;
  a.scale = p->softmax_scale;
  a.sums = static_cast<float*>(workspace);
  if (s.splits > 1) a.stats = a.sums + (size_t)B * H * s.splits * d;
  return status(launch_paged_decode(a, p->dtype == GF_BF16, reinterpret_cast<hipStream_t>(hip_stream)));
}

gf_status gformer_paged_fill(const void* k, const void* v, void* kpages, void* vpages, const int32_t* table, const int32_t* start,
                             const int32_t* cu, int n_seqs, int total, int Hkv, int d, int n_pages, int table_width,
                             const gformer_paged_params* p, void* hip_stream) {
  PagedFillArgs a;
  memset(&a, 0, sizeof(a));
  int room;
  gf_status st = check_paged(Hkv, d, n_pages, p, &a.shift, a.kps, a.vps);
  if (st != GF_OK) return st;
  if ((st = check_table(table_width, a.shift, 0, &room)) != GF_OK) return st;
  if (n_seqs < 0 || total < 0) return GF_ERR_INVALID_ARG;
  if (total > kMaxCached || n_seqs > kMaxCached) return GF_ERR_UNSUPPORTED;
  if ((st = strides2(p->k_stride, a.ks, Hkv, d)) != GF_OK || (st = strides2(p->v_stride, a.vs, Hkv, d)) != GF_OK) return st;
  if (!paged_fill_fits(total, n_seqs, Hkv)) return GF_ERR_UNSUPPORTED;
  if (total == 0 || n_seqs == 0 || table_width == 0 || n_pages == 0) return GF_OK;
  if (!k || !v || !kpages || !vpages || !table || !start || !cu) return GF_ERR_INVALID_ARG;
  if (misaligned(bits(k, v, kpages, vpages), 16) || misaligned(bits(table, start, cu), 4)) return GF_ERR_INVALID_ARG;
  if (kpages == vpages) return GF_ERR_INVALID_ARG;
  if ((st = check_device(hip_stream)) != GF_OK) return st;
  a.k = k;
  a.v = v;
  a.kpages = kpages;
  a.vpages = vpages;
  a.table = table;
  a.start = start;
  a.cu = cu;
  a.n_seqs = n_seqs;
  a.total = total;
  a.Hkv = Hkv;
  a.d = d;
  a.n_pages = n_pages;
  a.width = table_width;
  return status(launch_paged_fill(a, p->dtype == GF_BF16, reinterpret_cast<hipStream_t>(hip_stream)));
}

gf_status gformer_pages_copy(void* kpages, void* vpages, const int32_t* src, const int32_t* dst, int n_copies, int Hkv, int d,
                             int n_pages, const gformer_paged_params* p, void* hip_stream) {
  PagesCopyArgs a;
  memset(&a, 0, sizeof(a));
  int shift;
  gf_status st = check_paged(Hkv, d, n_pages, p, &shift, a.kps, a.vps);
  if (st != GF_OK) return st;
  if (n_copies < 0) return GF_ERR_INVALID_ARG;
  if ((int64_t)n_copies * Hkv > most_workgroups(kPagedThreads)) return GF_ERR_UNSUPPORTED;
  if (n_copies == 0) return GF_OK;
  if (!kpages || !vpages || !src || !dst || kpages == vpages) return GF_ERR_INVALID_ARG;
  if (misaligned(bits(kpages, vpages), 16) || misaligned(bits(src, dst), 4)) return GF_ERR_INVALID_ARG;
  if ((st = check_device(hip_stream)) != GF_OK) return st;
  a.kpages = kpages;
  a.vpages = vpages;
  a.src = src;
  a.dst = dst;
  a.n_copies = n_copies;
  a.Hkv = Hkv;
  a.d = d;
  a.n_pages = n_pages;
  a.page = p->page_size;
  return status(launch_pages_copy(a, p->dtype == GF_BF16, reinterpret_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
