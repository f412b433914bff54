// C-ABI entry points: context and layer handles, argument checking, and the
// launch sequences of the draft step (Eq. 5), the verify block (Eq. 4 grouped
// by the union of Eq. 2 / Eq. 3) and greedy acceptance (Algorithm 1).
#include <new>

#include "dx_internal.cuh"

bool dx_bf16_hidden_supported(int H);
void dx_cache_forget_layer(dx_cache* c, dx_layer* L);

extern "C" const char* dx_status_string(dx_status s) {
  switch (s) {
    case DX_OK: return "ok";
    case DX_ERR_INVALID_ARG: return "invalid argument";
    case DX_ERR_SHAPE: return "shape mismatch";
    case DX_ERR_CUDA: return "CUDA runtime error";
    case DX_ERR_OOM: return "out of memory";
    case DX_ERR_NOT_RESIDENT: return "expert not resident";
    case DX_ERR_TIMEOUT: return "timed out";
    case DX_ERR_CACHE_FULL: return "expert cache full";
    case DX_ERR_UNSUPPORTED: return "unsupported configuration";
    default: return "unknown status";
  }
}

extern "C" dx_status dx_create(int device, dx_ctx** out) {
  if (!out) return DX_ERR_INVALID_ARG;
  *out = nullptr;
  int n = 0;
  if (cudaGetDeviceCount(&n) != cudaSuccess || device < 0 || device >= n) return DX_ERR_CUDA;
  dx_ctx* ctx = new (std::nothrow) dx_ctx();
  if (!ctx) return DX_ERR_OOM;
  ctx->device = device;
  ctx->last_cuda = cudaSuccess;
  ctx->launches = 0;
  ctx->pdl_mask = DX_PDL_ROUTE | DX_PDL_EXPERTS;
  ctx->accept_keep_bytes = 0;
  ctx->wait_limit = DX_WAIT_LIMIT_DEFAULT;
  cudaError_t e = cudaSetDevice(device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&ctx->sm_count, cudaDevAttrMultiProcessorCount, device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&ctx->smem_optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, device);
  if (e == cudaSuccess) e = cudaMalloc(&ctx->work, sizeof(DxWork));
  if (e == cudaSuccess) e = cudaMalloc(&ctx->ticket, sizeof(unsigned int) * 4);
  if (e == cudaSuccess) e = cudaMalloc(&ctx->keys, sizeof(unsigned long long) * DX_MAX_M);
  if (e == cudaSuccess) e = cudaMalloc(&ctx->dev_status, sizeof(int32_t));
  if (e == cudaSuccess) e = cudaMalloc(&ctx->handover, 4 * sizeof(unsigned int));
  if (e == cudaSuccess) e = cudaMemset(ctx->handover, 0, 4 * sizeof(unsigned int));
  if (e == cudaSuccess) e = cudaMalloc(&ctx->conf_part, sizeof(float2) * 8 * ctx->sm_count * DX_MAX_M);
  if (e == cudaSuccess) e = cudaMalloc(&ctx->route_counts, sizeof(int32_t) * DX_ROUTE_CTAS_PER_SM * ctx->sm_count * DX_MAX_E);
  if (e == cudaSuccess) e = dx_logprobs_prepare();
  if (e == cudaSuccess) e = dx_distill_prepare(ctx);
  if (e == cudaSuccess) e = cudaMalloc(&ctx->scratch_i32, sizeof(int32_t) * 2);
  if (e == cudaSuccess) e = cudaMalloc(&ctx->union_dev, sizeof(int32_t) * (DX_MAX_E + 1 + DX_MAX_TOPK));
  if (e == cudaSuccess) e = cudaHostAlloc((void**)&ctx->union_host, sizeof(int32_t) * (DX_MAX_E + 1 + DX_MAX_TOPK),
                                          cudaHostAllocMapped);
  if (e == cudaSuccess) e = cudaHostGetDevicePointer((void**)&ctx->union_host_dev, ctx->union_host, 0);
  if (e == cudaSuccess) e = cudaMemset(ctx->work, 0, sizeof(DxWork));
  if (e == cudaSuccess) e = cudaMemset(ctx->ticket, 0, sizeof(unsigned int) * 4);
  if (e == cudaSuccess) e = cudaMemset(ctx->keys, 0, sizeof(unsigned long long) * DX_MAX_M);
  if (e == cudaSuccess) e = cudaMemset(ctx->dev_status, 0, sizeof(int32_t));
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  if (e != cudaSuccess) {
    dx_destroy(ctx);
    return e == cudaErrorMemoryAllocation ? DX_ERR_OOM : DX_ERR_CUDA;
  }
  *out = ctx;
  return DX_OK;
}

extern "C" dx_status dx_destroy(dx_ctx* ctx) {
  if (!ctx) return DX_ERR_INVALID_ARG;
  cudaFree(ctx->work);
  cudaFree(ctx->ticket);
  cudaFree(ctx->keys);
  cudaFree(ctx->dev_status);
  cudaFree(ctx->handover);
  cudaFree(ctx->conf_part);
  cudaFree(ctx->route_counts);
  cudaFree(ctx->scratch_i32);
  cudaFree(ctx->union_dev);
  if (ctx->union_host) cudaFreeHost(ctx->union_host);
  delete ctx;
  return DX_OK;
}

extern "C" dx_status dx_last_device_status(dx_ctx* ctx, void* stream, int32_t* out) {
  if (!ctx || !out) return DX_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  DX_CUDA(ctx, cudaMemcpyAsync(out, ctx->dev_status, sizeof(int32_t), cudaMemcpyDeviceToHost, st));
  DX_CUDA(ctx, cudaMemsetAsync(ctx->dev_status, 0, sizeof(int32_t), st));
  DX_CUDA(ctx, cudaStreamSynchronize(st));
  return DX_OK;
}

extern "C" dx_status dx_set_activation_split(dx_ctx* ctx, int32_t on) {
  if (!ctx) return DX_ERR_INVALID_ARG;
  ctx->act_split = on ? 1 : 0;
  return DX_OK;
}

extern "C" dx_status dx_set_launch_overlap(dx_ctx* ctx, int32_t mask) {
  if (!ctx || mask < 0 || mask > (DX_PDL_ROUTE | DX_PDL_EXPERTS | DX_PDL_ACCEPT)) return DX_ERR_INVALID_ARG;
  ctx->pdl_mask = mask;
  return DX_OK;
}

extern "C" dx_status dx_set_wait_limit(dx_ctx* ctx, uint32_t polls) {
  if (!ctx) return DX_ERR_INVALID_ARG;
  ctx->wait_limit = polls ? polls : DX_WAIT_LIMIT_DEFAULT;
  return DX_OK;
}

extern "C" dx_status dx_set_accept_l2_keep(dx_ctx* ctx, size_t bytes) {
  if (!ctx) return DX_ERR_INVALID_ARG;
  ctx->accept_keep_bytes = bytes;
  return DX_OK;
}

// Small host -> device transfers by a kernel that reads the pinned buffer through its device mapping: a copy-engine
// transfer of a few ten KB costs more in set-up than in time on the link (measured: a 32 KB memcpy node in front of a
// decode step adds 13 us to it, this kernel 4 us).
namespace {
__global__ void dx_stage_block_kernel(uint4* dst, const uint4* src, size_t n16, unsigned char* dst_tail,
                                      const unsigned char* src_tail, int n_tail) {
  const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  // a routing kernel behind this one may become resident and fetch its router rows while the link is read; it waits
  // for this grid's completion before it touches the block
  dx_pdl_trigger();
  if (i < n16) {
    uint4 v;   // (a volatile load: the host rewrites the buffer between two calls, nothing may be served from a cache)
    asm volatile("ld.volatile.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(src + i));
    dst[i] = v;
  }
  if (i < (size_t)n_tail) dst_tail[i] = *reinterpret_cast<const volatile unsigned char*>(src_tail + i);
}
}  // namespace

extern "C" dx_status dx_stage_block(dx_ctx* ctx, void* dst, const void* src_host, size_t bytes, void* stream) {
  if (!ctx || !dst || !src_host) return DX_ERR_INVALID_ARG;
  if (bytes == 0) return DX_OK;
  cudaStream_t st = (cudaStream_t)stream;
  void* src_dev = nullptr;
  if (cudaHostGetDevicePointer(&src_dev, const_cast<void*>(src_host), 0) != cudaSuccess) {
    (void)cudaGetLastError();
    return DX_ERR_INVALID_ARG;   // not page-locked (or not mapped): the kernel could not read it
  }
  if (bytes > ((size_t)1 << 20) || ((uintptr_t)dst) % 16 || ((uintptr_t)src_dev) % 16) {
    DX_CUDA(ctx, cudaMemcpyAsync(dst, src_host, bytes, cudaMemcpyHostToDevice, st));   // large or unaligned: the copy engine
    return DX_OK;
  }
  const size_t n16 = bytes / 16;
  const int n_tail = (int)(bytes % 16);
  const size_t threads = n16 > (size_t)n_tail ? n16 : (size_t)n_tail;
  const int grid = (int)((threads + 255) / 256);
  dx_stage_block_kernel<<<grid, 256, 0, st>>>(reinterpret_cast<uint4*>(dst), reinterpret_cast<const uint4*>(src_dev), n16,
                                              reinterpret_cast<unsigned char*>(dst) + n16 * 16,
                                              reinterpret_cast<const unsigned char*>(src_dev) + n16 * 16, n_tail);
  DX_CUDA(ctx, cudaGetLastError());
  ctx->launches++;
  return DX_OK;
}

extern "C" int32_t dx_last_cuda_error(dx_ctx* ctx) { return ctx ? (int32_t)ctx->last_cuda : 0; }
extern "C" int64_t dx_kernel_launches(dx_ctx* ctx) { return ctx ? ctx->launches : 0; }

static dx_status check_desc(const dx_layer_desc* d) {
  if (!d) return DX_ERR_INVALID_ARG;
  if (d->hidden <= 0 || d->n_experts <= 0 || d->top_k <= 0 || d->inter <= 0 || d->n_shared < 0) return DX_ERR_SHAPE;
  if (d->top_k > d->n_experts) return DX_ERR_SHAPE;
  if (d->weight_dtype != DX_DTYPE_FP32 && d->weight_dtype != DX_DTYPE_BF16 && d->weight_dtype != DX_DTYPE_Q4 &&
      d->weight_dtype != DX_DTYPE_BF16_WIDE)
    return DX_ERR_INVALID_ARG;
  if (d->score_fn != DX_SCORE_SOFTMAX && d->score_fn != DX_SCORE_SIGMOID) return DX_ERR_INVALID_ARG;
  if (d->hidden > DX_MAX_H || d->hidden % 256 || d->n_experts > DX_MAX_E || d->top_k > DX_MAX_TOPK ||
      d->n_shared > DX_MAX_SHARED)
    return DX_ERR_UNSUPPORTED;
  if (d->inter % DX_TILE_I || (d->n_shared && (d->shared_inter <= 0 || d->shared_inter % DX_TILE_I)) ||
      d->draft_inter < 0 || d->draft_inter % DX_TILE_I)
    return DX_ERR_UNSUPPORTED;
  if (d->weight_dtype != DX_DTYPE_FP32 && !dx_bf16_hidden_supported(d->hidden)) return DX_ERR_UNSUPPORTED;
  // 4-bit experts: quantisation blocks of 32 along the rows of W_d [hidden, inter]
  if (d->weight_dtype == DX_DTYPE_Q4 &&
      (d->inter % 32 || (d->n_shared && d->shared_inter % 32) || d->draft_inter % 32))
    return DX_ERR_UNSUPPORTED;
  return DX_OK;
}

extern "C" dx_status dx_expert_blob_bytes(const dx_layer_desc* desc, int32_t inter, size_t* bytes_out) {
  if (!desc || !bytes_out) return DX_ERR_INVALID_ARG;
  if (inter <= 0 || inter % DX_TILE_I || desc->hidden <= 0 || desc->hidden % 256) return DX_ERR_UNSUPPORTED;
  if (desc->weight_dtype == DX_DTYPE_Q4) {
    if (inter % 32 || !dx_bf16_hidden_supported(desc->hidden)) return DX_ERR_UNSUPPORTED;
    *bytes_out = (size_t)inter * dx_chunk_bytes(desc->hidden, true);   // inter / 8 units of 8 chunks
    return DX_OK;
  }
  if (desc->weight_dtype == DX_DTYPE_BF16_WIDE && !dx_bf16_hidden_supported(desc->hidden)) return DX_ERR_UNSUPPORTED;
  *bytes_out = (size_t)3 * desc->hidden * inter * (desc->weight_dtype == DX_DTYPE_FP32 ? 4 : 2);
  return DX_OK;
}

extern "C" dx_status dx_pack_expert(dx_ctx* ctx, const dx_layer_desc* desc, int32_t inter, const void* Wg,
                                    const void* Wu, const void* Wd, void* blob_out, void* stream) {
  if (!ctx || !desc || !Wg || !Wu || !Wd || !blob_out) return DX_ERR_INVALID_ARG;
  if (inter <= 0 || inter % DX_TILE_I || desc->hidden <= 0 || desc->hidden % 256) return DX_ERR_UNSUPPORTED;
  if (((uintptr_t)blob_out) % 128) return DX_ERR_INVALID_ARG;
  if (desc->weight_dtype == DX_DTYPE_Q4) {
    if (inter % 32 || !dx_bf16_hidden_supported(desc->hidden)) return DX_ERR_UNSUPPORTED;
    if (((uintptr_t)Wg) % 2 || ((uintptr_t)Wu) % 2 || ((uintptr_t)Wd) % 2) return DX_ERR_INVALID_ARG;
    DX_CUDA(ctx, dx_launch_pack_q4(desc->hidden, inter, Wg, Wu, Wd, blob_out, (cudaStream_t)stream));
  } else if (desc->weight_dtype == DX_DTYPE_BF16_WIDE) {
    if (!dx_bf16_hidden_supported(desc->hidden)) return DX_ERR_UNSUPPORTED;
    DX_CUDA(ctx, dx_launch_pack_wide(desc->hidden, inter, Wg, Wu, Wd, blob_out, (cudaStream_t)stream));
  } else {
    DX_CUDA(ctx, dx_launch_pack(desc->weight_dtype, desc->hidden, inter, Wg, Wu, Wd, blob_out, (cudaStream_t)stream));
  }
  ctx->launches++;
  return DX_OK;
}

extern "C" dx_status dx_q4_expert_bytes(const dx_layer_desc* desc, int32_t inter, size_t* bytes_out) {
  if (!desc || !bytes_out) return DX_ERR_INVALID_ARG;
  if (desc->weight_dtype != DX_DTYPE_BF16 && desc->weight_dtype != DX_DTYPE_Q4) return DX_ERR_UNSUPPORTED;
  // blocks of 32 along the rows of W_g, W_u [inter, hidden] and of W_d [hidden, inter]
  if (inter <= 0 || inter % 32 || desc->hidden <= 0 || desc->hidden % 256) return DX_ERR_UNSUPPORTED;
  *bytes_out = (size_t)3 * desc->hidden * inter / 32 * 18;
  return DX_OK;
}

extern "C" dx_status dx_expand_q4_expert(dx_ctx* ctx, const dx_layer_desc* desc, int32_t inter, const void* q4_blob,
                                         void* blob_out, void* stream) {
  if (!ctx || !desc || !q4_blob || !blob_out) return DX_ERR_INVALID_ARG;
  if (desc->weight_dtype != DX_DTYPE_BF16) return DX_ERR_UNSUPPORTED;   // the result is a bf16 blob
  size_t need = 0;
  dx_status s = dx_q4_expert_bytes(desc, inter, &need);
  if (s != DX_OK) return s;
  if (((uintptr_t)blob_out) % 128 || ((uintptr_t)q4_blob) % 2) return DX_ERR_INVALID_ARG;
  DX_CUDA(ctx, dx_launch_expand_q4(desc->hidden, inter, q4_blob, blob_out, (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

extern "C" dx_status dx_layer_create(dx_ctx* ctx, const dx_layer_desc* desc, dx_layer** out) {
  if (!ctx || !out) return DX_ERR_INVALID_ARG;
  *out = nullptr;
  dx_status s = check_desc(desc);
  if (s != DX_OK) return s;
  dx_layer* L = new (std::nothrow) dx_layer();
  if (!L) return DX_ERR_OOM;
  L->ctx = ctx;
  L->desc = *desc;
  L->W_r = nullptr;
  L->bias = nullptr;
  L->table_len = desc->n_shared + 1 + desc->n_experts;
  L->table_host = new (std::nothrow) const void*[L->table_len]();
  L->table_dev = nullptr;
  L->dirty = true;
  L->cache = nullptr;
  L->cache_layer = -1;
  if (!L->table_host) { delete L; return DX_ERR_OOM; }
  cudaError_t e = cudaMalloc((void**)&L->table_dev, sizeof(void*) * L->table_len);
  if (e != cudaSuccess) {
    ctx->last_cuda = e;
    delete[] L->table_host;
    delete L;
    return DX_ERR_OOM;
  }
  *out = L;
  return DX_OK;
}

extern "C" dx_status dx_layer_destroy(dx_layer* L) {
  if (!L) return DX_ERR_INVALID_ARG;
  if (L->cache) dx_cache_forget_layer(L->cache, L);   // the cache must not patch a table that is gone
  cudaFree((void*)L->table_dev);
  delete[] L->table_host;
  delete L;
  return DX_OK;
}

extern "C" dx_status dx_layer_set_router(dx_layer* L, const void* W_r, const float* bias) {
  if (!L || !W_r) return DX_ERR_INVALID_ARG;
  if (((uintptr_t)W_r) % 16 || ((uintptr_t)bias) % 4) return DX_ERR_INVALID_ARG;
  L->W_r = W_r;
  L->bias = bias;
  return DX_OK;
}

static dx_status set_slot(dx_layer* L, int idx, const void* blob, bool allow_null) {
  if (!blob && !allow_null) return DX_ERR_INVALID_ARG;
  if (((uintptr_t)blob) % 128) return DX_ERR_INVALID_ARG;
  L->table_host[idx] = blob;
  L->dirty = true;
  return DX_OK;
}
extern "C" dx_status dx_layer_set_shared(dx_layer* L, int32_t s, const void* blob) {
  if (!L || s < 0 || s >= L->desc.n_shared) return DX_ERR_INVALID_ARG;
  return set_slot(L, s, blob, false);
}
extern "C" dx_status dx_layer_set_draft(dx_layer* L, const void* blob) {
  if (!L || L->desc.draft_inter <= 0) return DX_ERR_INVALID_ARG;
  return set_slot(L, L->desc.n_shared, blob, false);
}
extern "C" dx_status dx_layer_set_expert(dx_layer* L, int32_t e, const void* blob) {
  if (!L || e < 0 || e >= L->desc.n_experts) return DX_ERR_INVALID_ARG;
  return set_slot(L, L->desc.n_shared + 1 + e, blob, true);
}

static dx_status upload_table(dx_layer* L, cudaStream_t st) {
  if (!L->dirty) return DX_OK;
  // pageable source: the runtime stages the bytes before returning, the copy itself is stream-ordered
  DX_CUDA(L->ctx, cudaMemcpyAsync((void*)L->table_dev, L->table_host, sizeof(void*) * L->table_len,
                                  cudaMemcpyHostToDevice, st));
  L->dirty = false;
  return DX_OK;
}

struct RouteOut {
  int32_t* topk_ids;
  float* topk_w;
  uint64_t* union_mask;
  int32_t* union_ids;
  int32_t* union_count;
  int32_t* offsets;
  int32_t* perm;
};

static dx_status do_route(dx_layer* L, const float* h, int K, float* y, const RouteOut& o, bool draft, bool residual,
                          cudaStream_t st, int top_r = 1, bool use_draft_expert = true, bool paired = false,
                          bool skip_top1 = false, bool mirror_to_host = false) {
  dx_ctx* ctx = L->ctx;
  const dx_layer_desc& d = L->desc;
  if (!h || !y || h == y) return DX_ERR_INVALID_ARG;
  if (K < 1 || K > DX_MAX_K) return DX_ERR_UNSUPPORTED;
  if (!L->W_r) return DX_ERR_NOT_RESIDENT;
  for (int s = 0; s < d.n_shared; ++s)
    if (!L->table_host[s]) return DX_ERR_NOT_RESIDENT;
  if (draft && use_draft_expert && d.draft_inter > 0 && !L->table_host[d.n_shared]) return DX_ERR_NOT_RESIDENT;
  if (top_r < 0 || top_r > d.top_k) return DX_ERR_INVALID_ARG;
  if (((uintptr_t)h) % 16 || ((uintptr_t)y) % 16) return DX_ERR_INVALID_ARG;
  dx_status s = upload_table(L, st);
  if (s != DX_OK) return s;
  DxRouteParams p{};
  p.h = h; p.K = K; p.H = d.hidden; p.E = d.n_experts; p.k = d.top_k;
  p.score_fn = d.score_fn; p.norm_topk = d.norm_topk; p.scale = d.routed_scale; p.gamma = d.draft_gamma;
  p.W_r = L->W_r; p.bias = L->bias; p.table = L->table_dev;
  p.n_shared = d.n_shared;
  p.shared_tiles = d.n_shared ? d.shared_inter / DX_TILE_I : 0;
  p.routed_tiles = d.inter / DX_TILE_I;
  p.draft_tiles = draft && use_draft_expert ? d.draft_inter / DX_TILE_I : 0;
  p.draft_mode = draft ? 1 : 0;
  p.top_r = top_r;
  p.skip_top1 = skip_top1 ? 1 : 0;
  p.rms_norm = residual ? 1 : 0;
  p.residual = residual ? 1 : 0;
  p.y = y; p.work = ctx->work; p.dev_status = ctx->dev_status;
  p.handover = paired ? ctx->handover : nullptr;
  p.topk_ids = o.topk_ids; p.topk_w = o.topk_w;
  p.union_mask = (unsigned long long*)o.union_mask; p.union_ids = o.union_ids; p.union_count = o.union_count;
  p.offsets = o.offsets; p.perm = o.perm;
  p.host_mirror = mirror_to_host ? ctx->union_host_dev : nullptr;
  // (the router of a layer with 4-bit experts, or with experts in the wide layout, is bf16)
  DX_CUDA(ctx, dx_launch_route(ctx, p, d.weight_dtype == DX_DTYPE_FP32 ? DX_DTYPE_FP32 : DX_DTYPE_BF16, st));
  ctx->launches++;
  return DX_OK;
}

static dx_status do_experts(dx_layer* L, const float* h, int K, float* y, bool draft, bool residual,
                            cudaStream_t st, int first_routed = 0, int n_routed = -1, bool do_static = true,
                            bool paired = false, bool skip_shared = false,
                            const unsigned long long* subset = nullptr, bool tolerate_missing = false) {
  dx_ctx* ctx = L->ctx;
  const dx_layer_desc& d = L->desc;
  if (!h || !y || h == y) return DX_ERR_INVALID_ARG;
  if (K < 1 || K > DX_MAX_K) return DX_ERR_UNSUPPORTED;
  if (((uintptr_t)h) % 16 || ((uintptr_t)y) % 16) return DX_ERR_INVALID_ARG;   // 16-byte loads and reductions
  dx_status s = upload_table(L, st);
  if (s != DX_OK) return s;
  DxExpertParams p{};
  p.x = h;
  p.y = y;
  p.table = L->table_dev;
  p.table_len = L->table_len;
  p.work = ctx->work;
  p.dev_status = ctx->dev_status;
  p.H = d.hidden;
  p.K = K;
  p.rms_norm = residual ? 1 : 0;
  p.n_shared = d.n_shared;
  p.shared_tiles = d.n_shared ? d.shared_inter / DX_TILE_I : 0;
  p.draft_tiles = draft ? d.draft_inter / DX_TILE_I : 0;
  p.routed_tiles = d.inter / DX_TILE_I;
  p.gamma = d.draft_gamma;
  p.handover = paired ? ctx->handover : nullptr;
  p.wait_limit = ctx->wait_limit;
  p.first_routed = first_routed;
  p.n_routed = n_routed;
  p.do_static = do_static ? 1 : 0;
  p.skip_shared = skip_shared ? 1 : 0;
  p.use_subset = subset ? 1 : 0;
  p.tolerate_missing = tolerate_missing ? 1 : 0;
  for (int i = 0; i < DX_MAX_E / 64; ++i) p.subset[i] = subset ? subset[i] : 0ull;
  DX_CUDA(ctx, dx_launch_experts(ctx, p, L->desc.weight_dtype, K, st));
  ctx->launches++;
  if (L->cache) dx_cache_note_use(L->cache, L->cache_layer, st);
  return DX_OK;
}

// Routing kernel and expert kernel of one layer call, launched back to back.  Only here the two kernels use the
// device-side hand-over (bf16 blobs): the routing kernel sets the words, the expert kernel that is certain to
// follow consumes and clears them.
static dx_status do_pair(dx_layer* L, const float* h, int K, float* y, const RouteOut& o, bool draft, bool residual,
                         cudaStream_t st, int top_r = 1, bool use_draft_expert = true) {
  const bool paired = L->desc.weight_dtype != DX_DTYPE_FP32;
  dx_status s = do_route(L, h, K, y, o, draft, residual, st, top_r, use_draft_expert, paired);
  if (s != DX_OK) return s;
  s = do_experts(L, h, K, y, draft && use_draft_expert, residual, st, 0, -1, true, paired);
  if (s != DX_OK && paired) cudaMemsetAsync(L->ctx->handover, 0, 4 * sizeof(unsigned int), st);
  return s;
}

extern "C" dx_status moe_draft_step(dx_layer* L, const float* h, float* y, int32_t* topk_ids, float* topk_w,
                                    void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  RouteOut o{topk_ids, topk_w, nullptr, nullptr, nullptr, nullptr, nullptr};
  return do_pair(L, h, 1, y, o, true, false, st);
}

extern "C" dx_status moe_draft_step_residual(dx_layer* L, const float* h_in, float* h_out, int32_t* topk_ids,
                                             float* topk_w, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  RouteOut o{topk_ids, topk_w, nullptr, nullptr, nullptr, nullptr, nullptr};
  return do_pair(L, h_in, 1, h_out, o, true, true, st);
}

extern "C" dx_status moe_verify_route(dx_layer* L, const float* h, int32_t K, float* y, int32_t* topk_ids,
                                      float* topk_w, uint64_t* union_mask, int32_t* union_ids, int32_t* union_count,
                                      int32_t* offsets, int32_t* perm, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  RouteOut o{topk_ids, topk_w, union_mask, union_ids, union_count, offsets, perm};
  return do_route(L, h, K, y, o, false, false, (cudaStream_t)stream);
}

extern "C" dx_status moe_verify_experts(dx_layer* L, const float* h, int32_t K, float* y, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  return do_experts(L, h, K, y, false, false, (cudaStream_t)stream);
}

extern "C" dx_status moe_verify_experts_range(dx_layer* L, const float* h, int32_t K, float* y, int32_t first_union,
                                              int32_t n_union, int32_t include_shared, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  if (first_union < 0 || n_union < 0) return DX_ERR_INVALID_ARG;
  return do_experts(L, h, K, y, false, false, (cudaStream_t)stream, first_union, n_union, include_shared != 0);
}

extern "C" dx_status moe_draft_step_topr(dx_layer* L, const float* h, float* y, int32_t top_r,
                                         int32_t use_draft_expert, int32_t* topk_ids, float* topk_w, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  RouteOut o{topk_ids, topk_w, nullptr, nullptr, nullptr, nullptr, nullptr};
  if (top_r < 1) return DX_ERR_INVALID_ARG;
  return do_pair(L, h, 1, y, o, true, false, st, top_r, use_draft_expert != 0);
}

extern "C" dx_status moe_draft_step_topr_residual(dx_layer* L, const float* h_in, float* h_out, int32_t top_r,
                                                  int32_t use_draft_expert, int32_t* topk_ids, float* topk_w,
                                                  void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  RouteOut o{topk_ids, topk_w, nullptr, nullptr, nullptr, nullptr, nullptr};
  if (top_r < 1) return DX_ERR_INVALID_ARG;
  return do_pair(L, h_in, 1, h_out, o, true, true, (cudaStream_t)stream, top_r, use_draft_expert != 0);
}

extern "C" dx_status moe_draft_route(dx_layer* L, const float* h, float* y, int32_t* topk_ids, float* topk_w,
                                     void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  RouteOut o{topk_ids, topk_w, nullptr, nullptr, nullptr, nullptr, nullptr};
  return do_route(L, h, 1, y, o, true, false, (cudaStream_t)stream);
}

extern "C" dx_status moe_draft_experts(dx_layer* L, const float* h, float* y, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  return do_experts(L, h, 1, y, true, false, (cudaStream_t)stream);
}

extern "C" dx_status moe_verify_block(dx_layer* L, const float* h, int32_t K, float* y, int32_t* topk_ids,
                                      float* topk_w, uint64_t* union_mask, int32_t* union_ids, int32_t* union_count,
                                      int32_t* offsets, int32_t* perm, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  RouteOut o{topk_ids, topk_w, union_mask, union_ids, union_count, offsets, perm};
  return do_pair(L, h, K, y, o, false, false, (cudaStream_t)stream);
}

extern "C" dx_status moe_verify_block_residual(dx_layer* L, const float* h_in, float* h_out, int32_t K,
                                               int32_t* topk_ids, float* topk_w, uint64_t* union_mask,
                                               int32_t* union_ids, int32_t* union_count, int32_t* offsets,
                                               int32_t* perm, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  RouteOut o{topk_ids, topk_w, union_mask, union_ids, union_count, offsets, perm};
  return do_pair(L, h_in, K, h_out, o, false, true, st);
}

// ---- layers whose routed experts come through an expert cache (Sec. 3.5, Algorithm 1) ------------------------
int dx_cache_slot_of(const dx_cache* c, int layer, int expert);
int dx_cache_slots(const dx_cache* c);

// The one round trip on-demand loading needs (the routing decision is made on the device, the copies are issued by
// the host): the routing kernel itself writes what the host needs into page-locked host memory (a device -> host copy
// behind it costs ~10 us of copy-engine set-up for a few ten bytes), and the host waits for the stream.
static dx_status wait_for_routing(dx_ctx* ctx, cudaStream_t st) {
  DX_CUDA(ctx, cudaStreamSynchronize(st));
  return DX_OK;
}

extern "C" dx_status moe_verify_block_cached(dx_layer* L, const float* h, int32_t K, float* y, int32_t residual,
                                             int32_t* topk_ids, float* topk_w, uint64_t* union_mask,
                                             int32_t* union_ids, int32_t* union_count, int32_t* offsets,
                                             int32_t* perm, int32_t* host_union_ids, int32_t* host_union_count,
                                             void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  if (!L->cache) return DX_ERR_INVALID_ARG;
  dx_ctx* ctx = L->ctx;
  dx_cache* c = L->cache;
  cudaStream_t st = (cudaStream_t)stream;
  const int E = L->desc.n_experts;
  // the union goes to the context's scratch if the caller does not want it, and from there to the host
  int32_t* uid = union_ids ? union_ids : ctx->union_dev;
  int32_t* ucnt = union_count ? union_count : ctx->union_dev + DX_MAX_E;
  RouteOut o{topk_ids, topk_w, union_mask, uid, ucnt, offsets, perm};
  dx_status s = do_route(L, h, K, y, o, false, residual != 0, st, 1, true, false, false, true);
  if (s != DX_OK) return s;
  const int cap = E < K * L->desc.top_k ? E : K * L->desc.top_k;
  s = wait_for_routing(ctx, st);
  if (s != DX_OK) return s;
  const int n = ctx->union_host[DX_MAX_E];
  if (n < 0 || n > cap) return DX_ERR_CUDA;
  if (host_union_count) *host_union_count = n;
  if (host_union_ids)
    for (int i = 0; i < n; ++i) host_union_ids[i] = ctx->union_host[i];
  // Waves of at most S experts: the ones the cache already holds (landed or in flight) first, so that no load of
  // this block can evict them before they are used, then the missing ones in ascending id order.
  const int S = dx_cache_slots(c);
  int32_t order[DX_MAX_E];
  int m = 0;
  for (int i = 0; i < n; ++i)
    if (dx_cache_slot_of(c, L->cache_layer, ctx->union_host[i]) >= 0) order[m++] = ctx->union_host[i];
  for (int i = 0; i < n; ++i)
    if (dx_cache_slot_of(c, L->cache_layer, ctx->union_host[i]) < 0) order[m++] = ctx->union_host[i];
  int first = 0;
  do {
    const int cnt = n - first < S ? n - first : S;
    unsigned long long subset[DX_MAX_E / 64] = {};
    for (int i = 0; i < cnt; ++i) subset[order[first + i] >> 6] |= 1ull << (order[first + i] & 63);
    s = expert_cache_stage(c, L->cache_layer, order + first, cnt, stream);
    if (s != DX_OK) return s;
    s = do_experts(L, h, K, y, false, residual != 0, st, 0, -1, first == 0, false, false, subset);
    if (s != DX_OK) return s;
    first += cnt;
  } while (first < n);
  return DX_OK;
}

extern "C" dx_status moe_draft_step_cached(dx_layer* L, const float* h, float* y, int32_t residual,
                                           int32_t* topk_ids, float* topk_w, int32_t* host_topk_ids, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  if (!L->cache) return DX_ERR_INVALID_ARG;
  dx_ctx* ctx = L->ctx;
  cudaStream_t st = (cudaStream_t)stream;
  const int k = L->desc.top_k;
  int32_t* ids = topk_ids ? topk_ids : ctx->union_dev + DX_MAX_E + 1;
  RouteOut o{ids, topk_w, nullptr, nullptr, nullptr, nullptr, nullptr};
  int32_t* host = ctx->union_host + DX_MAX_E + 1;
  dx_status s;
  const int dt = L->desc.weight_dtype;
  if ((dt == DX_DTYPE_BF16 || dt == DX_DTYPE_Q4) && dx_cache_layer_quiet(L->cache, L->cache_layer)) {
    // Most selections are of experts the cache already holds, so -- while none of the layer's copies is in flight:
    // otherwise the stream would have to wait for all of them, not just for the one it may need -- the expert kernel
    // is launched beside the routing kernel, as for a resident layer, before the host knows the selection: the blob
    // table is first brought up to date (it then names exactly what the cache holds), the kernel leaves a routed
    // expert out if the table has no blob for it, and only in that case the expert is loaded and evaluated by a
    // second launch.  The cache sees the same calls in the same order either way.
    s = dx_cache_prepare_layer(L->cache, L->cache_layer, st);
    if (s != DX_OK) return s;
    s = do_route(L, h, 1, y, o, true, residual != 0, st, 1, true, true, false, true);
    if (s != DX_OK) return s;
    s = do_experts(L, h, 1, y, true, residual != 0, st, 0, -1, true, true, false, nullptr, true);
    if (s != DX_OK) { cudaMemsetAsync(ctx->handover, 0, 4 * sizeof(unsigned int), st); return s; }
    s = wait_for_routing(ctx, st);
    if (s != DX_OK) return s;
    if (host_topk_ids)
      for (int j = 0; j < k; ++j) host_topk_ids[j] = host[j];
    const int32_t e1 = host[0];
    if (e1 < 0 || e1 >= L->desc.n_experts) return DX_ERR_CUDA;
    const bool was_resident = dx_cache_slot_of(L->cache, L->cache_layer, e1) >= 0;
    s = expert_cache_stage(L->cache, L->cache_layer, &e1, 1, stream);   // the bookkeeping of a hit, or the load
    if (s != DX_OK || was_resident) return s;
    return do_experts(L, h, 1, y, true, residual != 0, st, 0, -1, false);   // the routed expert alone, now that it is there
  }
  s = do_route(L, h, 1, y, o, true, residual != 0, st, 1, true, false, false, true);
  if (s != DX_OK) return s;
  s = wait_for_routing(ctx, st);
  if (s != DX_OK) return s;
  if (host_topk_ids)
    for (int j = 0; j < k; ++j) host_topk_ids[j] = host[j];
  const int32_t e1 = host[0];
  s = expert_cache_stage(L->cache, L->cache_layer, &e1, 1, stream);   // hit, in flight (waited for) or on demand
  if (s != DX_OK) return s;
  return do_experts(L, h, 1, y, true, residual != 0, st);
}

// ---- exercising the bounded waits without a fault -------------------------------------------------------------
extern "C" dx_status dx_selftest_wait_expiry(dx_layer* L, const float* h, int32_t K, float* y, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  dx_ctx* ctx = L->ctx;
  if (L->desc.weight_dtype == DX_DTYPE_FP32) return DX_ERR_UNSUPPORTED;   // the fp32 kernels have no hand-over
  if (ctx->wait_limit > (1u << 16)) return DX_ERR_INVALID_ARG;            // keep the give-up short: set a limit first
  cudaStream_t st = (cudaStream_t)stream;
  // hand-over words as a routing kernel leaves them before it publishes anything, and then no routing kernel
  DX_CUDA(ctx, cudaMemsetAsync(ctx->handover, 0, 4 * sizeof(unsigned int), st));
  DX_CUDA(ctx, cudaMemsetAsync(ctx->work, 0, sizeof(DxWork), st));
  return do_experts(L, h, K, y, false, false, st, 0, -1, true, true);
}

// ---- draft stack: Eq. 5 through a whole stack of layers in one persistent kernel -----------------------------
extern "C" dx_status dx_stack_create(dx_ctx* ctx, dx_layer* const* layers, int32_t n_layers, dx_stack** out) {
  if (!ctx || !layers || !out) return DX_ERR_INVALID_ARG;
  *out = nullptr;
  if (n_layers < 1 || n_layers > 1024) return DX_ERR_UNSUPPORTED;
  for (int l = 0; l < n_layers; ++l) {
    dx_layer* L = layers[l];
    if (!L || L->ctx != ctx) return DX_ERR_INVALID_ARG;
    const dx_layer_desc &d = L->desc, &d0 = layers[0]->desc;
    if ((d.weight_dtype != DX_DTYPE_BF16 && d.weight_dtype != DX_DTYPE_Q4) || L->cache)
      return DX_ERR_UNSUPPORTED;   // resident bf16 / 4-bit experts in the streaming layout only
    if (d.weight_dtype != d0.weight_dtype) return DX_ERR_SHAPE;
    if (d.hidden != d0.hidden || d.n_experts != d0.n_experts || d.top_k != d0.top_k || d.inter != d0.inter ||
        d.n_shared != d0.n_shared || d.shared_inter != d0.shared_inter || d.draft_inter != d0.draft_inter ||
        d.score_fn != d0.score_fn || d.norm_topk != d0.norm_topk || d.routed_scale != d0.routed_scale)
      return DX_ERR_SHAPE;
    if (!L->W_r) return DX_ERR_NOT_RESIDENT;
  }
  dx_stack* s = new (std::nothrow) dx_stack();
  if (!s) return DX_ERR_OOM;
  s->ctx = ctx;
  s->n_layers = n_layers;
  s->layers = new (std::nothrow) dx_layer*[n_layers];
  s->desc_host = new (std::nothrow) DxStackLayer[n_layers]();
  s->desc_dev = nullptr; s->scratch = nullptr;
  if (!s->layers || !s->desc_host) { delete[] s->layers; delete[] s->desc_host; delete s; return DX_ERR_OOM; }
  for (int l = 0; l < n_layers; ++l) s->layers[l] = layers[l];
  const dx_layer_desc& d = layers[0]->desc;
  cudaError_t e = cudaMalloc(&s->desc_dev, sizeof(DxStackLayer) * n_layers);
  s->zword_off = sizeof(float) * (size_t)n_layers * DX_STACK_COPIES * d.hidden;
  s->sync_off = s->zword_off + sizeof(unsigned long long) * (size_t)n_layers * d.n_experts;
  s->scratch_bytes = s->sync_off + sizeof(unsigned int) * n_layers;
  if (e == cudaSuccess) e = cudaMalloc(&s->scratch, s->scratch_bytes);
  if (e != cudaSuccess) {
    ctx->last_cuda = e;
    dx_stack_destroy(s);
    return e == cudaErrorMemoryAllocation ? DX_ERR_OOM : DX_ERR_CUDA;
  }
  *out = s;
  return DX_OK;
}

extern "C" dx_status dx_stack_destroy(dx_stack* s) {
  if (!s) return DX_ERR_INVALID_ARG;
  cudaFree(s->desc_dev);
  cudaFree(s->scratch);
  delete[] s->layers;
  delete[] s->desc_host;
  delete s;
  return DX_OK;
}

extern "C" dx_status moe_draft_stack(dx_stack* s, const float* h_in, float* h_out, int32_t* topk_ids, float* topk_w,
                                     void* stream) {
  if (!s || !h_in || !h_out || h_in == h_out) return DX_ERR_INVALID_ARG;
  if (((uintptr_t)h_in) % 16 || ((uintptr_t)h_out) % 16) return DX_ERR_INVALID_ARG;
  dx_ctx* ctx = s->ctx;
  cudaStream_t st = (cudaStream_t)stream;
  const dx_layer_desc& d = s->layers[0]->desc;
  // every expert of every layer has to be resident, and the layers' tables and the descriptors up to date
  bool changed = false;
  for (int l = 0; l < s->n_layers; ++l) {
    dx_layer* L = s->layers[l];
    for (int i = 0; i < L->table_len; ++i)
      if (!L->table_host[i] && !(i == d.n_shared && d.draft_inter == 0)) return DX_ERR_NOT_RESIDENT;
    dx_status u = upload_table(L, st);
    if (u != DX_OK) return u;
    DxStackLayer now{};
    now.table = L->table_dev;
    now.W_r = L->W_r;
    now.bias = L->bias;
    now.gamma = L->desc.draft_gamma;
    DxStackLayer& have = s->desc_host[l];
    if (have.table != now.table || have.W_r != now.W_r || have.bias != now.bias || have.gamma != now.gamma) {
      have = now;
      changed = true;
    }
  }
  // (the source outlives the copy: it belongs to the stack)
  cudaError_t e = cudaSuccess;
  if (changed)
    e = cudaMemcpyAsync(s->desc_dev, s->desc_host, sizeof(DxStackLayer) * s->n_layers, cudaMemcpyHostToDevice, st);
  if (e == cudaSuccess) e = cudaMemsetAsync(s->scratch, 0, s->scratch_bytes, st);
  DX_CUDA(ctx, e);
  DxStackParams p{};
  p.layers = s->desc_dev;
  p.n_layers = s->n_layers;
  p.h_in = h_in;
  p.h_out = h_out;
  p.delta = reinterpret_cast<float*>(s->scratch);
  p.zword = reinterpret_cast<unsigned long long*>(s->scratch + s->zword_off);
  p.sync = reinterpret_cast<unsigned int*>(s->scratch + s->sync_off);
  p.topk_ids = topk_ids;
  p.topk_w = topk_w;
  p.dev_status = ctx->dev_status;
  p.H = d.hidden; p.E = d.n_experts; p.k = d.top_k; p.score_fn = d.score_fn; p.norm_topk = d.norm_topk;
  p.scale = d.routed_scale;
  p.n_shared = d.n_shared;
  p.shared_tiles = d.n_shared ? d.shared_inter / DX_TILE_I : 0;
  p.draft_tiles = d.draft_inter / DX_TILE_I;
  p.routed_tiles = d.inter / DX_TILE_I;
  p.q4 = d.weight_dtype == DX_DTYPE_Q4 ? 1 : 0;
  p.wait_limit = ctx->wait_limit;
  DX_CUDA(ctx, dx_launch_draft_stack(ctx, p, st));
  ctx->launches++;
  return DX_OK;
}

// ---- evaluation terms of Sec. 3.3 (no training involved) -----------------------------------------------------
extern "C" dx_status moe_missing_residual(dx_layer* L, const float* h, int32_t K, float* m, int32_t* topk_ids,
                                          float* topk_w, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  cudaStream_t st = (cudaStream_t)stream;
  RouteOut o{topk_ids, topk_w, nullptr, nullptr, nullptr, nullptr, nullptr};
  // Eq. 6 is the routed sum of Eq. 4 without each row's first selected expert: same kernels, that pair's weight
  // set to zero (and its expert left out of the union unless another pair selects it), shared experts skipped
  dx_status s = do_route(L, h, K, m, o, false, false, st, 1, true, false, true);
  if (s != DX_OK) return s;
  return do_experts(L, h, K, m, false, false, st, 0, -1, false);
}

extern "C" dx_status moe_draft_expert_term(dx_layer* L, const float* h, int32_t K, float* out, void* stream) {
  if (!L) return DX_ERR_INVALID_ARG;
  if (L->desc.draft_inter <= 0) return DX_ERR_UNSUPPORTED;
  cudaStream_t st = (cudaStream_t)stream;
  RouteOut o{nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr};
  // gamma * E^d(h_t) for K rows: the drafter's kernels with no routed group and the shared experts skipped
  dx_status s = do_route(L, h, K, out, o, true, false, st, 0, true);
  if (s != DX_OK) return s;
  return do_experts(L, h, K, out, true, false, st, 0, -1, true, false, true);
}

extern "C" dx_status moe_router_agreement(dx_layer* L, const float* h_star, const float* h_draft, int32_t K, float* kl,
                                          int32_t* agree, void* stream) {
  if (!L || !h_star || !h_draft || (!kl && !agree)) return DX_ERR_INVALID_ARG;
  if (K < 1) return DX_ERR_SHAPE;
  if (!L->W_r) return DX_ERR_NOT_RESIDENT;
  DX_CUDA(L->ctx, dx_launch_router_agreement(L, h_star, h_draft, K, kl, agree, (cudaStream_t)stream));
  L->ctx->launches++;
  return DX_OK;
}

extern "C" dx_status dx_squared_error(dx_ctx* ctx, const float* a, const float* b, int64_t n, float* out,
                                      void* stream) {
  if (!ctx || !a || !b || !out) return DX_ERR_INVALID_ARG;
  if (n < 0) return DX_ERR_SHAPE;
  DX_CUDA(ctx, dx_launch_squared_error(a, b, (long long)n, out, (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

extern "C" dx_status spec_accept(dx_ctx* ctx, const float* h, int32_t M, const void* W_lm, int32_t V, int32_t H,
                                 int32_t w_dtype, const int32_t* draft, int32_t K, int32_t rms_norm, int32_t* target,
                                 int32_t* n_accept, int32_t* next_token, void* stream) {
  if (!ctx || !h || !W_lm || !target || !n_accept || !next_token) return DX_ERR_INVALID_ARG;
  if (K > 0 && !draft) return DX_ERR_INVALID_ARG;
  if (M < 1 || V < 1 || K < 0) return DX_ERR_SHAPE;
  if (w_dtype != DX_DTYPE_FP32 && w_dtype != DX_DTYPE_BF16) return DX_ERR_INVALID_ARG;
  if (M > DX_MAX_M || K > DX_MAX_K || H <= 0 || H > DX_MAX_H || H % 256) return DX_ERR_UNSUPPORTED;
  if (((uintptr_t)h) % 16 || ((uintptr_t)W_lm) % 16) return DX_ERR_INVALID_ARG;
  if (w_dtype == DX_DTYPE_BF16) {
    const size_t smem = (size_t)((M + 7) / 8) * H * 32;
    if (smem > (size_t)ctx->smem_optin) return DX_ERR_UNSUPPORTED;
  }
  DX_CUDA(ctx, dx_launch_accept(ctx, h, M, W_lm, V, H, w_dtype, draft, K, rms_norm, target, n_accept, next_token,
                                nullptr, (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

extern "C" dx_status spec_draft_token(dx_ctx* ctx, const float* h, int32_t M, const void* W_lm, int32_t V, int32_t H,
                                      int32_t w_dtype, int32_t rms_norm, int32_t* token, float* confidence,
                                      void* stream) {
  if (!ctx || !h || !W_lm || !token || !confidence) return DX_ERR_INVALID_ARG;
  if (M < 1 || V < 1) return DX_ERR_SHAPE;
  if (w_dtype != DX_DTYPE_FP32 && w_dtype != DX_DTYPE_BF16) return DX_ERR_INVALID_ARG;
  if (M > DX_MAX_M || H <= 0 || H > DX_MAX_H || H % 256) return DX_ERR_UNSUPPORTED;
  if (((uintptr_t)h) % 16 || ((uintptr_t)W_lm) % 16) return DX_ERR_INVALID_ARG;
  if (w_dtype == DX_DTYPE_BF16 && (size_t)((M + 7) / 8) * H * 32 > (size_t)ctx->smem_optin) return DX_ERR_UNSUPPORTED;
  DX_CUDA(ctx, dx_launch_accept(ctx, h, M, W_lm, V, H, w_dtype, nullptr, 0, rms_norm, token, ctx->scratch_i32,
                                ctx->scratch_i32 + 1, confidence, (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

// ---- whole batches of tokens ------------------------------------------------------------------------------------
namespace {

// the context's GPU for the length of a call
struct DeviceScope {
  int before = -1;
  cudaError_t err;
  explicit DeviceScope(int device) {
    err = cudaGetDevice(&before);
    if (err == cudaSuccess && before != device) err = cudaSetDevice(device);
    if (err == cudaSuccess && before == device) before = -1;
  }
  ~DeviceScope() {
    if (before >= 0) (void)cudaSetDevice(before);
  }
};

dx_status check_rows(const void* p, int32_t dtype, int32_t N, int32_t len, int64_t ld) {
  if (dtype != DX_DTYPE_FP32 && dtype != DX_DTYPE_BF16) return DX_ERR_INVALID_ARG;
  if (N < 0 || len < 1 || ld < len) return DX_ERR_SHAPE;
  const int64_t elem = dtype == DX_DTYPE_FP32 ? 4 : 2;
  if (N > 0 && (!p || (uintptr_t)p % elem)) return DX_ERR_INVALID_ARG;
  // (the last row's end must be addressable)
  if (ld > (INT64_MAX / 8) / (N > 0 ? N : 1)) return DX_ERR_SHAPE;
  return DX_OK;
}
// [N rows of len elements, ld apart] against another such matrix of the same element size
bool rows_overlap(const void* a, int64_t ld_a, const void* b, int64_t ld_b, int32_t N, int32_t len, int64_t elem) {
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  const uintptr_t a1 = a0 + (uintptr_t)(((int64_t)(N - 1) * ld_a + len) * elem);
  const uintptr_t b1 = b0 + (uintptr_t)(((int64_t)(N - 1) * ld_b + len) * elem);
  if (!(a0 < b1 && b0 < a1)) return false;
  if (ld_a != ld_b || N == 1) return true;
  // one pitch: rows of the one may lie between the rows of the other
  const int64_t pitch = ld_a * elem, row = (int64_t)len * elem;
  const int64_t d = (((int64_t)(b0 - a0)) % pitch + pitch) % pitch;
  return d < row || d > pitch - row;
}
bool temperature_ok(float t) { return t >= 1e-4f && t <= 1e4f; }

dx_status check_route(const dx_route_desc* d, bool groups) {
  if (!d) return DX_ERR_INVALID_ARG;
  if (d->score_fn != DX_SCORE_SOFTMAX && d->score_fn != DX_SCORE_SIGMOID) return DX_ERR_INVALID_ARG;
  if (d->n_experts < 1 || d->top_k < 1 || d->top_k > d->n_experts) return DX_ERR_SHAPE;
  if (d->n_experts > DX_MAX_E || d->top_k > DX_MAX_TOPK) return DX_ERR_UNSUPPORTED;
  if (!groups) return DX_OK;
  if (d->group_score != DX_GROUP_MAX && d->group_score != DX_GROUP_TOP2) return DX_ERR_INVALID_ARG;
  if (d->n_groups < 1 || d->n_experts % d->n_groups || d->topk_groups < 1 || d->topk_groups > d->n_groups)
    return DX_ERR_SHAPE;
  if (d->topk_groups * (d->n_experts / d->n_groups) < d->top_k) return DX_ERR_SHAPE;
  if (d->n_groups > DX_MAX_GROUPS) return DX_ERR_UNSUPPORTED;
  return DX_OK;
}

}  // namespace

extern "C" dx_status spec_token_logprobs(dx_ctx* ctx, const void* logits, int32_t dtype, int32_t N, int32_t V, int64_t ld,
                                         const int32_t* tokens, float temperature, int32_t n_top, float* logprob,
                                         float* entropy, int32_t* top_ids, float* top_logprobs, void* stream) {
  if (!ctx || !temperature_ok(temperature)) return DX_ERR_INVALID_ARG;
  dx_status s = check_rows(logits, dtype, N, V, ld);
  if (s != DX_OK) return s;
  if (n_top < 0 || n_top > V) return DX_ERR_SHAPE;
  if (n_top > DX_MAX_TOP) return DX_ERR_UNSUPPORTED;
  if (N == 0) return DX_OK;
  if ((tokens == nullptr) != (logprob == nullptr)) return DX_ERR_INVALID_ARG;
  if (n_top > 0 && (!top_ids || !top_logprobs)) return DX_ERR_INVALID_ARG;
  if (!logprob && !entropy && n_top == 0) return DX_ERR_INVALID_ARG;
  DeviceScope scope(ctx->device);
  DX_CUDA(ctx, scope.err);
  DX_CUDA(ctx, dx_launch_logprobs(ctx, logits, dtype, N, V, (long long)ld, tokens, temperature, n_top, logprob, entropy,
                                  top_ids, top_logprobs, (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

extern "C" dx_status spec_distill_topk(dx_ctx* ctx, const void* logits, int32_t dtype, int32_t N, int32_t V, int64_t ld,
                                       const int32_t* teacher_ids, const float* teacher_logprobs, int32_t k, int32_t tail,
                                       float temperature, const float* row_weight, float* loss, void* dlogits,
                                       int64_t ld_d, void* stream) {
  if (!ctx || !temperature_ok(temperature) || (tail != 0 && tail != 1)) return DX_ERR_INVALID_ARG;
  dx_status s = check_rows(logits, dtype, N, V, ld);
  if (s != DX_OK) return s;
  if (k < 1) return DX_ERR_SHAPE;
  if (k > DX_MAX_TEACHER || N > DX_MAX_ROWS) return DX_ERR_UNSUPPORTED;
  const int64_t elem = dtype == DX_DTYPE_FP32 ? 4 : 2;
  if ((uint64_t)V * (uint64_t)elem > (uint64_t)dx_distill_max_row_bytes(ctx)) return DX_ERR_UNSUPPORTED;
  if (dlogits) {
    s = check_rows(dlogits, dtype, N, V, ld_d);
    if (s != DX_OK) return s;
  }
  if (N == 0) return DX_OK;
  if (!teacher_ids || !teacher_logprobs || (!loss && !dlogits)) return DX_ERR_INVALID_ARG;
  if (dlogits && !(dlogits == logits && ld == ld_d) && rows_overlap(logits, ld, dlogits, ld_d, N, V, elem))
    return DX_ERR_INVALID_ARG;
  DeviceScope scope(ctx->device);
  DX_CUDA(ctx, scope.err);
  DX_CUDA(ctx, dx_launch_distill(ctx, logits, dtype, N, V, (long long)ld, teacher_ids, teacher_logprobs, k, tail,
                                 temperature, row_weight, loss, dlogits, (long long)ld_d, (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

extern "C" dx_status moe_route_tokens(dx_ctx* ctx, const dx_route_desc* desc, const void* logits, int32_t dtype, int32_t N,
                                      int64_t ld, const float* select_bias, int32_t* topk_ids, float* topk_w,
                                      int32_t* offsets, int32_t* perm, void* stream) {
  if (!ctx) return DX_ERR_INVALID_ARG;
  dx_status s = check_route(desc, true);
  if (s != DX_OK) return s;
  s = check_rows(logits, dtype, N, desc->n_experts, ld);
  if (s != DX_OK) return s;
  if ((int64_t)N * desc->top_k > INT32_MAX) return DX_ERR_UNSUPPORTED;
  if (N > 0 && (!topk_ids || !topk_w || (offsets == nullptr) != (perm == nullptr))) return DX_ERR_INVALID_ARG;
  DeviceScope scope(ctx->device);
  DX_CUDA(ctx, scope.err);
  if (N == 0) {   // no pairs: every expert's run is empty
    if (offsets)
      DX_CUDA(ctx, cudaMemsetAsync(offsets, 0, sizeof(int32_t) * (desc->n_experts + 1), (cudaStream_t)stream));
    return DX_OK;
  }
  int n = 0;
  DX_CUDA(ctx, dx_launch_batch_route(ctx, *desc, logits, dtype, N, (long long)ld, select_bias, topk_ids, topk_w, offsets,
                                     perm, (cudaStream_t)stream, &n));
  ctx->launches += n;
  return DX_OK;
}

extern "C" dx_status moe_route_tokens_backward(dx_ctx* ctx, const dx_route_desc* desc, const void* logits, int32_t dtype,
                                               int32_t N, int64_t ld, const int32_t* topk_ids, const float* d_topk_w,
                                               void* d_logits, int64_t ld_d, void* stream) {
  if (!ctx) return DX_ERR_INVALID_ARG;
  dx_status s = check_route(desc, false);
  if (s != DX_OK) return s;
  s = check_rows(logits, dtype, N, desc->n_experts, ld);
  if (s == DX_OK) s = check_rows(d_logits, dtype, N, desc->n_experts, ld_d);
  if (s != DX_OK) return s;
  if (N == 0) return DX_OK;
  if (!topk_ids || !d_topk_w) return DX_ERR_INVALID_ARG;
  if (rows_overlap(logits, ld, d_logits, ld_d, N, desc->n_experts, dtype == DX_DTYPE_FP32 ? 4 : 2))
    return DX_ERR_INVALID_ARG;
  DeviceScope scope(ctx->device);
  DX_CUDA(ctx, scope.err);
  DX_CUDA(ctx, dx_launch_route_grad(ctx, *desc, logits, dtype, N, (long long)ld, topk_ids, d_topk_w, d_logits,
                                    (long long)ld_d, (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

// ---- whole batches of tokens: the experts, their combination, the loss -------------------------------------------------
namespace {

constexpr int32_t kMostRows = INT32_MAX - 2048;      // (what 32 bits count, less the largest step that is added to it)

// a matrix of the tensor-core products: address, pitch and width in whole 16-byte vectors of bf16 (8 elements)
dx_status check_matrix(const void* p, int64_t rows, int64_t cols, int64_t ld) {
  if (rows < 0 || cols < 1 || ld < cols) return DX_ERR_SHAPE;
  if (cols % 8 || ld % 8) return DX_ERR_UNSUPPORTED;
  if (rows > INT32_MAX || ld > (int64_t(1) << 38) || (rows > 0 && ld > (INT64_MAX / 16) / rows)) return DX_ERR_SHAPE;
  if (rows * (ld / 8) > UINT32_MAX) return DX_ERR_UNSUPPORTED;      // (a row's place is counted in 16-byte pieces of bf16)
  if (rows > 0 && (!p || (uintptr_t)p % 16)) return DX_ERR_INVALID_ARG;
  return DX_OK;
}
struct Range {
  uintptr_t lo, hi;
};
Range rows_range(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t elem) {
  const uintptr_t lo = (uintptr_t)p;
  return {lo, rows > 0 && p ? lo + (uintptr_t)(((rows - 1) * ld + cols) * elem) : lo};
}
bool overlap(Range a, Range b) { return a.lo < b.hi && b.lo < a.hi && a.lo < a.hi && b.lo < b.hi; }

dx_status check_groups(const dx_grouped_desc* d, const void* w) {
  if (!d || !w || (uintptr_t)w % 16) return DX_ERR_INVALID_ARG;
  if (d->n_groups < 1 || d->n_rows < 0 || d->n < 1 || d->k < 1 || d->ld_w < d->k) return DX_ERR_SHAPE;
  if (d->ld_w > (int64_t(1) << 36) || d->stride_w < (int64_t)(d->n - 1) * d->ld_w + d->k ||
      d->stride_w > (int64_t(1) << 38)) return DX_ERR_SHAPE;
  if (d->n_groups > DX_MAX_E || d->n % 8 || d->k % 8 || d->ld_w % 8 || d->stride_w % 8) return DX_ERR_UNSUPPORTED;
  // (rows, columns and tiles are numbered in 32 bits, up to a tile behind the last)
  if (d->n_rows > kMostRows || d->n > kMostRows || d->k > kMostRows) return DX_ERR_UNSUPPORTED;
  const int64_t a = (d->n + 63) / 64, b = (d->k + 63) / 64, rows = d->n_rows / 64 + d->n_groups;
  const int64_t most = a > b ? a : b;
  if (a * b > INT32_MAX / d->n_groups || rows * most > INT32_MAX) return DX_ERR_UNSUPPORTED;
  return DX_OK;
}
Range groups_range(const dx_grouped_desc* d, const void* w, int64_t elem) {
  return rows_range(w, d->n_groups, (int64_t)(d->n - 1) * d->ld_w + d->k, d->stride_w, elem);
}
bool dense_dtype(int32_t t) { return t == DX_DTYPE_FP32 || t == DX_DTYPE_BF16; }

}  // namespace

extern "C" dx_status moe_grouped_mm(dx_ctx* ctx, const dx_grouped_desc* desc, const void* x, int32_t x_rows, int64_t ldx,
                                    const void* w, int32_t transposed, const int32_t* offsets, const int32_t* gather,
                                    int32_t gather_div, const int32_t* scatter, void* y, int32_t y_dtype, int32_t y_rows,
                                    int64_t ldy, void* stream) {
  if (!ctx || (transposed != 0 && transposed != 1) || !dense_dtype(y_dtype) || gather_div < 1) return DX_ERR_INVALID_ARG;
  dx_status s = check_groups(desc, w);
  if (s != DX_OK) return s;
  const int n_in = transposed ? desc->n : desc->k, n_out = transposed ? desc->k : desc->n;
  s = check_matrix(x, x_rows, n_in, ldx);
  if (s == DX_OK) s = check_matrix(y, y_rows, n_out, ldy);
  if (s != DX_OK) return s;
  if (desc->n_rows == 0) return DX_OK;
  if (!offsets) return DX_ERR_INVALID_ARG;
  if (x_rows < (gather ? 1 : desc->n_rows) || y_rows < (scatter ? 1 : desc->n_rows)) return DX_ERR_SHAPE;
  const Range out = rows_range(y, y_rows, n_out, ldy, y_dtype == DX_DTYPE_FP32 ? 4 : 2);
  if (overlap(out, rows_range(x, x_rows, n_in, ldx, 2)) || overlap(out, groups_range(desc, w, 2))) return DX_ERR_INVALID_ARG;
  DeviceScope scope(ctx->device);
  DX_CUDA(ctx, scope.err);
  DxGroupedMm a = {};
  a.x = x; a.x_rows = x_rows; a.ldx = ldx;
  a.w = w; a.n_groups = desc->n_groups; a.n = desc->n; a.k = desc->k; a.ldw = desc->ld_w; a.w_stride = desc->stride_w;
  a.transposed = transposed;
  a.offsets = offsets; a.n_rows = desc->n_rows; a.gather = gather; a.gather_div = gather ? gather_div : 1; a.scatter = scatter;
  a.y = y; a.y_fp32 = y_dtype == DX_DTYPE_FP32; a.y_rows = y_rows; a.ldy = ldy;
  DX_CUDA(ctx, dx_launch_grouped_mm(ctx, a, (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

extern "C" dx_status moe_grouped_mm_dw(dx_ctx* ctx, const dx_grouped_desc* desc, const void* dy, int32_t dy_rows, int64_t ld_dy,
                                       const int32_t* gather_dy, int32_t dy_div, const void* x, int32_t x_rows, int64_t ldx,
                                       const int32_t* gather_x, int32_t x_div, const int32_t* offsets, void* dw,
                                       int32_t dw_dtype, void* stream) {
  if (!ctx || !dense_dtype(dw_dtype) || dy_div < 1 || x_div < 1) return DX_ERR_INVALID_ARG;
  dx_status s = check_groups(desc, dw);
  if (s == DX_OK) s = check_matrix(dy, dy_rows, desc->n, ld_dy);
  if (s == DX_OK) s = check_matrix(x, x_rows, desc->k, ldx);
  if (s != DX_OK) return s;
  const int64_t elem = dw_dtype == DX_DTYPE_FP32 ? 4 : 2;
  const Range out = groups_range(desc, dw, elem);
  if (overlap(out, rows_range(x, x_rows, desc->k, ldx, 2)) || overlap(out, rows_range(dy, dy_rows, desc->n, ld_dy, 2)))
    return DX_ERR_INVALID_ARG;
  if (desc->n_rows > 0) {
    if (!offsets) return DX_ERR_INVALID_ARG;
    if (dy_rows < (gather_dy ? 1 : desc->n_rows) || x_rows < (gather_x ? 1 : desc->n_rows)) return DX_ERR_SHAPE;
  }
  DeviceScope scope(ctx->device);
  DX_CUDA(ctx, scope.err);
  if (desc->n_rows == 0) {   // every group is empty
    for (int e = 0; e < desc->n_groups; ++e)
      DX_CUDA(ctx, cudaMemset2DAsync(reinterpret_cast<unsigned char*>(dw) + (size_t)e * desc->stride_w * elem,
                                     desc->ld_w * elem, 0, desc->k * elem, desc->n, (cudaStream_t)stream));
    return DX_OK;
  }
  DxGroupedDw a = {};
  a.dy = dy; a.dy_rows = dy_rows; a.ld_dy = ld_dy; a.gather_dy = gather_dy; a.dy_div = dy_div;
  a.x = x; a.x_rows = x_rows; a.ldx = ldx; a.gather_x = gather_x; a.x_div = x_div;
  a.n_groups = desc->n_groups; a.n = desc->n; a.k = desc->k; a.offsets = offsets; a.n_rows = desc->n_rows;
  a.dw = dw; a.dw_fp32 = dw_dtype == DX_DTYPE_FP32; a.ld_dw = desc->ld_w; a.dw_stride = desc->stride_w;
  DX_CUDA(ctx, dx_launch_grouped_dw(ctx, a, (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

extern "C" dx_status moe_grouped_swiglu(dx_ctx* ctx, const dx_grouped_desc* desc, const void* x, int32_t x_rows, int64_t ldx,
                                        const void* w_gate_up, const int32_t* offsets, const int32_t* gather,
                                        int32_t gather_div, void* act, int64_t ld_act, void* gate_up, int64_t ld_gate_up,
                                        void* stream) {
  if (!ctx || gather_div < 1) return DX_ERR_INVALID_ARG;
  dx_status s = check_groups(desc, w_gate_up);
  if (s != DX_OK) return s;
  if (desc->n % 2) return DX_ERR_SHAPE;
  if (desc->n % 16) return DX_ERR_UNSUPPORTED;
  const int n_inter = desc->n / 2, P = desc->n_rows;
  s = check_matrix(x, x_rows, desc->k, ldx);
  if (s == DX_OK) s = check_matrix(act, P, n_inter, ld_act);
  if (s == DX_OK && gate_up) s = check_matrix(gate_up, P, desc->n, ld_gate_up);
  if (s != DX_OK) return s;
  if (P == 0) return DX_OK;
  if (!offsets) return DX_ERR_INVALID_ARG;
  if (x_rows < (gather ? 1 : P)) return DX_ERR_SHAPE;
  const Range in[2] = {rows_range(x, x_rows, desc->k, ldx, 2), groups_range(desc, w_gate_up, 2)};
  const Range out[2] = {rows_range(act, P, n_inter, ld_act, 2), rows_range(gate_up, gate_up ? P : 0, desc->n, ld_gate_up, 2)};
  if (overlap(out[0], out[1])) return DX_ERR_INVALID_ARG;
  for (const Range& o : out)
    for (const Range& i : in)
      if (overlap(o, i)) return DX_ERR_INVALID_ARG;
  DeviceScope scope(ctx->device);
  DX_CUDA(ctx, scope.err);
  DxGroupedMm a = {};
  a.x = x; a.x_rows = x_rows; a.ldx = ldx;
  a.w = w_gate_up; a.n_groups = desc->n_groups; a.n = desc->n; a.k = desc->k; a.ldw = desc->ld_w; a.w_stride = desc->stride_w;
  a.offsets = offsets; a.n_rows = P; a.gather = gather; a.gather_div = gather ? gather_div : 1;
  a.y = act; a.y_rows = P; a.ldy = ld_act;
  DX_CUDA(ctx, dx_launch_grouped_swiglu(ctx, a, gate_up, ld_gate_up, (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

extern "C" dx_status moe_grouped_swiglu_backward_workspace(const dx_grouped_desc* desc, size_t* bytes_out) {
  if (!desc || !bytes_out) return DX_ERR_INVALID_ARG;
  if (desc->n_rows < 0 || desc->k < 1) return DX_ERR_SHAPE;
  *bytes_out = (size_t)dx_swiglu_grad_parts(desc->k) * (size_t)desc->n_rows * sizeof(float);
  return DX_OK;
}

extern "C" dx_status moe_grouped_swiglu_backward(dx_ctx* ctx, const dx_grouped_desc* desc, const void* dy, int32_t dy_rows,
                                                 int64_t ld_dy, const void* w_down, const void* gate_up, int64_t ld_gate_up,
                                                 const float* pair_w, int32_t n_pairs, const int32_t* offsets,
                                                 const int32_t* gather, int32_t gather_div, void* d_gate_up, int64_t ld_d,
                                                 void* act_w, int64_t ld_act, float* d_pair_w, void* workspace,
                                                 size_t workspace_bytes, void* stream) {
  if (!ctx || gather_div < 1) return DX_ERR_INVALID_ARG;
  dx_status s = check_groups(desc, w_down);
  if (s != DX_OK) return s;
  const int n_inter = desc->k, P = desc->n_rows;
  if (n_pairs < 0 || n_inter > INT32_MAX / 2) return DX_ERR_SHAPE;
  s = check_matrix(dy, dy_rows, desc->n, ld_dy);
  if (s == DX_OK) s = check_matrix(gate_up, P, 2 * (int64_t)n_inter, ld_gate_up);
  if (s == DX_OK) s = check_matrix(d_gate_up, P, 2 * (int64_t)n_inter, ld_d);
  if (s == DX_OK) s = check_matrix(act_w, P, n_inter, ld_act);
  if (s != DX_OK) return s;
  if (P == 0) return DX_OK;
  if (!offsets) return DX_ERR_INVALID_ARG;
  if (dy_rows < (gather ? 1 : (P - 1) / gather_div + 1) || n_pairs < (gather ? 1 : P)) return DX_ERR_SHAPE;
  if (d_pair_w) {
    size_t need = 0;
    moe_grouped_swiglu_backward_workspace(desc, &need);
    if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < need) return DX_ERR_INVALID_ARG;
  }
  const Range in[3] = {rows_range(dy, dy_rows, desc->n, ld_dy, 2), groups_range(desc, w_down, 2),
                       rows_range(gate_up, P, 2 * (int64_t)n_inter, ld_gate_up, 2)};
  const Range out[2] = {rows_range(d_gate_up, P, 2 * (int64_t)n_inter, ld_d, 2), rows_range(act_w, P, n_inter, ld_act, 2)};
  if (overlap(out[0], out[1])) return DX_ERR_INVALID_ARG;
  for (const Range& o : out)
    for (const Range& i : in)
      if (overlap(o, i)) return DX_ERR_INVALID_ARG;
  DeviceScope scope(ctx->device);
  DX_CUDA(ctx, scope.err);
  DxGroupedMm a = {};
  a.x = dy; a.x_rows = dy_rows; a.ldx = ld_dy;
  a.w = w_down; a.n_groups = desc->n_groups; a.n = desc->n; a.k = desc->k; a.ldw = desc->ld_w; a.w_stride = desc->stride_w;
  a.offsets = offsets; a.n_rows = P; a.gather = gather; a.gather_div = gather_div;
  a.y = d_gate_up; a.y_rows = P; a.ldy = ld_d;
  int n = 0;
  DX_CUDA(ctx, dx_launch_grouped_swiglu_grad(ctx, a, gate_up, ld_gate_up, pair_w, n_pairs, act_w, ld_act,
                                             reinterpret_cast<float*>(workspace), d_pair_w, (cudaStream_t)stream, &n));
  ctx->launches += n;
  return DX_OK;
}

namespace {
// rows of moe_combine_tokens: 16-byte vectors of eight elements (fp32: two)
dx_status check_combine(const dx_ctx* ctx, int32_t N, int32_t k, int32_t H) {
  if (!ctx) return DX_ERR_INVALID_ARG;
  if (N < 0 || k < 1 || H < 1) return DX_ERR_SHAPE;
  if (k > DX_MAX_TOPK || (int64_t)N * k > kMostRows || H > kMostRows) return DX_ERR_UNSUPPORTED;
  return DX_OK;
}
}  // namespace

extern "C" dx_status moe_combine_tokens(dx_ctx* ctx, const void* z, int32_t z_dtype, int64_t ldz, const float* topk_w,
                                        int32_t N, int32_t top_k, int32_t H, void* y, int32_t y_dtype, int64_t ldy,
                                        void* stream) {
  dx_status s = check_combine(ctx, N, top_k, H);
  if (s != DX_OK) return s;
  if (!dense_dtype(z_dtype) || !dense_dtype(y_dtype)) return DX_ERR_INVALID_ARG;
  s = check_matrix(z, (int64_t)N * top_k, H, ldz);
  if (s == DX_OK) s = check_matrix(y, N, H, ldy);
  if (s != DX_OK) return s;
  if (N == 0) return DX_OK;
  const int z32 = z_dtype == DX_DTYPE_FP32, y32 = y_dtype == DX_DTYPE_FP32;
  if (overlap(rows_range(z, (int64_t)N * top_k, H, ldz, z32 ? 4 : 2), rows_range(y, N, H, ldy, y32 ? 4 : 2)))
    return DX_ERR_INVALID_ARG;
  DeviceScope scope(ctx->device);
  DX_CUDA(ctx, scope.err);
  DX_CUDA(ctx, dx_launch_combine(ctx, z, z32, ldz, topk_w, N, top_k, H, y, y32, ldy, (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

extern "C" dx_status moe_combine_tokens_backward(dx_ctx* ctx, const void* dy, int64_t ld_dy, const void* z, int64_t ldz,
                                                 int32_t dtype, const float* topk_w, int32_t N, int32_t top_k, int32_t H,
                                                 void* dz, int64_t ld_dz, float* d_topk_w, void* stream) {
  dx_status s = check_combine(ctx, N, top_k, H);
  if (s != DX_OK) return s;
  if (!dense_dtype(dtype)) return DX_ERR_INVALID_ARG;
  const int64_t P = (int64_t)N * top_k, elem = dtype == DX_DTYPE_FP32 ? 4 : 2;
  s = check_matrix(dy, N, H, ld_dy);
  if (s == DX_OK && d_topk_w) s = check_matrix(z, P, H, ldz);
  if (s == DX_OK && dz) s = check_matrix(dz, P, H, ld_dz);
  if (s != DX_OK) return s;
  if (N == 0) return DX_OK;
  if (!dz && !d_topk_w) return DX_ERR_INVALID_ARG;
  if (dz && (overlap(rows_range(dz, P, H, ld_dz, elem), rows_range(dy, N, H, ld_dy, elem)) ||
             (d_topk_w && overlap(rows_range(dz, P, H, ld_dz, elem), rows_range(z, P, H, ldz, elem)))))
    return DX_ERR_INVALID_ARG;
  DeviceScope scope(ctx->device);
  DX_CUDA(ctx, scope.err);
  DX_CUDA(ctx, dx_launch_combine_grad(ctx, dy, z, dtype == DX_DTYPE_FP32, ld_dy, ldz, topk_w, N, top_k, H, dz, ld_dz, d_topk_w,
                                      (cudaStream_t)stream));
  ctx->launches++;
  return DX_OK;
}

namespace {
// (tiles, pieces and rows are numbered in 32 bits)
bool head_countable(int32_t N, int32_t V, int32_t H) {
  return ((int64_t)N / 128 + 1) * ((int64_t)V / 256 + 1) <= INT32_MAX && V <= kMostRows && N <= kMostRows && H <= kMostRows;
}
}  // namespace

extern "C" dx_status spec_head_loss_workspace(dx_ctx* ctx, int32_t N, int32_t V, int32_t H, int32_t grad, size_t* least_out,
                                              size_t* best_out) {
  if (!ctx || !least_out || !best_out) return DX_ERR_INVALID_ARG;
  if (N < 0 || V < 1 || H < 1) return DX_ERR_SHAPE;
  if (!head_countable(N, V, H)) return DX_ERR_UNSUPPORTED;
  *least_out = *best_out = 0;
  if (N > 0) dx_head_loss_workspace(ctx->sm_count, N, V, H, grad, least_out, best_out);
  return DX_OK;
}

extern "C" dx_status spec_head_loss(dx_ctx* ctx, const void* h, int32_t N, int64_t ldh, const void* W_lm, int32_t V, int64_t ldw,
                                    int32_t H, const int32_t* targets, const float* row_weight, float* loss, void* dh,
                                    int64_t ld_dh, void* dW, int64_t ld_dW, void* workspace, size_t workspace_bytes,
                                    void* stream) {
  if (!ctx) return DX_ERR_INVALID_ARG;
  if (V < 1) return DX_ERR_SHAPE;
  dx_status s = check_matrix(h, N, H, ldh);
  if (s == DX_OK) s = check_matrix(W_lm, V, H, ldw);
  if (s == DX_OK && dh) s = check_matrix(dh, N, H, ld_dh);
  if (s == DX_OK && dW) s = check_matrix(dW, V, H, ld_dW);
  if (s != DX_OK) return s;
  if (!head_countable(N, V, H)) return DX_ERR_UNSUPPORTED;
  if (!loss && !dh && !dW) return DX_ERR_INVALID_ARG;
  const Range in[2] = {rows_range(h, N, H, ldh, 2), rows_range(W_lm, V, H, ldw, 2)};
  const Range out[2] = {rows_range(dh, dh ? N : 0, H, ld_dh, 2), rows_range(dW, dW ? V : 0, H, ld_dW, 2)};
  if (overlap(out[0], out[1])) return DX_ERR_INVALID_ARG;
  for (const Range& o : out)
    for (const Range& i : in)
      if (overlap(o, i)) return DX_ERR_INVALID_ARG;
  size_t least = 0, best = 0;
  if (N > 0) {
    dx_head_loss_workspace(ctx->sm_count, N, V, H, dh || dW, &least, &best);
    if (!targets || !workspace || (uintptr_t)workspace % 256 || workspace_bytes < least) return DX_ERR_INVALID_ARG;
  }
  DeviceScope scope(ctx->device);
  DX_CUDA(ctx, scope.err);
  if (N == 0) {
    if (dW) DX_CUDA(ctx, cudaMemset2DAsync(dW, ld_dW * 2, 0, (size_t)H * 2, V, (cudaStream_t)stream));
    return DX_OK;
  }
  DxHeadLoss a = {};
  a.h = h; a.ldh = ldh; a.W = W_lm; a.ldw = ldw; a.N = N; a.V = V; a.H = H;
  a.targets = targets; a.row_weight = row_weight; a.loss = loss;
  a.dh = dh; a.ld_dh = ld_dh; a.dW = dW; a.ld_dW = ld_dW;
  a.workspace = workspace; a.workspace_bytes = workspace_bytes < best ? workspace_bytes : best;
  int n = 0;
  DX_CUDA(ctx, dx_launch_head_loss(ctx, a, (cudaStream_t)stream, &n));
  ctx->launches += n;
  return DX_OK;
}
