// C ABI of the verify/arbitrate round: host-side validation, workspace
// sizing, the device error word and dispatch to the kernel launchers.
#include <cuda.h>
#include <math.h>
#include <stdint.h>

#include <atomic>
#include <mutex>

#include "../../include/cospec.h"
#include "cospec_internal.h"

namespace cospec {

namespace {
__device__ int g_error_word;   // one per device context; bits COSPEC_DEVERR_*

constexpr int MAX_DEV = 64;
// Lazily filled per-device values; a race between host threads only
// repeats the same query.
std::atomic<int> g_num_sms[MAX_DEV];
std::atomic<int*> g_err_ptr[MAX_DEV];
std::mutex g_limits_mutex;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

// The calling thread's device, with its primary context made current the
// first time (a host thread that has made no CUDA call yet has no current
// context, and the tensor-map encoder needs one).
int current_device() {
  static thread_local int bound = -1;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return -1;
  if (bound != dev) {
    if (cudaSetDevice(dev) != cudaSuccess) return -1;
    bound = dev;
  }
  return dev;
}

int device_num_sms() {
  const int dev = current_device();
  if (dev < 0 || dev >= MAX_DEV) return 0;
  int n = g_num_sms[dev].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    g_num_sms[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

int* device_error_word() {
  const int dev = current_device();
  if (dev < 0 || dev >= MAX_DEV) return nullptr;
  int* ptr = g_err_ptr[dev].load(std::memory_order_acquire);
  if (!ptr) {
    void* p = nullptr;
    if (cudaGetSymbolAddress(&p, g_error_word) != cudaSuccess) return nullptr;
    ptr = static_cast<int*>(p);
    g_err_ptr[dev].store(ptr, std::memory_order_release);
  }
  return ptr;
}

cudaError_t ensure_kernel_limits(const void* kern, KernelLimits& lim, size_t smem_bytes,
                                 bool cluster) {
  const int dev = current_device();
  if (dev < 0 || dev >= KL_MAX_DEV) return cudaErrorInvalidDevice;
  if (lim.smem[dev].load(std::memory_order_acquire) >= smem_bytes &&
      (!cluster || lim.cluster[dev].load(std::memory_order_acquire)))
    return cudaSuccess;
  std::lock_guard<std::mutex> guard(g_limits_mutex);
  if (lim.smem[dev].load(std::memory_order_relaxed) < smem_bytes) {
    const cudaError_t e =
        cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes);
    if (e != cudaSuccess) return e;
    lim.smem[dev].store(smem_bytes, std::memory_order_release);
  }
  if (cluster && !lim.cluster[dev].load(std::memory_order_relaxed)) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    lim.cluster[dev].store(true, std::memory_order_release);
  }
  return cudaSuccess;
}

int resident_clusters(const void* kern, KernelLimits& lim, int dev, int key, int threads, size_t smem_bytes, int S, int num_sms) {
  if (dev < 0 || dev >= KL_MAX_DEV) return num_sms / S > 0 ? num_sms / S : 1;
  int n = lim.resident[dev][key].load(std::memory_order_relaxed);
  if (n == 0) {
    cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(S * num_sms));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem_bytes;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)S;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n < 1) {
      cudaGetLastError();
      n = num_sms / S > 0 ? num_sms / S : 1;
    }
    lim.resident[dev][key].store(n, std::memory_order_relaxed);
  }
  return n;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

bool encode_tensor_map_bf16(void* map, const void* base, int rank, const uint64_t* dims,
                            const uint64_t* strides, const uint32_t* box, int swizzle) {
  static std::atomic<EncodeTiledFn> fn_cache{nullptr};
  EncodeTiledFn fn = fn_cache.load(std::memory_order_acquire);
  if (!fn) {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault,
                                         &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      return false;
    fn = reinterpret_cast<EncodeTiledFn>(ptr);
    fn_cache.store(fn, std::memory_order_release);
  }
  if (rank < 1 || rank > 5) return false;
  cuuint64_t d[5];
  cuuint64_t st[4];
  cuuint32_t bx[5], es[5];
  for (int i = 0; i < rank; ++i) {
    d[i] = dims[i];
    bx[i] = box[i];
    es[i] = 1;
    if (i > 0) st[i - 1] = strides[i - 1];
  }
  return fn(static_cast<CUtensorMap*>(map), CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank,
            const_cast<void*>(base), d, st, bx, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            swizzle == 32 ? CU_TENSOR_MAP_SWIZZLE_32B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace cospec

using namespace cospec;

#define CS_CHECK_ARG(cond)                 \
  do {                                     \
    if (!(cond)) return COSPEC_ERR_INVALID_ARG; \
  } while (0)

// The CUDA error behind this host thread's last COSPEC_ERR_CUDA.
static thread_local cudaError_t t_last_cuda_error = cudaSuccess;

int cospec::cuda_status(cudaError_t e) {
  if (e == cudaSuccess) return COSPEC_OK;
  t_last_cuda_error = e;
  return COSPEC_ERR_CUDA;
}

int cospec::cuda_lookup_failed() {
  const cudaError_t e = cudaPeekAtLastError();
  return cuda_status(e == cudaSuccess ? cudaErrorUnknown : e);
}

extern "C" {

COSPEC_API const char* cospec_status_string(int status) {
  switch (status) {
    case COSPEC_OK: return "ok";
    case COSPEC_ERR_INVALID_ARG: return "invalid argument";
    case COSPEC_ERR_UNSUPPORTED: return "unsupported shape";
    case COSPEC_ERR_WORKSPACE: return "workspace missing or too small";
    case COSPEC_ERR_CUDA: return "CUDA runtime error";
    case COSPEC_ERR_DEVICE_CHECK: return "device-side check failed";
    default: return "unknown status";
  }
}

COSPEC_API int cospec_num_sms(void) { return device_num_sms(); }

COSPEC_API const char* cospec_last_cuda_error(void) { return cudaGetErrorName(t_last_cuda_error); }

COSPEC_API int cospec_get_device_error(int* flags, void* stream) {
  CS_CHECK_ARG(flags != nullptr);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int* dptr = device_error_word();
  if (!dptr) return cuda_lookup_failed();
  int v = 0;
  cudaError_t e = cudaStreamSynchronize(st);
  if (e == cudaSuccess) e = cudaMemcpyAsync(&v, dptr, sizeof(int), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaMemsetAsync(dptr, 0, sizeof(int), st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return cuda_status(e);
  *flags = v;
  return v ? COSPEC_ERR_DEVICE_CHECK : COSPEC_OK;
}

// ---------------------------------------------------------------- attention
static int check_attn_dims(const cospec_attn_dims* d) {
  if (!d) return COSPEC_ERR_INVALID_ARG;
  if (d->batch < 0 || d->rows < 1 || d->num_q_heads < 1 || d->num_kv_heads < 1 ||
      d->head_dim < 1 || d->page_size < 1 || d->max_pages_per_seq < 1 || d->num_pages < 1)
    return COSPEC_ERR_INVALID_ARG;
  if (d->num_q_heads % d->num_kv_heads != 0) return COSPEC_ERR_INVALID_ARG;
  if (isnan(d->softmax_scale) || isinf(d->softmax_scale)) return COSPEC_ERR_INVALID_ARG;
  if (d->flags & ~(COSPEC_ATTN_KV_STABLE | COSPEC_ATTN_BLOCK_FULL)) return COSPEC_ERR_INVALID_ARG;
  if (d->head_dim != 64 && d->head_dim != 128) return COSPEC_ERR_UNSUPPORTED;
  if (d->page_size != 16) return COSPEC_ERR_UNSUPPORTED;
  if (d->rows > 64) return COSPEC_ERR_UNSUPPORTED;
  if ((d->num_q_heads / d->num_kv_heads) * d->rows > 512) return COSPEC_ERR_UNSUPPORTED;
  return COSPEC_OK;
}

// Clusters of S CTAs of a plan's attention variant resident at once (the
// occupancy query, cached per device; it depends on the variant and its shared
// memory, not on the grid).  The tcgen05 kernels answer alike: each takes all of
// an SM's TMEM and at least 118 KB, so one CTA per SM, and clusters of one size fit alike.
static long long resident_clusters(int D, const AttnPlan& pl, int S, int Hkv, int B, int R) {
  // [dev][D==128][variant][block keys / 16 - 1][S - 1]: count + 1 (0: not yet queried)
  static std::atomic<int> cache[MAX_DEV][2][5][4][16];
  const int kbr = (R + 15) & ~15;
  int dev = 0;
  cudaGetDevice(&dev);
  const int di = D == 128 ? 1 : 0;
  const int mi = pl.kind == 1 ? 4 : (pl.mt == 1 ? 0 : pl.mt == 2 ? 1 : pl.mt == 4 ? 2 : 3);
  if (S < 1 || S > 16) return 0;
  std::atomic<int>& slot = cache[dev < MAX_DEV ? dev : MAX_DEV - 1][di][mi][kbr / 16 - 1][S - 1];
  int c = slot.load(std::memory_order_relaxed);
  if (c == 0) {
    c = 1 + (pl.kind == 1 ? attn_tcq_max_active_clusters(D, S, Hkv, B, pl.rg)
                          : attn_max_active_clusters(D, pl.mt, pl.wk, S, Hkv, B, kbr));
    slot.store(c, std::memory_order_relaxed);
  }
  return c - 1;
}

static AttnPlan attn_plan(const cospec_attn_dims* d, int max_ctx, int sms) {
  return plan_verify_attn(d->batch, d->rows, d->num_q_heads, d->num_kv_heads, d->head_dim,
                          max_ctx, sms, (d->flags & COSPEC_ATTN_KV_STABLE) != 0,
                          [d](const AttnPlan& pl, int S) {
                            return resident_clusters(d->head_dim, pl, S, d->num_kv_heads,
                                                     d->batch > 0 ? d->batch : 1, d->rows);
                          });
}

COSPEC_API int cospec_verify_attn_plan(const cospec_attn_dims* d, int max_ctx, int* kernel,
                                       int* splits) {
  const int st = check_attn_dims(d);
  if (st != COSPEC_OK) return st;
  CS_CHECK_ARG(kernel && splits);
  CS_CHECK_ARG(max_ctx >= 0 && max_ctx <= d->max_pages_per_seq * d->page_size);
  const int sms = device_num_sms();
  if (sms <= 0) return cuda_lookup_failed();
  const AttnPlan pl = attn_plan(d, max_ctx, sms);
  *kernel = pl.kind;
  *splits = pl.cluster;
  return COSPEC_OK;
}

COSPEC_API int cospec_verify_attn_variant(const cospec_attn_dims* d, int max_ctx, int* variant) {
  const int st = check_attn_dims(d);
  if (st != COSPEC_OK) return st;
  CS_CHECK_ARG(variant);
  CS_CHECK_ARG(max_ctx >= 0 && max_ctx <= d->max_pages_per_seq * d->page_size);
  const int sms = device_num_sms();
  if (sms <= 0) return cuda_lookup_failed();
  const AttnPlan pl = attn_plan(d, max_ctx, sms);
  *variant = pl.kind == 1 ? 1 + pl.two : 0;
  return COSPEC_OK;
}

COSPEC_API int cospec_verify_attn_plan_model(const cospec_attn_dims* d, int max_ctx, int num_sms,
                                             cospec_resident_fn resident, void* user, int* kernel,
                                             int* splits) {
  const int st = check_attn_dims(d);
  if (st != COSPEC_OK) return st;
  CS_CHECK_ARG(kernel && splits && resident && num_sms >= 1);
  CS_CHECK_ARG(max_ctx >= 0 && max_ctx <= d->max_pages_per_seq * d->page_size);
  const int kbr = (d->rows + 15) & ~15;
  const AttnPlan pl = plan_verify_attn(
      d->batch, d->rows, d->num_q_heads, d->num_kv_heads, d->head_dim, max_ctx, num_sms,
      (d->flags & COSPEC_ATTN_KV_STABLE) != 0,
      [=](const AttnPlan& p, int S) -> long long {
        return resident(p.kind, p.kind >= 1 ? p.nt : p.nrp, kbr, S, user);
      });
  *kernel = pl.kind;
  *splits = pl.cluster;
  return COSPEC_OK;
}

COSPEC_API int cospec_verify_attn(const cospec_attn_dims* d, int max_ctx, const uint16_t* q,
                                  const uint16_t* k_blk, const uint16_t* v_blk,
                                  const uint16_t* k_pages, const uint16_t* v_pages,
                                  const int32_t* page_table, const int32_t* ctx_len, uint16_t* out,
                                  void* stream) {
  const int st = check_attn_dims(d);
  if (st != COSPEC_OK) return st;
  CS_CHECK_ARG(max_ctx >= 0 && max_ctx <= d->max_pages_per_seq * d->page_size);
  if (d->batch == 0) return COSPEC_OK;
  CS_CHECK_ARG(q && k_blk && v_blk && k_pages && v_pages && page_table && ctx_len && out);
  CS_CHECK_ARG(aligned16(q) && aligned16(k_blk) && aligned16(v_blk) && aligned16(k_pages) &&
               aligned16(v_pages) && aligned16(out));
  const int sms = device_num_sms();
  if (sms <= 0) return cuda_lookup_failed();
  const AttnPlan pl = attn_plan(d, max_ctx, sms);
  int* err = device_error_word();
  if (!err) return cuda_lookup_failed();
  AttnArgs a{};
  a.q = reinterpret_cast<const __nv_bfloat16*>(q);
  a.k_blk = reinterpret_cast<const __nv_bfloat16*>(k_blk);
  a.v_blk = reinterpret_cast<const __nv_bfloat16*>(v_blk);
  a.k_pages = reinterpret_cast<const __nv_bfloat16*>(k_pages);
  a.v_pages = reinterpret_cast<const __nv_bfloat16*>(v_pages);
  a.page_table = page_table;
  a.ctx_len = ctx_len;
  a.out = reinterpret_cast<__nv_bfloat16*>(out);
  a.B = d->batch;
  a.R = d->rows;
  a.Hq = d->num_q_heads;
  a.Hkv = d->num_kv_heads;
  a.D = d->head_dim;
  a.P = d->page_size;
  a.max_pages = d->max_pages_per_seq;
  a.num_pages = d->num_pages;
  a.scale = d->softmax_scale > 0.f ? d->softmax_scale : 1.0f / sqrtf((float)d->head_dim);
  a.max_ctx = max_ctx;
  a.kv_stable = (d->flags & COSPEC_ATTN_KV_STABLE) ? 1 : 0;
  a.block_full = (d->flags & COSPEC_ATTN_BLOCK_FULL) ? 1 : 0;
  return cuda_status(launch_verify_attn(a, pl, err, static_cast<cudaStream_t>(stream)));
}

// ---------------------------------------------------------------- LM head
COSPEC_API size_t cospec_lmhead_workspace(int M, int d, int V) {
  if (M < 1 || d < 64 || V < 1) return 0;
  const int sms = device_num_sms();
  return plan_lmhead(M, d, V, sms > 0 ? sms : 148).ws_bytes;
}

COSPEC_API int cospec_lmhead_argmax_features(int M, int d, int V, const uint16_t* hidden,
                                             const uint16_t* w, const int32_t* draft_for_row,
                                             int32_t* argmax, float* stats, void* ws,
                                             size_t ws_bytes, void* stream) {
  CS_CHECK_ARG(M >= 0 && d > 0 && V > 0);
  if (M == 0) return COSPEC_OK;
  CS_CHECK_ARG(hidden && w && draft_for_row && argmax && stats);
  if (d % 64 != 0) return COSPEC_ERR_UNSUPPORTED;
  if ((long long)V > 0x7fffff00LL) return COSPEC_ERR_UNSUPPORTED;
  CS_CHECK_ARG(aligned16(hidden) && aligned16(w));
  const int sms = device_num_sms();
  if (sms <= 0) return cuda_lookup_failed();
  const LmheadPlan pl = plan_lmhead(M, d, V, sms);
  if (!ws || ws_bytes < pl.ws_bytes || !aligned16(ws)) return COSPEC_ERR_WORKSPACE;
  int* err = device_error_word();
  if (!err) return cuda_lookup_failed();
  return cuda_status(launch_lmhead(M, d, V, reinterpret_cast<const __nv_bfloat16*>(hidden),
                                 reinterpret_cast<const __nv_bfloat16*>(w), draft_for_row, argmax,
                                 stats, ws, LM_WS_ENTRIES, pl, err, static_cast<cudaStream_t>(stream)));
}

COSPEC_API int cospec_lmhead_sample_features(int M, int d, int V, const uint16_t* hidden,
                                             const uint16_t* w, const int32_t* draft_for_row,
                                             float temperature, const uint64_t* seed,
                                             int32_t* sample, float* stats, void* ws,
                                             size_t ws_bytes, void* stream) {
  CS_CHECK_ARG(M >= 0 && d > 0 && V > 0);
  CS_CHECK_ARG(temperature > 0.f && isfinite(temperature) && isfinite(1.0f / temperature));
  if (M == 0) return COSPEC_OK;
  CS_CHECK_ARG(hidden && w && draft_for_row && sample && stats && seed);
  CS_CHECK_ARG((reinterpret_cast<uintptr_t>(seed) & 7u) == 0);
  if (d % 64 != 0) return COSPEC_ERR_UNSUPPORTED;
  if ((long long)V > 0x7fffff00LL) return COSPEC_ERR_UNSUPPORTED;
  CS_CHECK_ARG(aligned16(hidden) && aligned16(w));
  const int sms = device_num_sms();
  if (sms <= 0) return cuda_lookup_failed();
  const LmheadPlan pl = plan_lmhead(M, d, V, sms);
  if (!ws || ws_bytes < pl.ws_bytes || !aligned16(ws)) return COSPEC_ERR_WORKSPACE;
  int* err = device_error_word();
  if (!err) return cuda_lookup_failed();
  return cuda_status(launch_lmhead(M, d, V, reinterpret_cast<const __nv_bfloat16*>(hidden),
                                 reinterpret_cast<const __nv_bfloat16*>(w), draft_for_row, sample,
                                 stats, ws, LM_WS_ENTRIES, pl, err, static_cast<cudaStream_t>(stream),
                                 reinterpret_cast<const unsigned long long*>(seed),
                                 1.0f / temperature));
}

COSPEC_API int cospec_lmhead_logits_features(int M, int d, int V, const uint16_t* hidden,
                                             const uint16_t* w, const int32_t* draft_for_row,
                                             float temperature, int32_t* argmax, float* stats,
                                             float* logits, void* ws, size_t ws_bytes,
                                             void* stream) {
  CS_CHECK_ARG(M >= 0 && d > 0 && V > 0);
  CS_CHECK_ARG(temperature > 0.f && isfinite(temperature) && isfinite(1.0f / temperature));
  if (M == 0) return COSPEC_OK;
  CS_CHECK_ARG(hidden && w && draft_for_row && argmax && stats && logits);
  if (d % 64 != 0) return COSPEC_ERR_UNSUPPORTED;
  if ((long long)V > 0x7fffff00LL) return COSPEC_ERR_UNSUPPORTED;
  CS_CHECK_ARG(aligned16(hidden) && aligned16(w) && (reinterpret_cast<uintptr_t>(logits) & 3u) == 0);
  const int sms = device_num_sms();
  if (sms <= 0) return cuda_lookup_failed();
  const LmheadPlan pl = plan_lmhead(M, d, V, sms);
  if (!ws || ws_bytes < pl.ws_bytes || !aligned16(ws)) return COSPEC_ERR_WORKSPACE;
  int* err = device_error_word();
  if (!err) return cuda_lookup_failed();
  return cuda_status(launch_lmhead(M, d, V, reinterpret_cast<const __nv_bfloat16*>(hidden),
                                   reinterpret_cast<const __nv_bfloat16*>(w), draft_for_row,
                                   argmax, stats, ws, LM_WS_ENTRIES, pl, err, static_cast<cudaStream_t>(stream),
                                   nullptr, 1.0f / temperature, logits));
}

// ---------------------------------------------------------------- speculative sampling
COSPEC_API size_t cospec_sps_workspace(int B) {
  if (B < 1) return 0;
  return (size_t)B * SPS_MAX_SLICES * 16 + (size_t)B * 4 + 256;
}

COSPEC_API int cospec_sps_accept(int B, int K, int V, const int32_t* draft, const float* stats,
                                 const float* logits, const float* q, const uint64_t* seed,
                                 int32_t* target, uint8_t* accept, float* ratio, void* ws,
                                 size_t ws_bytes, void* stream) {
  CS_CHECK_ARG(B >= 0 && K >= 0 && V > 0);
  if (K > 31) return COSPEC_ERR_UNSUPPORTED;
  if (B == 0) return COSPEC_OK;
  CS_CHECK_ARG(stats && logits && seed && target);
  CS_CHECK_ARG(K == 0 || (draft && q && accept && ratio));
  CS_CHECK_ARG((reinterpret_cast<uintptr_t>(seed) & 7u) == 0);
  if (!ws || ws_bytes < cospec_sps_workspace(B) || !aligned16(ws)) return COSPEC_ERR_WORKSPACE;
  const int sms = device_num_sms();
  if (sms <= 0) return cuda_lookup_failed();
  int* err = device_error_word();
  if (!err) return cuda_lookup_failed();
  SpsArgs a{};
  a.B = B;
  a.K = K;
  a.V = V;
  a.draft = draft;
  a.stats = stats;
  a.logits = logits;
  a.q = q;
  a.seed = reinterpret_cast<const unsigned long long*>(seed);
  a.target = target;
  a.accept = accept;
  a.ratio = ratio;
  a.ws = ws;
  return cuda_status(launch_sps(a, sms, err, static_cast<cudaStream_t>(stream)));
}

// ---------------------------------------------------------------- arbitration
COSPEC_API int cospec_arbitrate(int B, int K, const int32_t* draft, const int32_t* argmax,
                                const float* stats, int mlp_hidden, const float* w1,
                                const float* b1, const float* w2, float b2, float lambda,
                                int policy_mode, float* p_out, uint8_t* accept, void* stream) {
  CS_CHECK_ARG(B >= 0 && K >= 0);
  if (K > 31) return COSPEC_ERR_UNSUPPORTED;
  CS_CHECK_ARG(policy_mode >= 0 && policy_mode <= 2);
  CS_CHECK_ARG(!isnan(lambda));
  if (B == 0 || K == 0) return COSPEC_OK;
  CS_CHECK_ARG(draft && argmax && stats && p_out && accept);
  if (policy_mode == COSPEC_POLICY_MLP) {
    CS_CHECK_ARG(w1 && b1 && w2 && mlp_hidden >= 1 && !isnan(b2));
    if (mlp_hidden > 1024) return COSPEC_ERR_UNSUPPORTED;
  }
  return cuda_status(launch_arbitrate(B, K, draft, argmax, stats, mlp_hidden, w1, b1, w2, b2, lambda,
                                    policy_mode, p_out, accept, static_cast<cudaStream_t>(stream)));
}

// ---------------------------------------------------------------- accept + commit
COSPEC_API int cospec_accept_commit(int B, int K, int num_layers, const cospec_attn_dims* dims,
                                    const int32_t* draft, const int32_t* argmax,
                                    const uint8_t* accept, const uint16_t* k_blk,
                                    const uint16_t* v_blk, uint16_t* k_pages, uint16_t* v_pages,
                                    long long pool_layer_stride, const int32_t* page_table,
                                    int32_t* ctx_len, int32_t* accept_len, int32_t* emitted,
                                    void* stream) {
  CS_CHECK_ARG(B >= 0 && K >= 0 && num_layers >= 0);
  if (K > 31) return COSPEC_ERR_UNSUPPORTED;
  const int st = check_attn_dims(dims);
  if (st != COSPEC_OK) return st;
  CS_CHECK_ARG(dims->batch == B && dims->rows == K + 1);
  if (B == 0) return COSPEC_OK;
  CS_CHECK_ARG(argmax && ctx_len && accept_len && emitted && page_table);
  CS_CHECK_ARG(K == 0 || (draft && accept));
  const long long pool_elems = (long long)dims->num_pages * dims->num_kv_heads * dims->page_size *
                               dims->head_dim;
  if (num_layers > 0) {
    CS_CHECK_ARG(k_blk && v_blk && k_pages && v_pages);
    CS_CHECK_ARG(aligned16(k_blk) && aligned16(v_blk) && aligned16(k_pages) && aligned16(v_pages));
    // Several layers need pools of their own: with one pool shared by all
    // layers, every layer's rows would land in the same cells and the
    // committed bytes would depend on which write came last.
    CS_CHECK_ARG(num_layers == 1 || pool_layer_stride >= pool_elems);
    CS_CHECK_ARG(pool_layer_stride % 8 == 0);
  }
  int* err = device_error_word();
  if (!err) return cuda_lookup_failed();
  CommitArgs a{};
  a.B = B;
  a.K = K;
  a.L = num_layers;
  a.Hkv = dims->num_kv_heads;
  a.D = dims->head_dim;
  a.P = dims->page_size;
  a.max_pages = dims->max_pages_per_seq;
  a.num_pages = dims->num_pages;
  a.pool_layer_stride = pool_layer_stride;
  a.draft = draft;
  a.argmax = argmax;
  a.accept = accept;
  a.k_blk = reinterpret_cast<const __nv_bfloat16*>(k_blk);
  a.v_blk = reinterpret_cast<const __nv_bfloat16*>(v_blk);
  a.k_pages = reinterpret_cast<__nv_bfloat16*>(k_pages);
  a.v_pages = reinterpret_cast<__nv_bfloat16*>(v_pages);
  a.page_table = page_table;
  a.ctx_len = ctx_len;
  a.accept_len = accept_len;
  a.emitted = emitted;
  return cuda_status(launch_accept_commit(a, err, static_cast<cudaStream_t>(stream)));
}

COSPEC_API int cospec_accept_commit_launches(const cospec_attn_dims* dims, int num_layers) {
  const int st = check_attn_dims(dims);
  if (st != COSPEC_OK) return st;
  if (num_layers < 0) return COSPEC_ERR_INVALID_ARG;
  if (dims->rows > 32) return COSPEC_ERR_UNSUPPORTED;
  return accept_commit_launches(dims->batch, dims->rows - 1, num_layers, dims->num_kv_heads, dims->head_dim);
}

// ---------------------------------------------------------------- 8-bit KV cache
// Checks a pool's geometry and arrays and fills `p` with the addresses of layer `layer`.
static int kv8_pool(const cospec_kv8_pool* s, int layer, bool summaries, Kv8Pool* p) {
  CS_CHECK_ARG(s && s->layers >= 1 && s->num_pages >= 1 && s->num_kv_heads >= 1);
  if (s->head_dim != 64 && s->head_dim != 128) return COSPEC_ERR_UNSUPPORTED;
  CS_CHECK_ARG(layer >= 0 && layer < s->layers);
  CS_CHECK_ARG(s->k && s->v && s->scale);
  CS_CHECK_ARG(!summaries || (s->summary && s->summary_scale));
  CS_CHECK_ARG((s->summary == nullptr) == (s->summary_scale == nullptr));
  CS_CHECK_ARG(aligned16(s->k) && aligned16(s->v) && aligned16(s->scale) && aligned16(s->summary) &&
               aligned16(s->summary_scale));
  const size_t heads = (size_t)layer * s->num_pages * s->num_kv_heads;
  p->k = s->k + heads * 16 * s->head_dim;
  p->v = s->v + heads * 16 * s->head_dim;
  p->scale = s->scale + heads * 2;
  p->summary = s->summary ? s->summary + heads * s->head_dim : nullptr;
  p->summary_scale = s->summary_scale ? s->summary_scale + heads : nullptr;
  return COSPEC_OK;
}

static int kv8_src(const uint16_t* x, const cospec_kv8_strides* st, Kv8Src* s) {
  CS_CHECK_ARG(x && st && aligned16(x));
  CS_CHECK_ARG(st->layer % 8 == 0 && st->batch % 8 == 0 && st->row % 8 == 0);
  s->p = reinterpret_cast<const __nv_bfloat16*>(x);
  s->layer = st->layer;
  s->batch = st->batch;
  s->row = st->row;
  return COSPEC_OK;
}

// The geometry shared by the selection and the attention.
static int check_kv8_dims(const cospec_attn_dims* d, const cospec_kv8_pool* pool) {
  const int st = check_attn_dims(d);
  if (st != COSPEC_OK) return st;
  CS_CHECK_ARG(pool && pool->num_pages == d->num_pages && pool->num_kv_heads == d->num_kv_heads &&
               pool->head_dim == d->head_dim);
  if ((long long)d->max_pages_per_seq * 16 > 0x7fffffffLL) return COSPEC_ERR_UNSUPPORTED;
  return COSPEC_OK;
}

COSPEC_API int cospec_kv8_append(const cospec_kv8_pool* pool, int first_layer, int num_layers,
                                 int batch, int rows, int num_q_heads, const cospec_rope* rope,
                                 const uint16_t* q, const cospec_kv8_strides* q_strides,
                                 const uint16_t* k, const cospec_kv8_strides* k_strides,
                                 const uint16_t* v, const cospec_kv8_strides* v_strides,
                                 const int32_t* page_table, int max_pages_per_seq,
                                 const int32_t* start, const int32_t* num_rows, uint16_t* q_out,
                                 uint16_t* k_out, void* stream) {
  CS_CHECK_ARG(pool && num_layers >= 0 && batch >= 0 && rows >= 0);
  Kv8AppendArgs a{};
  if (pool->k) {
    const int st = kv8_pool(pool, first_layer, false, &a.pool);
    if (st != COSPEC_OK) return st;
    CS_CHECK_ARG(num_layers <= pool->layers - first_layer);
  } else {
    CS_CHECK_ARG(pool->num_kv_heads >= 1);
    if (pool->head_dim != 64 && pool->head_dim != 128) return COSPEC_ERR_UNSUPPORTED;
  }
  if (num_layers == 0 || batch == 0 || rows == 0) return COSPEC_OK;
  CS_CHECK_ARG(start);
  int st = COSPEC_OK;
  if (pool->k || k_out) st = kv8_src(k, k_strides, &a.k);
  if (st == COSPEC_OK && pool->k) st = kv8_src(v, v_strides, &a.v);
  if (st == COSPEC_OK && q_out) st = kv8_src(q, q_strides, &a.q);
  if (st != COSPEC_OK) return st;
  if (pool->k) {
    CS_CHECK_ARG(page_table && max_pages_per_seq >= 1);
    if ((long long)max_pages_per_seq * 16 > 0x7fffffffLL) return COSPEC_ERR_UNSUPPORTED;
  }
  CS_CHECK_ARG(!q_out || num_q_heads >= 1);
  CS_CHECK_ARG(aligned16(q_out) && aligned16(k_out));
  if (rope) {
    CS_CHECK_ARG(rope->cos && rope->sin && rope->positions >= 1);
    CS_CHECK_ARG(aligned16(rope->cos) && aligned16(rope->sin));
    CS_CHECK_ARG(rope->rot_dim >= 8 && rope->rot_dim % 8 == 0 && rope->rot_dim <= pool->head_dim);
    a.cos = rope->cos;
    a.sin = rope->sin;
    a.positions = rope->positions;
    a.rot = rope->rot_dim;
    a.inter = rope->interleaved ? 1 : 0;
  }
  a.L = num_layers;
  a.B = batch;
  a.R = rows;
  a.Hq = q_out ? num_q_heads : 0;
  a.Hkv = pool->num_kv_heads;
  a.D = pool->head_dim;
  a.num_pages = pool->num_pages;
  a.max_pages = max_pages_per_seq;
  a.page_table = page_table;
  a.start = start;
  a.num_rows = num_rows;
  a.q_out = reinterpret_cast<__nv_bfloat16*>(q_out);
  a.k_out = reinterpret_cast<__nv_bfloat16*>(k_out);
  int* err = device_error_word();
  if (!err) return cuda_lookup_failed();
  return cuda_status(launch_kv8_append(a, err, static_cast<cudaStream_t>(stream)));
}

COSPEC_API int cospec_kv8_select(const cospec_attn_dims* d, const cospec_kv8_pool* pool, int layer,
                                 const uint16_t* q, const cospec_kv8_strides* q_strides,
                                 const int32_t* page_table, const int32_t* ctx_len, int pages,
                                 int sink, int recent, int32_t* sel, void* stream) {
  int st = check_kv8_dims(d, pool);
  if (st != COSPEC_OK) return st;
  Kv8SelectArgs a{};
  st = kv8_pool(pool, layer, true, &a.pool);
  if (st != COSPEC_OK) return st;
  CS_CHECK_ARG(pages >= 1 && sink >= 0 && recent >= 0 && sink <= pages && recent <= pages - sink);
  if (d->max_pages_per_seq > 32768 || d->num_q_heads / d->num_kv_heads > 256 || d->batch > 65535)
    return COSPEC_ERR_UNSUPPORTED;
  if (d->batch == 0) return COSPEC_OK;
  st = kv8_src(q, q_strides, &a.q);
  if (st != COSPEC_OK) return st;
  CS_CHECK_ARG(page_table && ctx_len && sel);
  a.B = d->batch;
  a.R = d->rows;
  a.Hq = d->num_q_heads;
  a.Hkv = d->num_kv_heads;
  a.D = d->head_dim;
  a.num_pages = d->num_pages;
  a.max_pages = d->max_pages_per_seq;
  a.page_table = page_table;
  a.ctx_len = ctx_len;
  a.pages = pages;
  a.sink = sink;
  a.recent = recent;
  a.sel = sel;
  int* err = device_error_word();
  if (!err) return cuda_lookup_failed();
  return cuda_status(launch_kv8_select(a, err, static_cast<cudaStream_t>(stream)));
}

COSPEC_API int cospec_kv8_attn(const cospec_attn_dims* d, int max_ctx, const cospec_kv8_pool* pool,
                               int layer, const uint16_t* q, const cospec_kv8_strides* q_strides,
                               const uint16_t* k_blk, const cospec_kv8_strides* k_strides,
                               const uint16_t* v_blk, const cospec_kv8_strides* v_strides,
                               const int32_t* page_table, const int32_t* ctx_len,
                               const int32_t* sel, int pages, uint16_t* out, void* stream) {
  int st = check_kv8_dims(d, pool);
  if (st != COSPEC_OK) return st;
  CS_CHECK_ARG(max_ctx >= 0 && max_ctx <= d->max_pages_per_seq * d->page_size);
  Kv8AttnArgs a{};
  st = kv8_pool(pool, layer, false, &a.pool);
  if (st != COSPEC_OK) return st;
  CS_CHECK_ARG(!sel || (pages >= 1 && pages <= 0x7fffffff / 16));
  if (d->batch == 0) return COSPEC_OK;
  if ((st = kv8_src(q, q_strides, &a.q)) != COSPEC_OK || (st = kv8_src(k_blk, k_strides, &a.k_blk)) != COSPEC_OK ||
      (st = kv8_src(v_blk, v_strides, &a.v_blk)) != COSPEC_OK)
    return st;
  CS_CHECK_ARG(page_table && ctx_len && out && aligned16(out));
  a.B = d->batch;
  a.R = d->rows;
  a.Hq = d->num_q_heads;
  a.Hkv = d->num_kv_heads;
  a.D = d->head_dim;
  a.num_pages = d->num_pages;
  a.max_pages = d->max_pages_per_seq;
  a.page_table = page_table;
  a.ctx_len = ctx_len;
  a.sel = sel;
  a.pages = sel ? pages : 0;
  a.out = reinterpret_cast<__nv_bfloat16*>(out);
  a.scale = d->softmax_scale > 0.f ? d->softmax_scale : 1.0f / sqrtf((float)d->head_dim);
  a.max_ctx = max_ctx;
  a.kv_stable = (d->flags & COSPEC_ATTN_KV_STABLE) ? 1 : 0;
  a.block_full = (d->flags & COSPEC_ATTN_BLOCK_FULL) ? 1 : 0;
  int* err = device_error_word();
  if (!err) return cuda_lookup_failed();
  return cuda_status(launch_kv8_attn(a, err, static_cast<cudaStream_t>(stream)));
}

// ---------------------------------------------------------------- low-rank adapters
// The checks shared by the two passes; x or dy may be the rows that come in.
static int lora_args(const cospec_lora_dims* d, const uint64_t* seed, LoraArgs* p) {
  CS_CHECK_ARG(d && d->rows >= 0 && d->in_features >= 1 && d->out_features >= 1 && d->rank >= 1 && d->num_adapters >= 1);
  CS_CHECK_ARG(d->dropout >= 0.f && d->dropout < 1.f);
  if (d->in_features % 8 != 0 || d->out_features % 8 != 0 || d->rank % 8 != 0 || d->rank > 128 || d->num_adapters > 65535)
    return COSPEC_ERR_UNSUPPORTED;
  // 32-bit element offsets inside the kernels' tiles, and a launch's rows and columns
  if (d->in_features > (1 << 24) || d->out_features > (1 << 24) || d->rows > 8 << 20) return COSPEC_ERR_UNSUPPORTED;
  const double thr = floor((double)d->dropout * 65536.0 + 0.5);
  if (thr > 65535.0) return COSPEC_ERR_UNSUPPORTED;
  CS_CHECK_ARG(thr == 0.0 || (seed && (reinterpret_cast<uintptr_t>(seed) & 7u) == 0));
  const long long K = d->in_features, N = d->out_features;
  p->ldx = d->x_stride ? d->x_stride : K;
  p->ldy = d->y_stride ? d->y_stride : N;
  p->lddx = d->dx_stride ? d->dx_stride : K;
  CS_CHECK_ARG(p->ldx >= K && p->ldy >= N && p->lddx >= K);
  CS_CHECK_ARG(p->ldx % 8 == 0 && p->ldy % 8 == 0 && p->lddx % 8 == 0);
  if (p->ldx > 1LL << 30 || p->ldy > 1LL << 30 || p->lddx > 1LL << 30) return COSPEC_ERR_UNSUPPORTED;
  p->M = d->rows;
  p->K = d->in_features;
  p->N = d->out_features;
  p->r = d->rank;
  p->n = d->num_adapters;
  p->thr = (uint32_t)thr;
  p->site = d->site;
  p->seed = reinterpret_cast<const unsigned long long*>(seed);
  return COSPEC_OK;
}

COSPEC_API int cospec_lora_forward(const cospec_lora_dims* dims, const uint16_t* x, const uint16_t* w,
                                   const uint16_t* a, const uint16_t* b, const float* scaling,
                                   const int32_t* adapter, const uint64_t* seed, float* u, uint16_t* y,
                                   void* stream) {
  LoraArgs p{};
  const int st = lora_args(dims, seed, &p);
  if (st != COSPEC_OK) return st;
  if (p.M == 0) return COSPEC_OK;
  CS_CHECK_ARG(x && w && a && b && scaling && adapter && u && y);
  CS_CHECK_ARG(aligned16(x) && aligned16(w) && aligned16(a) && aligned16(b) && aligned16(u) && aligned16(y));
  p.x = reinterpret_cast<const __nv_bfloat16*>(x);
  p.w = reinterpret_cast<const __nv_bfloat16*>(w);
  p.a = reinterpret_cast<const __nv_bfloat16*>(a);
  p.b = reinterpret_cast<const __nv_bfloat16*>(b);
  p.scaling = scaling;
  p.adapter = adapter;
  p.u = u;
  p.y = reinterpret_cast<__nv_bfloat16*>(y);
  const int sms = device_num_sms();
  if (sms <= 0) return cuda_lookup_failed();
  int* err = device_error_word();
  if (!err) return cuda_lookup_failed();
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = launch_lora_low(p, false, sms, err, s);
  if (e != cudaSuccess) return cuda_status(e);
  return cuda_status(launch_lora_gemm(p, false, sms, err, s));
}

COSPEC_API int cospec_lora_backward(const cospec_lora_dims* dims, const uint16_t* dy, const uint16_t* x,
                                    const uint16_t* w, const uint16_t* a, const uint16_t* b,
                                    const float* scaling, const int32_t* adapter, const uint64_t* seed,
                                    const float* u, float* t, uint16_t* dx, float* da, float* db,
                                    int flags, void* stream) {
  LoraArgs p{};
  const int st = lora_args(dims, seed, &p);
  if (st != COSPEC_OK) return st;
  CS_CHECK_ARG((flags & ~COSPEC_LORA_ACCUMULATE) == 0);
  CS_CHECK_ARG(aligned16(da) && aligned16(db) && aligned16(dx));
  if (p.M > 0 && (dx || da || db)) {
    CS_CHECK_ARG(dy && adapter && aligned16(dy));
    if (dx || da) CS_CHECK_ARG(b && scaling && t && aligned16(b) && aligned16(t));
    if (dx) CS_CHECK_ARG(w && a && aligned16(w) && aligned16(a));
    if (da) CS_CHECK_ARG(x && aligned16(x));
    if (db) CS_CHECK_ARG(u && aligned16(u));
  }
  p.dy = reinterpret_cast<const __nv_bfloat16*>(dy);
  p.x = reinterpret_cast<const __nv_bfloat16*>(x);
  p.w = reinterpret_cast<const __nv_bfloat16*>(w);
  p.a = reinterpret_cast<const __nv_bfloat16*>(a);
  p.b = reinterpret_cast<const __nv_bfloat16*>(b);
  p.scaling = scaling;
  p.adapter = adapter;
  p.u = const_cast<float*>(u);
  p.t = t;
  p.dx = reinterpret_cast<__nv_bfloat16*>(dx);
  p.da = da;
  p.db = db;
  p.accumulate = flags & COSPEC_LORA_ACCUMULATE;
  const int sms = device_num_sms();
  if (sms <= 0) return cuda_lookup_failed();
  int* err = device_error_word();
  if (!err) return cuda_lookup_failed();
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (p.M > 0 && (dx || da)) e = launch_lora_low(p, true, sms, err, s);
  if (e == cudaSuccess && (da || db)) e = launch_lora_grad(p, sms, err, s);
  if (e == cudaSuccess && p.M > 0 && dx) e = launch_lora_gemm(p, true, sms, err, s);
  return cuda_status(e);
}

// ---------------------------------------------------------------- policy loss
COSPEC_API size_t cospec_arbitrate_loss_workspace(int mlp_hidden) {
  return mlp_hidden < 1 || mlp_hidden > 1024 ? 0 : arb_loss_ws_bytes(mlp_hidden);
}

COSPEC_API int cospec_arbitrate_loss(int num_rounds, int K, const int32_t* draft, const int32_t* argmax,
                                     const float* stats, int mlp_hidden, const float* w1, const float* b1,
                                     const float* w2, const float* b2, const uint8_t* accept,
                                     const uint8_t* eff, const float* adv, const float* p_old,
                                     const float* p_ref, const cospec_rl_params* params, float grad_scale,
                                     float* loss, float* p_new, float* dz, float* dw1, float* db1,
                                     float* dw2, float* db2, void* ws, size_t ws_bytes, void* stream) {
  CS_CHECK_ARG(num_rounds >= 0 && K >= 1 && mlp_hidden >= 1 && params);
  CS_CHECK_ARG(params->clip_eps >= 0.f && isfinite(params->clip_eps) && isfinite(params->beta_h) && isfinite(params->beta_kl) &&
               isfinite(grad_scale));
  if (K > 64 || mlp_hidden > 1024 || (long long)num_rounds * K > (1LL << 31) - 4096) return COSPEC_ERR_UNSUPPORTED;
  CS_CHECK_ARG(w1 && b1 && w2 && b2 && loss && dw1 && db1 && dw2 && db2 && aligned16(w1));
  CS_CHECK_ARG(num_rounds == 0 || (draft && argmax && stats && accept && eff && adv && p_old && p_ref && p_new && dz));
  if (!ws || ws_bytes < arb_loss_ws_bytes(mlp_hidden) || !aligned16(ws)) return COSPEC_ERR_WORKSPACE;
  const int sms = device_num_sms();
  if (sms <= 0) return cuda_lookup_failed();
  ArbLossArgs a{num_rounds, K, mlp_hidden, draft, argmax, stats, w1, b1, w2, b2, accept, eff, adv, p_old, p_ref,
                params->clip_eps, params->beta_h, params->beta_kl, grad_scale, loss, p_new, dz, dw1, db1, dw2, db2, ws};
  return cuda_status(launch_arb_loss(a, sms, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
