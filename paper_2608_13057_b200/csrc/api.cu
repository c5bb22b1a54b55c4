// Host side of the C ABI: argument checks, tensor-map encoding, kernel launches.
// Nothing here synchronises, allocates or reads device memory.
#include <cuda.h>
#include <cuda_runtime.h>

#include "tempo_kernels.cuh"

namespace tempo {

// ---- helpers ------------------------------------------------------------------------------------
constexpr int kMaxE = 1024, kMaxG = 1024, kMaxR = 8, kMaxTopK = 32;

static int check_shape(const tempo_shape* s) {
  if (s == nullptr) return TEMPO_ERR_NULL;
  if (s->T <= 0 || s->k <= 0 || s->E <= 0 || s->G_max <= 0 || s->R_max <= 0 || s->d <= 0 || s->f <= 0 || s->M_cap <= 0)
    return TEMPO_ERR_SHAPE;
  if (s->d % 128 || s->f % 128 || s->M_cap % 128) return TEMPO_ERR_SHAPE;
  if (s->E > kMaxE || s->G_max > kMaxG || s->R_max > kMaxR || s->k > kMaxTopK) return TEMPO_ERR_UNSUPPORTED;
  if (static_cast<long long>(s->T) * s->k > 0x7fff0000ll || static_cast<long long>(s->M_cap) > 0x7fff0000ll)
    return TEMPO_ERR_UNSUPPORTED;
  if (dispatch_smem_bytes(s->E, s->R_max, s->G_max) > 220 * 1024) return TEMPO_ERR_UNSUPPORTED;
  if (dispatch_sampled_smem_bytes(s->E, s->R_max, s->G_max) > 220 * 1024) return TEMPO_ERR_UNSUPPORTED;
  return TEMPO_OK;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiledFn resolve_encode_fn() {
  void* ptr = nullptr;
  cudaDriverEntryPointQueryResult q;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &q) == cudaSuccess &&
      q == cudaDriverEntryPointSuccess)
    return reinterpret_cast<EncodeTiledFn>(ptr);
  return nullptr;
}

static EncodeTiledFn encode_fn() {
  // A pure host-side driver routine, looked up once; the initialisation of a function-local static
  // is thread-safe, so concurrent first calls from several threads are fine.
  static const EncodeTiledFn fn = resolve_encode_fn();
  return fn;
}

// u8 matrix [rows, cols] row-major, box = 128 columns x box_rows rows, 128-byte swizzle.
static bool make_map(CUtensorMap* map, const void* base, uint64_t rows, uint64_t cols, uint32_t box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (fn == nullptr) return false;
  const cuuint64_t dims[2] = {cols, rows};
  const cuuint64_t strides[1] = {cols};
  const cuuint32_t box[2] = {128, box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Scale bytes per token of the per-token quantised activations: one per 128 columns, rounded up to 4.
static int token_sf_stride(int d) { return 4 * (((d / 128) + 3) / 4); }

static int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  return n;
}

// run_mask bit 0: gate/up tiles, bit 1: down tiles.  Buffers a side does not use may be NULL.
static int launch_ffn_host(int run_mask, const tempo_shape* s, const void* a_q, const uint8_t* a_sf, const void* packed,
                           const int32_t* inst_off, const int32_t* m_pad, void* h_q, uint8_t* h_sf, void* y,
                           uint32_t* status, void* workspace, cudaStream_t stream, int max_m = 0,
                           const int32_t* inst_count = nullptr, unsigned long long wait_ns = kDefaultWaitNs,
                           const uint8_t* x_q = nullptr, const uint8_t* x_sf = nullptr, const int32_t* row_pair = nullptr) {
  const PackLayout L = pack_layout(s->G_max, s->d, s->f);
  const uint8_t* blob = static_cast<const uint8_t*>(packed);
  const int sms = sm_count();
  if (sms <= 0) return TEMPO_ERR_CUDA;
  CUtensorMap tmA1, tmA2, tmY;
  // a side that does not run still needs a well-formed map; point it at a buffer that exists
  const bool gather = x_q != nullptr;              // gate/up rows fetched from the per-token buffers: no a_q
  if (!make_map(&tmA1, (run_mask & 1) && !gather ? a_q : h_q, s->M_cap, (run_mask & 1) && !gather ? s->d : s->f, 128))
    return TEMPO_ERR_CUDA;
  if (!make_map(&tmA2, h_q, s->M_cap, s->f, 128)) return TEMPO_ERR_CUDA;
  // Y stores: 32-row x 128-byte boxes (bf16 seen as bytes: 2d per row)
  if (!make_map(&tmY, (run_mask & 2) ? y : h_q, s->M_cap, (run_mask & 2) ? 2ull * s->d : s->f, 32)) return TEMPO_ERR_CUDA;
  FfnParams p{};
  p.side[0] = GemmSide{s->d / 128, L.J1, L.NT1, blob + L.off_w13, a_sf, blob + L.off_sf13};
  p.side[1] = GemmSide{s->f / 128, L.J2, L.NT2, blob + L.off_w2, h_sf, blob + L.off_sf2};
  p.run_mask = run_mask;
  p.G_max = s->G_max;
  p.M_cap = s->M_cap;
  p.d = s->d;
  p.f = s->f;
  p.J_h = L.J2;
  p.inst_off = inst_off;
  p.m_pad = m_pad;
  p.stride_tiles = max_m / 128;
  p.inst_count = inst_count;
  p.h_q = static_cast<uint8_t*>(h_q);
  p.h_sf = h_sf;
  p.y = static_cast<__nv_bfloat16*>(y);
  p.ready = static_cast<int32_t*>(workspace);
  p.done = p.ready ? p.ready + s->M_cap / 128 : nullptr;
  p.status = status;
  p.wait_ns = wait_ns;
  if (gather) {
    p.x_q = x_q;
    p.x_sf = x_sf;
    p.row_pair = row_pair;
    p.x_sf_stride = token_sf_stride(s->d);
    p.k = s->k;
    p.T = s->T;
    return launch_ffn_gather(tmA2, tmY, p, sms, stream) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
  }
  return launch_ffn(tmA1, tmA2, tmY, p, sms, stream) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

// ---- scratch for tempo_grouped_ffn_static ---------------------------------------------------------
// The H-ready / down-seen counters of the fused FFN kernel, two int32 per 128-row tile, for callers
// that cannot hand in a scratch buffer of their own.  Lives in every GPU that loads the library
// (128 KB) until the process ends.  The name is a host-side handle here: the device address is
// looked up once per device with cudaGetSymbolAddress and cached.
constexpr int kStaticMaxTiles = 16384;                       // M_cap <= 128 * 16384 = 2,097,152 rows
static __device__ __align__(256) int32_t g_ffn_scratch[2 * kStaticMaxTiles];
constexpr int kMaxDevices = 64;
static std::atomic<int32_t*> g_ffn_scratch_addr[kMaxDevices];   // zero-initialised; every writer stores the same value

static int32_t* static_scratch_for_current_device() {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
  int32_t* addr = g_ffn_scratch_addr[dev].load(std::memory_order_acquire);
  if (addr == nullptr) {
    void* ptr = nullptr;
    if (cudaGetSymbolAddress(&ptr, g_ffn_scratch) != cudaSuccess || ptr == nullptr) return nullptr;
    addr = static_cast<int32_t*>(ptr);
    g_ffn_scratch_addr[dev].store(addr, std::memory_order_release);
  }
  return addr;
}

}  // namespace tempo

using namespace tempo;

extern "C" {

int tempo_version(void) { return 1; }

const char* tempo_status_string(int code) {
  switch (code) {
    case TEMPO_OK: return "ok";
    case TEMPO_ERR_NULL: return "a required pointer is NULL";
    case TEMPO_ERR_SHAPE: return "a size is not positive or not a multiple of 128";
    case TEMPO_ERR_UNSUPPORTED: return "a size exceeds a documented limit";
    case TEMPO_ERR_CUDA: return "a CUDA call failed";
    case TEMPO_ERR_ALIGN: return "a pointer is not aligned as its comment asks";
    default: return "unknown code";
  }
}

int tempo_m_cap_bound(const tempo_shape* s, int32_t* m_cap) {
  if (s == nullptr || m_cap == nullptr) return TEMPO_ERR_NULL;
  if (s->T <= 0 || s->k <= 0 || s->G_max <= 0) return TEMPO_ERR_SHAPE;
  const long long v = ((static_cast<long long>(s->T) * s->k + 127) / 128) * 128 + 128ll * s->G_max;
  if (v > 0x7fff0000ll) return TEMPO_ERR_UNSUPPORTED;
  *m_cap = static_cast<int32_t>(v);
  return TEMPO_OK;
}

int tempo_sf_bytes(int32_t rows, int32_t cols, size_t* bytes) {
  if (bytes == nullptr) return TEMPO_ERR_NULL;
  if (rows <= 0 || cols <= 0 || rows % 128 || cols % 128) return TEMPO_ERR_SHAPE;
  *bytes = static_cast<size_t>(rows / 128) * (((cols / 128) + 3) / 4) * 512;
  return TEMPO_OK;
}

int tempo_workspace_bytes(const tempo_shape* s, size_t* bytes) {
  if (bytes == nullptr) return TEMPO_ERR_NULL;
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  *bytes = ffn_workspace_bytes(s->M_cap);
  return TEMPO_OK;
}

int tempo_packed_weight_bytes(const tempo_shape* s, size_t* bytes) {
  if (bytes == nullptr) return TEMPO_ERR_NULL;
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  *bytes = pack_layout(s->G_max, s->d, s->f).total;
  return TEMPO_OK;
}

int tempo_pack_weights(const tempo_shape* s, const void* w13_q, const float* w13_s, const void* w2_q,
                       const float* w2_s, void* packed, uint32_t* status, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!w13_q || !w13_s || !w2_q || !w2_s || !packed || !status) return TEMPO_ERR_NULL;
  return launch_pack(s->G_max, s->d, s->f, static_cast<const uint8_t*>(w13_q), w13_s,
                     static_cast<const uint8_t*>(w2_q), w2_s, static_cast<uint8_t*>(packed), status,
                     static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_count_dispatch(const tempo_shape* s, const int32_t* topk_ids, const int32_t* n_valid,
                         const int32_t* replica_map, const int32_t* quota, uint32_t* cum_counts,
                         int32_t* counts, int32_t* inst_count, int32_t* inst_off, int32_t* pair_row,
                         int32_t* row_pair, int32_t* tile_inst, int32_t* m_pad, uint32_t* status, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!topk_ids || !replica_map || !quota || !counts || !inst_count || !inst_off || !pair_row || !row_pair ||
      !tile_inst || !m_pad || !status)
    return TEMPO_ERR_NULL;
  DispatchParams p{s->T, s->k, s->E, s->G_max, s->R_max, s->M_cap, topk_ids, n_valid, replica_map, quota,
                   cum_counts, counts, inst_count, inst_off, pair_row, row_pair, tile_inst, m_pad, status};
  return launch_count_dispatch(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_count_dispatch_sampled(const tempo_shape* s, const int32_t* topk_ids, const int32_t* n_valid,
                                 const int32_t* replica_map, const float* table, uint64_t seed, uint32_t layer,
                                 uint32_t* cum_counts, int32_t* counts, int32_t* inst_count, int32_t* inst_off,
                                 int32_t* pair_row, int32_t* row_pair, int32_t* tile_inst, int32_t* m_pad,
                                 uint32_t* status, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!topk_ids || !replica_map || !table || !counts || !inst_count || !inst_off || !pair_row || !row_pair ||
      !tile_inst || !m_pad || !status)
    return TEMPO_ERR_NULL;
  SampledParams p{s->T, s->k, s->E, s->G_max, s->R_max, s->M_cap, topk_ids, n_valid, replica_map, table,
                  static_cast<unsigned long long>(seed), layer, cum_counts, counts, inst_count, inst_off, pair_row,
                  row_pair, tile_inst, m_pad, status};
  return launch_count_dispatch_sampled(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_permute_pad(const tempo_shape* s, const void* x_bf16, const int32_t* row_pair, const int32_t* pair_row,
                      const int32_t* m_pad, void* a_q, uint8_t* a_sf, uint32_t* status, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!x_bf16 || !row_pair || !m_pad || !a_q || !a_sf || !status) return TEMPO_ERR_NULL;
  PermuteParams p{s->k, s->d, s->M_cap, static_cast<const __nv_bfloat16*>(x_bf16), row_pair, s->T, pair_row, nullptr, m_pad,
                  static_cast<uint8_t*>(a_q), a_sf};
  return launch_permute_pad(p, sm_count(), static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_ffn_gate_up(const tempo_shape* s, const void* a_q, const uint8_t* a_sf, const void* packed,
                      const int32_t* inst_off, const int32_t* m_pad, void* h_q, uint8_t* h_sf, uint32_t* status,
                      void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!a_q || !a_sf || !packed || !inst_off || !m_pad || !h_q || !h_sf || !status) return TEMPO_ERR_NULL;
  return launch_ffn_host(1, s, a_q, a_sf, packed, inst_off, m_pad, h_q, h_sf, nullptr, status, nullptr,
                         static_cast<cudaStream_t>(stream));
}

int tempo_ffn_down(const tempo_shape* s, const void* h_q, const uint8_t* h_sf, const void* packed,
                   const int32_t* inst_off, const int32_t* m_pad, void* y_bf16, uint32_t* status, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!h_q || !h_sf || !packed || !inst_off || !m_pad || !y_bf16 || !status) return TEMPO_ERR_NULL;
  return launch_ffn_host(2, s, nullptr, nullptr, packed, inst_off, m_pad, const_cast<void*>(h_q),
                         const_cast<uint8_t*>(h_sf), y_bf16, status, nullptr, static_cast<cudaStream_t>(stream));
}

int tempo_grouped_ffn(const tempo_shape* s, const void* a_q, const uint8_t* a_sf, const void* packed,
                      const int32_t* inst_off, const int32_t* m_pad, void* h_q, uint8_t* h_sf, void* y_bf16,
                      uint32_t* status, void* workspace, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!a_q || !a_sf || !packed || !inst_off || !m_pad || !h_q || !h_sf || !y_bf16 || !status || !workspace)
    return TEMPO_ERR_NULL;
  return launch_ffn_host(3, s, a_q, a_sf, packed, inst_off, m_pad, h_q, h_sf, y_bf16, status, workspace,
                         static_cast<cudaStream_t>(stream));
}

int tempo_token_sf_bytes(const tempo_shape* s, size_t* bytes) {
  if (bytes == nullptr) return TEMPO_ERR_NULL;
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  *bytes = static_cast<size_t>(s->T) * token_sf_stride(s->d);
  return TEMPO_OK;
}

int tempo_quantize_tokens(const tempo_shape* s, const void* x_bf16, const int32_t* n_valid, void* x_q, uint8_t* x_sf,
                          uint32_t* status, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!x_bf16 || !x_q || !x_sf || !status) return TEMPO_ERR_NULL;
  QuantizeParams p{s->T, s->d, token_sf_stride(s->d), static_cast<const __nv_bfloat16*>(x_bf16), n_valid,
                   static_cast<uint8_t*>(x_q), x_sf};
  return launch_quantize_tokens(p, sm_count(), static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_grouped_ffn_gather(const tempo_shape* s, const void* x_q, const uint8_t* x_sf, const int32_t* row_pair,
                             const void* packed, const int32_t* inst_off, const int32_t* m_pad, void* h_q,
                             uint8_t* h_sf, void* y_bf16, uint32_t* status, void* workspace, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!x_q || !x_sf || !row_pair || !packed || !inst_off || !m_pad || !h_q || !h_sf || !y_bf16 || !status || !workspace)
    return TEMPO_ERR_NULL;
  return launch_ffn_host(3, s, nullptr, nullptr, packed, inst_off, m_pad, h_q, h_sf, y_bf16, status, workspace,
                         static_cast<cudaStream_t>(stream), 0, nullptr, kDefaultWaitNs, static_cast<const uint8_t*>(x_q),
                         x_sf, row_pair);
}

int tempo_grouped_ffn_bounded(const tempo_shape* s, const void* a_q, const uint8_t* a_sf, const void* packed,
                              const int32_t* inst_off, const int32_t* m_pad, void* h_q, uint8_t* h_sf, void* y_bf16,
                              uint32_t* status, void* workspace, uint64_t wait_limit_ns, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!a_q || !a_sf || !packed || !inst_off || !m_pad || !h_q || !h_sf || !y_bf16 || !status || !workspace)
    return TEMPO_ERR_NULL;
  if (wait_limit_ns == 0) return TEMPO_ERR_SHAPE;
  return launch_ffn_host(3, s, a_q, a_sf, packed, inst_off, m_pad, h_q, h_sf, y_bf16, status, workspace,
                         static_cast<cudaStream_t>(stream), 0, nullptr, wait_limit_ns);
}

int tempo_grouped_ffn_static(const tempo_shape* s, const void* a_q, const uint8_t* a_sf, const void* packed,
                             const int32_t* inst_off, const int32_t* m_pad, void* h_q, uint8_t* h_sf, void* y_bf16,
                             uint32_t* status, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!a_q || !a_sf || !packed || !inst_off || !m_pad || !h_q || !h_sf || !y_bf16 || !status) return TEMPO_ERR_NULL;
  if (s->M_cap / 128 > kStaticMaxTiles) return TEMPO_ERR_UNSUPPORTED;      // beyond the built-in scratch
  int32_t* scratch = static_scratch_for_current_device();
  if (scratch == nullptr) return TEMPO_ERR_CUDA;
  // the array keeps whatever the last call left (normally zeros; not after a timed-out call): start clean
  if (cudaMemsetAsync(scratch, 0, 2 * sizeof(int32_t) * static_cast<size_t>(s->M_cap / 128),
                      static_cast<cudaStream_t>(stream)) != cudaSuccess)
    return TEMPO_ERR_CUDA;
  return launch_ffn_host(3, s, a_q, a_sf, packed, inst_off, m_pad, h_q, h_sf, y_bf16, status, scratch,
                         static_cast<cudaStream_t>(stream));
}

// ---- masked layout ------------------------------------------------------------------------------------
static int check_masked(const tempo_shape* s, int32_t max_m) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (max_m <= 0 || max_m % 128 != 0) return TEMPO_ERR_SHAPE;
  if (static_cast<long long>(s->G_max) * max_m > s->M_cap) return TEMPO_ERR_SHAPE;
  return TEMPO_OK;
}

int tempo_count_dispatch_masked(const tempo_shape* s, int32_t max_m, const int32_t* topk_ids, const int32_t* n_valid,
                                const int32_t* replica_map, const int32_t* quota, uint32_t* cum_counts,
                                int32_t* counts, int32_t* inst_count, int32_t* inst_off, int32_t* pair_row,
                                int32_t* row_pair, int32_t* tile_inst, int32_t* m_pad, uint32_t* status, void* stream) {
  const int rc = check_masked(s, max_m);
  if (rc != TEMPO_OK) return rc;
  if (!topk_ids || !replica_map || !quota || !counts || !inst_count || !inst_off || !pair_row || !row_pair ||
      !tile_inst || !m_pad || !status)
    return TEMPO_ERR_NULL;
  DispatchParams p{s->T, s->k, s->E, s->G_max, s->R_max, s->M_cap, topk_ids, n_valid, replica_map, quota,
                   cum_counts, counts, inst_count, inst_off, pair_row, row_pair, tile_inst, m_pad, status, max_m};
  return launch_count_dispatch(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_permute_pad_masked(const tempo_shape* s, const void* x_bf16, const int32_t* row_pair, const int32_t* pair_row,
                             const int32_t* tile_inst, const int32_t* m_pad, void* a_q, uint8_t* a_sf,
                             uint32_t* status, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!x_bf16 || !row_pair || !pair_row || !tile_inst || !m_pad || !a_q || !a_sf || !status) return TEMPO_ERR_NULL;
  PermuteParams p{s->k, s->d, s->M_cap, static_cast<const __nv_bfloat16*>(x_bf16), row_pair, s->T, pair_row, tile_inst,
                  m_pad, static_cast<uint8_t*>(a_q), a_sf};
  return launch_permute_pad(p, sm_count(), static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_grouped_ffn_masked(const tempo_shape* s, int32_t max_m, const void* a_q, const uint8_t* a_sf,
                             const void* packed, const int32_t* inst_count, void* h_q, uint8_t* h_sf, void* y_bf16,
                             uint32_t* status, void* workspace, void* stream) {
  const int rc = check_masked(s, max_m);
  if (rc != TEMPO_OK) return rc;
  if (!a_q || !a_sf || !packed || !inst_count || !h_q || !h_sf || !y_bf16 || !status || !workspace) return TEMPO_ERR_NULL;
  return launch_ffn_host(3, s, a_q, a_sf, packed, nullptr, nullptr, h_q, h_sf, y_bf16, status, workspace,
                         static_cast<cudaStream_t>(stream), max_m, inst_count);
}

// ---- bf16 variant of steps 2 and 3 -------------------------------------------------------------------
int tempo_packed_weight_bytes_bf16(const tempo_shape* s, size_t* bytes) {
  if (bytes == nullptr) return TEMPO_ERR_NULL;
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  *bytes = pack_layout_bf16(s->G_max, s->d, s->f).total;
  return TEMPO_OK;
}

int tempo_pack_weights_bf16(const tempo_shape* s, const void* w13_bf16, const void* w2_bf16, void* packed, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!w13_bf16 || !w2_bf16 || !packed) return TEMPO_ERR_NULL;
  return launch_pack_bf16(s->G_max, s->d, s->f, static_cast<const __nv_bfloat16*>(w13_bf16),
                          static_cast<const __nv_bfloat16*>(w2_bf16), static_cast<uint8_t*>(packed),
                          static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_permute_pad_bf16(const tempo_shape* s, const void* x_bf16, const int32_t* row_pair, const int32_t* m_pad,
                           void* a_bf16, uint32_t* status, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!x_bf16 || !row_pair || !m_pad || !a_bf16 || !status) return TEMPO_ERR_NULL;
  PermuteParams p{s->k, s->d, s->M_cap, static_cast<const __nv_bfloat16*>(x_bf16), row_pair, s->T, nullptr, nullptr, m_pad, nullptr, nullptr};
  return launch_permute_pad_bf16(p, static_cast<__nv_bfloat16*>(a_bf16), sm_count(), static_cast<cudaStream_t>(stream)) ==
                 cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_grouped_ffn_bf16(const tempo_shape* s, const void* a_bf16, const void* packed, const int32_t* inst_off,
                           const int32_t* m_pad, void* h_bf16, void* y_bf16, uint32_t* status, void* workspace,
                           void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!a_bf16 || !packed || !inst_off || !m_pad || !h_bf16 || !y_bf16 || !status || !workspace) return TEMPO_ERR_NULL;
  const PackLayout L = pack_layout_bf16(s->G_max, s->d, s->f);
  const uint8_t* blob = static_cast<const uint8_t*>(packed);
  const int sms = sm_count();
  if (sms <= 0) return TEMPO_ERR_CUDA;
  CUtensorMap tmA1, tmA2, tmY;    // bf16 matrices seen as bytes: 2d / 2f per row
  if (!make_map(&tmA1, a_bf16, s->M_cap, 2ull * s->d, 128)) return TEMPO_ERR_CUDA;
  if (!make_map(&tmA2, h_bf16, s->M_cap, 2ull * s->f, 128)) return TEMPO_ERR_CUDA;
  if (!make_map(&tmY, y_bf16, s->M_cap, 2ull * s->d, 32)) return TEMPO_ERR_CUDA;
  FfnParams p{};
  p.side[0] = GemmSide{s->d / 64, 0, L.NT1, blob + L.off_w13, nullptr, nullptr};
  p.side[1] = GemmSide{s->f / 64, 0, L.NT2, blob + L.off_w2, nullptr, nullptr};
  p.run_mask = 3;
  p.G_max = s->G_max;
  p.M_cap = s->M_cap;
  p.d = s->d;
  p.f = s->f;
  p.inst_off = inst_off;
  p.m_pad = m_pad;
  p.h_q = static_cast<uint8_t*>(h_bf16);
  p.y = static_cast<__nv_bfloat16*>(y_bf16);
  p.ready = static_cast<int32_t*>(workspace);
  p.done = p.ready + s->M_cap / 128;
  p.status = status;
  p.wait_ns = kDefaultWaitNs;
  return launch_ffn_bf16(tmA1, tmA2, tmY, p, sms, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK
                                                                                                         : TEMPO_ERR_CUDA;
}

int tempo_unpermute_combine(const tempo_shape* s, const void* y_bf16, const int32_t* pair_row, const float* topk_w,
                            const int32_t* n_valid, void* out_bf16, uint32_t* status, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!y_bf16 || !pair_row || !topk_w || !out_bf16 || !status) return TEMPO_ERR_NULL;
  CombineParams p{s->T, s->k, s->d, static_cast<const __nv_bfloat16*>(y_bf16), pair_row, topk_w, n_valid,
                  static_cast<__nv_bfloat16*>(out_bf16)};
  return launch_combine(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

// ---- norms around the block ----------------------------------------------------------------------------
static bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

static int check_norm(const tempo_norm* s) {
  if (s == nullptr) return TEMPO_ERR_NULL;
  if (s->T <= 0 || s->d <= 0) return TEMPO_ERR_SHAPE;
  if (s->kind != TEMPO_NORM_RMS && s->kind != TEMPO_NORM_LAYER) return TEMPO_ERR_UNSUPPORTED;
  if (s->d > 16384) return TEMPO_ERR_UNSUPPORTED;
  return TEMPO_OK;
}

// The widest vector (elements) that the width, every pitch and every pointer of the launch allow.
static int norm_vec(const NormParams& p) {
  for (int vec = 8; vec > 1; vec /= 2) {
    const size_t b16 = 2 * vec, f32 = vec >= 4 ? 16 : 4 * vec;
    const size_t rs = p.stream_f32 ? f32 : b16, ps = p.param_f32 ? f32 : b16;
    bool ok = p.d % vec == 0 && aligned(p.r, rs) && p.ld_r % vec == 0 && aligned(p.x, b16) && (!p.x || p.ld_x % vec == 0);
    ok = ok && aligned(p.next_w, ps) && aligned(p.next_b, ps) && aligned(p.post_w, ps) && aligned(p.post_b, ps);
    if (p.y != nullptr) ok = ok && aligned(p.y, b16) && p.ld_y % vec == 0 && aligned(p.r_out, rs) && p.ld_r_out % vec == 0;
    if (ok) return vec;
  }
  return 1;
}

static int run_norm(NormParams& p, cudaStream_t stream) {
  const int sms = sm_count();
  if (sms <= 0) return TEMPO_ERR_CUDA;
  const int vec = norm_vec(p);
  p.shift = norm_shifts(p, vec);
  const int pv = p.shift ? 8 : vec;
  const size_t gs = p.gate_f32 ? (pv >= 4 ? 16 : 4 * pv) : 2 * pv;
  p.gate_vec = p.gate != nullptr && p.gate_col == 1 && p.gate_row % pv == 0 && aligned(p.gate, gs) ? 1 : 0;
  p.param_vec = aligned(p.next_w, 16) && aligned(p.next_b, 16) && aligned(p.post_w, 16) && aligned(p.post_b, 16);
  return launch_norm(p, vec, sms, stream) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_norm_in(const tempo_norm* s, const void* r, const void* w, const void* b, const int32_t* n_valid, void* x_bf16,
                  void* stream) {
  const int rc = check_norm(s);
  if (rc != TEMPO_OK) return rc;
  if (!r || !w || !x_bf16) return TEMPO_ERR_NULL;
  if (s->ld_r < s->d || s->ld_x < s->d) return TEMPO_ERR_SHAPE;
  if (!aligned(r, s->stream_f32 ? 4 : 2) || !aligned(w, s->param_f32 ? 4 : 2) || !aligned(b, s->param_f32 ? 4 : 2) ||
      !aligned(x_bf16, 2))
    return TEMPO_ERR_ALIGN;
  NormParams p{};
  p.T = s->T; p.d = s->d; p.layer = s->kind == TEMPO_NORM_LAYER;
  p.stream_f32 = s->stream_f32; p.param_f32 = s->param_f32;
  p.r = r; p.next_w = w; p.next_b = b; p.n_valid = n_valid;
  p.x = static_cast<__nv_bfloat16*>(x_bf16);
  p.ld_r = s->ld_r; p.ld_x = s->ld_x; p.eps = s->eps;
  return run_norm(p, static_cast<cudaStream_t>(stream));
}

int tempo_norm_out(const tempo_norm* s, const void* y_bf16, const void* r, const void* post_w, const void* post_b,
                   const void* gate, const void* next_w, const void* next_b, const int32_t* n_valid, void* r_out,
                   void* x_bf16, void* stream) {
  const int rc = check_norm(s);
  if (rc != TEMPO_OK) return rc;
  if (!y_bf16 || !r || !r_out || (x_bf16 && !next_w) || (post_b && !post_w)) return TEMPO_ERR_NULL;
  if (s->ld_y < s->d || s->ld_r < s->d || s->ld_r_out < s->d || (x_bf16 && s->ld_x < s->d)) return TEMPO_ERR_SHAPE;
  if (gate && (s->gate_row < 0 || s->gate_col < 0)) return TEMPO_ERR_SHAPE;
  const size_t rs = s->stream_f32 ? 4 : 2, ps = s->param_f32 ? 4 : 2;
  if (!aligned(y_bf16, 2) || !aligned(r, rs) || !aligned(r_out, rs) || !aligned(x_bf16, 2) || !aligned(post_w, ps) ||
      !aligned(post_b, ps) || !aligned(next_w, ps) || !aligned(next_b, ps) || !aligned(gate, s->gate_f32 ? 4 : 2))
    return TEMPO_ERR_ALIGN;
  NormParams p{};
  p.T = s->T; p.d = s->d; p.layer = s->kind == TEMPO_NORM_LAYER;
  p.stream_f32 = s->stream_f32; p.param_f32 = s->param_f32; p.gate_f32 = s->gate_f32;
  p.y = static_cast<const __nv_bfloat16*>(y_bf16);
  p.r = r; p.post_w = post_w; p.post_b = post_b; p.gate = gate;
  p.next_w = x_bf16 ? next_w : nullptr; p.next_b = x_bf16 ? next_b : nullptr; p.n_valid = n_valid;
  p.r_out = r_out; p.x = static_cast<__nv_bfloat16*>(x_bf16);
  p.ld_y = s->ld_y; p.ld_r = s->ld_r; p.ld_r_out = s->ld_r_out; p.ld_x = s->ld_x;
  p.gate_row = s->gate_row; p.gate_col = s->gate_col;
  p.eps = s->eps; p.r_scale = s->r_scale; p.y_scale = s->y_scale;
  return run_norm(p, static_cast<cudaStream_t>(stream));
}

// ---- router ----------------------------------------------------------------------------------------------
int tempo_route(const tempo_shape* s, int32_t score, int32_t renormalise, float scale, const void* x_bf16,
                const void* w_router_bf16, const float* bias, const int32_t* n_valid, int32_t* topk_ids, float* topk_w,
                uint32_t* status, void* stream) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (!x_bf16 || !w_router_bf16 || !topk_ids || !topk_w || !status) return TEMPO_ERR_NULL;
  if (s->k > s->E) return TEMPO_ERR_SHAPE;
  if (s->E > 512 || (score != TEMPO_ROUTE_SOFTMAX && score != TEMPO_ROUTE_SIGMOID)) return TEMPO_ERR_UNSUPPORTED;
  if (!aligned(x_bf16, 16) || !aligned(w_router_bf16, 16) || !aligned(topk_ids, 4) || !aligned(topk_w, 4) || !aligned(bias, 4))
    return TEMPO_ERR_ALIGN;
  const int sms = sm_count();
  if (sms <= 0) return TEMPO_ERR_CUDA;
  const RoutePlan plan = route_plan(s->T, s->E, s->d, sms);
  CUtensorMap tmX, tmW;      // bf16 matrices seen as bytes: 2d per row
  if (!make_map(&tmX, x_bf16, s->T, 2ull * s->d, plan.x_box)) return TEMPO_ERR_CUDA;
  if (!make_map(&tmW, w_router_bf16, s->E, 2ull * s->d, plan.w_box)) return TEMPO_ERR_CUDA;
  RouteParams p{};
  p.T = s->T; p.k = s->k; p.E = s->E; p.Kb = s->d / 64;
  p.sigmoid = score == TEMPO_ROUTE_SIGMOID; p.renormalise = renormalise != 0; p.scale = scale;
  p.bias = bias; p.n_valid = n_valid; p.ids = topk_ids; p.w = topk_w; p.status = status;
  return launch_route(tmX, tmW, p, plan, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

// ---- the layer's experts for a few tokens ---------------------------------------------------------------
static int check_few(const tempo_shape* s, int sms) {
  const int rc = check_shape(s);
  if (rc != TEMPO_OK) return rc;
  if (s->T > kFewMaxT || s->T * s->k > kFewMaxPairs) return TEMPO_ERR_UNSUPPORTED;
  // run arithmetic in 32 bits: (blocks of the larger product) * CTAs, bf16 blocks (64 values) being the more
  const long long A = s->G_max < s->T * s->k ? s->G_max : s->T * s->k;
  const long long b1 = A * (s->f / 128) * (s->d / 64), b2 = A * ((s->d + 255) / 256) * (s->f / 64);
  if (((b1 > b2 ? b1 : b2) + 1) * sms > 0xffffffffll) return TEMPO_ERR_UNSUPPORTED;
  return TEMPO_OK;
}

int tempo_few_workspace_bytes(const tempo_shape* s, size_t* bytes) {
  if (bytes == nullptr) return TEMPO_ERR_NULL;
  const int rc = check_few(s, kFewMaxSms);
  if (rc != TEMPO_OK) return rc;
  *bytes = few_layout(s->T, s->k, s->G_max, s->d, s->f, kFewMaxSms).total;
  return TEMPO_OK;
}

static int run_few(bool bf16, const tempo_shape* s, const void* x, const int32_t* ids, const float* w, const int32_t* n_valid,
                   const int32_t* replica_map, const void* packed, void* out, uint32_t* status, void* workspace, void* stream) {
  const int rc = check_few(s, kFewMaxSms);
  if (rc != TEMPO_OK) return rc;
  if (!x || !ids || !w || !replica_map || !packed || !out || !status || !workspace) return TEMPO_ERR_NULL;
  if (!aligned(x, 16) || !aligned(packed, 256) || !aligned(out, 16) || !aligned(workspace, 256) || !aligned(ids, 4) ||
      !aligned(w, 4) || !aligned(replica_map, 4))
    return TEMPO_ERR_ALIGN;
  const int sms = min(sm_count(), kFewMaxSms);
  if (sms <= 0) return TEMPO_ERR_CUDA;
  const PackLayout L = bf16 ? pack_layout_bf16(s->G_max, s->d, s->f) : pack_layout(s->G_max, s->d, s->f);
  const FewLayout F = few_layout(s->T, s->k, s->G_max, s->d, s->f, kFewMaxSms);
  const uint8_t* blob = static_cast<const uint8_t*>(packed);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const int kblock = bf16 ? 64 : 128;
  FewParams p{};
  p.T = s->T; p.k = s->k; p.E = s->E; p.R = s->R_max; p.G = s->G_max; p.d = s->d;
  p.Kb1 = s->d / kblock; p.Kb2 = s->f / kblock; p.NT1 = L.NT1; p.NT2 = L.NT2; p.J1 = L.J1; p.J2 = L.J2;
  p.ids = ids; p.w = w; p.n_valid = n_valid; p.replica_map = replica_map;
  p.x = static_cast<const __nv_bfloat16*>(x);
  p.w13 = blob + L.off_w13; p.w2 = blob + L.off_w2; p.sf13 = blob + L.off_sf13; p.sf2 = blob + L.off_sf2;
  p.leave = reinterpret_cast<unsigned int*>(ws + F.off_leave);
  p.counters = reinterpret_cast<int32_t*>(ws + F.off_counters);
  p.counter_ints = F.counter_ints;
  p.x_img = ws + F.off_x; p.h_img = ws + F.off_h;
  p.gu_part = reinterpret_cast<float*>(ws + F.off_gu); p.y_part = reinterpret_cast<float*>(ws + F.off_y);
  p.out = static_cast<__nv_bfloat16*>(out); p.status = status; p.wait_ns = kDefaultWaitNs;
  return launch_few(p, bf16, sms, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_few_ffn(const tempo_shape* s, const void* x_bf16, const int32_t* topk_ids, const float* topk_w,
                  const int32_t* n_valid, const int32_t* replica_map, const void* packed, void* out_bf16, uint32_t* status,
                  void* workspace, void* stream) {
  return run_few(false, s, x_bf16, topk_ids, topk_w, n_valid, replica_map, packed, out_bf16, status, workspace, stream);
}

int tempo_few_ffn_bf16(const tempo_shape* s, const void* x_bf16, const int32_t* topk_ids, const float* topk_w,
                       const int32_t* n_valid, const int32_t* replica_map, const void* packed, void* out_bf16,
                       uint32_t* status, void* workspace, void* stream) {
  return run_few(true, s, x_bf16, topk_ids, topk_w, n_valid, replica_map, packed, out_bf16, status, workspace, stream);
}

// ---- the attention half of a layer ------------------------------------------------------------------------
static int check_cache(const tempo_cache* c) {
  if (c == nullptr) return TEMPO_ERR_NULL;
  if (c->n_pages <= 0 || c->Hkv <= 0) return TEMPO_ERR_SHAPE;
  if ((c->D != 64 && c->D != 128) || c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return TEMPO_ERR_UNSUPPORTED;
  if (static_cast<long long>(c->n_pages) * c->page_size > 0x7fffffffll || c->Hkv > 65536) return TEMPO_ERR_UNSUPPORTED;
  if (9.0 * c->D * c->page_size / 8 * c->Hkv * c->n_pages > 1e12) return TEMPO_ERR_UNSUPPORTED;   // units are numbered in 32 bits
  return TEMPO_OK;
}

int tempo_cache_bytes(const tempo_cache* c, size_t* bytes) {
  if (bytes == nullptr) return TEMPO_ERR_NULL;
  const int rc = check_cache(c);
  if (rc != TEMPO_OK) return rc;
  *bytes = 9ull * c->D * c->page_size / 8 * c->Hkv * c->n_pages;
  return TEMPO_OK;
}

static bool vectors8(const void* p, int64_t ld, int64_t hd) { return aligned(p, 16) && ld % 8 == 0 && hd % 8 == 0; }

// Heads of D elements at these pitches; those of an output do not overlap (rows of heads, or heads of rows).
static bool pitches(int64_t ld, int64_t hd) { return ld >= 0 && hd >= 0 && ld < (1ll << 40) && hd < (1ll << 40); }
static bool apart(int64_t ld, int64_t hd, int64_t T, int64_t H, int D) {
  return pitches(ld, hd) && (H == 1 || hd >= D) && (T == 1 || ld >= D) && (H == 1 || T == 1 || ld >= (H - 1) * hd + D || hd >= (T - 1) * ld + D);
}

static int check_heads(const tempo_heads* a, bool append) {
  if (a == nullptr) return TEMPO_ERR_NULL;
  if (a->T <= 0 || a->Hq < 0 || a->Hkv < 0 || a->Hq + static_cast<int64_t>(a->Hkv) == 0 || (append && a->Hkv == 0)) return TEMPO_ERR_SHAPE;
  if (a->D <= 0 || a->D % 8 || a->rot < 0 || a->rot > a->D || a->rot % 2 || (a->rot > 0 && a->n_pos <= 0)) return TEMPO_ERR_SHAPE;
  if (a->D > 256 || a->Hq > 65536 || a->Hkv > 65536 || (a->interleaved != 0 && a->interleaved != 1)) return TEMPO_ERR_UNSUPPORTED;
  if (a->Hq > 0 && (!pitches(a->ld_q, a->hd_q) || !apart(a->ld_q_out, a->hd_q_out, a->T, a->Hq, a->D))) return TEMPO_ERR_SHAPE;
  if (a->Hkv > 0 && !pitches(a->ld_k, a->hd_k)) return TEMPO_ERR_SHAPE;
  if (append && !pitches(a->ld_v, a->hd_v)) return TEMPO_ERR_SHAPE;
  if (!append && a->Hkv > 0 && !apart(a->ld_k_out, a->hd_k_out, a->T, a->Hkv, a->D)) return TEMPO_ERR_SHAPE;
  return TEMPO_OK;
}

static int run_heads(const tempo_heads* a, const tempo_cache* c, const void* q, const void* k, const void* v, const void* q_w,
                     const void* k_w, const int32_t* positions, const float* cos_sin, const int32_t* slots, const int32_t* n_valid,
                     void* q_out, void* k_out, void* cache, uint32_t* status, void* stream) {
  const bool append = c != nullptr;
  if (!status || (a->Hq > 0 && (!q || !q_out)) || (a->Hkv > 0 && !k) || (a->rot > 0 && (!positions || !cos_sin))) return TEMPO_ERR_NULL;
  if (append ? !v || !slots || !cache : a->Hkv > 0 && !k_out) return TEMPO_ERR_NULL;
  const size_t ws = a->w_f32 ? 4 : 2;
  if (!aligned(q, 2) || !aligned(k, 2) || !aligned(v, 2) || !aligned(q_out, 2) || !aligned(k_out, 2) || !aligned(q_w, ws) ||
      !aligned(k_w, ws) || !aligned(positions, 4) || !aligned(cos_sin, 4) || !aligned(slots, 4) || !aligned(n_valid, 4) ||
      !aligned(cache, 16) || !aligned(status, 4))
    return TEMPO_ERR_ALIGN;
  HeadsParams p{};
  p.T = a->T; p.Hq = a->Hq; p.Hkv = a->Hkv; p.D = a->D; p.rot = a->rot; p.interleaved = a->interleaved; p.n_pos = a->n_pos;
  p.w_f32 = a->w_f32;
  p.q_vec = vectors8(q, a->ld_q, a->hd_q); p.k_vec = vectors8(k, a->ld_k, a->hd_k); p.v_vec = vectors8(v, a->ld_v, a->hd_v);
  p.q_out_vec = vectors8(q_out, a->ld_q_out, a->hd_q_out); p.k_out_vec = vectors8(k_out, a->ld_k_out, a->hd_k_out);
  p.w_vec = aligned(q_w, 16) && aligned(k_w, 16);
  p.rot_vec = aligned(cos_sin, 16) && a->rot % (a->interleaved ? 8 : 16) == 0;
  const auto quads = [&](const void* x, int64_t ld, int64_t hd) { return aligned(x, 8) && ld % 4 == 0 && hd % 4 == 0; };
  p.quads = a->rot % 8 == 0 && aligned(cos_sin, 16) && aligned(q_w, 4 * ws) && aligned(k_w, 4 * ws) && quads(q, a->ld_q, a->hd_q) &&
            quads(q_out, a->ld_q_out, a->hd_q_out) && (append || (quads(k, a->ld_k, a->hd_k) && quads(k_out, a->ld_k_out, a->hd_k_out)));
  p.inverse_d = 1.0f / a->D;
  p.q = static_cast<const __nv_bfloat16*>(q); p.k = static_cast<const __nv_bfloat16*>(k); p.v = static_cast<const __nv_bfloat16*>(v);
  p.q_w = q_w; p.k_w = k_w; p.positions = positions; p.cos_sin = cos_sin; p.n_valid = n_valid;
  p.q_out = static_cast<__nv_bfloat16*>(q_out); p.k_out = static_cast<__nv_bfloat16*>(k_out);
  p.ld_q = a->ld_q; p.hd_q = a->hd_q; p.ld_k = a->ld_k; p.hd_k = a->hd_k; p.ld_v = a->ld_v; p.hd_v = a->hd_v;
  p.ld_q_out = a->ld_q_out; p.hd_q_out = a->hd_q_out; p.ld_k_out = a->ld_k_out; p.hd_k_out = a->hd_k_out;
  p.eps = a->eps; p.status = status;
  if (append) {
    p.n_pages = c->n_pages; p.page_size = c->page_size; p.slots = slots; p.cache = static_cast<uint8_t*>(cache);
  }
  const int sms = sm_count();
  if (sms <= 0) return TEMPO_ERR_CUDA;
  return launch_heads(p, append, sms, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_qk_rotate(const tempo_heads* a, const void* q, const void* k, const void* q_w, const void* k_w, const int32_t* positions,
                    const float* cos_sin, const int32_t* n_valid, void* q_out, void* k_out, uint32_t* status, void* stream) {
  const int rc = check_heads(a, false);
  if (rc != TEMPO_OK) return rc;
  return run_heads(a, nullptr, q, k, nullptr, q_w, k_w, positions, cos_sin, nullptr, n_valid, q_out, k_out, nullptr, status, stream);
}

int tempo_kv_append(const tempo_heads* a, const tempo_cache* c, const void* q, const void* k, const void* v, const void* q_w,
                    const void* k_w, const int32_t* positions, const float* cos_sin, const int32_t* slots, const int32_t* n_valid,
                    void* q_out, void* cache, uint32_t* status, void* stream) {
  int rc = check_cache(c);
  if (rc == TEMPO_OK) rc = check_heads(a, true);
  if (rc != TEMPO_OK) return rc;
  if (a->D != c->D || a->Hkv != c->Hkv) return TEMPO_ERR_SHAPE;
  return run_heads(a, c, q, k, v, q_w, k_w, positions, cos_sin, slots, n_valid, q_out, nullptr, cache, status, stream);
}

int tempo_kv_read(const tempo_cache* c, const void* cache, const int32_t* slots, int32_t n, void* k, void* v, uint32_t* status,
                  void* stream) {
  const int rc = check_cache(c);
  if (rc != TEMPO_OK) return rc;
  if (n <= 0) return TEMPO_ERR_SHAPE;
  if (!cache || !slots || !k || !v || !status) return TEMPO_ERR_NULL;
  if (!aligned(cache, 16) || !aligned(slots, 4) || !aligned(k, 16) || !aligned(v, 16) || !aligned(status, 4)) return TEMPO_ERR_ALIGN;
  KvReadParams p{n, c->n_pages, c->page_size, c->Hkv, static_cast<const uint8_t*>(cache), slots, static_cast<__half*>(k),
                 static_cast<__half*>(v), status};
  return launch_kv_read(p, c->D, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_attend_workspace_bytes(const tempo_cache* c, int32_t Hq, size_t* bytes) {
  if (bytes == nullptr) return TEMPO_ERR_NULL;
  const int rc = check_cache(c);
  if (rc != TEMPO_OK) return rc;
  if (Hq <= 0 || Hq % c->Hkv) return TEMPO_ERR_SHAPE;
  *bytes = attend_layout(c->D).total;
  return TEMPO_OK;
}

int tempo_attend_padded(const tempo_attention* a, const tempo_cache* c, const void* q, const void* cache, const int32_t* page_table,
                        const int32_t* lens, const int32_t* q_start, const int32_t* n_valid, void* out, uint32_t* status,
                        void* workspace, void* stream) {
  const int rc = check_cache(c);
  if (rc != TEMPO_OK) return rc;
  if (a == nullptr || !q || !cache || !page_table || !lens || !out || !status || !workspace) return TEMPO_ERR_NULL;
  if (a->B <= 0 || a->T <= 0 || a->Hq <= 0 || a->Hq % c->Hkv || a->max_pages <= 0 || a->max_q <= 0 || (!q_start && a->B != a->T))
    return TEMPO_ERR_SHAPE;
  if (!pitches(a->ld_q, a->hd_q) || !apart(a->ld_out, a->hd_out, a->T, a->Hq, c->D)) return TEMPO_ERR_SHAPE;
  if (!(a->scale > -1e30f && a->scale < 1e30f)) return TEMPO_ERR_UNSUPPORTED;
  if (a->B > kAttendMaxB || a->Hq > 65536 || static_cast<long long>(a->max_pages) * c->page_size > 0x7fffff00ll ||
      static_cast<long long>(a->T) * (a->Hq / c->Hkv) > 0x7fffff00ll)
    return TEMPO_ERR_UNSUPPORTED;
  if (!vectors8(q, a->ld_q, a->hd_q) || !vectors8(out, a->ld_out, a->hd_out) || !aligned(cache, 16) || !aligned(page_table, 4) ||
      !aligned(lens, 4) || !aligned(q_start, 4) || !aligned(n_valid, 4) || !aligned(status, 4) || !aligned(workspace, 256))
    return TEMPO_ERR_ALIGN;
  const int sms = min(sm_count(), kAttendMaxSms);
  if (sms <= 0) return TEMPO_ERR_CUDA;
  const AttendLayout L = attend_layout(c->D);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  AttendParams p{};
  p.B = a->B; p.T = a->T; p.Hkv = c->Hkv; p.group = a->Hq / c->Hkv;
  p.max_pages = a->max_pages; p.page_size = c->page_size; p.n_pages = c->n_pages;
  while ((1 << p.page_shift) < c->page_size) ++p.page_shift;
  p.q = static_cast<const __nv_bfloat16*>(q); p.cache = static_cast<const uint8_t*>(cache);
  p.page_table = page_table; p.lens = lens; p.q_start = q_start; p.n_valid = n_valid; p.out = static_cast<__nv_bfloat16*>(out);
  p.ld_q = a->ld_q; p.hd_q = a->hd_q; p.ld_out = a->ld_out; p.hd_out = a->hd_out;
  p.wide = aligned(q, 32) && a->ld_q % 16 == 0 && a->hd_q % 16 == 0 && aligned(out, 32) && a->ld_out % 16 == 0 && a->hd_out % 16 == 0;
  p.scale_log2 = a->scale * 1.4426950408889634f; p.status = status;
  p.counters = reinterpret_cast<unsigned int*>(ws + L.off_counters);
  p.groups = reinterpret_cast<unsigned int*>(ws + L.off_groups);
  p.stats = reinterpret_cast<float*>(ws + L.off_stats); p.part = reinterpret_cast<float*>(ws + L.off_out);
  p.wait_ns = kDefaultWaitNs;
  p.idle_ns = 4096 * kDefaultWaitNs;                     // 10^9 tiles, the most of a call, take 14 s on 148 SMs
  return launch_attend(p, a->max_q, c->D, sms, static_cast<cudaStream_t>(stream)) == cudaSuccess ? TEMPO_OK : TEMPO_ERR_CUDA;
}

int tempo_attend(const tempo_attention* a, const tempo_cache* c, const void* q, const void* cache, const int32_t* page_table,
                 const int32_t* lens, const int32_t* q_start, void* out, uint32_t* status, void* workspace, void* stream) {
  return tempo_attend_padded(a, c, q, cache, page_table, lens, q_start, nullptr, out, status, workspace, stream);
}

}  // extern "C"
