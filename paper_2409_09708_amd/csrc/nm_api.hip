// C ABI of the N:M-sparse linear layer: argument validation on the host, then kernel launches on
// the caller's stream.  Declarations and the contract of every call are in include/nm_sparse.h.
#include "nm_sparse.h"

#include "nm_device.h"
#include "nm_launch.h"

#include <atomic>

namespace {

thread_local int32_t g_last_hip_error = 0;

// Scratch of nm_linear_forward_static: device memory that exists as long as the library is loaded, one copy on
// every device the library runs on.  In host code the array's name is only a handle; the memory's address on the
// current device comes from hipGetSymbolAddress (asked once per device) and is what the kernels receive.
constexpr size_t kStaticScratchBytes = (size_t)8 << 20;
__device__ __align__(256) unsigned char scratch[kStaticScratchBytes];
std::atomic<unsigned char*> g_scratch_ptr[nm::kMaxDevices];

hipError_t static_scratch(unsigned char** ptr) {
  int dev = 0;
  hipError_t e = nm::current_device_slot(&dev);
  if (e != hipSuccess) return e;
  unsigned char* p = g_scratch_ptr[dev].load(std::memory_order_acquire);
  if (p == nullptr) {
    void* addr = nullptr;
    if ((e = hipGetSymbolAddress(&addr, HIP_SYMBOL(scratch))) != hipSuccess) return e;
    if (addr == nullptr) return hipErrorInvalidSymbol;
    p = static_cast<unsigned char*>(addr);
    g_scratch_ptr[dev].store(p, std::memory_order_release);
  }
  *ptr = p;
  return hipSuccess;
}

inline int32_t device_status(hipError_t e) {
  if (e == hipSuccess) return NM_OK;
  g_last_hip_error = (int32_t)e;
  return NM_ERR_DEVICE;
}

inline bool level_ok(int32_t N, int32_t M) { return (M == 4 || M == 8 || M == 16) && N >= 1 && N <= M; }

inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// shape of a weight: level first (so that an illegal M never reaches a modulo), then sizes
inline int32_t check_weight(int64_t O, int64_t K, int32_t N, int32_t M) {
  if (!level_ok(N, M)) return NM_ERR_LEVEL;
  if (O <= 0 || K <= 0 || (K % M) != 0) return NM_ERR_SHAPE;
  if (O > (int64_t)1 << 31 || K > (int64_t)1 << 31) return NM_ERR_SHAPE;
  if (O * K > (int64_t)1 << 40) return NM_ERR_SHAPE;  // every launcher's grid (at most one block per 1024 weights) fits 2^31 - 1
  return NM_OK;
}

}  // namespace

extern "C" {

const char* nm_status_string(int32_t status) {
  switch (status) {
    case NM_OK: return "ok";
    case NM_ERR_NULL: return "a required pointer is NULL";
    case NM_ERR_SHAPE: return "illegal shape (sizes must be positive, K a multiple of M, leading dimensions >= row length)";
    case NM_ERR_LEVEL: return "illegal N:M level (M in {4, 8, 16}, 1 <= N <= M)";
    case NM_ERR_ALIGN: return "a pointer is not aligned as documented";
    case NM_ERR_DTYPE: return "unknown output type";
    case NM_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
    case NM_ERR_DEVICE: return "a HIP call failed (see nm_last_hip_error)";
    case NM_ERR_EXHAUSTED: return "random numbers exhausted before a configuration fell into the interval";
    default: return "unknown status";
  }
}

int32_t nm_last_hip_error(void) { return g_last_hip_error; }

size_t nm_values_bytes(int64_t O, int64_t K, int32_t N, int32_t M) {
  if (check_weight(O, K, N, M) != NM_OK) return 0;
  return (size_t)O * (size_t)nm::values_per_row(K, N, M) * sizeof(nm_bf16);
}

size_t nm_index_bytes(int64_t O, int64_t K, int32_t N, int32_t M) {
  if (check_weight(O, K, N, M) != NM_OK) return 0;
  return (size_t)O * (size_t)nm::index_words_per_row(K, N, M) * sizeof(uint32_t);
}

size_t nm_mask_bytes(int64_t O, int64_t K) {
  if (O <= 0 || K <= 0) return 0;
  return (size_t)O * (size_t)nm::mask_words_per_row(K) * sizeof(uint32_t);
}

size_t nm_spmm_workspace_bytes(int64_t O, int64_t K, int32_t N, int32_t M, int64_t T) {
  if (check_weight(O, K, N, M) != NM_OK || T <= 0) return 0;
  return nm::spmm_workspace_bytes(O, K, N, M, T);
}

int32_t nm_prune(const nm_bf16* W, int64_t O, int64_t K, int64_t ldw, int32_t N, int32_t M, uint32_t* mask,
                 nm_bf16* W_masked, void* stream) {
  if (!W || !mask) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, N, M)) return s;
  if (ldw < K) return NM_ERR_SHAPE;
  if (!aligned(W, 2) || !aligned(mask, 4) || !aligned(W_masked, 2)) return NM_ERR_ALIGN;
  return device_status(nm::launch_prune(W, O, K, ldw, N, M, mask, W_masked, (hipStream_t)stream));
}

int32_t nm_pack(const nm_bf16* W, int64_t O, int64_t K, int64_t ldw, int32_t N, int32_t M, const uint32_t* mask,
                nm_bf16* values, uint32_t* indices, void* stream) {
  if (!W || !values || !indices) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, N, M)) return s;
  if (ldw < K) return NM_ERR_SHAPE;
  if (!aligned(W, 2) || !aligned(values, 2) || !aligned(indices, 4) || !aligned(mask, 4)) return NM_ERR_ALIGN;
  return device_status(nm::launch_pack(W, O, K, ldw, N, M, mask, values, indices, (hipStream_t)stream));
}

int32_t nm_pack_batched(const nm_pack_desc* descs, int32_t count, void* stream) {
  if (!descs) return NM_ERR_NULL;
  if (count <= 0) return NM_ERR_SHAPE;
  static_assert(sizeof(nm_pack_desc) == sizeof(nm::PackDesc), "descriptor layouts must match");
  for (int32_t i = 0; i < count; ++i) {
    const nm_pack_desc& d = descs[i];
    if (!d.W || !d.values || !d.indices) return NM_ERR_NULL;
    if (int32_t s = check_weight(d.O, d.K, d.N, d.M)) return s;
    if (!aligned(d.W, 2) || !aligned(d.values, 2) || !aligned(d.indices, 4)) return NM_ERR_ALIGN;
  }
  return device_status(nm::launch_pack_batched(reinterpret_cast<const nm::PackDesc*>(descs), count, (hipStream_t)stream));
}

int32_t nm_pack_prepare_batched(const nm_layer_desc* descs, int32_t count, void* stream) {
  if (!descs) return NM_ERR_NULL;
  if (count <= 0) return NM_ERR_SHAPE;
  static_assert(sizeof(nm_layer_desc) == sizeof(nm::LayerDesc), "descriptor layouts must match");
  for (int32_t i = 0; i < count; ++i) {
    const nm_layer_desc& d = descs[i];
    if (!d.W || !d.values || !d.indices) return NM_ERR_NULL;
    if (int32_t s = check_weight(d.O, d.K, d.N, d.M)) return s;
    if (d.T <= 0 || d.T > (int64_t)1 << 31) return NM_ERR_SHAPE;
    if (!aligned(d.W, 2) || !aligned(d.values, 2) || !aligned(d.indices, 4)) return NM_ERR_ALIGN;
  }
  bool workspace_short = false;
  hipError_t e = nm::launch_pack_prepare_batched(reinterpret_cast<const nm::LayerDesc*>(descs), count,
                                                 (hipStream_t)stream, &workspace_short);
  if (workspace_short) return NM_ERR_WORKSPACE;
  return device_status(e);
}

int32_t nm_unpack(const nm_bf16* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N, int32_t M,
                  nm_bf16* W_dense, int64_t ldw, void* stream) {
  if (!values || !indices || !W_dense) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, N, M)) return s;
  if (ldw < K) return NM_ERR_SHAPE;
  if (!aligned(values, 2) || !aligned(indices, 4) || !aligned(W_dense, 2)) return NM_ERR_ALIGN;
  return device_status(nm::launch_unpack(values, indices, O, K, N, M, W_dense, ldw, (hipStream_t)stream));
}

size_t nm_rank_bytes(int64_t O, int64_t K) {
  if (O <= 0 || K <= 0 || (K % 4) != 0) return 0;
  return (size_t)O * (size_t)K / 2;
}

int32_t nm_rank(const nm_bf16* W, int64_t O, int64_t K, int64_t ldw, int32_t M, uint8_t* rank, void* stream) {
  if (!W || !rank) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, M, M)) return s;
  if (ldw < K) return NM_ERR_SHAPE;
  if (!aligned(W, 2)) return NM_ERR_ALIGN;
  return device_status(nm::launch_rank(W, O, K, ldw, M, rank, (hipStream_t)stream));
}

int32_t nm_rank_batched(const nm_rank_desc* descs, int32_t count, void* stream) {
  if (!descs) return NM_ERR_NULL;
  if (count <= 0) return NM_ERR_SHAPE;
  static_assert(sizeof(nm_rank_desc) == sizeof(nm::RankDesc), "descriptor layouts must match");
  for (int32_t i = 0; i < count; ++i) {
    const nm_rank_desc& d = descs[i];
    if (!d.W || !d.rank) return NM_ERR_NULL;
    if (int32_t s = check_weight(d.O, d.K, d.M, d.M)) return s;
    if (!aligned(d.W, 2)) return NM_ERR_ALIGN;
  }
  return device_status(nm::launch_rank_batched(reinterpret_cast<const nm::RankDesc*>(descs), count, (hipStream_t)stream));
}

int32_t nm_rank_mask(const uint8_t* rank, int64_t O, int64_t K, int32_t N, int32_t M, uint32_t* mask, void* stream) {
  if (!rank || !mask) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, N, M)) return s;
  if (!aligned(mask, 4)) return NM_ERR_ALIGN;
  return device_status(nm::launch_rank_mask(rank, O, K, N, mask, (hipStream_t)stream));
}

int32_t nm_pack_ranked(const nm_bf16* W, const uint8_t* rank, int64_t O, int64_t K, int64_t ldw, int32_t N, int32_t M,
                       nm_bf16* values, uint32_t* indices, void* stream) {
  if (!W || !rank || !values || !indices) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, N, M)) return s;
  if (ldw < K) return NM_ERR_SHAPE;
  if (!aligned(W, 2) || !aligned(values, 2) || !aligned(indices, 4)) return NM_ERR_ALIGN;
  return device_status(nm::launch_pack_ranked(W, rank, O, K, ldw, N, M, values, indices, (hipStream_t)stream));
}

int32_t nm_pack_ranked_batched(const nm_pack_ranked_desc* descs, int32_t count, void* stream) {
  if (!descs) return NM_ERR_NULL;
  if (count <= 0) return NM_ERR_SHAPE;
  static_assert(sizeof(nm_pack_ranked_desc) == sizeof(nm::PackRankedDesc), "descriptor layouts must match");
  for (int32_t i = 0; i < count; ++i) {
    const nm_pack_ranked_desc& d = descs[i];
    if (!d.W || !d.rank || !d.values || !d.indices) return NM_ERR_NULL;
    if (int32_t s = check_weight(d.O, d.K, d.N, d.M)) return s;
    if (!aligned(d.W, 2) || !aligned(d.values, 2) || !aligned(d.indices, 4)) return NM_ERR_ALIGN;
  }
  return device_status(nm::launch_pack_ranked_batched(reinterpret_cast<const nm::PackRankedDesc*>(descs), count,
                                                      (hipStream_t)stream));
}

int32_t nm_mask_check(const uint32_t* mask, int64_t O, int64_t K, int32_t N, int32_t M, uint32_t* bad_groups,
                      void* stream) {
  if (!mask || !bad_groups) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, N, M)) return s;
  if (!aligned(mask, 4) || !aligned(bad_groups, 4)) return NM_ERR_ALIGN;
  return device_status(nm::launch_mask_check(mask, O, K, N, M, bad_groups, (hipStream_t)stream));
}

}  // extern "C"

namespace {

// validation shared by the product calls; fills the launch arguments
int32_t spmm_check(const nm_bf16* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N, int32_t M,
                   const nm_bf16* X, int64_t T, int64_t ldx, const float* bias, void* Y, int64_t ldy, int32_t out_dtype,
                   void* workspace, size_t workspace_bytes, bool product, nm::SpmmArgs* a) {
  if (!values || !indices || (product && (!X || !Y))) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, N, M)) return s;
  if (T <= 0 || T > (int64_t)1 << 31) return NM_ERR_SHAPE;
  if (product && (ldx < K || ldy < O)) return NM_ERR_SHAPE;
  if (out_dtype != NM_OUT_F32 && out_dtype != NM_OUT_BF16) return NM_ERR_DTYPE;
  if (!aligned(values, 2) || !aligned(indices, 4) || !aligned(X, 2) || !aligned(bias, 4) ||
      !aligned(Y, out_dtype == NM_OUT_F32 ? 4 : 2))
    return NM_ERR_ALIGN;
  a->values = values; a->indices = indices; a->O = O; a->K = K; a->N = N; a->M = M;
  a->X = X; a->T = T; a->ldx = product ? ldx : K; a->bias = bias; a->Y = Y; a->ldy = ldy;
  a->out_bf16 = (out_dtype == NM_OUT_BF16);
  a->workspace = workspace; a->workspace_bytes = workspace_bytes;
  a->scratch = nullptr; a->scratch_bytes = 0;
  return NM_OK;
}

int32_t spmm_entry(const nm_bf16* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N, int32_t M,
                   const nm_bf16* X, int64_t T, int64_t ldx, const float* bias, void* Y, int64_t ldy, int32_t out_dtype,
                   void* workspace, size_t workspace_bytes, void* scratch, size_t scratch_bytes, void* stream, int phases) {
  nm::SpmmArgs a;
  if (int32_t st = spmm_check(values, indices, O, K, N, M, X, T, ldx, bias, Y, ldy, out_dtype, workspace, workspace_bytes,
                              phases & nm::SPMM_PRODUCT, &a))
    return st;
  a.scratch = scratch; a.scratch_bytes = scratch_bytes;
  if (phases & nm::SPMM_PREPARE) nm::spmm_scratch_behind_operand(&a);
  bool workspace_short = false;
  hipError_t e = nm::launch_spmm(a, (hipStream_t)stream, &workspace_short, phases);
  if (workspace_short) return NM_ERR_WORKSPACE;
  return device_status(e);
}

int32_t forward_args(const nm_forward_desc& d, nm::SpmmArgs* a) {
  return spmm_check(d.values, d.indices, d.O, d.K, d.N, d.M, d.X, d.T, d.ldx, d.bias, d.Y, d.ldy, d.out_dtype, d.workspace,
                    d.workspace_bytes, true, a);
}
// f(layers, how many) for runs of descriptors, converted without an allocation; ends with the first status that is not NM_OK
template <class F>
int32_t forward_chunks(const nm_forward_desc* descs, int32_t count, F&& f) {
  constexpr int kChunk = 64;
  nm::SpmmArgs layers[kChunk];
  for (int32_t first = 0; first < count; first += kChunk) {
    const int n = count - first < kChunk ? count - first : kChunk;
    for (int i = 0; i < n; ++i)
      if (int32_t st = forward_args(descs[first + i], &layers[i])) return st;
    if (int32_t st = f(layers, n)) return st;
  }
  return NM_OK;
}

// the int8 layer from the dense weight + mask (values == NULL) or from the compressed form (Wq == NULL)
int32_t i8_entry(const int8_t* Wq, int64_t O, int64_t K, int64_t ldw, const uint32_t* mask, const int8_t* values,
                 const uint32_t* indices, int32_t N, int32_t M, const int8_t* Xq, int64_t T, int64_t ldx, float x_scale,
                 const float* w_scale, const float* bias, void* Y, int64_t ldy, int32_t out_dtype, void* workspace,
                 size_t workspace_bytes, void* stream, int phases) {
  const bool product = phases & nm::SPMM_PRODUCT;
  const bool packed = values != nullptr || indices != nullptr;
  if (packed ? (!values || !indices) : (!Wq || !mask)) return NM_ERR_NULL;
  if (product && (!Xq || !Y)) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, N, M)) return s;
  if (T <= 0 || T > (int64_t)1 << 31 || (!packed && ldw < K)) return NM_ERR_SHAPE;
  if (product && (ldx < K || ldy < O)) return NM_ERR_SHAPE;
  if (out_dtype != NM_OUT_F32 && out_dtype != NM_OUT_BF16 && out_dtype != NM_OUT_I32) return NM_ERR_DTYPE;
  if (!aligned(mask, 4) || !aligned(indices, 4) || !aligned(w_scale, 4) || !aligned(bias, 4) ||
      !aligned(Y, out_dtype == NM_OUT_BF16 ? 2 : 4))
    return NM_ERR_ALIGN;
  nm::I8LinearArgs a;
  a.Wq = packed ? nullptr : Wq; a.ldw = ldw; a.mask = mask; a.values = values; a.indices = indices;
  a.O = O; a.K = K; a.N = N; a.M = M;
  a.X = Xq; a.T = T; a.ldx = ldx; a.x_scale = x_scale; a.w_scale = w_scale; a.bias = bias;
  a.Y = Y; a.ldy = ldy; a.out_kind = out_dtype;
  a.workspace = workspace; a.workspace_bytes = workspace_bytes;
  bool workspace_short = false;
  hipError_t e = nm::launch_linear_i8(a, (hipStream_t)stream, &workspace_short, phases);
  if (workspace_short) return NM_ERR_WORKSPACE;
  return device_status(e);
}

}  // namespace

extern "C" {

int32_t nm_linear_forward(const nm_bf16* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N, int32_t M,
                          const nm_bf16* X, int64_t T, int64_t ldx, const float* bias, void* Y, int64_t ldy,
                          int32_t out_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  return spmm_entry(values, indices, O, K, N, M, X, T, ldx, bias, Y, ldy, out_dtype, workspace, workspace_bytes, nullptr, 0,
                    stream, nm::SPMM_PREPARE | nm::SPMM_PRODUCT);
}

int32_t nm_spmm(const nm_bf16* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N, int32_t M,
                const nm_bf16* X, int64_t T, int64_t ldx, void* Y, int64_t ldy, int32_t out_dtype, void* workspace,
                size_t workspace_bytes, void* stream) {
  return spmm_entry(values, indices, O, K, N, M, X, T, ldx, nullptr, Y, ldy, out_dtype, workspace, workspace_bytes,
                    nullptr, 0, stream, nm::SPMM_PREPARE | nm::SPMM_PRODUCT);
}

int32_t nm_spmm_prepare(const nm_bf16* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N, int32_t M,
                        int64_t T, void* workspace, size_t workspace_bytes, void* stream) {
  return spmm_entry(values, indices, O, K, N, M, nullptr, T, K, nullptr, nullptr, O, NM_OUT_F32, workspace,
                    workspace_bytes, nullptr, 0, stream, nm::SPMM_PREPARE);
}

int32_t nm_linear_forward_prepared(const nm_bf16* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N,
                                   int32_t M, const nm_bf16* X, int64_t T, int64_t ldx, const float* bias, void* Y,
                                   int64_t ldy, int32_t out_dtype, const void* workspace, size_t workspace_bytes,
                                   void* stream) {
  return nm_linear_forward_prepared_scratch(values, indices, O, K, N, M, X, T, ldx, bias, Y, ldy, out_dtype, workspace,
                                            workspace_bytes, nullptr, 0, stream);
}

size_t nm_prepared_scratch_bytes(int64_t O, int64_t K, int32_t N, int32_t M, int64_t T) {
  if (check_weight(O, K, N, M) != NM_OK || T <= 0) return 0;
  return nm::spmm_partial_bytes(O, K, N, M, T);
}

int32_t nm_linear_forward_prepared_scratch(const nm_bf16* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N,
                                           int32_t M, const nm_bf16* X, int64_t T, int64_t ldx, const float* bias, void* Y,
                                           int64_t ldy, int32_t out_dtype, const void* workspace, size_t workspace_bytes,
                                           void* scratch, size_t scratch_bytes, void* stream) {
  // (the product alone writes Y and the scratch, never the workspace)
  return spmm_entry(values, indices, O, K, N, M, X, T, ldx, bias, Y, ldy, out_dtype, const_cast<void*>(workspace),
                    workspace_bytes, scratch, scratch_bytes, stream, nm::SPMM_PRODUCT);
}

size_t nm_static_scratch_bytes(void) { return kStaticScratchBytes; }

int32_t nm_linear_forward_static(const nm_bf16* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N,
                                 int32_t M, const nm_bf16* X, int64_t T, int64_t ldx, const float* bias, void* Y,
                                 int64_t ldy, int32_t out_dtype, void* stream) {
  nm::SpmmArgs a;
  if (int32_t st = spmm_check(values, indices, O, K, N, M, X, T, ldx, bias, Y, ldy, out_dtype, nullptr, 0, true, &a))
    return st;
  if (nm::spmm_operand_workspace_bytes(O, K, N, M, T) > kStaticScratchBytes) return NM_ERR_WORKSPACE;
  unsigned char* ws = nullptr;
  if (int32_t st = device_status(static_scratch(&ws))) return st;
  a.workspace = ws;
  a.workspace_bytes = kStaticScratchBytes;
  nm::spmm_scratch_behind_operand(&a);
  bool workspace_short = false;
  hipError_t e = nm::launch_spmm_on_scratch(a, (hipStream_t)stream, &workspace_short);
  if (workspace_short) return NM_ERR_WORKSPACE;
  return device_status(e);
}

size_t nm_backward_weight_workspace_bytes(int64_t O, int64_t K, int64_t T) {
  if (O <= 0 || K <= 0 || T <= 0) return 0;
  return nm::backward_weight_workspace_bytes(O, K, T);
}

size_t nm_backward_input_workspace_bytes(int64_t O, int64_t K, int64_t T) {
  if (O <= 0 || K <= 0 || T <= 0) return 0;
  return nm::backward_input_workspace_bytes(O, K, T);
}

namespace {
int32_t backward_input(const nm_bf16* Ws, int64_t O, int64_t K, int64_t ldw, const nm_bf16* dY, int64_t T, int64_t ldy, void* dX,
                       int64_t ldx, int32_t out_dtype, void* workspace, size_t workspace_bytes, void* stream, bool optional) {
  if (!Ws || !dY || !dX) return NM_ERR_NULL;
  if (O <= 0 || K <= 0 || T <= 0 || O > (int64_t)1 << 31 || K > (int64_t)1 << 31 || T > (int64_t)1 << 31)
    return NM_ERR_SHAPE;
  if (ldw < K || ldy < O || ldx < K) return NM_ERR_SHAPE;
  if (out_dtype != NM_OUT_F32 && out_dtype != NM_OUT_BF16) return NM_ERR_DTYPE;
  if (!aligned(Ws, 2) || !aligned(dY, 2) || !aligned(dX, out_dtype == NM_OUT_F32 ? 4 : 2)) return NM_ERR_ALIGN;
  bool workspace_short = false;
  hipError_t e = nm::launch_backward_input(Ws, O, K, ldw, dY, T, ldy, dX, ldx, out_dtype == NM_OUT_BF16, workspace,
                                           workspace_bytes, (hipStream_t)stream, optional, &workspace_short);
  if (workspace_short) return NM_ERR_WORKSPACE;
  return device_status(e);
}
}  // namespace

int32_t nm_linear_backward_input(const nm_bf16* Ws, int64_t O, int64_t K, int64_t ldw, const nm_bf16* dY, int64_t T,
                                 int64_t ldy, void* dX, int64_t ldx, int32_t out_dtype, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  return backward_input(Ws, O, K, ldw, dY, T, ldy, dX, ldx, out_dtype, workspace, workspace_bytes, stream, false);
}

size_t nm_backward_input_scratch_bytes(int64_t O, int64_t K, int64_t T) {
  if (O <= 0 || K <= 0 || T <= 0) return 0;
  return nm::backward_input_scratch_bytes(O, K, T);
}

int32_t nm_backward_input_scratch_pays(int64_t O, int64_t K, int64_t T, int32_t out_dtype, void* stream) {
  if (O <= 0 || K <= 0 || T <= 0) return 0;
  return nm::backward_input_scratch_pays(O, K, T, out_dtype == NM_OUT_BF16, (hipStream_t)stream);
}

int32_t nm_linear_backward_input_scratch(const nm_bf16* Ws, int64_t O, int64_t K, int64_t ldw, const nm_bf16* dY, int64_t T,
                                         int64_t ldy, void* dX, int64_t ldx, int32_t out_dtype, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  return backward_input(Ws, O, K, ldw, dY, T, ldy, dX, ldx, out_dtype, workspace, workspace_bytes, stream, true);
}

namespace {
int32_t backward_weight(const nm_bf16* dY, int64_t T, int64_t O, int64_t ldy, const nm_bf16* X, int64_t K,
                                  int64_t ldx, const uint32_t* mask, void* dW, int64_t lddw, int32_t out_dtype,
                                  void* workspace, size_t workspace_bytes, void* stream, bool used_only) {
  if (!dY || !X || !dW) return NM_ERR_NULL;
  if (O <= 0 || K <= 0 || T <= 0 || O > (int64_t)1 << 31 || K > (int64_t)1 << 31 || T > (int64_t)1 << 31)
    return NM_ERR_SHAPE;
  if (ldy < O || ldx < K || lddw < K) return NM_ERR_SHAPE;
  if (out_dtype != NM_OUT_F32 && out_dtype != NM_OUT_BF16) return NM_ERR_DTYPE;
  if (!aligned(dY, 2) || !aligned(X, 2) || !aligned(mask, 4) || !aligned(dW, out_dtype == NM_OUT_F32 ? 4 : 2))
    return NM_ERR_ALIGN;
  bool workspace_short = false;
  hipError_t e = nm::launch_backward_weight(dY, T, O, ldy, X, K, ldx, mask, dW, lddw, out_dtype == NM_OUT_BF16, workspace,
                                            workspace_bytes, (hipStream_t)stream, used_only, &workspace_short);
  if (workspace_short) return NM_ERR_WORKSPACE;
  return device_status(e);
}
}  // namespace

int32_t nm_linear_backward_weight(const nm_bf16* dY, int64_t T, int64_t O, int64_t ldy, const nm_bf16* X, int64_t K,
                                  int64_t ldx, const uint32_t* mask, void* dW, int64_t lddw, int32_t out_dtype,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  return backward_weight(dY, T, O, ldy, X, K, ldx, mask, dW, lddw, out_dtype, workspace, workspace_bytes, stream, false);
}

size_t nm_backward_weight_scratch_bytes(int64_t O, int64_t K, int64_t T) {
  if (O <= 0 || K <= 0 || T <= 0) return 0;
  return nm::backward_weight_scratch_bytes(O, K, T);
}

int32_t nm_linear_backward_weight_scratch(const nm_bf16* dY, int64_t T, int64_t O, int64_t ldy, const nm_bf16* X, int64_t K,
                                  int64_t ldx, const uint32_t* mask, void* dW, int64_t lddw, int32_t out_dtype,
                                  void* workspace, size_t workspace_bytes, void* stream) {
  return backward_weight(dY, T, O, ldy, X, K, ldx, mask, dW, lddw, out_dtype, workspace, workspace_bytes, stream, true);
}

size_t nm_i8_workspace_bytes(int64_t O, int64_t K, int32_t N, int32_t M, int64_t T) {
  if (check_weight(O, K, N, M) != NM_OK || T <= 0) return 0;
  return nm::i8_workspace_bytes(O, K, N, M, T);
}

int32_t nm_linear_forward_i8(const int8_t* Wq, int64_t O, int64_t K, int64_t ldw, const uint32_t* mask, int32_t N,
                             int32_t M, const int8_t* Xq, int64_t T, int64_t ldx, float x_scale, const float* w_scale,
                             const float* bias, void* Y, int64_t ldy, int32_t out_dtype, void* workspace,
                             size_t workspace_bytes, void* stream) {
  return i8_entry(Wq, O, K, ldw, mask, nullptr, nullptr, N, M, Xq, T, ldx, x_scale, w_scale, bias, Y, ldy, out_dtype, workspace,
                  workspace_bytes, stream, nm::SPMM_PREPARE | nm::SPMM_PRODUCT);
}

int32_t nm_i8_prepare(const int8_t* Wq, int64_t O, int64_t K, int64_t ldw, const uint32_t* mask, int32_t N, int32_t M,
                      int64_t T, void* workspace, size_t workspace_bytes, void* stream) {
  return i8_entry(Wq, O, K, ldw, mask, nullptr, nullptr, N, M, nullptr, T, K, 1.f, nullptr, nullptr, nullptr, O, NM_OUT_F32,
                  workspace, workspace_bytes, stream, nm::SPMM_PREPARE);
}

int32_t nm_linear_forward_i8_prepared(const int8_t* Wq, int64_t O, int64_t K, int64_t ldw, const uint32_t* mask,
                                      int32_t N, int32_t M, const int8_t* Xq, int64_t T, int64_t ldx, float x_scale,
                                      const float* w_scale, const float* bias, void* Y, int64_t ldy, int32_t out_dtype,
                                      void* workspace, size_t workspace_bytes, void* stream) {
  return i8_entry(Wq, O, K, ldw, mask, nullptr, nullptr, N, M, Xq, T, ldx, x_scale, w_scale, bias, Y, ldy, out_dtype, workspace,
                  workspace_bytes, stream, nm::SPMM_PRODUCT);
}

size_t nm_values_i8_bytes(int64_t O, int64_t K, int32_t N, int32_t M) {
  if (check_weight(O, K, N, M) != NM_OK) return 0;
  return (size_t)O * (size_t)nm::values_per_row(K, N, M);
}

int32_t nm_pack_i8(const int8_t* Wq, int64_t O, int64_t K, int64_t ldw, int32_t N, int32_t M, const uint32_t* mask,
                   int8_t* values, uint32_t* indices, void* stream) {
  if (!Wq || !mask || !values || !indices) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, N, M)) return s;
  if (ldw < K) return NM_ERR_SHAPE;
  if (!aligned(mask, 4) || !aligned(indices, 4)) return NM_ERR_ALIGN;
  return device_status(nm::launch_pack_i8(Wq, O, K, ldw, N, M, mask, values, indices, (hipStream_t)stream));
}

int32_t nm_unpack_i8(const int8_t* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N, int32_t M,
                     int8_t* Wq_dense, int64_t ldw, void* stream) {
  if (!values || !indices || !Wq_dense) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, N, M)) return s;
  if (ldw < K) return NM_ERR_SHAPE;
  if (!aligned(indices, 4)) return NM_ERR_ALIGN;
  return device_status(nm::launch_unpack_i8(values, indices, O, K, N, M, Wq_dense, ldw, (hipStream_t)stream));
}

int32_t nm_linear_forward_i8_packed(const int8_t* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N,
                                    int32_t M, const int8_t* Xq, int64_t T, int64_t ldx, float x_scale,
                                    const float* w_scale, const float* bias, void* Y, int64_t ldy, int32_t out_dtype,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!values || !indices) return NM_ERR_NULL;
  return i8_entry(nullptr, O, K, K, nullptr, values, indices, N, M, Xq, T, ldx, x_scale, w_scale, bias, Y, ldy, out_dtype,
                  workspace, workspace_bytes, stream, nm::SPMM_PREPARE | nm::SPMM_PRODUCT);
}

int32_t nm_i8_prepare_packed(const int8_t* values, const uint32_t* indices, int64_t O, int64_t K, int32_t N, int32_t M,
                             int64_t T, void* workspace, size_t workspace_bytes, void* stream) {
  if (!values || !indices) return NM_ERR_NULL;
  return i8_entry(nullptr, O, K, K, nullptr, values, indices, N, M, nullptr, T, K, 1.f, nullptr, nullptr, nullptr, O,
                  NM_OUT_F32, workspace, workspace_bytes, stream, nm::SPMM_PREPARE);
}

int32_t nm_linear_forward_i8_packed_prepared(const int8_t* values, const uint32_t* indices, int64_t O, int64_t K,
                                             int32_t N, int32_t M, const int8_t* Xq, int64_t T, int64_t ldx,
                                             float x_scale, const float* w_scale, const float* bias, void* Y,
                                             int64_t ldy, int32_t out_dtype, void* workspace, size_t workspace_bytes,
                                             void* stream) {
  if (!values || !indices) return NM_ERR_NULL;
  return i8_entry(nullptr, O, K, K, nullptr, values, indices, N, M, Xq, T, ldx, x_scale, w_scale, bias, Y, ldy, out_dtype,
                  workspace, workspace_bytes, stream, nm::SPMM_PRODUCT);
}

int32_t nm_prune_scored(const float* score, int64_t O, int64_t K, int64_t lds, int32_t N, int32_t M, uint32_t* mask,
                        void* stream) {
  if (!score || !mask) return NM_ERR_NULL;
  if (int32_t s = check_weight(O, K, N, M)) return s;
  if (lds < K) return NM_ERR_SHAPE;
  if (!aligned(score, 4) || !aligned(mask, 4)) return NM_ERR_ALIGN;
  return device_status(nm::launch_score_mask(score, O, K, lds, N, M, mask, (hipStream_t)stream));
}

namespace {
constexpr int64_t kMost = (int64_t)1 << 31, kMostColumns = (int64_t)1 << 24;
inline bool type_ok(int32_t t) { return t == NM_OUT_F32 || t == NM_OUT_BF16; }
inline bool type_aligned(const void* p, int32_t t) { return aligned(p, t == NM_OUT_F32 ? 4 : 2); }
inline bool workspace_ok(const void* p, size_t bytes, size_t need) { return need == 0 || (p && bytes >= need && aligned(p, 256)); }

// rows of D elements at two strides: an input may repeat itself, an output's rows must not overlap
inline bool strides_ok(int64_t T, int64_t H, int64_t D, int64_t token, int64_t head, bool output) {
  if (token < 0 || head < 0) return false;
  if (!output) return true;
  if (T == 1 || H == 1) return (T == 1 || token >= D) && (H == 1 || head >= D);
  // the heads of a token side by side (or those of all tokens, head after head)
  return (head >= D && token >= (H - 1) * head + D) || (token >= D && head >= (T - 1) * token + D);
}
// The rotary turn of a call: the pairs of each axis.
int32_t rotary_check(const int32_t* sections, int32_t axes, int64_t rotated, int64_t D, int (&section_end)[nm::kMaxRotaryAxes]) {
  if (rotated <= 0 || rotated > D || rotated % 2 || axes < 1 || axes > nm::kMaxRotaryAxes) return NM_ERR_SHAPE;
  int64_t end = 0;
  for (int x = 0; x < nm::kMaxRotaryAxes; ++x) {
    if (x < axes && (sections[x] < 0 || sections[x] > rotated / 2)) return NM_ERR_SHAPE;
    end += x < axes ? sections[x] : 0;
    section_end[x] = x < axes - 1 ? (int)end : (int)(rotated / 2);
  }
  return end == rotated / 2 ? NM_OK : NM_ERR_SHAPE;
}
}  // namespace

int32_t nm_layer_norm(const void* X, int64_t ldx, int32_t x_dtype, const void* R, int64_t ldr, int64_t T, int64_t C,
                      const float* weight, const float* bias, float eps, void* Y, int64_t ldy, int32_t y_dtype, void* S,
                      int64_t lds, float* stats, void* stream) {
  if (!X || !Y) return NM_ERR_NULL;
  if (T <= 0 || C <= 0 || T > kMost || C > kMostColumns || T * C > (int64_t)1 << 40) return NM_ERR_SHAPE;
  const bool sum = R != nullptr && S != nullptr;
  if (ldx < C || ldy < C || (R && ldr < C) || (sum && lds < C) || !(eps >= 0.f)) return NM_ERR_SHAPE;
  if (!type_ok(x_dtype) || !type_ok(y_dtype)) return NM_ERR_DTYPE;
  if (!type_aligned(X, x_dtype) || !type_aligned(R, x_dtype) || !type_aligned(S, x_dtype) || !type_aligned(Y, y_dtype) ||
      !aligned(weight, 4) || !aligned(bias, 4) || !aligned(stats, 8))
    return NM_ERR_ALIGN;
  nm::NormCall c;
  c.X = X; c.R = R; c.w = weight; c.b = bias; c.Y = Y; c.S = sum ? S : nullptr; c.stats = stats;
  c.T = T; c.C = C; c.ldx = ldx; c.ldr = ldr; c.ldy = ldy; c.lds = lds; c.eps = eps;
  c.x_f32 = x_dtype == NM_OUT_F32; c.y_f32 = y_dtype == NM_OUT_F32;
  return device_status(nm::launch_norm(c, (hipStream_t)stream));
}

size_t nm_layer_norm_backward_workspace_bytes(int64_t T, int64_t C) {
  if (T <= 0 || C <= 0 || T > kMost || C > kMostColumns) return 0;
  return nm::norm_grad_workspace_bytes(T, C);
}

int32_t nm_layer_norm_backward(const void* dY, int64_t lddy, int32_t dy_dtype, const void* S, int64_t lds, int32_t s_dtype,
                               const float* stats, const float* weight, const void* dS, int64_t ldds, int64_t T, int64_t C,
                               void* dX, int64_t lddx, int32_t dx_dtype, float* dweight, float* dbias, void* workspace,
                               size_t workspace_bytes, void* stream) {
  if (!dY || !S || !stats || !dX || (dweight == nullptr) != (dbias == nullptr)) return NM_ERR_NULL;
  if (T <= 0 || C <= 0 || T > kMost || C > kMostColumns || T * C > (int64_t)1 << 40) return NM_ERR_SHAPE;
  if (lddy < C || lds < C || lddx < C || (dS && ldds < C)) return NM_ERR_SHAPE;
  if (!type_ok(dy_dtype) || !type_ok(s_dtype) || !type_ok(dx_dtype)) return NM_ERR_DTYPE;
  if (!type_aligned(dY, dy_dtype) || !type_aligned(dS, dy_dtype) || !type_aligned(S, s_dtype) || !type_aligned(dX, dx_dtype) ||
      !aligned(stats, 8) || !aligned(weight, 4) || !aligned(dweight, 4) || !aligned(dbias, 4))
    return NM_ERR_ALIGN;
  if (dweight && !workspace_ok(workspace, workspace_bytes, nm::norm_grad_workspace_bytes(T, C))) return NM_ERR_WORKSPACE;
  nm::NormGradCall c;
  c.dY = dY; c.S = S; c.stats = stats; c.w = weight; c.dS = dS; c.dX = dX; c.dw = dweight; c.db = dbias;
  c.T = T; c.C = C; c.lddy = lddy; c.lds = lds; c.ldds = ldds; c.lddx = lddx;
  c.dy_f32 = dy_dtype == NM_OUT_F32; c.s_f32 = s_dtype == NM_OUT_F32; c.dx_f32 = dx_dtype == NM_OUT_F32;
  c.workspace = workspace;
  return device_status(nm::launch_norm_grad(c, (hipStream_t)stream));
}

int32_t nm_rotary(const void* X, int32_t x_dtype, int64_t T, int64_t H, int64_t D, int64_t x_token, int64_t x_head,
                  const void* positions, int32_t positions_f32, const float* freqs, const int32_t* sections, int32_t axes,
                  int64_t rotated, int32_t interleaved, int32_t inverse, void* Y, int32_t y_dtype, int64_t y_token,
                  int64_t y_head, void* stream) {
  if (!X || !Y || !positions || !freqs || !sections) return NM_ERR_NULL;
  if (T <= 0 || H <= 0 || D <= 0 || T > kMost || H > 1 << 20 || D > 1 << 20 || H * D > 1 << 20) return NM_ERR_SHAPE;
  nm::RotaryCall c;
  if (int32_t st = rotary_check(sections, axes, rotated, D, c.section_end)) return st;
  if (!strides_ok(T, H, D, x_token, x_head, false) || !strides_ok(T, H, D, y_token, y_head, true)) return NM_ERR_SHAPE;
  if (!type_ok(x_dtype) || !type_ok(y_dtype)) return NM_ERR_DTYPE;
  if (!type_aligned(X, x_dtype) || !type_aligned(Y, y_dtype) || !aligned(positions, 4) || !aligned(freqs, 4)) return NM_ERR_ALIGN;
  c.X = X; c.Y = Y; c.positions = positions; c.freqs = freqs;
  c.T = T; c.H = H; c.D = D; c.R = rotated;
  c.x_token = x_token; c.x_head = x_head; c.y_token = y_token; c.y_head = y_head;
  c.axes = axes;
  c.positions_f32 = positions_f32 != 0; c.interleaved = interleaved != 0; c.inverse = inverse != 0;
  c.x_f32 = x_dtype == NM_OUT_F32; c.y_f32 = y_dtype == NM_OUT_F32;
  return device_status(nm::launch_rotary(c, (hipStream_t)stream));
}

namespace {
constexpr int64_t kMostTokens = (int64_t)1 << 30;
bool attention_sizes_ok(int64_t Tq, int64_t sequences, int64_t heads_q, int64_t heads_kv, int64_t head_size, int64_t max_q,
                        int64_t max_k) {
  return Tq > 0 && Tq <= kMostTokens && sequences >= 1 && sequences <= 65535 && heads_q >= 1 && heads_kv >= 1 &&
         heads_q % heads_kv == 0 && sequences * heads_q <= 1 << 20 && head_size >= 1 && head_size <= 128 && max_q >= 0 && max_k >= 0;
}

int32_t attention_check(const nm_attention_desc* d, bool backward, nm::AttentionCall* c) {
  if (!d) return NM_ERR_NULL;
  const bool keys = d->Tk != 0;
  if (!d->Q.data || !d->O.data || (keys && (!d->K.data || !d->V.data))) return NM_ERR_NULL;
  if (backward && (!d->dO.data || !d->dQ.data || (keys && (!d->dK.data || !d->dV.data)) || !d->lse)) return NM_ERR_NULL;
  if ((!d->offsets_q || !d->offsets_k) && d->sequences != 1) return d->sequences < 1 ? NM_ERR_SHAPE : NM_ERR_NULL;
  if (!attention_sizes_ok(d->Tq, d->sequences, d->heads_q, d->heads_kv, d->head_size, d->max_q, d->max_k)) return NM_ERR_SHAPE;
  if (d->Tk < 0 || d->Tk > kMostTokens) return NM_ERR_SHAPE;
  if (!(d->scale > 0.f) || d->scale > 3.0e38f) return NM_ERR_SHAPE;
  auto take = [&](const nm_heads& h, nm::HeadRows* r, int64_t T, int64_t H, bool output) {
    *r = nm::HeadRows{h.data, h.token, h.head};
    return T == 0 || strides_ok(T, H, d->head_size, h.token, h.head, output);
  };
  *c = nm::AttentionCall{};
  if (!take(d->Q, &c->Q, d->Tq, d->heads_q, false) || !take(d->K, &c->K, d->Tk, d->heads_kv, false) ||
      !take(d->V, &c->V, d->Tk, d->heads_kv, false) || !take(d->O, &c->O, d->Tq, d->heads_q, !backward))
    return NM_ERR_SHAPE;
  if (backward && (!take(d->dO, &c->dO, d->Tq, d->heads_q, false) || !take(d->dQ, &c->dQ, d->Tq, d->heads_q, true) ||
                   !take(d->dK, &c->dK, d->Tk, d->heads_kv, true) || !take(d->dV, &c->dV, d->Tk, d->heads_kv, true)))
    return NM_ERR_SHAPE;
  for (const void* p : {d->Q.data, d->K.data, d->V.data, d->O.data, c->dO.p, c->dQ.p, c->dK.p, c->dV.p})
    if (!aligned(p, 2)) return NM_ERR_ALIGN;
  for (const void* p : {(const void*)d->lse, (const void*)d->offsets_q, (const void*)d->offsets_k, (const void*)d->lengths_k})
    if (!aligned(p, 4)) return NM_ERR_ALIGN;
  c->lse = d->lse; c->offsets_q = d->offsets_q; c->offsets_k = d->offsets_k; c->lengths_k = d->lengths_k;
  c->Tq = d->Tq; c->Tk = d->Tk;
  c->B = d->sequences; c->Hq = d->heads_q; c->Hkv = d->heads_kv; c->D = d->head_size;
  c->max_q = d->max_q < d->Tq ? d->max_q : d->Tq;
  c->max_k = d->max_k < d->Tk ? d->max_k : d->Tk;
  c->causal = d->causal != 0;
  c->scale = d->scale;
  return NM_OK;
}
}  // namespace

size_t nm_attention_workspace_bytes(int64_t Tq, int32_t sequences, int32_t heads_q, int32_t heads_kv, int32_t head_size,
                                    int64_t max_q, int64_t max_k) {
  if (!attention_sizes_ok(Tq, sequences, heads_q, heads_kv, head_size, max_q, max_k)) return 0;
  // (the call cuts max_k to its number of keys, which this does not know)
  return nm::attention_workspace_most(Tq, sequences, heads_q, heads_kv, head_size, max_q < Tq ? max_q : Tq, max_k < kMostTokens ? max_k : kMostTokens);
}

int32_t nm_attention(const nm_attention_desc* desc, void* workspace, size_t workspace_bytes, void* stream) {
  nm::AttentionCall c;
  if (int32_t st = attention_check(desc, false, &c)) return st;
  if (!workspace_ok(workspace, workspace_bytes, nm::attention_workspace_bytes(c.Tq, c.B, c.Hq, c.Hkv, c.D, c.max_q, c.max_k)))
    return NM_ERR_WORKSPACE;
  c.workspace = workspace;
  return device_status(nm::launch_attention(c, (hipStream_t)stream));
}

size_t nm_attention_backward_workspace_bytes(int64_t Tq, int64_t Tk, int32_t sequences, int32_t heads_q, int32_t heads_kv,
                                             int32_t head_size, int64_t max_q, int64_t max_k, int32_t causal) {
  if (!attention_sizes_ok(Tq, sequences, heads_q, heads_kv, head_size, max_q, max_k) || Tk < 0 || Tk > kMostTokens) return 0;
  return nm::attention_grad_workspace_bytes(Tq, Tk, sequences, heads_q, heads_kv, head_size, max_q < Tq ? max_q : Tq,
                                            max_k < Tk ? max_k : Tk, causal != 0);
}

int32_t nm_attention_backward(const nm_attention_desc* desc, void* workspace, size_t workspace_bytes, void* stream) {
  nm::AttentionCall c;
  if (int32_t st = attention_check(desc, true, &c)) return st;
  if (!workspace_ok(workspace, workspace_bytes, nm::attention_grad_workspace_bytes(c.Tq, c.Tk, c.B, c.Hq, c.Hkv, c.D, c.max_q,
                                                                                 c.max_k, c.causal)))
    return NM_ERR_WORKSPACE;
  c.workspace = workspace;
  return device_status(nm::launch_attention_grad(c, (hipStream_t)stream));
}

namespace {
int32_t head_norm_check(const nm_head_norm_desc* d, bool backward, nm::HeadNormCall* c) {
  if (!d || !d->X.data || !d->Y.data || (backward && !d->dY.data)) return NM_ERR_NULL;
  const bool turned = d->positions != nullptr;
  if (turned && (!d->freqs || !d->sections)) return NM_ERR_NULL;
  if (backward && d->dweight && !d->weight) return NM_ERR_NULL;
  const int64_t T = d->T, H = d->H, D = d->D;
  if (T <= 0 || H <= 0 || D <= 0 || T > kMost || H > 1 << 20 || D > 512 || H * D > 1 << 20) return NM_ERR_SHAPE;
  if (d->heads < 1 || d->heads > H || !(d->eps >= 0.f)) return NM_ERR_SHAPE;
  *c = nm::HeadNormCall{};
  if (turned)
    if (int32_t st = rotary_check(d->sections, d->axes, d->rotated, D, c->section_end)) return st;
  if (!strides_ok(T, H, D, d->X.token, d->X.head, false) || !strides_ok(T, H, D, d->Y.token, d->Y.head, true) ||
      (backward && !strides_ok(T, H, D, d->dY.token, d->dY.head, false)))
    return NM_ERR_SHAPE;
  if (!type_ok(d->X.dtype) || !type_ok(d->Y.dtype) || (backward && !type_ok(d->dY.dtype))) return NM_ERR_DTYPE;
  if (!type_aligned(d->X.data, d->X.dtype) || !type_aligned(d->Y.data, d->Y.dtype) || (backward && !type_aligned(d->dY.data, d->dY.dtype)))
    return NM_ERR_ALIGN;
  for (const void* p : {(const void*)d->weight, (const void*)d->dweight, d->positions, (const void*)d->freqs})
    if (!aligned(p, 4)) return NM_ERR_ALIGN;
  c->X = d->X.data; c->Y = d->Y.data; c->w = d->weight;
  c->T = T; c->H = H; c->D = D; c->heads = d->heads;
  // (a stride over one token, or one head, is not used)
  auto stride = [](int64_t s, int64_t n) { return n == 1 ? (int64_t)0 : s; };
  c->x_token = stride(d->X.token, T); c->x_head = stride(d->X.head, H);
  c->y_token = stride(d->Y.token, T); c->y_head = stride(d->Y.head, H);
  if (backward) {
    c->dy_token = stride(d->dY.token, T);
    c->dy_head = stride(d->dY.head, H);
  }
  for (int64_t s : {c->x_token, c->x_head, c->y_token, c->y_head, c->dy_token, c->dy_head})
    if (s > 0x7FFFFFFF) return NM_ERR_SHAPE;
  c->eps = d->eps; c->centred = d->centred != 0;
  c->x_f32 = d->X.dtype == NM_OUT_F32; c->y_f32 = d->Y.dtype == NM_OUT_F32;
  if (turned) {
    c->R = d->rotated; c->axes = d->axes; c->positions = d->positions; c->freqs = d->freqs;
    c->positions_f32 = d->positions_f32 != 0; c->interleaved = d->interleaved != 0;
  }
  if (backward) {
    c->dY = d->dY.data; c->dy_f32 = d->dY.dtype == NM_OUT_F32;
    c->dw = d->dweight;
  }
  return NM_OK;
}
}  // namespace

int32_t nm_head_norm(const nm_head_norm_desc* desc, void* stream) {
  nm::HeadNormCall c;
  if (int32_t st = head_norm_check(desc, false, &c)) return st;
  return device_status(nm::launch_head_norm(c, (hipStream_t)stream));
}

size_t nm_head_norm_backward_workspace_bytes(int64_t T, int64_t H, int64_t heads, int64_t D, int64_t rotated) {
  if (T <= 0 || H <= 0 || D <= 0 || T > kMost || H > 1 << 20 || D > 512 || H * D > 1 << 20 || heads < 1 || heads > H) return 0;
  if (rotated < 0 || rotated > D || rotated % 2) return 0;
  return nm::head_norm_grad_workspace_bytes(T, H, heads, D, rotated);
}

int32_t nm_head_norm_backward(const nm_head_norm_desc* desc, void* workspace, size_t workspace_bytes, void* stream) {
  nm::HeadNormCall c;
  if (int32_t st = head_norm_check(desc, true, &c)) return st;
  if (c.dw && !workspace_ok(workspace, workspace_bytes, nm::head_norm_grad_workspace_bytes(c.T, c.H, c.heads, c.D, c.R)))
    return NM_ERR_WORKSPACE;
  c.workspace = workspace;
  return device_status(nm::launch_head_norm_grad(c, (hipStream_t)stream));
}

namespace {
constexpr int64_t kMostPageTokens = (int64_t)1 << 30;
// whether elements of three nested strides, `extent` of them in a row, are all different places
bool apart(int64_t extent, int64_t s0, int64_t n0, int64_t s1, int64_t n1, int64_t s2, int64_t n2) {
  int64_t s[3] = {s0, s1, s2}, n[3] = {n0, n1, n2};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (s[j] > s[j + 1]) {
        const int64_t t = s[j], m = n[j];
        s[j] = s[j + 1]; n[j] = n[j + 1];
        s[j + 1] = t; n[j + 1] = m;
      }
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) continue;
    if (s[i] < extent) return false;
    extent += s[i] * (n[i] - 1);
  }
  return true;
}

int32_t pages_check(const nm_pages* d, bool written, nm::PagesCall* c) {
  if (!d || !d->K || !d->V || !d->table || !d->lengths) return NM_ERR_NULL;
  if (d->dtype != NM_OUT_BF16 && d->dtype != NM_E4M3) return NM_ERR_DTYPE;
  const bool codes = d->dtype == NM_E4M3;
  if (codes && (!d->K_scales || !d->V_scales)) return NM_ERR_NULL;
  if (d->pages < 1 || d->pages > 0x7FFFFFFF || d->page_size < 1 || d->page_size > 1 << 20 || d->table_width < 1 ||
      (int64_t)d->table_width * d->page_size > kMostPageTokens)
    return NM_ERR_SHAPE;
  if (d->sequences < 1 || d->sequences > 65535 || d->heads < 1 || (int64_t)d->sequences * d->heads > 1 << 20 || d->head_size < 1 ||
      d->head_size > 128)
    return NM_ERR_SHAPE;
  const int64_t most = (int64_t)1 << 40;
  for (int64_t s : {d->page, d->token, d->head, d->scale_page, d->scale_token, d->scale_head})
    if (s < 0 || s > most) return NM_ERR_SHAPE;
  if (written && (!apart(d->head_size, d->page, d->pages, d->token, d->page_size, d->head, d->heads) ||
                  (codes && !apart(1, d->scale_page, d->pages, d->scale_token, d->page_size, d->scale_head, d->heads))))
    return NM_ERR_SHAPE;
  if (!aligned(d->K, codes ? 1 : 2) || !aligned(d->V, codes ? 1 : 2) || !aligned(d->table, 4) || !aligned(d->lengths, 4)) return NM_ERR_ALIGN;
  c->K = d->K; c->V = d->V; c->K_scales = d->K_scales; c->V_scales = d->V_scales;
  c->page = d->page; c->token = d->token; c->head = d->head;
  c->scale_page = d->scale_page; c->scale_token = d->scale_token; c->scale_head = d->scale_head;
  c->table = d->table; c->lengths = d->lengths; c->pages = d->pages;
  c->page_size = d->page_size; c->width = d->table_width; c->B = d->sequences; c->H = d->heads; c->D = d->head_size;
  c->e4m3 = codes;
  return NM_OK;
}

// packed tokens beside a cache: K and V, their offsets
int32_t packed_check(const nm_pages& d, const nm_heads* K, const nm_heads* V, const int32_t* offsets, int64_t T, bool output, nm::HeadRows* k,
                     nm::HeadRows* v) {
  if (!K || !V || !K->data || !V->data) return NM_ERR_NULL;
  if (T <= 0 || T > kMostTokens || (!offsets && T % d.sequences)) return NM_ERR_SHAPE;
  if (!strides_ok(T, d.heads, d.head_size, K->token, K->head, output) || !strides_ok(T, d.heads, d.head_size, V->token, V->head, output))
    return NM_ERR_SHAPE;
  if (!aligned(K->data, 2) || !aligned(V->data, 2) || !aligned(offsets, 4)) return NM_ERR_ALIGN;
  *k = nm::HeadRows{K->data, K->token, K->head};
  *v = nm::HeadRows{V->data, V->token, V->head};
  return NM_OK;
}
}  // namespace

int32_t nm_cache_write(const nm_pages* pages, const nm_heads* K, const nm_heads* V, const int32_t* offsets, int64_t T, void* stream) {
  nm::CacheWriteCall c = {};
  if (int32_t st = pages_check(pages, true, &c.p)) return st;
  if (int32_t st = packed_check(*pages, K, V, offsets, T, false, &c.K, &c.V)) return st;
  c.offsets = offsets;
  c.T = T;
  return device_status(nm::launch_cache_write(c, (hipStream_t)stream));
}

int32_t nm_cache_read(const nm_pages* pages, const nm_heads* K, const nm_heads* V, const int32_t* offsets, const int32_t* first, int64_t T,
                      void* stream) {
  nm::CacheReadCall c = {};
  if (int32_t st = pages_check(pages, false, &c.p)) return st;
  if (int32_t st = packed_check(*pages, K, V, offsets, T, true, &c.K, &c.V)) return st;
  if (!aligned(first, 4)) return NM_ERR_ALIGN;
  c.offsets = offsets;
  c.first = first;
  c.T = T;
  return device_status(nm::launch_cache_read(c, (hipStream_t)stream));
}

namespace {
bool paged_sizes_ok(int64_t Tq, int64_t sequences, int64_t heads_q, int64_t heads_kv, int64_t head_size, int64_t max_q) {
  return attention_sizes_ok(Tq, sequences, heads_q, heads_kv, head_size, max_q, 0) && Tq * heads_q <= kMostTokens;
}
}  // namespace

size_t nm_attention_paged_workspace_bytes(int64_t Tq, int32_t sequences, int32_t heads_q, int32_t heads_kv, int32_t head_size, int64_t max_q) {
  if (!paged_sizes_ok(Tq, sequences, heads_q, heads_kv, head_size, max_q)) return 0;
  return nm::paged_workspace_most(Tq, sequences, heads_q, heads_kv, head_size, max_q < Tq ? max_q : Tq);
}

int32_t nm_attention_paged(const nm_paged_desc* d, void* workspace, size_t workspace_bytes, void* stream) {
  if (!d || !d->Q.data || !d->O.data) return NM_ERR_NULL;
  nm::PagedCall c = {};
  if (int32_t st = pages_check(&d->pages, false, &c.p)) return st;
  const nm_pages& p = d->pages;
  if (!paged_sizes_ok(d->Tq, p.sequences, d->heads_q, p.heads, p.head_size, d->max_q) || d->max_k < 0) return NM_ERR_SHAPE;
  if (!d->offsets_q && d->Tq % p.sequences) return NM_ERR_SHAPE;
  if (d->window < 0 || d->sinks < 0 || !(d->scale > 0.f) || d->scale > 3.0e38f) return NM_ERR_SHAPE;
  if (!strides_ok(d->Tq, d->heads_q, p.head_size, d->Q.token, d->Q.head, false) ||
      !strides_ok(d->Tq, d->heads_q, p.head_size, d->O.token, d->O.head, true))
    return NM_ERR_SHAPE;
  if (!aligned(d->Q.data, 2) || !aligned(d->O.data, 2) || !aligned(d->lse, 4) || !aligned(d->offsets_q, 4)) return NM_ERR_ALIGN;
  c.Q = nm::HeadRows{d->Q.data, d->Q.token, d->Q.head};
  c.O = nm::HeadRows{d->O.data, d->O.token, d->O.head};
  c.lse = d->lse; c.offsets_q = d->offsets_q;
  c.Tq = d->Tq; c.Hq = d->heads_q;
  const int64_t room = (int64_t)p.table_width * p.page_size;
  c.max_q = d->max_q < d->Tq ? d->max_q : d->Tq;
  c.max_k = d->max_k < room ? d->max_k : room;
  c.window = d->window < kMostPageTokens ? d->window : (int)kMostPageTokens;  // (no sequence is longer; positions less it fit 32 bits)
  c.sinks = d->sinks; c.scale = d->scale;
  if (!workspace_ok(workspace, workspace_bytes, nm::paged_workspace_bytes(c)))
    return NM_ERR_WORKSPACE;
  c.workspace = workspace;
  return device_status(nm::launch_paged(c, (hipStream_t)stream));
}

size_t nm_probe_sink_bytes(void) { return nm::probe_sink_bytes(); }

int32_t nm_probe_matrix_rate(int32_t kind, int32_t iters, void* sink, int64_t* ops, void* stream) {
  if (!sink || !ops) return NM_ERR_NULL;
  if (kind != 0 && kind != 1) return NM_ERR_DTYPE;
  if (iters <= 0) return NM_ERR_SHAPE;
  if (!aligned(sink, 4)) return NM_ERR_ALIGN;
  return device_status(nm::launch_probe_matrix(kind, iters, static_cast<float*>(sink), ops, (hipStream_t)stream));
}

int32_t nm_probe_copy(const void* src, void* dst, size_t bytes, void* stream) {
  if (!src || !dst) return NM_ERR_NULL;
  if (bytes == 0 || (bytes % 16) != 0) return NM_ERR_SHAPE;
  if (!aligned(src, 16) || !aligned(dst, 16)) return NM_ERR_ALIGN;
  return device_status(nm::launch_probe_copy(src, dst, bytes, (hipStream_t)stream));
}

int32_t nm_linear_forward_prepared_batched(const nm_forward_desc* descs, int32_t count, void* stream) {
  return nm_linear_forward_prepared_batched_scratch(descs, count, nullptr, 0, stream);
}

size_t nm_prepared_batched_scratch_bytes(const nm_forward_desc* descs, int32_t count) {
  if (!descs) return 0;
  size_t most = 0;
  const int32_t st = forward_chunks(descs, count, [&](nm::SpmmArgs* layers, int n) {
    const size_t bytes = nm::spmm_batched_scratch(layers, n, nullptr, 0);
    most = bytes > most ? bytes : most;
    return (int32_t)NM_OK;
  });
  return st == NM_OK ? most : 0;
}

int32_t nm_linear_forward_prepared_batched_scratch(const nm_forward_desc* descs, int32_t count, void* scratch,
                                                   size_t scratch_bytes, void* stream) {
  if (!descs) return NM_ERR_NULL;
  if (count <= 0) return NM_ERR_SHAPE;
  // every argument error is reported before anything is launched
  for (int32_t i = 0; i < count; ++i) {
    nm::SpmmArgs a;
    if (int32_t st = forward_args(descs[i], &a)) return st;
    if (nm::spmm_workspace_short(a)) return NM_ERR_WORKSPACE;
  }
  // the launches of one run of layers follow those of the one before, so that all runs use the scratch from its start
  return forward_chunks(descs, count, [&](nm::SpmmArgs* layers, int n) {
    nm::spmm_batched_scratch(layers, n, scratch, scratch_bytes);
    return device_status(nm::launch_spmm_batched(layers, n, (hipStream_t)stream));
  });
}

}  // extern "C"
