// C ABI of the SVD-Attention forward pass: argument checks, workspace layout,
// kernel selection.  Every host-visible error is returned before any launch.
#include <atomic>

#include "solar_internal.cuh"

namespace solar {
namespace {
std::atomic<int> g_slice_limit{0};     // solar_set_slice_limit
}  // namespace
int slice_limit() { return g_slice_limit.load(std::memory_order_relaxed); }
}  // namespace solar

using namespace solar;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

solar_status_t check_dims(int B, int M, int N, int d, int r, solar_dtype_t dt) {
  if (dt != SOLAR_F32 && dt != SOLAR_BF16) return SOLAR_ERR_UNSUPPORTED;
  if (B < 0 || M < 0 || N < 1 || r < 1) return SOLAR_ERR_INVALID_ARG;
  if (d != 32 && d != 64 && d != 128) return SOLAR_ERR_UNSUPPORTED;
  if (r > d || r > N) return SOLAR_ERR_INVALID_ARG;
  if (r > 64 || B > 65535) return SOLAR_ERR_UNSUPPORTED;
  return SOLAR_OK;
}

solar_status_t check_ptr(const void* p) {
  return (p != nullptr && aligned16(p)) ? SOLAR_OK : SOLAR_ERR_INVALID_ARG;
}

solar_status_t check_ws(const void* ws, size_t have, size_t need) {
  if (ws == nullptr || !aligned16(ws) || have < need) return SOLAR_ERR_WORKSPACE;
  return SOLAR_OK;
}

#define SOLAR_TRY(expr)                       \
  do {                                        \
    const solar_status_t st__ = (expr);       \
    if (st__ != SOLAR_OK) return st__;        \
  } while (0)

solar_status_t from_cuda(cudaError_t e) { return e == cudaSuccess ? SOLAR_OK : SOLAR_ERR_CUDA; }

// Scores, softmax, weighted sum from a prepared workspace.  early_c: an earlier kernel of the
// same library call has already waited for whatever ran before the call, so the candidate tile
// may be fetched ahead of this kernel's own wait.
solar_status_t attn_apply_impl(int B, int M, int d, int r, solar_dtype_t dt, const void* C, unsigned flags,
                               void* O, const char* ws, bool early_c, cudaStream_t st) {
  if (attn_umma_supported(d, dt))
    return from_cuda(launch_attn_umma(B, M, d, r, C, flags, O, ws, attn_ws_layout(d, r), early_c, st));
  return from_cuda(launch_attn_simt(B, M, d, r, dt, C, flags, O, ws, attn_ws_layout(d, r), early_c, st));
}

// The streaming pass and the eigensolve of one call, on a workspace laid out by `plan`.
solar_status_t gram_impl(int B, int N, int d, solar_dtype_t dt, const void* H, void* workspace, const GramPlan& plan,
                         cudaStream_t st) {
  float* gpart = static_cast<float*>(workspace);
  int* status = reinterpret_cast<int*>(static_cast<char*>(workspace) + gram_status_offset(B, d, plan));
  if (gram_umma_supported(N, d, dt)) return from_cuda(launch_gram_umma(B, N, d, H, gpart, status, plan, st));
  return from_cuda(launch_gram_simt(B, N, d, dt, H, gpart, status, plan, st));
}

solar_status_t eig_impl(int B, int d, int r, solar_dtype_t dt, int route, int sweep_cap, int force_iters, float* S,
                        float* V, int* info, int* route_taken, void* workspace, const GramPlan& plan, cudaStream_t st) {
  char* ws = static_cast<char*>(workspace);
  const int* status = reinterpret_cast<const int*>(ws + gram_status_offset(B, d, plan));
  float* gsum = reinterpret_cast<float*>(ws + gram_sum_offset(B, d, plan));
  return from_cuda(launch_eig(B, d, r, dt, route, sweep_cap, force_iters, reinterpret_cast<const float*>(ws), status,
                              plan.parts, plan.splits, gsum, S, V, info, route_taken, st));
}

// A token tensor [B,T,H,d]: strides of the first three dimensions in elements (NULL: dense), whole 16-byte pieces.
struct Tokens {
  long long sb, st, sh;
};
solar_status_t token_strides(int B, int T, int H, int d, solar_dtype_t dt, const void* p, const long long* strides, Tokens* out) {
  SOLAR_TRY(check_ptr(p));
  if (strides == nullptr) {
    *out = {(long long)T * H * d, (long long)H * d, d};
    return SOLAR_OK;
  }
  *out = {strides[0], strides[1], strides[2]};
  const long long piece = 16 / (long long)elem_size(dt);
  const long long n[3] = {B, T, H};
  for (int i = 0; i < 3; ++i)
    if (strides[i] < 0 || (n[i] > 1 && strides[i] % piece != 0)) return SOLAR_ERR_INVALID_ARG;
  return SOLAR_OK;
}
solar_status_t token_input(int B, int T, int H, int d, solar_dtype_t dt, const void* p, const long long* strides, LinearOperand* out) {
  Tokens t;
  SOLAR_TRY(token_strides(B, T, H, d, dt, p, strides, &t));
  *out = {p, t.sb, t.st, t.sh};
  return SOLAR_OK;
}
// An output's rows may not lie over one another: each dimension steps over all of the smaller ones.
solar_status_t token_output(int B, int T, int H, int d, solar_dtype_t dt, const void* p, const long long* strides, Tokens* out) {
  SOLAR_TRY(token_strides(B, T, H, d, dt, p, strides, out));
  long long n[3] = {B, T, H}, s[3] = {out->sb, out->st, out->sh};
  for (int i = 0; i < 3; ++i)
    for (int k = i + 1; k < 3; ++k)
      if (s[k] < s[i]) { const long long a = s[i], c = n[i]; s[i] = s[k]; n[i] = n[k]; s[k] = a; n[k] = c; }
  long long extent = d;
  for (int i = 0; i < 3; ++i) {
    if (n[i] <= 1) continue;
    if (s[i] < extent) return SOLAR_ERR_INVALID_ARG;
    extent += (n[i] - 1) * s[i];
  }
  return SOLAR_OK;
}
solar_status_t check_linear(int B, int T, int H, int d, solar_dtype_t dt) {
  if (dt != SOLAR_F32 && dt != SOLAR_BF16) return SOLAR_ERR_UNSUPPORTED;
  if (B < 0 || T < 0 || H < 1) return SOLAR_ERR_INVALID_ARG;
  if (d != 32 && d != 64 && d != 128) return SOLAR_ERR_UNSUPPORTED;
  if (B > 65535 || H > 65535 / 3 || T > (1 << 30)) return SOLAR_ERR_UNSUPPORTED;
  return SOLAR_OK;
}
solar_status_t check_cache(int N) {
  if (N < 0 || N % SOLAR_CACHE_BLOCK != 0) return SOLAR_ERR_INVALID_ARG;
  return N > (1 << 30) ? SOLAR_ERR_UNSUPPORTED : SOLAR_OK;
}
solar_status_t check_optional(const void* p, unsigned align) {
  return (reinterpret_cast<uintptr_t>(p) & (align - 1)) == 0 ? SOLAR_OK : SOLAR_ERR_INVALID_ARG;
}
solar_status_t check_word_ptr(const void* p) { return p == nullptr ? SOLAR_ERR_INVALID_ARG : check_optional(p, 4); }

}  // namespace

extern "C" {

const char* solar_status_string(solar_status_t st) {
  switch (st) {
    case SOLAR_OK: return "ok";
    case SOLAR_ERR_INVALID_ARG: return "invalid argument";
    case SOLAR_ERR_UNSUPPORTED: return "unsupported size, dtype or flag";
    case SOLAR_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
    case SOLAR_ERR_CUDA: return "CUDA error";
  }
  return "unknown status";
}

size_t solar_workspace_bytes(int B, int M, int N, int d, int r, solar_dtype_t dt) {
  if (check_dims(B, M, N, d, r, dt) != SOLAR_OK) return 0;
  const size_t f = factor_ws_reserve(B, N, d, slice_limit()), a = attn_ws_bytes(B, d, r);
  const size_t need = f > a ? f : a;
  return need ? need : 256;
}

int solar_set_slice_limit(int max_slices) {
  if (max_slices < 0) max_slices = 0;
  return solar::g_slice_limit.exchange(max_slices);
}

int solar_gram_splits(int B, int N, int d, solar_dtype_t dt) {
  if (check_dims(B, 0, N, d, 1, dt) != SOLAR_OK) return 0;
  return gram_plan(B, N, d, dt, slice_limit()).parts;
}

int solar_gram_slices(int B, int N, int d, solar_dtype_t dt) {
  if (check_dims(B, 0, N, d, 1, dt) != SOLAR_OK) return 0;
  return gram_plan(B, N, d, dt, slice_limit()).splits;
}

solar_status_t solar_gram_partials(int B, int N, int d, solar_dtype_t dt, const void* H,
                                   void* workspace, size_t workspace_bytes, void* stream) {
  SOLAR_TRY(check_dims(B, 0, N, d, 1, dt));
  if (B == 0) return SOLAR_OK;
  SOLAR_TRY(check_ptr(H));
  const GramPlan plan = gram_plan(B, N, d, dt, slice_limit());
  SOLAR_TRY(check_ws(workspace, workspace_bytes, factor_ws_bytes(B, d, plan)));
  return gram_impl(B, N, d, dt, H, workspace, plan, static_cast<cudaStream_t>(stream));
}

solar_status_t solar_eig_from_partials_ex(int B, int N, int d, int r, solar_dtype_t dt, int route,
                                          float* S, float* V, int* info, int* route_taken,
                                          void* workspace, size_t workspace_bytes, void* stream) {
  SOLAR_TRY(check_dims(B, 0, N, d, r, dt));
  const int base_route = route & 0xff, sweep_cap = (route >> 8) & 0xff, force_iters = (route >> 16) & 0xff;
  if ((route & ~0xffffff) != 0 || base_route > SOLAR_ROUTE_TRIDIAG) return SOLAR_ERR_INVALID_ARG;
  if (B == 0) return SOLAR_OK;
  SOLAR_TRY(check_ptr(S));
  SOLAR_TRY(check_ptr(V));
  if (info != nullptr && (reinterpret_cast<uintptr_t>(info) & 3u)) return SOLAR_ERR_INVALID_ARG;
  if (route_taken != nullptr && (reinterpret_cast<uintptr_t>(route_taken) & 3u))
    return SOLAR_ERR_INVALID_ARG;
  const GramPlan plan = gram_plan(B, N, d, dt, slice_limit());
  SOLAR_TRY(check_ws(workspace, workspace_bytes, factor_ws_bytes(B, d, plan)));
  return eig_impl(B, d, r, dt, base_route, sweep_cap, force_iters, S, V, info, route_taken, workspace, plan,
                  static_cast<cudaStream_t>(stream));
}

solar_status_t solar_eig_from_partials(int B, int N, int d, int r, solar_dtype_t dt, float* S,
                                       float* V, int* info, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  return solar_eig_from_partials_ex(B, N, d, r, dt, SOLAR_ROUTE_AUTO, S, V, info, nullptr,
                                    workspace, workspace_bytes, stream);
}

solar_status_t solar_project_us(int B, int N, int d, int r, solar_dtype_t dt, const void* H,
                                const float* V, void* US, void* stream) {
  SOLAR_TRY(check_dims(B, 0, N, d, r, dt));
  if (B == 0) return SOLAR_OK;
  SOLAR_TRY(check_ptr(H));
  SOLAR_TRY(check_ptr(V));
  SOLAR_TRY(check_ptr(US));
  return from_cuda(launch_project_us(B, N, d, r, dt, H, V, US, false, static_cast<cudaStream_t>(stream)));
}

solar_status_t solar_lowrank_factor(int B, int M, int N, int d, int r, solar_dtype_t dt,
                                    const void* H, float* S, float* V, void* US, int* info,
                                    void* workspace, size_t workspace_bytes, void* stream) {
  (void)M;
  SOLAR_TRY(check_dims(B, 0, N, d, r, dt));
  if (B == 0) return SOLAR_OK;
  SOLAR_TRY(check_ptr(H));
  SOLAR_TRY(check_ptr(S));
  SOLAR_TRY(check_ptr(V));
  if (US != nullptr) SOLAR_TRY(check_ptr(US));
  if (info != nullptr && (reinterpret_cast<uintptr_t>(info) & 3u)) return SOLAR_ERR_INVALID_ARG;
  const GramPlan plan = gram_plan(B, N, d, dt, slice_limit());
  SOLAR_TRY(check_ws(workspace, workspace_bytes, factor_ws_bytes(B, d, plan)));
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  SOLAR_TRY(gram_impl(B, N, d, dt, H, workspace, plan, st));
  SOLAR_TRY(eig_impl(B, d, r, dt, SOLAR_ROUTE_AUTO, 0, 0, S, V, info, nullptr, workspace, plan, st));
  if (US != nullptr) SOLAR_TRY(from_cuda(launch_project_us(B, N, d, r, dt, H, V, US, true, st)));
  return SOLAR_OK;
}

solar_status_t solar_attn_prepare(int B, int d, int r, solar_dtype_t dt, const float* S,
                                  const float* V, const void* Wq, const void* Wk, const void* Wv,
                                  float scale, void* workspace, size_t workspace_bytes,
                                  void* stream) {
  SOLAR_TRY(check_dims(B, 0, r, d, r, dt));
  if (B == 0) return SOLAR_OK;
  SOLAR_TRY(check_ptr(S));
  SOLAR_TRY(check_ptr(V));
  SOLAR_TRY(check_ptr(Wq));
  SOLAR_TRY(check_ptr(Wk));
  SOLAR_TRY(check_ptr(Wv));
  SOLAR_TRY(check_ws(workspace, workspace_bytes, attn_ws_bytes(B, d, r)));
  return from_cuda(launch_attn_prepare(B, d, r, dt, S, V, Wq, Wk, Wv, scale,
                                       static_cast<char*>(workspace), attn_ws_layout(d, r), true, nullptr,
                                       static_cast<cudaStream_t>(stream)));
}

solar_status_t solar_attn_apply(int B, int M, int d, int r, solar_dtype_t dt, const void* C,
                                unsigned flags, void* O, void* workspace, size_t workspace_bytes,
                                void* stream) {
  SOLAR_TRY(check_dims(B, M, r, d, r, dt));
  if (flags & ~(unsigned)SOLAR_FLAG_NO_SOFTMAX) return SOLAR_ERR_UNSUPPORTED;
  if (B == 0 || M == 0) return SOLAR_OK;
  SOLAR_TRY(check_ptr(C));
  SOLAR_TRY(check_ptr(O));
  SOLAR_TRY(check_ws(workspace, workspace_bytes, attn_ws_bytes(B, d, r)));
  return attn_apply_impl(B, M, d, r, dt, C, flags, O, static_cast<const char*>(workspace), false,
                         static_cast<cudaStream_t>(stream));
}

solar_status_t solar_svd_attention_fwd(int B, int M, int N, int d, int r, solar_dtype_t dt,
                                       const void* C, const float* S, const float* V,
                                       const void* Wq, const void* Wk, const void* Wv, float scale,
                                       unsigned flags, void* O, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  (void)N;
  SOLAR_TRY(check_dims(B, M, r, d, r, dt));
  if (flags & ~(unsigned)SOLAR_FLAG_NO_SOFTMAX) return SOLAR_ERR_UNSUPPORTED;
  if (B == 0 || M == 0) return SOLAR_OK;
  SOLAR_TRY(check_ptr(C));
  SOLAR_TRY(check_ptr(O));
  SOLAR_TRY(check_ptr(S));
  SOLAR_TRY(check_ptr(V));
  SOLAR_TRY(check_ptr(Wq));
  SOLAR_TRY(check_ptr(Wk));
  SOLAR_TRY(check_ptr(Wv));
  SOLAR_TRY(check_ws(workspace, workspace_bytes, attn_ws_bytes(B, d, r)));
  if (attn_own_supported(B, M, d, r, dt))
    return from_cuda(launch_attn_own(B, M, r, C, S, V, Wq, Wk, Wv, scale, flags, O, static_cast<char*>(workspace),
                                     attn_ws_layout(d, r), static_cast<cudaStream_t>(stream)));
  SOLAR_TRY(from_cuda(launch_attn_prepare(B, d, r, dt, S, V, Wq, Wk, Wv, scale, static_cast<char*>(workspace),
                                          attn_ws_layout(d, r), false, nullptr, static_cast<cudaStream_t>(stream))));
  return attn_apply_impl(B, M, d, r, dt, C, flags, O, static_cast<const char*>(workspace), true,
                         static_cast<cudaStream_t>(stream));
}

size_t solar_fused_workspace_bytes(int B, int M, int N, int d, int r, solar_dtype_t dt) {
  if (check_dims(B, M, N, d, r, dt) != SOLAR_OK) return 0;
  return align_up(factor_ws_reserve(B, N, d, slice_limit()), 256) + align_up(attn_ws_bytes(B, d, r), 256);
}

solar_status_t solar_svd_attention_fused(int B, int M, int N, int d, int r, solar_dtype_t dt,
                                         const void* H, const void* C, const void* Wq, const void* Wk,
                                         const void* Wv, float scale, unsigned flags, float* S, float* V,
                                         void* O, int* info, void* workspace, size_t workspace_bytes,
                                         void* stream) {
  SOLAR_TRY(check_dims(B, M, N, d, r, dt));
  if (flags & ~(unsigned)SOLAR_FLAG_NO_SOFTMAX) return SOLAR_ERR_UNSUPPORTED;
  if (B == 0) return SOLAR_OK;
  SOLAR_TRY(check_ptr(H));
  SOLAR_TRY(check_ptr(S));
  SOLAR_TRY(check_ptr(V));
  SOLAR_TRY(check_ptr(Wq));
  SOLAR_TRY(check_ptr(Wk));
  SOLAR_TRY(check_ptr(Wv));
  if (M > 0) { SOLAR_TRY(check_ptr(C)); SOLAR_TRY(check_ptr(O)); }
  if (info != nullptr && (reinterpret_cast<uintptr_t>(info) & 3u)) return SOLAR_ERR_INVALID_ARG;
  // the factorization's workspace, then the attention's
  const GramPlan plan = gram_plan(B, N, d, dt, slice_limit());
  const size_t attn_off = align_up(factor_ws_bytes(B, d, plan), 256);
  SOLAR_TRY(check_ws(workspace, workspace_bytes, attn_off + align_up(attn_ws_bytes(B, d, r), 256)));
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  char* attn_ws = ws + attn_off;
  // streaming pass over H (the first kernel of the call: it waits for what ran before)
  SOLAR_TRY(gram_impl(B, N, d, dt, H, workspace, plan, st));
  // eigensolve; every user's CTA ends with that user's factor-token projections
  const int* status = reinterpret_cast<const int*>(ws + gram_status_offset(B, d, plan));
  float* gsum = reinterpret_cast<float*>(ws + gram_sum_offset(B, d, plan));
  const EigFuse fuse = {Wq, Wk, Wv, scale, attn_ws};
  SOLAR_TRY(from_cuda(launch_eig_tridiag(B, d, r, dt, SOLAR_ROUTE_AUTO, kMaxSweeps, reinterpret_cast<const float*>(ws),
                                         status, plan.parts, plan.splits, gsum, S, V, info, nullptr, &fuse, st)));
  if (M == 0) return SOLAR_OK;
  return attn_apply_impl(B, M, d, r, dt, C, flags, O, attn_ws, true, st);
}

size_t solar_backward_workspace_bytes(int B, int M, int N, int d, int r, solar_dtype_t dt) {
  if (check_dims(B, M, N, d, r, dt) != SOLAR_OK) return 0;
  const size_t a = bwd_ws_layout(B, M, d, r).total, k = (size_t)B * d * d * sizeof(float);
  return a > k ? a : k;
}

solar_status_t solar_svd_attention_bwd(int B, int M, int N, int d, int r, solar_dtype_t dt,
                                       const void* C, const float* S, const float* V,
                                       const void* Wq, const void* Wk, const void* Wv,
                                       float scale, unsigned flags, const void* dO,
                                       void* dC, float* dWq, float* dWk, float* dWv,
                                       float* dS, float* dV,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  (void)N;
  SOLAR_TRY(check_dims(B, M, r, d, r, dt));
  if (flags & ~(unsigned)SOLAR_FLAG_NO_SOFTMAX) return SOLAR_ERR_UNSUPPORTED;
  if (B == 0) return SOLAR_OK;
  if (M > 0) { SOLAR_TRY(check_ptr(C)); SOLAR_TRY(check_ptr(dO)); SOLAR_TRY(check_ptr(dC)); }
  SOLAR_TRY(check_ptr(S));
  SOLAR_TRY(check_ptr(V));
  SOLAR_TRY(check_ptr(Wq));
  SOLAR_TRY(check_ptr(Wk));
  SOLAR_TRY(check_ptr(Wv));
  SOLAR_TRY(check_ptr(dWq));
  SOLAR_TRY(check_ptr(dWk));
  SOLAR_TRY(check_ptr(dWv));
  SOLAR_TRY(check_ptr(dS));
  SOLAR_TRY(check_ptr(dV));
  const BwdWs bl = bwd_ws_layout(B, M, d, r);
  SOLAR_TRY(check_ws(workspace, workspace_bytes, bl.total));
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const AttnWs lay = attn_ws_layout(d, r);
  char* ws = static_cast<char*>(workspace);
  // T_b and Value_r as in the forward call
  SOLAR_TRY(from_cuda(launch_attn_prepare(B, d, r, dt, S, V, Wq, Wk, Wv, scale, ws, lay, false, ws + bl.pk_off, st)));
  return from_cuda(launch_attn_bwd(B, M, d, r, dt, C, dO, S, V, Wq, Wk, Wv, scale, flags, dC, dWq, dWk, dWv,
                                   dS, dV, ws, lay, bl, st));
}

solar_status_t solar_svd_backward(int B, int N, int d, int r, solar_dtype_t dt, const void* H,
                                  const float* S, const float* V, const float* dS, const float* dV,
                                  float eps_rel, void* dH, void* workspace, size_t workspace_bytes,
                                  void* stream) {
  SOLAR_TRY(check_dims(B, 0, N, d, r, dt));
  if (!(eps_rel >= 0.f)) return SOLAR_ERR_INVALID_ARG;
  if (B == 0) return SOLAR_OK;
  SOLAR_TRY(check_ptr(H));
  SOLAR_TRY(check_ptr(S));
  SOLAR_TRY(check_ptr(V));
  SOLAR_TRY(check_ptr(dS));
  SOLAR_TRY(check_ptr(dV));
  SOLAR_TRY(check_ptr(dH));
  SOLAR_TRY(check_ws(workspace, workspace_bytes, (size_t)B * d * d * sizeof(float)));
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  float* K = static_cast<float*>(workspace);
  SOLAR_TRY(from_cuda(launch_svd_grad(B, d, r, S, V, dS, dV, eps_rel, K, st)));
  // dH_b = H_b K_b: the right-multiplication kernel of the left factor, with q = d columns
  return from_cuda(launch_project_us(B, N, d, d, dt, H, K, dH, true, st));
}

solar_status_t solar_factored_softmax_attention_fwd(int B, int M, int N, int d, int r, solar_dtype_t dt,
                                                    const void* C, const void* US, const float* V,
                                                    const void* Wq, const void* Wk, const void* Wv,
                                                    float scale, void* O, void* workspace,
                                                    size_t workspace_bytes, void* stream) {
  SOLAR_TRY(check_dims(B, M, N, d, r, dt));
  if (!flash_factored_supported(d, r, dt)) return SOLAR_ERR_UNSUPPORTED;
  if (B == 0 || M == 0) return SOLAR_OK;
  SOLAR_TRY(check_ptr(C));
  SOLAR_TRY(check_ptr(US));
  SOLAR_TRY(check_ptr(V));
  SOLAR_TRY(check_ptr(Wq));
  SOLAR_TRY(check_ptr(Wk));
  SOLAR_TRY(check_ptr(Wv));
  SOLAR_TRY(check_ptr(O));
  SOLAR_TRY(check_ws(workspace, workspace_bytes, attn_ws_bytes(B, d, r)));
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const AttnWs lay = attn_ws_layout(d, r);
  // The packed operands of the kernel are the prepare kernel's with unit singular values:
  // T^T becomes (scale log2e W_Q W_K^T V)^T and Value_r^T becomes (V^T W_V)^T.
  char* ws = static_cast<char*>(workspace);
  const FlashSplit split = flash_split(B, M, N, d, r, workspace_bytes);
  int* counters = split.ranges > 1 ? reinterpret_cast<int*>(ws + split.counter_off) : nullptr;
  SOLAR_TRY(from_cuda(launch_attn_prepare(B, d, r, dt, nullptr, V, Wq, Wk, Wv, scale * 1.4426950408889634f, ws, lay, false,
                                          nullptr, st, counters, split.items_per_user)));
  return from_cuda(launch_flash_factored(B, M, N, d, r, C, US, O, ws, lay, split, st));
}

solar_status_t solar_linear_attention_fwd(int B, int T, int H, int d, solar_dtype_t dt, const void* Q, const long long* q_strides,
                                          const void* K, const long long* k_strides, const void* V, const long long* v_strides,
                                          const float* log_decay, float scale, const int* lengths, const float* state0,
                                          void* O, const long long* o_strides, float* state, void* stream) {
  SOLAR_TRY(check_linear(B, T, H, d, dt));
  if (B == 0) return SOLAR_OK;
  LinearParams prm = {};
  prm.roles = 1; prm.T = T; prm.H = H; prm.lengths = lengths; prm.log_decay = log_decay;
  LinearRole& r = prm.role[0];
  if (T > 0) {
    SOLAR_TRY(token_input(B, T, H, d, dt, Q, q_strides, &r.q));
    SOLAR_TRY(token_input(B, T, H, d, dt, K, k_strides, &r.k));
    SOLAR_TRY(token_input(B, T, H, d, dt, V, v_strides, &r.v));
    Tokens o;
    SOLAR_TRY(token_output(B, T, H, d, dt, O, o_strides, &o));
    if (O == Q || O == K || O == V) return SOLAR_ERR_INVALID_ARG;              // other CTAs still read them
    r.o = O; r.ob = o.sb; r.ot = o.st; r.oh = o.sh;
  }
  SOLAR_TRY(check_word_ptr(log_decay));
  SOLAR_TRY(check_optional(lengths, 4));
  SOLAR_TRY(check_optional(state0, 16));
  SOLAR_TRY(check_optional(state, 16));
  if (state != nullptr && state == state0) return SOLAR_ERR_INVALID_ARG;       // other segments still read it
  if (T == 0 && state == nullptr) return SOLAR_OK;
  r.s0 = state0; r.s0_r = d; r.s0_c = 1; r.s1 = state;
  r.ap = scale; r.aq = scale; r.ak = 1.f;
  return from_cuda(launch_linear_attention(B, d, dt, prm, static_cast<cudaStream_t>(stream)));
}

solar_status_t solar_linear_attention_bwd(int B, int T, int H, int d, solar_dtype_t dt, const void* Q, const long long* q_strides,
                                          const void* K, const long long* k_strides, const void* V, const long long* v_strides,
                                          const float* log_decay, float scale, const int* lengths, const float* state0,
                                          const void* dO, const long long* do_strides, const float* dstate,
                                          void* dQ, const long long* dq_strides, void* dK, const long long* dk_strides,
                                          void* dV, const long long* dv_strides, float* dstate0, void* stream) {
  SOLAR_TRY(check_linear(B, T, H, d, dt));
  if (B == 0) return SOLAR_OK;
  LinearOperand q = {}, k = {}, v = {}, g = {};
  Tokens out[3] = {};
  if (T > 0) {
    SOLAR_TRY(token_input(B, T, H, d, dt, Q, q_strides, &q));
    SOLAR_TRY(token_input(B, T, H, d, dt, K, k_strides, &k));
    SOLAR_TRY(token_input(B, T, H, d, dt, V, v_strides, &v));
    SOLAR_TRY(token_input(B, T, H, d, dt, dO, do_strides, &g));
    SOLAR_TRY(token_output(B, T, H, d, dt, dQ, dq_strides, &out[0]));
    SOLAR_TRY(token_output(B, T, H, d, dt, dK, dk_strides, &out[1]));
    SOLAR_TRY(token_output(B, T, H, d, dt, dV, dv_strides, &out[2]));
    const void* made[3] = {dQ, dK, dV};
    for (int i = 0; i < 3; ++i)
      if (made[i] == Q || made[i] == K || made[i] == V || made[i] == dO || made[i] == made[(i + 1) % 3]) return SOLAR_ERR_INVALID_ARG;
  }
  SOLAR_TRY(check_word_ptr(log_decay));
  SOLAR_TRY(check_optional(lengths, 4));
  SOLAR_TRY(check_optional(state0, 16));
  SOLAR_TRY(check_optional(dstate, 16));
  SOLAR_TRY(check_optional(dstate0, 16));
  if (dstate0 != nullptr && (dstate0 == dstate || dstate0 == state0)) return SOLAR_ERR_INVALID_ARG;
  if (T == 0 && dstate0 == nullptr) return SOLAR_OK;
  LinearParams prm = {};
  prm.roles = 3; prm.T = T; prm.H = H; prm.lengths = lengths; prm.log_decay = log_decay;
  auto role = [&](int i, const LinearOperand& a, const LinearOperand& b, const LinearOperand& c, void* o, const float* s0, bool transposed) {
    LinearRole& r = prm.role[i];
    r.q = a; r.k = b; r.v = c;
    r.o = o; r.ob = out[i].sb; r.ot = out[i].st; r.oh = out[i].sh;
    r.s0 = s0; r.s0_r = transposed ? 1 : d; r.s0_c = transposed ? d : 1;
    r.reverse = i > 0; r.ap = scale; r.aq = i > 0 ? 1.f : scale; r.ak = i > 0 ? scale : 1.f;
  };
  role(0, g, v, k, dQ, state0, true);
  role(1, v, g, q, dK, dstate, true);
  role(2, k, q, g, dV, dstate, false);
  prm.role[2].s1 = dstate0;
  return from_cuda(launch_linear_attention(B, d, dt, prm, static_cast<cudaStream_t>(stream)));
}

solar_status_t solar_linear_attention_step(int B, int H, int d, solar_dtype_t dt, const void* Q, const long long* q_strides,
                                           const void* K, const long long* k_strides, const void* V, const long long* v_strides,
                                           const float* log_decay, float scale, float* state, void* O, const long long* o_strides,
                                           void* stream) {
  SOLAR_TRY(check_linear(B, 1, H, d, dt));
  if (B == 0) return SOLAR_OK;
  LinearOperand op[3];
  const void* in[3] = {Q, K, V};
  const long long* strides[3] = {q_strides, k_strides, v_strides};
  for (int i = 0; i < 3; ++i) {
    const long long s[3] = {strides[i] ? strides[i][0] : 0, 0, strides[i] ? strides[i][1] : 0};
    SOLAR_TRY(token_input(B, 1, H, d, dt, in[i], strides[i] ? s : nullptr, &op[i]));
  }
  Tokens o;
  const long long s[3] = {o_strides ? o_strides[0] : 0, 0, o_strides ? o_strides[1] : 0};
  SOLAR_TRY(token_output(B, 1, H, d, dt, O, o_strides ? s : nullptr, &o));
  if (O == Q || O == K || O == V) return SOLAR_ERR_INVALID_ARG;
  SOLAR_TRY(check_word_ptr(log_decay));
  SOLAR_TRY(check_ptr(state));
  return from_cuda(launch_linear_step(B, H, d, dt, op[0], op[1], op[2], log_decay, scale, state, O, o.sb, o.sh,
                                      static_cast<cudaStream_t>(stream)));
}

solar_status_t solar_history_cache_append(int B, int T, int H, int N, int d, solar_dtype_t dt, const void* K, const long long* k_strides,
                                          const void* V, const long long* v_strides, const int* start, const int* counts,
                                          void* k8, void* v8, float* k_scale, float* v_scale, void* stream) {
  SOLAR_TRY(check_linear(B, T, H, d, dt));
  SOLAR_TRY(check_cache(N));
  if (B == 0 || T == 0 || N == 0) return SOLAR_OK;
  LinearOperand k, v;
  SOLAR_TRY(token_input(B, T, H, d, dt, K, k_strides, &k));
  SOLAR_TRY(token_input(B, T, H, d, dt, V, v_strides, &v));
  SOLAR_TRY(check_word_ptr(start));
  SOLAR_TRY(check_optional(counts, 4));
  SOLAR_TRY(check_ptr(k8));
  SOLAR_TRY(check_ptr(v8));
  SOLAR_TRY(check_word_ptr(k_scale));
  SOLAR_TRY(check_word_ptr(v_scale));
  return from_cuda(launch_history_append(B, T, H, N, d, dt, k, v, start, counts, static_cast<uint8_t*>(k8), static_cast<uint8_t*>(v8),
                                         k_scale, v_scale, static_cast<cudaStream_t>(stream)));
}

solar_status_t solar_history_cache_attention(int B, int M, int Hq, int H, int N, int d, solar_dtype_t dt, const void* Q,
                                             const long long* q_strides, const void* k8, const void* v8, const float* k_scale,
                                             const float* v_scale, const int* lengths, float scale, unsigned flags, void* O,
                                             const long long* o_strides, void* stream) {
  SOLAR_TRY(check_linear(B, M, H, d, dt));
  SOLAR_TRY(check_cache(N));
  if (flags & ~(unsigned)SOLAR_FLAG_CAUSAL) return SOLAR_ERR_UNSUPPORTED;
  if (Hq < 1 || Hq % H != 0) return SOLAR_ERR_INVALID_ARG;
  if (B == 0 || M == 0) return SOLAR_OK;
  HistoryCall c = {};
  Tokens o;
  SOLAR_TRY(token_input(B, M, Hq, d, dt, Q, q_strides, &c.q));
  SOLAR_TRY(token_output(B, M, Hq, d, dt, O, o_strides, &o));
  if (N > 0) {
    SOLAR_TRY(check_ptr(k8));
    SOLAR_TRY(check_ptr(v8));
    SOLAR_TRY(check_word_ptr(k_scale));
    SOLAR_TRY(check_word_ptr(v_scale));
  }
  SOLAR_TRY(check_word_ptr(lengths));
  c.B = B; c.M = M; c.H = H; c.G = Hq / H; c.N = N;
  c.o = O; c.ob = o.sb; c.ot = o.st; c.oh = o.sh;
  c.k8 = static_cast<const uint8_t*>(k8); c.v8 = static_cast<const uint8_t*>(v8); c.k_scale = k_scale; c.v_scale = v_scale;
  c.lengths = lengths; c.scale = scale; c.causal = (flags & SOLAR_FLAG_CAUSAL) != 0;
  if (history_flash_supported(d, dt, c)) return from_cuda(launch_history_flash(d, c, static_cast<cudaStream_t>(stream)));
  return from_cuda(launch_history_attention(d, dt, c, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
