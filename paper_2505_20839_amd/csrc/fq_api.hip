// C entry points of the W4A8-FP library: argument validation, kernel choice, launch.
// Declarations and the contract of every call are in include/fireq.h.
#include "../../include/fireq.h"
#include "../../include/fireq_chunk.h"
#include "../../include/fireq_kv4_ws.h"
#include "../../include/fireq_norm.h"
#include "../../include/fireq_norm_block.h"
#include "../../include/fireq_paged.h"
#include "../../include/fireq_sample.h"
#include "../../include/fireq_wquant_ws.h"
#include "fq_common.h"
#include "fq_kernels.h"

#include <cstdlib>
#include <cstring>
#include <atomic>
#include <mutex>

// Scratch of fq_w4a8_gemm_static: one array per GPU the library runs on, part of the code object, held
// until the process ends.  In host code the name is only a handle for hipGetSymbolAddress.
#define FQ_STATIC_SCRATCH_BYTES (16u << 20)
static __device__ __align__(256) unsigned char scratch[FQ_STATIC_SCRATCH_BYTES];

namespace {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int after_launch() { return hipGetLastError() == hipSuccess ? FQ_OK : FQ_ERR_LAUNCH; }

enum class GemmKernel { Auto, Simple, Large, Small, KSplit };

// FQ_FORCE_KERNEL=simple|large|small overrides the choice (tests use it to cross-check kernels).
GemmKernel parse_kernel(const char* e) {
    if (!e || !*e) return GemmKernel::Auto;
    if (!std::strcmp(e, "simple")) return GemmKernel::Simple;
    if (!std::strcmp(e, "large")) return GemmKernel::Large;
    if (!std::strcmp(e, "small")) return GemmKernel::Small;
    if (!std::strcmp(e, "ksplit")) return GemmKernel::KSplit;
    return GemmKernel::Auto;
}

// The environment is read when the library is loaded; fq_test_force_kernel changes the choice later.
std::atomic<int> g_forced{static_cast<int>(parse_kernel(std::getenv("FQ_FORCE_KERNEL")))};

GemmKernel forced_kernel() { return static_cast<GemmKernel>(g_forced.load(std::memory_order_relaxed)); }

// The GEMM kernels address every operand through 32-bit buffer offsets: each of A, the packed
// weights, the group scales and the workspace must stay below 4 GiB, and a band of 256 output rows too.
bool gemm_operands_addressable(int M, int N, int K) {
    const unsigned long long lim = 0xFFFFFF00ull, m = (unsigned long long)M, n = (unsigned long long)N,
                             k = (unsigned long long)K, g = k / FQ_GROUP;
    return m * k < lim && ((n + 31) / 32) * 32 * k / 2 < lim && n * g < lim && 256ull * n * 2 < lim &&
           (unsigned long long)fq_gemm_large_workspace_bytes(M, K) < lim;
}

// Argument checks shared by the GEMM entry points (M == 0 is valid and needs no pointers).
int check_gemm_args(const void* A, const void* a_scale, const void* W, const void* gs, const void* Y,
                    int M, int N, int K) {
    if (M < 0 || N < 0 || K <= 0 || (K % FQ_GROUP) != 0) return FQ_ERR_SHAPE;
    if (M == 0) return FQ_OK;
    if (N == 0) return FQ_ERR_SHAPE;
    if (!A || !a_scale || !W || !gs || !Y) return FQ_ERR_NULL;
    if (!aligned16(A) || !aligned16(W) || !aligned16(gs) || !aligned16(Y)) return FQ_ERR_ALIGN;
    if (!gemm_operands_addressable(M, N, K)) return FQ_ERR_SHAPE;
    return FQ_OK;
}

// Large also stands for the K-split kernel, which shares its workspace: ksplit_choice picks between the two.
GemmKernel choose_kernel(int M) {
    const GemmKernel k = forced_kernel();
    if (k == GemmKernel::KSplit) return GemmKernel::Large;
    return k != GemmKernel::Auto ? k : (M <= 64 ? GemmKernel::Small : GemmKernel::Large);
}

// 0: the large-M kernel's own tiles; 1, 2, 3: a shape of the K-split kernel (never with the fused gate/up epilogue).
// Forcing "large" keeps the large-M kernel, forcing "ksplit" takes the K-split kernel wherever it can run.
int ksplit_choice(int M, int N, int K, bool swiglu) {
    const GemmKernel k = forced_kernel();
    if (swiglu || k == GemmKernel::Large || k == GemmKernel::Simple || k == GemmKernel::Small) return 0;
    if (k == GemmKernel::KSplit) return (K / FQ_GROUP >= 8) ? (M <= 512 ? 2 : 1) : 0;
    return fq_gemm_ksplit_choice(M, N, K, fq_device_cus());
}

// The top of 16 < M <= 64: the K-split kernel on 64 x 64 tiles instead of the M <= 64 kernel (never when a kernel is forced,
// never with the fused gate/up epilogue)
bool ksplit64_choice(int M, int N, int K, bool swiglu) {
    return !swiglu && forced_kernel() == GemmKernel::Auto && fq_gemm_ksplit64_serves(M, N, K, fq_device_cus());
}

}  // namespace

extern "C" {

int fq_layout_version(void) { return FQ_LAYOUT_VERSION; }

const char* fq_status_string(int status) {
    switch (status) {
        case FQ_OK: return "ok";
        case FQ_ERR_NULL: return "a required pointer is NULL";
        case FQ_ERR_SHAPE: return "invalid shape (sizes must be non-negative, K a positive multiple of 128)";
        case FQ_ERR_ALIGN: return "a base pointer is not 16-byte aligned";
        case FQ_ERR_LAUNCH: return "the HIP runtime rejected the kernel launch";
        case FQ_ERR_MEMORY: return "workspace missing or too small (fq_w4a8_gemm_static: the problem needs more than the "
                                   "built-in scratch holds), or the library could not allocate its own";
        default: return "unknown status";
    }
}

size_t fq_packed_weight_bytes(int N, int K) {
    if (N <= 0 || K <= 0 || (K % FQ_GROUP) != 0) return 0;
    return (size_t)((N + 31) / 32) * 32u * (size_t)K / 2u;
}

int fq_pack_weights(const int8_t* q, uint8_t* Wq_packed, int N, int K, void* stream) {
    if (N < 0 || K <= 0 || (K % FQ_GROUP) != 0) return FQ_ERR_SHAPE;
    if (N == 0) return FQ_OK;
    if (!q || !Wq_packed) return FQ_ERR_NULL;
    if (!aligned16(Wq_packed)) return FQ_ERR_ALIGN;
    fq_launch_pack(q, Wq_packed, N, K, static_cast<hipStream_t>(stream));
    return after_launch();
}

int fq_unpack_weights(const uint8_t* Wq_packed, int8_t* q, int N, int K, void* stream) {
    if (N < 0 || K <= 0 || (K % FQ_GROUP) != 0) return FQ_ERR_SHAPE;
    if (N == 0) return FQ_OK;
    if (!q || !Wq_packed) return FQ_ERR_NULL;
    if (!aligned16(Wq_packed)) return FQ_ERR_ALIGN;
    fq_launch_unpack(Wq_packed, q, N, K, static_cast<hipStream_t>(stream));
    return after_launch();
}

int fq_quantize_act(const uint16_t* X_bf16, uint8_t* A_fp8, float* a_scale, int M, int K, void* stream) {
    if (M < 0 || K <= 0 || (K % 8) != 0) return FQ_ERR_SHAPE;
    if (M == 0) return FQ_OK;
    if (!X_bf16 || !A_fp8 || !a_scale) return FQ_ERR_NULL;
    if (!aligned16(X_bf16) || !aligned16(A_fp8)) return FQ_ERR_ALIGN;
    if (((size_t)K * 2u) % 16u != 0 || ((size_t)K % 8u) != 0) return FQ_ERR_SHAPE;
    fq_launch_quantize(X_bf16, A_fp8, a_scale, M, K, static_cast<hipStream_t>(stream));
    return after_launch();
}

int fq_cas_scales(const uint16_t* W_bf16, float target, float* lambda, int N, int K, void* stream) {
    return fq_cas_scales_ws(W_bf16, target, lambda, N, K, nullptr, 0, stream);
}

size_t fq_cas_scales_workspace_bytes(int N, int K) { return N > 0 && K > 0 ? fq_cas_scales_scratch(N, K) : 0; }

int fq_cas_scales_ws(const uint16_t* W_bf16, float target, float* lambda, int N, int K, void* workspace, size_t workspace_bytes,
                     void* stream) {
    if (N <= 0 || K <= 0 || !(target > 0.f)) return FQ_ERR_SHAPE;
    if (!W_bf16 || !lambda) return FQ_ERR_NULL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const size_t need = workspace ? fq_cas_scales_scratch(N, K) : 0;
    if (need != 0) {
        if (!aligned16(workspace)) return FQ_ERR_ALIGN;
        if (workspace_bytes < need) return FQ_ERR_MEMORY;
    }
    if (need != 0 && aligned16(W_bf16)) fq_launch_cas_scales_split(W_bf16, target, lambda, N, K, workspace, s);
    else fq_launch_cas_scales(W_bf16, target, lambda, N, K, s);
    return after_launch();
}

int fq_pts_exponent(const uint16_t* W_bf16, const float* lambda, int* n_out, int N, int K, void* stream) {
    return fq_pts_exponent_ws(W_bf16, lambda, n_out, N, K, nullptr, 0, stream);
}

size_t fq_pts_exponent_workspace_bytes(int N, int K) {
    return N > 0 && K > 0 && (K % FQ_GROUP) == 0 ? fq_pts_exponent_scratch(K) : 0;
}

int fq_pts_exponent_ws(const uint16_t* W_bf16, const float* lambda, int* n_out, int N, int K, void* workspace,
                       size_t workspace_bytes, void* stream) {
    if (N <= 0 || K <= 0 || (K % FQ_GROUP) != 0) return FQ_ERR_SHAPE;
    if (!W_bf16 || !n_out) return FQ_ERR_NULL;
    const size_t need = workspace ? fq_pts_exponent_scratch(K) : 0;
    if (!aligned16(W_bf16) || !aligned16(n_out) || (need != 0 && !aligned16(workspace))) return FQ_ERR_ALIGN;
    if (workspace_bytes < need) return FQ_ERR_MEMORY;
    fq_launch_pts_exponent(W_bf16, lambda, n_out, N, K, need != 0 ? workspace : nullptr, static_cast<hipStream_t>(stream));
    return after_launch();
}

int fq_quantize_weights(const uint16_t* W_bf16, const float* lambda, int n_pts, int sigma_nearest,
                        int8_t* q, uint8_t* w_gscale, int N, int K, void* stream) {
    if (N < 0 || K <= 0 || (K % FQ_GROUP) != 0 || n_pts < 0 || n_pts > 126) return FQ_ERR_SHAPE;
    if (N == 0) return FQ_OK;
    if (!W_bf16 || !q || !w_gscale) return FQ_ERR_NULL;
    if (!aligned16(W_bf16) || !aligned16(q) || (lambda && !aligned16(lambda))) return FQ_ERR_ALIGN;
    fq_launch_quantize_weights(W_bf16, lambda, n_pts, sigma_nearest != 0, q, w_gscale, N, K,
                               static_cast<hipStream_t>(stream));
    return after_launch();
}

int fq_test_force_kernel(const char* name) {
    g_forced.store(static_cast<int>(parse_kernel(name)), std::memory_order_relaxed);
    return FQ_OK;
}

size_t fq_diag_stream_read_sink_bytes(void) { return (size_t)fq_stream_read_blocks() * sizeof(unsigned); }

int fq_diag_stream_read(const void* src, size_t bytes, void* sink, void* stream) {
    if (bytes == 0) return FQ_OK;
    if (!src || !sink) return FQ_ERR_NULL;
    if (!aligned16(src) || (bytes & 15u) != 0) return FQ_ERR_ALIGN;
    fq_launch_stream_read(src, bytes, static_cast<unsigned*>(sink), static_cast<hipStream_t>(stream));
    return after_launch();
}

int fq_w4a8_gemm_plan(int M, int N, int K, int cus, int* plan) {
    if (M <= 0 || N <= 0 || K <= 0 || (K % FQ_GROUP) != 0 || cus < 0) return FQ_ERR_SHAPE;
    if (!plan) return FQ_ERR_NULL;
    for (int i = 0; i < 8; ++i) plan[i] = 0;
    const GemmKernel k = choose_kernel(M);
    plan[0] = k == GemmKernel::Simple ? 0 : k == GemmKernel::Small ? (!fq_gemm_small_serves(M, K) ? 0 : M <= 16 ? 1 : 2) : 3;
    if (k == GemmKernel::Small && forced_kernel() == GemmKernel::Auto &&
        fq_gemm_ksplit64_serves(M, N, K, cus > 0 ? cus : fq_device_cus())) {
        plan[0] = 6;
        plan[5] = (N + 63) / 64;
        plan[6] = 1;
    }
    if (k == GemmKernel::Large) {
        const int c = cus > 0 ? cus : fq_device_cus();
        const GemmKernel f = forced_kernel();
        const int ks = f == GemmKernel::Large ? 0
                     : f == GemmKernel::KSplit ? ((K / FQ_GROUP >= 8) ? (M <= 512 ? 2 : 1) : 0)
                                               : fq_gemm_ksplit_choice(M, N, K, c);
        if (ks != 0) {
            const int bm = ks == 1 ? 256 : 128, bn = ks == 2 ? 64 : 128;
            plan[0] = ks == 3 ? 7 : 3 + ks;
            plan[5] = ((M + bm - 1) / bm) * ((N + bn - 1) / bn);
            plan[6] = fq_gemm_ksplit_slices(ks, M, N, K, c);
        } else {
            fq_gemm_large_plan(M, N, c, plan + 1);
        }
    }
    return FQ_OK;
}

size_t fq_w4a8_gemm_workspace_bytes(int M, int N, int K) {
    if (M <= 0 || N <= 0 || K <= 0 || (K % FQ_GROUP) != 0) return 0;
    if (choose_kernel(M) != GemmKernel::Large) return 0;
    // (the fused gate/up epilogue never takes the K-split kernel and leaves the partial tiles unused)
    return fq_gemm_large_workspace_bytes(M, K) +
           fq_gemm_ksplit_partial_bytes(ksplit_choice(M, N, K, false), M, N, K, fq_device_cus());
}

int fq_quantize_act_ws(const uint16_t* X_bf16, uint8_t* A_fp8, float* a_scale, int M, int K,
                       void* workspace, size_t workspace_bytes, void* stream) {
    if (M < 0 || K <= 0 || (K % FQ_GROUP) != 0) return FQ_ERR_SHAPE;
    if (M == 0) return FQ_OK;
    if (!X_bf16 || !A_fp8 || !a_scale) return FQ_ERR_NULL;
    if (!aligned16(X_bf16) || !aligned16(A_fp8)) return FQ_ERR_ALIGN;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (choose_kernel(M) != GemmKernel::Large) {          // that GEMM takes no workspace: the plain quantiser
        fq_launch_quantize(X_bf16, A_fp8, a_scale, M, K, s);
        return after_launch();
    }
    if (!workspace || workspace_bytes < fq_gemm_large_workspace_bytes(M, K)) return FQ_ERR_MEMORY;
    if (!aligned16(workspace)) return FQ_ERR_ALIGN;
    if (fq_quantize_can_write_zero_point(K)) {
        fq_launch_quantize_zp(X_bf16, A_fp8, a_scale, M, K, workspace, s);
    } else {                                              // very long rows: two kernels
        fq_launch_quantize(X_bf16, A_fp8, a_scale, M, K, s);
        fq_launch_zero_point(A_fp8, workspace, M, K, s);
    }
    return after_launch();
}

namespace {

int gemm_ws(const uint8_t* A_fp8, const float* a_scale, const uint8_t* Wq_packed, const uint8_t* w_gscale,
            float w_tscale, uint16_t* out, int M, int N, int K, void* workspace, size_t workspace_bytes,
            int workspace_prepared, bool swiglu, const uint16_t* R, bool with_residual, void* stream) {
    const int rc = check_gemm_args(A_fp8, a_scale, Wq_packed, w_gscale, out, M, N, K);
    if (rc != FQ_OK) return rc;
    if (swiglu && (N & 1)) return FQ_ERR_SHAPE;
    if (M == 0) return FQ_OK;
    if (with_residual) {
        if (!R) return FQ_ERR_NULL;
        if (!aligned16(R)) return FQ_ERR_ALIGN;
        if (R != out) {                                   // the very same array is fine, a shifted overlap is not
            const uintptr_t r0 = reinterpret_cast<uintptr_t>(R), y0 = reinterpret_cast<uintptr_t>(out);
            const uintptr_t bytes = (uintptr_t)M * (uintptr_t)N * 2u;
            if (r0 < y0 + bytes && y0 < r0 + bytes) return FQ_ERR_SHAPE;
        }
    }
    const size_t need = fq_w4a8_gemm_workspace_bytes(M, N, K);
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return FQ_ERR_MEMORY;
        if (!aligned16(workspace)) return FQ_ERR_ALIGN;
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    switch (choose_kernel(M)) {
        case GemmKernel::Simple:
            fq_launch_gemm_simple(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, out, M, N, K, swiglu, R, s);
            break;
        case GemmKernel::Small:
            if (ksplit64_choice(M, N, K, swiglu))
                fq_launch_gemm_ksplit64(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, out, M, N, K, R, s);
            else if (!fq_launch_gemm_small(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, out, M, N, K, swiglu, R, s))
                fq_launch_gemm_simple(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, out, M, N, K, swiglu, R, s);
            break;
        default: {
            const int ks = ksplit_choice(M, N, K, swiglu);
            if (ks != 0)
                fq_launch_gemm_ksplit(ks, A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, out, M, N, K, workspace,
                                      workspace_prepared != 0, R, s);
            else
                fq_launch_gemm_large(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, out, M, N, K, workspace,
                                     workspace_prepared != 0, swiglu, R, s);
            break;
        }
    }
    return after_launch();
}

}  // namespace

int fq_w4a8_gemm_ws(const uint8_t* A_fp8, const float* a_scale, const uint8_t* Wq_packed,
                    const uint8_t* w_gscale, float w_tscale, uint16_t* Y_bf16,
                    int M, int N, int K, void* workspace, size_t workspace_bytes, int workspace_prepared,
                    void* stream) {
    return gemm_ws(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, Y_bf16, M, N, K, workspace, workspace_bytes,
                   workspace_prepared, false, nullptr, false, stream);
}

int fq_w4a8_gemm_add_ws(const uint8_t* A_fp8, const float* a_scale, const uint8_t* Wq_packed,
                        const uint8_t* w_gscale, float w_tscale, const uint16_t* R_bf16, uint16_t* Y_bf16,
                        int M, int N, int K, void* workspace, size_t workspace_bytes, int workspace_prepared,
                        void* stream) {
    return gemm_ws(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, Y_bf16, M, N, K, workspace, workspace_bytes,
                   workspace_prepared, false, R_bf16, true, stream);
}

int fq_w4a8_gemm_swiglu_ws(const uint8_t* A_fp8, const float* a_scale, const uint8_t* Wq_packed,
                           const uint8_t* w_gscale, float w_tscale, uint16_t* H_bf16,
                           int M, int N, int K, void* workspace, size_t workspace_bytes, int workspace_prepared,
                           void* stream) {
    return gemm_ws(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, H_bf16, M, N, K, workspace, workspace_bytes,
                   workspace_prepared, true, nullptr, false, stream);
}

int fq_w4a8_gemm_swiglu_quant_ws(const uint8_t* A_fp8, const float* a_scale, const uint8_t* Wq_packed,
                                 const uint8_t* w_gscale, float w_tscale, uint16_t* H_bf16,
                                 uint8_t* H_fp8, float* h_scale, int M, int N, int K,
                                 void* workspace, size_t workspace_bytes, int workspace_prepared,
                                 void* next_workspace, size_t next_workspace_bytes, void* stream) {
    const int rc = check_gemm_args(A_fp8, a_scale, Wq_packed, w_gscale, H_bf16, M, N, K);
    if (rc != FQ_OK) return rc;
    if (N & 1) return FQ_ERR_SHAPE;
    if (M == 0) return FQ_OK;
    const int NH = N / 2;
    if ((NH % 8) != 0) return FQ_ERR_SHAPE;               // the quantiser works on whole 16-byte chunks of a row
    if (!H_fp8 || !h_scale) return FQ_ERR_NULL;
    if (!aligned16(H_fp8)) return FQ_ERR_ALIGN;
    hipStream_t s = static_cast<hipStream_t>(stream);
    // zero-point terms for a GEMM that takes H_fp8 as its input: only where that GEMM has a workspace and the
    // quantiser can write them (rows of at most 16384 codes, whole groups)
    const bool next_large = next_workspace != nullptr && choose_kernel(M) == GemmKernel::Large &&
                            (NH % FQ_GROUP) == 0 && fq_quantize_can_write_zero_point(NH);
    if (next_workspace) {
        if (!next_large) return FQ_ERR_SHAPE;
        if (next_workspace_bytes < fq_gemm_large_workspace_bytes(M, NH)) return FQ_ERR_MEMORY;
        if (!aligned16(next_workspace)) return FQ_ERR_ALIGN;
    }
    // The gate/up GEMM, then the quantiser, which reads a row once, search included.  Row maxima raised by the GEMM's epilogue
    // (an atomic per row and tile, into scales that another launch has cleared) save the search and cost more than it: 1000 x 22016
    // x 4096 and the layer behind it 155 us with them, 151 without; 2048 x 22016 x 4096 alone 201, 192; 65 x 22016 x 4096 39.5, 35.5.
    // (Only rows of more than 32768 outputs over a short K show the search: 2048 x 65792 x 512 179, 192.)
    const int g = fq_w4a8_gemm_swiglu_ws(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, H_bf16, M, N, K, workspace,
                                         workspace_bytes, workspace_prepared, stream);
    if (g != FQ_OK) return g;
    if (next_workspace) fq_launch_quantize_zp(H_bf16, H_fp8, h_scale, M, NH, next_workspace, s);
    else fq_launch_quantize(H_bf16, H_fp8, h_scale, M, NH, s);
    return after_launch();
}

namespace {

inline size_t round16(size_t v) { return (v + 15u) & ~(size_t)15u; }

// one kernel for the whole layer: a few rows, and no kernel forced from outside
bool linear_is_fused(int M, int N, int K) {
    const GemmKernel k = forced_kernel();
    return (k == GemmKernel::Auto || k == GemmKernel::Small) && fq_linear_small_serves(M, N, K);
}

}  // namespace

size_t fq_w4a8_linear_workspace_bytes(int M, int N, int K) {
    if (M <= 0 || N <= 0 || K <= 0 || (K % FQ_GROUP) != 0) return 0;
    // (more rows and longer ones keep the size they have had, whichever kernels run)
    if (M <= 6 && K <= 4096 && linear_is_fused(M, N, K)) return 0;
    return round16((size_t)M * (size_t)K) + round16((size_t)M * sizeof(float)) + fq_w4a8_gemm_workspace_bytes(M, N, K);
}

int fq_w4a8_linear_ws(const uint16_t* X_bf16, const uint8_t* Wq_packed, const uint8_t* w_gscale, float w_tscale,
                      uint16_t* Y_bf16, int M, int N, int K, void* workspace, size_t workspace_bytes, void* stream) {
    // the GEMM's checks, with X in the place of the codes (same alignment rule, twice the bytes)
    const int rc = check_gemm_args(X_bf16, X_bf16, Wq_packed, w_gscale, Y_bf16, M, N, K);
    if (rc != FQ_OK || M == 0) return rc;
    if ((unsigned long long)M * (unsigned long long)K * 2ull >= 0xFFFFFF00ull) return FQ_ERR_SHAPE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const size_t need = fq_w4a8_linear_workspace_bytes(M, N, K);
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return FQ_ERR_MEMORY;
        if (!aligned16(workspace)) return FQ_ERR_ALIGN;
    }
    // Y over X (the layer in place): in one kernel a workgroup would write what others have not read yet; of two kernels the first
    // reads all of X.  Shapes without a workspace have one kernel only.
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(X_bf16), y0 = reinterpret_cast<uintptr_t>(Y_bf16);
    const bool apart = y0 >= x0 + (size_t)M * (size_t)K * 2 || x0 >= y0 + (size_t)M * (size_t)N * 2;
    if ((apart || need == 0) && linear_is_fused(M, N, K)) {
        if (fq_launch_linear_small(X_bf16, Wq_packed, w_gscale, w_tscale, Y_bf16, M, N, K, s)) return after_launch();
        return FQ_ERR_LAUNCH;                             // (the predicate and the launcher agree; not reached)
    }
    uint8_t* A = static_cast<uint8_t*>(workspace);
    float* a_scale = reinterpret_cast<float*>(A + round16((size_t)M * (size_t)K));
    uint8_t* gemm_ws = reinterpret_cast<uint8_t*>(a_scale) + round16((size_t)M * sizeof(float));
    const size_t gemm_ws_bytes = fq_w4a8_gemm_workspace_bytes(M, N, K);
    int q;
    if (gemm_ws_bytes > 0) q = fq_quantize_act_ws(X_bf16, A, a_scale, M, K, gemm_ws, gemm_ws_bytes, stream);
    else                   q = fq_quantize_act(X_bf16, A, a_scale, M, K, stream);
    if (q != FQ_OK) return q;
    return fq_w4a8_gemm_ws(A, a_scale, Wq_packed, w_gscale, w_tscale, Y_bf16, M, N, K, gemm_ws, gemm_ws_bytes,
                           gemm_ws_bytes > 0 ? 1 : 0, stream);
}

int fq_w4a8_gemm_lut(const uint8_t* A_fp8, const float* a_scale, const uint8_t* Wq_packed,
                     const uint8_t* w_gscale, float w_tscale, uint16_t* Y_bf16,
                     int M, int N, int K, void* stream) {
    const int rc = check_gemm_args(A_fp8, a_scale, Wq_packed, w_gscale, Y_bf16, M, N, K);
    if (rc != FQ_OK || M == 0) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (forced_kernel() == GemmKernel::Simple)
        fq_launch_gemm_simple(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, Y_bf16, M, N, K, false, nullptr, s, true);
    else
        fq_launch_gemm_large(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, Y_bf16, M, N, K, nullptr, true, false, nullptr, s,
                             true);
    return after_launch();
}

size_t fq_kv4_packed_bytes(int H, int T, int values) {
    if (H <= 0 || T <= 0) return 0;
    return (size_t)H * (values ? fq_kv4_value_bytes(T) : fq_kv4_key_bytes(T));
}

int fq_kv4_pack(const int8_t* codes, uint8_t* packed, int H, int T, int values, void* stream) {
    if (H < 0 || T < 0) return FQ_ERR_SHAPE;
    if (H == 0 || T == 0) return FQ_OK;
    if (!codes || !packed) return FQ_ERR_NULL;
    if (!aligned16(packed)) return FQ_ERR_ALIGN;
    if (fq_kv4_packed_bytes(1, T, values) >= 0xFFFFFF00ull || H > 65535) return FQ_ERR_SHAPE;
    fq_launch_kv4_pack(codes, packed, H, T, values != 0, static_cast<hipStream_t>(stream));
    return after_launch();
}

int fq_kv4_unpack(const uint8_t* packed, int8_t* codes, int H, int T, int values, void* stream) {
    if (H < 0 || T < 0) return FQ_ERR_SHAPE;
    if (H == 0 || T == 0) return FQ_OK;
    if (!codes || !packed) return FQ_ERR_NULL;
    if (!aligned16(packed)) return FQ_ERR_ALIGN;
    if (fq_kv4_packed_bytes(1, T, values) >= 0xFFFFFF00ull || H > 65535) return FQ_ERR_SHAPE;
    fq_launch_kv4_unpack(packed, codes, H, T, values != 0, static_cast<hipStream_t>(stream));
    return after_launch();
}

int fq_kv4_scores(const uint8_t* Q_fp8, const float* q_scale, const uint8_t* K_packed, const uint8_t* k_scale,
                  float out_scale, uint16_t* S_bf16, int H, int R, int T, void* stream) {
    if (H < 0 || R < 0 || T < 0 || R > 64 || H > 65535) return FQ_ERR_SHAPE;
    if (H == 0 || R == 0 || T == 0) return FQ_OK;
    if (!Q_fp8 || !q_scale || !K_packed || !k_scale || !S_bf16) return FQ_ERR_NULL;
    if (!aligned16(Q_fp8) || !aligned16(K_packed)) return FQ_ERR_ALIGN;
    if (fq_kv4_key_bytes(T) >= 0xFFFFFF00ull) return FQ_ERR_SHAPE;
    fq_launch_kv4_scores(Q_fp8, q_scale, K_packed, k_scale, out_scale, S_bf16, H, R, T, static_cast<hipStream_t>(stream));
    return after_launch();
}

size_t fq_kv4_output_workspace_bytes(int H, int R, int T) {
    if (H <= 0 || R <= 0 || T <= 0 || R > 32) return 0;
    return fq_kv4_output_scratch_bytes(H, R, T);
}

int fq_kv4_output_ws(const uint8_t* P_fp8, const float* p_scale, const uint8_t* V_packed, const uint8_t* v_scale,
                     uint16_t* O_bf16, int H, int R, int T, int ldp, void* workspace, size_t workspace_bytes, void* stream) {
    if (H < 0 || R < 0 || T < 0 || R > 32 || ldp < T) return FQ_ERR_SHAPE;
    if (H == 0 || R == 0) return FQ_OK;
    if (T == 0) return FQ_ERR_SHAPE;                      // an empty sum: nothing to attend to
    if (!P_fp8 || !p_scale || !V_packed || !v_scale || !O_bf16) return FQ_ERR_NULL;
    if (!aligned16(V_packed)) return FQ_ERR_ALIGN;
    if (fq_kv4_value_bytes(T) >= 0xFFFFFF00ull) return FQ_ERR_SHAPE;
    const size_t need = workspace ? fq_kv4_output_workspace_bytes(H, R, T) : 0;
    if (need > 0) {
        if (workspace_bytes < need) return FQ_ERR_MEMORY;
        if (!aligned16(workspace)) return FQ_ERR_ALIGN;
    }
    fq_launch_kv4_output(P_fp8, p_scale, V_packed, v_scale, O_bf16, H, R, T, ldp, need > 0 ? workspace : nullptr,
                         static_cast<hipStream_t>(stream));
    return after_launch();
}

int fq_kv4_output(const uint8_t* P_fp8, const float* p_scale, const uint8_t* V_packed, const uint8_t* v_scale,
                  uint16_t* O_bf16, int H, int R, int T, int ldp, void* stream) {
    return fq_kv4_output_ws(P_fp8, p_scale, V_packed, v_scale, O_bf16, H, R, T, ldp, nullptr, 0, stream);
}

}  // extern "C"

namespace {

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    return p < q + nb && q < p + na;
}

// The bytes of a paged cache's tiles: n1 x n2 blocks of `per` bytes at two strides.  What lies between them is somebody else's (other layers
// of a pool).
struct blocks {
    const void* base;
    int64_t n1, s1, n2, s2, per;
};
bool overlap(const void* p, size_t n, const blocks& c) {
    if (n == 0 || c.n1 <= 0 || c.n2 <= 0) return false;
    const bool first = c.n1 > 1 && (c.n2 == 1 || c.s1 >= c.s2);                       // the larger stride outside
    const __int128 N = first ? c.n1 : c.n2, S = first ? c.s1 : c.s2, m = first ? c.n2 : c.n1, s = first ? c.s2 : c.s1, per = c.per;
    const __int128 a = (__int128)reinterpret_cast<uintptr_t>(p) - (__int128)reinterpret_cast<uintptr_t>(c.base), b = a + (__int128)n, w = (m - 1) * s + per;
    if (b <= 0 || a >= (N - 1) * S + w) return false;
    if (N > 1 && w > S) return true;                      // (not one inside the other: the whole span)
    const __int128 i0 = a < w ? 0 : (a - w) / S + 1, i1 = N == 1 ? 0 : (b - 1) / S;
    for (__int128 i = i0; i <= i1 && i < N; ++i) {        // (one that is not the first or the last lies in the range as a whole)
        const __int128 x = a - i * S, y = b - i * S, j0 = x < per ? 0 : (x - per) / s + 1;
        if (y > 0 && j0 < m && j0 * s < y) return true;
    }
    return false;
}

// Whether an array meets one of `n` others; empty ones do not.
struct bytes {
    const void* p;
    size_t n;
};
bool meet(const bytes& out, const bytes* others, int n) {
    for (int i = 0; i < n; ++i)
        if (out.n > 0 && others[i].n > 0 && overlap(out.p, out.n, others[i].p, others[i].n)) return true;
    return false;
}

// Checks shared by the norms; `out`: Y_bf16 or A_fp8, `per`: its bytes per number.
int check_norm(const uint16_t* X, const uint16_t* R, const uint16_t* w, float eps, const uint16_t* H, const void* out, size_t per, int M, int K) {
    // (a grid holds fewer than 2^32 threads, 1024 of them for a long row)
    if (M < 0 || M >= 1 << 22 || K <= 0 || (K % 8) != 0 || !(eps > 0.f) || !(eps <= 3.402823466e38f)) return FQ_ERR_SHAPE;
    if (M == 0) return FQ_OK;
    if (!X || !w || !out || (R != nullptr) != (H != nullptr)) return FQ_ERR_NULL;
    if (!aligned16(X) || !aligned16(w) || !aligned16(out) || !aligned16(R) || !aligned16(H)) return FQ_ERR_ALIGN;
    const size_t n = (size_t)M * K * 2, no = (size_t)M * K * per;
    if (H && ((H != X && overlap(H, n, X, n)) || (H != R && overlap(H, n, R, n)) || overlap(H, n, w, (size_t)K * 2) || overlap(H, n, out, no)))
        return FQ_ERR_SHAPE;
    const bool whole = per == 2;                          // a bf16 output may take an input's place
    if (overlap(out, no, w, (size_t)K * 2) || (!(whole && out == X) && overlap(out, no, X, n)) || (R && !(whole && out == R) && overlap(out, no, R, n)))
        return FQ_ERR_SHAPE;
    return FQ_OK;
}

// The GEMM's workspace, where a quantising norm is to prepare it: NULL in `planes` where there is nothing to prepare.
int norm_workspace(int M, int K, void* workspace, size_t workspace_bytes, void*& planes) {
    planes = nullptr;
    if (!workspace || choose_kernel(M) != GemmKernel::Large) return FQ_OK;
    if (!fq_quantize_can_write_zero_point(K)) return FQ_ERR_SHAPE;
    if (workspace_bytes < fq_gemm_large_workspace_bytes(M, K)) return FQ_ERR_MEMORY;
    if (!aligned16(workspace)) return FQ_ERR_ALIGN;
    planes = workspace;
    return FQ_OK;
}

// Both forms of the norm between two blocks (Y, or A and a_scale).
int norm_block(const uint16_t* X, const uint16_t* post, const uint16_t* gate, const int32_t* gate_rows, int gates, float scale, const uint16_t* R,
               const uint16_t* w, float eps, uint16_t* H, uint16_t* Y, uint8_t* A, float* a_scale, int M, int K, void* workspace, size_t workspace_bytes,
               void* stream) {
    const void* out = Y ? static_cast<const void*>(Y) : A;
    int rc = check_norm(X, R, w, eps, H, out, Y ? 2 : 1, M, K);
    if (rc != FQ_OK) return rc;
    if (!(scale >= -3.402823466e38f && scale <= 3.402823466e38f)) return FQ_ERR_SHAPE;
    if (gate && (gates < 1 || (!gate_rows && gates != 1 && gates != M))) return FQ_ERR_SHAPE;
    if (M == 0) return FQ_OK;
    if (!R || (!Y && !a_scale) || (gate_rows && !gate)) return FQ_ERR_NULL;
    if (!aligned16(post) || !aligned16(gate)) return FQ_ERR_ALIGN;
    void* planes;
    rc = norm_workspace(M, K, workspace, workspace_bytes, planes);
    if (rc != FQ_OK) return rc;
    const size_t n = (size_t)M * K;
    const bytes in[] = {{post, post ? (size_t)K * 2 : 0}, {gate, gate ? (size_t)gates * K * 2 : 0}, {gate_rows, gate_rows ? (size_t)M * 4 : 0},
                        {X, n * 2}, {R, n * 2}, {w, (size_t)K * 2}, {H, n * 2}, {out, n * (Y ? 2 : 1)},
                        {a_scale, a_scale ? (size_t)M * 4 : 0}, {planes, planes ? fq_gemm_large_workspace_bytes(M, K) : 0}};
    if (meet(in[6], in, 3) || meet(in[7], in, 3) || meet(in[8], in, 8) || meet(in[9], in, 9)) return FQ_ERR_SHAPE;
    fq_launch_rmsnorm_block(X, {post, gate, gate_rows, gate ? gates : 1, scale}, R, w, eps, H, Y, A, a_scale, M, K, planes, static_cast<hipStream_t>(stream));
    return after_launch();
}

// A paged cache's geometry.
int check_paged(const uint8_t* cache, int64_t page_stride, int64_t head_stride, int pages, int page, int heads) {
    if (pages < 0 || page <= 0 || page % FQ_KV4_TILE_TOKENS != 0 || heads <= 0 || heads > 65535) return FQ_ERR_SHAPE;
    const int64_t per = (int64_t)(page / FQ_KV4_TILE_TOKENS) * FQ_KV4_TILE_BYTES;
    if (page_stride <= 0 || head_stride <= 0 || page_stride % 16 != 0 || head_stride % 16 != 0 || per > 0x7FFFFFFF) return FQ_ERR_SHAPE;
    // (the kernels count a page's 16-byte units and a cache's tiles in 32 bits)
    if ((page_stride >> 36) != 0 || (int64_t)pages * (page / FQ_KV4_TILE_TOKENS) > 0xFFFFFFFFll) return FQ_ERR_SHAPE;
    if ((heads > 1 && head_stride < per) || (pages > 1 && page_stride < per)) return FQ_ERR_SHAPE;
    if (pages > 0 && !cache) return FQ_ERR_NULL;
    if (!aligned16(cache)) return FQ_ERR_ALIGN;
    return FQ_OK;
}

blocks paged_blocks(const uint8_t* cache, int64_t page_stride, int64_t head_stride, int pages, int page, int heads) {
    return {cache, pages, page_stride, heads, head_stride, (int64_t)(page / FQ_KV4_TILE_TOKENS) * FQ_KV4_TILE_BYTES};
}

// The sizes that the attention takes.
bool attention_sizes(int B, int Hq, int Hkv, int max_len, int prefix_len) {
    return B >= 0 && B <= 65535 && Hq > 0 && Hq <= 65535 && Hkv > 0 && Hq % Hkv == 0 && (int64_t)B * Hq <= 1 << 23 &&
           (int64_t)Hkv * ((Hq / Hkv + 15) / 16) <= 65535 && max_len >= 0 && max_len <= 1 << 30 && prefix_len >= 0 && prefix_len <= 1 << 30;
}

int attend(const uint8_t* Q_fp8, const float* q_scale, const uint8_t* cache, int64_t page_stride, int64_t head_stride, int pages, int page,
           const int32_t* prefix_pages, int prefix_len, const int32_t* block_table, int table_width, const int32_t* seq_lens,
           float out_scale, uint16_t* O_bf16, int B, int Hq, int Hkv, int max_len, void* workspace, size_t workspace_bytes, void* stream) {
    if (!attention_sizes(B, Hq, Hkv, max_len, prefix_len) || table_width < 0 || !(out_scale > 0.f) || !(out_scale <= 3.402823466e38f)) return FQ_ERR_SHAPE;
    const int rc = check_paged(cache, page_stride, head_stride, pages, page, Hkv);
    if (rc != FQ_OK) return rc;
    if (B == 0) return FQ_OK;
    if (!Q_fp8 || !q_scale || !seq_lens || !O_bf16 || (table_width > 0 && !block_table) || (prefix_len > 0 && !prefix_pages)) return FQ_ERR_NULL;
    if (!aligned16(Q_fp8) || !aligned16(O_bf16)) return FQ_ERR_ALIGN;
    if (pages == 0 && (prefix_len > 0 || (table_width > 0 && max_len > 0))) return FQ_ERR_SHAPE;   // no page to fall back on
    const size_t need = fq_attend_scratch_bytes(B, Hq, Hkv, max_len, prefix_len);
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return FQ_ERR_MEMORY;
        if (!aligned16(workspace)) return FQ_ERR_ALIGN;
    }
    // (workgroups that have not begun still read what an output would have changed)
    const size_t rows = (size_t)B * Hq;
    const bytes in[] = {{Q_fp8, rows * 128}, {q_scale, rows * 4}, {block_table, (size_t)B * table_width * 4}, {seq_lens, (size_t)B * 4},
                        {prefix_pages, ((size_t)prefix_len + page - 1) / page * 4}, {workspace, need}};
    const blocks c = paged_blocks(cache, page_stride, head_stride, pages, page, Hkv);
    if (meet({O_bf16, rows * 256}, in, 6) || overlap(O_bf16, rows * 256, c) || meet({workspace, need}, in, 5) || overlap(workspace, need, c)) return FQ_ERR_SHAPE;
    const fq_attend_args a = {Q_fp8, q_scale, {const_cast<uint8_t*>(cache), page_stride, head_stride, pages, page}, prefix_pages, block_table,
                              seq_lens, prefix_len, table_width, out_scale, O_bf16, B, Hq, Hkv, max_len};
    fq_launch_attend(a, workspace, static_cast<hipStream_t>(stream));
    return after_launch();
}

// axis_of_pair NULL: one axis for all pairs.
int append(const uint16_t* QKV_bf16, int64_t ld, const float* cos_sin, int max_positions, const int32_t* positions, int axes, const int8_t* axis_of_pair,
           const int64_t* slots, int interleaved, uint8_t* Q_fp8, float* q_scale, uint8_t* cache, int64_t page_stride, int64_t head_stride, int pages,
           int page, int T, int Hq, int Hkv, void* stream) {
    if (T < 0 || Hq <= 0 || Hq > 65535 || Hkv <= 0 || Hq % Hkv != 0 || max_positions < 0) return FQ_ERR_SHAPE;
    const int rc = check_paged(cache, page_stride, head_stride, pages, page, Hkv);
    if (rc != FQ_OK) return rc;
    const int64_t heads = (int64_t)Hq + 2 * (int64_t)Hkv;
    if (ld < heads * 128 || ld % 8 != 0 || (int64_t)T * heads > (int64_t)0x0FFFFFF0 || T >= 1 << 23) return FQ_ERR_SHAPE;
    if (T == 0) return FQ_OK;
    if (!QKV_bf16 || !positions || !slots || !Q_fp8 || !q_scale || (max_positions > 0 && !cos_sin)) return FQ_ERR_NULL;
    if (!aligned16(QKV_bf16) || !aligned16(cos_sin) || !aligned16(Q_fp8)) return FQ_ERR_ALIGN;
    const size_t rows = (size_t)T * Hq;
    const bytes in[] = {{cos_sin, (size_t)max_positions * 512}, {positions, (size_t)T * 4 * axes}, {slots, (size_t)T * 8}, {Q_fp8, rows * 128}, {q_scale, rows * 4}};
    const blocks all = paged_blocks(cache, page_stride, head_stride, pages, page, Hkv), tokens = {QKV_bf16, T, ld * 2, 1, 0, heads * 256};
    if (meet(in[3], in, 3) || meet(in[4], in, 4) || overlap(Q_fp8, rows * 128, tokens) || overlap(q_scale, rows * 4, tokens) ||
        overlap(QKV_bf16, ((size_t)(T - 1) * ld + heads * 128) * 2, all))
        return FQ_ERR_SHAPE;
    for (const bytes& x : in)
        if (overlap(x.p, x.n, all)) return FQ_ERR_SHAPE;
    const fq_paged_cache c = {cache, page_stride, head_stride, pages, page};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    bool one = true;                                      // all pairs turn by one axis: 6001 tokens 24 us, 27 by the form for several
    for (int j = 0; axis_of_pair && j < 64; ++j) one = one && axis_of_pair[j] == axis_of_pair[0] && axis_of_pair[0] >= 0;
    if (one) {
        if (axis_of_pair) positions += (size_t)axis_of_pair[0] * T;
        fq_launch_kv4_append(QKV_bf16, ld, cos_sin, max_positions, positions, slots, interleaved != 0, Q_fp8, q_scale, c, T, Hq, Hkv, st);
        return after_launch();
    }
    fq_pair_axes axis;
    std::memcpy(axis.four, axis_of_pair, 64);
    axis.axes = axes;
    axis.used = 0;
    for (int j = 0; j < 64; ++j)
        if (axis_of_pair[j] >= 0 && axis_of_pair[j] < 32) axis.used |= 1u << axis_of_pair[j];
    fq_launch_kv4_append_axes(QKV_bf16, ld, cos_sin, max_positions, positions, axis, slots, interleaved != 0, Q_fp8, q_scale, c, T, Hq, Hkv, st);
    return after_launch();
}

// The sizes that the attention of new tokens takes.
bool chunk_sizes(int T, int B, int Hq, int Hkv, int max_new, int max_len) {
    return T >= 0 && T < 1 << 23 && B >= 0 && B <= 65535 && Hq > 0 && Hq <= 65535 && Hkv > 0 && Hq % Hkv == 0 && (int64_t)T * Hq <= 1 << 25 &&
           ((int64_t)T * (Hq / Hkv) / 16 + B) * Hkv < 1 << 24 && max_new >= 0 && max_len >= 0 && max_len <= 1 << 30;
}

int attend_chunk(const fq_chunk_args& a, void* workspace, size_t workspace_bytes, void* stream) {
    if (!chunk_sizes(a.T, a.B, a.Hq, a.Hkv, a.max_new, a.max_len) || a.width < 0 || a.window < 0 || !(a.out_scale > 0.f) || !(a.out_scale <= 3.402823466e38f) ||
        !(a.cap == 0.f || (a.cap >= 0x1p-60f && a.cap <= 3.402823466e38f)) || (a.cap > 0.f && !(a.out_scale / a.cap <= 3.402823466e38f)))
        return FQ_ERR_SHAPE;
    const fq_paged_cache& c = a.c;
    const int rc = check_paged(c.base, c.page_stride, c.head_stride, c.pages, c.page, a.Hkv);
    if (rc != FQ_OK) return rc;
    if (a.T == 0 || a.B == 0) return FQ_OK;
    if (!a.Q || !a.q_scale || !a.starts || !a.lens || !a.O || (a.width > 0 && !a.table)) return FQ_ERR_NULL;
    if (!aligned16(a.Q) || !aligned16(a.O)) return FQ_ERR_ALIGN;
    if (c.pages == 0 && a.width > 0 && a.max_len > 0) return FQ_ERR_SHAPE;   // no page to fall back on
    const size_t need = fq_chunk_scratch_bytes(a.T, a.B, a.Hq, a.Hkv, a.max_new, a.max_len);
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return FQ_ERR_MEMORY;
        if (!aligned16(workspace)) return FQ_ERR_ALIGN;
    }
    const size_t rows = (size_t)a.T * a.Hq;
    const bytes in[] = {{a.Q, rows * 128}, {a.q_scale, rows * 4}, {a.table, (size_t)a.B * a.width * 4}, {a.starts, (size_t)a.B * 4 + 4}, {a.lens, (size_t)a.B * 4},
                        {a.first, a.first ? (size_t)a.T * 4 : 0}, {a.end, a.end ? (size_t)a.T * 4 : 0}, {a.slopes, a.slopes ? (size_t)a.Hq * 4 : 0}, {workspace, need}};
    const blocks all = paged_blocks(c.base, c.page_stride, c.head_stride, c.pages, c.page, a.Hkv);
    if (meet({a.O, rows * 256}, in, 9) || overlap(a.O, rows * 256, all) || meet({workspace, need}, in, 8) || overlap(workspace, need, all)) return FQ_ERR_SHAPE;
    fq_launch_chunk(a, workspace, static_cast<hipStream_t>(stream));
    return after_launch();
}

int sample(const fq_sample_args& a, void* workspace, size_t workspace_bytes, void* stream) {
    const size_t size = a.wide ? 4 : 2;
    if (a.B < 0 || a.B > 65535 || a.V < 1 || a.V > 1 << 20 || a.ld < a.V || a.ld > (int64_t)1 << 40) return FQ_ERR_SHAPE;
    if (a.B == 0) return FQ_OK;
    if (!a.logits || !a.u || !a.token) return FQ_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(a.logits) % size != 0) return FQ_ERR_ALIGN;
    const size_t need = fq_sample_scratch_bytes(a.B, a.V);
    if (need > 0) {
        if (!workspace || workspace_bytes < need) return FQ_ERR_MEMORY;
        if (!aligned16(workspace)) return FQ_ERR_ALIGN;
    }
    const size_t n = (size_t)a.B * 4;
    const blocks rows = {a.logits, a.B, (int64_t)(a.ld * size), 1, 0, (int64_t)(a.V * size)};
    const bytes all[] = {{a.u, n}, {a.temperature, a.temperature ? n : 0}, {a.top_k, a.top_k ? n : 0}, {a.top_p, a.top_p ? n : 0}, {a.min_p, a.min_p ? n : 0},
                         {a.token, n}, {a.logprob, a.logprob ? n : 0}, {workspace, need}};
    for (int i = 5; i < 8; ++i)
        if (meet(all[i], all, i) || overlap(all[i].p, all[i].n, rows)) return FQ_ERR_SHAPE;
    fq_launch_sample(a, workspace, static_cast<hipStream_t>(stream));
    return after_launch();
}

}  // namespace

extern "C" {

int fq_rmsnorm(const uint16_t* X_bf16, const uint16_t* R_bf16, const uint16_t* w_bf16, float eps, uint16_t* H_bf16, uint16_t* Y_bf16,
               int M, int K, void* stream) {
    const int rc = check_norm(X_bf16, R_bf16, w_bf16, eps, H_bf16, Y_bf16, 2, M, K);
    if (rc != FQ_OK || M == 0) return rc;
    fq_launch_rmsnorm(X_bf16, R_bf16, w_bf16, eps, H_bf16, Y_bf16, M, K, static_cast<hipStream_t>(stream));
    return after_launch();
}

int fq_rmsnorm_quant_ws(const uint16_t* X_bf16, const uint16_t* R_bf16, const uint16_t* w_bf16, float eps, uint16_t* H_bf16,
                        uint8_t* A_fp8, float* a_scale, int M, int K, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_norm(X_bf16, R_bf16, w_bf16, eps, H_bf16, A_fp8, 1, M, K);
    if (rc != FQ_OK || M == 0) return rc;
    if (!a_scale) return FQ_ERR_NULL;
    void* planes = nullptr;
    const int ws = norm_workspace(M, K, workspace, workspace_bytes, planes);
    if (ws != FQ_OK) return ws;
    const size_t n = (size_t)M * K;
    const bytes in[] = {{X_bf16, n * 2}, {R_bf16, R_bf16 ? n * 2 : 0}, {w_bf16, (size_t)K * 2}, {H_bf16, H_bf16 ? n * 2 : 0}, {A_fp8, n},
                        {planes, planes ? fq_gemm_large_workspace_bytes(M, K) : 0}};
    if (meet({a_scale, (size_t)M * 4}, in, 6) || meet(in[5], in, 5)) return FQ_ERR_SHAPE;
    fq_launch_rmsnorm_quant(X_bf16, R_bf16, w_bf16, eps, H_bf16, A_fp8, a_scale, M, K, planes, static_cast<hipStream_t>(stream));
    return after_launch();
}

int fq_kv4_append(const uint16_t* QKV_bf16, int64_t ld, const float* cos_sin, int max_positions, const int32_t* positions,
                  const int64_t* slots, int interleaved, uint8_t* Q_fp8, float* q_scale, uint8_t* cache, int64_t page_stride,
                  int64_t head_stride, int pages, int page, int T, int Hq, int Hkv, void* stream) {
    return append(QKV_bf16, ld, cos_sin, max_positions, positions, 1, nullptr, slots, interleaved, Q_fp8, q_scale, cache, page_stride, head_stride, pages,
                  page, T, Hq, Hkv, stream);
}

int fq_kv4_append_axes(const uint16_t* QKV_bf16, int64_t ld, const float* cos_sin, int max_positions, const int32_t* positions, int axes,
                       const int8_t* axis_of_pair, const int64_t* slots, int interleaved, uint8_t* Q_fp8, float* q_scale, uint8_t* cache,
                       int64_t page_stride, int64_t head_stride, int pages, int page, int T, int Hq, int Hkv, void* stream) {
    if (axes < 1 || axes > 127) return FQ_ERR_SHAPE;
    if (!axis_of_pair) return T == 0 ? FQ_OK : FQ_ERR_NULL;
    for (int j = 0; j < 64; ++j)
        if (axis_of_pair[j] < -1 || axis_of_pair[j] >= axes) return FQ_ERR_SHAPE;
    return append(QKV_bf16, ld, cos_sin, max_positions, positions, axes, axis_of_pair, slots, interleaved, Q_fp8, q_scale, cache, page_stride,
                  head_stride, pages, page, T, Hq, Hkv, stream);
}

int fq_kv4_read(const uint8_t* cache, int64_t page_stride, int64_t head_stride, int pages, int page, const int64_t* slots,
                uint16_t* K_bf16, uint16_t* V_bf16, int n, int Hkv, void* stream) {
    if (n < 0) return FQ_ERR_SHAPE;
    const int rc = check_paged(cache, page_stride, head_stride, pages, page, Hkv);
    if (rc != FQ_OK) return rc;
    if ((int64_t)n * Hkv > (int64_t)0x0FFFFFF0) return FQ_ERR_SHAPE;
    if (n == 0) return FQ_OK;
    if (!slots || !K_bf16 || !V_bf16) return FQ_ERR_NULL;
    if (!aligned16(K_bf16) || !aligned16(V_bf16)) return FQ_ERR_ALIGN;
    const size_t out = (size_t)n * Hkv * 256;
    const bytes in[] = {{slots, (size_t)n * 8}, {K_bf16, out}};
    const blocks all = paged_blocks(cache, page_stride, head_stride, pages, page, Hkv);
    if (meet({K_bf16, out}, in, 1) || meet({V_bf16, out}, in, 2) || overlap(K_bf16, out, all) || overlap(V_bf16, out, all)) return FQ_ERR_SHAPE;
    const fq_paged_cache c = {const_cast<uint8_t*>(cache), page_stride, head_stride, pages, page};
    fq_launch_kv4_read(c, slots, K_bf16, V_bf16, n, Hkv, static_cast<hipStream_t>(stream));
    return after_launch();
}

size_t fq_kv4_attention_workspace_bytes(int B, int Hq, int Hkv, int max_len, int prefix_len) {
    if (B <= 0 || !attention_sizes(B, Hq, Hkv, max_len, prefix_len)) return 0;
    return fq_attend_scratch_bytes(B, Hq, Hkv, max_len, prefix_len);
}

int fq_kv4_attention_ws(const uint8_t* Q_fp8, const float* q_scale, const uint8_t* cache, int64_t page_stride, int64_t head_stride,
                        int pages, int page, const int32_t* block_table, int table_width, const int32_t* seq_lens, float out_scale,
                        uint16_t* O_bf16, int B, int Hq, int Hkv, int max_len, void* workspace, size_t workspace_bytes, void* stream) {
    return attend(Q_fp8, q_scale, cache, page_stride, head_stride, pages, page, nullptr, 0, block_table, table_width, seq_lens, out_scale,
                  O_bf16, B, Hq, Hkv, max_len, workspace, workspace_bytes, stream);
}

int fq_kv4_attention_prefix_ws(const uint8_t* Q_fp8, const float* q_scale, const uint8_t* cache, int64_t page_stride,
                               int64_t head_stride, int pages, int page, const int32_t* prefix_pages, int prefix_len,
                               const int32_t* block_table, int table_width, const int32_t* seq_lens, float out_scale,
                               uint16_t* O_bf16, int B, int Hq, int Hkv, int max_len, void* workspace, size_t workspace_bytes,
                               void* stream) {
    return attend(Q_fp8, q_scale, cache, page_stride, head_stride, pages, page, prefix_pages, prefix_len, block_table, table_width, seq_lens,
                  out_scale, O_bf16, B, Hq, Hkv, max_len, workspace, workspace_bytes, stream);
}

int fq_rmsnorm_block(const uint16_t* X_bf16, const uint16_t* post_bf16, const uint16_t* gate_bf16, const int32_t* gate_rows, int gates,
                     float scale, const uint16_t* R_bf16, const uint16_t* w_bf16, float eps, uint16_t* H_bf16, uint16_t* Y_bf16, int M, int K,
                     void* stream) {
    if (M > 0 && !Y_bf16) return FQ_ERR_NULL;
    return norm_block(X_bf16, post_bf16, gate_bf16, gate_rows, gates, scale, R_bf16, w_bf16, eps, H_bf16, Y_bf16, nullptr, nullptr, M, K, nullptr, 0,
                      stream);
}

int fq_rmsnorm_block_quant_ws(const uint16_t* X_bf16, const uint16_t* post_bf16, const uint16_t* gate_bf16, const int32_t* gate_rows,
                              int gates, float scale, const uint16_t* R_bf16, const uint16_t* w_bf16, float eps, uint16_t* H_bf16,
                              uint8_t* A_fp8, float* a_scale, int M, int K, void* workspace, size_t workspace_bytes, void* stream) {
    return norm_block(X_bf16, post_bf16, gate_bf16, gate_rows, gates, scale, R_bf16, w_bf16, eps, H_bf16, nullptr, A_fp8, a_scale, M, K, workspace,
                      workspace_bytes, stream);
}

size_t fq_kv4_attention_chunk_workspace_bytes(int T, int B, int Hq, int Hkv, int max_new, int max_len) {
    if (T <= 0 || B <= 0 || !chunk_sizes(T, B, Hq, Hkv, max_new, max_len)) return 0;
    return fq_chunk_scratch_bytes(T, B, Hq, Hkv, max_new, max_len);
}

int fq_kv4_attention_chunk_ws(const uint8_t* Q_fp8, const float* q_scale, const uint8_t* cache, int64_t page_stride, int64_t head_stride,
                              int pages, int page, const int32_t* block_table, int table_width, const int32_t* starts,
                              const int32_t* seq_lens, const int32_t* first, const int32_t* end, int window, float cap, const float* slopes,
                              float out_scale, uint16_t* O_bf16, int T, int B, int Hq, int Hkv, int max_new, int max_len, void* workspace,
                              size_t workspace_bytes, void* stream) {
    return attend_chunk({Q_fp8, q_scale, {const_cast<uint8_t*>(cache), page_stride, head_stride, pages, page}, block_table, starts, seq_lens, first, end,
                         slopes, table_width, window, T, B, Hq, Hkv, max_new, max_len, out_scale, cap, O_bf16},
                        workspace, workspace_bytes, stream);
}

size_t fq_sample_workspace_bytes(int B, int V) { return B > 0 && B <= 65535 && V > 0 && V <= 1 << 20 ? fq_sample_scratch_bytes(B, V) : 0; }

int fq_sample_bf16_ws(const uint16_t* logits, int64_t ld, const float* u, const float* temperature, const int32_t* top_k,
                      const float* top_p, const float* min_p, int32_t* token, float* logprob, int B, int V, void* workspace,
                      size_t workspace_bytes, void* stream) {
    return sample({logits, false, ld, u, temperature, top_p, min_p, top_k, token, logprob, B, V}, workspace, workspace_bytes, stream);
}

int fq_sample_fp32_ws(const float* logits, int64_t ld, const float* u, const float* temperature, const int32_t* top_k, const float* top_p,
                      const float* min_p, int32_t* token, float* logprob, int B, int V, void* workspace, size_t workspace_bytes, void* stream) {
    return sample({logits, true, ld, u, temperature, top_p, min_p, top_k, token, logprob, B, V}, workspace, workspace_bytes, stream);
}

size_t fq_w4a8_gemm_static_max_workspace(void) { return FQ_STATIC_SCRATCH_BYTES; }

int fq_w4a8_gemm_static(const uint8_t* A_fp8, const float* a_scale, const uint8_t* Wq_packed,
                        const uint8_t* w_gscale, float w_tscale, uint16_t* Y_bf16,
                        int M, int N, int K, void* stream) {
    const int rc = check_gemm_args(A_fp8, a_scale, Wq_packed, w_gscale, Y_bf16, M, N, K);
    if (rc != FQ_OK || M == 0) return rc;
    const size_t need = fq_w4a8_gemm_workspace_bytes(M, N, K);
    if (need > FQ_STATIC_SCRATCH_BYTES) return FQ_ERR_MEMORY;
    // the device address of this GPU's copy of the array, looked up once per device
    static std::mutex m;
    static void* ptr[FQ_MAX_DEVICES];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= FQ_MAX_DEVICES) {
        (void)hipGetLastError();
        return FQ_ERR_LAUNCH;
    }
    void* ws;
    {
        std::lock_guard<std::mutex> lock(m);
        if (!ptr[dev]) {
            void* p = nullptr;
            if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) {
                (void)hipGetLastError();
                return FQ_ERR_MEMORY;
            }
            ptr[dev] = p;
        }
        ws = ptr[dev];
    }
    // every byte of the scratch this call reads is written by this call first (the zero-point pre-pass
    // fills all units of all M rows), so nothing needs clearing between calls
    return fq_w4a8_gemm_ws(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, Y_bf16, M, N, K, ws, FQ_STATIC_SCRATCH_BYTES, 0,
                           stream);
}

int fq_w4a8_gemm(const uint8_t* A_fp8, const float* a_scale, const uint8_t* Wq_packed,
                 const uint8_t* w_gscale, float w_tscale, uint16_t* Y_bf16,
                 int M, int N, int K, void* stream) {
    const int rc = check_gemm_args(A_fp8, a_scale, Wq_packed, w_gscale, Y_bf16, M, N, K);
    if (rc != FQ_OK || M == 0) return rc;
    // the library's own workspace: one grow-only device buffer, shared by every call of the process
    // (the mutex keeps the bookkeeping whole when several host threads call; the kernels of overlapping
    // calls still share the buffer, as the header says)
    static std::mutex ws_mutex;
    static void* ws = nullptr;
    static size_t ws_bytes = 0;
    const size_t need = fq_w4a8_gemm_workspace_bytes(M, N, K);
    std::lock_guard<std::mutex> lock(ws_mutex);
    if (need > ws_bytes) {
        if (ws) (void)hipFree(ws);
        ws = nullptr;
        ws_bytes = 0;
        if (hipMalloc(&ws, need) != hipSuccess) {
            (void)hipGetLastError();
            return FQ_ERR_MEMORY;
        }
        ws_bytes = need;
    }
    return fq_w4a8_gemm_ws(A_fp8, a_scale, Wq_packed, w_gscale, w_tscale, Y_bf16, M, N, K, ws, ws_bytes, 0, stream);
}

}  // extern "C"
