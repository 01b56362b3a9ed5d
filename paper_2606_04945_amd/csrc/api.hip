// C ABI of libstarquant: argument checks, workspace layout and kernel dispatch.
// Every argument is checked before the first launch; on failure nothing is
// enqueued and the reason is kept in a thread-local message.
#include <stdarg.h>
#include <stdlib.h>
#include <stdio.h>

#include <math.h>

#include <atomic>
#include <mutex>

#include "../../include/starquant.h"
#include "layer.hpp"
#include "norm_plan.hpp"
#include "serve.hpp"

namespace {

thread_local char g_err[512] = "";

int fail(int code, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return code;
}

// SQ_DEBUG_SYNC set to anything but "" or "0" (read once, at the first call):
// every launch is followed by a device-wide synchronisation and an error
// check, so an asynchronous fault is reported by the call whose kernel raised
// it, named in the message.  For debugging only: it serialises the device and
// cannot be used under stream capture.
bool debug_sync() {
    static const bool on = [] {
        const char* v = getenv("SQ_DEBUG_SYNC");
        return v != nullptr && v[0] != '\0' && !(v[0] == '0' && v[1] == '\0');
    }();
    return on;
}

int hip_status(hipError_t e, const char* what) {
    if (e == hipSuccess && debug_sync()) {
        e = hipDeviceSynchronize();
        if (e == hipSuccess) e = hipGetLastError();
    }
    if (e == hipSuccess) return SQ_OK;
    return fail(SQ_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// Whether two ranges of bytes have none in common.
bool apart(const void* a, size_t na, const void* b, size_t nb) {
    return (uintptr_t)a + na <= (uintptr_t)b || (uintptr_t)b + nb <= (uintptr_t)a;
}

// Row-tiled launches put row tiles (at least 64 rows each) on the second grid
// axis, which holds at most 65535 workgroups.
constexpr int32_t kMaxTiledRows = 65535 * 64;

constexpr size_t kAlign = 256;
size_t round_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

int check_K(int32_t K) {
    if (K < 64 || K > 131072 || K % 64)
        return fail(SQ_ERR_SHAPE, "K=%d: need 64 <= K <= 131072 and K %% 64 == 0", K);
    return SQ_OK;
}

int check_band(int32_t K, int32_t dm, int32_t du) {
    if (dm < 0 || du < 0 || (int64_t)dm + du >= K)
        return fail(SQ_ERR_SHAPE, "bands d_m=%d d_u=%d: need d_m, d_u >= 0 and d_m + d_u < K=%d", dm, du, K);
    return SQ_OK;
}

int check_tac(int32_t C, int32_t g) {
    if (g < 1 || g > 128 || (g & (g - 1)) || C % g)
        return fail(SQ_ERR_SHAPE, "TAC block g=%d: need a power of two in [1, 128] dividing C=%d", g, C);
    return SQ_OK;
}

#define SQ_REQUIRE(cond, code, ...) \
    do {                            \
        if (!(cond)) return fail(code, __VA_ARGS__); \
    } while (0)

#define SQ_TRY(expr)                 \
    do {                             \
        int _rc = (expr);            \
        if (_rc != SQ_OK) return _rc; \
    } while (0)

}  // namespace

extern "C" {

const char* sq_last_error(void) { return g_err; }

const char* sq_version(void) { return "starquant 0.1 gfx950"; }

int32_t sq_tac_default_block(int32_t C) {
    if (C <= 0) return 0;
    for (int g = 16; g > 1; --g)
        if (C % g == 0) return g;
    return 1;
}

size_t sq_quant_act_workspace_bytes(int32_t M, int32_t K, int32_t has_P, int32_t has_tac) {
    if (M <= 0 || K <= 0) return 0;
    size_t n = 0;
    if (has_tac) n += round_up((size_t)M * K * sizeof(uint16_t));
    if (has_P) n += round_up((size_t)M * K * sizeof(float));
    return n;
}

size_t sq_prepare_weights_workspace_bytes(int32_t N, int32_t K, int32_t has_P) {
    if (N <= 0 || K <= 0 || !has_P) return 0;
    return round_up((size_t)N * K * sizeof(float));
}

size_t sq_gemm_workspace_bytes(int32_t M, int32_t N, int32_t K) {
    if (M <= 0 || N <= 0 || K <= 0) return 0;
    return round_up(sq::gemm_workspace_bytes(M, N, K, 4));
}

size_t sq_gemm_w8_workspace_bytes(int32_t M, int32_t N, int32_t K) {
    if (M <= 0 || N <= 0 || K <= 0) return 0;
    return round_up(sq::gemm_workspace_bytes(M, N, K, 8));
}

}  // extern "C"

namespace {

int prepare_weights(const uint16_t* W, const float* P, int32_t N, int32_t K, uint8_t* Wq, float* s_w, void* ws,
                    size_t ws_bytes, void* stream, int bits, const char* name) {
    SQ_TRY(check_K(K));
    SQ_REQUIRE(N >= 0, SQ_ERR_SHAPE, "N=%d < 0", N);
    if (N == 0) return SQ_OK;
    SQ_REQUIRE(W && Wq && s_w, SQ_ERR_NULL, "%s: W, Wq and s_w are required", name);
    SQ_REQUIRE(aligned16(W) && aligned16(Wq) && aligned16(s_w) && aligned16(P) && aligned16(ws), SQ_ERR_ALIGN,
               "%s: pointers must be 16-byte aligned", name);
    const size_t need = sq_prepare_weights_workspace_bytes(N, K, P != nullptr);
    SQ_REQUIRE(ws_bytes >= need && (need == 0 || ws), SQ_ERR_WORKSPACE, "%s: workspace %zu B < %zu B", name,
               ws_bytes, need);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (!P) return hip_status(sq::launch_quant_f16(W, nullptr, N, K, 0, 0, Wq, s_w, st, bits), "quant_f16");
    float* wp = static_cast<float*>(ws);
    SQ_TRY(hip_status(sq::launch_transform(W, nullptr, P, N, K, 0, 0, wp, st), "transform"));
    return hip_status(sq::launch_quant_f32(wp, N, K, Wq, s_w, st, bits), "quant_f32");
}

int quantize(const float* Xp, int32_t M, int32_t K, uint8_t* Aq, float* s, void* stream, int bits,
             const char* name) {
    SQ_TRY(check_K(K));
    SQ_REQUIRE(M >= 0, SQ_ERR_SHAPE, "M=%d < 0", M);
    if (M == 0) return SQ_OK;
    SQ_REQUIRE(Xp && Aq && s, SQ_ERR_NULL, "%s: Xp, Aq and s are required", name);
    SQ_REQUIRE(aligned16(Xp) && aligned16(Aq) && aligned16(s), SQ_ERR_ALIGN, "%s: pointers must be 16-byte aligned",
               name);
    return hip_status(sq::launch_quant_f32(Xp, M, K, Aq, s, static_cast<hipStream_t>(stream), bits), "quant_f32");
}

int quant_act(const uint16_t* X, const uint8_t* state, const float* P, int32_t M, int32_t K, int32_t d_m,
              int32_t d_u, const uint16_t* tac_M, const uint16_t* tac_d, int32_t g, uint8_t* Aq, float* s_a,
              void* ws, size_t ws_bytes, void* stream, int bits, const char* name) {
    SQ_TRY(check_K(K));
    SQ_TRY(check_band(K, d_m, d_u));
    SQ_REQUIRE(M >= 0, SQ_ERR_SHAPE, "M=%d < 0", M);
    if (tac_M) {
        SQ_REQUIRE(tac_d, SQ_ERR_NULL, "%s: tac_d is required with tac_M", name);
        SQ_TRY(check_tac(K, g));
        SQ_REQUIRE(M <= kMaxTiledRows, SQ_ERR_SHAPE, "%s: M=%d: at most %d rows per call with TAC", name, M,
                   kMaxTiledRows);
    }
    if (M == 0) return SQ_OK;
    SQ_REQUIRE(X && Aq && s_a, SQ_ERR_NULL, "%s: X, Aq and s_a are required", name);
    SQ_REQUIRE(aligned16(X) && aligned16(Aq) && aligned16(s_a) && aligned16(P) && aligned16(ws) &&
                   aligned16(tac_M) && aligned16(tac_d),
               SQ_ERR_ALIGN, "%s: pointers must be 16-byte aligned", name);
    const size_t need = sq_quant_act_workspace_bytes(M, K, P != nullptr, tac_M != nullptr);
    SQ_REQUIRE(ws_bytes >= need && (need == 0 || ws), SQ_ERR_WORKSPACE, "%s: workspace %zu B < %zu B", name,
               ws_bytes, need);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (tac_M && !P && sq::tac_quant_fusable(K, g))
        return hip_status(sq::launch_tac_quant(X, tac_M, tac_d, state, M, K, g, d_m, d_u, Aq, s_a, st, bits),
                          "tac_quant");
    uint8_t* wsb = static_cast<uint8_t*>(ws);
    const uint16_t* src = X;
    if (tac_M) {
        uint16_t* z = reinterpret_cast<uint16_t*>(wsb);
        SQ_TRY(hip_status(sq::launch_tac(X, tac_M, tac_d, M, K, g, z, st), "tac"));
        src = z;
        wsb += round_up((size_t)M * K * sizeof(uint16_t));
    }
    if (!P) return hip_status(sq::launch_quant_f16(src, state, M, K, d_m, d_u, Aq, s_a, st, bits), "quant_f16");
    float* xp = reinterpret_cast<float*>(wsb);
    SQ_TRY(hip_status(sq::launch_transform(src, state, P, M, K, d_m, d_u, xp, st), "transform"));
    return hip_status(sq::launch_quant_f32(xp, M, K, Aq, s_a, st, bits), "quant_f32");
}

int gemm(const uint8_t* Aq, const float* s_a, const uint8_t* Wq, const float* s_w, int32_t M, int32_t N, int32_t K,
         uint16_t* Y, int32_t* acc, void* ws, size_t ws_bytes, void* stream, int bits, const char* name) {
    SQ_TRY(check_K(K));
    SQ_REQUIRE(bits == 4 || K <= 65536, SQ_ERR_SHAPE, "%s: K=%d: 8-bit codes need K <= 65536", name, K);
    SQ_REQUIRE(M >= 0 && N >= 0, SQ_ERR_SHAPE, "M=%d N=%d: need >= 0", M, N);
    SQ_REQUIRE(M <= kMaxTiledRows, SQ_ERR_SHAPE, "%s: M=%d: at most %d rows per call", name, M, kMaxTiledRows);
    SQ_REQUIRE(N % 8 == 0, SQ_ERR_SHAPE, "N=%d: need N %% 8 == 0", N);
    // operand rows are addressed with 32-bit buffer offsets
    const size_t row_bytes = (size_t)K * bits / 8;
    SQ_REQUIRE((size_t)M * row_bytes < (1u << 31) && (size_t)N * row_bytes < (1u << 31), SQ_ERR_SHAPE,
               "%s: each operand must be under 2 GiB (M=%d N=%d K=%d)", name, M, N, K);
    if (M == 0 || N == 0) return SQ_OK;
    SQ_REQUIRE(Aq && s_a && Wq && s_w && (Y || acc), SQ_ERR_NULL,
               "%s: Aq, s_a, Wq, s_w and one of Y / acc are required", name);
    SQ_REQUIRE(aligned16(Aq) && aligned16(s_a) && aligned16(Wq) && aligned16(s_w) && aligned16(Y) &&
                   aligned16(acc) && aligned16(ws),
               SQ_ERR_ALIGN, "%s: pointers must be 16-byte aligned", name);
    const size_t need = bits == 8 ? sq_gemm_w8_workspace_bytes(M, N, K) : sq_gemm_workspace_bytes(M, N, K);
    SQ_REQUIRE(ws_bytes >= need && (need == 0 || ws), SQ_ERR_WORKSPACE, "%s: workspace %zu B < %zu B", name,
               ws_bytes, need);
    return hip_status(
        sq::launch_gemm(Aq, s_a, Wq, s_w, M, N, K, Y, acc, ws, static_cast<hipStream_t>(stream), bits), "gemm");
}

// Shared argument checks of the fragment-ordered GEMM entry points; *done is
// set when there is nothing to compute (M == 0 or N == 0).
int check_gemm_frag(const uint8_t* Aq, const float* s_a, const uint8_t* Wf, const float* s_w, int32_t M, int32_t N,
                    int32_t K, uint16_t* Y, int32_t* acc, int bits, const char* name, int* done) {
    SQ_TRY(check_K(K));
    SQ_REQUIRE(bits == 4 || K <= 65536, SQ_ERR_SHAPE, "%s: K=%d: 8-bit codes need K <= 65536", name, K);
    SQ_REQUIRE(M >= 0 && N >= 0, SQ_ERR_SHAPE, "M=%d N=%d: need >= 0", M, N);
    SQ_REQUIRE(M <= kMaxTiledRows, SQ_ERR_SHAPE, "%s: M=%d: at most %d rows per call", name, M, kMaxTiledRows);
    SQ_REQUIRE(N % 8 == 0, SQ_ERR_SHAPE, "N=%d: need N %% 8 == 0", N);
    // the fragment layout counts a row in int4 codes: an 8-bit row of K bytes is 2 K of them
    SQ_REQUIRE((size_t)M * K * bits / 8 < (1u << 31) && sq::frag_weight_bytes(N, K * bits / 4) < (1u << 31),
               SQ_ERR_SHAPE, "%s: each operand must be under 2 GiB (M=%d N=%d K=%d)", name, M, N, K);
    *done = M == 0 || N == 0;
    if (*done) return SQ_OK;
    SQ_REQUIRE(Aq && s_a && Wf && s_w && (Y || acc), SQ_ERR_NULL,
               "%s: Aq, s_a, Wf, s_w and one of Y / acc are required", name);
    SQ_REQUIRE(aligned16(Aq) && aligned16(s_a) && aligned16(Wf) && aligned16(s_w) && aligned16(Y) && aligned16(acc),
               SQ_ERR_ALIGN, "%s: pointers must be 16-byte aligned", name);
    return SQ_OK;
}

int weights_to_frag(const uint8_t* Wq, int32_t N, int32_t K, uint8_t* Wf, void* stream, bool glu, const char* name) {
    SQ_TRY(check_K(K));
    SQ_REQUIRE(N >= 0, SQ_ERR_SHAPE, "%s: N=%d < 0", name, N);
    SQ_REQUIRE(!glu || N % 16 == 0, SQ_ERR_SHAPE, "%s: N=%d: gates and ups need N %% 16 == 0", name, N);
    SQ_REQUIRE(sq::frag_weight_bytes(N, K) < (1u << 31), SQ_ERR_SHAPE,
               "%s: the fragment-ordered weights must be under 2 GiB (N=%d K=%d)", name, N, K);
    if (N == 0) return SQ_OK;
    SQ_REQUIRE(Wq && Wf, SQ_ERR_NULL, "%s: Wq and Wf are required", name);
    SQ_REQUIRE(aligned16(Wq) && aligned16(Wf), SQ_ERR_ALIGN, "%s: pointers must be 16-byte aligned", name);
    SQ_REQUIRE(apart(Wq, (size_t)N * K / 2, Wf, sq::frag_weight_bytes(N, K)), SQ_ERR_SHAPE, "%s: Wf overlaps Wq", name);
    hipStream_t st = static_cast<hipStream_t>(stream);
    return hip_status(
        glu ? sq::launch_weights_to_frag_glu(Wq, N, K, Wf, st) : sq::launch_weights_to_frag(Wq, N, K, Wf, st),
        "weights_to_frag");
}

// Scratch of w4a4_gemm_frag_noalloc: a file-scope device array, which every
// GPU the library runs on holds (its own copy) until the process ends.  It
// takes the K-split partial sums, the only scratch the GEMM uses; those are
// written in full before they are read, so nothing has to start at zero.
// Host code never passes the array's name to a kernel: it stands for a host
// symbol there.  The device address comes from hipGetSymbolAddress, once per
// device, on the first call that needs it with that device current.
constexpr size_t kNoallocScratchBytes = SQ_NOALLOC_SCRATCH_BYTES;
__device__ __align__(256) uint8_t scratch[kNoallocScratchBytes];
std::atomic<void*> g_scratch_ptr[sq::kMaxDevices];
std::mutex g_scratch_mu;

int scratch_for(void* stream, void** out) {
    int dev = -1;
    SQ_TRY(hip_status(hipGetDevice(&dev), "hipGetDevice"));
    SQ_REQUIRE(dev >= 0 && dev < sq::kMaxDevices, SQ_ERR_HIP, "device %d out of range", dev);
    if (stream) {   // the address belongs to the current device, so the stream must too
        hipDevice_t sdev = -1;
        SQ_TRY(hip_status(hipStreamGetDevice(static_cast<hipStream_t>(stream), &sdev), "hipStreamGetDevice"));
        SQ_REQUIRE(sdev == dev, SQ_ERR_SHAPE, "the stream belongs to device %d, not the current device %d",
                   (int)sdev, dev);
    }
    void* p = g_scratch_ptr[dev].load(std::memory_order_acquire);
    if (!p) {
        std::lock_guard<std::mutex> lock(g_scratch_mu);
        p = g_scratch_ptr[dev].load(std::memory_order_relaxed);
        if (!p) {
            SQ_TRY(hip_status(hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)), "hipGetSymbolAddress(scratch)"));
            SQ_REQUIRE(p, SQ_ERR_HIP, "hipGetSymbolAddress(scratch) gave a null address");
            g_scratch_ptr[dev].store(p, std::memory_order_release);
        }
    }
    *out = p;
    return SQ_OK;
}

}  // namespace

extern "C" {

int sgat_prepare_weights(const uint16_t* W, const float* P, int32_t N, int32_t K, uint8_t* Wq, float* s_w,
                         void* ws, size_t ws_bytes, void* stream) {
    return prepare_weights(W, P, N, K, Wq, s_w, ws, ws_bytes, stream, 4, "sgat_prepare_weights");
}

int sgat_prepare_weights_w8(const uint16_t* W, const float* P, int32_t N, int32_t K, int8_t* Wq, float* s_w,
                            void* ws, size_t ws_bytes, void* stream) {
    return prepare_weights(W, P, N, K, reinterpret_cast<uint8_t*>(Wq), s_w, ws, ws_bytes, stream, 8,
                           "sgat_prepare_weights_w8");
}

int sgat_transform(const uint16_t* X, const uint8_t* state, const float* P, int32_t M, int32_t K, int32_t d_m,
                   int32_t d_u, float* Xp, void* stream) {
    SQ_TRY(check_K(K));
    SQ_TRY(check_band(K, d_m, d_u));
    SQ_REQUIRE(M >= 0, SQ_ERR_SHAPE, "M=%d < 0", M);
    if (M == 0) return SQ_OK;
    SQ_REQUIRE(X && Xp, SQ_ERR_NULL, "sgat_transform: X and Xp are required");
    SQ_REQUIRE(aligned16(X) && aligned16(Xp) && aligned16(P), SQ_ERR_ALIGN,
               "sgat_transform: X, P and Xp must be 16-byte aligned");
    return hip_status(sq::launch_transform(X, state, P, M, K, d_m, d_u, Xp, static_cast<hipStream_t>(stream)),
                      "transform");
}

int sgat_quantize(const float* Xp, int32_t M, int32_t K, uint8_t* Aq, float* s, void* stream) {
    return quantize(Xp, M, K, Aq, s, stream, 4, "sgat_quantize");
}

int sgat_quantize_w8(const float* Xp, int32_t M, int32_t K, int8_t* Aq, float* s, void* stream) {
    return quantize(Xp, M, K, reinterpret_cast<uint8_t*>(Aq), s, stream, 8, "sgat_quantize_w8");
}

int sgat_quant_act(const uint16_t* X, const uint8_t* state, const float* P, int32_t M, int32_t K, int32_t d_m,
                   int32_t d_u, const uint16_t* tac_M, const uint16_t* tac_d, int32_t g, uint8_t* Aq, float* s_a,
                   void* ws, size_t ws_bytes, void* stream) {
    return quant_act(X, state, P, M, K, d_m, d_u, tac_M, tac_d, g, Aq, s_a, ws, ws_bytes, stream, 4,
                     "sgat_quant_act");
}

int sgat_quant_act_w8(const uint16_t* X, const uint8_t* state, const float* P, int32_t M, int32_t K, int32_t d_m,
                      int32_t d_u, const uint16_t* tac_M, const uint16_t* tac_d, int32_t g, int8_t* Aq,
                      float* s_a, void* ws, size_t ws_bytes, void* stream) {
    return quant_act(X, state, P, M, K, d_m, d_u, tac_M, tac_d, g, reinterpret_cast<uint8_t*>(Aq), s_a, ws,
                     ws_bytes, stream, 8, "sgat_quant_act_w8");
}

int w4a4_gemm(const uint8_t* Aq, const float* s_a, const uint8_t* Wq, const float* s_w, int32_t M, int32_t N,
              int32_t K, uint16_t* Y, int32_t* acc, void* ws, size_t ws_bytes, void* stream) {
    return gemm(Aq, s_a, Wq, s_w, M, N, K, Y, acc, ws, ws_bytes, stream, 4, "w4a4_gemm");
}

int w8a8_gemm(const int8_t* Aq, const float* s_a, const int8_t* Wq, const float* s_w, int32_t M, int32_t N,
              int32_t K, uint16_t* Y, int32_t* acc, void* ws, size_t ws_bytes, void* stream) {
    return gemm(reinterpret_cast<const uint8_t*>(Aq), s_a, reinterpret_cast<const uint8_t*>(Wq), s_w, M, N, K, Y,
                acc, ws, ws_bytes, stream, 8, "w8a8_gemm");
}

int tac_apply(const uint16_t* Z, const uint16_t* tac_M, const uint16_t* tac_d, int32_t M, int32_t C, int32_t g,
              uint16_t* Z_out, void* stream) {
    SQ_TRY(check_K(C));
    SQ_TRY(check_tac(C, g));
    SQ_REQUIRE(M >= 0, SQ_ERR_SHAPE, "M=%d < 0", M);
    SQ_REQUIRE(M <= kMaxTiledRows, SQ_ERR_SHAPE, "tac_apply: M=%d: at most %d rows per call", M, kMaxTiledRows);
    if (M == 0) return SQ_OK;
    SQ_REQUIRE(Z && tac_M && tac_d && Z_out, SQ_ERR_NULL, "tac_apply: Z, tac_M, tac_d and Z_out are required");
    SQ_REQUIRE(aligned16(Z) && aligned16(tac_M) && aligned16(tac_d) && aligned16(Z_out), SQ_ERR_ALIGN,
               "tac_apply: pointers must be 16-byte aligned");
    const uintptr_t a0 = (uintptr_t)Z, a1 = a0 + (size_t)M * C * 2;
    const uintptr_t b0 = (uintptr_t)Z_out, b1 = b0 + (size_t)M * C * 2;
    SQ_REQUIRE(a1 <= b0 || b1 <= a0, SQ_ERR_SHAPE, "tac_apply: Z_out overlaps Z");
    return hip_status(sq::launch_tac(Z, tac_M, tac_d, M, C, g, Z_out, static_cast<hipStream_t>(stream)), "tac");
}

size_t sq_fp6_row_bytes(int32_t K) {
    if (K < 64 || K > 131072 || K % 64) return 0;
    return sq::fp6_row_bytes(K);
}

int sq_codes_to_fp6(const uint8_t* codes, int32_t R, int32_t K, uint8_t* out, void* stream) {
    SQ_TRY(check_K(K));
    SQ_REQUIRE(R >= 0, SQ_ERR_SHAPE, "sq_codes_to_fp6: R=%d < 0", R);
    SQ_REQUIRE((size_t)R * sq::fp6_row_bytes(K) < (1u << 31), SQ_ERR_SHAPE,
               "sq_codes_to_fp6: the FP6 operand must be under 2 GiB (R=%d K=%d)", R, K);
    if (R == 0) return SQ_OK;
    SQ_REQUIRE(codes && out, SQ_ERR_NULL, "sq_codes_to_fp6: codes and out are required");
    SQ_REQUIRE(aligned16(codes) && aligned16(out), SQ_ERR_ALIGN, "sq_codes_to_fp6: pointers must be 16-byte aligned");
    const uintptr_t a0 = (uintptr_t)codes, a1 = a0 + (size_t)R * K / 2;
    const uintptr_t b0 = (uintptr_t)out, b1 = b0 + (size_t)R * sq::fp6_row_bytes(K);
    SQ_REQUIRE(a1 <= b0 || b1 <= a0, SQ_ERR_SHAPE, "sq_codes_to_fp6: out overlaps codes");
    return hip_status(sq::launch_codes_to_fp6(codes, R, K, out, static_cast<hipStream_t>(stream)), "codes_to_fp6");
}

int w4a4_gemm_fp6(const uint8_t* A6, const float* s_a, const uint8_t* W6, const float* s_w, int32_t M, int32_t N,
                  int32_t K, uint16_t* Y, int32_t* acc, void* stream) {
    SQ_TRY(check_K(K));
    SQ_REQUIRE(M >= 0 && N >= 0, SQ_ERR_SHAPE, "M=%d N=%d: need >= 0", M, N);
    SQ_REQUIRE(N % 8 == 0, SQ_ERR_SHAPE, "N=%d: need N %% 8 == 0", N);
    const size_t rb = sq::fp6_row_bytes(K);
    SQ_REQUIRE((size_t)M * rb < (1u << 31) && (size_t)N * rb < (1u << 31), SQ_ERR_SHAPE,
               "w4a4_gemm_fp6: each operand must be under 2 GiB (M=%d N=%d K=%d)", M, N, K);
    if (M == 0 || N == 0) return SQ_OK;
    SQ_REQUIRE(A6 && s_a && W6 && s_w && (Y || acc), SQ_ERR_NULL,
               "w4a4_gemm_fp6: A6, s_a, W6, s_w and one of Y / acc are required");
    SQ_REQUIRE(aligned16(A6) && aligned16(s_a) && aligned16(W6) && aligned16(s_w) && aligned16(Y) &&
                   aligned16(acc),
               SQ_ERR_ALIGN, "w4a4_gemm_fp6: pointers must be 16-byte aligned");
    return hip_status(sq::launch_gemm_fp6(A6, s_a, W6, s_w, M, N, K, Y, acc, static_cast<hipStream_t>(stream)),
                      "gemm_fp6");
}

size_t sq_frag_weight_bytes(int32_t N, int32_t K) {
    if (N < 0 || K < 64 || K > 131072 || K % 64) return 0;
    return sq::frag_weight_bytes(N, K);
}

int sq_weights_to_frag(const uint8_t* Wq, int32_t N, int32_t K, uint8_t* Wf, void* stream) {
    return weights_to_frag(Wq, N, K, Wf, stream, false, "sq_weights_to_frag");
}

int w4a4_gemm_frag(const uint8_t* Aq, const float* s_a, const uint8_t* Wf, const float* s_w, int32_t M, int32_t N,
                   int32_t K, uint16_t* Y, int32_t* acc, void* ws, size_t ws_bytes, void* stream) {
    int done = 0;
    SQ_TRY(check_gemm_frag(Aq, s_a, Wf, s_w, M, N, K, Y, acc, 4, "w4a4_gemm_frag", &done));
    if (done) return SQ_OK;
    SQ_REQUIRE(aligned16(ws), SQ_ERR_ALIGN, "w4a4_gemm_frag: pointers must be 16-byte aligned");
    const size_t need = sq_gemm_workspace_bytes(M, N, K);
    SQ_REQUIRE(ws_bytes >= need && (need == 0 || ws), SQ_ERR_WORKSPACE, "w4a4_gemm_frag: workspace %zu B < %zu B",
               ws_bytes, need);
    return hip_status(
        sq::launch_gemm_frag(Aq, s_a, Wf, s_w, M, N, K, Y, acc, ws, static_cast<hipStream_t>(stream), 4),
        "gemm_frag");
}

size_t sq_frag_weight_w8_bytes(int32_t N, int32_t K) {
    if (K < 64 || K > 65536 || K % 64) return 0;
    return sq_frag_weight_bytes(N, 2 * K);
}

int sq_weights_to_frag_w8(const int8_t* Wq, int32_t N, int32_t K, uint8_t* Wf, void* stream) {
    SQ_REQUIRE(K <= 65536, SQ_ERR_SHAPE, "sq_weights_to_frag_w8: K=%d: 8-bit codes need K <= 65536", K);
    SQ_TRY(check_K(K));
    // a row of K int8 codes is reordered as a row of 2 K int4 codes: the same K bytes
    return sq_weights_to_frag(reinterpret_cast<const uint8_t*>(Wq), N, 2 * K, Wf, stream);
}

int w8a8_gemm_frag(const int8_t* Aq, const float* s_a, const uint8_t* Wf, const float* s_w, int32_t M, int32_t N,
                   int32_t K, uint16_t* Y, int32_t* acc, void* ws, size_t ws_bytes, void* stream) {
    int done = 0;
    const uint8_t* A8 = reinterpret_cast<const uint8_t*>(Aq);
    SQ_TRY(check_gemm_frag(A8, s_a, Wf, s_w, M, N, K, Y, acc, 8, "w8a8_gemm_frag", &done));
    if (done) return SQ_OK;
    SQ_REQUIRE(aligned16(ws), SQ_ERR_ALIGN, "w8a8_gemm_frag: pointers must be 16-byte aligned");
    const size_t need = sq_gemm_w8_workspace_bytes(M, N, K);
    SQ_REQUIRE(ws_bytes >= need && (need == 0 || ws), SQ_ERR_WORKSPACE, "w8a8_gemm_frag: workspace %zu B < %zu B",
               ws_bytes, need);
    return hip_status(
        sq::launch_gemm_frag(A8, s_a, Wf, s_w, M, N, K, Y, acc, ws, static_cast<hipStream_t>(stream), 8),
        "gemm_frag_w8");
}

int w4a4_gemm_frag_noalloc(const uint8_t* Aq, const float* s_a, const uint8_t* Wf, const float* s_w, int32_t M,
                           int32_t N, int32_t K, uint16_t* Y, int32_t* acc, void* stream) {
    int done = 0;
    SQ_TRY(check_gemm_frag(Aq, s_a, Wf, s_w, M, N, K, Y, acc, 4, "w4a4_gemm_frag_noalloc", &done));
    if (done) return SQ_OK;
    const size_t need = sq_gemm_workspace_bytes(M, N, K);
    SQ_REQUIRE(need <= kNoallocScratchBytes, SQ_ERR_WORKSPACE,
               "w4a4_gemm_frag_noalloc: this shape needs %zu B of scratch, above the %zu B the library holds "
               "(M=%d N=%d K=%d)", need, kNoallocScratchBytes, M, N, K);
    void* ws = nullptr;
    if (need > 0) SQ_TRY(scratch_for(stream, &ws));
    return hip_status(
        sq::launch_gemm_frag(Aq, s_a, Wf, s_w, M, N, K, Y, acc, ws, static_cast<hipStream_t>(stream), 4),
        "gemm_frag_noalloc");
}

size_t sq_tac_calibrate_workspace_bytes(int32_t N, int32_t C, int32_t g) {
    if (N <= 0 || C < 64 || C % 64 || g < 1 || g > 128 || (g & (g - 1)) || C % g) return 0;
    return sq::tac_calib_workspace_bytes(N, C, g);
}

int tac_calibrate(const uint16_t* Z_fp, const uint16_t* Z_q, int32_t N, int32_t C, int32_t g, double rho,
                  double eps, double eta, double alpha, uint16_t* tac_M, uint16_t* tac_d, double* M64,
                  double* d64, void* ws, size_t ws_bytes, void* stream) {
    SQ_TRY(check_K(C));
    SQ_TRY(check_tac(C, g));
    SQ_REQUIRE(N >= 1, SQ_ERR_SHAPE, "tac_calibrate: N=%d: need at least one token", N);
    SQ_REQUIRE(rho >= 0.0 && eps >= 0.0 && eta >= 0.0 && eta <= 1.0 && alpha >= 0.0 && alpha <= 1.0 &&
                   rho < 1e300 && eps < 1e300,
               SQ_ERR_SHAPE, "tac_calibrate: need rho, eps >= 0 (finite) and eta, alpha in [0, 1]");
    SQ_REQUIRE(Z_fp && Z_q && tac_M && tac_d && ws, SQ_ERR_NULL,
               "tac_calibrate: Z_fp, Z_q, tac_M, tac_d and ws are required");
    SQ_REQUIRE(aligned16(Z_fp) && aligned16(Z_q) && aligned16(tac_M) && aligned16(tac_d) && aligned16(M64) &&
                   aligned16(d64) && aligned16(ws),
               SQ_ERR_ALIGN, "tac_calibrate: pointers must be 16-byte aligned");
    const size_t need = sq::tac_calib_workspace_bytes(N, C, g);
    SQ_REQUIRE(ws_bytes >= need, SQ_ERR_WORKSPACE, "tac_calibrate: workspace %zu B < %zu B", ws_bytes, need);
    return hip_status(sq::launch_tac_calib(Z_fp, Z_q, N, C, g, rho, eps, eta, alpha, tac_M, tac_d, M64, d64, ws,
                                           static_cast<hipStream_t>(stream)),
                      "tac_calibrate");
}

int sgat_split_basis(const float* P, int32_t K, uint16_t* Ps, void* stream) {
    SQ_TRY(check_K(K));
    SQ_REQUIRE((size_t)K * K * 4 < (1u << 31), SQ_ERR_SHAPE,
               "sgat_split_basis: K=%d: the split basis (4 K^2 bytes) must be under 2 GiB", K);
    SQ_REQUIRE(P && Ps, SQ_ERR_NULL, "sgat_split_basis: P and Ps are required");
    SQ_REQUIRE(aligned16(P) && aligned16(Ps), SQ_ERR_ALIGN, "sgat_split_basis: pointers must be 16-byte aligned");
    return hip_status(sq::launch_split_basis(P, K, Ps, static_cast<hipStream_t>(stream)), "split_basis");
}

int sgat_transform_fast(const uint16_t* X, const uint8_t* state, const uint16_t* Ps, int32_t M, int32_t K,
                        int32_t d_m, int32_t d_u, float* Xp, void* stream) {
    SQ_TRY(check_K(K));
    SQ_TRY(check_band(K, d_m, d_u));
    SQ_REQUIRE(M >= 0, SQ_ERR_SHAPE, "M=%d < 0", M);
    SQ_REQUIRE((size_t)K * K * 4 < (1u << 31), SQ_ERR_SHAPE,
               "sgat_transform_fast: K=%d: the split basis (4 K^2 bytes) must be under 2 GiB", K);
    SQ_REQUIRE((size_t)M * K * 2 < (1u << 31), SQ_ERR_SHAPE,
               "sgat_transform_fast: X must be under 2 GiB (M=%d K=%d)", M, K);
    if (M == 0) return SQ_OK;
    SQ_REQUIRE(X && Ps && Xp, SQ_ERR_NULL, "sgat_transform_fast: X, Ps and Xp are required");
    SQ_REQUIRE(aligned16(X) && aligned16(Ps) && aligned16(Xp), SQ_ERR_ALIGN,
               "sgat_transform_fast: X, Ps and Xp must be 16-byte aligned");
    return hip_status(sq::launch_transform_fast(X, state, Ps, M, K, d_m, d_u, Xp, static_cast<hipStream_t>(stream)),
                      "transform_fast");
}

}  // extern "C"

// ---- rotary positions, the paged 8-bit cache, attention over it, weight-only products ----

namespace {

bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

constexpr int32_t kMaxTokens = 1 << 24, kMaxPositions = 1 << 28;
constexpr int64_t kMaxBlocks = 1 << 24;      // workgroups of 256 threads that one launch's grid holds
constexpr int32_t kMaxSequences = 1 << 14;   // every workgroup looks through them, 64 at a time

// Strides of a [T][H][D] tensor, dense in D; those of an extent of one do not count.
int check_strides(int64_t token, int64_t head, int32_t T, int32_t H, int32_t D, bool out, const char* name,
                  const char* what) {
    const int64_t t = T > 1 ? token : 0, h = H > 1 ? head : 0;
    if (t < 0 || h < 0 || t % 8 || h % 8 || t > ((int64_t)1 << 40) || h > ((int64_t)1 << 40))
        return fail(SQ_ERR_SHAPE, "%s: strides of %s (%lld, %lld): need multiples of 8, not negative", name, what,
                    (long long)token, (long long)head);
    const bool apart = (T == 1 && H == 1) || (T == 1 && h >= D) || (H == 1 && t >= D) ||
                       (h >= D && t >= (H - 1) * h + D) || (t >= D && h >= (T - 1) * t + D);
    if (out && !apart)
        return fail(SQ_ERR_SHAPE, "%s: strides of %s (%lld, %lld): its rows overlap", name, what, (long long)token,
                    (long long)head);
    return SQ_OK;
}

int check_rotation(int32_t rot, int32_t layout, float amplitude, int32_t D, const char* name) {
    SQ_REQUIRE(rot >= 2 && rot <= D && rot % 2 == 0, SQ_ERR_SHAPE, "%s: rot=%d: need an even 2 .. %d", name, rot, D);
    SQ_REQUIRE(layout == SQ_ROPE_HALF || layout == SQ_ROPE_PAIRS, SQ_ERR_SHAPE, "%s: layout=%d", name, layout);
    SQ_REQUIRE(isfinite(amplitude), SQ_ERR_SHAPE, "%s: the amplitude is not finite", name);
    return SQ_OK;
}

int check_cache(const sq_kv_cache* c, const char* name) {
    SQ_REQUIRE(c, SQ_ERR_NULL, "%s: cache is required", name);
    SQ_REQUIRE(c->page == 16 || c->page == 32 || c->page == 64 || c->page == 128, SQ_ERR_SHAPE,
               "%s: page=%d: need 16, 32, 64 or 128 tokens", name, c->page);
    SQ_REQUIRE(c->dim >= 16 && c->dim <= 256 && c->dim % 16 == 0, SQ_ERR_SHAPE,
               "%s: dim=%d: need a multiple of 16 in 16 .. 256", name, c->dim);
    SQ_REQUIRE(c->heads >= 1 && c->heads <= 1024, SQ_ERR_SHAPE, "%s: heads=%d: need 1 .. 1024", name, c->heads);
    SQ_REQUIRE(c->pages >= 1, SQ_ERR_SHAPE, "%s: pages=%d: need at least one", name, c->pages);
    SQ_REQUIRE(c->k && c->v && c->k_scale && c->v_scale, SQ_ERR_NULL, "%s: the cache's four tensors are required",
               name);
    SQ_REQUIRE(aligned16(c->k) && aligned16(c->v) && aligned16(c->k_scale) && aligned16(c->v_scale), SQ_ERR_ALIGN,
               "%s: pointers must be 16-byte aligned", name);
    return SQ_OK;
}

int check_batch(const sq_kv_cache* c, const int32_t* cu, const int32_t* lens, const int32_t* table, int32_t T,
                int32_t B, int32_t max_pages, const char* name) {
    SQ_REQUIRE(T >= 0 && T <= kMaxTokens && B >= 0 && B <= kMaxSequences, SQ_ERR_SHAPE,
               "%s: T=%d B=%d: need 0 <= T <= %d, 0 <= B <= %d", name, T, B, kMaxTokens, kMaxSequences);
    SQ_REQUIRE(max_pages >= 0 && (int64_t)max_pages * c->page <= kMaxPositions, SQ_ERR_SHAPE,
               "%s: max_pages=%d: need at most %d positions", name, max_pages, kMaxPositions);
    if (T == 0 || B == 0) return SQ_OK;
    SQ_REQUIRE(cu && lens && (table || max_pages == 0), SQ_ERR_NULL, "%s: cu, lens and table are required", name);
    SQ_REQUIRE(aligned4(cu) && aligned4(lens) && aligned4(table), SQ_ERR_ALIGN,
               "%s: cu, lens and table must be 4-byte aligned", name);
    return SQ_OK;
}

int check_group(int32_t N, int32_t K, int32_t group, const char* name) {
    SQ_TRY(check_K(K));
    SQ_REQUIRE((group == 32 || group == 64 || (group > 0 && group % 128 == 0)) && K % group == 0, SQ_ERR_SHAPE,
               "%s: group=%d: need 32, 64 or a multiple of 128, dividing K=%d", name, group, K);
    SQ_REQUIRE(N >= 0 && N % 8 == 0, SQ_ERR_SHAPE, "%s: N=%d: need N %% 8 == 0", name, N);
    return SQ_OK;
}

}  // namespace

extern "C" {

int sq_rope_frequencies(int32_t rot, double base, int32_t scaling, double factor, double original, double beta_fast,
                        double beta_slow, double* freq, void* stream) {
    SQ_REQUIRE(rot >= 2 && rot <= 1024 && rot % 2 == 0, SQ_ERR_SHAPE,
               "sq_rope_frequencies: rot=%d: need an even 2 .. 1024", rot);
    SQ_REQUIRE(scaling >= SQ_ROPE_NONE && scaling <= SQ_ROPE_YARN, SQ_ERR_SHAPE, "sq_rope_frequencies: scaling=%d",
               scaling);
    SQ_REQUIRE(base > 1.0 && isfinite(base), SQ_ERR_SHAPE, "sq_rope_frequencies: base=%g: need a finite base > 1",
               base);
    SQ_REQUIRE(scaling == SQ_ROPE_NONE || (factor >= 1.0 && isfinite(factor)), SQ_ERR_SHAPE,
               "sq_rope_frequencies: factor=%g: need a finite factor >= 1", factor);
    SQ_REQUIRE(scaling != SQ_ROPE_YARN || (original > 0 && isfinite(original) && beta_slow >= 0 &&
                                           beta_fast > beta_slow && isfinite(beta_fast)),
               SQ_ERR_SHAPE, "sq_rope_frequencies: original=%g beta_fast=%g beta_slow=%g: need original > 0 and "
               "beta_fast > beta_slow >= 0", original, beta_fast, beta_slow);
    SQ_REQUIRE(freq, SQ_ERR_NULL, "sq_rope_frequencies: freq is required");
    SQ_REQUIRE(aligned16(freq), SQ_ERR_ALIGN, "sq_rope_frequencies: freq must be 16-byte aligned");
    return hip_status(sq::launch_rope_frequencies(rot, base, scaling, factor, original, beta_fast, beta_slow, freq,
                                                  static_cast<hipStream_t>(stream)),
                      "rope_frequencies");
}

double sq_rope_amplitude(int32_t scaling, double factor) {
    return scaling == SQ_ROPE_YARN && factor > 1.0 ? 0.1 * log(factor) + 1.0 : 1.0;
}

int sq_rope(const uint16_t* X, int64_t x_token, int64_t x_head, const int32_t* pos, const double* freq, int32_t T,
            int32_t H, int32_t D, int32_t rot, int32_t layout, int32_t transpose, float amplitude, uint16_t* Y,
            int64_t y_token, int64_t y_head, void* stream) {
    SQ_REQUIRE(D >= 16 && D <= 1024 && D % 16 == 0, SQ_ERR_SHAPE, "sq_rope: D=%d: need a multiple of 16 in 16 .. 1024",
               D);
    SQ_TRY(check_rotation(rot, layout, amplitude, D, "sq_rope"));
    // (a pair a thread where rot % 16 != 0, and the last workgroup's threads are all there)
    SQ_REQUIRE(T >= 0 && H >= 0 && (double)T * H * D < (rot % 16 ? 0x1p33 - 511 : 0x1p33), SQ_ERR_SHAPE,
               "sq_rope: T=%d H=%d: need T H D < 2^33, at most 2^33 - 512 for rot %% 16 != 0", T, H);
    if (T == 0 || H == 0) return SQ_OK;
    SQ_TRY(check_strides(x_token, x_head, T, H, D, false, "sq_rope", "X"));
    SQ_TRY(check_strides(y_token, y_head, T, H, D, true, "sq_rope", "Y"));
    SQ_REQUIRE(X && Y && freq, SQ_ERR_NULL, "sq_rope: X, Y and freq are required");
    SQ_REQUIRE(aligned16(X) && aligned16(Y) && aligned16(freq) && aligned4(pos), SQ_ERR_ALIGN,
               "sq_rope: X, Y and freq must be 16-byte aligned, pos 4-byte");
    SQ_REQUIRE(X != Y || ((T == 1 || x_token == y_token) && (H == 1 || x_head == y_head)), SQ_ERR_SHAPE,
               "sq_rope: in place needs the same strides");
    return hip_status(sq::launch_rope(X, x_token, x_head, pos, freq, T, H, D, rot, layout, transpose != 0, amplitude, Y,
                                      y_token, y_head, static_cast<hipStream_t>(stream)),
                      "rope");
}

int kv_append(const sq_kv_cache* cache, const uint16_t* K, int64_t k_token, int64_t k_head, const uint16_t* V,
              int64_t v_token, int64_t v_head, const int32_t* cu, const int32_t* lens, const int32_t* table, int32_t T,
              int32_t B, int32_t max_pages, const int32_t* pos, const double* freq, int32_t rot, int32_t layout,
              float amplitude, const uint16_t* Q, int64_t q_token, int64_t q_head, int32_t Hq, uint16_t* Qr,
              int64_t r_token, int64_t r_head, void* stream) {
    SQ_TRY(check_cache(cache, "kv_append"));
    const sq_kv_cache& c = *cache;
    SQ_TRY(check_batch(cache, cu, lens, table, T, B, max_pages, "kv_append"));
    if (freq) SQ_TRY(check_rotation(rot, layout, amplitude, c.dim, "kv_append"));
    SQ_REQUIRE(!Q || (freq && Qr), SQ_ERR_NULL, "kv_append: Q needs freq and Qr");
    SQ_REQUIRE(!Q || (Hq >= 1 && Hq <= 1024), SQ_ERR_SHAPE, "kv_append: Hq=%d: need 1 .. 1024", Hq);
    const int64_t per = freq && rot % 16 ? 512 : 4096;       // entries of Q that a workgroup rotates, at least
    SQ_REQUIRE(((int64_t)T / c.page + 2 * (int64_t)B) * c.heads + (Q ? ((int64_t)T * Hq * c.dim + per - 1) / per : 0) <
                   kMaxBlocks,
               SQ_ERR_SHAPE, "kv_append: T=%d B=%d: too many rows for one call", T, B);
    if (T == 0 || B == 0) return SQ_OK;
    SQ_TRY(check_strides(k_token, k_head, T, c.heads, c.dim, false, "kv_append", "K"));
    SQ_TRY(check_strides(v_token, v_head, T, c.heads, c.dim, false, "kv_append", "V"));
    SQ_REQUIRE(K && V, SQ_ERR_NULL, "kv_append: K and V are required");
    SQ_REQUIRE(aligned16(K) && aligned16(V) && aligned16(freq) && aligned16(Q) && aligned16(Qr) && aligned4(pos),
               SQ_ERR_ALIGN, "kv_append: K, V, Q, Qr and freq must be 16-byte aligned, pos 4-byte");
    if (Q) {
        SQ_TRY(check_strides(q_token, q_head, T, Hq, c.dim, false, "kv_append", "Q"));
        SQ_TRY(check_strides(r_token, r_head, T, Hq, c.dim, true, "kv_append", "Qr"));
        SQ_REQUIRE(Q != Qr || ((T == 1 || q_token == r_token) && (Hq == 1 || q_head == r_head)), SQ_ERR_SHAPE,
                   "kv_append: rotating Q in place needs the same strides");
    }
    return hip_status(
        sq::launch_kv_append(c.k, c.v, c.k_scale, c.v_scale, c.pages, c.page, c.heads, c.dim, K, k_token, k_head, V,
                             v_token, v_head, cu, lens, table, pos, T, B, max_pages, freq, freq ? rot : 0, layout,
                             amplitude, Q, q_token, q_head, Hq, Qr, r_token, r_head, static_cast<hipStream_t>(stream)),
        "kv_append");
}

int kv_read(const sq_kv_cache* cache, const int32_t* list, int32_t n, uint16_t* K, uint16_t* V, void* stream) {
    SQ_TRY(check_cache(cache, "kv_read"));
    const sq_kv_cache& c = *cache;
    SQ_REQUIRE(n >= 0 && (int64_t)n * c.heads < kMaxBlocks, SQ_ERR_SHAPE, "kv_read: n=%d: need n heads < 2^24", n);
    if (n == 0) return SQ_OK;
    SQ_REQUIRE(list && K && V, SQ_ERR_NULL, "kv_read: list, K and V are required");
    SQ_REQUIRE(aligned4(list) && aligned16(K) && aligned16(V), SQ_ERR_ALIGN,
               "kv_read: K and V must be 16-byte aligned, list 4-byte");
    return hip_status(sq::launch_kv_read(c.k, c.v, c.k_scale, c.v_scale, c.pages, c.page, c.heads, c.dim, list, n, K, V,
                                         static_cast<hipStream_t>(stream)),
                      "kv_read");
}

size_t sq_attn_kv8_workspace_bytes(int32_t T, int32_t B, int32_t Hq, int32_t heads, int32_t dim, int32_t max_len) {
    if (T <= 0 || B <= 0 || heads <= 0 || Hq <= 0 || Hq % heads || dim <= 0 || max_len < 0) return 0;
    return round_up(sq::attn_workspace_bytes(T, B, Hq, heads, dim, max_len));
}

int attn_kv8(const uint16_t* Q, int64_t q_token, int64_t q_head, const sq_kv_cache* cache, const int32_t* cu,
             const int32_t* lens, const int32_t* table, int32_t T, int32_t B, int32_t max_pages, int32_t Hq,
             int32_t causal, int32_t window, float scale, uint16_t* O, float* lse, void* ws, size_t ws_bytes,
             void* stream) {
    SQ_TRY(check_cache(cache, "attn_kv8"));
    const sq_kv_cache& c = *cache;
    SQ_TRY(check_batch(cache, cu, lens, table, T, B, max_pages, "attn_kv8"));
    SQ_REQUIRE(Hq >= 1 && Hq <= 1024 && Hq % c.heads == 0, SQ_ERR_SHAPE,
               "attn_kv8: Hq=%d: need a multiple of heads=%d, at most 1024", Hq, c.heads);
    // workgroups of up to 512 threads; and sums of weights stay below 2^63, whatever cu holds
    SQ_REQUIRE((int64_t)T * Hq / 16 + (int64_t)B * c.heads < kMaxBlocks / 2 &&
                   (double)T * Hq * (Hq / c.heads) * B * ((double)max_pages * c.page + 64) < 0x1p63,
               SQ_ERR_SHAPE, "attn_kv8: T=%d B=%d max_pages=%d: too much for one call", T, B, max_pages);
    SQ_REQUIRE(window >= 0, SQ_ERR_SHAPE, "attn_kv8: window=%d < 0", window);
    SQ_REQUIRE(isfinite(scale), SQ_ERR_SHAPE, "attn_kv8: the scale is not finite");
    if (T == 0 || B == 0) return SQ_OK;
    SQ_TRY(check_strides(q_token, q_head, T, Hq, c.dim, false, "attn_kv8", "Q"));
    SQ_REQUIRE(Q && O, SQ_ERR_NULL, "attn_kv8: Q and O are required");
    SQ_REQUIRE(aligned16(Q) && aligned16(O) && aligned16(lse) && aligned16(ws), SQ_ERR_ALIGN,
               "attn_kv8: pointers must be 16-byte aligned");
    SQ_REQUIRE(Q != O, SQ_ERR_SHAPE, "attn_kv8: O must not overlap Q");
    const size_t need = sq_attn_kv8_workspace_bytes(T, B, Hq, c.heads, c.dim, max_pages * c.page);
    SQ_REQUIRE(ws_bytes >= need && (need == 0 || ws), SQ_ERR_WORKSPACE, "attn_kv8: workspace %zu B < %zu B", ws_bytes,
               need);
    return hip_status(sq::launch_attn(Q, q_token, q_head, c.k, c.v, c.k_scale, c.v_scale, c.pages, c.page, c.heads,
                                      c.dim, cu, lens, table, T, B, max_pages, Hq, causal != 0, window, scale, O, lse,
                                      ws, static_cast<hipStream_t>(stream)),
                      "attn_kv8");
}

int sq_quantize_weights_group(const uint16_t* W, int32_t N, int32_t K, int32_t group, uint8_t* Wq, uint16_t* s_w,
                              void* stream) {
    SQ_TRY(check_group(N, K, group, "sq_quantize_weights_group"));
    SQ_REQUIRE((int64_t)N * (K / group) < 4 * kMaxBlocks, SQ_ERR_SHAPE,
               "sq_quantize_weights_group: N=%d: too many groups for one call", N);
    if (N == 0) return SQ_OK;
    SQ_REQUIRE(W && Wq && s_w, SQ_ERR_NULL, "sq_quantize_weights_group: W, Wq and s_w are required");
    SQ_REQUIRE(aligned16(W) && aligned16(Wq) && aligned16(s_w), SQ_ERR_ALIGN,
               "sq_quantize_weights_group: pointers must be 16-byte aligned");
    return hip_status(sq::launch_quantize_group(W, N, K, group, Wq, s_w, static_cast<hipStream_t>(stream)),
                      "quantize_group");
}

int w4a16_gemm_frag(const uint16_t* X, const uint8_t* Wf, const uint16_t* s_w, int32_t M, int32_t N, int32_t K,
                    int32_t group, uint16_t* Y, void* stream) {
    SQ_TRY(check_group(N, K, group, "w4a16_gemm_frag"));
    SQ_REQUIRE(M >= 0 && M <= 65535 * 16, SQ_ERR_SHAPE, "w4a16_gemm_frag: M=%d: need 0 .. %d rows", M, 65535 * 16);
    SQ_REQUIRE(sq::frag_weight_bytes(N, K) < ((size_t)1 << 31), SQ_ERR_SHAPE,
               "w4a16_gemm_frag: the fragment-ordered weights must be under 2 GiB (N=%d K=%d)", N, K);
    if (M == 0 || N == 0) return SQ_OK;
    SQ_REQUIRE(X && Wf && s_w && Y, SQ_ERR_NULL, "w4a16_gemm_frag: X, Wf, s_w and Y are required");
    SQ_REQUIRE(aligned16(X) && aligned16(Wf) && aligned16(s_w) && aligned16(Y), SQ_ERR_ALIGN,
               "w4a16_gemm_frag: pointers must be 16-byte aligned");
    SQ_REQUIRE(X != Y, SQ_ERR_SHAPE, "w4a16_gemm_frag: Y must not overlap X");
    return hip_status(sq::launch_w4a16_frag(X, Wf, s_w, M, N, K, group, Y, static_cast<hipStream_t>(stream)),
                      "w4a16_gemm_frag");
}

}  // extern "C"

namespace {

// What the fused epilogue adds to a product's own rules.  in, in_bytes: the rows multiplied.
int check_epilogue(const sq_epilogue& e, int32_t M, int32_t N, const void* in, size_t in_bytes, const void* Wf,
                   size_t wf_bytes, const void* s_w, size_t s_bytes, const void* s_a, void* Y, const char* name) {
    SQ_REQUIRE(e.act >= 0 && e.act < sq::kActs, SQ_ERR_SHAPE, "%s: act=%d: need 0 .. %d", name, e.act, sq::kActs - 1);
    SQ_REQUIRE(!e.glu || N % 16 == 0, SQ_ERR_SHAPE, "%s: N=%d: gates and ups need N %% 16 == 0", name, N);
    // a tile's rows of outputs are addressed with 32-bit buffer offsets
    SQ_REQUIRE((e.glu ? N / 2 : N) <= 1 << 22, SQ_ERR_SHAPE, "%s: N=%d: at most 2^22 outputs a row", name, N);
    if (M == 0 || N == 0) return SQ_OK;
    SQ_REQUIRE(aligned16(e.bias) && aligned16(e.residual), SQ_ERR_ALIGN, "%s: pointers must be 16-byte aligned", name);
    const size_t out = (size_t)M * (e.glu ? N / 2 : N) * (e.f32 ? 4 : 2);
    SQ_REQUIRE(!e.residual || e.residual == Y || apart(Y, out, e.residual, out), SQ_ERR_SHAPE,
               "%s: Y overlaps a residual that it is not", name);
    SQ_REQUIRE(apart(Y, out, in, in_bytes) && apart(Y, out, Wf, wf_bytes) && apart(Y, out, s_w, s_bytes) &&
                   (!s_a || apart(Y, out, s_a, (size_t)M * 4)) && (!e.bias || apart(Y, out, e.bias, (size_t)N * 2)),
               SQ_ERR_SHAPE, "%s: Y overlaps an input", name);
    return SQ_OK;
}

sq::EpilogueArgs epilogue_args(const sq_epilogue& e, void* Y) {
    return sq::EpilogueArgs{e.bias, e.residual, Y, e.act, e.f32 != 0};
}

int linear(const uint8_t* Aq, const float* s_a, const uint8_t* Wf, const float* s_w, int32_t M, int32_t N, int32_t K,
           const sq_epilogue* epilogue, void* Y, void* ws, size_t ws_bytes, void* stream, int bits, const char* name) {
    const sq_epilogue e = epilogue ? *epilogue : sq_epilogue{};
    int done = 0;
    SQ_TRY(check_gemm_frag(Aq, s_a, Wf, s_w, M, N, K, static_cast<uint16_t*>(Y), nullptr, bits, name, &done));
    SQ_TRY(check_epilogue(e, M, N, Aq, (size_t)M * K * bits / 8, Wf, sq::frag_weight_bytes(N, K * bits / 4), s_w,
                          (size_t)N * 4, s_a, Y, name));
    if (done) return SQ_OK;
    SQ_REQUIRE(aligned16(ws), SQ_ERR_ALIGN, "%s: pointers must be 16-byte aligned", name);
    const size_t need = bits == 8 ? sq_gemm_w8_workspace_bytes(M, N, K) : sq_gemm_workspace_bytes(M, N, K);
    SQ_REQUIRE(ws_bytes >= need && (need == 0 || ws), SQ_ERR_WORKSPACE, "%s: workspace %zu B < %zu B", name, ws_bytes,
               need);
    return hip_status(sq::launch_linear(Aq, s_a, Wf, s_w, M, N, K, epilogue_args(e, Y), e.glu != 0, ws,
                                        static_cast<hipStream_t>(stream), bits),
                      name);
}

}  // namespace

extern "C" {

int sq_weights_to_frag_glu(const uint8_t* Wq, int32_t N, int32_t K, uint8_t* Wf, void* stream) {
    return weights_to_frag(Wq, N, K, Wf, stream, true, "sq_weights_to_frag_glu");
}

int sq_weights_to_frag_glu_w8(const int8_t* Wq, int32_t N, int32_t K, uint8_t* Wf, void* stream) {
    SQ_TRY(check_K(K));
    SQ_REQUIRE(K <= 65536, SQ_ERR_SHAPE, "sq_weights_to_frag_glu_w8: K=%d: 8-bit codes need K <= 65536", K);
    return weights_to_frag(reinterpret_cast<const uint8_t*>(Wq), N, 2 * K, Wf, stream, true,
                           "sq_weights_to_frag_glu_w8");
}

int w4a4_linear(const uint8_t* Aq, const float* s_a, const uint8_t* Wf, const float* s_w, int32_t M, int32_t N,
                int32_t K, const sq_epilogue* epilogue, void* Y, void* ws, size_t ws_bytes, void* stream) {
    return linear(Aq, s_a, Wf, s_w, M, N, K, epilogue, Y, ws, ws_bytes, stream, 4, "w4a4_linear");
}

int w8a8_linear(const int8_t* Aq, const float* s_a, const uint8_t* Wf, const float* s_w, int32_t M, int32_t N,
                int32_t K, const sq_epilogue* epilogue, void* Y, void* ws, size_t ws_bytes, void* stream) {
    return linear(reinterpret_cast<const uint8_t*>(Aq), s_a, Wf, s_w, M, N, K, epilogue, Y, ws, ws_bytes, stream, 8,
                  "w8a8_linear");
}

int w4a16_linear(const uint16_t* X, const uint8_t* Wf, const uint16_t* s_w, int32_t M, int32_t N, int32_t K,
                 int32_t group, const sq_epilogue* epilogue, void* Y, void* stream) {
    const sq_epilogue e = epilogue ? *epilogue : sq_epilogue{};
    SQ_TRY(check_group(N, K, group, "w4a16_linear"));
    SQ_REQUIRE(M >= 0 && M <= 65535 * 16, SQ_ERR_SHAPE, "w4a16_linear: M=%d: need 0 .. %d rows", M, 65535 * 16);
    SQ_REQUIRE(sq::frag_weight_bytes(N, K) < ((size_t)1 << 31), SQ_ERR_SHAPE,
               "w4a16_linear: the fragment-ordered weights must be under 2 GiB (N=%d K=%d)", N, K);
    if (M > 0 && N > 0) {
        SQ_REQUIRE(X && Wf && s_w && Y, SQ_ERR_NULL, "w4a16_linear: X, Wf, s_w and Y are required");
        SQ_REQUIRE(aligned16(X) && aligned16(Wf) && aligned16(s_w) && aligned16(Y), SQ_ERR_ALIGN,
                   "w4a16_linear: pointers must be 16-byte aligned");
    }
    SQ_TRY(check_epilogue(e, M, N, X, (size_t)M * K * 2, Wf, sq::frag_weight_bytes(N, K), s_w,
                          (size_t)(K / group) * N * 2, nullptr, Y, "w4a16_linear"));
    if (M == 0 || N == 0) return SQ_OK;
    return hip_status(sq::launch_w4a16_linear(X, Wf, s_w, M, N, K, group, epilogue_args(e, Y), e.glu != 0,
                                              static_cast<hipStream_t>(stream)),
                      "w4a16_linear");
}

int sq_norm(const sq_norm_args* args, int32_t M, int32_t K, void* stream) {
    SQ_REQUIRE(args, SQ_ERR_NULL, "sq_norm: the arguments are required");
    const sq_norm_args& a = *args;
    SQ_REQUIRE(K >= 8 && K <= sq::kNormMaxK && K % 8 == 0, SQ_ERR_SHAPE,
               "sq_norm: K=%d: need 8 <= K <= %d and K %% 8 == 0", K, sq::kNormMaxK);
    SQ_REQUIRE(M >= 0 && M <= kMaxTiledRows, SQ_ERR_SHAPE, "sq_norm: M=%d: need 0 .. %d rows", M, kMaxTiledRows);
    // (1 / sqrt(eps), the r of a row of zeros, is finite in fp32)
    SQ_REQUIRE(isfinite(a.alpha) && isfinite(a.eps) && a.eps >= 1e-30, SQ_ERR_SHAPE,
               "sq_norm: alpha=%g eps=%g: need finite values and eps >= 1e-30", a.alpha, a.eps);
    const bool rows = a.gate || a.scale || a.shift;
    SQ_REQUIRE(!rows || a.seqs >= 1, SQ_ERR_SHAPE, "sq_norm: seqs=%d < 1", a.seqs);
    if (rows && a.seqs > 1) {
        auto bad = [&](const uint16_t* p, int64_t row) {
            return p && row != 0 && (row < K || row % 8 || row > ((int64_t)1 << 32));
        };
        SQ_REQUIRE(!bad(a.gate, a.gate_row) && !bad(a.scale, a.scale_row) && !bad(a.shift, a.shift_row), SQ_ERR_SHAPE,
                   "sq_norm: rows of gate, scale and shift must be multiples of 8 and at least K=%d apart, or 0", K);
    }
    if (a.codes || a.s) {
        SQ_REQUIRE(a.bits == 4 || a.bits == 8, SQ_ERR_SHAPE, "sq_norm: bits=%d: need 4 or 8", a.bits);
        SQ_TRY(check_K(K));
        SQ_TRY(check_band(K, a.d_m, a.d_u));
    }
    if (M == 0) return SQ_OK;
    SQ_REQUIRE(a.h && (a.h_out || a.X || a.codes) && !a.codes == !a.s, SQ_ERR_NULL,
               "sq_norm: h, one of h_out, X and codes, and codes with s are required");
    SQ_REQUIRE(!(a.y_weight || a.gate) || a.y, SQ_ERR_NULL, "sq_norm: y_weight and gate need y");
    const void* all[] = {a.h, a.y, a.y_weight, a.gate, a.scale, a.shift, a.weight, a.h_out, a.X, a.codes, a.s};
    for (const void* p : all) SQ_REQUIRE(aligned16(p), SQ_ERR_ALIGN, "sq_norm: pointers must be 16-byte aligned");
    SQ_REQUIRE(aligned4(a.seq), SQ_ERR_ALIGN, "sq_norm: seq must be 4-byte aligned");
    // outputs against inputs and against each other
    const size_t n = (size_t)M * K, stream_bytes = n * (a.f32 ? 4 : 2);
    auto table = [&](int64_t row) { return ((size_t)(a.seqs - 1) * (size_t)(a.seqs > 1 ? row : 0) + K) * 2; };
    struct Range {
        const void* p;
        size_t bytes;
    };
    const Range in[] = {{a.h, stream_bytes}, {a.y, n * 2}, {a.y_weight, (size_t)K * 2}, {a.weight, (size_t)K * 2},
                        {a.gate, table(a.gate_row)}, {a.scale, table(a.scale_row)}, {a.shift, table(a.shift_row)},
                        {a.seq, (size_t)M * 4}, {a.state, (size_t)M}};
    const Range out[] = {{a.h_out, stream_bytes}, {a.X, n * 2}, {a.codes, a.codes ? n * (size_t)a.bits / 8 : 0},
                         {a.s, (size_t)M * 4}};
    for (const Range& o : out) {
        if (!o.p) continue;
        for (const Range& i : in)
            SQ_REQUIRE(!i.p || (&o == out && &i == in && o.p == i.p) || apart(o.p, o.bytes, i.p, i.bytes), SQ_ERR_SHAPE,
                       "sq_norm: an output overlaps an input");       // (h_out may be h)
        for (const Range& q : out)
            SQ_REQUIRE(&q == &o || !q.p || apart(o.p, o.bytes, q.p, q.bytes), SQ_ERR_SHAPE,
                       "sq_norm: two outputs overlap");
    }
    sq::NormArgs k{};
    k.h = a.h, k.y = a.y, k.post = a.y_weight, k.gate = a.gate, k.scale = a.scale, k.shift = a.shift;
    k.gate_row = a.gate_row, k.scale_row = a.scale_row, k.shift_row = a.shift_row;
    k.seq = rows && a.seqs > 1 ? a.seq : nullptr;
    k.weight = a.weight, k.state = a.state, k.h_out = a.h_out, k.X = a.X;
    k.codes = static_cast<uint8_t*>(a.codes), k.s = a.s;
    k.alpha = a.alpha, k.eps = a.eps, k.seqs = a.seqs, k.f32 = a.f32 != 0, k.center = a.center != 0, k.bits = a.bits;
    k.d_m = a.d_m, k.d_u = a.d_u;
    return hip_status(sq::launch_norm(k, M, K, static_cast<hipStream_t>(stream)), "sq_norm");
}

}  // extern "C"
