// Products with a fused epilogue: bias, activation (gated or not) and residual applied to a
// tile's sums while they are in registers (the kernels of gemm_kernels.hpp, the
// epilogue of epilogue.hpp).
#include "gemm_kernels.hpp"
#include "layer.hpp"

namespace sq {

hipError_t launch_linear(const uint8_t* Aq, const float* s_a, const uint8_t* Wf, const float* s_w, int M, int N, int K,
                         const EpilogueArgs& e, bool glu, void* ws, hipStream_t st, int bits) {
    if (glu) return run_frag(Aq, s_a, Wf, s_w, M, N, K, nullptr, nullptr, ws, st, bits, Fused<true>{e});
    return run_frag(Aq, s_a, Wf, s_w, M, N, K, nullptr, nullptr, ws, st, bits, Fused<false>{e});
}

}  // namespace sq
