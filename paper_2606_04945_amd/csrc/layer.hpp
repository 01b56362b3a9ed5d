// Launchers of what stands between a layer's quantised products: norms with the residual
// stream, products with a fused epilogue.
#pragma once
#include "epilogue.hpp"

namespace sq {

// Products with bias, activation and residual (gemm_linear.hip, w4a16.hip); workspace as
// gemm_workspace_bytes(M, N, K, bits).
hipError_t launch_linear(const uint8_t* Aq, const float* s_a, const uint8_t* Wf, const float* s_w, int M, int N, int K,
                         const EpilogueArgs& e, bool glu, void* ws, hipStream_t st, int bits);
hipError_t launch_weights_to_frag_glu(const uint8_t* Wq, int N, int K, uint8_t* Wf, hipStream_t st);
hipError_t launch_w4a16_linear(const uint16_t* X, const uint8_t* Wf, const uint16_t* s_w, int M, int N, int K, int group,
                               const EpilogueArgs& e, bool glu, hipStream_t st);

// Norm with the residual stream (norm.hip).  Pointers as in the header's sq_norm_args.
struct NormArgs {
    const void* h;             // [M][K] fp16, or fp32 if f32
    const uint16_t *y, *post;  // [M][K], [K]
    const uint16_t *gate, *scale, *shift;              // [seqs] rows of K
    int64_t gate_row, scale_row, shift_row;            // elements between their rows
    const int32_t* seq;        // [M] or NULL
    const uint16_t* weight;    // [K] or NULL
    const uint8_t* state;      // [M] or NULL
    void* h_out;
    uint16_t* X;
    uint8_t* codes;
    float* s;
    float alpha;
    double eps;
    int seqs, f32, center, bits, d_m, d_u;
};
hipError_t launch_norm(const NormArgs& a, int M, int K, hipStream_t st);

}  // namespace sq
