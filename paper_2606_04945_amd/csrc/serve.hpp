// Launchers of the operators around the quantised linears: rotary positions, the paged
// 8-bit cache, attention over it, weight-only products.
#pragma once
#include "sq_internal.hpp"

namespace sq {

// Rotary positions and the paged 8-bit cache (kv_cache.hip); strides in elements.
hipError_t launch_rope_frequencies(int rot, double base, int scaling, double factor, double original, double beta_fast,
                                   double beta_slow, double* freq, hipStream_t st);
hipError_t launch_rope(const uint16_t* X, int64_t x_token, int64_t x_head, const int32_t* pos, const double* freq, int T,
                       int H, int D, int rot, int layout, bool transpose, float amp, uint16_t* Y, int64_t y_token,
                       int64_t y_head, hipStream_t st);
hipError_t launch_kv_append(int8_t* k, int8_t* v, float* k_scale, float* v_scale, int pages, int page, int heads, int D,
                            const uint16_t* K, int64_t k_token, int64_t k_head, const uint16_t* V, int64_t v_token,
                            int64_t v_head, const int32_t* cu, const int32_t* lens, const int32_t* table,
                            const int32_t* pos, int T, int B, int max_pages, const double* freq, int rot, int layout,
                            float amp, const uint16_t* Q, int64_t q_token, int64_t q_head, int Hq, uint16_t* Qr,
                            int64_t r_token, int64_t r_head, hipStream_t st);
hipError_t launch_kv_read(const int8_t* k, const int8_t* v, const float* k_scale, const float* v_scale, int pages,
                          int page, int heads, int D, const int32_t* list, int n, uint16_t* Ko, uint16_t* Vo,
                          hipStream_t st);

// Attention over that cache (attn.hip)
size_t attn_workspace_bytes(int T, int B, int Hq, int heads, int D, int max_len);
hipError_t launch_attn(const uint16_t* Q, int64_t q_token, int64_t q_head, const int8_t* k, const int8_t* v,
                       const float* k_scale, const float* v_scale, int pages, int page, int heads, int D,
                       const int32_t* cu, const int32_t* lens, const int32_t* table, int T, int B, int max_pages, int Hq,
                       bool causal, int window, float scale, uint16_t* O, float* lse, void* ws, hipStream_t st);

// Weight-only products with group scales (w4a16.hip)
hipError_t launch_quantize_group(const uint16_t* W, int N, int K, int group, uint8_t* Wq, uint16_t* s_w,
                                 hipStream_t st);
hipError_t launch_w4a16_frag(const uint16_t* X, const uint8_t* Wf, const uint16_t* s_w, int M, int N, int K, int group,
                             uint16_t* Y, hipStream_t st);

}  // namespace sq
