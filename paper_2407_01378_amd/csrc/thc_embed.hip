// Embedding lookup and its gradient.
//
// Simple form of the gradient: a workgroup per row of the table looks through all tokens.
#include "thc_fp8.h"
#include "thc_internal.h"

#pragma clang fp contract(off)

namespace thc {
namespace {

constexpr uint32_t kThreads = 256;

__device__ __forceinline__ int64_t token_at(const EmbedArgs& a, uint32_t i) {
    return a.wide_tokens ? static_cast<const int64_t*>(a.tokens)[i] : (int64_t)static_cast<const int32_t*>(a.tokens)[i];
}
__device__ __forceinline__ float load1(const void* p, bool bf16, uint64_t at) {
    return bf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16) : static_cast<const float*>(p)[at];
}
__device__ __forceinline__ void store1(void* p, bool bf16, uint64_t at, float v) {
    if (bf16) static_cast<uint16_t*>(p)[at] = bf16_bits(v);
    else static_cast<float*>(p)[at] = v;
}

__global__ __launch_bounds__(kThreads) void embed_forward_kernel(EmbedArgs a) {
    for (uint32_t i = blockIdx.x; i < a.count; i += gridDim.x) {
        const int64_t v = token_at(a, i);
        const bool in = v >= 0 && v < (int64_t)a.vocab;
        for (uint32_t d = threadIdx.x; d < a.dim; d += kThreads)
            store1(a.out, a.out_bf16, (uint64_t)i * a.ld_out + d,
                   in ? a.scale * load1(a.in, a.in_bf16, (uint64_t)v * a.ld_in + d) : 0.0f);
    }
}

__global__ __launch_bounds__(kThreads) void embed_backward_simple_kernel(EmbedArgs a) {
    __shared__ uint32_t s_found[kThreads];
    __shared__ uint32_t s_count[kThreads / 64u];
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = t >> 6;
    for (uint32_t v = blockIdx.x; v < a.vocab; v += gridDim.x) {
        for (uint32_t d0 = 0; d0 < a.dim; d0 += kThreads) {
            const uint32_t d = d0 + t;
            float sum = 0.0f;
            bool any = false;
            for (uint64_t i0 = 0; i0 < a.count; i0 += kThreads) {
                const uint64_t i = i0 + t;
                const bool match = i < a.count && token_at(a, (uint32_t)i) == (int64_t)v;
                const uint64_t mask = __ballot(match);
                if (lane == 0u) s_count[wave] = __popcll(mask);
                __syncthreads();
                uint32_t before = 0, total = 0;
                for (uint32_t w = 0; w < kThreads / 64u; ++w) {
                    before += w < wave ? s_count[w] : 0u;
                    total += s_count[w];
                }
                if (match) s_found[before + __popcll(mask & ((1ull << lane) - 1ull))] = (uint32_t)i;
                __syncthreads();
                any = any || total != 0u;
                if (d < a.dim)
                    for (uint32_t k = 0; k < total; ++k) sum += load1(a.in, a.in_bf16, (uint64_t)s_found[k] * a.ld_in + d);
                __syncthreads();
            }
            if (d < a.dim && (any || !a.accumulate)) {
                const uint64_t at = (uint64_t)v * a.ld_out + d;
                float r = any ? sum * a.scale : 0.0f;
                if (a.accumulate) r += load1(a.out, a.out_bf16, at);
                store1(a.out, a.out_bf16, at, r);
            }
        }
    }
}

uint32_t grid_for(uint64_t blocks) { return (uint32_t)(blocks < (1u << 20) ? blocks : (1u << 20)); }

}  // namespace

hipError_t launch_embed_forward(const EmbedArgs& a, hipStream_t stream) {
    embed_forward_kernel<<<grid_for(a.count), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

uint64_t embed_backward_workspace_bytes(uint64_t, uint64_t, uint64_t) { return 0; }

hipError_t launch_embed_backward(const EmbedArgs& a, hipStream_t stream) {
    embed_backward_simple_kernel<<<grid_for(a.vocab), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace thc
