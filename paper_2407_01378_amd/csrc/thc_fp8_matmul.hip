// C = A B^T of two 8-bit matrices with a power-of-two scale for each block of 128 along k.
//
// Simple form: a wave per 16 x 16 tile of C, operands straight from memory.
#include "thc_fp8.h"
#include "thc_internal.h"

#pragma clang fp contract(off)

namespace thc {
namespace {

__device__ __forceinline__ i32x8 load_codes(const uint8_t* row, uint32_t k, uint32_t quarter) {
    const uint4 lo = *reinterpret_cast<const uint4*>(row + k + 16u * quarter);
    const uint4 hi = *reinterpret_cast<const uint4*>(row + k + 64u + 16u * quarter);
    return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}

template <int FA, int FB, bool EXACT>
__global__ __launch_bounds__(256) void fp8_matmul_simple_kernel(Fp8MatmulArgs a, uint32_t tiles_n, uint64_t tiles) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, x = lane & 15u, g = lane >> 4;
    const uint32_t blocks = (a.K + 127u) / 128u;
    const uint64_t ld = (uint64_t)blocks * 128u;
    for (uint64_t tile = (uint64_t)blockIdx.x * 4u + wave; tile < tiles; tile += (uint64_t)gridDim.x * 4u) {
        const uint32_t m = (uint32_t)(tile / tiles_n) * 16u + x, n0 = (uint32_t)(tile % tiles_n) * 16u;
        const uint32_t mr = m < a.M ? m : a.M - 1u, nr = n0 + x < a.N ? n0 + x : a.N - 1u;
        const uint8_t* pa = a.a + mr * ld;
        const uint8_t* pb = a.b + nr * ld;
        f32x4 d = {0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t j = 0; j < blocks; ++j) {
            const uint32_t sa = a.a_scales[(uint64_t)(j >> 2) * a.M + mr] >> (8u * (j & 3u));
            const uint32_t sb = a.b_scales[(uint64_t)(j >> 2) * a.N + nr] >> (8u * (j & 3u));
            const i32x8 va = load_codes(pa, j * 128u, g), vb = load_codes(pb, j * 128u, g);
            d = EXACT ? bf16_mfma16<FB, FA>(vb, va, d, sb, sa) : fp8_mfma16<FB, FA>(vb, va, d, sb, sa);
        }
        if (m >= a.M) continue;
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) {
            const uint32_t n = n0 + 4u * g + i;
            if (n >= a.N) continue;
            const uint64_t at = (uint64_t)m * a.ldc + n;
            float v = d[i];
            if (a.out_bf16) {
                uint16_t* c = static_cast<uint16_t*>(a.c) + at;
                if (a.accumulate) v += __uint_as_float((uint32_t)*c << 16);
                *c = (uint16_t)bf16_rne(v);
            } else {
                float* c = static_cast<float*>(a.c) + at;
                if (a.accumulate) v += *c;
                *c = v;
            }
        }
    }
}

}  // namespace

uint64_t fp8_matmul_workspace_bytes(uint64_t, uint64_t, uint64_t) { return 0; }

hipError_t launch_fp8_matmul(const Fp8MatmulArgs& a, hipStream_t stream) {
    const uint32_t tiles_n = (a.N + 15u) / 16u;
    const uint64_t tiles = (uint64_t)tiles_n * ((a.M + 15u) / 16u), blocks = (tiles + 3u) / 4u;
    const uint32_t grid = (uint32_t)(blocks < (1u << 20) ? blocks : (1u << 20));
    auto go = [&](auto FA, auto FB) {
        constexpr int A = decltype(FA)::value, B = decltype(FB)::value;
        if (a.out_bf16) fp8_matmul_simple_kernel<A, B, false><<<grid, 256, 0, stream>>>(a, tiles_n, tiles);
        else fp8_matmul_simple_kernel<A, B, true><<<grid, 256, 0, stream>>>(a, tiles_n, tiles);
    };
    auto with_b = [&](auto FA) {
        a.b_e5m2 ? go(FA, std::integral_constant<int, 1>{}) : go(FA, std::integral_constant<int, 0>{});
    };
    a.a_e5m2 ? with_b(std::integral_constant<int, 1>{}) : with_b(std::integral_constant<int, 0>{});
    return hipGetLastError();
}

}  // namespace thc
