// C = A B^T of two 8-bit matrices where A has few rows (tokens of a few sequences), and y = Q(x) B^T in one launch.
//
// B is read once, and that is what the time is: a workgroup takes 16 rows of B and all rows of A, its waves take the blocks
// of 128 along k in turn, with operands straight from memory in the layout of the 16 x 16 matrix instruction
// (a lane holds 32 neighbouring codes of a row, four lanes a whole line), several blocks in flight.  The waves' sums are
// added in their order through LDS.
// With x in fp32 or bf16 a lane quantizes the 32 values it needs itself: every workgroup quantizes all of x, which for few rows
// costs less than a launch.
#include "thc_fp8.h"
#include "thc_internal.h"

#pragma clang fp contract(off)

namespace thc {
namespace {

// 32 values of one row of x, of which `valid` exist, as codes; returns the block's scale byte.  All 64 lanes take part: the
// lanes l, l ^ 16, l ^ 32, l ^ 48 hold one block.
template <bool BF16, bool E5M2>
struct Raw {
    uint4 w[BF16 ? 4 : 8];
    __device__ __forceinline__ void load(const void* x, uint64_t at, uint32_t valid, bool vector) {
        if (vector && valid >= 32u) {
            const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(x) + at * (BF16 ? 2u : 4u));
#pragma unroll
            for (int i = 0; i < (BF16 ? 4 : 8); ++i) w[i] = p[i];
            return;
        }
        uint32_t v[BF16 ? 16 : 32];
#pragma unroll
        for (uint32_t i = 0; i < 32u; ++i) {
            if (BF16) {
                const uint32_t b = i < valid ? static_cast<const uint16_t*>(x)[at + i] : 0u;
                if (i & 1u) v[i >> 1] |= b << 16;
                else v[i >> 1] = b;
            } else {
                v[i] = i < valid ? static_cast<const uint32_t*>(x)[at + i] : 0u;
            }
        }
#pragma unroll
        for (int i = 0; i < (BF16 ? 4 : 8); ++i) w[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    }
    __device__ __forceinline__ uint32_t quantize(i32x8& codes) const {
        constexpr int kWords = BF16 ? 16 : 32;
        uint32_t v[kWords];
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
            v[4 * i] = w[i].x;
            v[4 * i + 1] = w[i].y;
            v[4 * i + 2] = w[i].z;
            v[4 * i + 3] = w[i].w;
        }
        uint32_t top = 0u;
        if (BF16) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) top = max_u16x2(top, v[i] & 0x7FFF7FFFu);
            top = (top & 0xFFFFu) > (top >> 16) ? top << 16 : top & 0xFFFF0000u;
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                const uint32_t m = v[i] & 0x7FFFFFFFu;
                top = m > top ? m : top;
            }
        }
        uint32_t y = (uint32_t)__shfl_xor((int)top, 16);
        top = y > top ? y : top;
        y = (uint32_t)__shfl_xor((int)top, 32);
        top = y > top ? y : top;
        const uint32_t e = fp8_scale_byte<E5M2>(top);
        const float scale = fp8_scale(e);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t c;
            if constexpr (BF16)
                c = fp8_codes_bf16<E5M2>(v[2 * i], v[2 * i + 1], scale);
            else
                c = fp8_codes<E5M2>(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]),
                                    __uint_as_float(v[4 * i + 3]), scale);
            codes[i] = (int)(e == 255u ? 0x7F7F7F7Fu : c);
        }
        return e;
    }
};

__device__ __forceinline__ i32x8 load32(const uint8_t* p) {
    const uint4 lo = reinterpret_cast<const uint4*>(p)[0], hi = reinterpret_cast<const uint4*>(p)[1];
    return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}

// SOURCE: 0 = A in codes, 1 = bf16 values, 2 = fp32 values.  MF: 16 rows of A each.
template <int FA, int FB, bool EXACT, int SOURCE, int MF, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void fp8_narrow_kernel(Fp8NarrowArgs a, bool vector_x, bool vector_c) {
    constexpr uint32_t kPitch = 20u;
    constexpr uint32_t kAhead = WAVES * MF < 32 ? 4u : 2u;                   // blocks of a wave in flight
    constexpr uint32_t kAheadX = SOURCE == 1 && WAVES * MF < 32 ? 2u : 1u;   // blocks of x held unquantized (its rows come from the cache)
    __shared__ __attribute__((aligned(16))) float s_sum[WAVES][16 * MF][kPitch];
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = t >> 6, r = lane & 15u, g = lane >> 4;
    const uint32_t n0 = blockIdx.x * 16u, steps = (a.K + 127u) / 128u;
    const uint64_t ld = (uint64_t)steps * 128u;
    const uint32_t n = n0 + r < a.N ? n0 + r : a.N - 1u;
    const uint8_t* b = a.b + n * ld + 32u * g;
    const uint8_t* sb = reinterpret_cast<const uint8_t*>(a.b_scales + n);
    uint32_t m[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) m[f] = 16u * f + r < a.M ? 16u * f + r : a.M - 1u;
    f32x4 acc[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) acc[f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t j0 = wave; j0 < steps; j0 += WAVES * kAhead) {
        i32x8 vb[kAhead];
        uint32_t eb[kAhead];
        i32x8 va[SOURCE ? 1 : MF][kAhead];
        uint32_t ea[SOURCE ? 1 : MF][kAhead];
        Raw<SOURCE == 1, FA == 1> raw[SOURCE ? MF : 1][kAheadX];
#pragma unroll
        for (uint32_t q = 0; q < kAhead; ++q) {
            const uint32_t j = j0 + q * WAVES;
            if (j >= steps) continue;
            vb[q] = load32(b + (uint64_t)j * 128u);
            eb[q] = sb[(uint64_t)(j >> 2) * a.N * 4u + (j & 3u)];
#pragma unroll
            for (int f = 0; f < MF; ++f) {
                if constexpr (SOURCE == 0) {
                    va[f][q] = load32(a.a + m[f] * ld + j * 128u + 32u * g);
                    ea[f][q] = reinterpret_cast<const uint8_t*>(a.a_scales + (uint64_t)(j >> 2) * a.M + m[f])[j & 3u];
                }
            }
        }
#pragma unroll
        for (uint32_t q = 0; q < kAhead; ++q) {
            if (SOURCE && q % kAheadX == 0u) {
#pragma unroll
                for (uint32_t p = 0; p < kAheadX; ++p)
#pragma unroll
                    for (int f = 0; f < MF; ++f) {
                        const uint32_t j = j0 + (q + p) * WAVES, k = j * 128u + 32u * g;
                        if (j < steps) raw[f][p].load(a.x, (uint64_t)m[f] * a.ldx + k, k < a.K ? a.K - k : 0u, vector_x);
                    }
            }
            if (j0 + q * WAVES >= steps) continue;
#pragma unroll
            for (int f = 0; f < MF; ++f) {
                i32x8 v;
                uint32_t e;
                if constexpr (SOURCE == 0) {
                    v = va[f][q];
                    e = ea[f][q];
                } else {
                    e = raw[f][q % kAheadX].quantize(v);
                }
                acc[f] = EXACT ? bf16_mfma16<FB, FA>(vb[q], v, acc[f], eb[q], e) : fp8_mfma16<FB, FA>(vb[q], v, acc[f], eb[q], e);
            }
        }
    }
#pragma unroll
    for (int f = 0; f < MF; ++f)
        *reinterpret_cast<float4*>(&s_sum[wave][16 * f + r][4u * g]) = make_float4(acc[f][0], acc[f][1], acc[f][2], acc[f][3]);
    __syncthreads();
    for (uint32_t i = t; i < 64u * MF; i += 64u * WAVES) {
        const uint32_t row = i >> 2, c4 = 4u * (i & 3u);
        if (row >= a.M || n0 + c4 >= a.N) continue;
        f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float4 p = *reinterpret_cast<const float4*>(&s_sum[w][row][c4]);
            v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
        }
        uint8_t* c = static_cast<uint8_t*>(a.c) + ((uint64_t)row * a.ldc + n0 + c4) * (EXACT ? 4u : 2u);
        if (vector_c && !a.accumulate && n0 + c4 + 4u <= a.N) {
            if (EXACT) *reinterpret_cast<float4*>(c) = make_float4(v[0], v[1], v[2], v[3]);
            else *reinterpret_cast<uint2*>(c) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 4u; ++e)
                if (n0 + c4 + e < a.N) store1<!EXACT>(c + e * (EXACT ? 4u : 2u), v[e], a.accumulate);
        }
    }
}

template <int MF>
hipError_t launch(const Fp8NarrowArgs& a, hipStream_t stream) {
    const uint32_t grid = (a.N + 15u) / 16u, steps = (a.K + 127u) / 128u;
    const bool vector_x = (reinterpret_cast<uintptr_t>(a.x) & 15u) == 0 && a.ldx * (a.source == 1 ? 2u : 4u) % 16u == 0;
    const bool vector_c = (reinterpret_cast<uintptr_t>(a.c) & 15u) == 0 && a.ldc * (a.out_bf16 ? 2u : 4u) % 16u == 0;
    auto go = [&](auto FA, auto FB, auto SOURCE, auto EXACT) {
        constexpr int A = decltype(FA)::value, B = decltype(FB)::value, S = decltype(SOURCE)::value;
        constexpr bool E = decltype(EXACT)::value;
        // 16 waves where a column of workgroups would leave compute units idle and there are blocks enough for them.  (Sizes alone
        // decide: codes and values have to be added in one order.)
        if (grid < 512u && steps >= 32u) fp8_narrow_kernel<A, B, E, S, MF, 16><<<grid, 1024, 0, stream>>>(a, vector_x, vector_c);
        else fp8_narrow_kernel<A, B, E, S, MF, 8><<<grid, 512, 0, stream>>>(a, vector_x, vector_c);
        return hipGetLastError();
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    auto out = [&](auto FA, auto FB, auto S) { return a.out_bf16 ? go(FA, FB, S, std::false_type{}) : go(FA, FB, S, std::true_type{}); };
    auto source = [&](auto FA, auto FB) { return a.source == 0 ? out(FA, FB, I0{}) : a.source == 1 ? out(FA, FB, I1{}) : out(FA, FB, I2{}); };
    auto with_b = [&](auto FA) { return a.b_e5m2 ? source(FA, I1{}) : source(FA, I0{}); };
    return a.a_e5m2 ? with_b(I1{}) : with_b(I0{});
}

}  // namespace

hipError_t launch_fp8_narrow(const Fp8NarrowArgs& a, hipStream_t stream) {
    if (a.M > kFp8NarrowRows || a.K == 0u) return hipErrorInvalidValue;
    return a.M <= 16u ? launch<1>(a, stream) : launch<2>(a, stream);
}

}  // namespace thc
