// C = A B^T of two 8-bit matrices straight from memory: few rows (tokens of a few sequences), where the time is that of reading B
// once, and fp32 products of too few tiles for the tiled kernel; and y = Q(x) B^T in one launch for few rows.
//
// A workgroup takes 16 MF rows of A and 16 NF rows of B.  Its waves take the blocks of 128 along k in turn, with operands
// straight from memory in the layout of the 16 x 16 matrix instruction (four lanes hold a row's 128 codes, 16 of each 64
// neighbouring ones a lane), several blocks in flight; their sums are added in their order through LDS.  Where the tiles are too few
// for the device the blocks along k are also divided among workgroups, whose sums a second launch adds.
// With x in fp32 or bf16 a lane quantizes the 32 values it needs itself: every workgroup quantizes its part of x, which for up to 16
// rows costs less than a launch.
//
// What bounds it: the latency of memory, then its bandwidth.  One token, 2048 along k, 8192 rows of weights: 6.1 us for 16.8 MB, 2.7 TB/s (an
// empty launch takes 2 us of it); 16 rows and 16384 rows of weights 11.4 us, 2.9 TB/s.  8 waves to a workgroup:
// the token's product in 4, 8 and 16 waves took 6.9, 6.4 and 8.0 us, from codes 5.4, 5.5 and 7.3 us.
#include "thc_fp8.h"
#include "thc_internal.h"

#pragma clang fp contract(off)

namespace thc {
namespace {

// 32 values of one row of x, two runs of 16 that are 64 apart, as codes; `quantize` returns the block's scale byte.  All 64
// lanes take part: the lanes l, l ^ 16, l ^ 32, l ^ 48 hold one block.
template <bool BF16, bool E5M2>
struct Raw {
    uint4 w[BF16 ? 4 : 8];
    // left: values from the first one to the end of the row (0 or less: none)
    __device__ __forceinline__ void load(const void* x, uint64_t at, int32_t left) {
        constexpr int kHalf = BF16 ? 2 : 4;
        if (left >= 80) {
            const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(x) + at * (BF16 ? 2u : 4u));
#pragma unroll
            for (int i = 0; i < kHalf; ++i) {
                w[i] = load16(p + i);
                w[kHalf + i] = load16(p + 4 * kHalf + i);
            }
            return;
        }
        uint32_t v[BF16 ? 16 : 32];
#pragma unroll
        for (int32_t i = 0; i < 32; ++i) {
            const int32_t k = i < 16 ? i : 48 + i;
            if (BF16) {
                const uint32_t b = k < left ? static_cast<const uint16_t*>(x)[at + k] : 0u;
                if (i & 1) v[i >> 1] |= b << 16;
                else v[i >> 1] = b;
            } else {
                v[i] = k < left ? static_cast<const uint32_t*>(x)[at + k] : 0u;
            }
        }
#pragma unroll
        for (int i = 0; i < 2 * kHalf; ++i) w[i] = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
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

// A lane's 32 codes of a row: every load takes 64 neighbouring bytes of 16 rows.
__device__ __forceinline__ i32x8 load32(const uint8_t* p) {
    const uint4 lo = reinterpret_cast<const uint4*>(p)[0], hi = reinterpret_cast<const uint4*>(p)[4];
    return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
}

// SOURCE: 0 = A in codes, 1 = bf16 values, 2 = fp32 values.
template <int FA, int FB, bool EXACT, int SOURCE, int MF, int NF, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void fp8_direct_kernel(Fp8DirectArgs a, uint32_t tiles_m, uint32_t tiles_n) {
    constexpr uint32_t kCols = 16u * NF, kPitch = kCols + 4u;
    constexpr uint32_t kAhead = NF > 1 ? 2u : 4u;          // blocks of a wave in flight
    constexpr uint32_t kAheadX = SOURCE == 1 ? 2u : 1u;    // blocks of x held unquantized (128 registers: two workgroups to a compute unit)
    __shared__ __attribute__((aligned(16))) float s_sum[WAVES][16][kPitch];
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = t >> 6, r = lane & 15u, g = lane >> 4;
    uint32_t tm, tn;
    place_tile(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn);
    const uint32_t m0 = tm * 16u * MF, n0 = tn * kCols, steps = (a.K + 127u) / 128u;
    const uint32_t begin = blockIdx.y * a.share, end = begin + a.share < steps ? begin + a.share : steps;
    const uint64_t ld = (uint64_t)steps * 128u;
    uint32_t m[MF], n[NF];
#pragma unroll
    for (int f = 0; f < MF; ++f) m[f] = m0 + 16u * f + r < a.M ? m0 + 16u * f + r : a.M - 1u;
#pragma unroll
    for (int f = 0; f < NF; ++f) n[f] = n0 + 16u * f + r < a.N ? n0 + 16u * f + r : a.N - 1u;
    f32x4 acc[MF][NF];
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int i = 0; i < NF; ++i) acc[f][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t j0 = begin + wave; j0 < end; j0 += WAVES * kAhead) {
        i32x8 vb[NF][kAhead], va[SOURCE ? 1 : MF][kAhead];
        uint32_t eb[NF][kAhead], ea[SOURCE ? 1 : MF][kAhead];
        Raw<SOURCE == 1, FA == 1> raw[SOURCE ? MF : 1][kAheadX];
        auto load_x = [&](uint32_t first) {
#pragma unroll
            for (uint32_t p = 0; p < kAheadX; ++p)
#pragma unroll
                for (int f = 0; f < MF; ++f) {
                    const uint32_t j = j0 + (first + p) * WAVES, k = j * 128u + 16u * g;
                    if (j < end) raw[f][p].load(a.x, (uint64_t)m[f] * a.ldx + k, (int32_t)a.K - (int32_t)k);
                }
        };
        if constexpr (SOURCE != 0) load_x(0);   // (before B: what is loaded first arrives first, and there is work to do on it)
#pragma unroll
        for (uint32_t q = 0; q < kAhead; ++q) {
            const uint32_t ahead = j0 + q * WAVES, j = ahead < end ? ahead : j0;
            if (NF == 1 && ahead >= end) continue;   // (tiles: loaded, not used, which keeps the loads in one run)
#pragma unroll
            for (int i = 0; i < NF; ++i) {
                vb[i][q] = load32(a.b + n[i] * ld + j * 128u + 16u * g);
                eb[i][q] = reinterpret_cast<const uint8_t*>(a.b_scales + (uint64_t)(j >> 2) * a.N + n[i])[j & 3u];
            }
            if constexpr (SOURCE == 0) {
#pragma unroll
                for (int f = 0; f < MF; ++f) {
                    va[f][q] = load32(a.a + m[f] * ld + j * 128u + 16u * g);
                    ea[f][q] = reinterpret_cast<const uint8_t*>(a.a_scales + (uint64_t)(j >> 2) * a.M + m[f])[j & 3u];
                }
            }
        }
#pragma unroll
        for (uint32_t q = 0; q < kAhead; ++q) {
            if constexpr (SOURCE != 0) {
                if (q != 0u && q % kAheadX == 0u) load_x(q);
            }
            if (j0 + q * WAVES >= end) continue;
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
#pragma unroll
                for (int i = 0; i < NF; ++i)
                    acc[f][i] = EXACT ? bf16_mfma16<FB, FA>(vb[i][q], v, acc[f][i], eb[i][q], e)
                                      : fp8_mfma16<FB, FA>(vb[i][q], v, acc[f][i], eb[i][q], e);
            }
        }
    }
    const uint64_t pitch = fp8_part_pitch(a.N);
    float* part = a.share < steps ? a.workspace + blockIdx.y * a.M * pitch : nullptr;
#pragma unroll
    for (int f = 0; f < MF; ++f) {   // 16 rows at a time
        if (f) __syncthreads();
#pragma unroll
        for (int i = 0; i < NF; ++i)
            *reinterpret_cast<float4*>(&s_sum[wave][r][16u * i + 4u * g]) = make_float4(acc[f][i][0], acc[f][i][1], acc[f][i][2], acc[f][i][3]);
        __syncthreads();
        for (uint32_t i = t; i < 64u * NF; i += 64u * WAVES) {
            const uint32_t row = i / (4u * NF), c4 = 4u * (i % (4u * NF)), mm = m0 + 16u * f + row, nn = n0 + c4;
            if (mm >= a.M || nn >= a.N) continue;
            f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float4 p = *reinterpret_cast<const float4*>(&s_sum[w][row][c4]);
                v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
            }
            if (part) {   // (rows of the parts have room up to a multiple of 8)
                *reinterpret_cast<float4*>(part + mm * pitch + nn) = make_float4(v[0], v[1], v[2], v[3]);
                continue;
            }
            uint8_t* c = static_cast<uint8_t*>(a.c) + ((uint64_t)mm * a.ldc + nn) * (EXACT ? 4u : 2u);
            store4<!EXACT>(c, v, a.N - nn, a.accumulate);
        }
    }
}

constexpr int kFewWaves = 8;

using I0 = std::integral_constant<int, 0>;
using I1 = std::integral_constant<int, 1>;
using I2 = std::integral_constant<int, 2>;

// Calls go(FA, FB, EXACT) for the formats and result type of a.
template <typename F>
hipError_t with_types(const Fp8MatmulArgs& a, F&& go) {
    auto out = [&](auto FA, auto FB) { return a.out_bf16 ? go(FA, FB, std::false_type{}) : go(FA, FB, std::true_type{}); };
    auto with_b = [&](auto FA) { return a.b_e5m2 ? out(FA, I1{}) : out(FA, I0{}); };
    return a.a_e5m2 ? with_b(I1{}) : with_b(I0{});
}

}  // namespace

hipError_t launch_fp8_direct(const Fp8DirectArgs& args, hipStream_t stream) {
    Fp8DirectArgs a = args;
    const bool few = fp8_rows_are_few(a.M, a.N, a.K);
    const uint32_t cols = few ? 16u : 64u, rows = few && a.M > 16u ? 32u : cols, wanted = few ? fp8_few_rows_parts(a.M, a.N, a.K) : 1u, steps = (a.K + 127u) / 128u;
    const uint32_t tiles_m = (a.M + rows - 1u) / rows, tiles_n = (a.N + cols - 1u) / cols;
    // (few rows: at most 1536 workgroups along B, tiles of 64: fewer than 192)
    if (steps == 0u || (a.source != 0u && !(few && rows == 16u))) return hipErrorInvalidValue;   // (no caller asks for it)
    a.share = (steps + wanted - 1u) / wanted;
    const uint32_t parts = (steps + a.share - 1u) / a.share;
    const dim3 grid(tiles_m * tiles_n, parts);
    const hipError_t rc = with_types(a, [&](auto FA, auto FB, auto EXACT) {
        constexpr int A = decltype(FA)::value, B = decltype(FB)::value;
        constexpr bool E = decltype(EXACT)::value;
        auto go = [&](auto S) {
            constexpr int kSource = decltype(S)::value;
            fp8_direct_kernel<A, B, E, kSource, 1, 1, kFewWaves><<<grid, 64 * kFewWaves, 0, stream>>>(a, tiles_m, tiles_n);
        };
        if (!few) {
            if constexpr (E) fp8_direct_kernel<A, B, true, 0, 4, 4, 4><<<grid, 256, 0, stream>>>(a, tiles_m, tiles_n);
            else return hipErrorInvalidValue;   // (no plan)
        } else if (rows == 32u) fp8_direct_kernel<A, B, E, 0, 2, 1, kFewWaves><<<grid, 64 * kFewWaves, 0, stream>>>(a, tiles_m, tiles_n);
        else if (a.source == 0u) go(I0{});
        else if (a.source == 1u) go(I1{});
        else go(I2{});
        return hipGetLastError();
    });
    return rc != hipSuccess || parts == 1u ? rc : launch_fp8_join(a, parts, stream);
}

}  // namespace thc
