// Matrices to 8-bit floating point with a power-of-two scale for each block of 128, and back.
//
// One workgroup takes a 128 x 128 tile of x: 16 lanes hold a row's 128 values, 8 each, so that a row's largest
// magnitude is a maximum over 16 lanes (inside the vector ALU) and a column's a maximum over the workgroup (through
// LDS).  Both forms, along the rows and along the columns, come from one read of x; the codes of the
// transposed form pass through LDS so that every store is a whole piece of a row.
// What bounds it: memory, 2 or 4 bytes read and 1 written per value and form.
#include "thc_device.h"
#include "thc_fp8.h"
#include "thc_internal.h"

#pragma clang fp contract(off)

namespace thc {
namespace {

constexpr uint32_t kTile = 128, kThreads = 256;

// Largest over the 16 lanes of a row of lanes, in every one of them.
__device__ __forceinline__ uint32_t row16_umax(uint32_t x) {
    auto step = [&](auto ctrl) {
        const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, false);
        x = y > x ? y : x;
    };
    step(std::integral_constant<int, 0xB1>{});    // lane ^ 1
    step(std::integral_constant<int, 0x4E>{});    // lane ^ 2
    step(std::integral_constant<int, 0x141>{});   // the other quad of the half row
    step(std::integral_constant<int, 0x140>{});   // the other half row
    return x;
}

// 8 neighbouring values, of which `valid` exist.
template <bool BF16>
__device__ __forceinline__ void load8(const void* x, uint64_t at, uint32_t valid, float (&v)[8]) {
    if (valid >= 8u) {
        if (BF16) {
            const uint4 q = load16(static_cast<const uint16_t*>(x) + at);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                v[2 * d] = bf16_low(w[d]);
                v[2 * d + 1] = bf16_high(w[d]);
            }
        } else {
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const uint4 q = load16(static_cast<const float*>(x) + at + 4 * d);
                v[4 * d] = __uint_as_float(q.x);
                v[4 * d + 1] = __uint_as_float(q.y);
                v[4 * d + 2] = __uint_as_float(q.z);
                v[4 * d + 3] = __uint_as_float(q.w);
            }
        }
        return;
    }
#pragma unroll
    for (uint32_t e = 0; e < 8u; ++e) {
        float f = 0.0f;
        if (e < valid)
            f = BF16 ? bf16_low(static_cast<const uint16_t*>(x)[at + e]) : static_cast<const float*>(x)[at + e];
        v[e] = f;
    }
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The byte of block j in its scale word, and zeros behind the last block.
__device__ __forceinline__ void store_scale(uint32_t* scales, uint32_t rows, uint32_t r, uint32_t j, uint32_t blocks, uint32_t e) {
    uint8_t* w = reinterpret_cast<uint8_t*>(scales + (uint64_t)(j >> 2) * rows + r);
    w[j & 3u] = (uint8_t)e;
    if (j + 1u == blocks)
        for (uint32_t k = (j & 3u) + 1u; k < 4u; ++k) w[k] = 0;
}

template <bool BF16, bool E5M2, bool TILE>
__global__ __launch_bounds__(kThreads) void fp8_quantize_kernel(Fp8QuantizeArgs a, uint32_t tiles_c, uint64_t tiles) {
    __shared__ uint32_t s_max[16][kTile];
    __shared__ uint2 s_code[kTile][16];
    __shared__ uint32_t s_row[kTile], s_col[kTile];
    const uint32_t t = threadIdx.x, cg = t & 15u, rg = t >> 4;
    const uint64_t q_ld = (uint64_t)tiles_c * kTile;
    const uint32_t tiles_r = (a.rows + kTile - 1u) / kTile;
    const uint64_t qt_ld = (uint64_t)tiles_r * kTile;
    for (uint64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint32_t tr = (uint32_t)(tile / tiles_c), tc = (uint32_t)(tile % tiles_c);
        const uint32_t r0 = tr * kTile + rg * 8u, c0 = tc * kTile + cg * 8u;
        float v[8][8];
#pragma unroll
        for (uint32_t p = 0; p < 8u; ++p) {
            const uint32_t r = r0 + p, valid = r < a.rows && c0 < a.cols ? a.cols - c0 : 0u;
            load8<BF16>(a.x, (uint64_t)r * a.ld + c0, valid, v[p]);
        }
        uint32_t rm[8], cm[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) rm[i] = cm[i] = 0u;
#pragma unroll
        for (int p = 0; p < 8; ++p)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t m = magnitude(v[p][j]);
                rm[p] = m > rm[p] ? m : rm[p];
                cm[j] = m > cm[j] ? m : cm[j];
            }
#pragma unroll
        for (int p = 0; p < 8; ++p) rm[p] = row16_umax(rm[p]);
        if (TILE) {
            uint32_t m = 0u;
#pragma unroll
            for (int p = 0; p < 8; ++p) m = rm[p] > m ? rm[p] : m;
            if (cg == 0u) s_max[0][rg] = m;
            __syncthreads();
            m = row16_umax(s_max[0][cg]);
#pragma unroll
            for (int p = 0; p < 8; ++p) rm[p] = m;
            if (t < kTile) s_row[t] = s_col[t] = fp8_scale_byte<E5M2>(m);
        } else {
            if (cg < 8u) {
                uint32_t m = 0u;
#pragma unroll
                for (uint32_t p = 0; p < 8u; ++p) m = cg == p ? rm[p] : m;
                s_row[rg * 8u + cg] = fp8_scale_byte<E5M2>(m);
            }
            if (a.q_t) {
#pragma unroll
                for (int j = 0; j < 8; ++j) s_max[rg][cg * 8u + j] = cm[j];
            }
        }
        __syncthreads();
        if (!TILE && a.q_t) {
            if (t < kTile) {
                uint32_t m = 0u;
#pragma unroll
                for (int g = 0; g < 16; ++g) {
                    const uint32_t y = s_max[g][t];
                    m = y > m ? y : m;
                }
                s_col[t] = fp8_scale_byte<E5M2>(m);
            }
            __syncthreads();
        }
        if (a.q) {
#pragma unroll
            for (uint32_t p = 0; p < 8u; ++p) {
                if (r0 + p >= a.rows) continue;
                const uint32_t e = fp8_scale_byte<E5M2>(rm[p]);
                const float scale = fp8_scale(e);
                uint2 w;
                w.x = fp8_codes<E5M2>(v[p][0], v[p][1], v[p][2], v[p][3], scale);
                w.y = fp8_codes<E5M2>(v[p][4], v[p][5], v[p][6], v[p][7], scale);
                if (e == 255u) w.x = w.y = 0x7F7F7F7Fu;
                *reinterpret_cast<uint2*>(a.q + (uint64_t)(r0 + p) * q_ld + c0) = w;
            }
            if (t < kTile && tr * kTile + t < a.rows) store_scale(a.scales, a.rows, tr * kTile + t, tc, tiles_c, s_row[t]);
        }
        if (a.q_t) {
#pragma unroll
            for (uint32_t j = 0; j < 8u; ++j) {
                const uint32_t e = s_col[cg * 8u + j];
                const float scale = fp8_scale(e);
                uint2 w;
                w.x = fp8_codes<E5M2>(v[0][j], v[1][j], v[2][j], v[3][j], scale);
                w.y = fp8_codes<E5M2>(v[4][j], v[5][j], v[6][j], v[7][j], scale);
                if (e == 255u) w.x = w.y = 0x7F7F7F7Fu;
                s_code[cg * 8u + j][rg ^ cg] = w;   // (columns 8 apart fall into the same banks)
            }
            __syncthreads();
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) {
                const uint32_t piece = t + i * kThreads, c = piece >> 3, g = 2u * (piece & 7u);
                if (tc * kTile + c >= a.cols) continue;
                const uint2 lo = s_code[c][g ^ (c >> 3)], hi = s_code[c][(g + 1u) ^ (c >> 3)];
                *reinterpret_cast<uint4*>(a.q_t + (uint64_t)(tc * kTile + c) * qt_ld + (uint64_t)tr * kTile + g * 8u) =
                    make_uint4(lo.x, lo.y, hi.x, hi.y);
            }
            if (t < kTile && tc * kTile + t < a.cols) store_scale(a.scales_t, a.cols, tc * kTile + t, tr, tiles_r, s_col[t]);
        }
        __syncthreads();   // the next tile writes the shared arrays
    }
}

// Along the rows only: 16 lanes take a block, a wave 4 neighbouring blocks of a row, which share their scale word.
template <bool BF16, bool E5M2>
__global__ __launch_bounds__(kThreads) void fp8_quantize_rows_kernel(Fp8QuantizeArgs a, uint32_t groups, uint64_t total) {
    const uint32_t lane = threadIdx.x & 63u, cg = lane & 15u, blocks = (a.cols + 127u) / 128u;
    const uint64_t q_ld = (uint64_t)blocks * 128u, step = (uint64_t)gridDim.x * (kThreads / 64u);
    for (uint64_t i = (uint64_t)blockIdx.x * (kThreads / 64u) + (threadIdx.x >> 6); i < total; i += step) {
        const uint32_t r = (uint32_t)(i / groups), group = (uint32_t)(i % groups), j = 4u * group + (lane >> 4), c = j * 128u + cg * 8u;
        float v[8];
        load8<BF16>(a.x, (uint64_t)r * a.ld + c, c < a.cols ? a.cols - c : 0u, v);
        uint32_t m = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t y = magnitude(v[e]);
            m = y > m ? y : m;
        }
        m = row16_umax(m);
        const uint32_t e = fp8_scale_byte<E5M2>(m);
        const float scale = fp8_scale(e);
        uint2 w;
        w.x = fp8_codes<E5M2>(v[0], v[1], v[2], v[3], scale);
        w.y = fp8_codes<E5M2>(v[4], v[5], v[6], v[7], scale);
        if (e == 255u) w.x = w.y = 0x7F7F7F7Fu;
        if (j < blocks) *reinterpret_cast<uint2*>(a.q + r * q_ld + c) = w;   // (behind the last block: zeros, and scale 0)
        uint32_t word = e << (8u * (lane >> 4));
        word |= (uint32_t)__shfl_xor((int)word, 16);
        word |= (uint32_t)__shfl_xor((int)word, 32);
        if (lane == 0u) a.scales[(uint64_t)group * a.rows + r] = word;
    }
}

// 16 codes a thread.
template <bool E5M2, bool BF16OUT>
__global__ __launch_bounds__(kThreads) void fp8_dequantize_kernel(const uint8_t* q, const uint32_t* scales, uint32_t rows,
                                                                  uint32_t cols, uint32_t pieces, void* out, uint64_t ld) {
    const uint64_t total = (uint64_t)rows * pieces, step = (uint64_t)gridDim.x * kThreads;
    const uint64_t q_ld = (cols + 127u) / 128u * 128u;
    for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += step) {
        const uint32_t r = (uint32_t)(i / pieces), c = (uint32_t)(i % pieces) * 16u, j = c >> 7;
        const uint4 w = *reinterpret_cast<const uint4*>(q + (uint64_t)r * q_ld + c);
        const uint32_t e = (scales[(uint64_t)(j >> 2) * rows + r] >> (8u * (j & 3u))) & 0xFFu;
        const uint32_t word[4] = {w.x, w.y, w.z, w.w};
        float v[16];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const auto lo = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8((int)word[k], false) : __builtin_amdgcn_cvt_pk_f32_fp8((int)word[k], false);
            const auto hi = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8((int)word[k], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)word[k], true);
            v[4 * k] = lo[0]; v[4 * k + 1] = lo[1]; v[4 * k + 2] = hi[0]; v[4 * k + 3] = hi[1];
        }
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = e == 255u ? __uint_as_float(0x7FC00000u) : ldexpf(v[k], (int)e - 127);
        if (c + 16u <= cols) {
            uint8_t* o = static_cast<uint8_t*>(out) + ((uint64_t)r * ld + c) * (BF16OUT ? 2u : 4u);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float half[8] = {v[8 * k], v[8 * k + 1], v[8 * k + 2], v[8 * k + 3], v[8 * k + 4], v[8 * k + 5], v[8 * k + 6], v[8 * k + 7]};
                Row8<BF16OUT>::store(o + k * (BF16OUT ? 16 : 32), half);
            }
            continue;
        }
#pragma unroll
        for (uint32_t k = 0; k < 16u; ++k) {
            if (c + k >= cols) continue;
            const uint64_t at = (uint64_t)r * ld + c + k;
            if (BF16OUT) static_cast<uint16_t*>(out)[at] = bf16_bits(v[k]);
            else static_cast<float*>(out)[at] = v[k];
        }
    }
}

uint32_t grid_for(uint64_t blocks) { return (uint32_t)(blocks < (1u << 20) ? blocks : (1u << 20)); }

}  // namespace

hipError_t launch_fp8_quantize(const Fp8QuantizeArgs& a, bool bf16, bool e5m2, bool tile, hipStream_t stream) {
    const uint32_t tiles_c = (uint32_t)(fp8_row_bytes(a.cols) / kTile);
    const uint64_t tiles = (uint64_t)tiles_c * (fp8_row_bytes(a.rows) / kTile);
    if (!a.q_t && !tile) {
        const uint32_t groups = (a.cols + 511u) / 512u;
        const uint64_t total = (uint64_t)a.rows * groups;
        const uint32_t grid = grid_for((total + kThreads / 64u - 1u) / (kThreads / 64u));
        auto rows = [&](auto B, auto E) {
            fp8_quantize_rows_kernel<decltype(B)::value, decltype(E)::value><<<grid, kThreads, 0, stream>>>(a, groups, total);
        };
        auto with_format = [&](auto B) { e5m2 ? rows(B, std::true_type{}) : rows(B, std::false_type{}); };
        bf16 ? with_format(std::true_type{}) : with_format(std::false_type{});
        return hipGetLastError();
    }
    auto go = [&](auto B, auto E, auto T) {
        fp8_quantize_kernel<decltype(B)::value, decltype(E)::value, decltype(T)::value>
            <<<grid_for(tiles), kThreads, 0, stream>>>(a, tiles_c, tiles);
    };
    auto with_tile = [&](auto B, auto E) { tile ? go(B, E, std::true_type{}) : go(B, E, std::false_type{}); };
    auto with_format = [&](auto B) { e5m2 ? with_tile(B, std::true_type{}) : with_tile(B, std::false_type{}); };
    bf16 ? with_format(std::true_type{}) : with_format(std::false_type{});
    return hipGetLastError();
}

hipError_t launch_fp8_dequantize(const uint8_t* q, const uint32_t* scales, bool e5m2, uint32_t rows, uint32_t cols,
                                 bool out_bf16, void* out, uint64_t ld, hipStream_t stream) {
    const uint32_t pieces = (cols + 15u) / 16u;
    const uint32_t grid = grid_for(((uint64_t)rows * pieces + kThreads - 1u) / kThreads);
    auto go = [&](auto E, auto B) {
        fp8_dequantize_kernel<decltype(E)::value, decltype(B)::value>
            <<<grid, kThreads, 0, stream>>>(q, scales, rows, cols, pieces, out, ld);
    };
    auto with_out = [&](auto E) { out_bf16 ? go(E, std::true_type{}) : go(E, std::false_type{}); };
    e5m2 ? with_out(std::true_type{}) : with_out(std::false_type{});
    return hipGetLastError();
}

}  // namespace thc
