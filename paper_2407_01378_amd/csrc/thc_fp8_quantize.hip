// Matrices to 8-bit floating point with a power-of-two scale for each block of 128, and back.
//
// One workgroup takes a 128 x 128 tile of x: 16 lanes hold a row's 128 values, 8 each, so that a row's largest
// magnitude is a maximum over 16 lanes (inside the vector ALU) and a column's a maximum over the workgroup (through
// LDS).  Both forms, along the rows and along the columns, come from one read of x; the codes of the
// transposed form pass through LDS so that every store is a whole piece of a row.
// What bounds it: memory, 2 or 4 bytes read and 1 written per value and form.  Measured: 8192 x 8192 bf16, both forms, 61 us and
// 8192 x 2048 fp32 by tiles, both forms, 23 us, 4.4 TB/s each (a 4 GiB copy reaches 4.7); 8192 x 8192 bf16 along the rows only 42 us, 4.9 TB/s; back from codes 14.5 us (8192 x 2048 to fp32).  A
// small matrix, of fewer tiles than compute units, takes 6 us whatever its size: one tile's way through memory and LDS.
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

// 8 neighbouring values, of which `valid` exist, as they lie in memory.
template <bool BF16>
struct Eight {
    static constexpr int kWords = BF16 ? 4 : 8;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void* x, uint64_t at, uint32_t valid) {
        if (valid >= 8u) {
#pragma unroll
            for (int d = 0; d < kWords / 4; ++d) {
                const uint4 q = load16(static_cast<const uint8_t*>(x) + at * (BF16 ? 2u : 4u) + 16 * d);
                w[4 * d] = q.x;
                w[4 * d + 1] = q.y;
                w[4 * d + 2] = q.z;
                w[4 * d + 3] = q.w;
            }
            return;
        }
#pragma unroll
        for (uint32_t e = 0; e < 8u; ++e) {
            if (BF16) {
                const uint32_t v = e < valid ? static_cast<const uint16_t*>(x)[at + e] : 0u;
                if (e & 1u) w[e >> 1] |= v << 16;
                else w[e >> 1] = v;
            } else {
                w[BF16 ? 0 : e] = e < valid ? static_cast<const uint32_t*>(x)[at + e] : 0u;
            }
        }
    }
    // the larger magnitude, word by word (bf16: of both halves)
    static __device__ __forceinline__ uint32_t larger(uint32_t top, uint32_t word) {
        if (BF16) return max_u16x2(top, word & 0x7FFF7FFFu);
        const uint32_t m = word & 0x7FFFFFFFu;
        return m > top ? m : top;
    }
    // of both halves, as fp32 bits
    static __device__ __forceinline__ uint32_t whole(uint32_t top) {
        if (!BF16) return top;
        const uint32_t lo = top << 16, hi = top & 0xFFFF0000u;
        return lo > hi ? lo : hi;
    }
    __device__ __forceinline__ uint32_t amax() const {
        uint32_t m = 0u;
#pragma unroll
        for (int d = 0; d < kWords; ++d) m = larger(m, w[d]);
        return whole(m);
    }
    template <bool E5M2>
    __device__ __forceinline__ uint2 codes(uint32_t e) const {
        const float scale = fp8_scale(e);
        uint2 c;
        if constexpr (BF16) {
            c.x = fp8_codes_bf16<E5M2>(w[0], w[1], scale);
            c.y = fp8_codes_bf16<E5M2>(w[2], w[3], scale);
        } else {
            c.x = fp8_codes<E5M2>(value(0), value(1), value(2), value(3), scale);
            c.y = fp8_codes<E5M2>(value(4), value(5), value(6), value(7), scale);
        }
        if (e == 255u) c.x = c.y = 0x7F7F7F7Fu;
        return c;
    }
    __device__ __forceinline__ float value(int e) const { return __uint_as_float(w[e]); }   // (fp32 only)
};

// Codes of column j of 8 rows.
template <bool BF16, bool E5M2>
__device__ __forceinline__ uint2 column_codes(const Eight<BF16> (&v)[8], int j, uint32_t e) {
    const float scale = fp8_scale(e);
    uint2 c;
    if constexpr (BF16) {
        const uint32_t halves = j & 1 ? 0x07060302u : 0x05040100u;   // of the second word and the first
        uint32_t pair[4];
#pragma unroll
        for (int p = 0; p < 4; ++p) pair[p] = __builtin_amdgcn_perm(v[2 * p + 1].w[j >> 1], v[2 * p].w[j >> 1], halves);
        c.x = fp8_codes_bf16<E5M2>(pair[0], pair[1], scale);
        c.y = fp8_codes_bf16<E5M2>(pair[2], pair[3], scale);
    } else {
        c.x = fp8_codes<E5M2>(v[0].value(j), v[1].value(j), v[2].value(j), v[3].value(j), scale);
        c.y = fp8_codes<E5M2>(v[4].value(j), v[5].value(j), v[6].value(j), v[7].value(j), scale);
    }
    if (e == 255u) c.x = c.y = 0x7F7F7F7Fu;
    return c;
}

// The byte of block j in its scale word, and zeros behind the last block.
__device__ __forceinline__ void store_scale(uint32_t* scales, uint32_t rows, uint32_t r, uint32_t j, uint32_t blocks, uint32_t e) {
    uint8_t* w = reinterpret_cast<uint8_t*>(scales + (uint64_t)(j >> 2) * rows + r);
    w[j & 3u] = (uint8_t)e;
    if (j + 1u == blocks)
        for (uint32_t k = (j & 3u) + 1u; k < 4u; ++k) w[k] = 0;
}

template <bool BF16, bool E5M2, bool TILE>
__global__ __launch_bounds__(kThreads) void fp8_quantize_kernel(Fp8QuantizeArgs a, uint32_t tiles_c, uint64_t tiles) {
    constexpr int kWords = Eight<BF16>::kWords;
    __shared__ uint32_t s_max[16][kTile];   // (bf16: two columns to a word)
    __shared__ uint2 s_code[kTile][16];
    __shared__ uint32_t s_row[kTile], s_col[kTile];
    const uint32_t t = threadIdx.x, cg = t & 15u, rg = t >> 4;
    const uint64_t q_ld = (uint64_t)tiles_c * kTile;
    const uint32_t tiles_r = (a.rows + kTile - 1u) / kTile;
    const uint64_t qt_ld = (uint64_t)tiles_r * kTile;
    for (uint64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint32_t tr = (uint32_t)(tile / tiles_c), tc = (uint32_t)(tile % tiles_c);
        const uint32_t r0 = tr * kTile + rg * 8u, c0 = tc * kTile + cg * 8u;
        Eight<BF16> v[8];
#pragma unroll
        for (uint32_t p = 0; p < 8u; ++p) {
            const uint32_t r = r0 + p, valid = r < a.rows && c0 < a.cols ? a.cols - c0 : 0u;
            v[p].load(a.x, (uint64_t)r * a.ld + c0, valid);
        }
        uint32_t rm[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) rm[p] = row16_umax(v[p].amax());
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
                for (int d = 0; d < kWords; ++d) {
                    uint32_t m = 0u;
#pragma unroll
                    for (int p = 0; p < 8; ++p) m = Eight<BF16>::larger(m, v[p].w[d]);
                    s_max[rg][cg * kWords + d] = m;
                }
            }
        }
        __syncthreads();
        if (!TILE && a.q_t) {
            if (t < kTile) {
                uint32_t m = 0u;
#pragma unroll
                for (int g = 0; g < 16; ++g) m = Eight<BF16>::larger(m, s_max[g][BF16 ? t >> 1 : t]);
                if (BF16) m = t & 1u ? m & 0xFFFF0000u : m << 16;
                s_col[t] = fp8_scale_byte<E5M2>(m);
            }
            __syncthreads();
        }
        if (a.q) {
#pragma unroll
            for (uint32_t p = 0; p < 8u; ++p)
                if (r0 + p < a.rows)
                    *reinterpret_cast<uint2*>(a.q + (uint64_t)(r0 + p) * q_ld + c0) = v[p].template codes<E5M2>(fp8_scale_byte<E5M2>(rm[p]));
            if (t < kTile && tr * kTile + t < a.rows) store_scale(a.scales, a.rows, tr * kTile + t, tc, tiles_c, s_row[t]);
        }
        if (a.q_t) {
#pragma unroll
            for (int j = 0; j < 8; ++j)   // (columns 8 apart fall into the same banks)
                s_code[cg * 8u + j][rg ^ cg] = column_codes<BF16, E5M2>(v, j, s_col[cg * 8u + j]);
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

// Along the rows only: 16 lanes take a block, a wave 4 neighbouring blocks of a row, which share their scale word.  (No tile has to
// come together, so a few rows are spread over the device: 24 x 8192 bf16 2.9 us.)
template <bool BF16, bool E5M2>
__global__ __launch_bounds__(kThreads) void fp8_quantize_rows_kernel(Fp8QuantizeArgs a, uint32_t groups, uint64_t total) {
    const uint32_t lane = threadIdx.x & 63u, cg = lane & 15u, blocks = (a.cols + 127u) / 128u;
    const uint64_t q_ld = (uint64_t)blocks * 128u, step = (uint64_t)gridDim.x * (kThreads / 64u);
    for (uint64_t i = (uint64_t)blockIdx.x * (kThreads / 64u) + (threadIdx.x >> 6); i < total; i += step) {
        const uint32_t r = (uint32_t)(i / groups), group = (uint32_t)(i % groups), j = 4u * group + (lane >> 4), c = j * 128u + cg * 8u;
        Eight<BF16> v;
        v.load(a.x, (uint64_t)r * a.ld + c, c < a.cols ? a.cols - c : 0u);
        const uint32_t e = fp8_scale_byte<E5M2>(row16_umax(v.amax()));
        const uint2 w = v.template codes<E5M2>(e);
        if (j < blocks) *reinterpret_cast<uint2*>(a.q + r * q_ld + c) = w;   // (behind the last block: zeros, and scale 0)
        uint32_t word = e << (8u * (lane >> 4));
        word |= (uint32_t)__shfl_xor((int)word, 16);
        word |= (uint32_t)__shfl_xor((int)word, 32);
        if (lane == 0u) a.scales[(uint64_t)group * a.rows + r] = word;
    }
}

// As many codes a thread as make 16 bytes of values.
template <bool E5M2, bool BF16OUT>
__global__ __launch_bounds__(kThreads) void fp8_dequantize_kernel(const uint8_t* q, const uint32_t* scales, uint32_t rows, uint32_t cols,
                                                                  uint32_t pieces, void* out, uint64_t ld) {
    constexpr uint32_t kEach = BF16OUT ? 8u : 4u;
    const uint64_t total = (uint64_t)rows * pieces, step = (uint64_t)gridDim.x * kThreads;
    const uint64_t q_ld = (cols + 127u) / 128u * 128u;
    for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += step) {
        const uint32_t r = (uint32_t)(i / pieces), c = (uint32_t)(i % pieces) * kEach, j = c >> 7;
        const uint32_t* w = reinterpret_cast<const uint32_t*>(q + (uint64_t)r * q_ld + c);
        const uint32_t e = (scales[(uint64_t)(j >> 2) * rows + r] >> (8u * (j & 3u))) & 0xFFu;
        float v[kEach];
#pragma unroll
        for (uint32_t k = 0; k < kEach / 4u; ++k) {
            const auto lo = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8((int)w[k], false) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false);
            const auto hi = E5M2 ? __builtin_amdgcn_cvt_pk_f32_bf8((int)w[k], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
            v[4 * k] = lo[0]; v[4 * k + 1] = lo[1]; v[4 * k + 2] = hi[0]; v[4 * k + 3] = hi[1];
        }
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k) v[k] = e == 255u ? __uint_as_float(0x7FC00000u) : ldexpf(v[k], (int)e - 127);
        uint8_t* o = static_cast<uint8_t*>(out) + ((uint64_t)r * ld + c) * (BF16OUT ? 2u : 4u);
        if (c + kEach <= cols) {
            if constexpr (BF16OUT) store16(o, make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])));
            else store16(o, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
            continue;
        }
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k)
            if (c + k < cols) store1<BF16OUT>(o + k * (BF16OUT ? 2u : 4u), v[k], false);
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
    const uint32_t each = out_bf16 ? 8u : 4u, pieces = (cols + each - 1u) / each;
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
