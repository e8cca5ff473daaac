// C = A B^T of two 8-bit matrices with a power-of-two scale for each block of 128 along k.
//
// Tiled form: a workgroup of 4 waves takes BM x BN of C and walks along k in steps of 128, one block of scales.  A step's
// codes go from memory to LDS without passing registers, two steps deep; each wave multiplies (BM / 2) x (BN / 2) with
// 32 x 32 matrix instructions while the codes of the next half step are read from LDS.
#include "thc_fp8.h"
#include "thc_internal.h"

#pragma clang fp contract(off)

namespace thc {
namespace {

constexpr uint32_t kStep = 128;
constexpr uint64_t kMaxGrid = 1ull << 23;   // workgroups of 256 threads: 2^31 threads

typedef __attribute__((address_space(3))) void lds_void;

// 8 neighbouring values of a row of C.
template <bool BF16>
__device__ __forceinline__ void store8(const Fp8MatmulArgs& a, uint32_t m, uint32_t n, float (&v)[8], bool vector) {
    const uint64_t at = (uint64_t)m * a.ldc + n;
    if (vector && n + 8u <= a.N) {
        if (BF16) {
            uint4* c = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.c) + at);
            if (a.accumulate) {
                const uint4 old = *c;
                const uint32_t o[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[2 * i] += __uint_as_float(o[i] << 16);
                    v[2 * i + 1] += __uint_as_float(o[i] & 0xFFFF0000u);
                }
            }
            uint32_t p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = bf16_rne(v[2 * i]) | bf16_rne(v[2 * i + 1]) << 16;
            *c = make_uint4(p[0], p[1], p[2], p[3]);
        } else {
            float4* c = reinterpret_cast<float4*>(static_cast<float*>(a.c) + at);
            if (a.accumulate) {
                const float4 x = c[0], y = c[1];
                v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
                v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
            }
            c[0] = make_float4(v[0], v[1], v[2], v[3]);
            c[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
        if (n + i >= a.N) continue;
        if (BF16) {
            uint16_t* c = static_cast<uint16_t*>(a.c) + at + i;
            *c = (uint16_t)bf16_rne(a.accumulate ? v[i] + __uint_as_float((uint32_t)*c << 16) : v[i]);
        } else {
            float* c = static_cast<float*>(a.c) + at + i;
            *c = a.accumulate ? v[i] + *c : v[i];
        }
    }
}

// The place of workgroup `id` among `total` tiles: workgroups go round the 8 dies in turn, and each die's workgroups take a
// contiguous run of tiles, in columns of 4 tiles in m, so that what a die reads at a time is few rows of A and B.
__device__ __forceinline__ void place_tile(uint32_t id, uint32_t total, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn) {
    const uint32_t die = id & 7u, of_die = id >> 3, share = total >> 3, rest = total & 7u;
    const uint32_t t = die * share + (die < rest ? die : rest) + of_die;
    const uint32_t group = t / (4u * tiles_n), first = group * 4u, high = tiles_m - first < 4u ? tiles_m - first : 4u;
    const uint32_t in_group = t - group * 4u * tiles_n;
    tm = first + in_group % high;
    tn = in_group / high;
}

template <int FA, int FB, bool EXACT, int MF, int NF>
__global__ __launch_bounds__(256, 1) void fp8_matmul_tiled_kernel(Fp8MatmulArgs a, uint32_t tiles_m, uint32_t tiles_n, bool vector) {
    constexpr uint32_t BM = 64u * MF, BN = 64u * NF;
    __shared__ __attribute__((aligned(1024))) uint8_t s0[(BM + BN) * kStep];
    __shared__ __attribute__((aligned(1024))) uint8_t s1[(BM + BN) * kStep];
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t x = lane & 31u, h = lane >> 5, wm = wave & 1u, wn = wave >> 1;
    uint32_t tm, tn;
    place_tile(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn);
    const uint32_t m0 = tm * BM, n0 = tn * BN, steps = (a.K + kStep - 1u) / kStep, ld = steps * kStep;

    // memory -> LDS: a wave moves 8 rows at a time, lane l the piece that belongs at place l % 8 of row l / 8
    const uint32_t left_m = a.M - m0, left_n = a.N - n0;
    const uint32_t rows_m = left_m < BM ? left_m : BM, rows_n = left_n < BN ? left_n : BN;
    const auto src_a = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.a + (uint64_t)m0 * ld), 0, rows_m * ld, 0x00020000);
    const auto src_b = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.b + (uint64_t)n0 * ld), 0, rows_n * ld, 0x00020000);
    uint32_t off_a[BM / 32u], off_b[BN / 32u];
    const uint32_t key_b = ((lane >> 3) & 3u) | (wave & 1u) << 2;
#pragma unroll
    for (uint32_t i = 0; i < BM / 32u; ++i) {
        const uint32_t r = 8u * (wave + 4u * i) + (lane >> 3);
        off_a[i] = (r < rows_m ? r : rows_m - 1u) * ld + (((lane & 7u) ^ (lane >> 3)) << 4);
    }
#pragma unroll
    for (uint32_t i = 0; i < BN / 32u; ++i) {
        const uint32_t r = 8u * (wave + 4u * i) + (lane >> 3);
        off_b[i] = (r < rows_n ? r : rows_n - 1u) * ld + (((lane & 7u) ^ key_b) << 4);
    }
    uint32_t base = wave * 1024u;
    auto fetch = [&](uint8_t* s, uint32_t k) {
        asm volatile("" : "+s"(base));   // (32 places in LDS, kept across the loop, would not fit the scalar registers)
#pragma unroll
        for (uint32_t i = 0; i < BM / 32u; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(src_a, (lds_void*)(s + base + i * 4096u), 16, (int)off_a[i], (int)k, 0, 0);
#pragma unroll
        for (uint32_t i = 0; i < BN / 32u; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(src_b, (lds_void*)(s + base + BM * kStep + i * 4096u), 16, (int)off_b[i], (int)k, 0, 0);
    };

    // LDS -> registers.  Rows of B are taken in the order with bits 2 and 3 exchanged, which gives a lane 8
    // neighbouring columns of C.
    const uint32_t xb = (x & 0x13u) | (x & 4u) << 1 | (x & 8u) >> 1;
    const uint32_t at_a = (wm * 32u * MF + x) * kStep + (((2u * h) ^ (x & 7u)) << 4);
    const uint32_t at_b = (BM + wn * 32u * NF + xb) * kStep + (((2u * h) ^ (x & 7u)) << 4);
    auto read = [&](const uint8_t* s, uint32_t half, i32x8 (&fa)[MF], i32x8 (&fb)[NF]) {
        auto piece = [&](uint32_t at) {
            const uint4 lo = *reinterpret_cast<const uint4*>(s + at), hi = *reinterpret_cast<const uint4*>(s + (at ^ 16u));
            return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        };
#pragma unroll
        for (uint32_t f = 0; f < MF; ++f) fa[f] = piece((at_a ^ (half << 6)) + f * 32u * kStep);
#pragma unroll
        for (uint32_t f = 0; f < NF; ++f) fb[f] = piece((at_b ^ (half << 6)) + f * 32u * kStep);
    };

    // a block's scale bytes
    uint32_t row_a[MF], row_b[NF];   // in bytes from the tile's first row
#pragma unroll
    for (uint32_t f = 0; f < MF; ++f) {
        const uint32_t r = wm * 32u * MF + f * 32u + x;
        row_a[f] = 4u * (r < rows_m ? r : rows_m - 1u);
    }
#pragma unroll
    for (uint32_t f = 0; f < NF; ++f) {
        const uint32_t r = wn * 32u * NF + f * 32u + xb;
        row_b[f] = 4u * (r < rows_n ? r : rows_n - 1u);
    }
    auto scales = [&](uint32_t j, uint32_t (&wa)[MF], uint32_t (&wb)[NF]) {
        const uint8_t* pa = reinterpret_cast<const uint8_t*>(a.a_scales + (uint64_t)(j >> 2) * a.M + m0) + (j & 3u);
        const uint8_t* pb = reinterpret_cast<const uint8_t*>(a.b_scales + (uint64_t)(j >> 2) * a.N + n0) + (j & 3u);
#pragma unroll
        for (uint32_t f = 0; f < MF; ++f) wa[f] = pa[row_a[f]];
#pragma unroll
        for (uint32_t f = 0; f < NF; ++f) wb[f] = pb[row_b[f]];
    };

    f32x16 acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    auto multiply = [&](const i32x8 (&fa)[MF], const i32x8 (&fb)[NF], const uint32_t (&sa)[MF], const uint32_t (&sb)[NF]) {
        if constexpr (EXACT) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                bf16x8 wa[MF], wb[NF];
#pragma unroll
                for (int i = 0; i < MF; ++i) wa[i] = fp8_widen<FA>(fa[i][2 * p], fa[i][2 * p + 1], fp8_scale(sa[i]));
#pragma unroll
                for (int j = 0; j < NF; ++j) wb[j] = fp8_widen<FB>(fb[j][2 * p], fb[j][2 * p + 1], fp8_scale(sb[j]));
#pragma unroll
                for (int i = 0; i < MF; ++i)
#pragma unroll
                    for (int j = 0; j < NF; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[j], wa[i], acc[i][j], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int j = 0; j < NF; ++j) acc[i][j] = fp8_mfma32<FB, FA>(fb[j], fa[i], acc[i][j], sb[j], sa[i]);
        }
    };
    // Keeps the products of a half between two points of the program: its codes are taken from here on, its sums are
    // formed here (a product is free to move across a barrier otherwise, and three halves of codes would be held).
    auto from_here = [&](i32x8 (&fa)[MF], i32x8 (&fb)[NF]) {
#pragma unroll
        for (int i = 0; i < MF; ++i) asm volatile("" : "+v"(fa[i]));
#pragma unroll
        for (int j = 0; j < NF; ++j) asm volatile("" : "+v"(fb[j]));
    };
    auto up_to_here = [&]() {
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j) asm volatile("" : "+a"(acc[i][j]));
        __builtin_amdgcn_sched_barrier(0);
    };

    // The order of a half: reads from LDS among its first products, fetches among the others.
    auto alternate = [&](bool fetches) {
#pragma unroll
        for (int i = 0; i < MF + NF; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, EXACT ? 4 : 1, 0);              // matrix instruction
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);                          // LDS read
            if (!fetches) __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);            // load
        }
#pragma unroll
        for (int i = 0; i < MF + NF; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, EXACT ? 4 : 1, 0);
            if (fetches) __builtin_amdgcn_sched_group_barrier(0x010, 2, 0);
        }
    };

    i32x8 fa0[MF], fb0[NF], fa1[MF], fb1[NF];
    uint32_t sa0[MF], sb0[NF], sa1[MF], sb1[NF];
    const uint32_t last = steps - 1u;
    fetch(s0, 0);
    scales(0, sa0, sb0);
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    __builtin_amdgcn_s_barrier();
    fetch(s1, last < 1u ? 0u : kStep);
    read(s0, 0, fa0, fb0);

    // One step: its second half is read while the first one is multiplied, the next step's first half (which has
    // arrived when every wave has waited for its part) while the second one is.  Behind the last step the last codes
    // are fetched again, and not used.
    auto step = [&](uint8_t* cur, uint8_t* nxt, uint32_t k, const uint32_t (&sa)[MF], const uint32_t (&sb)[NF],
                    uint32_t (&next_a)[MF], uint32_t (&next_b)[NF]) {
        from_here(fa0, fb0);
        read(cur, 1, fa1, fb1);
        scales(k + 1u < steps ? k + 1u : last, next_a, next_b);
        multiply(fa0, fb0, sa, sb);
        alternate(false);
        up_to_here();
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        from_here(fa1, fb1);
        read(nxt, 0, fa0, fb0);
        fetch(cur, (k + 2u < steps ? k + 2u : last) * kStep);
        multiply(fa1, fb1, sa, sb);
        alternate(true);
        up_to_here();
    };
    uint32_t k = 0;
    for (; k + 1u < steps; k += 2u) {
        step(s0, s1, k, sa0, sb0, sa1, sb1);
        step(s1, s0, k + 1u, sa1, sb1, sa0, sb0);
    }
    if (k < steps) step(s0, s1, k, sa0, sb0, sa1, sb1);

    // C by way of LDS, 32 rows of a wave at a time, so that a row of it is stored by neighbouring lanes.
    __builtin_amdgcn_s_waitcnt(0x0F70);   // (the last fetch)
    __builtin_amdgcn_s_barrier();
    constexpr uint32_t kPitch = 32u * NF + 4u;
    float* strip = reinterpret_cast<float*>(wave < 2u ? s0 : s1) + (wave & 1u) * 32u * kPitch;
#pragma unroll
    for (uint32_t i = 0; i < MF; ++i) {
#pragma unroll
        for (uint32_t j = 0; j < NF; ++j)
#pragma unroll
            for (uint32_t q = 0; q < 4u; ++q) {
                float* at = strip + x * kPitch + j * 32u + 16u * (q >> 1) + 8u * h + 4u * (q & 1u);
                *reinterpret_cast<float4*>(at) = make_float4(acc[i][j][4u * q], acc[i][j][4u * q + 1u], acc[i][j][4u * q + 2u], acc[i][j][4u * q + 3u]);
            }
        constexpr uint32_t kLanes = 4u * NF, kRows = 64u / kLanes;   // lanes of a row, rows at a time
#pragma unroll 1
        for (uint32_t r = lane / kLanes; r < 32u; r += kRows) {
            const uint32_t c = lane % kLanes * 8u, m = m0 + wm * 32u * MF + i * 32u + r, n = n0 + wn * 32u * NF + c;
            const float4 lo = *reinterpret_cast<const float4*>(strip + r * kPitch + c);
            const float4 hi = *reinterpret_cast<const float4*>(strip + r * kPitch + c + 4u);
            float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            if (m < a.M && n < a.N) store8<!EXACT>(a, m, n, v, vector);
        }
    }
}

// The empty sum: zeros.
__global__ __launch_bounds__(256) void zero_matrix_kernel(Fp8MatmulArgs a) {
    const uint64_t total = (uint64_t)a.M * a.N, step = (uint64_t)gridDim.x * 256u;
    for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < total; i += step) {
        const uint64_t at = i / a.N * a.ldc + i % a.N;
        if (a.out_bf16) static_cast<uint16_t*>(a.c)[at] = 0;
        else static_cast<float*>(a.c)[at] = 0.0f;
    }
}

}  // namespace

uint64_t fp8_matmul_workspace_bytes(uint64_t, uint64_t, uint64_t) { return 0; }

hipError_t launch_fp8_matmul(const Fp8MatmulArgs& a, hipStream_t stream) {
    if (a.K == 0u) {   // (there may be no codes and scales to read)
        if (a.accumulate) return hipSuccess;
        const uint64_t blocks = ((uint64_t)a.M * a.N + 255u) / 256u;
        zero_matrix_kernel<<<(uint32_t)(blocks < 4096u ? blocks : 4096u), 256, 0, stream>>>(a);
        return hipGetLastError();
    }
    const uint32_t size = a.out_bf16 ? 2u : 4u;
    const bool vector = (reinterpret_cast<uintptr_t>(a.c) & 15u) == 0 && a.ldc * size % 16u == 0;
    auto go = [&](auto FA, auto FB) {
        constexpr int A = decltype(FA)::value, B = decltype(FB)::value;
        const uint32_t tiles_m = (a.M + 255u) / 256u, tiles_n = (a.N + 255u) / 256u;
        if ((uint64_t)tiles_m * tiles_n > kMaxGrid) return hipErrorInvalidValue;
        if (a.out_bf16) fp8_matmul_tiled_kernel<A, B, false, 4, 4><<<tiles_m * tiles_n, 256, 0, stream>>>(a, tiles_m, tiles_n, vector);
        else fp8_matmul_tiled_kernel<A, B, true, 4, 4><<<tiles_m * tiles_n, 256, 0, stream>>>(a, tiles_m, tiles_n, vector);
        return hipGetLastError();
    };
    auto with_b = [&](auto FA) {
        return a.b_e5m2 ? go(FA, std::integral_constant<int, 1>{}) : go(FA, std::integral_constant<int, 0>{});
    };
    return a.a_e5m2 ? with_b(std::integral_constant<int, 1>{}) : with_b(std::integral_constant<int, 0>{});
}

}  // namespace thc
