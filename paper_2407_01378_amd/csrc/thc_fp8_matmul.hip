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

constexpr uint32_t kStep = 128, kHalf = 64;
constexpr uint64_t kMaxGrid = 1ull << 23;   // workgroups of 256 threads: 2^31 threads

typedef __attribute__((address_space(3))) void lds_void;

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
    static_assert(MF == NF, "the four units of a step have one size");
    // A step's codes are four units, the even and the odd halves of the waves' rows of A and of B; ten units fit LDS.  (Arrays of
    // their own: that a fetch to one does not touch what is read from another has to be seen.)
    constexpr uint32_t kUnitRows = 32u * MF, kUnit = kUnitRows * kStep, kSlots = 10;
    __shared__ __attribute__((aligned(1024))) uint8_t s0[kUnit], s1[kUnit], s2[kUnit], s3[kUnit], s4[kUnit], s5[kUnit], s6[kUnit],
        s7[kUnit], s8[kUnit], s9[kUnit];
    uint8_t* const slots[kSlots] = {s0, s1, s2, s3, s4, s5, s6, s7, s8, s9};
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t x = lane & 31u, h = lane >> 5, wm = wave & 1u, wn = wave >> 1;
    uint32_t tm, tn;
    place_tile(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn);
    const uint32_t m0 = tm * BM, n0 = tn * BN, steps = (a.K + kStep - 1u) / kStep, ld = steps * kStep;

    // memory -> LDS: a wave moves 8 rows (whole lines of memory) at a time, lane l the piece of 16 codes that belongs at place
    // l % 8 of row l / 8.  Piece c of a row lies at place c ^ key: two rows fill all banks, and of 16 lanes that read
    // one piece of their rows at a time no two may share a place in rows of the same parity.  key = bits 1, 2, 3 of the
    // row, in the order in which lanes take the rows.
    const uint32_t left_m = a.M - m0, left_n = a.N - n0;
    const uint32_t rows_m = left_m < BM ? left_m : BM, rows_n = left_n < BN ? left_n : BN;
    const auto src_a = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.a + (uint64_t)m0 * ld), 0, rows_m * ld, 0x00020000);
    const auto src_b = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.b + (uint64_t)n0 * ld), 0, rows_n * ld, 0x00020000);
    uint32_t off[4][MF];
    const uint32_t key_a = lane >> 4 | (wave & 1u) << 2, key_b = ((lane >> 4) & 1u) | (wave & 1u) << 1 | (lane >> 5) << 2;
#pragma unroll
    for (uint32_t i = 0; i < MF; ++i) {
        const uint32_t q = 8u * (wave + 4u * i) + (lane >> 3);   // row of the unit
        const uint32_t r = q / (16u * MF) * (32u * MF) + q % (16u * MF);
#pragma unroll
        for (uint32_t u = 0; u < 2u; ++u) {
            const uint32_t ru = r + u * 16u * MF;
            off[u][i] = (ru < rows_m ? ru : rows_m - 1u) * ld + (((lane & 7u) ^ key_a) << 4);
            off[2u + u][i] = (ru < rows_n ? ru : rows_n - 1u) * ld + (((lane & 7u) ^ key_b) << 4);
        }
    }
    uint32_t base = wave * 1024u;
    auto fetch = [&](uint8_t* s, auto unit, uint32_t step) {
        constexpr uint32_t u = decltype(unit)::value;
        asm volatile("" : "+s"(base));   // (all places in LDS, kept across the loop, would not fit the scalar registers)
        const int k = (int)(step < steps ? step * kStep : 0u);   // (behind the last step: not used)
#pragma unroll
        for (uint32_t i = 0; i < MF; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(u < 2u ? src_a : src_b, (lds_void*)(s + base + i * 4096u), 16, (int)off[u][i], k, 0, 0);
    };

    // LDS -> registers.  Rows of B are taken in the order with bits 2 and 3 exchanged, which gives a lane 8
    // neighbouring columns of C.
    const uint32_t xb = (x & 0x13u) | (x & 4u) << 1 | (x & 8u) >> 1;
    const uint32_t at_a = (wm * 16u * MF + x) * kStep + (((2u * h) ^ ((x >> 1) & 7u)) << 4);
    const uint32_t at_b = (wn * 16u * MF + xb) * kStep + (((2u * h) ^ ((x >> 1) & 7u)) << 4);
    auto read = [&](auto first, uint32_t half, i32x8 (&fa)[MF], i32x8 (&fb)[NF]) {   // first: the step's first unit
        constexpr uint32_t u = decltype(first)::value;
        auto piece = [&](const uint8_t* s, uint32_t at) {
            const uint4 lo = *reinterpret_cast<const uint4*>(s + at), hi = *reinterpret_cast<const uint4*>(s + (at ^ 16u));
            return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        };
#pragma unroll
        for (uint32_t f = 0; f < MF; ++f)
            fa[f] = piece(slots[(u + f / (MF / 2u)) % kSlots], (at_a ^ (half << 6)) + f % (MF / 2u) * 32u * kStep);
#pragma unroll
        for (uint32_t f = 0; f < NF; ++f)
            fb[f] = piece(slots[(u + 2u + f / (NF / 2u)) % kSlots], (at_b ^ (half << 6)) + f % (NF / 2u) * 32u * kStep);
    };

    // scale words: four blocks each
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
    auto scales = [&](uint32_t word, uint32_t (&wa)[MF], uint32_t (&wb)[NF]) {
        const uint8_t* pa = reinterpret_cast<const uint8_t*>(a.a_scales + (uint64_t)word * a.M + m0);
        const uint8_t* pb = reinterpret_cast<const uint8_t*>(a.b_scales + (uint64_t)word * a.N + n0);
#pragma unroll
        for (uint32_t f = 0; f < MF; ++f) wa[f] = *reinterpret_cast<const uint32_t*>(pa + row_a[f]);
#pragma unroll
        for (uint32_t f = 0; f < NF; ++f) wb[f] = *reinterpret_cast<const uint32_t*>(pb + row_b[f]);
    };

    const uint32_t words = (steps + 3u) / 4u;
    uint32_t sa[MF], sb[NF], next_a[MF], next_b[NF];
    f32x16 acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    auto multiply = [&](const i32x8 (&fa)[MF], const i32x8 (&fb)[NF]) {
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

    // A step's first half (64 k) is multiplied while its second one is read, and its second half while the next
    // step's first one is.  Behind the first half every wave has read all of the step's units and has waited for what
    // it fetched of the next step, with the 2 units fetched last still on their way: from there on two units of the step
    // after the next one, and in the next first half two of the one behind it, go where the step's were.
    i32x8 fa0[MF], fb0[NF], fa1[MF], fb1[NF];
    auto order = [&]() {   // reads from LDS among the first products, then fetches
#pragma unroll
        for (int i = 0; i < (MF + NF) / 2; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, EXACT ? MF : 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
        }
#pragma unroll
        for (int i = 0; i < 2 * MF; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, EXACT ? MF : 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
        }
        up_to_here();
    };
    auto step = [&](auto phase, uint32_t k) {   // phase: k mod 5
        constexpr uint32_t u = 4u * decltype(phase)::value;
        from_here(fa0, fb0);
        read(std::integral_constant<uint32_t, u>{}, 1, fa1, fb1);
        fetch(slots[(u + 8u) % kSlots], std::integral_constant<uint32_t, 0>{}, k + 2u);
        fetch(slots[(u + 9u) % kSlots], std::integral_constant<uint32_t, 1>{}, k + 2u);
        multiply(fa0, fb0);
        order();
        constexpr uint32_t kLeft = 2u * MF;
        __builtin_amdgcn_s_waitcnt((kLeft & 15u) | (kLeft >> 4) << 14 | 7u << 4);   // vmcnt(kLeft) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        from_here(fa1, fb1);
        read(std::integral_constant<uint32_t, u + 4u>{}, 0, fa0, fb0);
        fetch(slots[(u + 10u) % kSlots], std::integral_constant<uint32_t, 2>{}, k + 2u);
        fetch(slots[(u + 11u) % kSlots], std::integral_constant<uint32_t, 3>{}, k + 2u);
        multiply(fa1, fb1);
        order();
        if ((k & 3u) == 3u) {   // (moved, not renamed: a load that may be on its way would be waited for in every step)
#pragma unroll
            for (int i = 0; i < MF; ++i) asm volatile("v_mov_b32 %0, %1" : "=v"(sa[i]) : "v"(next_a[i]));
#pragma unroll
            for (int j = 0; j < NF; ++j) asm volatile("v_mov_b32 %0, %1" : "=v"(sb[j]) : "v"(next_b[j]));
            const uint32_t w = (k >> 2) + 2u;
            scales(w < words ? w : 0u, next_a, next_b);
        } else {
#pragma unroll
            for (int i = 0; i < MF; ++i) sa[i] >>= 8;
#pragma unroll
            for (int j = 0; j < NF; ++j) sb[j] >>= 8;
        }
    };
    scales(0, sa, sb);
    scales(words > 1u ? 1u : 0u, next_a, next_b);
    fetch(s0, std::integral_constant<uint32_t, 0>{}, 0);
    fetch(s1, std::integral_constant<uint32_t, 1>{}, 0);
    fetch(s2, std::integral_constant<uint32_t, 2>{}, 0);
    fetch(s3, std::integral_constant<uint32_t, 3>{}, 0);
    fetch(s4, std::integral_constant<uint32_t, 0>{}, 1);
    fetch(s5, std::integral_constant<uint32_t, 1>{}, 1);
    fetch(s6, std::integral_constant<uint32_t, 2>{}, 1);
    fetch(s7, std::integral_constant<uint32_t, 3>{}, 1);
    constexpr uint32_t kNext = 4u * MF;
    __builtin_amdgcn_s_waitcnt((kNext & 15u) | (kNext >> 4) << 14 | 0xF70u);   // vmcnt(kNext): step 0
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read(std::integral_constant<uint32_t, 0>{}, 0, fa0, fb0);
    __builtin_amdgcn_sched_barrier(0);
    uint32_t k = 0;
    for (; k + 4u < steps; k += 5u) {
        step(std::integral_constant<uint32_t, 0>{}, k);
        step(std::integral_constant<uint32_t, 1>{}, k + 1u);
        step(std::integral_constant<uint32_t, 2>{}, k + 2u);
        step(std::integral_constant<uint32_t, 3>{}, k + 3u);
        step(std::integral_constant<uint32_t, 4>{}, k + 4u);
    }
    if (k < steps) step(std::integral_constant<uint32_t, 0>{}, k);
    if (k + 1u < steps) step(std::integral_constant<uint32_t, 1>{}, k + 1u);
    if (k + 2u < steps) step(std::integral_constant<uint32_t, 2>{}, k + 2u);
    if (k + 3u < steps) step(std::integral_constant<uint32_t, 3>{}, k + 3u);
    __builtin_amdgcn_s_waitcnt(0x0F70);   // (what was fetched behind the last step)

    constexpr bool BF16 = !EXACT;
    constexpr uint32_t kSize = BF16 ? 2u : 4u, kCols = 32u * NF;
    const uint32_t mw = m0 + wm * 32u * MF, nw = n0 + wn * kCols;
    uint8_t* c = static_cast<uint8_t*>(a.c);
    if (vector && n0 + BN <= a.N) {
        // A whole tile with rows on the 16-byte grid: straight from the registers.
        auto rows = [&](auto add) {
#pragma unroll
            for (uint32_t i = 0; i < MF; ++i) {
                const uint32_t m = mw + i * 32u + x;
                if (m >= a.M) continue;
                uint8_t* at = c + ((uint64_t)m * a.ldc + nw + 8u * h) * kSize;
                Row8<BF16> old[NF][2];
                if (decltype(add)::value) {
#pragma unroll
                    for (uint32_t j = 0; j < 2u * NF; ++j) old[j >> 1][j & 1u].load(at + j * 16u * kSize);
                }
#pragma unroll
                for (uint32_t j = 0; j < 2u * NF; ++j) {
                    float v[8];
#pragma unroll
                    for (uint32_t e = 0; e < 8u; ++e) v[e] = acc[i][j >> 1][8u * (j & 1u) + e];
                    if (decltype(add)::value) old[j >> 1][j & 1u].add_to(v);
                    Row8<BF16>::store(at + j * 16u * kSize, v);
                }
            }
        };
        if (a.accumulate) rows(std::true_type{});
        else rows(std::false_type{});
        return;
    }
    // Otherwise by way of LDS, 32 rows of a wave at a time, so that neighbouring lanes store neighbouring values.
    __builtin_amdgcn_s_barrier();
    if (nw >= a.N) return;
    // (two units to a strip, one behind the other)
    constexpr uint32_t kPitch = kCols + 4u, kHalfRows = 16u;
    static_assert(kHalfRows * kPitch * sizeof(float) <= kUnit, "half a strip fits a unit");
    float* const lower = reinterpret_cast<float*>(wave == 0u ? s0 : wave == 1u ? s1 : wave == 2u ? s2 : s3);
    float* const upper = reinterpret_cast<float*>(wave == 0u ? s4 : wave == 1u ? s5 : wave == 2u ? s6 : s7);
    auto strip = [&](uint32_t r) { return (r < kHalfRows ? lower : upper) + (r % kHalfRows) * kPitch; };
    const uint32_t cols = a.N - nw < kCols ? a.N - nw : kCols;
#pragma unroll
    for (uint32_t i = 0; i < MF; ++i) {
#pragma unroll
        for (uint32_t j = 0; j < NF; ++j)
#pragma unroll
            for (uint32_t q = 0; q < 4u; ++q) {
                float* at = strip(x) + j * 32u + 16u * (q >> 1) + 8u * h + 4u * (q & 1u);
                *reinterpret_cast<float4*>(at) = make_float4(acc[i][j][4u * q], acc[i][j][4u * q + 1u], acc[i][j][4u * q + 2u], acc[i][j][4u * q + 3u]);
            }
        const uint32_t m1 = mw + i * 32u, rows = m1 >= a.M ? 0u : a.M - m1 < 32u ? a.M - m1 : 32u;
        if (BF16 && !a.accumulate) {
            // pairs on the 4-byte grid, then the values left over at a row's ends
#pragma unroll 4
            for (uint32_t r = 0; r < rows; ++r) {
                uint8_t* at = c + ((uint64_t)(m1 + r) * a.ldc + nw) * 2u;
                const uint32_t n = 2u * lane + (uint32_t)(reinterpret_cast<uintptr_t>(at) >> 1 & 1u);
                if (n + 1u < cols) *reinterpret_cast<uint32_t*>(at + 2u * n) = bf16_pair(strip(r)[n], strip(r)[n + 1u]);
            }
            const uint32_t r = lane >> 1;
            if (r < rows) {
                uint8_t* at = c + ((uint64_t)(m1 + r) * a.ldc + nw) * 2u;
                const uint32_t odd = (uint32_t)(reinterpret_cast<uintptr_t>(at) >> 1 & 1u), n = lane & 1u ? cols - 1u : 0u;
                if (lane & 1u ? ((cols - odd) & 1u) != 0u && n >= odd : odd != 0u) store1<true>(at + 2u * n, strip(r)[n], false);
            }
        } else {
#pragma unroll 2
            for (uint32_t r = 0; r < rows; ++r)
#pragma unroll
                for (uint32_t n = lane; n < kCols; n += 64u)
                    if (n < cols) store1<BF16>(c + ((uint64_t)(m1 + r) * a.ldc + nw + n) * kSize, strip(r)[n], a.accumulate);
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
    if (a.M <= kFp8NarrowRows) {
        Fp8NarrowArgs narrow{};
        static_cast<Fp8MatmulArgs&>(narrow) = a;
        return launch_fp8_narrow(narrow, stream);
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
