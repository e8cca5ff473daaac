// C = A B^T of two 8-bit matrices with a power-of-two scale for each block of 128 along k.
//
// c[m][n] = sum over blocks j of 2^(ea[m][j] + eb[n][j] - 254) times the sum of the products of the codes in block j.
//
// A workgroup of 4 waves takes 256 x 256 or 128 x 128 of C and walks along k in steps of 128, one block of scales.  A step's
// codes go from memory to LDS without passing registers, up to two and a half steps ahead; each wave multiplies a
// quarter of the tile with 32 x 32 matrix instructions while the codes of the next half step are read from LDS.
//
// What bounds it: the matrix unit and the power it takes.  16384 x 8192 x 8192 to bf16 705 us (3.1 PFLOP/s) on codes of few values
// and 760 to 830 us (2.7 to 2.9) on codes of normal values, which clock the device lower (a library product of plain 8-bit matrices: 2.7 to
// 3.2); the matrix unit is busy 78 % of the cycles.  To fp32, in bf16 products of widened codes, 2048 x 8192 x 8192 184 to 191 us (1.45 PFLOP/s; a
// library product in bf16 1.5 to 1.6), busy 73 %.  Why 256 x 256: each step brings 64 KB to a compute unit for 1000 cycles of products
// (8192 x 2048 x 8192 to bf16 97 us, 120 in tiles of 128 x 128).  A step is not read until it lies in LDS whole; with one step ahead instead of two
// to two and a half the loop waited for memory.  No bank of LDS is asked twice at a time.
#include <initializer_list>

#include "thc_fp8.h"
#include "thc_internal.h"

#pragma clang fp contract(off)

namespace thc {
namespace {

constexpr uint32_t kStep = 128;
constexpr uint32_t kUnits = 256;   // compute units (a multiple of the dies, so that a workgroup's tiles are its die's)

typedef __attribute__((address_space(3))) void lds_void;

template <int FA, int FB, bool EXACT, int MF, int NF>
__global__ __launch_bounds__(256, 1) void fp8_matmul_tiled_kernel(Fp8MatmulArgs a, uint32_t tiles_m, uint32_t tiles_n) {
    constexpr uint32_t BM = 64u * MF, BN = 64u * NF;
    static_assert(MF == NF, "the four units of a step have one size");
    constexpr bool kWalks = MF == 4;   // one workgroup on a compute unit, which goes from tile to tile (two, a tile each, otherwise)
    // A step's codes are four units, the even and the odd halves of the waves' rows of A and of B; ten units fit LDS.  (Arrays of
    // their own: that a fetch to one does not touch what is read from another has to be seen.)
    constexpr uint32_t kUnitRows = 32u * MF, kUnit = kUnitRows * kStep, kSlots = 10;
    __shared__ __attribute__((aligned(1024))) uint8_t s0[kUnit], s1[kUnit], s2[kUnit], s3[kUnit], s4[kUnit], s5[kUnit], s6[kUnit],
        s7[kUnit], s8[kUnit], s9[kUnit];
    uint8_t* const slots[kSlots] = {s0, s1, s2, s3, s4, s5, s6, s7, s8, s9};
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t x = lane & 31u, h = lane >> 5, wm = wave & 1u, wn = wave >> 1;
    // this workgroup's part of the blocks along k
    const uint32_t blocks = (a.K + kStep - 1u) / kStep, ld = blocks * kStep, first = blockIdx.y * a.share;
    const uint32_t steps = blocks - first < a.share ? blocks - first : a.share;

    // memory -> LDS: a wave moves 8 rows (whole lines of memory) at a time, lane l the piece of 16 codes that belongs at place
    // l % 8 of row l / 8.  Piece c of a row lies at place c ^ key: two rows fill all banks, and of 16 lanes that read
    // one piece of their rows at a time no two may share a place in rows of the same parity.  key = bits 1, 2, 3 of the
    // row, in the order in which lanes take the rows.
    uint32_t m0, n0, rows_m, rows_n, off[4][MF];
    uint32_t row_a[MF], row_b[NF];   // of the scales, in bytes from the tile's first row
    auto go_to = [&](uint32_t tile) __attribute__((always_inline)) {
        uint32_t tm, tn, l = lane;
        asm volatile("" : "+v"(l));   // (worked out for each tile, not kept)
        const uint32_t x = l & 31u, xb = (x & 0x13u) | (x & 4u) << 1 | (x & 8u) >> 1;   // (rows of B: bits 2 and 3 exchanged)
        const uint32_t key_a = l >> 4 | (wave & 1u) << 2, key_b = ((l >> 4) & 1u) | (wave & 1u) << 1 | (l >> 5) << 2;
        place_tile(tile, tiles_m * tiles_n, tiles_m, tiles_n, tm, tn);
        m0 = tm * BM, n0 = a.first_n + tn * BN;
        rows_m = a.M - m0 < BM ? a.M - m0 : BM, rows_n = a.N - n0 < BN ? a.N - n0 : BN;
#pragma unroll
        for (uint32_t i = 0; i < MF; ++i) {
            const uint32_t q = 8u * (wave + 4u * i) + (l >> 3);   // row of the unit
            const uint32_t r = q / (16u * MF) * (32u * MF) + q % (16u * MF);
#pragma unroll
            for (uint32_t u = 0; u < 2u; ++u) {
                const uint32_t ru = r + u * 16u * MF;
                off[u][i] = (ru < rows_m ? ru : rows_m - 1u) * ld + (((l & 7u) ^ key_a) << 4);
                off[2u + u][i] = (ru < rows_n ? ru : rows_n - 1u) * ld + (((l & 7u) ^ key_b) << 4);
            }
        }
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
    };
    uint32_t base = wave * 1024u;
    auto fetch_one = [&](uint8_t* s, uint32_t unit, uint32_t i, uint32_t step) __attribute__((always_inline)) {
        const int k = (int)((first + (step < steps ? step : 0u)) * kStep);   // (behind the last step: not used)
        const auto src = unit < 2u ? __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.a + (uint64_t)m0 * ld), 0, rows_m * ld, 0x00020000)
                                   : __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.b + (uint64_t)n0 * ld), 0, rows_n * ld, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void*)(s + base + i * 4096u), 16, (int)off[unit][i], k, 0, 0);
    };
    auto fetch = [&](uint8_t* s, uint32_t unit, uint32_t step) __attribute__((always_inline)) {
        asm volatile("" : "+s"(base));   // (all places in LDS, kept across the loop, would not fit the scalar registers)
#pragma unroll
        for (uint32_t i = 0; i < MF; ++i) fetch_one(s, unit, i, step);
    };

    // LDS -> registers.  Rows of B are taken in the order with bits 2 and 3 exchanged, which gives a lane 8
    // neighbouring columns of C.
    const uint32_t xb = (x & 0x13u) | (x & 4u) << 1 | (x & 8u) >> 1;
    const uint32_t at_a = (wm * 16u * MF + x) * kStep + (((2u * h) ^ ((x >> 1) & 7u)) << 4);
    const uint32_t at_b = (wn * 16u * MF + xb) * kStep + (((2u * h) ^ ((x >> 1) & 7u)) << 4);
    auto read_one = [&](uint32_t u, uint32_t half, uint32_t f, i32x8 (&fa)[MF], i32x8 (&fb)[NF]) __attribute__((always_inline)) {   // u: the step's first unit
        auto piece = [&](const uint8_t* s, uint32_t at) {
            const uint4 lo = *reinterpret_cast<const uint4*>(s + at), hi = *reinterpret_cast<const uint4*>(s + (at ^ 16u));
            return i32x8{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w};
        };
        if (f < MF) fa[f] = piece(slots[(u + f / (MF / 2u)) % kSlots], (at_a ^ (half << 6)) + f % (MF / 2u) * 32u * kStep);
        else fb[f - MF] = piece(slots[(u + 2u + (f - MF) / (NF / 2u)) % kSlots], (at_b ^ (half << 6)) + (f - MF) % (NF / 2u) * 32u * kStep);
    };
    auto read = [&](uint32_t u, uint32_t half, i32x8 (&fa)[MF], i32x8 (&fb)[NF]) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t f = 0; f < MF + NF; ++f) read_one(u, half, f, fa, fb);
    };

    // scale words: four blocks each
    auto scales = [&](uint32_t word, uint32_t (&wa)[MF], uint32_t (&wb)[NF]) {
        const uint8_t* pa = reinterpret_cast<const uint8_t*>(a.a_scales + (uint64_t)word * a.M + m0);
        const uint8_t* pb = reinterpret_cast<const uint8_t*>(a.b_scales + (uint64_t)word * a.N + n0);
#pragma unroll
        for (uint32_t f = 0; f < MF; ++f) wa[f] = *reinterpret_cast<const uint32_t*>(pa + row_a[f]);
#pragma unroll
        for (uint32_t f = 0; f < NF; ++f) wb[f] = *reinterpret_cast<const uint32_t*>(pb + row_b[f]);
    };

    const uint32_t word0 = first >> 2, words = (blocks + 3u) / 4u;
    uint32_t sa[MF], sb[NF], next_a[MF], next_b[NF];
    f32x16 acc[MF][NF];
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
    // What is multiplied and what is widened to bfloat16 for the next 16 k meanwhile.
    bf16x8 wide[2][EXACT ? MF + NF : 1];
    auto widen = [&](uint32_t to, uint32_t f, uint32_t p, const i32x8 (&fa)[MF], const i32x8 (&fb)[NF], const uint32_t (&ea)[MF],
                     const uint32_t (&eb)[NF]) __attribute__((always_inline)) {
        if (f < MF) wide[to][f] = fp8_widen<FA>(fa[f][2 * p], fa[f][2 * p + 1], fp8_scale(ea[f]));
        else wide[to][f] = fp8_widen<FB>(fb[f - MF][2 * p], fb[f - MF][2 * p + 1], fp8_scale(eb[f - MF]));
    };
    // A half: the products of (fa, fb) with the scales sa, sb, while (ga, gb), the next half with the scales ea, eb, is read
    // from the step whose first unit is u, and two units from `unit` on, of two steps ahead, are fetched into the slots from `to` on.
    auto half_step = [&](i32x8 (&fa)[MF], i32x8 (&fb)[NF], uint32_t u, uint32_t half, i32x8 (&ga)[MF], i32x8 (&gb)[NF],
                         const uint32_t (&ea)[MF], const uint32_t (&eb)[NF], uint32_t to, uint32_t unit, uint32_t step) __attribute__((always_inline)) {
        from_here(fa, fb);
        if constexpr (EXACT) {
            constexpr uint32_t kOperands = MF + NF, kProducts = MF * NF / kOperands;   // products of 16 k beside each widened operand
            asm volatile("" : "+s"(base));
#pragma unroll
            for (uint32_t p = 0; p < 4; ++p)
#pragma unroll
                for (uint32_t f = 0; f < kOperands; ++f) {
                    if (p < 3) widen((p + 1u) & 1u, f, p + 1u, fa, fb, sa, sb);
                    else widen(0, f, 0, ga, gb, ea, eb);
#pragma unroll
                    for (uint32_t q = f * kProducts; q < (f + 1u) * kProducts; ++q)
                        acc[q / NF][q % NF] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wide[p & 1u][MF + q % NF], wide[p & 1u][q / NF], acc[q / NF][q % NF], 0, 0, 0);
                    if (p == 0) read_one(u, half, f, ga, gb);
                    if (p == 3) asm volatile("" : "+v"(wide[0][f]));   // (here, not in the next half)
                    if (p == 1) fetch_one(slots[(to + f / MF) % kSlots], unit + f / MF, f % MF, step);
                    __builtin_amdgcn_sched_barrier(0);
                }
        } else {
            read(u, half, ga, gb);
            fetch(slots[to % kSlots], unit, step);
            fetch(slots[(to + 1u) % kSlots], unit + 1u, step);
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int j = 0; j < NF; ++j) acc[i][j] = fp8_mfma32<FB, FA>(fb[j], fa[i], acc[i][j], sb[j], sa[i]);
            // four reads behind each of the first products, then fetches
#pragma unroll
            for (int i = 0; i < (MF + NF) / 2; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
            }
#pragma unroll
            for (int i = 0; i < 2 * MF; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
            }
        }
        up_to_here();
    };
    // For s_waitcnt: all but the youngest operations on memory (63 at most are counted).
    auto all_but = [](uint32_t left) {
        const uint32_t n = left < 63u ? left : 63u;
        return (n & 15u) | n >> 4 << 14;
    };
    auto step = [&](auto phase, uint32_t k) __attribute__((always_inline)) {   // phase: k mod 5
        constexpr uint32_t u = 4u * decltype(phase)::value;
        half_step(fa0, fb0, u, 1, fa1, fb1, sa, sb, u + 8u, 0, k + 2u);
        if (!kWalks || u != 0u || k != 0u) __builtin_amdgcn_s_waitcnt(all_but(2u * MF) | 0xF70u);
        __builtin_amdgcn_s_waitcnt(all_but(63u) | 0x070u);   // what was read
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        uint32_t ta[MF], tb[NF];   // the next step's scales
        if (((first + k) & 3u) == 3u) {   // (moved, not renamed: a load that may be on its way would be waited for in every step)
#pragma unroll
            for (int i = 0; i < MF; ++i) asm volatile("v_mov_b32 %0, %1" : "=v"(ta[i]) : "v"(next_a[i]));
#pragma unroll
            for (int j = 0; j < NF; ++j) asm volatile("v_mov_b32 %0, %1" : "=v"(tb[j]) : "v"(next_b[j]));
            const uint32_t w = ((first + k) >> 2) + 2u;
            scales(w < words ? w : 0u, next_a, next_b);
        } else {
#pragma unroll
            for (int i = 0; i < MF; ++i) ta[i] = sa[i] >> 8;
#pragma unroll
            for (int j = 0; j < NF; ++j) tb[j] = sb[j] >> 8;
        }
        __builtin_amdgcn_sched_barrier(0);
        half_step(fa1, fb1, u + 4u, 0, fa0, fb0, ta, tb, u + 10u, 2, k + 2u);
#pragma unroll
        for (int i = 0; i < MF; ++i) sa[i] = ta[i];
#pragma unroll
        for (int j = 0; j < NF; ++j) sb[j] = tb[j];
    };
    auto begin = [&]() __attribute__((always_inline)) {   // a tile's first scales and two steps
        scales(word0, sa, sb);
        scales(word0 + 1u < words ? word0 + 1u : 0u, next_a, next_b);
        __builtin_amdgcn_sched_barrier(0);
        fetch(s0, 0, 0);
        fetch(s1, 1, 0);
        fetch(s2, 2, 0);
        fetch(s3, 3, 0);
        fetch(s4, 0, 1);
        fetch(s5, 1, 1);
        fetch(s6, 2, 1);
        fetch(s7, 3, 1);
        __builtin_amdgcn_sched_barrier(0);
    };
    // 32 rows of a wave at a time by way of LDS, in the two units that the next tile's first steps leave free, so that a row leaves in
    // whole lines: stored as the matrix unit holds them, two lanes to a row, the writes of all workgroups took the caches ten times
    // as long.  Pieces of 16 bytes are kept at places exchanged by row, as above; fp32 sums leave in two halves of the columns.  One of
    // several parts keeps its sums in fp32, in rows with room up to a multiple of 8.
    auto emit = [&](auto wide, auto half, bool whole, uint32_t m1, uint32_t n1, void* out, uint64_t pitch, uint32_t columns, bool add) __attribute__((always_inline)) {
        constexpr bool kWide = decltype(wide)::value, kHalf16 = decltype(half)::value;   // sums kept in fp32; bf16 results
        constexpr uint32_t kPieces = 4u * NF, kEach = kWide ? 4u : 8u, kTurns = kWide ? 2u : 1u;   // of a strip's row, values of a piece
        static_assert(32u * kPieces * 16u <= kUnit / 2u, "a strip fits half a unit");
        uint8_t* strip = (wave < 2u ? s8 : s9) + (wave & 1u) * (kUnit / 2u);
        auto place = [&](uint32_t r, uint32_t piece) __attribute__((always_inline)) {
            return reinterpret_cast<uint4*>(strip + (r * kPieces + (piece ^ (kPieces >= 16u ? r & 15u : (r >> 1) & 7u))) * 16u);
        };
        uint32_t l = lane;   // (places are worked out here, in each variant by itself, not kept while products are formed)
        asm volatile("; %1" : "+v"(l) : "n"(kWide + 2 * kHalf16));
        asm volatile("s_nop 15\n s_nop 15");   // (the last products' results; the reads below are written out, else whole sums are copied and spilled)
        const uint32_t x = l & 31u, h = l >> 5;
#pragma unroll
        for (uint32_t turn = 0; turn < MF * kTurns; ++turn) {
            const uint32_t i = turn / kTurns, j0 = turn % kTurns * NF, nw = n1 + wn * 32u * NF + j0 * 16u;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (uint32_t j = 0; j < 2u * NF / kTurns; ++j) {
                float v[8];
#pragma unroll
                for (uint32_t e = 0; e < 8u; ++e)
                    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[e]) : "a"(acc[i][(j0 + j) >> 1][8u * ((j0 + j) & 1u) + e]));
                const uint32_t g = 2u * j + h;   // 8 columns
                if (kWide) {
                    *place(x, 2u * g) = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
                    *place(x, 2u * g + 1u) = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
                } else {
                    *place(x, g) = make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            const uint32_t r0 = l / kPieces, piece = l % kPieces, n = nw + piece * kEach, row = m1 + wm * 32u * MF + i * 32u + r0;
            if (whole) {
                uint8_t* at = static_cast<uint8_t*>(out) + (row * pitch + n) * (kHalf16 ? 2u : 4u);
                const uint64_t step = 64u / kPieces * pitch * (kHalf16 ? 2u : 4u);
                uint4 w[kPieces / 2u];
#pragma unroll
                for (uint32_t it = 0; it < kPieces / 2u; ++it) w[it] = *place(r0 + it * (64u / kPieces), piece);
#pragma unroll
                for (uint32_t it = 0; it < kPieces / 2u; ++it, at += step) store16(at, w[it]);
            } else {
#pragma unroll 1
                for (uint32_t it = 0; it < kPieces / 2u; ++it) {
                    const uint32_t m = row + it * (64u / kPieces);
                    const uint4 w = *place(r0 + it * (64u / kPieces), piece);
                    uint8_t* at = static_cast<uint8_t*>(out) + (m * pitch + n) * (kHalf16 ? 2u : 4u);
                    if (m >= a.M || n >= columns) continue;
                    if (kWide) {
                        store4<kHalf16>(at, f32x4{__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w)}, columns - n, add);
                    } else if (n + 8u <= columns) {
                        store16(at, w);
                    } else {
                        const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (uint32_t e = 0; e < 7u; ++e)
                            if (n + e < columns) reinterpret_cast<uint16_t*>(at)[e] = (uint16_t)(words[e >> 1] >> (e & 1u ? 16 : 0));
                    }
                }
                __builtin_amdgcn_s_waitcnt(0x0F70);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    go_to(blockIdx.x);
    begin();
    __builtin_amdgcn_s_waitcnt(all_but(kWalks ? 0u : 4u * MF) | 0xF70u);
    for (uint32_t tile = blockIdx.x;;) {
        float zero;
        asm volatile("v_mov_b32 %0, 0" : "=v"(zero));   // (else sixteen zeros are kept for the next tile)
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < NF; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = zero;
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < MF; ++i) sa[i] >>= 8u * (first & 3u);
#pragma unroll
        for (int j = 0; j < NF; ++j) sb[j] >>= 8u * (first & 3u);
        read(0, 0, fa0, fb0);
        if constexpr (EXACT)
#pragma unroll
            for (uint32_t f = 0; f < MF + NF; ++f) widen(0, f, 0, fa0, fb0, sa, sb);
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
        __builtin_amdgcn_s_waitcnt(0x0070);   // (what was fetched behind the last step, and read)
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        up_to_here();
        const uint32_t m = m0, n = n0;
        tile += gridDim.x;
        const bool more = kWalks && tile < tiles_m * tiles_n;
        if (more) {
            go_to(tile);
            begin();
        }
        // Whole tiles leave in a known number of stores, which are still on their way when the next tile begins: only its first two steps,
        // fetched before them, are waited for.  (They are waited for sooner than here: the compiler does not know a strip from the units
        // that are fetched to, and waits for all fetches before the first write to a strip.)
        // Tiles that are added to what is there take the ragged way out, piece by piece: 8192 x 8192 x 2048 373 us for 219 to fp32, 265 for
        // 115 to bf16; 2048 x 8192 x 8192 218 for 191 and 117 for 94.
        using yes = std::true_type;
        using no = std::false_type;
        const bool whole = m + BM <= a.M && n + BN <= a.N && !a.accumulate;
        if (!kWalks && a.share < blocks) {   // (the larger tiles are not divided)
            const uint64_t pitch = fp8_part_pitch(a.N);
            emit(yes{}, no{}, whole, m, n, a.workspace + blockIdx.y * a.M * pitch, pitch, (uint32_t)pitch, false);
            break;
        } else if (EXACT) {
            emit(yes{}, no{}, whole, m, n, a.c, a.ldc, a.N, a.accumulate);
            if (!more) break;
            __builtin_amdgcn_s_waitcnt(all_but(4u * MF * NF) | 0xF70u);
        } else if (a.accumulate) {   // (the old value is added before the only rounding)
            emit(yes{}, yes{}, false, m, n, a.c, a.ldc, a.N, true);
            if (!more) break;
        } else {
            emit(no{}, yes{}, whole, m, n, a.c, a.ldc, a.N, false);
            if (!more) break;
            __builtin_amdgcn_s_waitcnt(all_but(2u * MF * NF) | 0xF70u);
        }
    }
}

// The parts' sums, added in their order: four neighbouring values of a row to a thread.
template <bool BF16>
__global__ __launch_bounds__(256) void fp8_join_kernel(Fp8MatmulArgs a, uint32_t parts) {
    const uint32_t pieces = (a.N + 3u) / 4u;
    const uint64_t pitch = fp8_part_pitch(a.N), total = (uint64_t)a.M * pieces, step = (uint64_t)gridDim.x * 256u;
    for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < total; i += step) {
        const uint32_t m = (uint32_t)(i / pieces), n = (uint32_t)(i % pieces) * 4u;
        const float* at = a.workspace + m * pitch + n;
        float4 v = *reinterpret_cast<const float4*>(at);
#pragma unroll 8
        for (uint32_t p = 1; p < parts; ++p) {
            const float4 w = *reinterpret_cast<const float4*>(at + p * a.M * pitch);
            v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
        }
        uint8_t* c = static_cast<uint8_t*>(a.c) + (m * a.ldc + n) * (BF16 ? 2u : 4u);
        store4<BF16>(c, f32x4{v.x, v.y, v.z, v.w}, a.N - n, a.accumulate);
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

// How a product is done, by its sizes alone (an order of additions may depend on nothing else).  Measured on the device:
//  - up to 16 rows: direct, unless there are 24576 rows of B or more (2048 along k: one row and 8192 rows of B 7.5 us direct and
//    10.6 us tiled; 16 rows and 16384 rows of B 11.4 and 12.7 us, 24576 16 and 13 us, 50257 34 and 23 us);
//    up to 32 rows, for 4096 rows of B or fewer (32 rows: 2048 x 2048 5.8 and 9.1 us, 2048 x 8192 11 and 14 us, 8192 x 2048 11 and 10 us);
//  - tiles of 256 x 256 where they are expected to be shorter: 256 of them run at a time, 512 of 128 x 128, two on a compute unit
//    and 1.4 times as long for their size (bf16 results, which wait for memory) or 1.06 times (fp32), the last of them less.
//    Measured, in us with 256 and 128, bf16 and fp32: 2048 x 4096 x 2048 26 and 19, 46 and 30; 3000 x 4096 x 2048 29 and 29, 53 and 45;
//    4096 x 4096 x 2048 31 and 37, 57 and 58; 4608 x 4096 x 2048 48 and 43, 90 and 67; 7168 x 4096 x 2048 54 and 61, 104 and 96;
//    1024 x 50304 x 1024 66 and 73, 119 and 118; 16384 x 8192 x 8192 705 and 905; 8192^3 fp32 690 and 740;
//    The columns of tiles behind whole rounds of 256, if they are at most 512 tiles of 128 x 128, in those and a launch of their own, where that is
//    shorter (in tiles of 256, of 128 and of both: 1003 x 50257 x 1024 69, 71 and 64 us; 4608 x 4096 x 8192 149, 137 and 123 us, fp32
//    292, 223 and 220; 9216 x 4096 x 2048 76, 75 and 72 us; with 576 small ones, 6144 x 4096 x 2048, 51, 51 and 57 us);
//  - short fp32 products of few tiles of 128 x 128: direct, tiles of 64 x 64 (777 x 520 x 1000, 35 tiles: 8.4 and 9.4 us, to bf16
//    8.0 and 6.8; 512 x 512 x 1536 10.4 and 11.0 us, to bf16 9.8 and 7.6);
//  - tiles of 128 x 128 otherwise, the blocks along k divided among workgroups where that is expected to be
//    shorter: a block takes such a tile 0.45 us, a second launch 2 us, and the parts' sums pass memory twice at about 3 TB/s
//    (1024 x 1024 x 16384: 59 us undivided, 41, 29 and 31 us in 2, 4 and 8 parts; 512 x 2048 x 2048: 11, 15 and 20 us in 1, 2
//    and 4 parts).
struct Plan {
    uint32_t tile;      // of the tiled kernel: 256 or 128; of the direct one: 64, or 16 (few rows: all of A, 16 of B)
    uint32_t parts;     // among which the blocks along k are divided
    uint32_t columns;   // of tiles of 256 x 256: those of whole rounds, what is behind them in tiles of 128 x 128; 0: all
};
static Plan plan_for(uint64_t M, uint64_t N, uint64_t K, bool bf16) {
    auto tiles = [&](uint64_t rows, uint64_t cols) { return ((M + rows - 1) / rows) * ((N + cols - 1) / cols); };
    const uint64_t steps = (K + kStep - 1) / kStep;
    if ((M <= kFp8FewRows && N < 24576u) || (M <= 2u * kFp8FewRows && N <= 4096u)) {
        uint64_t parts = 256u / tiles(M > kFp8FewRows ? 2u * kFp8FewRows : kFp8FewRows, 16);   // (no part shorter than two blocks for each of 8 waves)
        parts = parts < steps / 16u ? parts : steps / 16u;
        return {16u, (uint32_t)(parts > 1u ? parts : 1u)};
    }
    const uint64_t count = tiles(128, 128);
    auto small = [&](uint64_t n) { return (bf16 ? 2.8 : 2.12) * (n > 512u ? n / 512.0 : 1.0); };
    const uint64_t high = (M + 255u) / 256u, all = tiles(256, 256), whole = all / kUnits * kUnits / high;   // columns of tiles in whole rounds
    const uint64_t rest = whole * 256u < N ? (M + 127u) / 128u * ((N - whole * 256u + 127u) / 128u) : 0u;
    const double large = 4.0 * ((all + kUnits - 1u) / kUnits), large_and_small = 4.0 * (all / kUnits) + (rest <= 256u ? bf16 ? 2.2 : 1.5 : bf16 ? 3.1 : 2.4);
    if (whole != 0u && rest != 0u && rest <= 512u && large_and_small < large && large_and_small < small(count)) return {256u, 1u, (uint32_t)whole};
    if (large < small(count)) return {256u, 1u};
    if (!bf16 && count < 48u && tiles(64, 64) >= 40u && steps <= 12u) return {64u, 1u};
    Plan best{128u, 1u};
    double least = 0.45 * steps;
    for (uint32_t parts = 2; parts * count <= 512u && parts * 4u <= steps; parts *= 2u) {
        const double time = 0.45 * ((steps + parts - 1u) / parts) + 2.0 + 8e-6 / 3.0 * parts * M * fp8_part_pitch(N);
        if (time < least) {
            least = time;
            best.parts = parts;
        }
    }
    return best;
}

bool fp8_rows_are_few(uint64_t M, uint64_t N, uint64_t K) { return plan_for(M, N, K, true).tile == 16u; }

uint64_t fp8_matmul_workspace_bytes(uint64_t M, uint64_t N, uint64_t K) {
    if (M == 0 || N == 0 || K == 0) return 0;
    uint64_t bytes = 0;   // enough for either type of results
    for (const bool bf16 : {false, true}) {
        const Plan p = plan_for(M, N, K, bf16);
        const uint64_t need = p.parts > 1u ? p.parts * M * fp8_part_pitch(N) * sizeof(float) : 0;
        bytes = need > bytes ? need : bytes;
    }
    return bytes;
}

uint32_t fp8_few_rows_parts(uint64_t M, uint64_t N, uint64_t K) { return plan_for(M, N, K, true).parts; }

hipError_t launch_fp8_matmul(const Fp8MatmulArgs& args, hipStream_t stream) {
    Fp8MatmulArgs a = args;
    if (a.K == 0u) {   // (there may be no codes and scales to read)
        if (a.accumulate) return hipSuccess;
        const uint64_t blocks = ((uint64_t)a.M * a.N + 255u) / 256u;
        zero_matrix_kernel<<<(uint32_t)(blocks < 4096u ? blocks : 4096u), 256, 0, stream>>>(a);
        return hipGetLastError();
    }
    const Plan plan = plan_for(a.M, a.N, a.K, a.out_bf16);
    if (plan.tile < 128u) {
        Fp8DirectArgs direct{};
        static_cast<Fp8MatmulArgs&>(direct) = a;
        return launch_fp8_direct(direct, stream);
    }
    const uint32_t blocks = (a.K + kStep - 1u) / kStep;
    uint32_t tm = (a.M + plan.tile - 1u) / plan.tile, tn = plan.columns ? plan.columns : (a.N + plan.tile - 1u) / plan.tile;
    a.first_n = 0u;
    a.share = (blocks + plan.parts - 1u) / plan.parts;
    const uint32_t parts = (blocks + a.share - 1u) / a.share;
    // (tiles of 256 x 256 are walked by a workgroup on each compute unit)
    const dim3 grid(plan.tile == 256u && tm * tn > kUnits ? kUnits : tm * tn, parts);
    auto go = [&](auto FA, auto FB, auto EXACT) {
        constexpr int A = decltype(FA)::value, B = decltype(FB)::value;
        constexpr bool E = decltype(EXACT)::value;
        if (plan.tile == 256u) fp8_matmul_tiled_kernel<A, B, E, 4, 4><<<grid, 256, 0, stream>>>(a, tm, tn);
        else fp8_matmul_tiled_kernel<A, B, E, 2, 2><<<grid, 256, 0, stream>>>(a, tm, tn);
        if (plan.columns) {
            a.first_n = plan.columns * 256u;
            tm = (a.M + 127u) / 128u;
            tn = (a.N - a.first_n + 127u) / 128u;
            fp8_matmul_tiled_kernel<A, B, E, 2, 2><<<tm * tn, 256, 0, stream>>>(a, tm, tn);
        }
        return hipGetLastError();
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    auto out = [&](auto FA, auto FB) { return a.out_bf16 ? go(FA, FB, std::false_type{}) : go(FA, FB, std::true_type{}); };
    auto with_b = [&](auto FA) { return a.b_e5m2 ? out(FA, I1{}) : out(FA, I0{}); };
    const hipError_t rc = a.a_e5m2 ? with_b(I1{}) : with_b(I0{});
    return rc != hipSuccess || parts == 1u ? rc : launch_fp8_join(a, parts, stream);
}

hipError_t launch_fp8_join(const Fp8MatmulArgs& a, uint32_t parts, hipStream_t stream) {
    const uint64_t join = ((uint64_t)a.M * ((a.N + 3u) / 4u) + 255u) / 256u;
    const uint32_t join_grid = (uint32_t)(join < 4096u ? join : 4096u);
    if (a.out_bf16) fp8_join_kernel<true><<<join_grid, 256, 0, stream>>>(a, parts);
    else fp8_join_kernel<false><<<join_grid, 256, 0, stream>>>(a, parts);
    return hipGetLastError();
}

}  // namespace thc
