// Embedding lookup and its gradient.
//
// Lookup: rows are gathered 16 bytes a lane; memory is what bounds it.
//
// Gradient: the tokens are sorted (stable, so that a row's terms keep their order), the sorted list is cut into pieces of equal
// length, and a group of lanes adds the rows of a piece, run by run of equal tokens: however often a token occurs,
// the work is divided evenly, and every sum has one order.  A run inside a piece is written directly; of a run that
// crosses a piece's border the piece keeps its part, and a last launch adds the parts.  Rows of the table whose token does not occur are
// zeroed by further workgroups of the sorting and the summing launches.
//
// What bounds it: memory.  Lookup: 8192 rows of 2048 bf16 10.2 us, 67 MB, 6.6 TB/s (rows that occur often come from the caches).  Gradient: the
// write of the whole table, 3.8 TB/s while the tokens are sorted beside it (8192 tokens, 50257 x 1024 to fp32: 66 us, 223 MB); then the way through
// memory that a piece's keys, its rows and the parts of the longest run take one after the other (the sums of 8192 x 1024 bf16 by
// themselves 15 us, the last launch 7 us).  The parts of one run are added by one group of lanes, 16 at a time: 16384 tokens, 30522 x 768 to bf16, take
// 50 us, 104 with 60 % of them on one row of the table and 140 with 95 % (42 and 40 where these are outside the table).
#include "thc_fp8.h"
#include "thc_internal.h"

#pragma clang fp contract(off)

namespace thc {
namespace {

constexpr uint32_t kThreads = 256;

// ---------------------------------------------------------------- values of a row, 8 a lane
template <bool BF16>
__device__ __forceinline__ void load_row(const void* p, uint64_t at, uint32_t valid, float (&v)[8]) {
    if (valid >= 8u) {
        Row8<BF16> r;
        r.load(static_cast<const uint8_t*>(p) + at * (BF16 ? 2u : 4u));
        r.values(v);   // (not added to zeros: -0 would become 0)
        return;
    }
#pragma unroll
    for (uint32_t e = 0; e < 8u; ++e)
        v[e] = e >= valid ? 0.0f : BF16 ? bf16_low(static_cast<const uint16_t*>(p)[at + e]) : static_cast<const float*>(p)[at + e];
}
template <bool BF16>
__device__ __forceinline__ void store_row(void* p, uint64_t at, uint32_t valid, const float (&v)[8]) {
    uint8_t* c = static_cast<uint8_t*>(p) + at * (BF16 ? 2u : 4u);
    if (valid >= 8u) {
        Row8<BF16>::store(c, v);
        return;
    }
#pragma unroll
    for (uint32_t e = 0; e < 8u; ++e)
        if (e < valid) store1<BF16>(c + e * (BF16 ? 2u : 4u), v[e], false);
}

__device__ __forceinline__ int64_t token_at(const EmbedArgs& a, uint64_t i) {
    return a.wide_tokens ? static_cast<const int64_t*>(a.tokens)[i] : (int64_t)static_cast<const int32_t*>(a.tokens)[i];
}

// ---------------------------------------------------------------- lookup
template <bool IN, bool OUT>
__global__ __launch_bounds__(kThreads) void embed_forward_kernel(EmbedArgs a, uint32_t pieces) {
    const uint64_t total = (uint64_t)a.count * pieces, step = (uint64_t)gridDim.x * kThreads;
    for (uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += step) {
        const uint64_t row = i / pieces;
        const uint32_t d = (uint32_t)(i % pieces) * 8u, valid = a.dim - d;
        const int64_t token = token_at(a, row);
        float v[8] = {};
        if (token >= 0 && token < (int64_t)a.vocab) {
            load_row<IN>(a.in, (uint64_t)token * a.ld_in + d, valid, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= a.scale;
        }
        store_row<OUT>(a.out, row * a.ld_out + d, valid, v);
    }
}

// ---------------------------------------------------------------- sorting the tokens
// Keys: the token, or `vocab` for one outside the table, which sorts behind all others.
__device__ __forceinline__ uint32_t key_at(const EmbedArgs& a, uint32_t i) {
    const int64_t t = token_at(a, i);
    return t >= 0 && t < (int64_t)a.vocab ? (uint32_t)t : a.vocab;
}

// Lanes that hold the same digit as this one, among those of `in`.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, uint32_t bits, uint64_t in) {
    uint64_t mask = in;
    for (uint32_t b = 0; b < bits; ++b) {
        const bool one = (digit >> b) & 1u;
        const uint64_t ones = __ballot(one);
        mask &= one ? ones : ~ones;
    }
    return mask;
}

// Zeros in rows [first, end) of the table, by workgroup `group` of `groups`.
template <bool OUT>
__device__ __forceinline__ void zero_rows(const EmbedArgs& a, uint32_t first, uint32_t end, uint32_t group, uint32_t groups) {
    constexpr uint32_t kEach = OUT ? 8u : 4u, kSize = OUT ? 2u : 4u;   // values in 16 bytes
    const uint32_t pieces = (a.dim + kEach - 1u) / kEach;
    const uint64_t total = (uint64_t)(end - first) * pieces, step = (uint64_t)groups * blockDim.x;
    for (uint64_t i = (uint64_t)group * blockDim.x + threadIdx.x; i < total; i += step) {
        const uint32_t d = (uint32_t)(i % pieces) * kEach;
        uint8_t* at = static_cast<uint8_t*>(a.out) + ((first + i / pieces) * a.ld_out + d) * kSize;
        if (d + kEach <= a.dim) {
            store16(at, make_uint4(0u, 0u, 0u, 0u));
            continue;
        }
        for (uint32_t e = 0; d + e < a.dim; ++e) store1<OUT>(at + e * kSize, 0.0f, false);
    }
}
// The workgroups of a sorting launch behind the first `sorters`: zeros in their launch's share of the table.
struct ZeroShare {
    uint32_t first, end;   // rows
};
__device__ __forceinline__ bool zeroes(const EmbedArgs& a, const ZeroShare& z, uint32_t sorters) {
    if (blockIdx.x < sorters) return false;
    if (a.out_bf16) zero_rows<true>(a, z.first, z.end, blockIdx.x - sorters, gridDim.x - sorters);
    else zero_rows<false>(a, z.first, z.end, blockIdx.x - sorters, gridDim.x - sorters);
    return true;
}

// Between the accesses of a wave's lanes to what other lanes of the wave have written in LDS.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// One pass of a stable radix sort.  The list is cut into at most 256 tiles, one per workgroup; `counts` holds every tile's number of keys per
// digit.
struct SortPass {
    const uint32_t* keys;    // null: the tokens themselves, in their order
    const uint32_t* places;
    uint32_t* keys_out;
    uint32_t* places_out;
    uint32_t* counts;        // tiles x digits
    uint32_t tile;           // keys of a tile, a multiple of 256
    uint32_t tiles;
    uint32_t shift, bits;
};

__global__ __launch_bounds__(kThreads) void sort_count_kernel(EmbedArgs a, SortPass s, ZeroShare z) {
    extern __shared__ uint32_t s_count[];
    if (zeroes(a, z, s.tiles)) return;
    const uint32_t digits = 1u << s.bits, first = blockIdx.x * s.tile, end = a.count - first < s.tile ? a.count : first + s.tile;
    for (uint32_t d = threadIdx.x; d < digits; d += kThreads) s_count[d] = 0u;
    __syncthreads();
    for (uint32_t i = first + threadIdx.x; i < end; i += kThreads) {
        const uint32_t key = s.keys ? s.keys[i] : key_at(a, i);
        atomicAdd(&s_count[(key >> s.shift) & (digits - 1u)], 1u);
    }
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < digits; d += kThreads) s.counts[(uint64_t)blockIdx.x * digits + d] = s_count[d];
}

// Sum of the values of lower threads.
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t* s_wave) {
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = t >> 6;
    uint32_t x = v;
#pragma unroll
    for (uint32_t o = 1; o < 64u; o <<= 1) {
        const uint32_t y = (uint32_t)__shfl_up((int)x, o);
        x += lane >= o ? y : 0u;
    }
    if (lane == 63u) s_wave[wave] = x;
    __syncthreads();
    uint32_t before = x - v;
    for (uint32_t w = 0; w < wave; ++w) before += s_wave[w];
    __syncthreads();
    return before;
}

__global__ __launch_bounds__(kThreads) void sort_scatter_kernel(EmbedArgs a, SortPass s, ZeroShare z) {
    extern __shared__ uint32_t s_next[];   // 4 waves x digits: first the numbers, then the next place of a digit; 2 x digits of scratch
    __shared__ uint32_t s_wave[kThreads / 64u];
    if (zeroes(a, z, s.tiles)) return;
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = t >> 6, digits = 1u << s.bits;
    const uint32_t first = blockIdx.x * s.tile, end = a.count - first < s.tile ? a.count : first + s.tile;
    const uint32_t from = first + wave * (s.tile / 4u), to = end < from + s.tile / 4u ? end : from + s.tile / 4u;
    uint32_t* mine = s_next + wave * digits;
    for (uint32_t d = t; d < 4u * digits; d += kThreads) s_next[d] = 0u;
    __syncthreads();
    // every wave has a run of the tile, of which it counts the digits ...
    for (uint32_t i0 = from; i0 < to; i0 += 64u) {
        const uint32_t i = i0 + lane;
        const bool in = i < to;
        const uint32_t digit = in ? ((s.keys ? s.keys[i] : key_at(a, i)) >> s.shift) & (digits - 1u) : 0u;
        const uint64_t same = same_digit(digit, s.bits, __ballot(in));
        if (in && (same & ((1ull << lane) - 1ull)) == 0ull) mine[digit] += (uint32_t)__popcll(same);
        wave_fence();
    }
    __syncthreads();
    // ... from which follows where its keys go: behind all smaller digits, and behind its own of earlier tiles and waves
    uint32_t *s_total = s_next + 4u * digits, *s_here = s_total + digits;
    for (uint32_t d = t; d < digits; d += kThreads) {
        uint32_t total = 0u, here = 0u;
        for (uint32_t tile = 0; tile < s.tiles; tile += 16u) {
            uint32_t n[16];
#pragma unroll
            for (uint32_t q = 0; q < 16u; ++q) n[q] = tile + q < s.tiles ? s.counts[(uint64_t)(tile + q) * digits + d] : 0u;
#pragma unroll
            for (uint32_t q = 0; q < 16u; ++q) {
                total += n[q];
                here += tile + q < blockIdx.x ? n[q] : 0u;
            }
        }
        s_total[d] = total;
        s_here[d] = here;
    }
    __syncthreads();
    const uint32_t each = (digits + kThreads - 1u) / kThreads, d0 = t * each < digits ? t * each : digits, d1 = digits - d0 < each ? digits : d0 + each;
    uint32_t total = 0u;
    for (uint32_t d = d0; d < d1; ++d) total += s_total[d];
    uint32_t at = sum_before(total, s_wave);
    for (uint32_t d = d0; d < d1; ++d) {
        uint32_t here = at + s_here[d];
        at += s_total[d];
        for (uint32_t w = 0; w < 4u; ++w) {
            const uint32_t n = s_next[w * digits + d];
            s_next[w * digits + d] = here;
            here += n;
        }
    }
    __syncthreads();
    for (uint32_t i0 = from; i0 < to; i0 += 64u) {
        const uint32_t i = i0 + lane;
        const bool in = i < to;
        const uint32_t key = in ? (s.keys ? s.keys[i] : key_at(a, i)) : 0u, digit = (key >> s.shift) & (digits - 1u);
        const uint64_t same = same_digit(digit, s.bits, __ballot(in)), below = same & ((1ull << lane) - 1ull);
        const uint32_t next = mine[digit];
        wave_fence();
        if (in) {
            const uint32_t place = next + (uint32_t)__popcll(below);
            s.keys_out[place] = key;
            s.places_out[place] = s.keys ? s.places[i] : i;
            if (below == 0ull) mine[digit] = next + (uint32_t)__popcll(same);
        }
        wave_fence();
    }
}

// Up to kFew tokens, in one launch: an entry's place is the number of entries that sort before it, counted by looking at all of them.  A
// workgroup holds all keys in LDS and counts for 16 entries; 16 neighbouring lanes take one entry each and a share of the keys, four at a
// time.  2784 tokens 5.7 us, 6144 13 us.  (A radix sort in one workgroup's LDS took 8 us longer for 2784; the launches above take 4 us longer
// for 5000 tokens and 1 us less for 8192.)
constexpr uint32_t kFew = 6144, kFewThreads = 512, kFewEntries = 16;
__global__ __launch_bounds__(kFewThreads) void sort_few_kernel(EmbedArgs a, uint32_t* keys_out, uint32_t* places_out, uint32_t sorters, ZeroShare z) {
    if (zeroes(a, z, sorters)) return;
    constexpr uint32_t kShares = kFewThreads / kFewEntries;
    __shared__ __attribute__((aligned(16))) uint32_t s_key[kFew];
    __shared__ uint32_t s_before[kShares][kFewEntries];
    const uint32_t t = threadIdx.x, entry = t % kFewEntries, share = t / kFewEntries, fours = (a.count + 3u) / 4u;
    for (uint32_t i = t; i < 4u * fours; i += kFewThreads) s_key[i] = i < a.count ? key_at(a, i) : ~0u;   // (behind the last: before nothing)
    __syncthreads();
    const uint32_t i = blockIdx.x * kFewEntries + entry, key = s_key[i < a.count ? i : 0u];
    uint32_t before = 0u;
    for (uint32_t f = share; f < fours; f += kShares) {
        const uint4 k = *reinterpret_cast<const uint4*>(&s_key[4u * f]);
        const uint32_t j = 4u * f;   // (of equal keys the earlier ones; key + 1 <= 2^31)
        before += k.x < key + (j < i) ? 1u : 0u;
        before += k.y < key + (j + 1u < i) ? 1u : 0u;
        before += k.z < key + (j + 2u < i) ? 1u : 0u;
        before += k.w < key + (j + 3u < i) ? 1u : 0u;
    }
    s_before[share][entry] = before;
    __syncthreads();
    if (t >= kFewEntries || i >= a.count) return;
    uint32_t place = 0u;
#pragma unroll
    for (uint32_t q = 0; q < kShares; ++q) place += s_before[q][entry];
    keys_out[place] = key;
    places_out[place] = i;
}

// ---------------------------------------------------------------- sums of the runs
struct SumArgs {
    const uint32_t* keys;     // sorted
    const uint32_t* places;
    float* parts;             // 2 x pieces x pitch: what a piece has of a run begun before it, and of one that goes on behind it
    uint64_t pitch;           // dim rounded up to a multiple of 8
    uint32_t piece, pieces;   // entries of a piece, and how many
    uint32_t lanes;           // of a group: a power of two
    uint32_t slices;          // groups side by side on a row
    uint32_t sum_groups;      // workgroups that sum; the others write zeros
    uint32_t zero_from;                // rows from here on are set to zero by the sums' launch where they get no gradient
};

// First entry in [lo, hi) whose key is at least `key`.
__device__ __forceinline__ uint32_t lower_bound(const uint32_t* keys, uint32_t lo, uint32_t hi, uint32_t key) {
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2u;
        if (keys[mid] < key) lo = mid + 1u;
        else hi = mid;
    }
    return lo;
}

constexpr uint32_t kZeroRows = 32;   // rows of the table that a workgroup looks after

// Which of the rows v0 .. v0 + 31 have an entry among the sorted keys, one bit each, by a wave.  The entries of these rows are found by looking at 32
// keys at a time, the lower lanes for the first one and the upper ones for the end: three looks for up to 2^15 entries, where halving takes 15
// one after the other (of which each waits for memory).
__device__ __forceinline__ uint32_t rows_with_entries(const uint32_t* keys, uint32_t count, uint32_t v0, uint32_t vocab) {
    const uint32_t lane = threadIdx.x & 63u, sub = lane & 31u, past = vocab - v0 < kZeroRows ? vocab : v0 + kZeroRows;
    const uint32_t target = lane < 32u ? v0 : past;
    uint32_t lo = 0u, hi = count;
    while (__any(lo < hi)) {
        const uint32_t stride = (hi - lo + 31u) / 32u, at = lo + sub * stride;
        const bool less = at < hi && keys[at] < target;
        const uint64_t all = __ballot(less);
        const uint32_t n = (uint32_t)__popc((uint32_t)(lane < 32u ? all : all >> 32));
        if (n == 0u) {
            hi = lo;
        } else {
            const uint32_t next = lo + n * stride;
            lo = lo + (n - 1u) * stride + 1u;
            hi = next < hi ? next : hi;
        }
    }
    const uint32_t first = (uint32_t)__shfl((int)lo, 0), end = (uint32_t)__shfl((int)lo, 32);
    uint32_t mask = 0u;
    if (end - first <= 64u) {
        if (lane < end - first) mask = 1u << (keys[first + lane] - v0);
    } else if (lane < past - v0) {
        const uint32_t i = lower_bound(keys, first, end, v0 + lane);
        mask = i < end && keys[i] == v0 + lane ? 1u << lane : 0u;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) mask |= (uint32_t)__shfl_xor((int)mask, o);
    return mask;
}

// The 8 columns that a lane sums.  Rows need not be a multiple of 8 long: the last lane of a row takes its last 8 columns, of which the
// first `skip` are its neighbour's too, so that every load is a whole one; a row shorter than 8 is loaded value by value.
struct Columns {
    uint32_t d, skip, end;   // the lane writes columns d + skip .. d + end - 1
    __device__ __forceinline__ Columns(uint32_t chunk, uint32_t dim) {
        d = chunk * 8u;
        skip = 0u;
        end = 8u;
        if (dim < 8u) {
            end = dim;
        } else if (d + 8u > dim) {
            skip = d + 8u - dim;
            d = dim - 8u;
        }
    }
};

template <bool OUT>
__device__ __forceinline__ void finish_row(const EmbedArgs& a, uint32_t key, const Columns& c, const float (&sum)[8]) {
    constexpr uint32_t kSize = OUT ? 2u : 4u;
    uint8_t* at = static_cast<uint8_t*>(a.out) + ((uint64_t)key * a.ld_out + c.d) * kSize;
    if (c.skip == 0u && c.end == 8u) {
        float v[8] = {};
        if (a.accumulate) {
            Row8<OUT> old;
            old.load(at);
            old.values(v);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = a.accumulate ? v[e] + sum[e] * a.scale : sum[e] * a.scale;
        Row8<OUT>::store(at, v);
        return;
    }
#pragma unroll
    for (uint32_t e = 0; e < 8u; ++e)
        if (e >= c.skip && e < c.end) store1<OUT>(at + e * kSize, sum[e] * a.scale, a.accumulate);
}

template <bool IN, bool OUT>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(EmbedArgs a, SumArgs s) {
    if (blockIdx.x >= s.sum_groups) {
        // Rows whose token does not occur.
        __shared__ uint32_t s_present;
        constexpr uint32_t kEach = OUT ? 8u : 4u;   // values in 16 bytes
        const uint32_t t = threadIdx.x;
        for (uint64_t v0 = s.zero_from + (uint64_t)(blockIdx.x - s.sum_groups) * kZeroRows; v0 < a.vocab; v0 += (uint64_t)(gridDim.x - s.sum_groups) * kZeroRows) {
            if (t < 64u) {
                const uint32_t mask = rows_with_entries(s.keys, a.count, (uint32_t)v0, a.vocab);
                if (t == 0u) s_present = a.vocab - v0 < kZeroRows ? mask | ~0u << (a.vocab - v0) : mask;   // (none behind the table)
            }
            __syncthreads();
            const uint32_t absent = ~s_present;
            for (uint32_t r = 0; r < kZeroRows; ++r) {
                if (!((absent >> r) & 1u)) continue;
                uint8_t* row = static_cast<uint8_t*>(a.out) + (v0 + r) * a.ld_out * (OUT ? 2u : 4u);
                for (uint32_t c = kEach * t; c < a.dim; c += kEach * kThreads) {
                    if (c + kEach <= a.dim) {
                        store16(row + c * (OUT ? 2u : 4u), make_uint4(0u, 0u, 0u, 0u));
                        continue;
                    }
                    for (uint32_t d = c; d < a.dim; ++d) store1<OUT>(row + d * (OUT ? 2u : 4u), 0.0f, false);
                }
            }
            __syncthreads();
        }
        return;
    }
    const uint64_t group = ((uint64_t)blockIdx.x * kThreads + threadIdx.x) / s.lanes;
    const uint32_t p = (uint32_t)(group / s.slices), slice = (uint32_t)(group % s.slices);
    const uint32_t chunk = slice * s.lanes + threadIdx.x % s.lanes;
    if (p >= s.pieces || chunk * 8u >= a.dim) return;
    const Columns columns(chunk, a.dim);
    const uint32_t d = columns.d, begin = p * s.piece, end = a.count - begin < s.piece ? a.count : begin + s.piece;
    uint32_t key = s.keys[begin];
    bool open = begin != 0u && s.keys[begin - 1u] == key;   // the run has begun before the piece
    float sum[8] = {};
    float* part = s.parts + (uint64_t)p * s.pitch + d;
    auto keep = [&](float* to) { Row8<false>::store(to, sum); };
    // Rows are loaded several at a time, those of tokens outside the table at the border too (they are rows of grad_out like the
    // others); keys and places a step ahead.
    constexpr uint32_t kAhead = IN ? 16 : 8;
    uint32_t k[kAhead], place[kAhead];
    auto look = [&](uint32_t i) {
#pragma unroll
        for (uint32_t q = 0; q < kAhead; ++q) {
            const uint32_t j = i + q < end ? i + q : end - 1u;
            k[q] = s.keys[j];
            place[q] = s.places[j];
        }
    };
    look(begin);
    for (uint32_t i = begin; i < end; i += kAhead) {
        Row8<IN> v[kAhead];
        uint32_t now[kAhead];
        if (k[0] < a.vocab) {
            if (a.dim >= 8u) {
#pragma unroll
                for (uint32_t q = 0; q < kAhead; ++q)
                    v[q].load(static_cast<const uint8_t*>(a.in) + ((uint64_t)place[q] * a.ld_in + d) * (IN ? 2u : 4u));
            } else {
#pragma unroll
                for (uint32_t q = 0; q < kAhead; ++q) v[q].load_some(a.in, (uint64_t)place[q] * a.ld_in, a.dim);
            }
        }
#pragma unroll
        for (uint32_t q = 0; q < kAhead; ++q) now[q] = k[q];
        if (i + kAhead < end) look(i + kAhead);
#pragma unroll
        for (uint32_t q = 0; q < kAhead; ++q) {
            if (i + q >= end) continue;
            if (now[q] != key) {
                if (open) keep(part);
                else finish_row<OUT>(a, key, columns, sum);
                key = now[q];
                open = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
            }
            if (key < a.vocab) v[q].add_to(sum);
        }
        if (key >= a.vocab) return;   // (nothing but such follows)
    }
    if (open) keep(part);
    else if (end < a.count && s.keys[end] == key) keep(part + (uint64_t)s.pieces * s.pitch);
    else finish_row<OUT>(a, key, columns, sum);
}

// Runs that cross a border: the piece in which one begins adds what the others have of it, in their order.
template <bool OUT>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(EmbedArgs a, SumArgs s) {
    const uint64_t group = ((uint64_t)blockIdx.x * kThreads + threadIdx.x) / s.lanes;
    const uint32_t p = (uint32_t)(group / s.slices), slice = (uint32_t)(group % s.slices);
    const uint32_t chunk = slice * s.lanes + threadIdx.x % s.lanes;
    if (p + 1u >= s.pieces || chunk * 8u >= a.dim) return;
    const Columns columns(chunk, a.dim);
    const uint32_t d = columns.d;
    const uint32_t begin = p * s.piece, end = begin + s.piece, key = s.keys[end - 1u];
    const uint32_t after = s.keys[end], first_key = s.keys[begin], before = s.keys[begin != 0u ? begin - 1u : 0u];
    if (key >= a.vocab || after != key) return;                            // nothing goes on
    if (first_key == key && begin != 0u && before == key) return;          // it has begun before
    float sum[8] = {};
    Row8<false> mine;   // (added to zeros, as no part is -0: loaded in place the sum is waited for in every branch below, 13 us instead of 7)
    mine.load(s.parts + ((uint64_t)s.pieces + p) * s.pitch + d);
    mine.add_to(sum);
    // pieces that begin with the run, 16 at a time; their parts are loaded where there are such pieces (most runs end in the next one)
    constexpr uint32_t kAhead = 16;
    uint32_t first[kAhead];
    auto look = [&](uint32_t q) {
#pragma unroll
        for (uint32_t r = 0; r < kAhead; ++r) first[r] = s.keys[(q + r < s.pieces ? q + r : s.pieces - 1u) * s.piece];
    };
    look(p + 1u);
    bool more = true;
    for (uint32_t q = p + 1u; more && q < s.pieces; q += kAhead) {
        Row8<false> v[kAhead];
        bool in[kAhead];
#pragma unroll
        for (uint32_t r = 0; r < kAhead; ++r) {
            more = more && q + r < s.pieces && first[r] == key;
            in[r] = more;
            if (more) v[r].load(s.parts + (uint64_t)(q + r) * s.pitch + d);
        }
        if (more) look(q + kAhead);
#pragma unroll
        for (uint32_t r = 0; r < kAhead; ++r)
            if (in[r]) v[r].add_to(sum);
    }
    finish_row<OUT>(a, key, columns, sum);
}

// No tokens at all: zeros.
template <bool OUT>
__global__ __launch_bounds__(kThreads) void embed_zero_kernel(EmbedArgs a) {
    zero_rows<OUT>(a, 0u, a.vocab, blockIdx.x, gridDim.x);
}

constexpr uint32_t kZeroGroups = 1024;   // workgroups that write zeros beside others

uint32_t grid_for(uint64_t threads) {
    const uint64_t blocks = (threads + kThreads - 1u) / kThreads;
    return (uint32_t)(blocks < (1u << 20) ? blocks : (1u << 20));
}

// How the gradient's tokens are sorted and cut, by the sizes alone.
struct EmbedPlan {
    uint32_t key_bits, passes, bits, tile, tiles;   // of the sort
    uint32_t piece, pieces, lanes, slices;          // of the sums
    uint64_t pitch;
    uint64_t list, counts, parts;                   // words: of one sorted array, of the counts, of the parts
};
EmbedPlan plan_for(uint64_t count, uint64_t vocab, uint64_t dim) {
    EmbedPlan p{};
    while (vocab >> p.key_bits) ++p.key_bits;       // keys are 0 .. vocab
    p.passes = (p.key_bits + 10u) / 11u;
    p.bits = (p.key_bits + p.passes - 1u) / p.passes;
    // a tile for each workgroup, 256 keys (one look at 64 keys for each of its waves) or, from 2^16 tokens on, as many as make 256
    // tiles
    const uint64_t share = (count + 255u) / 256u;
    p.tile = (uint32_t)((share + 255u) / 256u * 256u);
    p.tiles = (uint32_t)((count + p.tile - 1u) / p.tile);
    // pieces of 16 entries or, from 2^15 tokens on, as many as make 2048 pieces: a run that crosses all of them is added by one group
    const uint64_t entries = (count + 2047u) / 2048u;
    p.piece = (uint32_t)(entries < 16u ? 16u : entries);
    p.pieces = (uint32_t)((count + p.piece - 1u) / p.piece);
    const uint64_t chunks = (dim + 7u) / 8u;
    p.lanes = 1u;
    while (p.lanes < 64u && p.lanes < chunks) p.lanes *= 2u;
    p.slices = (uint32_t)((chunks + p.lanes - 1u) / p.lanes);
    p.pitch = 8u * chunks;
    p.list = (count + 3u) / 4u * 4u;
    p.counts = count > kFew ? (uint64_t)p.tiles << p.bits : 0u;
    p.parts = 2u * p.pieces * p.pitch;
    return p;
}

}  // namespace

hipError_t launch_embed_forward(const EmbedArgs& a, hipStream_t stream) {
    const uint32_t pieces = (a.dim + 7u) / 8u, grid = grid_for((uint64_t)a.count * pieces);
    auto go = [&](auto I, auto O) {
        embed_forward_kernel<decltype(I)::value, decltype(O)::value><<<grid, kThreads, 0, stream>>>(a, pieces);
    };
    auto out = [&](auto I) { a.out_bf16 ? go(I, std::true_type{}) : go(I, std::false_type{}); };
    a.in_bf16 ? out(std::true_type{}) : out(std::false_type{});
    return hipGetLastError();
}

uint64_t embed_backward_workspace_bytes(uint64_t count, uint64_t vocab, uint64_t dim) {
    if (count == 0 || vocab == 0 || dim == 0) return 0;
    const EmbedPlan p = plan_for(count, vocab, dim);
    return 4u * (4u * p.list + (p.counts + 3u) / 4u * 4u + p.parts);
}

hipError_t launch_embed_backward(const EmbedArgs& a, hipStream_t stream) {
    if (a.count == 0u) {
        if (a.out_bf16) embed_zero_kernel<true><<<kZeroGroups, kThreads, 0, stream>>>(a);
        else embed_zero_kernel<false><<<kZeroGroups, kThreads, 0, stream>>>(a);
        return hipGetLastError();
    }
    const EmbedPlan p = plan_for(a.count, a.vocab, a.dim);
    uint32_t* list[4];
    for (int i = 0; i < 4; ++i) list[i] = a.workspace + i * p.list;
    uint32_t* counts = a.workspace + 4u * p.list;
    SumArgs s{};
    s.parts = reinterpret_cast<float*>(counts + (p.counts + 3u) / 4u * 4u);
    s.pitch = p.pitch;
    s.piece = p.piece;
    s.pieces = p.pieces;
    s.lanes = p.lanes;
    s.slices = p.slices;
    // Far fewer tokens than rows: the sorting launches, which leave most of the device idle, zero three quarters of the table beside it
    // (rows that get a gradient are written twice).  Of the rest, or of the whole table otherwise, the summing launch zeroes the rows
    // that get none.  (All beside the sort, three quarters and half: 4096 tokens, 50257 x 768 43, 40 and 47 us; 16384, 50257 x 2048
    // 133, 126 and 127 us; 300, 50257 x 1024 53, 47 and 48 us; 2048, 30522 x 768 in bf16 26, 27 and 28 us.)
    const bool zero_first = !a.accumulate && a.count < a.vocab / 2u;
    const uint32_t launches = a.count <= kFew ? 1u : 2u * p.passes, zeroers = zero_first ? kZeroGroups : 0u;
    s.zero_from = zero_first ? (uint32_t)((uint64_t)a.vocab * 3u / 4u) : 0u;
    auto share = [&](uint32_t launch) {
        return ZeroShare{(uint32_t)((uint64_t)s.zero_from * launch / launches), (uint32_t)((uint64_t)s.zero_from * (launch + 1u) / launches)};
    };
    if (a.count <= kFew) {
        const uint32_t sorters = (a.count + kFewEntries - 1u) / kFewEntries;
        sort_few_kernel<<<sorters + zeroers, kFewThreads, 0, stream>>>(a, list[0], list[1], sorters, share(0));
        s.keys = list[0];
        s.places = list[1];
    } else {
        for (uint32_t pass = 0; pass < p.passes; ++pass) {
            SortPass sort{};
            sort.keys = pass ? list[2u * ((pass - 1u) & 1u)] : nullptr;
            sort.places = pass ? list[2u * ((pass - 1u) & 1u) + 1u] : nullptr;
            sort.keys_out = list[2u * (pass & 1u)];
            sort.places_out = list[2u * (pass & 1u) + 1u];
            sort.counts = counts;
            sort.tile = p.tile;
            sort.shift = pass * p.bits;
            sort.bits = p.bits;
            sort.tiles = p.tiles;
            sort_count_kernel<<<p.tiles + zeroers, kThreads, 4u << p.bits, stream>>>(a, sort, share(2u * pass));
            sort_scatter_kernel<<<p.tiles + zeroers, kThreads, 24u << p.bits, stream>>>(a, sort, share(2u * pass + 1u));
            s.keys = sort.keys_out;
            s.places = sort.places_out;
        }
    }
    const uint64_t groups = (uint64_t)p.pieces * p.slices * p.lanes;
    s.sum_groups = (uint32_t)((groups + kThreads - 1u) / kThreads);
    const uint32_t zero_rows = (a.vocab - s.zero_from + kZeroRows - 1u) / kZeroRows;
    const uint32_t zero_groups = a.accumulate ? 0u : zero_rows < (1u << 20) ? zero_rows : 1u << 20;
    auto out = [&](auto O) {
        constexpr bool OUT = decltype(O)::value;
        if (a.in_bf16) embed_sum_kernel<true, OUT><<<s.sum_groups + zero_groups, kThreads, 0, stream>>>(a, s);
        else embed_sum_kernel<false, OUT><<<s.sum_groups + zero_groups, kThreads, 0, stream>>>(a, s);
        if (p.pieces > 1u) embed_join_kernel<OUT><<<s.sum_groups, kThreads, 0, stream>>>(a, s);
    };
    a.out_bf16 ? out(std::true_type{}) : out(std::false_type{});
    return hipGetLastError();
}

}  // namespace thc
