// Adapters of many requests beside one shared layer: every token t names its adapter i = ids[t], or none.
//
//   out[t] = base[t] + (x[t] A_i) B_i        A_i [K, r_i], B_i [r_i, N]
//   dx[t] = dx_base[t] + (dy[t] B_i^T) A_i^T,   dA_i = sum over i's tokens of x[t]^T (dy[t] B_i^T),   dB_i = sum of (x[t] A_i)^T dy[t]
//
// Tokens of one adapter are brought together into tiles, whose rows are read and written where they are: nothing is copied.
//   up to kDirectTokens tokens   a workgroup is a token, finds its fellows among the ids by comparisons across the wave, and goes on if
//                                it is the first of a tile of 16
//   few of them                  see few_tokens_kernel: all of it in one launch
//   more                         a launch in front orders the tokens by adapter (stable: sums over tokens have an order) and writes a table of tiles of 64
// Then  narrow_tile    t = in * factor (K or N columns down to r; fp32 sums over slices of the columns),
//       wide_tile      out = base + t * factor (r up to N or K columns),
//       outer_tile     the adapters' gradients, sums over tokens; beside wide_tile for dx in one launch.
// t goes into the second product as two bf16 values, t rounded and what is left of it: 16 bits of mantissa, so that results are as good as their own
// rounding (with t rounded once, as the layer does, errors were 1.4 times that).  In wide_tile the second value is free: an instruction
// that takes eight values a lane has room for four ranks of both.  (few_tokens_kernel keeps t in fp32, on the vector units.)
// All others on the matrix cores, though memory bounds each (2 r products a byte of x and out at most): tiles of 16 fill them however few rows are live, and
// what an adapter's factors lack in alignment or length is zeros in LDS.  Results do not depend on which other tokens a call holds, save that
// which of these forms it takes, and the number of slices, follow from its sizes.
#include <type_traits>

#include "salr_adapter_t.hpp"
#include "salr_eight.hpp"
#include "salr_internal.hpp"

namespace salr {

namespace {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef u32x2_t AnyUint2 __attribute__((aligned(2)));

// LDS of one wave alone: what was written is read by its other lanes, what was read may be written again.  (Its accesses are done in order;
// this keeps the compiler to it.)
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Whole waves.  128 tokens without an ordering launch against with one, 4096 x 14336 rank 16 of 32 adapters 18.8 us against 23.4, rank 64 of 64 adapters 44
// against 68, rank 64 of one 23.8 against 25.8; 256 tokens 30.5 against 24.7 (32 adapters) and 30.8 against 25.8 (one of rank 64).
constexpr int kDirectTokens = 128;
constexpr int kTileTokens = 64;   // of a launch that orders tokens

struct Tokens {   // how a kernel finds its rows
    const salr_adapter_t* list;
    const int32_t* ids;
    const int32_t* order;    // tokens by group: adapters, then those without one, then those whose id is none
    const int32_t* starts;   // [n + 2]
    const int32_t* counts;   // [n + 2]
    const int4* tiles;       // group (-1: none), live rows, place of the first in `order`, 0
    int T, n;
};

// Groups n and n + 1: no adapter; an id out of range.
__device__ __forceinline__ int group_of(int id, int n) { return id < 0 ? n : id < n ? id : n + 1; }

struct Tile {
    int group;   // -1: none left
    int count;   // live rows
    int first;   // of an ordered launch: position of the first
};

// What is the same for the wave and does not change while a kernel runs comes through the scalar cache: a trip for a table's entry or an adapter's record
// is what a workgroup's start consists of, and there it is half as long.
template <typename T>
__device__ __forceinline__ T scalar_load(const T* p) {
    typedef const T __attribute__((address_space(4))) * Constant;
    return *(Constant)(uintptr_t)p;
}
struct Adapter {
    const uint16_t *a, *b;
    int rank, pitch;   // never more ranks than the call names, whatever the record says; elements of a row of A: the record's
};
__device__ __forceinline__ Adapter adapter_of(const Tokens& k, int group, int max_rank) {
    const salr_adapter_t* record = k.list + group;
    const int64_t rank = scalar_load(&record->rank);
    return Adapter{scalar_load(&record->a), scalar_load(&record->b), rank < max_rank ? (int)rank : max_rank, (int)rank};
}

// Tile `self`; of a direct launch also its tokens in rows[kRows] (LDS, a barrier behind it).
template <bool kDirect, int kRows>
__device__ __forceinline__ Tile find_tile(const Tokens& k, int self, int* rows) {
    Tile tile{-1, 0, 0};
    if constexpr (kDirect) {
        constexpr int kChunks = kDirectTokens / kWave;
        const int lane = lane_id(), mine = group_of(scalar_load(k.ids + self), k.n);
        bool same[kChunks];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) same[c] = kWave * c + lane < k.T && group_of(k.ids[kWave * c + lane], k.n) == mine;
        int before = 0, all = 0, place[kChunks];   // fellows before this one, all of them, and before each
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const uint64_t mask = __ballot(same[c]);
            place[c] = all + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));   // fellows on the lanes before this one
            if (self >= kWave * (c + 1)) before += __popcll(mask);
            else if (self >= kWave * c) before += __popcll(mask & (((uint64_t)1 << (self - kWave * c)) - 1));
            all += __popcll(mask);
        }
        if (before % kRows != 0) return tile;   // the same for the workgroup
        tile.group = mine;
        tile.count = all - before < kRows ? all - before : kRows;
        if (threadIdx.x < kWave)
#pragma unroll
            for (int c = 0; c < kChunks; ++c)
                if (same[c] && place[c] >= before && place[c] < before + kRows) rows[place[c] - before] = kWave * c + lane;
        __syncthreads();
    } else {
        const AlignedUint4 t = scalar_load(reinterpret_cast<const AlignedUint4*>(k.tiles + self));
        tile = Tile{(int)t[0], (int)t[1], (int)t[2]};
    }
    return tile;
}

// Row j's token (j < count), and its place in the sums of a tile.
template <bool kDirect>
__device__ __forceinline__ int token_of(const Tokens& k, const Tile& tile, const int* rows, int j) {
    return kDirect ? rows[j] : k.order[tile.first + j];
}
template <bool kDirect>
__device__ __forceinline__ int64_t place_of(const Tile& tile, const int* rows, int j) {
    return kDirect ? rows[j] : tile.first + j;
}

// Sixteen bytes at any element's address of global memory.  (Said to the compiler: a pointer out of a record could point anywhere, and loads through
// such pointers are waited for together with LDS'.)
__device__ __forceinline__ uint4 load16(const uint16_t* p) {
    typedef const AnyUint4 __attribute__((address_space(1))) * Global;
    return __builtin_bit_cast(uint4, *(Global)(uintptr_t)p);
}

// The eight values `by` places on, zeros behind the first `left` of them.  (In 32-bit words: with 64-bit shifts one wave of a kernel that was
// being written here had NaN for its values.  Why was not shown; what was seen is that the shift's amount lay in the last vector register of that kernel.)
__device__ __forceinline__ uint4 from_place(uint4 q, int by, int left) {
    if (!__any(by > 0 || left < 8)) return q;   // (a wave in the middle of a row has nothing to do)
    const auto choose = [](bool there, uint32_t a, uint32_t b) { return there ? a : b; };
    uint32_t a = choose(by & 4, q.z, q.x), b = choose(by & 4, q.w, q.y), c = choose(by & 4, 0, q.z), d = choose(by & 4, 0, q.w);
    a = choose(by & 2, b, a), b = choose(by & 2, c, b), c = choose(by & 2, d, c), d = choose(by & 2, 0, d);
    a = choose(by & 1, a >> 16 | b << 16, a), b = choose(by & 1, b >> 16 | c << 16, b), c = choose(by & 1, c >> 16 | d << 16, c), d = choose(by & 1, d >> 16, d);
    const auto cut = [&](uint32_t v, int from) { return left >= from + 2 ? v : left > from ? v & 0xFFFFu : 0u; };
    return make_uint4(cut(a, 0), cut(b, 2), cut(c, 4), cut(d, 6));
}

// Columns c .. c + 7 of the row of C >= 8 that starts at element `start` of a matrix of `total`, in two steps, so that nothing waits for a request until it
// is used: raw_eight asks for them, in one request without a branch (kWhole, C % 8 == 0: at the row's last vector where c is past it; else pulled back
// from the matrix' end where it would leave it), and true_eight makes of what came the row's values, and zeros behind them, wherever c is.
template <bool kWhole>
__device__ __forceinline__ uint4 raw_eight(const uint16_t* m, int64_t start, int c, int C, int64_t total) {
    if constexpr (kWhole) {
        return load16(m + start + (c < C ? c : C - 8));
    } else {
        const int64_t at = start + (c < C ? c : C - 1);
        return load16(m + (at < total - 8 ? at : total - 8));
    }
}
template <bool kWhole>
__device__ __forceinline__ uint4 true_eight(uint4 q, int64_t start, int c, int C, int64_t total) {
    if constexpr (kWhole) {
        return c < C ? q : make_uint4(0, 0, 0, 0);
    } else {
        const int64_t at = start + (c < C ? c : C - 1), past = at - (total - 8);
        return from_place(q, past > 0 ? (int)past : 0, C - c);
    }
}

// Ranks r .. r + 7 of a row of a factor A [C, pitch], likewise; behind the last rank whatever comes, but nothing from behind the matrix.
__device__ __forceinline__ uint4 raw_ranks(const uint16_t* m, int64_t row, int r, int pitch, int64_t total) {
    const int64_t at = row * pitch + r;
    return load16(m + (at < total - 8 ? at : total - 8));
}
__device__ __forceinline__ uint4 true_ranks(uint4 q, int64_t row, int r, int pitch, int64_t total) {
    if ((pitch & 7) == 0) return q;   // (whole vectors are pulled back only where r >= pitch)
    const int64_t past = row * pitch + r - (total - 8);
    return from_place(q, past > 0 ? past < 8 ? (int)past : 7 : 0, 8);
}

// Four values as bf16 and what that leaves of them, as bf16 too.
__device__ __forceinline__ uint4 two_halves(f32x4 v) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        hi[e] = f32_to_bf16_rne(v[e]);
        const float rest = v[e] - bf16_bits_to_f32(hi[e]);
        lo[e] = fabsf(rest) <= fabsf(v[e]) ? f32_to_bf16_rne(rest) : 0u;   // (infinite or NaN: all of it is in the first)
    }
    return make_uint4(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16, lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
}

}  // namespace

// A workgroup a group: counts the tokens of the groups before its own, then puts its own in order.  Every group goes through all ids, which
// stay in the caches; no workgroup waits for another.  A thread takes eight ids side by side, so that up to 8192 tokens are read once.
// Group g, whose tokens start at place s, has the entries s / 64 + g and on of the table of tiles, up to the next group's, which are enough for its tiles
// whatever s: so nobody has to know how many tiles the groups before have.  What is left over is marked as empty.
constexpr int kOrderEach = 8;
__global__ __launch_bounds__(1024) void order_tokens_kernel(const int32_t* ids, int T, int n, int32_t* order, int32_t* starts, int32_t* counts, int4* tiles,
                                                            int chunk, int4* chunks) {
    __shared__ uint32_t scratch[17];
    __shared__ int total[2][16];
    const int group = blockIdx.x, wave = threadIdx.x >> 6;
    int less = 0, same = 0;
    uint32_t mine = 0;   // of the ids looked at last
    const auto look = [&](int64_t t0) {
        mine = 0;
        int g[kOrderEach];
        typedef int Four __attribute__((ext_vector_type(4), aligned(4)));
        const int64_t t = t0 + kOrderEach * threadIdx.x;
        if (t + kOrderEach <= T) {
            const Four lo = reinterpret_cast<const Four*>(ids + t)[0], hi = reinterpret_cast<const Four*>(ids + t)[1];
#pragma unroll
            for (int j = 0; j < kOrderEach; ++j) g[j] = group_of(j < 4 ? lo[j] : hi[j - 4], n);
        } else {
#pragma unroll
            for (int j = 0; j < kOrderEach; ++j) g[j] = t + j < T ? group_of(ids[t + j], n) : 2147483647;
        }
#pragma unroll
        for (int j = 0; j < kOrderEach; ++j) {
            less += g[j] < group;
            mine |= (uint32_t)(g[j] == group) << j;
        }
        same += __popc(mine);
    };
    for (int64_t t0 = 0; t0 < T; t0 += 1024 * kOrderEach) look(t0);
    less = (int)last_lane(wave_inclusive_scan((uint32_t)less));
    same = (int)last_lane(wave_inclusive_scan((uint32_t)same));
    if (lane_id() == 0) {
        total[0][wave] = less;
        total[1][wave] = same;
    }
    __syncthreads();
    int at = 0, count = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        at += total[0][w];
        count += total[1][w];
    }
    if (threadIdx.x == 0) {
        starts[group] = at;
        counts[group] = count;
    }
    const int entry = at / kTileTokens + group, entries = (at + count) / kTileTokens + group + 1 - entry;
    for (int i = threadIdx.x; i < entries; i += 1024) {
        const int left = count - kTileTokens * i;
        tiles[entry + i] = make_int4(left > 0 ? group : -1, left < kTileTokens ? left : kTileTokens, at + kTileTokens * i, 0);
    }
    if (chunks != nullptr) {   // the table of chunks, likewise: an adapter's first entry is there even without a token, for its gradients' zeros
        const int first = at / chunk + group, last = (at + count) / chunk + group;
        for (int i = threadIdx.x; first + i <= last; i += 1024) {
            const int left = count - chunk * i;
            chunks[first + i] = make_int4(group < n && (i == 0 || left > 0) ? group : -1, at + chunk * i, left < 0 ? 0 : left < chunk ? left : chunk,
                                          count > chunk ? 2 * (at / chunk) + i : -1);
        }
    }
    if (count == 0) return;
    for (int64_t t0 = 0; t0 < T; t0 += 1024 * kOrderEach) {
        if (T > 1024 * kOrderEach) look(t0);
        uint32_t here;
        uint32_t place = at + block_exclusive_scan<1024>(__popc(mine), scratch, here);
        for (uint32_t left = mine; left != 0; left &= left - 1) order[place++] = (int32_t)(t0 + kOrderEach * threadIdx.x + __builtin_ctz(left));
        at += (int)here;
    }
}

struct NarrowArgs {
    Tokens tokens;
    const uint16_t* in[2];    // x with A; dy with B
    int64_t C[2];
    float* part[2];           // [slices][t_rows][rpad]
    int slices[2];
    int64_t t_rows;
    int rpad, max_rank;
};

// part[z][row][r] = sum over the columns c of slice z of in[row][c] * factor(c, r).  A workgroup has a slice of a tile: every `slices`-th step of 128
// columns, so that the workgroups of a tile read side by side.  Rows of in and the factor's part come in by whole lines, four rows of 256 bytes a request, and
// through LDS: as MFMA operands straight from memory, 16 rows of 64 bytes a request, 4096 tokens of 4096 and 14336 columns at rank 32 took 51 us
// instead of 42, and three times the registers.  The requests of two steps are out while one is multiplied.  16x16x32 MFMAs with in as A operand; A's
// [128 columns, ranks], which lie the wrong way round, are read transposed.  Tiles of 64 rows: a wave has 16 of them; of 16 rows: each has 32 columns of a
// step, and their sums meet in LDS, in order.  16 kRT ranks a pass.
// Memory bounds the large case (40 us for 151 MB of x and dy that no cache has, 48 MB of factors past L2; without multiplying 39.7, without the factors 37.5;
// one or four workgroups a CU, half or twice as many slices, tiles or slices side by side: all within 2 us), trips to memory the small ones
// (64 tokens of 40 adapters 6.1 us, one token 3.5).
template <int kMB, int kRT>
struct NarrowLds {
    static constexpr int kCols = 128, kPitch = kCols + 8, kRankPitch = 16 * kRT + 8, kSumPitch = 16 * kRT + 4;
    static constexpr int kIn = 16 * kMB * kPitch, kFactor = 16 * kRT * kPitch > kCols * kRankPitch ? 16 * kRT * kPitch : kCols * kRankPitch;
    static constexpr int kSums = kMB == 1 ? 4 * 16 * kSumPitch : 1;
    uint16_t in[kIn], factor[kFactor];
    float sums[kSums];
    int rows[16 * kMB];
};

template <bool kDirect, int kMB, int kRT, bool kWhole, bool second>   // second: dy with B
__device__ __forceinline__ void narrow_tile(const NarrowArgs& a, const Tile& tile, int z, NarrowLds<kMB, kRT>& lds) {
    typedef NarrowLds<kMB, kRT> Lds;
    constexpr int kPitch = Lds::kPitch, kRankPitch = Lds::kRankPitch, kSumPitch = Lds::kSumPitch, kParts = kMB == 1 ? 1 : 4;
    static_assert(kMB == 1 || kMB == 4, "a block of rows for each wave, or one for all");
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, g = lane >> 4;
    const int slices = second ? a.slices[1] : a.slices[0];
    const uint16_t* in = second ? a.in[1] : a.in[0];
    const int C = (int)(second ? a.C[1] : a.C[0]);
    const int64_t in_total = (int64_t)a.tokens.T * C;
    float* part = (second ? a.part[1] : a.part[0]) + (int64_t)z * a.t_rows * a.rpad;
    const Adapter adapter = adapter_of(a.tokens, tile.group, a.max_rank);
    const int rank = adapter.rank, pitch = adapter.pitch;
    const uint16_t* factor = second ? adapter.b : adapter.a;
    const int64_t factor_total = (int64_t)(second ? rank : pitch) * C;
    const int steps = (C + Lds::kCols - 1) / Lds::kCols;
    const int vrow = threadIdx.x >> 4, vcol = 8 * (threadIdx.x & 15);
    int64_t row[kMB];   // (behind the last token the first one's: what comes of it is not stored)
#pragma unroll
    for (int i = 0; i < kMB; ++i) row[i] = (int64_t)token_of<kDirect>(a.tokens, tile, lds.rows, 16 * i + vrow < tile.count ? 16 * i + vrow : 0) * C;
    for (int rb = 0; rb < rank; rb += 16 * kRT) {
        const int rts = (rank - rb + 15) / 16 < kRT ? (rank - rb + 15) / 16 : kRT;
        f32x4 acc[kRT] = {};
        struct Step {
            uint4 x[kMB], f[kRT];
        } ahead[2];
        const auto request = [&](Step& q, int s) {
            const int c = Lds::kCols * s;
#pragma unroll
            for (int i = 0; i < kMB; ++i) q.x[i] = raw_eight<kWhole>(in, row[i], c + vcol, C, in_total);
#pragma unroll
            for (int i = 0; i < kRT; ++i) {
                if constexpr (second) {   // (behind the last rank its values again: what comes of them is dropped)
                    const int r = rb + 16 * i + vrow;
                    q.f[i] = raw_eight<kWhole>(factor, (int64_t)(r < rank ? r : rank - 1) * C, c + vcol, C, factor_total);
                } else {                  // vector v of [128][16 kRT]
                    const int v = threadIdx.x + 256 * i, k = c + v / (2 * kRT);
                    q.f[i] = raw_ranks(factor, k < C ? k : C - 1, rb + 8 * (v % (2 * kRT)), pitch, factor_total);
                }
            }
        };
        const auto step = [&](Step& q, int s) {
            const int c = Lds::kCols * s;
            if (s > z) __syncthreads();   // the step before has been multiplied by every wave
#pragma unroll
            for (int i = 0; i < kMB; ++i) *reinterpret_cast<uint4*>(lds.in + (16 * i + vrow) * kPitch + vcol) = true_eight<kWhole>(q.x[i], row[i], c + vcol, C, in_total);
#pragma unroll
            for (int i = 0; i < kRT; ++i) {
                if constexpr (second) {
                    const int r = rb + 16 * i + vrow;
                    *reinterpret_cast<uint4*>(lds.factor + (16 * i + vrow) * kPitch + vcol) =
                        true_eight<kWhole>(q.f[i], (int64_t)(r < rank ? r : rank - 1) * C, c + vcol, C, factor_total);
                } else {
                    const int v = threadIdx.x + 256 * i, k = c + v / (2 * kRT);
                    const uint4 f = true_ranks(q.f[i], k < C ? k : C - 1, rb + 8 * (v % (2 * kRT)), pitch, factor_total);
                    *reinterpret_cast<uint4*>(lds.factor + v / (2 * kRT) * kRankPitch + 8 * (v % (2 * kRT))) = k < C ? f : make_uint4(0, 0, 0, 0);
                }
            }
            if (s + 2 * slices < steps) request(q, s + 2 * slices);
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kParts; ++u) {
                const int block = kMB == 1 ? 0 : wave, col = 32 * (kMB == 1 ? wave : u);
                const bf16x8 x = as_bf16x8(*reinterpret_cast<const uint4*>(lds.in + (16 * block + i16) * kPitch + col + 8 * g));
#pragma unroll
                for (int rt = 0; rt < kRT; ++rt) {
                    if (rt >= rts) continue;
                    uint4 f;
                    if constexpr (second) {
                        f = *reinterpret_cast<const uint4*>(lds.factor + (16 * rt + i16) * kPitch + col + 8 * g);
                    } else {
                        const uint16_t* from = lds.factor + (col + 8 * g + (i16 >> 2)) * kRankPitch + 16 * rt + 4 * (i16 & 3);
                        const uint2 lo = lds_read_tr4(from), hi = lds_read_tr4(from + 4 * kRankPitch);
                        f = make_uint4(lo.x, lo.y, hi.x, hi.y);
                    }
                    acc[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, as_bf16x8(f), acc[rt], 0, 0, 0);
                }
            }
        };
        if (z < steps) request(ahead[0], z);
        if (z + slices < steps) request(ahead[1], z + slices);
        for (int s = z; s < steps; s += 2 * slices) {
            step(ahead[0], s);
            if (s + slices < steps) step(ahead[1], s + slices);
        }
        // accumulators: lane holds column i16 (rank), rows 4 g + e (tokens).  Zeros behind the last rank (zero times an infinity of in is none).
        if constexpr (kMB == 1) {
#pragma unroll
            for (int rt = 0; rt < kRT; ++rt)
#pragma unroll
                for (int e = 0; e < 4; ++e) lds.sums[(16 * wave + 4 * g + e) * kSumPitch + 16 * rt + i16] = acc[rt][e];
            __syncthreads();
            for (int i = threadIdx.x; i < tile.count * rts * 4; i += 256) {
                const int j = i / (rts * 4), c = 4 * (i % (rts * 4));
                f32x4 v = *reinterpret_cast<const f32x4*>(lds.sums + j * kSumPitch + c);
#pragma unroll
                for (int w = 1; w < 4; ++w) v += *reinterpret_cast<const f32x4*>(lds.sums + (16 * w + j) * kSumPitch + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = rb + c + e < rank ? v[e] : 0.f;
                *reinterpret_cast<f32x4*>(part + place_of<kDirect>(tile, lds.rows, j) * a.rpad + rb + c) = v;
            }
        } else {
#pragma unroll
            for (int rt = 0; rt < kRT; ++rt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = 16 * wave + 4 * g + e, r = rb + 16 * rt + i16;
                    if (rt < rts && j < tile.count) part[place_of<kDirect>(tile, lds.rows, j) * a.rpad + r] = r < rank ? acc[rt][e] : 0.f;
                }
        }
        __syncthreads();   // before the next pass
    }
}

template <bool kDirect, int kMB, int kRT, bool kWhole>
__global__ __launch_bounds__(256, kRT < 4 ? 4 : 3) void narrow_kernel(NarrowArgs a) {
    __shared__ __align__(16) NarrowLds<kMB, kRT> lds;
    // slices side by side, then tiles: workgroups that run at a time read whole rows between them
    const int slices = a.slices[0] + a.slices[1], slice = blockIdx.x % slices;
    const Tile tile = find_tile<kDirect, 16 * kMB>(a.tokens, blockIdx.x / slices, lds.rows);
    if (tile.group < 0 || tile.group >= a.tokens.n) return;
    if constexpr (kDirect) narrow_tile<kDirect, kMB, kRT, kWhole, false>(a, tile, slice, lds);
    else if (slice < a.slices[0]) narrow_tile<kDirect, kMB, kRT, kWhole, false>(a, tile, slice, lds);
    else narrow_tile<kDirect, kMB, kRT, kWhole, true>(a, tile, slice - a.slices[0], lds);
}

// t = the sum over the slices of part, four values a thread, as two_halves has them; y picks the product.
struct SumArgs {
    const float* part[2];
    uint4* t[2];
    int slices[2];
    int64_t count;   // of a slice
};
__global__ __launch_bounds__(256) void sum_slices_kernel(SumArgs a) {
    const bool second = blockIdx.y == 1;
    const float* part = second ? a.part[1] : a.part[0];
    const int slices = second ? a.slices[1] : a.slices[0];
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (4 * i >= a.count) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int z = 0; z < slices; ++z) s += *reinterpret_cast<const f32x4*>(part + z * a.count + 4 * i);
    (second ? a.t[1] : a.t[0])[i] = two_halves(s);
}

struct WideArgs {
    Tokens tokens;
    const float* part;      // [slices][t_rows][rpad], summed here; or, slices 0,
    const uint4* t;         // [t_rows][rpad / 4], as two_halves has them
    int slices;
    int64_t t_rows;
    int rpad, max_rank;
    int64_t C;              // columns of out
    int per_group;          // of a workgroup, whole steps of its waves
    const uint16_t* base;   // may be out, or null (zeros)
    uint16_t* out;
};

// out[row][c] = base[row][c] + sum over r of t[row][r] * factor(r, c).  A workgroup has some columns of a tile: t's rows once into LDS, then each wave takes 64
// columns at a time, the factor's part of them, zeros where ranks or columns end, through LDS of its own (kPass ranks a pass), the next one's on their
// way meanwhile.  The product is formed transposed, columns of out as rows of 16x16x32 MFMAs, and which column a row stands for is chosen so that a
// lane ends up with twice eight columns of one token side by side and four lanes with 64 bytes (row m of tile j is column 32 (j / 2) + 8 (m / 4)
// + 4 (j % 2) + m % 4): out is read and written in whole vectors.  An instruction takes 16 ranks: four of a lane with t's first half and the same four with its second.
// kFactorA: the factor is A [C, r] (dx), else B [r, C] (y).
// kRows: of a tile; of 64, two waves have one half each.
// The start is four trips to memory one behind the other (the tile, its tokens and the adapter's record, t, base and factor), and with the stores that is what
// bounds all but the largest calls: 64 tokens of 40 adapters, 4096 -> 14336, 10.5 us (26 MB); 2001 tokens, 2720 -> 2731, 13 us, 11 with N = 2736.  Three of
// them follow from each other; base and factor are only asked for behind the sum of t, on which they do not depend.
template <int kRows, int kMostR, bool kFactorA>
struct WideLds {
    static constexpr int kTPitch = 2 * kMostR + 8, kPass = 32, kPitch = kFactorA ? kPass + 8 : 64 + 8, kOutPitch = 64 + 8;
    static constexpr int kMB = kRows / 16 < 2 ? 1 : 2, kStage = (kFactorA ? 64 : kPass) * kPitch;   // kMB: blocks of rows of a wave
    static_assert(16 * kMB * kOutPitch <= kStage, "out goes through the factor's place");
    uint16_t t[kRows * kTPitch], stages[4][kStage];
    int rows[kRows];
};

template <bool kDirect, int kRows, int kMostR, bool kFactorA, bool kWhole>
__device__ __forceinline__ void wide_tile(const WideArgs& a, int block, WideLds<kRows, kMostR, kFactorA>& lds) {
    typedef WideLds<kRows, kMostR, kFactorA> Lds;
    constexpr int kTPitch = Lds::kTPitch, kPass = Lds::kPass, kVectors = kPass / 8, kPitch = Lds::kPitch, kOutPitch = Lds::kOutPitch;
    constexpr int kMB = Lds::kMB, kHalves = kRows / 16 / kMB, kStride = 256 / kHalves;   // columns of a workgroup's step
    int* rows = lds.rows;
    uint16_t* t = lds.t;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, g = lane >> 4;
    const int C = (int)a.C, across = (C + a.per_group - 1) / a.per_group;
    const Tile tile = find_tile<kDirect, kRows>(a.tokens, block / across, rows);
    if (tile.group < 0) return;
    const int c_begin = block % across * a.per_group, c_end = c_begin + a.per_group < C ? c_begin + a.per_group : C;
    if (tile.group >= a.tokens.n) {   // no adapter: base as it is; an id that is none: NaN
        const bool none = tile.group == a.tokens.n;
        if (none && a.base == a.out) return;
        const int width = (c_end - c_begin + 7) >> 3;
        for (int i = threadIdx.x; i < tile.count * width; i += 256) {
            const int64_t at = (int64_t)token_of<kDirect>(a.tokens, tile, rows, i / width) * C;
            const int c = c_begin + 8 * (i % width), left = c_end - c;
            Eight<false> q{{make_uint4(0, 0, 0, 0)}};
            if (none && a.base != nullptr) q = load_eight<false, false, false>(a.base + at + c, 0, left);
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = none ? q.get(j) : __uint_as_float(0x7FC00000u);
            store_eight<false, false>(a.out + at + c, 0, left, v);
        }
        return;
    }
    const Adapter adapter = adapter_of(a.tokens, tile.group, a.max_rank);
    const int rank = adapter.rank, rank16 = (rank + 15) & ~15, pitch = adapter.pitch;
    const uint16_t* factor = kFactorA ? adapter.a : adapter.b;
    const int64_t factor_total = (int64_t)(kFactorA ? pitch : rank) * C;
    uint4 q[kVectors];
    const auto request = [&](int c0, int rb) {   // the factor's part for 64 columns and kPass ranks
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
            if (!kFactorA && rb + 8 * v >= rank16) continue;   // the same for the workgroup
            if constexpr (kFactorA) {   // vectors of [64 columns][kPass ranks]
                const int i = lane + 64 * v, k = c0 + i / kVectors;
                q[v] = raw_ranks(factor, k < C ? k : C - 1, rb + 8 * (i % kVectors), pitch, factor_total);
            } else {                    // vectors of [kPass ranks][64 columns]
                const int r = rb + 8 * v + (lane >> 3);
                q[v] = raw_eight<kWhole>(factor, (int64_t)(r < rank ? r : rank - 1) * C, c0 + 8 * (lane & 7), C, factor_total);
            }
        }
    };
    const auto place = [&](uint16_t* stage, int c0, int rb) {   // what came of that into LDS, zeros behind the last rank
#pragma unroll
        for (int v = 0; v < kVectors; ++v) {
            const int i = lane + 64 * v;
            if constexpr (kFactorA) {
                const int k = c0 + i / kVectors, r = rb + 8 * (i % kVectors);
                const uint4 f = true_ranks(q[v], k < C ? k : C - 1, r, pitch, factor_total);
                *reinterpret_cast<uint4*>(stage + i / kVectors * kPitch + 8 * (i % kVectors)) = rank - r >= 8 ? f : from_place(f, 0, rank - r);
            } else {
                const int r = rb + 8 * v + (lane >> 3);
                if (rb + 8 * v >= rank16) continue;   // the same for the workgroup
                const uint4 f = true_eight<kWhole>(q[v], (int64_t)(r < rank ? r : rank - 1) * C, c0 + 8 * (lane & 7), C, factor_total);
                *reinterpret_cast<uint4*>(stage + (i >> 3) * kPitch + 8 * (i & 7)) = r < rank ? f : make_uint4(0, 0, 0, 0);
            }
        }
    };
    const int64_t out_total = (int64_t)a.tokens.T * C;
    const int first_row = wave % kHalves * 16 * kMB, vrow = lane >> 3, vcol = 8 * (lane & 7);
    int64_t row[2 * kMB];   // of the vectors of out that this lane reads and writes, eight rows apart; behind the last token -1
#pragma unroll
    for (int i = 0; i < 2 * kMB; ++i) {
        const int j = first_row + 8 * i + vrow;
        const int token = token_of<kDirect>(a.tokens, tile, rows, j < tile.count ? j : 0);
        row[i] = j < tile.count ? (int64_t)token * C : -1;
    }
    // t's live rows; what the others hold comes to nothing that is stored
    const int quads = rank16 / 4, items = tile.count * quads;
    if (kRows == 16 && a.slices > 0) {   // four lanes share a quad's slices, every fourth each, and are of one mind
        const int first = threadIdx.x & 3;
        for (int i = threadIdx.x >> 2; i < items; i += 64) {
            const int j = i / quads, r = 4 * (i % quads);
            const float* from = a.part + place_of<kDirect>(tile, rows, j) * a.rpad + r;
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int z = first; z < a.slices; z += 4) s += *reinterpret_cast<const f32x4*>(from + z * a.t_rows * a.rpad);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[e] += __shfl_xor(s[e], 1);
                s[e] += __shfl_xor(s[e], 2);
            }
            if (first == 0) *reinterpret_cast<uint4*>(t + j * kTPitch + 2 * r) = two_halves(s);
        }
    } else {
        for (int i = threadIdx.x; i < items; i += 256) {
            const int j = i / quads, r = 4 * (i % quads);
            const int64_t at = place_of<kDirect>(tile, rows, j) * a.rpad + r;
            uint4 h;
            if (a.slices > 0) {
                f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
                for (int z = 0; z < a.slices; ++z) s += *reinterpret_cast<const f32x4*>(a.part + z * a.t_rows * a.rpad + at);
                h = two_halves(s);
            } else {
                h = a.t[at >> 2];
            }
            *reinterpret_cast<uint4*>(t + j * kTPitch + 2 * r) = h;
        }
    }
    uint4 base[2 * kMB] = {};
    const auto request_base = [&](int c0) {   // (behind the last token any row: what comes of it is not stored)
        if (a.base == nullptr) return;
#pragma unroll
        for (int i = 0; i < 2 * kMB; ++i) base[i] = raw_eight<kWhole>(a.base, row[i] < 0 ? 0 : row[i], c0 + vcol, C, out_total);
    };
    int c0 = c_begin + 64 * (wave / kHalves), rb = 0;
    if (c0 < c_end) {
        request_base(c0);
        if (rank > 0) request(c0, 0);
    }
    __syncthreads();
    uint16_t* stage = lds.stages[wave];
    f32x4 acc[kMB][4];
    if (first_row >= tile.count) return;   // (no barrier follows)
    while (c0 < c_end) {
        if (rb == 0) {
#pragma unroll
            for (int mb = 0; mb < kMB; ++mb)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[mb][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int steps = (rank - rb + 15) / 16 < kPass / 16 ? (rank - rb + 15) / 16 : kPass / 16;
        if (rank > 0) place(stage, c0, rb);
        wave_sync();
        const int now = rb, c_now = c0;
        rb += kPass;
        if (rb >= rank) {
            rb = 0;
            c0 += kStride;
        }
        if (c0 < c_end && rank > 0) request(c0, rb);
#pragma unroll
        for (int st = 0; st < kPass / 16; ++st) {
            if (st < steps) {
                uint4 tq[kMB];
#pragma unroll
                for (int mb = 0; mb < kMB; ++mb) tq[mb] = *reinterpret_cast<const uint4*>(t + (first_row + 16 * mb + i16) * kTPitch + 2 * (now + 16 * st + 4 * g));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint2 f;
                    if constexpr (kFactorA) f = *reinterpret_cast<const uint2*>(stage + (32 * (j >> 1) + 8 * (i16 >> 2) + 4 * (j & 1) + (i16 & 3)) * kPitch + 16 * st + 4 * g);
                    else f = lds_read_tr4(stage + (16 * st + 4 * g + (i16 >> 2)) * kPitch + 32 * (j >> 1) + 8 * (i16 & 3) + 4 * (j & 1));
                    const bf16x8 twice = as_bf16x8(make_uint4(f.x, f.y, f.x, f.y));
#pragma unroll
                    for (int mb = 0; mb < kMB; ++mb)
                        if (16 * mb < tile.count) acc[mb][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(twice, as_bf16x8(tq[mb]), acc[mb][j], 0, 0, 0);
                }
            }
        }
        wave_sync();
        if (rb != 0) continue;
        // The accumulators hold columns 32 h + 8 g .. + 7 of row 16 mb + i16 in a lane.  base comes to them through the place of the factor in LDS, and out goes
        // back through it: to memory whole lines.  (16 rows of 64 bytes a request, as the accumulators have them, 4096 tokens of 4096 columns
        // took 23.8 us.)  base is used up before the next columns' is asked for.
#pragma unroll
        for (int i = 0; i < 2 * kMB; ++i)
            *reinterpret_cast<uint4*>(stage + (8 * i + vrow) * kOutPitch + vcol) = true_eight<kWhole>(base[i], row[i] < 0 ? 0 : row[i], c_now + vcol, C, out_total);
        wave_sync();
        if (c0 < c_end) request_base(c0);
#pragma unroll
        for (int mb = 0; mb < kMB; ++mb)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint16_t* at = stage + (16 * mb + i16) * kOutPitch + 32 * h + 8 * g;
                const Eight<false> from{{*reinterpret_cast<const uint4*>(at)}};
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = from.get(e) + acc[mb][2 * h + (e >> 2)][e & 3];
                store_eight<false>(at, 0, 8, v);
            }
        wave_sync();
#pragma unroll
        for (int i = 0; i < 2 * kMB; ++i) {
            const int c = c_now + vcol, left = C - c;
            const Eight<false> v{{*reinterpret_cast<const uint4*>(stage + (8 * i + vrow) * kOutPitch + vcol)}};
            if (row[i] < 0 || left <= 0) continue;
            if (kWhole || left >= 8) {
                *reinterpret_cast<AnyUint4*>(a.out + row[i] + c) = __builtin_bit_cast(AlignedUint4, v.q[0]);
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < left) a.out[row[i] + c + e] = (uint16_t)unit_elem(v.q[0], e);
            }
        }
        wave_sync();
    }
}

template <bool kDirect, int kRows, int kMostR, bool kWhole>
__global__ __launch_bounds__(256, kMostR > 64 && kRows > 16 ? 1 : 4) void wide_kernel(WideArgs a) {
    __shared__ __align__(16) WideLds<kRows, kMostR, false> lds;
    wide_tile<kDirect, kRows, kMostR, false, kWhole>(a, blockIdx.x, lds);
}

struct OuterArgs {
    Tokens tokens;
    const uint16_t* in[2];   // x (dA), dy (dB)
    const uint4* s[2];       // dy B^T (dA), x A (dB): [T][rpad / 4] by position, as two_halves has them
    int64_t C[2];
    int rpad, max_rank;
    int blocks0;             // of kOuterCols columns: of x
    const int4* chunks;      // adapter (-1: none), place of the first token, tokens, and where its sums go: -1 to the gradient, else one of
    float* sums;             // [slots][K rpad + rpad N]
};
constexpr int kOuterCols = 128;

// dA_i [K, r] and dB_i [r, N], sums over the adapter's tokens: workgroup (128 columns of x or dy, chunk of an adapter's tokens).  An adapter with more tokens than
// a chunk has its sums joined by the launch behind, in order; a workgroup that went through 4096 tokens, 1.4 us for each 64, would be all there is to
// wait for (one adapter of rank 64 at 4096 x 4096: 91 us).  Both operands lie with the tokens as rows and are transposed by LDS' transposing read, 32 tokens a step, kBatch steps a batch and up to two batches in flight.  Which of the two is the MFMA's
// first operand is chosen so that a lane holds four values side by side of the result.  An adapter without tokens gets zeros.
template <int kRT>
struct OuterLds {
    static constexpr int kCols = kOuterCols, kBatch = 2, kTokens = 32 * kBatch, kPitch = kCols + 8, kSPitch = 32 * kRT + 8;
    uint16_t in_tile[kTokens * kPitch];
    uint16_t s_tile[kTokens * kSPitch];
};

template <int kRT, bool kWhole, bool second>   // second: dB
__device__ __forceinline__ void outer_tile(const OuterArgs& a, int block, const AlignedUint4& chunk, uint16_t* in_tile, uint16_t* s_tile) {
    typedef OuterLds<kRT> Lds;
    constexpr int kCols = kOuterCols, kBatch = Lds::kBatch, kTokens = Lds::kTokens, kPitch = Lds::kPitch, kSPitch = Lds::kSPitch;
    constexpr int kCT = kCols / 64, kX = kTokens * kCols / 8 / 256, kS = kTokens * 4 * kRT / 256, kAcross = kCols / 8;
    // batches under way (two of rank 64 hold registers that a second workgroup would need: 4096 tokens at 4096 x 4096 39.5 us with one, 46.5 with two)
    constexpr int kDeep = kRT < 4 ? 2 : 1;
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, g = lane >> 4;
    const int group = (int)chunk[0], start = (int)chunk[1], count = (int)chunk[2], slot = (int)chunk[3];
    const salr_adapter_t* record = a.tokens.list + group;
    uint16_t* out = second ? scalar_load(&record->db) : scalar_load(&record->da);
    if (out == nullptr) return;
    const Adapter adapter = adapter_of(a.tokens, group, a.max_rank);
    const int rank = adapter.rank;
    const uint16_t* in = second ? a.in[1] : a.in[0];
    const uint4* s = (second ? a.s[1] : a.s[0]) + (int64_t)start * (a.rpad / 4);
    const int C = (int)(second ? a.C[1] : a.C[0]), c0 = kCols * (block - (second ? a.blocks0 : 0));
    const int64_t in_total = (int64_t)a.tokens.T * C;
    const int trow = threadIdx.x / kAcross, tvec = threadIdx.x % kAcross;
    for (int rb = 0; rb < rank; rb += 16 * kRT) {
        f32x4 acc[kCT][kRT] = {};
        struct Batch {
            uint4 x[kX], s[kS];
            int64_t row[kX];
        } ahead[kDeep];
        int token[kX];   // of the batch after the one requested last
        const auto find = [&](int b) {
#pragma unroll
            for (int d = 0; d < kX; ++d) {
                const int j = b + 256 / kAcross * d + trow;
                token[d] = a.tokens.order[start + (j < count ? j : count - 1)];
            }
        };
        const auto request = [&](Batch& q, int b) {   // tokens b .. b + kTokens - 1 of the adapter
#pragma unroll
            for (int d = 0; d < kX; ++d) {
                q.row[d] = (int64_t)token[d] * C;
                q.x[d] = raw_eight<kWhole>(in, q.row[d], c0 + 8 * tvec, C, in_total);
            }
#pragma unroll
            for (int v = 0; v < kS; ++v) {
                const int i = threadIdx.x + 256 * v, j = b + i / (4 * kRT), quad = rb / 4 + i % (4 * kRT), across = a.rpad / 4;
                q.s[v] = s[(int64_t)(j < count ? j : count - 1) * across + (quad < across ? quad : across - 1)];
            }
            find(b + kTokens);
        };
        const auto multiply = [&](Batch& q, int b) {
            if (b > 0) __syncthreads();   // the tiles of the batch before have been read by everyone
#pragma unroll
            for (int d = 0; d < kX; ++d) {   // (zeros behind the last token, in both)
                const int j = 256 / kAcross * d + trow;
                const uint4 x = true_eight<kWhole>(q.x[d], q.row[d], c0 + 8 * tvec, C, in_total);
                *reinterpret_cast<uint4*>(&in_tile[j * kPitch + 8 * tvec]) = b + j < count ? x : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int v = 0; v < kS; ++v) {
                const int i = threadIdx.x + 256 * v, j = i / (4 * kRT);
                *reinterpret_cast<uint4*>(&s_tile[j * kSPitch + 8 * (i % (4 * kRT))]) = b + j < count ? q.s[v] : make_uint4(0, 0, 0, 0);
            }
            if (b + kDeep * kTokens < count) request(q, b + kDeep * kTokens);
            __syncthreads();
#pragma unroll
            for (int d = 0; d < kBatch; ++d) {
                if (b + 32 * d >= count) continue;   // the same for the workgroup
                // four quads of a row side by side, or (s) every other one: the first halves, or the second
                const auto operand = [&](const uint16_t* tile, int pitch, int c, int apart) {
                    const uint16_t* col = tile + (32 * d + 8 * g + (i16 >> 2)) * pitch + c + apart * (i16 & 3);
                    const uint2 lo = lds_read_tr4(col), hi = lds_read_tr4(col + 4 * pitch);
                    return as_bf16x8(make_uint4(lo.x, lo.y, hi.x, hi.y));
                };
                bf16x8 x[kCT];
#pragma unroll
                for (int ct = 0; ct < kCT; ++ct) x[ct] = operand(in_tile, kPitch, 16 * (kCT * wave + ct), 4);
#pragma unroll
                for (int rt = 0; rt < kRT; ++rt)
                    if (rb + 16 * rt < rank)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const bf16x8 f = operand(s_tile, kSPitch, 32 * rt + 4 * h, 8);
#pragma unroll
                            for (int ct = 0; ct < kCT; ++ct) {
                                if constexpr (second) acc[ct][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[ct], f, acc[ct][rt], 0, 0, 0);
                                else acc[ct][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, x[ct], acc[ct][rt], 0, 0, 0);
                            }
                        }
            }
        };
        if (count > 0) {
            find(0);
            request(ahead[0], 0);
            if constexpr (kDeep == 2)
                if (kTokens < count) request(ahead[1], kTokens);
        }
        for (int b = 0; b < count; b += kDeep * kTokens) {
            multiply(ahead[0], b);
            if constexpr (kDeep == 2)
                if (b + kTokens < count) multiply(ahead[1], b + kTokens);
        }
        if (rb + 16 * kRT < rank) __syncthreads();   // before the next pass writes the tiles again
        // lane holds column i16 and rows 4 g + e of its accumulators: rows are columns of dy (dB) or ranks (dA)
#pragma unroll
        for (int ct = 0; ct < kCT; ++ct)
#pragma unroll
            for (int rt = 0; rt < kRT; ++rt) {
                const int r = rb + 16 * rt + (second ? i16 : 4 * g), c = c0 + 16 * (kCT * wave + ct) + (second ? 4 * g : i16);
                if (r >= rank || c >= C) continue;
                const int left = second ? C - c : rank - r;
                if (slot >= 0) {   // [K][rpad], then [rpad][N]
                    float* to = a.sums + (int64_t)slot * (a.C[0] + a.C[1]) * a.rpad + (second ? a.C[0] * a.rpad + (int64_t)r * C + c : (int64_t)c * a.rpad + r);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i < left) to[i] = acc[ct][rt][i];
                    continue;
                }
                uint16_t* to = second ? out + (int64_t)r * C + c : out + (int64_t)c * adapter.pitch + r;
                uint16_t e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) e[i] = f32_to_bf16_rne(acc[ct][rt][i]);
                if (left >= 4) {
                    *reinterpret_cast<AnyUint2*>(to) = u32x2_t{e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16};
                } else {
#pragma unroll
                    for (int i = 0; i < 3; ++i)
                        if (i < left) to[i] = e[i];
                }
            }
    }
}

// The second half of the backward pass in one launch: the adapters' gradients, which read what the first products have read, then dx.  (Two launches: 33 and 21 us for
// 4096 tokens at 4096 x 14336, rank 32, 53 so; 8 and 9 us for 777 tokens at 2720 x 2744, 13 so.)
struct BackwardArgs {
    OuterArgs outer;
    WideArgs wide;
    int across, outer_blocks;   // of a chunk, of all (0: not wanted)
};
template <int kRT, int kMostR, bool kWhole>
__global__ __launch_bounds__(256, kMostR > 64 ? 1 : 2) void backward_kernel(BackwardArgs a) {
    __shared__ __align__(16) union Lds {
        OuterLds<kRT> outer;
        WideLds<64, kMostR, true> wide;
    } lds;
    if ((int)blockIdx.x >= a.outer_blocks) {
        wide_tile<false, 64, kMostR, true, kWhole>(a.wide, (int)blockIdx.x - a.outer_blocks, lds.wide);
    } else {
        const AlignedUint4 chunk = scalar_load(reinterpret_cast<const AlignedUint4*>(a.outer.chunks + (int)blockIdx.x / a.across));
        const int block = (int)blockIdx.x % a.across;
        if ((int)chunk[0] < 0) return;
        if (block < a.outer.blocks0) outer_tile<kRT, kWhole, false>(a.outer, block, chunk, lds.outer.in_tile, lds.outer.s_tile);
        else outer_tile<kRT, kWhole, true>(a.outer, block, chunk, lds.outer.in_tile, lds.outer.s_tile);
    }
}

// The gradients of adapters of several chunks: workgroup (share of the values, adapter).
struct JoinArgs {
    Tokens tokens;
    const float* sums;
    int64_t K, N;
    int rpad, max_rank, chunk;
};
__global__ __launch_bounds__(256) void join_kernel(JoinArgs a) {
    const int group = blockIdx.y, count = scalar_load(a.tokens.counts + group), start = scalar_load(a.tokens.starts + group);
    if (count <= a.chunk) return;
    const salr_adapter_t* record = a.tokens.list + group;
    uint16_t *da = scalar_load(&record->da), *db = scalar_load(&record->db);
    const Adapter adapter = adapter_of(a.tokens, group, a.max_rank);
    const int rank = adapter.rank, slots = (count + a.chunk - 1) / a.chunk;
    const int64_t slot = (a.K + a.N) * a.rpad, of_a = a.K * rank, all = of_a + a.N * rank;
    const float* sums = a.sums + 2 * (start / a.chunk) * slot;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const bool second = i >= of_a;
        uint16_t* out = second ? db : da;
        if (out == nullptr) continue;
        const int64_t at = second ? i - of_a : i;
        const float* from = sums + (second ? a.K * a.rpad + at : at / rank * a.rpad + at % rank);
        float s = 0.f;
#pragma unroll 8
        for (int z = 0; z < slots; ++z) s += from[z * slot];
        out[second ? at : at / rank * adapter.pitch + at % rank] = f32_to_bf16_rne(s);
    }
}

// ---- host

namespace {

size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// Slices of a contraction of C columns: `want` of them, each of steps_least steps of 128 columns at least.
int slices_of(int64_t C, int64_t want, int64_t steps_least) {
    const int64_t steps = (C + 127) / 128;
    int64_t s = want;
    if (s > steps / steps_least) s = steps / steps_least;
    if (s > 16) s = 16;
    return s < 1 ? 1 : (int)s;
}

Tokens tokens_of(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p) {
    const char* w = static_cast<const char*>(a.workspace);
    const auto at = [&](size_t offset) { return reinterpret_cast<const int32_t*>(w + offset); };
    return p.direct ? Tokens{a.list, a.ids, nullptr, nullptr, nullptr, nullptr, (int)a.T, (int)a.n}
                    : Tokens{a.list, a.ids, at(p.order), at(p.starts), at(p.counts), reinterpret_cast<const int4*>(w + p.table), (int)a.T, (int)a.n};
}

void launch_order(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p) {
    char* w = static_cast<char*>(a.workspace);
    hipLaunchKernelGGL(order_tokens_kernel, dim3((unsigned)a.n + 2), dim3(1024), 0, a.stream, a.ids, (int)a.T, (int)a.n,
                       reinterpret_cast<int32_t*>(w + p.order), reinterpret_cast<int32_t*>(w + p.starts), reinterpret_cast<int32_t*>(w + p.counts),
                       reinterpret_cast<int4*>(w + p.table), p.chunk, p.chunk > 0 ? reinterpret_cast<int4*>(w + p.chunks) : nullptr);
}

template <typename Run>
void with_whole(bool whole, Run run) {   // rows of whole vectors
    if (whole) run(std::true_type());
    else run(std::false_type());
}

void launch_narrow(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p, bool x_too, bool dy_too) {
    char* w = static_cast<char*>(a.workspace);
    NarrowArgs n{tokens_of(a, p), {a.x, a.dy}, {a.K, a.N}, {reinterpret_cast<float*>(w + p.part_x), reinterpret_cast<float*>(w + p.part_dy)},
                 {x_too ? p.slices_x : 0, dy_too ? p.slices_dy : 0}, p.t_rows, p.rpad, p.max_rank};
    const dim3 grid((unsigned)(p.tiles * (n.slices[0] + n.slices[1])));
    const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, a.stream, n); };
    with_whole((!x_too || a.K % 8 == 0) && (!dy_too || a.N % 8 == 0), [&](auto whole) {
        constexpr bool kWhole = decltype(whole)::value;
        if (p.direct) p.rpad <= 16 ? run(narrow_kernel<true, 1, 1, kWhole>) : p.rpad <= 32 ? run(narrow_kernel<true, 1, 2, kWhole>) : run(narrow_kernel<true, 1, 4, kWhole>);
        else p.rpad <= 16 ? run(narrow_kernel<false, 4, 1, kWhole>) : p.rpad <= 32 ? run(narrow_kernel<false, 4, 2, kWhole>) : run(narrow_kernel<false, 4, 4, kWhole>);
    });
}

// Columns of a workgroup of wide_tile: 256, and twice as many as long as the chip has work for every place it has (six workgroups a CU, four of 64 tokens; ranks
// above 64, whose t takes 66 KB of LDS however many they are, leave place for one, which the rule does not know).
// 777 tokens, 2720 columns: 23 us in 1088 workgroups, 29 in 544 (and 26 in steps of 128 columns).
int per_group_of(const RequestAdaptersPlan& p, int64_t C) {
    int64_t per_group = 256;
    while (per_group < C && p.live * ((C + 2 * per_group - 1) / (2 * per_group)) >= (p.direct ? 1536 : 1024)) per_group *= 2;
    return (int)per_group;
}

void launch_forward_wide(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p) {
    const int per_group = per_group_of(p, a.N);
    const float* part = reinterpret_cast<const float*>(static_cast<char*>(a.workspace) + p.part_x);
    const WideArgs w{tokens_of(a, p), part, nullptr, p.slices_x, p.t_rows, p.rpad, p.max_rank, a.N, per_group, a.base, a.out};
    const dim3 grid((unsigned)(p.tiles * ((a.N + per_group - 1) / per_group)));
    const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, a.stream, w); };
    with_whole(a.N % 8 == 0, [&](auto whole) {
        constexpr bool kWhole = decltype(whole)::value;
        if (p.direct) p.rpad <= 32 ? run(wide_kernel<true, 16, 32, kWhole>) : p.rpad <= 64 ? run(wide_kernel<true, 16, 64, kWhole>) : run(wide_kernel<true, 16, 256, kWhole>);
        else p.rpad <= 32 ? run(wide_kernel<false, 64, 32, kWhole>) : p.rpad <= 64 ? run(wide_kernel<false, 64, 64, kWhole>) : run(wide_kernel<false, 64, 256, kWhole>);
    });
}

void launch_backward(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p, const uint4* t_x, const uint4* t_dy) {
    char* workspace = static_cast<char*>(a.workspace);
    float* sums = reinterpret_cast<float*>(workspace + p.sums);
    BackwardArgs b{};
    const int blocks0 = (int)((a.K + kOuterCols - 1) / kOuterCols), blocks1 = (int)((a.N + kOuterCols - 1) / kOuterCols), per_group = per_group_of(p, a.K);
    b.outer = OuterArgs{tokens_of(a, p), {a.x, a.dy}, {t_dy, t_x}, {a.K, a.N}, p.rpad, p.max_rank, blocks0, reinterpret_cast<const int4*>(workspace + p.chunks), sums};
    b.wide = WideArgs{tokens_of(a, p), nullptr, t_dy, 0, p.t_rows, p.rpad, p.max_rank, a.K, per_group, a.base, a.out};
    b.across = blocks0 + blocks1;
    b.outer_blocks = a.want_dadb ? (int)(b.across * (a.T / p.chunk + a.n)) : 0;
    const int64_t wide_blocks = a.T > 0 && a.out != nullptr ? p.tiles * ((a.K + per_group - 1) / per_group) : 0;
    if (b.outer_blocks + wide_blocks == 0) return;
    const dim3 grid((unsigned)(b.outer_blocks + wide_blocks));
    const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, a.stream, b); };
    with_whole(a.K % 8 == 0 && a.N % 8 == 0, [&](auto whole) {
        constexpr bool kWhole = decltype(whole)::value;
        if (p.rpad <= 32) p.rpad <= 16 ? run(backward_kernel<1, 32, kWhole>) : run(backward_kernel<2, 32, kWhole>);
        else p.rpad <= 64 ? run(backward_kernel<4, 64, kWhole>) : run(backward_kernel<4, 256, kWhole>);
    });
    if (a.want_dadb && a.T > p.chunk)
        hipLaunchKernelGGL(join_kernel, dim3((unsigned)(a.n < 16 ? 2048 / a.n : 128), (unsigned)a.n), dim3(256), 0, a.stream, JoinArgs{tokens_of(a, p), sums, a.K, a.N, p.rpad, p.max_rank, p.chunk});
}

// Tokens of a chunk of the gradients' sums.  Adapters enough for two workgroups a CU: 4096, since a chunk less costs a launch, and the sums a trip through memory
// (4096 tokens of eight adapters, 4096 x 14336, rank 32: 97 us so, 112 with chunks of 1024).  Else as few as there are workgroups for, if the
// batch were one adapter's: 4096 tokens of one adapter at 512 x 512 rank 16 43 us in one chunk, 13 so; at 4096 x 4096 rank 64 91 and 45.
int chunk_of(int64_t T, int64_t K, int64_t N, int64_t n) {
    const int64_t across = (K + N + kOuterCols - 1) / kOuterCols;
    if (across * (n < T ? n : T) >= 512) return 4096;
    int chunk = 1024;
    while (chunk > 256 && across * (T / chunk) < 512) chunk /= 2;
    return chunk;
}

}  // namespace

RequestAdaptersPlan request_adapters_plan(int64_t T, int64_t K, int64_t N, int64_t n, int64_t max_rank, bool backward, bool want_dadb) {
    RequestAdaptersPlan p{};
    p.direct = !backward && T <= kDirectTokens;
    p.rows = p.direct ? 16 : kTileTokens;
    const int64_t groups = n + 2 < T ? n + 2 : T;   // that hold a token
    p.tiles = p.direct ? T : T / kTileTokens + n + 2;
    p.t_rows = T;
    p.max_rank = (int)max_rank;
    p.rpad = (int)((max_rank + 15) / 16 * 16);
    if (p.rpad == 0) p.rpad = 16;
    p.live = p.direct ? (n < T ? n : T) : (T + kTileTokens - 1) / kTileTokens + groups / 2;   // tiles to expect
    if (p.live == 0) p.live = 1;
    if (p.direct) {
        p.slices_x = slices_of(K, 1024 / p.live, 1);
    } else {
        // four workgroups a CU, all at once; the backward pass' two products take as long as each other
        const int64_t all = 1024 / p.live, of_x = backward && want_dadb ? (all * K + (K + N) / 2) / (K + N) : 0;
        p.slices_x = slices_of(K, backward ? of_x : all, backward ? 2 : 4);
        p.slices_dy = slices_of(N, all - of_x, 2);
    }
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        const size_t here = at;
        at += padded(bytes);
        return here;
    };
    if (!p.direct) {
        p.order = take((size_t)T * 4);
        p.starts = take((size_t)(n + 2) * 4);
        p.counts = take((size_t)(n + 2) * 4);
        p.table = take((size_t)p.tiles * 16);
    }
    if (backward) {
        p.chunk = chunk_of(T, K, N, n);
        p.chunks = take((size_t)(T / p.chunk + n + 2) * 16);
        if (want_dadb && T > p.chunk) p.sums = take((size_t)(2 * (T / p.chunk) + 2) * (K + N) * p.rpad * 4);
    }
    const size_t row = (size_t)T * p.rpad;
    if (!backward || want_dadb) p.part_x = take(row * 4 * p.slices_x);
    if (backward) {
        p.part_dy = take(row * 4 * p.slices_dy);
        if (want_dadb) p.t_x = take(row * 4);
        p.t_dy = take(row * 4);
    }
    p.bytes = at;
    return p;
}

// Few tokens in one launch: a workgroup is a token and 512 columns of its output, and forms all of the token's t for them.  What memory brings twice that way costs less
// than a second launch, as long as it is not much.  Threads are vectors of eight ranks, then columns of x: A comes in as it lies; t is fp32 throughout.  The
// second product's operands are asked for before the first one's sums go round.
struct FewArgs {
    Tokens tokens;
    const uint16_t *x, *base;   // base may be out, or null (zeros)
    uint16_t* out;
    int K, N, max_rank, pieces;
};
constexpr int kFewColumns = 512, kFewRank = 64;
template <int kRT, bool kWhole>
__global__ __launch_bounds__(1024) void few_tokens_kernel(FewArgs a) {
    constexpr int kWaves = 16, kDeep = 8;
    __shared__ float t_sums[kWaves][16 * kRT];
    __shared__ f32x4 out_sums[kWaves][kFewColumns / 4];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces * kFewColumns, column = piece + (int)threadIdx.x;
    const bool writes = threadIdx.x < kFewColumns && column < a.N;
    const int64_t place = (int64_t)token * a.N + column;
    uint32_t before = 0;
    if (writes && a.base != nullptr) before = a.base[place];
    const int group = group_of(scalar_load(a.tokens.ids + token), a.tokens.n);
    Adapter adapter{nullptr, nullptr, 0, 0};
    if (group < a.tokens.n) adapter = adapter_of(a.tokens, group, a.max_rank);
    const int rank = adapter.rank;
    float y = 0.f;
    if (rank > 0) {   // the same for the workgroup
        uint4 b[kRT];
        const int64_t b_total = (int64_t)rank * a.N, a_total = (int64_t)adapter.pitch * a.K;
#pragma unroll
        for (int i = 0; i < kRT; ++i) {
            const int r = wave + kWaves * i;
            b[i] = raw_eight<kWhole>(adapter.b, (int64_t)(r < rank ? r : rank - 1) * a.N, piece + 8 * lane, a.N, b_total);
        }
        const int vectors = (rank + 7) / 8, shift = vectors <= 1 ? 0 : 32 - __builtin_clz(vectors - 1);   // a row's, and of how many threads
        const int v = threadIdx.x & ((1 << shift) - 1), step = 1024 >> shift;
        const uint16_t* x = a.x + (int64_t)token * a.K;
        float acc[8] = {};
        for (int c = threadIdx.x >> shift; c < a.K; c += kDeep * step) {
            uint4 q[kDeep];
            uint16_t xs[kDeep];
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {   // (behind the last column that one again, left out below)
                const int at = c + i * step < a.K ? c + i * step : a.K - 1;
                q[i] = raw_ranks(adapter.a, at, 8 * v, adapter.pitch, a_total);
                xs[i] = x[at];
            }
#pragma unroll
            for (int i = 0; i < kDeep; ++i) {
                if (c + i * step >= a.K) break;
                const uint4 f = true_ranks(q[i], c + i * step, 8 * v, adapter.pitch, a_total);
                const float xv = bf16_bits_to_f32(xs[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[j] = fmaf(xv, bf16_bits_to_f32(unit_elem(f, j)), acc[j]);
            }
        }
        // sums over the lanes with the same v: three exchanges halve what a lane has, until it is one rank
        float four[4], two[2];
        const bool h5 = lane & 32, h4 = lane & 16, h3 = lane & 8;
#pragma unroll
        for (int j = 0; j < 4; ++j) four[j] = (h5 ? acc[j + 4] : acc[j]) + __shfl_xor(h5 ? acc[j] : acc[j + 4], 32);
#pragma unroll
        for (int j = 0; j < 2; ++j) two[j] = (h4 ? four[j + 2] : four[j]) + __shfl_xor(h4 ? four[j] : four[j + 2], 16);
        float one = (h3 ? two[1] : two[0]) + __shfl_xor(h3 ? two[0] : two[1], 8);
        for (int apart = 1 << shift; apart < 8; apart *= 2) one += __shfl_xor(one, apart);
        if ((lane & 7) < (1 << shift) && v < vectors) t_sums[wave][8 * v + 4 * h5 + 2 * h4 + h3] = one;
        __syncthreads();
        // a wave has every sixteenth rank: sixteen lanes add up the waves' sums of each
        float t = 0.f;
        const int mine = wave + kWaves * (lane >> 4);
        if (mine < rank) t = t_sums[lane & 15][mine];
#pragma unroll
        for (int apart = 1; apart < 16; apart *= 2) t += __shfl_xor(t, apart);
        f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kRT; ++i) {
            const int r = wave + kWaves * i;
            if (r >= rank) break;
            const float ti = __shfl(t, 16 * i);
            const uint4 f = true_eight<kWhole>(b[i], (int64_t)r * a.N, piece + 8 * lane, a.N, b_total);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                lo[j] = fmaf(ti, bf16_bits_to_f32(unit_elem(f, j)), lo[j]);
                hi[j] = fmaf(ti, bf16_bits_to_f32(unit_elem(f, j + 4)), hi[j]);
            }
        }
        out_sums[wave][2 * lane] = lo;
        out_sums[wave][2 * lane + 1] = hi;
        __syncthreads();
        if (threadIdx.x < kFewColumns)
#pragma unroll
            for (int w = 0; w < kWaves; ++w) y += reinterpret_cast<const float*>(out_sums[w])[threadIdx.x];
    }
    if (writes) a.out[place] = group > a.tokens.n ? 0x7FC0 : rank > 0 ? f32_to_bf16_rne(bf16_bits_to_f32(before) + y) : before;
}

// Where that is faster than two launches.  One token, 4096 x 4096 rank 16 6.6 us against 8.2 (kernels alone; a call 4.9 to 6.5 against 8.25), 2048 x 8192 rank 32
// 7.3 against 8.8, 1024 x 4096 rank 64 7.0 against 9.8; sixteen tokens 512 x 512 rank 16 6.4 against 8.2.  Outside: one token, 4096 x 14336 rank 16 (28
// workgroups) 8.0 against 8.3, 14336 x 4096 10.8 against 9.6, 4096 x 4096 rank 64 12.3 against 10.2; four tokens 4096 x 4096 rank 16 8.5 against 8.3.
// The limit of A is on the safe side: in calls of one token one launch took 5.8 us against 8.3 at 80 K values of it (5120 x 4096 rank 16), 6.4 to 7.0 against 8.6 to 9.5 at 128 K
// (8192 x 4096 rank 16, 4096 x 4096 rank 32, 2048 x 4096 rank 64), 7.9 against 9.2 at 192 K (12288 x 4096 rank 16) and 9.0 against 9.4 at 224 K.
bool few_tokens(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p) {
    const int64_t pieces = (a.N + kFewColumns - 1) / kFewColumns;
    return p.rpad <= kFewRank && a.K * p.rpad <= 65536 && a.T * pieces <= 16;
}
void launch_few_tokens(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p) {
    const int pieces = (int)((a.N + kFewColumns - 1) / kFewColumns);
    const FewArgs f{tokens_of(a, p), a.x, a.base, a.out, (int)a.K, (int)a.N, p.max_rank, pieces};
    const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(a.T * pieces)), dim3(1024), 0, a.stream, f); };
    with_whole(a.N % 8 == 0, [&](auto whole) {
        constexpr bool kWhole = decltype(whole)::value;
        p.rpad <= 16 ? run(few_tokens_kernel<1, kWhole>) : p.rpad <= 32 ? run(few_tokens_kernel<2, kWhole>) : run(few_tokens_kernel<4, kWhole>);
    });
}

hipError_t launch_request_adapters(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p) {
    if (few_tokens(a, p)) {   // (leaves the workspace alone)
        launch_few_tokens(a, p);
        return hipGetLastError();
    }
    if (!p.direct) launch_order(a, p);
    launch_narrow(a, p, true, false);
    launch_forward_wide(a, p);
    return hipGetLastError();
}

hipError_t launch_request_adapters_backward(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p) {
    char* w = static_cast<char*>(a.workspace);
    uint4 *t_x = reinterpret_cast<uint4*>(w + p.t_x), *t_dy = reinterpret_cast<uint4*>(w + p.t_dy);
    launch_order(a, p);
    if (a.T > 0) {
        launch_narrow(a, p, a.want_dadb, true);
        const SumArgs s{{reinterpret_cast<const float*>(w + p.part_dy), reinterpret_cast<const float*>(w + p.part_x)}, {t_dy, t_x}, {p.slices_dy, p.slices_x}, a.T * p.rpad};
        hipLaunchKernelGGL(sum_slices_kernel, dim3((unsigned)((s.count / 4 + 255) / 256), a.want_dadb ? 2 : 1), dim3(256), 0, a.stream, s);
    }
    launch_backward(a, p, t_x, t_dy);
    return hipGetLastError();
}

}  // namespace salr
