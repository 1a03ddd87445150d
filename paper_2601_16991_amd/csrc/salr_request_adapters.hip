// Adapters of many requests beside one shared layer: every token t names its adapter i = ids[t], or none.
//
//   out[t] = base[t] + (x[t] A_i) B_i        A_i [K, r_i], B_i [r_i, N]
//   dx[t] = dx_base[t] + (dy[t] B_i^T) A_i^T,   dA_i = sum over i's tokens of x[t]^T (dy[t] B_i^T),   dB_i = sum of (x[t] A_i)^T dy[t]
//
// Tokens of one adapter are brought together into tiles, whose rows are read and written where they are: nothing is copied.
//   up to kDirectTokens tokens   a workgroup is a token, finds its fellows among the ids by one comparison across the wave, and goes on if it
//                                is the first of a tile of 16
//   more                         a launch in front orders the tokens by adapter (stable: sums over tokens have an order); a workgroup finds the
//                                adapter of its tile of 64 in the counts
// Then  narrow_kernel  t = in * factor (K or N columns down to r; fp32 sums over slices of the columns),
//       wide_kernel    out = base + t * factor (r up to N or K columns), t rounded to bf16 as the layer rounds its own,
//       outer_kernel   the adapters' gradients, sums over tokens.
// All on the matrix cores, though memory bounds each (2 r products a byte of x and out at most): tiles of 16 fill them however few rows are live, and
// what an adapter's factors lack in alignment or length is zeros in LDS.  Results do not depend on which other tokens a call holds, save that
// the number of slices follows from its sizes.
#include "salr_adapter_t.hpp"
#include "salr_eight.hpp"
#include "salr_internal.hpp"

namespace salr {

namespace {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef u32x2_t AnyUint2 __attribute__((aligned(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// LDS of one wave alone: what was written is read by its other lanes, what was read may be written again.  (Its accesses are done in order;
// this keeps the compiler to it.)
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int kDirectTokens = 64;
constexpr int kTileTokens = 64;   // of a launch that orders tokens

struct Tokens {   // how a kernel finds its rows
    const salr_adapter_t* list;
    const int32_t* ids;
    const int32_t* order;    // tokens by group: adapters, then those without one, then those whose id is none
    const int32_t* starts;   // [n + 2]
    const int32_t* counts;   // [n + 2]
    int T, n;
};

// Groups n and n + 1: no adapter; an id out of range.
__device__ __forceinline__ int group_of(int id, int n) { return id < 0 ? n : id < n ? id : n + 1; }

struct Tile {
    int group;   // -1: none left
    int count;   // live rows
    int first;   // of an ordered launch: position of the first
};

// The tile of this workgroup and, in rows[kRows] (LDS), its tokens, -1 behind the last.  Every thread calls it; ends with a barrier.
template <bool kDirect, int kRows>
__device__ __forceinline__ Tile find_tile(const Tokens& k, int* rows) {
    const int lane = lane_id();
    Tile tile{-1, 0, 0};
    if constexpr (kDirect) {
        const int self = blockIdx.x, group = lane < k.T ? group_of(k.ids[lane], k.n) : -2;
        const int mine = __builtin_amdgcn_readlane(group, self);
        const uint64_t same = __ballot(group == mine), below = same & (((uint64_t)1 << self) - 1);
        const int before = __popcll(below);
        if (before % kRows != 0) return tile;   // the same for the workgroup
        const int place = __popcll(same & (((uint64_t)1 << lane) - 1)) - before, left = __popcll(same) - before;
        tile.group = mine;
        tile.count = left < kRows ? left : kRows;
        if (threadIdx.x < kRows) rows[threadIdx.x] = -1;
        __syncthreads();
        if (threadIdx.x < kWave && group == mine && place >= 0 && place < kRows) rows[place] = lane;
    } else {
        int before = 0;   // tiles of the groups already looked at
        for (int g0 = 0; g0 < k.n + 2; g0 += kWave) {
            const int count = g0 + lane < k.n + 2 ? k.counts[g0 + lane] : 0;
            const int tiles = (count + kRows - 1) / kRows, upto = before + (int)wave_inclusive_scan((uint32_t)tiles);
            const uint64_t past = __ballot(upto > (int)blockIdx.x);
            if (past != 0) {
                const int at = __builtin_ctzll(past);
                const int done = kRows * ((int)blockIdx.x - __builtin_amdgcn_readlane(upto - tiles, at));
                const int left = __builtin_amdgcn_readlane(count, at) - done;
                tile.group = g0 + at;
                tile.count = left < kRows ? left : kRows;
                tile.first = k.starts[tile.group] + done;
                break;
            }
            before = __builtin_amdgcn_readlane(upto, kWave - 1);
        }
        if (tile.group < 0) return tile;
        if (threadIdx.x < kRows) rows[threadIdx.x] = (int)threadIdx.x < tile.count ? k.order[tile.first + threadIdx.x] : -1;
    }
    __syncthreads();
    return tile;
}

// Row j's place in the sums of a tile.
template <bool kDirect>
__device__ __forceinline__ int64_t place_of(const Tile& tile, const int* rows, int j) {
    return kDirect ? rows[j] : tile.first + j;
}

__device__ __forceinline__ uint4 eight_of(const uint16_t* row, int64_t c, int64_t C) {   // columns c .. c + 7 of a row of C, zeros behind it
    const int64_t left = C - c;
    return load_eight<false, false, false>(row + c, 0, left < 8 ? (int)left : 8).q[0];
}

}  // namespace

// A workgroup a group: counts the tokens of the groups before its own, then puts its own in order.  Every group goes through all ids, which
// stay in the caches; no workgroup waits for another.
__global__ __launch_bounds__(1024) void order_tokens_kernel(const int32_t* ids, int T, int n, int32_t* order, int32_t* starts, int32_t* counts) {
    __shared__ uint32_t scratch[17];
    __shared__ int total[2];
    const int group = blockIdx.x;
    if (threadIdx.x < 2) total[threadIdx.x] = 0;
    __syncthreads();
    int less = 0, same = 0;
    for (int t = threadIdx.x; t < T; t += 1024) {
        const int g = group_of(ids[t], n);
        less += g < group;
        same += g == group;
    }
    less = (int)last_lane(wave_inclusive_scan((uint32_t)less));
    same = (int)last_lane(wave_inclusive_scan((uint32_t)same));
    if (lane_id() == 0) {   // (whole numbers: in any order)
        atomicAdd(&total[0], less);
        atomicAdd(&total[1], same);
    }
    __syncthreads();
    int at = total[0];
    const int count = total[1];
    if (threadIdx.x == 0) {
        starts[group] = at;
        counts[group] = count;
    }
    if (count == 0) return;
    for (int t0 = 0; t0 < T; t0 += 1024) {
        const int t = t0 + threadIdx.x;
        const bool mine = t < T && group_of(ids[t], n) == group;
        uint32_t here;
        const uint32_t place = block_exclusive_scan<1024>(mine ? 1u : 0u, scratch, here);
        if (mine) order[at + place] = t;
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
    int rpad;
};

// part[z][row][r] = sum over the columns c of slice z of in[row][c] * factor(c, r).  Workgroup (tile, slice); its four waves take every fourth step
// of 32 columns, with 16 kMB rows and 16 kRT ranks each (more ranks: another pass), and are added through LDS, in order.  in's rows are the A
// operand of 16x16x32 MFMAs as they lie; A's [32 columns, ranks], which lie the wrong way round, go through LDS and its transposing
// read, B's [ranks, columns] are the B operand as they lie.  A step's requests are out while the one before is multiplied.
template <bool kDirect, int kMB, int kRT>
__global__ __launch_bounds__(256) void narrow_kernel(NarrowArgs a) {
    constexpr int kPitch = 16 * kRT + 8, kSumPitch = 16 * kRT + 4;
    __shared__ int rows[16 * kMB];
    __shared__ __align__(16) uint16_t stages[4][32 * kPitch];
    __shared__ __align__(16) float sums[16 * kMB * kSumPitch];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, g = lane >> 4;
    const Tile tile = find_tile<kDirect, 16 * kMB>(a.tokens, rows);
    if (tile.group < 0 || tile.group >= a.tokens.n) return;
    const bool second = (int)blockIdx.y >= a.slices[0];
    const int z = second ? (int)blockIdx.y - a.slices[0] : (int)blockIdx.y, slices = second ? a.slices[1] : a.slices[0];
    const uint16_t* in = second ? a.in[1] : a.in[0];
    const int64_t C = second ? a.C[1] : a.C[0];
    float* part = (second ? a.part[1] : a.part[0]) + (int64_t)z * a.t_rows * a.rpad;
    const salr_adapter_t& adapter = a.tokens.list[tile.group];
    const int rank = (int)adapter.rank;
    const uint16_t* factor = second ? adapter.b : adapter.a;
    const int steps = (int)((C + 31) >> 5), s_begin = (int)((int64_t)steps * z / slices), s_end = (int)((int64_t)steps * (z + 1) / slices);
    const uint16_t* row[kMB];
#pragma unroll
    for (int mb = 0; mb < kMB; ++mb) {
        const int token = rows[16 * mb + i16];
        row[mb] = token < 0 ? nullptr : in + (int64_t)token * C;
    }
    uint16_t* stage = stages[wave];
    for (int rb = 0; rb < rank; rb += 16 * kRT) {
        const int rts = (rank - rb + 15) / 16 < kRT ? (rank - rb + 15) / 16 : kRT;
        f32x4 acc[kMB][kRT] = {};
        uint4 xq[kMB], fq[kRT];
        const auto request = [&](int s) {
            const int64_t c = 32 * (int64_t)s;
#pragma unroll
            for (int mb = 0; mb < kMB; ++mb) xq[mb] = row[mb] != nullptr ? eight_of(row[mb], c + 8 * g, C) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int rt = 0; rt < kRT; ++rt) {
                fq[rt] = make_uint4(0, 0, 0, 0);
                if (second) {
                    const int r = rb + 16 * rt + i16;
                    if (r < rank) fq[rt] = eight_of(factor + (int64_t)r * C, c + 8 * g, C);
                } else {   // vector v of [32][16 kRT]
                    const int v = lane + 64 * rt, k = v / (2 * kRT), r = rb + 8 * (v % (2 * kRT));
                    if (c + k < C && r < rank) fq[rt] = eight_of(factor + (c + k) * rank, r, rank);
                }
            }
        };
        if (s_begin + wave < s_end) request(s_begin + wave);
        for (int s = s_begin + wave; s < s_end; s += 4) {
            bf16x8 x[kMB], f[kRT];
#pragma unroll
            for (int mb = 0; mb < kMB; ++mb) x[mb] = as_bf16x8(xq[mb]);
            if (second) {
#pragma unroll
                for (int rt = 0; rt < kRT; ++rt) f[rt] = as_bf16x8(fq[rt]);
            } else {
#pragma unroll
                for (int rt = 0; rt < kRT; ++rt) {
                    const int v = lane + 64 * rt;
                    *reinterpret_cast<uint4*>(stage + v / (2 * kRT) * kPitch + 8 * (v % (2 * kRT))) = fq[rt];
                }
                wave_sync();
#pragma unroll
                for (int rt = 0; rt < kRT; ++rt) {
                    const uint16_t* col = stage + (8 * g + (i16 >> 2)) * kPitch + 16 * rt + 4 * (i16 & 3);
                    const uint2 lo = lds_read_tr4(col), hi = lds_read_tr4(col + 4 * kPitch);
                    f[rt] = as_bf16x8(make_uint4(lo.x, lo.y, hi.x, hi.y));
                }
                wave_sync();
            }
            if (s + 4 < s_end) request(s + 4);
#pragma unroll
            for (int rt = 0; rt < kRT; ++rt)
                if (rt < rts)
#pragma unroll
                    for (int mb = 0; mb < kMB; ++mb)
                        if (16 * mb < tile.count) acc[mb][rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[mb], f[rt], acc[mb][rt], 0, 0, 0);
        }
        // accumulators: lane holds column i16 (rank), rows 4 g + e (tokens)
        for (int w = 0; w < 4; ++w) {
            if (w == wave)
#pragma unroll
                for (int mb = 0; mb < kMB; ++mb)
#pragma unroll
                    for (int rt = 0; rt < kRT; ++rt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float* to = sums + (16 * mb + 4 * g + e) * kSumPitch + 16 * rt + i16;
                            *to = w == 0 ? acc[mb][rt][e] : *to + acc[mb][rt][e];
                        }
            __syncthreads();
        }
        for (int i = threadIdx.x; i < tile.count * rts * 4; i += 256) {
            const int j = i / (rts * 4), c = 4 * (i % (rts * 4));
            f32x4 v = *reinterpret_cast<const f32x4*>(sums + j * kSumPitch + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = rb + c + e < rank ? v[e] : 0.f;   // (zero times an infinity of in, where the ranks are padded)
            *reinterpret_cast<f32x4*>(part + place_of<kDirect>(tile, rows, j) * a.rpad + rb + c) = v;
        }
        __syncthreads();   // before the next pass
    }
}

// t = bf16(sum over the slices of part), four values a thread; y picks the product.
struct SumArgs {
    const float* part[2];
    uint16_t* t[2];
    int slices[2];
    int64_t count;   // of a slice
};
__global__ __launch_bounds__(256) void sum_slices_kernel(SumArgs a) {
    const bool second = blockIdx.y == 1;
    const float* part = second ? a.part[1] : a.part[0];
    const int slices = second ? a.slices[1] : a.slices[0];
    const int64_t i = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
    if (i >= a.count) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int z = 0; z < slices; ++z) s += *reinterpret_cast<const f32x4*>(part + z * a.count + i);
    uint16_t* to = (second ? a.t[1] : a.t[0]) + i;
    *reinterpret_cast<uint2*>(to) = make_uint2(f32_to_bf16_rne(s[0]) | (uint32_t)f32_to_bf16_rne(s[1]) << 16, f32_to_bf16_rne(s[2]) | (uint32_t)f32_to_bf16_rne(s[3]) << 16);
}

struct WideArgs {
    Tokens tokens;
    const float* part;      // [slices][t_rows][rpad], summed here; or, slices 0,
    const uint16_t* t;      // [t_rows][rpad]
    int slices;
    int64_t t_rows;
    int rpad;
    int64_t C;              // columns of out
    int64_t per_group;      // of a workgroup, whole 256s
    const uint16_t* base;   // may be out, or null (zeros)
    uint16_t* out;
};

// out[row][c] = base[row][c] + sum over r of t[row][r] * factor(r, c).  Workgroup (tile, columns): t's rows once into LDS, then each wave takes 64
// columns at a time, the factor's part of them, zeros where ranks or columns end, through LDS of its own (64 ranks a pass).  The product is
// formed transposed, columns of out as rows of 16x16x16 MFMAs, and which column a row stands for is chosen so that a lane ends up with 16
// columns of one token side by side (row m of tile j is column 16 (m / 4) + 4 j + m % 4): out is read and written in whole vectors.
// kFactorA: the factor is A [C, r] (dx), else B [r, C] (y).
template <bool kDirect, int kMB, int kMostR, bool kFactorA>
__global__ __launch_bounds__(256) void wide_kernel(WideArgs a) {
    constexpr int kTPitch = kMostR + 8, kPitch = 64 + 8;
    __shared__ int rows[16 * kMB];
    __shared__ __align__(16) uint16_t t[16 * kMB * kTPitch];
    __shared__ __align__(16) uint16_t stages[4][64 * kPitch];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, g = lane >> 4;
    const Tile tile = find_tile<kDirect, 16 * kMB>(a.tokens, rows);
    if (tile.group < 0) return;
    const int64_t c_begin = (int64_t)blockIdx.y * a.per_group, c_end = c_begin + a.per_group < a.C ? c_begin + a.per_group : a.C;
    if (tile.group >= a.tokens.n) {   // no adapter: base as it is; an id that is none: NaN
        const bool none = tile.group == a.tokens.n;
        if (none && a.base == a.out) return;
        const int width = (int)((c_end - c_begin + 7) >> 3);
        for (int i = threadIdx.x; i < tile.count * width; i += 256) {
            const int64_t at = (int64_t)rows[i / width] * a.C, c = c_begin + 8 * (i % width);
            const int left = c_end - c < 8 ? (int)(c_end - c) : 8;
            Eight<false> q{{make_uint4(0, 0, 0, 0)}};
            if (none && a.base != nullptr) q = load_eight<false, false, false>(a.base + at + c, 0, left);
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = none ? q.get(j) : __uint_as_float(0x7FC00000u);
            store_eight<false, false>(a.out + at + c, 0, left, v);
        }
        return;
    }
    const salr_adapter_t& adapter = a.tokens.list[tile.group];
    const int rank = (int)adapter.rank, rank16 = (rank + 15) & ~15;
    const uint16_t* factor = kFactorA ? adapter.a : adapter.b;
    for (int i = threadIdx.x; i < 16 * kMB * (rank16 / 4); i += 256) {
        const int j = i / (rank16 / 4), r = 4 * (i % (rank16 / 4));
        uint2 q = make_uint2(0, 0);
        if (j < tile.count) {
            const int64_t at = place_of<kDirect>(tile, rows, j) * a.rpad + r;
            if (a.slices > 0) {
                f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
                for (int z = 0; z < a.slices; ++z) s += *reinterpret_cast<const f32x4*>(a.part + z * a.t_rows * a.rpad + at);
                q = make_uint2(f32_to_bf16_rne(s[0]) | (uint32_t)f32_to_bf16_rne(s[1]) << 16, f32_to_bf16_rne(s[2]) | (uint32_t)f32_to_bf16_rne(s[3]) << 16);
            } else {
                q = *reinterpret_cast<const uint2*>(a.t + at);
            }
        }
        *reinterpret_cast<uint2*>(t + j * kTPitch + r) = q;
    }
    __syncthreads();
    uint16_t* stage = stages[wave];
    for (int64_t c0 = c_begin + 64 * wave; c0 < c_end; c0 += 256) {
        f32x4 acc[kMB][4] = {};
        for (int rb = 0; rb < rank; rb += 64) {
            const int ranks = rank - rb < 64 ? rank - rb : 64, steps = (ranks + 15) / 16;
            uint4 q[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                if (v >= 2 * steps) break;
                q[v] = make_uint4(0, 0, 0, 0);
                if constexpr (kFactorA) {   // vectors of [64 columns][16 steps ranks]
                    const int i = lane + 64 * v, k = i / (2 * steps), r = 8 * (i % (2 * steps));
                    if (c0 + k < a.C && r < ranks) q[v] = eight_of(factor + (c0 + k) * rank, rb + r, rank);
                } else {                    // vectors of [16 steps ranks][64 columns]
                    const int r = 8 * v + (lane >> 3);
                    if (r < ranks) q[v] = eight_of(factor + (int64_t)(rb + r) * a.C, c0 + 8 * (lane & 7), a.C);
                }
            }
            wave_sync();
#pragma unroll
            for (int v = 0; v < 8; ++v) {
                if (v >= 2 * steps) break;
                const int i = lane + 64 * v;
                if constexpr (kFactorA) *reinterpret_cast<uint4*>(stage + i / (2 * steps) * kPitch + 8 * (i % (2 * steps))) = q[v];
                else *reinterpret_cast<uint4*>(stage + (i >> 3) * kPitch + 8 * (i & 7)) = q[v];
            }
            wave_sync();
#pragma unroll
            for (int st = 0; st < 4; ++st) {
                if (st >= steps) break;
                uint2 tq[kMB];
#pragma unroll
                for (int mb = 0; mb < kMB; ++mb) tq[mb] = *reinterpret_cast<const uint2*>(t + (16 * mb + i16) * kTPitch + rb + 16 * st + 4 * g);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint2 f;
                    if constexpr (kFactorA) f = *reinterpret_cast<const uint2*>(stage + (16 * (i16 >> 2) + 4 * j + (i16 & 3)) * kPitch + 16 * st + 4 * g);
                    else f = lds_read_tr4(stage + (16 * st + 4 * g + (i16 >> 2)) * kPitch + 16 * (i16 & 3) + 4 * j);
#pragma unroll
                    for (int mb = 0; mb < kMB; ++mb)
                        if (16 * mb < tile.count)
                            acc[mb][j] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, f), __builtin_bit_cast(s16x4, tq[mb]), acc[mb][j], 0, 0, 0);
                }
            }
        }
        // lane holds columns c0 + 16 g .. + 15 of token 16 mb + i16
#pragma unroll
        for (int mb = 0; mb < kMB; ++mb) {
            const int token = rows[16 * mb + i16];
            if (token < 0) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t c = c0 + 16 * g + 8 * h;
                const int left = a.C - c < 8 ? (int)(a.C - c) : 8;
                if (left <= 0) continue;
                const int64_t at = (int64_t)token * a.C + c;
                Eight<false> q{{make_uint4(0, 0, 0, 0)}};
                if (a.base != nullptr) q = load_eight<false, false, false>(a.base + at, 0, left);
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = q.get(e) + acc[mb][2 * h + (e >> 2)][e & 3];
                store_eight<false, false>(a.out + at, 0, left, v);
            }
        }
    }
}

struct OuterArgs {
    Tokens tokens;
    const uint16_t* in[2];   // x (dA), dy (dB)
    const uint16_t* s[2];    // dy B^T (dA), x A (dB): [T][rpad] by position
    int64_t C[2];
    int rpad;
    int blocks0;             // of 64 columns: of x
};

// dA_i [K, r] and dB_i [r, N], sums over the adapter's tokens: workgroup (64 columns of x or dy, adapter).  Both operands lie with the tokens as
// rows and are transposed by LDS' transposing read, 32 tokens a step and kBatch steps in flight.  Which of the two is the MFMA's first
// operand is chosen so that a lane holds four values side by side of the result.  An adapter without tokens gets zeros.
template <int kRT>
__global__ __launch_bounds__(256) void outer_kernel(OuterArgs a) {
    constexpr int kBatch = 4, kPitch = 64 + 8, kSPitch = 16 * kRT + 8;
    __shared__ __align__(16) uint16_t in_tile[2][kBatch * 32 * kPitch];
    __shared__ __align__(16) uint16_t s_tile[2][kBatch * 32 * kSPitch];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, g = lane >> 4;
    const salr_adapter_t& adapter = a.tokens.list[blockIdx.y];
    const bool second = (int)blockIdx.x >= a.blocks0;
    uint16_t* out = second ? adapter.db : adapter.da;
    if (out == nullptr) return;
    const int rank = (int)adapter.rank, count = a.tokens.counts[blockIdx.y], start = a.tokens.starts[blockIdx.y];
    const uint16_t* in = second ? a.in[1] : a.in[0];
    const uint16_t* s = (second ? a.s[1] : a.s[0]) + (int64_t)start * a.rpad;
    const int64_t C = second ? a.C[1] : a.C[0], c0 = 64 * (int64_t)((int)blockIdx.x - (second ? a.blocks0 : 0));
    const int trow = threadIdx.x >> 3, tvec = threadIdx.x & 7;
    for (int rb = 0; rb < rank; rb += 16 * kRT) {
        f32x4 acc[kRT] = {};
        uint4 xq[kBatch], sq[kRT];
        const auto request = [&](int b) {   // tokens b .. b + 32 kBatch - 1 of the adapter
#pragma unroll
            for (int d = 0; d < kBatch; ++d) {
                const int j = b + 32 * d + trow;
                xq[d] = make_uint4(0, 0, 0, 0);
                if (j < count) xq[d] = eight_of(in + (int64_t)a.tokens.order[start + j] * C, c0 + 8 * tvec, C);
            }
#pragma unroll
            for (int v = 0; v < kRT; ++v) {
                const int i = threadIdx.x + 256 * v, j = b + i / (2 * kRT), r = rb + 8 * (i % (2 * kRT));
                sq[v] = make_uint4(0, 0, 0, 0);
                if (j < count && r < a.rpad) sq[v] = *reinterpret_cast<const uint4*>(s + (int64_t)j * a.rpad + r);
            }
        };
        if (count > 0) request(0);
        int buf = 0;
        for (int b = 0; b < count; b += 32 * kBatch, buf ^= 1) {
#pragma unroll
            for (int d = 0; d < kBatch; ++d) *reinterpret_cast<uint4*>(&in_tile[buf][(32 * d + trow) * kPitch + 8 * tvec]) = xq[d];
#pragma unroll
            for (int v = 0; v < kRT; ++v) {
                const int i = threadIdx.x + 256 * v;
                *reinterpret_cast<uint4*>(&s_tile[buf][i / (2 * kRT) * kSPitch + 8 * (i % (2 * kRT))]) = sq[v];
            }
            if (b + 32 * kBatch < count) request(b + 32 * kBatch);
            __syncthreads();   // the tiles are complete; those of the other buffer have been read by everyone
#pragma unroll
            for (int d = 0; d < kBatch; ++d) {
                if (b + 32 * d >= count) break;   // the same for the workgroup
                const auto operand = [&](const uint16_t* tile, int pitch, int c) {
                    const uint16_t* col = tile + (32 * d + 8 * g + (i16 >> 2)) * pitch + c + 4 * (i16 & 3);
                    const uint2 lo = lds_read_tr4(col), hi = lds_read_tr4(col + 4 * pitch);
                    return as_bf16x8(make_uint4(lo.x, lo.y, hi.x, hi.y));
                };
                const bf16x8 x = operand(in_tile[buf], kPitch, 16 * wave);
#pragma unroll
                for (int rt = 0; rt < kRT; ++rt) {
                    const bf16x8 f = operand(s_tile[buf], kSPitch, 16 * rt);
                    acc[rt] = second ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, f, acc[rt], 0, 0, 0) : __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, x, acc[rt], 0, 0, 0);
                }
            }
        }
        __syncthreads();   // before the next pass writes buffer 0 again
        // lane holds column i16 and rows 4 g + e of its accumulators: rows are columns of dy (dB) or ranks (dA)
#pragma unroll
        for (int rt = 0; rt < kRT; ++rt) {
            const int r = rb + 16 * rt + (second ? i16 : 4 * g);
            const int64_t c = c0 + 16 * wave + (second ? 4 * g : i16);
            if (r >= rank || c >= C) continue;
            const int64_t left = second ? C - c : rank - r;
            uint16_t* to = second ? out + (int64_t)r * C + c : out + c * rank + r;
            uint16_t e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = f32_to_bf16_rne(acc[rt][i]);
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

// ---- host

namespace {

size_t padded(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// Slices of a contraction of C columns: workgroups enough for the chip, two steps of 32 columns a wave at least (one where tokens are few).
int slices_of(int64_t C, int64_t tiles, int64_t want, int64_t steps_least) {
    const int64_t steps = (C + 31) / 32;
    int64_t s = (want + tiles - 1) / tiles;
    if (s > steps / steps_least) s = steps / steps_least;
    if (s > 32) s = 32;
    return s < 1 ? 1 : (int)s;
}

Tokens tokens_of(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p) {
    const char* w = static_cast<const char*>(a.workspace);
    const auto at = [&](size_t offset) { return reinterpret_cast<const int32_t*>(w + offset); };
    return p.direct ? Tokens{a.list, a.ids, nullptr, nullptr, nullptr, (int)a.T, (int)a.n}
                    : Tokens{a.list, a.ids, at(p.order), at(p.starts), at(p.counts), (int)a.T, (int)a.n};
}

void launch_order(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p) {
    char* w = static_cast<char*>(a.workspace);
    hipLaunchKernelGGL(order_tokens_kernel, dim3((unsigned)a.n + 2), dim3(1024), 0, a.stream, a.ids, (int)a.T, (int)a.n,
                       reinterpret_cast<int32_t*>(w + p.order), reinterpret_cast<int32_t*>(w + p.starts), reinterpret_cast<int32_t*>(w + p.counts));
}

void launch_narrow(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p, bool x_too, bool dy_too) {
    char* w = static_cast<char*>(a.workspace);
    NarrowArgs n{tokens_of(a, p), {a.x, a.dy}, {a.K, a.N}, {reinterpret_cast<float*>(w + p.part_x), reinterpret_cast<float*>(w + p.part_dy)},
                 {x_too ? p.slices_x : 0, dy_too ? p.slices_dy : 0}, p.t_rows, p.rpad};
    const dim3 grid((unsigned)p.tiles, (unsigned)(n.slices[0] + n.slices[1]));
    const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, a.stream, n); };
    if (p.direct) p.rpad <= 16 ? run(narrow_kernel<true, 1, 1>) : p.rpad <= 32 ? run(narrow_kernel<true, 1, 2>) : run(narrow_kernel<true, 1, 4>);
    else p.rpad <= 16 ? run(narrow_kernel<false, 4, 1>) : p.rpad <= 32 ? run(narrow_kernel<false, 4, 2>) : run(narrow_kernel<false, 4, 4>);
}

template <bool kFactorA>
void launch_wide(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p, const float* part, const uint16_t* t, int slices, int64_t C) {
    int64_t per_group = 256;
    while (p.tiles * ((C + 2 * per_group - 1) / (2 * per_group)) >= 1024) per_group *= 2;
    const WideArgs w{tokens_of(a, p), part, t, slices, p.t_rows, p.rpad, C, per_group, a.base, a.out};
    const dim3 grid((unsigned)p.tiles, (unsigned)((C + per_group - 1) / per_group));
    const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, a.stream, w); };
    if constexpr (!kFactorA)
        if (p.direct) return p.rpad <= 64 ? run(wide_kernel<true, 1, 64, false>) : run(wide_kernel<true, 1, 256, false>);
    p.rpad <= 64 ? run(wide_kernel<false, 4, 64, kFactorA>) : run(wide_kernel<false, 4, 256, kFactorA>);
}

}  // namespace

RequestAdaptersPlan request_adapters_plan(int64_t T, int64_t K, int64_t N, int64_t n, int64_t max_rank, bool backward, bool want_dadb) {
    RequestAdaptersPlan p{};
    p.direct = !backward && T <= kDirectTokens;
    p.rows = p.direct ? 16 : kTileTokens;
    const int64_t groups = n + 2 < T ? n + 2 : T;   // that hold a token
    p.tiles = p.direct ? T : T / kTileTokens + groups;
    p.t_rows = T;
    p.rpad = (int)((max_rank + 15) / 16 * 16);
    if (p.rpad == 0) p.rpad = 16;
    const int64_t live = p.direct ? (n < T ? n : T) : (T + kTileTokens - 1) / kTileTokens + groups / 2;   // tiles to expect
    p.slices_x = slices_of(K, live > 0 ? live : 1, p.direct ? 512 : 768, p.direct ? 4 : 8);
    p.slices_dy = slices_of(N, live > 0 ? live : 1, p.direct ? 512 : 768, p.direct ? 4 : 8);
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
    }
    const size_t row = (size_t)T * p.rpad;
    if (!backward || want_dadb) p.part_x = take(row * 4 * p.slices_x);
    if (backward) {
        p.part_dy = take(row * 4 * p.slices_dy);
        if (want_dadb) p.t_x = take(row * 2);
        p.t_dy = take(row * 2);
    }
    p.bytes = at;
    return p;
}

hipError_t launch_request_adapters(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p) {
    if (!p.direct) launch_order(a, p);
    launch_narrow(a, p, true, false);
    launch_wide<false>(a, p, reinterpret_cast<const float*>(static_cast<char*>(a.workspace) + p.part_x), nullptr, p.slices_x, a.N);
    return hipGetLastError();
}

hipError_t launch_request_adapters_backward(const RequestAdaptersArgs& a, const RequestAdaptersPlan& p) {
    char* w = static_cast<char*>(a.workspace);
    uint16_t *t_x = reinterpret_cast<uint16_t*>(w + p.t_x), *t_dy = reinterpret_cast<uint16_t*>(w + p.t_dy);
    launch_order(a, p);
    if (a.T > 0) {
        launch_narrow(a, p, a.want_dadb, true);
        const SumArgs s{{reinterpret_cast<const float*>(w + p.part_dy), reinterpret_cast<const float*>(w + p.part_x)}, {t_dy, t_x}, {p.slices_dy, p.slices_x}, a.T * p.rpad};
        hipLaunchKernelGGL(sum_slices_kernel, dim3((unsigned)((s.count / 4 + 255) / 256), a.want_dadb ? 2 : 1), dim3(256), 0, a.stream, s);
        if (a.out != nullptr) launch_wide<true>(a, p, nullptr, t_dy, 0, a.K);
    }
    if (a.want_dadb) {
        const int blocks0 = (int)((a.K + 63) / 64), blocks1 = (int)((a.N + 63) / 64);
        const OuterArgs o{tokens_of(a, p), {a.x, a.dy}, {t_dy, t_x}, {a.K, a.N}, p.rpad, blocks0};
        const dim3 grid((unsigned)(blocks0 + blocks1), (unsigned)a.n);
        const auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, a.stream, o); };
        p.rpad <= 16 ? run(outer_kernel<1>) : p.rpad <= 32 ? run(outer_kernel<2>) : run(outer_kernel<4>);
    }
    return hipGetLastError();
}

}  // namespace salr
