// Softmax cross entropy of a language-model head, l = h w^T, without storing the logits:
//
//   loss_t = lse_t - l[t, target_t],   dh = G w,   dw = G^T h,   G = grad_t (softmax(l) - onehot(target))
//
// Without dw one pass over the vocabulary makes loss and dh (two products, what the result needs).  It goes in pieces of the
// vocabulary; in each
//   logits  a tile of 256 tokens x 256 columns at a time: E = 2^(l log2 e - M_tile) in bf16, M_tile a multiple of 128 near the
//           tile's largest exponent of the row, and the row's sum of E in fp32;
//   rows    M_row = the running maximum of the M_tile, the running sum; E of tiles with another M is brought to M_row, a subtraction
//           from its exponents (what falls below bf16's normal numbers is lost);
//   dh      sums = 2^(M_row before - M_row) sums + E w.
// The column of the target is left out of E and of the sum S' and joins at the end, dh = grad (E w - S' w_target) / (S' + e_target):
// a token that is predicted well has 1 - p_target = S' / S to full precision, not the difference of rounded numbers.
//
// With dw G is needed itself.  Where the vocabulary is one piece (up to 128 M logits), E is kept in fp32 and G made from it; else the statistics come
// first (a product more, on the logits: 1131 us against 925 for 1111 x 2720 x 50003) and the pieces hold G.
//
// Sums and statistics are fp32; E and G are rounded once to bf16, as operands of the matrix cores.
// A masked token (target < 0) has loss 0 and gradient 0 whatever its hidden state holds.
#include "salr_device.hpp"
#include "salr_internal.hpp"
#include "salr_linear_common.hpp"
#include "salr_tile_product.hpp"

namespace salr {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

enum CeMode { kStatistics, kExponentials, kExponentials32, kGradients };   // what a tile of logits becomes: nothing but its statistics, E in bf16 or fp32, G

struct CeRow {   // of a token, once its statistics are complete
    float M, alpha, beta;   // G = alpha 2^(l log2 e - M), of the target's column -beta; M at or above the reference of E by a whole number
    int32_t live;
};

__device__ __forceinline__ uint32_t pack_two_bf16(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}

// The reference of a tile's row: the multiple of 128 next to its largest exponent, so that its E lie below 2^65.  bf16 and fp32 hold those
// as well as numbers below 1, and hardly any row has tiles of two references: with logits within 44 of zero it is 0.  What is 2^-62 of the row's largest
// and less may be 0 then, which a sum over the words does not see.  E in fp32, which becomes operands of a sum over the tokens (dw: a word's may all be
// small), is kept from the largest exponent itself on, down to 2^-126 of it.
// Logits of 2^30 and more (-1e30 rules a word out) are 128 or further apart where they differ, and fp32 has no multiples of 128 much above: there
// the reference is twice the largest logit, E 1 where l is that one, else 0.  (2^127 and more counts as infinite.)
constexpr float kReferenceStep = 128.f, kLargeLogit = 0x1p30f, kLargeReference = 2.f * kLargeLogit;
template <int kMode>
__device__ __forceinline__ float tile_exponent(float most) {
    constexpr float kStep = kMode == kExponentials32 ? 1.f : kReferenceStep;
    return fabsf(most) < kLargeLogit ? kStep * rintf(most * (kLog2e / kStep)) : 2.f * most;
}

// x 2^by for a whole `by` that may be -infinity; 2^-128 is no normal number, so not by multiplying.
__device__ __forceinline__ float times_power(float x, float by) { return __builtin_amdgcn_ldexpf(x, (int)fminf(fmaxf(by, -1000.f), 1000.f)); }

// Of the four lanes that hold a row's columns: all of them get `with` of the four, without a trip through LDS.
template <class With>
__device__ __forceinline__ float over_groups(float x, With with) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = with(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return with(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// l = h w^T of one tile and what becomes of it.  `w`: the piece's first row, `columns` of it exist; `pitch`: of `out` [T][pitch].
// 2048 x 4096 x 131072, statistics: 1573 us a call, 1400 TFLOP/s (the product by itself, with its result stored, takes the library 1515 to 1545); E of
// 4096 x 32768: 830 us, 1325 TFLOP/s.  A tile of 256 x 256 has 7 us outside the k loop without E and 12 with it: start and first loads 3, the exponentials and
// statistics 4, E through LDS and out.  Up to 64 tokens the head's bytes count: 1 x 4096 x 131072 173 us, 6.2 TB/s.
template <class Shape, int kMode>
__global__ __launch_bounds__(Shape::kThreads) void ce_logits_kernel(const uint16_t* __restrict__ h, int64_t T, int64_t K, const uint16_t* __restrict__ w,
                                                        int64_t columns, int64_t first, const int64_t* __restrict__ targets, int m_tiles, int n_tiles,
                                                        float2* __restrict__ stats, float* __restrict__ target_logit, const CeRow* __restrict__ rows,
                                                        void* __restrict__ out, int64_t pitch) {
    constexpr int kMI = Shape::kMI, kNI = Shape::kNI, kWN = Shape::kWN, kM = Shape::kM, kN = Shape::kN;
    constexpr int kOutPitch = 2 * kN + 16;   // bytes of a row of E in LDS
    constexpr bool kBf16 = kMode == kExponentials || kMode == kGradients;
    constexpr int kTile = kBf16 ? kM * kOutPitch : 0;
    constexpr int kEnd = kTile + 2 * kWN * kM * 4;
    __shared__ __attribute__((aligned(16))) char lds[kEnd > Shape::kLdsBytes ? kEnd : Shape::kLdsBytes];
    const TilePlace at(m_tiles, n_tiles, 1);
    if (!at.any) return;   // uniform for the workgroup, before any barrier
    const int64_t m0 = (int64_t)at.mt * kM, n0 = (int64_t)at.nt * kN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / kWN, wn = wave % kWN, i16 = lane & 15, g = lane >> 4;

    f32x4 acc[kMI][kNI];
#pragma unroll
    for (int i = 0; i < kMI; ++i)
#pragma unroll
        for (int j = 0; j < kNI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const auto target_at = [&](int i) {
        const int64_t m = m0 + 16 * (wm * kMI + i) + i16;
        return m < T ? targets[m] : -1;
    };
    // Targets come during the products (2048 x 4096 x 131072 1566 us, 1607 if afterwards), but up to 32 tokens not ahead of the head (24 x 8192 x
    // 32000 108 us so, 107 afterwards).
    constexpr bool kAhead = kM > 32;
    int64_t target_of[kMI];
    if constexpr (kAhead) {
#pragma unroll
        for (int i = 0; i < kMI; ++i) target_of[i] = target_at(i);
    }
    const TileSource<false, kM, Shape::kWaves> hs(h + m0 * K, K, T - m0, K, wave, lane);
    const TileSource<false, kN, Shape::kWaves> ws(w + n0 * K, K, columns - n0, K, wave, lane);
    tile_product<Shape, false, false>(hs, ws, 0, (int)((K + kProductStep - 1) / kProductStep), lds, acc);

    // A lane holds columns 16 (wn kNI + j) + 4 g + r of row 16 (wm kMI + i) + i16.  What few lanes have to do (columns past the end, the
    // target's) is tested once for a wave: over a tile the exponentials alone are 2 us, every other instruction an element 0.5.
    float* largest = reinterpret_cast<float*>(lds + kTile);   // [kWN][kM]
    float* sums = largest + kWN * kM;
    const int here = (int)(columns - n0 < kN ? columns - n0 : kN);   // columns that exist
    const int first_n = 16 * wn * kNI + 4 * g;
    if (here < kN) {
#pragma unroll
        for (int i = 0; i < kMI; ++i)
#pragma unroll
            for (int j = 0; j < kNI; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (first_n + 16 * j + r >= here) acc[i][j][r] = -__builtin_inff();
    }
    int target[kMI];   // column in this wave's part of the tile, from the lane's first one on; others: none of its columns
#pragma unroll
    for (int i = 0; i < kMI; ++i) {
        const int64_t m = m0 + 16 * (wm * kMI + i) + i16;
        const int64_t t = (kAhead ? target_of[i] : target_at(i)) - first - n0;
        target[i] = t >= 0 && t < here ? (int)t - first_n : -1;
        if constexpr (kMode != kGradients) {
            if (__any(target[i] >= 0 && target[i] < 16 * kNI)) {
#pragma unroll
                for (int j = 0; j < kNI; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (16 * j + r == target[i]) {
                            target_logit[m] = acc[i][j][r];
                            acc[i][j][r] = -__builtin_inff();
                        }
            }
        }
    }
    if constexpr (kMode != kGradients) {
#pragma unroll
        for (int i = 0; i < kMI; ++i) {
            float most = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < kNI; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) most = fmaxf(most, acc[i][j][r]);
            most = over_groups(most, [](float a, float b) { return fmaxf(a, b); });
            if (g == 0) largest[wn * kM + 16 * (wm * kMI + i) + i16] = most;
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kMI; ++i) {
        const int row = 16 * (wm * kMI + i) + i16;
        float M, alpha = 1.f;
        CeRow of{};
        if constexpr (kMode == kGradients) {
            if (m0 + row < T) of = rows[m0 + row];
            M = of.M, alpha = of.alpha;
            if (__any(!of.live)) {   // a masked token: M and alpha are 0 in its CeRow, l here, whatever h held
#pragma unroll
                for (int j = 0; j < kNI; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] = of.live ? acc[i][j][r] : 0.f;
            }
        } else {
            float most = largest[row];
#pragma unroll
            for (int q = 1; q < kWN; ++q) most = fmaxf(most, largest[q * kM + row]);
            M = tile_exponent<kMode>(most);
            M = M == -__builtin_inff() ? 0.f : M;   // (nothing in the row: every E is 2^-inf)
        }
        const bool large = fabsf(M) >= kLargeReference;   // E = 2^(l - that logit): 1 or 0
        const float slope = large ? 1.f : kLog2e, origin = large ? 0.5f * M : M;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < kNI; ++j) {
            float e[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                e[r] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], slope, -origin));
                if constexpr (kMode == kGradients) e[r] *= alpha;
            }
            if constexpr (kMode == kGradients) {
                if (__any(target[i] >= 16 * j && target[i] < 16 * j + 4)) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) e[r] = 16 * j + r == target[i] ? -of.beta : e[r];
                }
            }
            sum += (e[0] + e[1]) + (e[2] + e[3]);
            if constexpr (kMode == kExponentials32) {
                if (m0 + row < T) *reinterpret_cast<float4*>(static_cast<float*>(out) + (m0 + row) * pitch + n0 + first_n + 16 * j) = make_float4(e[0], e[1], e[2], e[3]);
            }
            if constexpr (kBf16)
                *reinterpret_cast<uint2*>(lds + row * kOutPitch + 32 * (wn * kNI + j) + 8 * g) = make_uint2(pack_two_bf16(e[0], e[1]), pack_two_bf16(e[2], e[3]));
        }
        if constexpr (kMode != kGradients) {
            sum = over_groups(sum, [](float a, float b) { return a + b; });
            if (g == 0) sums[wn * kM + row] = sum;
        }
    }
    __syncthreads();
    if constexpr (kMode != kGradients) {
        for (int row = threadIdx.x; row < kM; row += Shape::kThreads) {
            if (m0 + row >= T) break;
            float most = largest[row], sum = sums[row];
#pragma unroll
            for (int q = 1; q < kWN; ++q) {
                most = fmaxf(most, largest[q * kM + row]);
                sum += sums[q * kM + row];
            }
            stats[(int64_t)at.nt * T + m0 + row] = make_float2(tile_exponent<kMode>(most), sum);
        }
    }
    if constexpr (kBf16) {
        // 16 bytes a lane; of wide tiles not kept in this XCD's cache, where h and w are: 784 x 768 x 106368 with dh 327 us for 336, 4096 x 4096 x
        // 131072 1 % (a small E is: 48 x 512 x 4099 24.8 us and 25.3)
        constexpr int kVecs = kN / 8, kRowsAtOnce = Shape::kThreads / kVecs;
        const int vec = threadIdx.x % kVecs;
        for (int row = threadIdx.x / kVecs; row < kM; row += kRowsAtOnce) {
            if (m0 + row >= T) break;
            const u32x4 q = *reinterpret_cast<const u32x4*>(lds + row * kOutPitch + 16 * vec);
            u32x4* to = reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + (m0 + row) * pitch + n0 + 8 * vec);
            if constexpr (kN == 256) __builtin_nontemporal_store(q, to);
            else *to = q;
        }
    }
}

struct CeRowArgs {
    const float2* stats;       // [n_tiles][T]: M and sum of a tile
    int n_tiles;
    bool first, last;          // piece of the vocabulary
    float2* running;           // [T]: M and sum so far
    float* rescale;            // [T]: M before - M now
    uint16_t* e;               // E of the piece, brought to M now where a tile's M is another; null: there is none
    int64_t pitch;
    int width;                 // columns of a tile: 64 or 256
    const float* target_logit;
    const int64_t* targets;
    const float* grad_loss;    // null: ones
    int64_t T, V;
    float* loss;
    float* lse;
    CeRow* rows;
};

// Maximum of references and the sum with respect to it.  References are whole numbers, -infinity (no column) or +infinity.
struct CeSum {
    float M, sum, least;   // least: smallest reference of a tile that has one
    __device__ __forceinline__ void add(float M2, float sum2, float least2) {
        const float top = fmaxf(M, M2), M_ref = top == -__builtin_inff() ? 0.f : top;
        sum = times_power(sum, M - M_ref) + times_power(sum2, M2 - M_ref);
        M = top;
        least = fminf(least, least2);
    }
};

// kRows rows a workgroup, 1024 / kRows threads a row; the tiles dealt out to them in turn.  4 to 7 us: two trips to memory and a launch.
template <int kRows>
__global__ __launch_bounds__(1024) void ce_rows_kernel(CeRowArgs a) {
    constexpr int kParts = 1024 / kRows;
    __shared__ CeSum part[16][kRows];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = threadIdx.x % kRows, first_tile = threadIdx.x / kRows;
    const int64_t t = (int64_t)blockIdx.x * kRows + row;
    const bool here = t < a.T;
    const float inf = __builtin_inff();
    CeSum all{-inf, 0.f, inf};
    if (here) {
#pragma unroll 8
        for (int n = first_tile; n < a.n_tiles; n += kParts) {
            const float2 s = a.stats[(int64_t)n * a.T + t];
            all.add(s.x, s.y, s.x > -inf ? s.x : inf);
        }
    }
#pragma unroll
    for (int o = kRows; o < 64; o <<= 1) {
        const CeSum other{__shfl_xor(all.M, o), __shfl_xor(all.sum, o), __shfl_xor(all.least, o)};
        all.add(other.M, other.sum, other.least);
    }
    if (lane < kRows) part[wave][row] = all;
    __syncthreads();
    const float2 before = here && !a.first ? a.running[t] : make_float2(-inf, 0.f);
    all = CeSum{before.x, before.y, inf};
    for (int q = 0; q < 16; ++q) all.add(part[q][row].M, part[q][row].sum, part[q][row].least);
    const float M = all.M == -inf ? 0.f : all.M, sum = all.sum;
    if (a.e != nullptr && __any(here && all.least < M)) {
        // The exponents of E in tiles with a reference below the row's, lowered by the difference: exact, but for what then lies below bf16's normal
        // numbers (2^-62 of the row's largest and less: 0, or another number as small).  The wave goes through such tiles
        // four at a time, its lanes through the columns.
        for (int n0 = 0; n0 < a.n_tiles; n0 += kParts) {
            const int n = n0 + first_tile;
            const float reference = here && n < a.n_tiles ? a.stats[(int64_t)n * a.T + t].x : -inf;   // (-infinity: every E is 0)
            const float behind = reference > -inf ? M - reference : 0.f;
            uint64_t todo = __ballot(behind > 0.f);
            while (todo != 0) {
                uint2* at[4] = {};
                uint2 q[4];
                uint32_t by[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int of = __ffsll((unsigned long long)todo) - 1;   // the same in all lanes; -1: no more
                    if (of < 0) break;
                    todo &= todo - 1;
                    const int64_t at_row = (int64_t)blockIdx.x * kRows + (wave * 64 + of) % kRows, at_tile = n0 + (wave * 64 + of) / kRows;
                    by[u] = __shfl(behind, of) > kReferenceStep ? 0xFFFFFFFFu : ((uint32_t)(int)kReferenceStep << 7) * 0x00010001u;
                    if (4 * lane >= a.width) continue;
                    at[u] = reinterpret_cast<uint2*>(a.e + at_row * a.pitch + at_tile * a.width) + lane;
                    q[u] = *at[u];
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (at[u] == nullptr) continue;
                    const u16x2 lower = __builtin_bit_cast(u16x2, by[u]);
                    q[u].x = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, q[u].x), lower));
                    q[u].y = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, q[u].y), lower));
                    *at[u] = q[u];
                }
            }
        }
    }
    if (threadIdx.x >= kRows || !here) return;
    a.running[t] = make_float2(all.M, sum);
    a.rescale[t] = before.x - M;
    if (!a.last) return;
    // S' = sum of 2^(l log2 e - M) over the other columns, e the target's (M may lie below the target's own exponent)
    const int64_t target = a.targets[t];
    const float nan = __builtin_nanf("");
    float loss = 0.f, lse = 0.f, alpha = 0.f, beta = 0.f, above = M;
    if (target >= a.V) {
        loss = lse = alpha = beta = nan;
    } else if (target >= 0) {
        const float l = a.target_logit[t];
        const bool large = fabsf(M) >= kLargeReference;   // M is twice a logit then
        float up = fmaf(l, kLog2e, -M);
        if (large) {
            const float off = l - 0.5f * M;
            up = off > kLargeLogit && l < inf ? kLargeLogit : off * kLog2e;
        }
        const float top = up > 0.f || all.M == -inf ? ceilf(up) : 0.f;
        const float e = __builtin_amdgcn_exp2f(up - top), rest = times_power(sum, -top), total = rest + e;
        const float gl = a.grad_loss != nullptr ? a.grad_loss[t] : 1.f;
        lse = kLn2 * (M + top);
        if (large) lse = top > 0.f ? l : 0.5f * M;
        lse += logf(total);
        const float ratio = rest / e;   // (where the target is far below the others it leaves fp32)
        loss = ratio < 1e6f ? log1pf(ratio) : lse - l;
        // 2^-top and the exponent of the sum go to M, as long as that is exact, so that 2^(l log2 e - M) is as small as G is and no smaller:
        // alpha times 2^-top would leave fp32 where the target is far above the others, 2^(l log2 e - M) where M is far above them all
        const bool exact = fabsf(M) <= 0x1p23f && top <= 1000.f && total > 0.f && total < inf;
        above = exact ? M + top + (float)__builtin_amdgcn_frexp_expf(total) : M;
        alpha = sum == 0.f ? 0.f : times_power(gl / (exact ? __builtin_amdgcn_frexp_mantf(total) : total), exact ? 0.f : -top);
        beta = gl * (rest / total);
        if (!(total > 0.f && total < inf)) loss = lse = alpha = beta = nan;
    }
    a.loss[t] = loss;
    a.lse[t] = lse;
    a.rows[t] = CeRow{target >= 0 ? above : 0.f, alpha, beta, target >= 0};   // (2^-M of a masked token may leave fp32, and 0 times infinity is NaN)
}

// G from E in fp32 and the tiles' references, eight columns a thread, up to a whole step of columns.  Bound by memory (1111 x 50003: 60 us, 5.6 TB/s).
// E is read for the last time, not kept in the caches: 2000 x 2048 x 65536 1099 us a call for 1128, smaller ones level.
__global__ __launch_bounds__(256) void ce_gradients_kernel(const float* __restrict__ e, int64_t T, int64_t columns, int64_t pitch, const float2* __restrict__ stats,
                                                           int width, const CeRow* __restrict__ rows, const int64_t* __restrict__ targets,
                                                           uint16_t* __restrict__ out) {
    const int64_t n = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 8, t = blockIdx.x;
    if (n >= (columns + kProductStep - 1) / kProductStep * kProductStep) return;
    const CeRow of = rows[t];
    const int64_t target = targets[t];
    const f32x4* from = reinterpret_cast<const f32x4*>(e + t * pitch + n);
    const f32x4 a = __builtin_nontemporal_load(from), b = __builtin_nontemporal_load(from + 1);
    const float by = stats[n / width * T + t].x - of.M;
    float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
    for (int c = 0; c < 8; ++c) x[c] = n + c == target ? -of.beta : of.alpha * times_power(x[c], by);
    const uint4 q = make_uint4(pack_two_bf16(x[0], x[1]), pack_two_bf16(x[2], x[3]), pack_two_bf16(x[4], x[5]), pack_two_bf16(x[6], x[7]));
    *reinterpret_cast<uint4*>(out + t * pitch + n) = of.live ? q : make_uint4(0, 0, 0, 0);
}

// sums = 2^rescale sums + E w over the columns of a piece (contracted), slice kz of them.  `rescale` null: zeros.
template <class Shape>
__global__ __launch_bounds__(Shape::kThreads) void ce_dh_kernel(const uint16_t* __restrict__ e, int64_t T, int64_t pitch, const uint16_t* __restrict__ w,
                                                    int64_t columns, int64_t K, int m_tiles, int n_tiles, int slices, const float* __restrict__ rescale,
                                                    bool first, float* __restrict__ sums) {
    constexpr int kMI = Shape::kMI, kNI = Shape::kNI, kWN = Shape::kWN, kM = Shape::kM;
    __shared__ __attribute__((aligned(16))) char lds[Shape::kLdsBytes];
    const TilePlace at(m_tiles, n_tiles, slices);
    if (!at.any) return;
    const int64_t m0 = (int64_t)at.mt * kM, n0 = (int64_t)at.nt * 256;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / kWN, wn = wave % kWN, i16 = lane & 15, g = lane >> 4;
    const int64_t steps = (columns + kProductStep - 1) / kProductStep;   // (E is written in whole steps)
    f32x4 acc[kMI][kNI];
#pragma unroll
    for (int i = 0; i < kMI; ++i) {
        const int64_t m = m0 + 16 * (wm * kMI + i) + i16;
        const float by = !first && m < T && rescale != nullptr ? rescale[m] : 0.f;
#pragma unroll
        for (int j = 0; j < kNI; ++j) {
            const int64_t n = n0 + 16 * (wn * kNI + j) + 4 * g;
            f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
            if (!first && m < T && n < K) {
                v = *reinterpret_cast<const f32x4*>(sums + ((int64_t)at.kz * T + m) * K + n);
#pragma unroll
                for (int r = 0; r < 4; ++r) v[r] = times_power(v[r], by);
            }
            acc[i][j] = v;
        }
    }
    const TileSource<false, kM, Shape::kWaves> es(e + m0 * pitch, pitch, T - m0, pitch, wave, lane);
    const TileSource<true, 256, Shape::kWaves> ws(w + n0, K, K - n0, columns, wave, lane);
    tile_product<Shape, false, true>(es, ws, (int)(steps * at.kz / slices), (int)(steps * (at.kz + 1) / slices), lds, acc);
#pragma unroll
    for (int i = 0; i < kMI; ++i) {
        const int64_t m = m0 + 16 * (wm * kMI + i) + i16;
#pragma unroll
        for (int j = 0; j < kNI; ++j) {
            const int64_t n = n0 + 16 * (wn * kNI + j) + 4 * g;
            if (m < T && n < K) *reinterpret_cast<f32x4*>(sums + ((int64_t)at.kz * T + m) * K + n) = acc[i][j];
        }
    }
}

// dh from the slices' sums, eight columns a thread.  kPlain: the sums are dh itself.  Bound by memory (4096 x 4096, one slice: 21 us, 5.6 TB/s).
template <bool kPlain>
__global__ __launch_bounds__(256) void ce_dh_finish_kernel(const float* __restrict__ sums, int slices, int64_t T, int64_t K, const CeRow* __restrict__ rows,
                                                           const float2* __restrict__ running, const int64_t* __restrict__ targets, int64_t V,
                                                           const uint16_t* __restrict__ w, uint16_t* __restrict__ dh) {
    const int64_t per_row = K / 8, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= T * per_row) return;
    const int64_t t = id / per_row, k = (id - t * per_row) * 8;
    const int64_t target = targets[t];
    const CeRow of = rows[t];
    float x[8] = {};
#pragma unroll 4
    for (int z = 0; z < slices; ++z) {
        const float4* from = reinterpret_cast<const float4*>(sums + ((int64_t)z * T + t) * K + k);
        const float4 a = from[0], b = from[1];
        x[0] += a.x, x[1] += a.y, x[2] += a.z, x[3] += a.w, x[4] += b.x, x[5] += b.y, x[6] += b.z, x[7] += b.w;
    }
    if constexpr (!kPlain) {
        const float reference = running[t].x, by = (reference == -__builtin_inff() ? 0.f : reference) - of.M;   // of E, below of.M
        const uint4 wt = target >= 0 && target < V ? *reinterpret_cast<const uint4*>(w + target * K + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int c = 0; c < 8; ++c) x[c] = times_power(of.alpha * x[c], by) - of.beta * bf16_bits_to_f32(unit_elem(wt, c));
    }
    uint4 q = make_uint4(pack_two_bf16(x[0], x[1]), pack_two_bf16(x[2], x[3]), pack_two_bf16(x[4], x[5]), pack_two_bf16(x[6], x[7]));
    if (target < 0) q = make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4*>(dh + t * K + k) = q;
}

// dw of a piece: G^T h, both operands across the contraction.  1111 x 2720 x 50003: 279 us, 1083 TFLOP/s; of the 34 us of a tile its 18 steps take 26.
// With few tokens the stores count: 315 x 7872 x 44416 7 us of steps in the 16 of a tile.
template <class Shape>
__global__ __launch_bounds__(Shape::kThreads) void ce_dw_kernel(const uint16_t* __restrict__ gr, int64_t T, int64_t pitch, const uint16_t* __restrict__ h, int64_t K,
                                                    int64_t columns, int m_tiles, int n_tiles, uint16_t* __restrict__ dw) {
    constexpr int kMI = Shape::kMI, kNI = Shape::kNI, kWN = Shape::kWN;
    __shared__ __attribute__((aligned(16))) char lds[Shape::kLdsBytes];
    const TilePlace at(m_tiles, n_tiles, 1);
    if (!at.any) return;
    const int64_t m0 = (int64_t)at.mt * 256, n0 = (int64_t)at.nt * 256;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / kWN, wn = wave % kWN, i16 = lane & 15, g = lane >> 4;
    f32x4 acc[kMI][kNI];
#pragma unroll
    for (int i = 0; i < kMI; ++i)
#pragma unroll
        for (int j = 0; j < kNI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const TileSource<true, 256, Shape::kWaves> gs(gr + m0, pitch, pitch - m0, T, wave, lane);
    const TileSource<true, 256, Shape::kWaves> hs(h + n0, K, K - n0, T, wave, lane);
    tile_product<Shape, true, true>(gs, hs, 0, (int)((T + kProductStep - 1) / kProductStep), lds, acc);
    // through LDS, so that rows leave as whole vectors, side by side, and not into the caches, where G and h are (315 x 7872 x 44416 639 us a call for 668)
    constexpr int kOutPitch = 512 + 16;
#pragma unroll
    for (int i = 0; i < kMI; ++i)
#pragma unroll
        for (int j = 0; j < kNI; ++j)
            *reinterpret_cast<uint2*>(lds + (16 * (wm * kMI + i) + i16) * kOutPitch + 32 * (wn * kNI + j) + 8 * g) =
                make_uint2(pack_two_bf16(acc[i][j][0], acc[i][j][1]), pack_two_bf16(acc[i][j][2], acc[i][j][3]));
    __syncthreads();
    const int vec = threadIdx.x % 32;
    if (n0 + 8 * vec >= K) return;
    for (int row = threadIdx.x / 32; row < 256 && m0 + row < columns; row += Shape::kThreads / 32)
        __builtin_nontemporal_store(*reinterpret_cast<const u32x4*>(lds + row * kOutPitch + 16 * vec), reinterpret_cast<u32x4*>(dw + (m0 + row) * K + n0 + 8 * vec));
}

// Hidden states with those of masked tokens as zeros: G is zero there, but not what it is multiplied by.
__global__ __launch_bounds__(256) void ce_live_rows_kernel(const uint16_t* __restrict__ h, const int64_t* __restrict__ targets, int64_t T, int64_t K,
                                                           uint16_t* __restrict__ out) {
    const int64_t per_row = K / 8, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= T * per_row) return;
    const uint4 q = reinterpret_cast<const uint4*>(h)[id];
    reinterpret_cast<uint4*>(out)[id] = targets[id / per_row] >= 0 ? q : make_uint4(0, 0, 0, 0);
}

// Tiles: 256 columns wide, or 64 where few tokens on a small vocabulary would leave CUs without one.
typedef TileShape<8, 4, 2, 4, 2, 3> Shape256;
typedef TileShape<4, 4, 2, 4, 3, 3> Shape128;
typedef TileShape<4, 2, 1, 8, 2, 2> Shape64;
typedef TileShape<2, 2, 1, 8, 2, 2> Shape32;
typedef TileShape<1, 2, 1, 8, 2, 2> Shape16;
typedef TileShape<4, 1, 2, 4, 3, 3> Narrow128;
typedef TileShape<4, 1, 1, 4, 4, 4> Narrow64;
typedef TileShape<2, 1, 1, 4, 4, 4> Narrow32;
typedef TileShape<1, 1, 1, 4, 4, 4> Narrow16;

constexpr int64_t kCus = 256;

// What a launch of `tiles` workgroups, one to a CU, takes in rounds of all CUs: a round that is part full costs 55 to 95 % of a full one
// (2048 to 32768 columns, 4096 deep: 640 tiles 2.7 rounds, 512 exactly 2, 128 tiles 0.85).
static double tile_rounds(int64_t tiles) {
    const double f = (double)(tiles % kCus) / kCus;
    return (double)(tiles / kCus) + (f > 0.0 ? 0.55 + 0.4 * f : 0.0);
}
// A round of tiles of 128 tokens against one of 256, a step of them takes 0.9 us and 1.56.  Logits: over 140 to 1100 tokens, 5760 to 100000 columns, 1024 and
// 4096 deep, what it chooses is within 1 % of the better one (with 0.6 or 0.56 up to 8 %).  dh: over such sizes 0.7 %
// from the best of several on average and 3 % at most (with 0.52 1.7 and 10, 0.56 and 0.64 0.8 and 4).
constexpr double kHalfTile = 0.58, kHalfTileDh = 0.6;

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

CePlan ce_plan(int64_t T, int64_t K, int64_t V, bool want_dh, bool want_dw) {
    CePlan p{};
    const bool pieces = want_dh || want_dw;
    const int64_t all = ceil_div(V, 256) * 256;
    p.piece = all;
    if (pieces) {
        const int64_t most = kCePieceBytes / (512 * (T > 0 ? T : 1)), cap = (most > 1 ? most : 1) * 256, n = ceil_div(all, cap);
        if (n > 0) p.piece = ceil_div(ceil_div(all, n), 256) * 256;
    }
    // tokens of a tile: the fewest that hold them all up to 64; from there the faster of 128 and 256
    // (66 against 91 us for 256 x 4096 x 32768, 214 against 194 for 777)
    const int64_t few = T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : 128, tiles = p.piece / 256;
    p.rows = few;
    if (T > 128 && tile_rounds(ceil_div(T, 256) * tiles) <= kHalfTile * tile_rounds(ceil_div(T, 128) * tiles)) p.rows = 256;
    p.m_tiles = ceil_div(T, p.rows);
    // columns of a tile: 64 where wide ones are too few to go round.  A CU draws about 45 GB/s from memory, so more of them count even where each
    // reads the tokens again (24 x 8192 x 32000: 104 us against 165; 256 x 4096 x 8192 35 against 48, but 512 x 4096 x 8192 53 against 53)
    p.width = few <= 64 ? (tiles < 384 ? 64 : 256) : p.rows == 128 && p.m_tiles * tiles <= 96 ? 64 : 256;
    p.dh_rows = few, p.slices = 1;
    if (want_dh) {
        const int64_t n_tiles = ceil_div(K, 256), steps = p.piece / kProductStep;
        if (few <= 64) {   // bound by memory: two workgroups to a CU, four steps at least
            while (n_tiles * p.slices < 384 && p.slices * 8 <= steps && p.slices < 64) p.slices *= 2;
        } else {
            // a slice more costs a pass over [T, K] in fp32, there and back
            double best = 0.0;
            for (int64_t rows = 128; rows <= (T > 128 ? 256 : 128); rows *= 2)
                for (int64_t s = 1; s <= 16 && s * 4 <= steps; ++s) {
                    const double us = tile_rounds(ceil_div(T, rows) * n_tiles * s) * (rows == 128 ? kHalfTileDh : 1.0) * 1.56 * (double)steps / s +
                                      (double)s * T * K * 8 / 5e6;
                    if (best == 0.0 || us < best) best = us, p.dh_rows = rows, p.slices = s;
                }
        }
    }
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_up_256(bytes);
        return here;
    };
    p.stats = take((size_t)((want_dh && !want_dw ? p.piece : all) / p.width) * T * sizeof(float2));
    p.running = take((size_t)T * sizeof(float2));
    p.rescale = take((size_t)T * 4);
    p.target_logit = take((size_t)T * 4);
    p.of_rows = take((size_t)T * sizeof(CeRow));
    if (pieces) p.e = take((size_t)T * p.piece * 2);
    p.holds_e32 = want_dw && p.piece == all;
    if (p.holds_e32) p.e32 = take((size_t)T * p.piece * 4);
    if (want_dh) p.sums = take((size_t)p.slices * T * K * 4);
    if (want_dw) p.h_live = take((size_t)T * K * 2);
    p.bytes = at;
    return p;
}

// Whether every launch of such a call keeps below 2^32 threads.  (Tiles are taken at the 512 threads of the largest; the narrow ones of 256 are
// few.)
bool ce_launches_fit(const CePlan& p, int64_t T, int64_t K, int64_t V, bool want_dh, bool want_dw) {
    const auto tiles_fit = [](int64_t a, int64_t b, int64_t c) {
        constexpr int64_t most = kMostThreads / 512 / kProductXcds * kProductXcds;   // (the grid is a multiple of the XCDs)
        return a == 0 || b == 0 || (b <= most / a && c <= most / (a * b));
    };
    const int64_t k_tiles = ceil_div(K, 256), columns = want_dh && !want_dw ? (V < p.piece ? V : p.piece) : V;
    if (!tiles_fit(p.m_tiles, ceil_div(columns, p.width), 1) || T > kMostThreads / 1024 * 64) return false;
    if (want_dh && !tiles_fit(ceil_div(T, p.dh_rows), k_tiles, p.slices)) return false;
    if (want_dw && !tiles_fit(ceil_div(V < p.piece ? V : p.piece, 256), k_tiles, 1)) return false;
    if ((want_dh || want_dw) && T * (K / 8) > kMostThreads / 256 * 256) return false;
    return !p.holds_e32 || T <= kMostThreads / 256;
}

namespace {

struct CeRun {   // one call
    const CeArgs& a;
    const CePlan& p;
    char* ws;
    template <class T>
    T* at(size_t offset) const { return reinterpret_cast<T*>(ws + offset); }

    template <class Shape, int kMode>
    void logits_on(int64_t first, int64_t columns) const {
        const int64_t tiles = (columns + Shape::kN - 1) / Shape::kN;
        hipLaunchKernelGGL((ce_logits_kernel<Shape, kMode>), dim3(product_grid(p.m_tiles * tiles)), dim3(Shape::kThreads), 0, a.stream, a.h, a.T, a.K,
                           a.w + first * a.K, columns, first, a.targets, (int)p.m_tiles, (int)tiles, at<float2>(p.stats), at<float>(p.target_logit),
                           at<const CeRow>(p.of_rows), kMode == kExponentials32 ? at<void>(p.e32) : at<void>(p.e), p.piece);
    }
    template <int kMode>
    void logits(int64_t first, int64_t columns) const {
        const bool narrow = p.width == 64;
        switch (p.rows) {
            case 16: return narrow ? logits_on<Narrow16, kMode>(first, columns) : logits_on<Shape16, kMode>(first, columns);
            case 32: return narrow ? logits_on<Narrow32, kMode>(first, columns) : logits_on<Shape32, kMode>(first, columns);
            case 64: return narrow ? logits_on<Narrow64, kMode>(first, columns) : logits_on<Shape64, kMode>(first, columns);
            case 128: return narrow ? logits_on<Narrow128, kMode>(first, columns) : logits_on<Shape128, kMode>(first, columns);
            default: return logits_on<Shape256, kMode>(first, columns);
        }
    }
    void rows(int64_t columns, bool first, bool last, bool with_e) const {
        CeRowArgs r{};
        r.stats = at<const float2>(p.stats);
        r.n_tiles = (int)((columns + p.width - 1) / p.width);
        r.first = first, r.last = last;
        r.running = at<float2>(p.running), r.rescale = at<float>(p.rescale);
        r.e = with_e ? at<uint16_t>(p.e) : nullptr, r.pitch = p.piece, r.width = (int)p.width;
        r.target_logit = at<const float>(p.target_logit), r.targets = a.targets, r.grad_loss = a.grad_loss;
        r.T = a.T, r.V = a.V, r.loss = a.loss, r.lse = a.lse, r.rows = at<CeRow>(p.of_rows);
        // fewer rows a workgroup where there are few: a thread's chain over the tiles stays short
        if (a.T <= 256) hipLaunchKernelGGL(ce_rows_kernel<4>, dim3((unsigned)ceil_div(a.T, 4)), dim3(1024), 0, a.stream, r);
        else if (a.T <= 4096) hipLaunchKernelGGL(ce_rows_kernel<16>, dim3((unsigned)ceil_div(a.T, 16)), dim3(1024), 0, a.stream, r);
        else hipLaunchKernelGGL(ce_rows_kernel<64>, dim3((unsigned)ceil_div(a.T, 64)), dim3(1024), 0, a.stream, r);
    }
    int n_tiles() const { return (int)((a.K + 255) / 256); }
    unsigned units() const { return (unsigned)((a.T * (a.K / 8) + 255) / 256); }   // workgroups with eight columns of a row a thread

    template <class Shape>
    void dh_on(int64_t first, int64_t columns, bool rescaled) const {
        const int64_t m_tiles = ceil_div(a.T, Shape::kM);
        hipLaunchKernelGGL(ce_dh_kernel<Shape>, dim3(product_grid(m_tiles * n_tiles() * p.slices)), dim3(Shape::kThreads), 0, a.stream, at<const uint16_t>(p.e),
                           a.T, p.piece, a.w + first * a.K, columns, a.K, (int)m_tiles, n_tiles(), (int)p.slices, rescaled ? at<const float>(p.rescale) : nullptr,
                           first == 0, at<float>(p.sums));
    }
    void dh(int64_t first, int64_t columns, bool rescaled) const {
        if (n_tiles() == 0) return;
        switch (p.dh_rows) {
            case 16: return dh_on<Shape16>(first, columns, rescaled);
            case 32: return dh_on<Shape32>(first, columns, rescaled);
            case 64: return dh_on<Shape64>(first, columns, rescaled);
            case 128: return dh_on<Shape128>(first, columns, rescaled);
            default: return dh_on<Shape256>(first, columns, rescaled);
        }
    }
    template <bool kPlain>
    void dh_finish() const {
        if (units() == 0) return;
        hipLaunchKernelGGL(ce_dh_finish_kernel<kPlain>, dim3(units()), dim3(256), 0, a.stream, at<const float>(p.sums), (int)p.slices, a.T, a.K,
                           at<const CeRow>(p.of_rows), at<const float2>(p.running), a.targets, a.V, a.w, a.dh);
    }
    void gradients() const {
        const unsigned across = (unsigned)ceil_div(a.V, 2048);
        hipLaunchKernelGGL(ce_gradients_kernel, dim3((unsigned)a.T, across), dim3(256), 0, a.stream, at<const float>(p.e32), a.T, a.V, p.piece, at<const float2>(p.stats),
                           (int)p.width, at<const CeRow>(p.of_rows), a.targets, at<uint16_t>(p.e));
    }
    void live_rows() const {
        if (units() == 0) return;
        hipLaunchKernelGGL(ce_live_rows_kernel, dim3(units()), dim3(256), 0, a.stream, a.h, a.targets, a.T, a.K, at<uint16_t>(p.h_live));
    }
    void dw(int64_t first, int64_t columns) const {
        if (n_tiles() == 0) return;
        const int64_t tiles = (columns + 255) / 256;
        hipLaunchKernelGGL(ce_dw_kernel<Shape256>, dim3(product_grid(tiles * n_tiles())), dim3(Shape256::kThreads), 0, a.stream, at<const uint16_t>(p.e), a.T, p.piece,
                           at<const uint16_t>(p.h_live), a.K, columns, (int)tiles, n_tiles(), a.dw + first * a.K);
    }
};

}  // namespace

hipError_t launch_cross_entropy(const CeArgs& a, void* workspace) {
    const CePlan p = ce_plan(a.T, a.K, a.V, a.dh != nullptr, a.dw != nullptr);
    const CeRun run{a, p, static_cast<char*>(workspace)};
    if (a.T == 0) {   // no tokens: dw is zero
        for (int64_t first = 0; first < a.V; first += p.piece) run.dw(first, a.V - first < p.piece ? a.V - first : p.piece);
        return hipGetLastError();
    }
    const bool one_pass = a.dh != nullptr && a.dw == nullptr;   // on E; else the statistics come first, and pieces of G where they are wanted
    if (!one_pass) {
        p.holds_e32 ? run.logits<kExponentials32>(0, a.V) : run.logits<kStatistics>(0, a.V);
        run.rows(a.V, true, true, false);
        if (a.dw == nullptr) return hipGetLastError();
        run.live_rows();
    }
    for (int64_t first = 0; first < a.V; first += p.piece) {
        const int64_t columns = a.V - first < p.piece ? a.V - first : p.piece;
        if (one_pass) {
            run.logits<kExponentials>(first, columns);
            run.rows(columns, first == 0, first + columns == a.V, true);
        } else if (p.holds_e32) {
            run.gradients();
        } else {
            run.logits<kGradients>(first, columns);
        }
        if (a.dh != nullptr) run.dh(first, columns, one_pass);
        if (a.dw != nullptr) run.dw(first, columns);
    }
    if (a.dh != nullptr) one_pass ? run.dh_finish<false>() : run.dh_finish<true>();
    return hipGetLastError();
}

}  // namespace salr
