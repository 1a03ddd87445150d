// Softmax cross entropy of a language-model head, l = h w^T, without keeping the logits:
//
//   loss_t = lse_t - l[t, target_t],   dh = G w,   dw = G^T h,   G = grad_t (softmax(l) - onehot(target))
//
// Without dw one pass over the vocabulary makes loss and dh (two products, what the result needs).  It goes in pieces of the
// vocabulary; in each
//   logits  a tile of 256 tokens x 256 columns at a time: E = 2^(l log2 e - M_tile) in bf16, M_tile a multiple of 128 near the
//           tile's largest exponent of the row, and the row's sum of E in fp32;
//   rows    M_row = the running maximum of the M_tile, the running sum; E of tiles with another M is brought to M_row, a subtraction
//           from its exponents;
//   dh      sums = 2^(M_row before - M_row) sums + E w.
// The column of the target is left out of E and of the sum S' and joins at the end, dh = grad (E w - S' w_target) / (S' + e_target):
// a token that is predicted well has 1 - p_target = S' / S to full precision, not the difference of rounded numbers.
//
// With dw G is needed itself, so the statistics come first (a third product, on the logits) and the pieces hold G.
//
// Sums and statistics are fp32; E and G are rounded once to bf16, as operands of the matrix cores.
// A masked token (target < 0) has loss 0 and gradient 0 whatever its hidden state holds.
#include "salr_device.hpp"
#include "salr_internal.hpp"
#include "salr_linear_common.hpp"
#include "salr_tile_product.hpp"

namespace salr {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

enum CeMode { kStatistics, kExponentials, kGradients };

struct CeRow {   // of a token, once its statistics are complete
    float M, alpha, beta;   // G = alpha 2^(l log2 e - M), of the target's column -beta
    int32_t live;
};

__device__ __forceinline__ uint32_t pack_two_bf16(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}

// The reference of a tile's row: the multiple of 128 next to its largest exponent, so that its E lie below 2^65.  bf16 and fp32 hold those
// as well as numbers below 1, and hardly any row has tiles of two references: with logits within 44 of zero it is 0.
constexpr float kReferenceStep = 128.f;
__device__ __forceinline__ float tile_exponent(float most) { return kReferenceStep * rintf(most * (kLog2e / kReferenceStep)); }

// l = h w^T of one tile and what becomes of it.  `w`: the piece's first row, `columns` of it exist; `pitch`: of `out` [T][pitch].
template <class Shape, int kMode>
__global__ __launch_bounds__(Shape::kThreads) void ce_logits_kernel(const uint16_t* __restrict__ h, int64_t T, int64_t K, const uint16_t* __restrict__ w,
                                                        int64_t columns, int64_t first, const int64_t* __restrict__ targets, int m_tiles, int n_tiles,
                                                        float2* __restrict__ stats, float* __restrict__ target_logit, const CeRow* __restrict__ rows,
                                                        uint16_t* __restrict__ out, int64_t pitch) {
    constexpr int kMI = Shape::kMI, kNI = Shape::kNI, kWN = Shape::kWN, kM = Shape::kM;
    constexpr int kOutPitch = 512 + 16;   // bytes of a row of E in LDS
    constexpr int kTile = kMode == kStatistics ? 0 : kM * kOutPitch;
    constexpr int kEnd = kTile + 2 * kWN * kM * 4;
    __shared__ __attribute__((aligned(16))) char lds[kEnd > Shape::kLdsBytes ? kEnd : Shape::kLdsBytes];
    const TilePlace at(m_tiles, n_tiles, 1);
    if (!at.any) return;   // uniform for the workgroup, before any barrier
    const int64_t m0 = (int64_t)at.mt * kM, n0 = (int64_t)at.nt * 256;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / kWN, wn = wave % kWN, i16 = lane & 15, g = lane >> 4;

    f32x4 acc[kMI][kNI];
#pragma unroll
    for (int i = 0; i < kMI; ++i)
#pragma unroll
        for (int j = 0; j < kNI; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const TileSource<false, kM, Shape::kWaves> hs(h + m0 * K, K, T - m0, K, wave, lane);
    const TileSource<false, 256, Shape::kWaves> ws(w + n0 * K, K, columns - n0, K, wave, lane);
    tile_product<Shape, false, false>(hs, ws, 0, (int)((K + kProductStep - 1) / kProductStep), lds, acc);

    // A lane holds columns 16 (wn kNI + j) + 4 g + r of row 16 (wm kMI + i) + i16.  What few lanes have to do (columns past the end, the
    // target's) is tested once for a wave: over a tile the exponentials alone are 2 us, every other instruction an element 0.5.
    float* largest = reinterpret_cast<float*>(lds + kTile);   // [kWN][kM]
    float* sums = largest + kWN * kM;
    const int here = (int)(columns - n0 < 256 ? columns - n0 : 256);   // columns that exist
    const int first_n = 16 * wn * kNI + 4 * g;
    if (here < 256) {
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
        const int64_t t = m < T ? targets[m] - first - n0 : -1;
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
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
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
            if (__any(!of.live)) {   // a masked token: alpha and M are 0
#pragma unroll
                for (int j = 0; j < kNI; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[i][j][r] = of.live ? acc[i][j][r] : 0.f;
            }
        } else {
            float most = largest[row];
#pragma unroll
            for (int q = 1; q < kWN; ++q) most = fmaxf(most, largest[q * kM + row]);
            M = tile_exponent(most);
            M = M == -__builtin_inff() ? 0.f : M;   // (nothing in the row: every E is 2^-inf)
        }
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < kNI; ++j) {
            float e[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                e[r] = __builtin_amdgcn_exp2f(fmaf(acc[i][j][r], kLog2e, -M));
                if constexpr (kMode == kGradients) e[r] *= alpha;
            }
            if constexpr (kMode == kGradients) {
                if (__any(target[i] >= 16 * j && target[i] < 16 * j + 4)) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) e[r] = 16 * j + r == target[i] ? -of.beta : e[r];
                }
            }
            sum += (e[0] + e[1]) + (e[2] + e[3]);
            if constexpr (kMode != kStatistics)
                *reinterpret_cast<uint2*>(lds + row * kOutPitch + 32 * (wn * kNI + j) + 8 * g) = make_uint2(pack_two_bf16(e[0], e[1]), pack_two_bf16(e[2], e[3]));
        }
        if constexpr (kMode != kGradients) {
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
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
            stats[(int64_t)at.nt * T + m0 + row] = make_float2(tile_exponent(most), sum);
        }
    }
    if constexpr (kMode != kStatistics) {
        for (int row = wave * 2 + (lane >> 5); row < kM; row += 2 * Shape::kWaves) {
            if (m0 + row >= T) break;
            *reinterpret_cast<uint4*>(out + (m0 + row) * pitch + n0 + 8 * (lane & 31)) = *reinterpret_cast<const uint4*>(lds + row * kOutPitch + 16 * (lane & 31));
        }
    }
}

struct CeRowArgs {
    const float2* stats;       // [n_tiles][T]: M and sum of a tile
    int n_tiles;
    bool first, last;          // piece of the vocabulary
    float2* running;           // [T]: M and sum so far
    float* rescale;            // [T]: 2^(M before - M now)
    uint16_t* e;               // E of the piece, brought to M now where a tile's M is another; null: there is none
    int64_t pitch;
    const float* target_logit;
    const int64_t* targets;
    const float* grad_loss;    // null: ones
    int64_t T, V;
    float* loss;
    float* lse;
    CeRow* rows;               // null: not wanted
};

// Sixteen waves on 64 rows, a lane a row; wave q takes every sixteenth tile.
__global__ __launch_bounds__(1024) void ce_rows_kernel(CeRowArgs a) {
    __shared__ float part[2][16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t = (int64_t)blockIdx.x * 64 + lane;
    const bool here = t < a.T;
    const float inf = __builtin_inff();
    float most = -inf, sum = 0.f;
    if (here) {
#pragma unroll 8
        for (int n = wave; n < a.n_tiles; n += 16) most = fmaxf(most, a.stats[(int64_t)n * a.T + t].x);
    }
    part[0][wave][lane] = most;
    __syncthreads();
    for (int q = 0; q < 16; ++q) most = fmaxf(most, part[0][q][lane]);
    const float2 before = here && !a.first ? a.running[t] : make_float2(-inf, 0.f);
    most = fmaxf(most, before.x);
    const float M = most == -inf ? 0.f : most;
    if (here) {
#pragma unroll 8
        for (int n = wave; n < a.n_tiles; n += 16) {
            const float2 s = a.stats[(int64_t)n * a.T + t];
            sum += s.y * __builtin_amdgcn_exp2f(s.x - M);
        }
    }
    part[1][wave][lane] = sum;
    if (a.e != nullptr) {
        // The exponents of E in tiles with a reference below the row's, lowered by the difference: exact.  The wave goes through such
        // rows one by one, its lanes through the tile's columns.
        for (int n = wave; n < a.n_tiles; n += 16) {
            const float behind = here ? M - a.stats[(int64_t)n * a.T + t].x : 0.f;
            uint64_t rows = __ballot(behind > 0.f && behind < inf);
            while (rows != 0) {
                const int of = __ffsll((unsigned long long)rows) - 1;
                rows &= rows - 1;
                uint2* at = reinterpret_cast<uint2*>(a.e + ((int64_t)blockIdx.x * 64 + of) * a.pitch + (int64_t)n * 256) + lane;
                const bool gone = __shfl(behind, of) > kReferenceStep;
                const u16x2 by = gone ? u16x2{0xFFFF, 0xFFFF} : u16x2{(uint16_t)kReferenceStep << 7, (uint16_t)kReferenceStep << 7};
                uint2 q = *at;
                q.x = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, q.x), by));
                q.y = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(u16x2, q.y), by));
                *at = q;
            }
        }
    }
    __syncthreads();
    if (wave != 0 || !here) return;
    const float scale = __builtin_amdgcn_exp2f(before.x - M);
    sum = a.first ? 0.f : before.y * scale;
    for (int q = 0; q < 16; ++q) sum += part[1][q][lane];
    a.running[t] = make_float2(most, sum);
    a.rescale[t] = scale;
    if (!a.last) return;
    // S' = sum of 2^(l log2 e - M) over the other columns, e the target's (M may lie below the target's own exponent)
    const int64_t target = a.targets[t];
    const float nan = __builtin_nanf("");
    float loss = 0.f, lse = 0.f, alpha = 0.f, beta = 0.f;
    if (target >= a.V) {
        loss = lse = alpha = beta = nan;
    } else if (target >= 0) {
        const float l = a.target_logit[t], up = fmaf(l, kLog2e, -M), top = up > 0.f ? ceilf(up) : 0.f;
        const float e = __builtin_amdgcn_exp2f(up - top), lower = __builtin_amdgcn_exp2f(-top), rest = sum * lower, all = rest + e;
        const float gl = a.grad_loss != nullptr ? a.grad_loss[t] : 1.f;
        lse = kLn2 * (M + top) + logf(all);
        loss = e > 1e-30f ? log1pf(rest / e) : lse - l;
        alpha = gl * lower / all;
        beta = gl * (rest / all);
        if (!(all > 0.f && all < inf)) loss = lse = alpha = beta = nan;
    }
    a.loss[t] = loss;
    a.lse[t] = lse;
    if (a.rows != nullptr) a.rows[t] = CeRow{M, alpha, beta, target >= 0};
}

// sums = rescale sums + E w over the columns of a piece (contracted), slice kz of them.  `rescale` null: ones.
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
    // slices start at whole tiles of 256 columns: four steps
    const int tiles = (int)((columns + 255) / 256), t_begin = (int)((int64_t)tiles * at.kz / slices), t_end = (int)((int64_t)tiles * (at.kz + 1) / slices);
    f32x4 acc[kMI][kNI];
#pragma unroll
    for (int i = 0; i < kMI; ++i) {
        const int64_t m = m0 + 16 * (wm * kMI + i) + i16;
        const float scale = !first && m < T && rescale != nullptr ? rescale[m] : 1.f;
#pragma unroll
        for (int j = 0; j < kNI; ++j) {
            const int64_t n = n0 + 16 * (wn * kNI + j) + 4 * g;
            f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
            if (!first && m < T && n < K) v = *reinterpret_cast<const f32x4*>(sums + ((int64_t)at.kz * T + m) * K + n) * scale;
            acc[i][j] = v;
        }
    }
    const TileSource<false, kM, Shape::kWaves> es(e + m0 * pitch, pitch, T - m0, pitch, wave, lane);
    const TileSource<true, 256, Shape::kWaves> ws(w + n0, K, K - n0, columns, wave, lane);
    tile_product<Shape, false, true>(es, ws, 4 * t_begin, 4 * t_end, lds, acc);
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

// dh from the slices' sums, eight columns a thread; a row a blockIdx.y.  kPlain: the sums are dh itself.
template <bool kPlain>
__global__ __launch_bounds__(256) void ce_dh_finish_kernel(const float* __restrict__ sums, int slices, int64_t T, int64_t K, const CeRow* __restrict__ rows,
                                                           const int64_t* __restrict__ targets, int64_t V, const uint16_t* __restrict__ w,
                                                           uint16_t* __restrict__ dh) {
    const int64_t per_row = K / 8, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= T * per_row) return;
    const int64_t t = id / per_row, k = (id - t * per_row) * 8;
    const int64_t target = targets[t];
    const CeRow of = rows[t];
    float x[8] = {};
    for (int z = 0; z < slices; ++z) {
        const float4* from = reinterpret_cast<const float4*>(sums + ((int64_t)z * T + t) * K + k);
        const float4 a = from[0], b = from[1];
        x[0] += a.x, x[1] += a.y, x[2] += a.z, x[3] += a.w, x[4] += b.x, x[5] += b.y, x[6] += b.z, x[7] += b.w;
    }
    if constexpr (!kPlain) {
        const uint4 wt = target >= 0 && target < V ? *reinterpret_cast<const uint4*>(w + target * K + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int c = 0; c < 8; ++c) x[c] = of.alpha * x[c] - of.beta * bf16_bits_to_f32(unit_elem(wt, c));
    }
    uint4 q = make_uint4(pack_two_bf16(x[0], x[1]), pack_two_bf16(x[2], x[3]), pack_two_bf16(x[4], x[5]), pack_two_bf16(x[6], x[7]));
    if (target < 0) q = make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4*>(dh + t * K + k) = q;
}

// dw of a piece: G^T h, both operands across the contraction.
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
#pragma unroll
    for (int i = 0; i < kMI; ++i) {
        const int64_t m = m0 + 16 * (wm * kMI + i) + i16;
#pragma unroll
        for (int j = 0; j < kNI; ++j) {
            const int64_t n = n0 + 16 * (wn * kNI + j) + 4 * g;
            if (m < columns && n < K)
                *reinterpret_cast<uint2*>(dw + m * K + n) = make_uint2(pack_two_bf16(acc[i][j][0], acc[i][j][1]), pack_two_bf16(acc[i][j][2], acc[i][j][3]));
        }
    }
}

// Hidden states with those of masked tokens as zeros: G is zero there, but not what it is multiplied by.
__global__ __launch_bounds__(256) void ce_live_rows_kernel(const uint16_t* __restrict__ h, const int64_t* __restrict__ targets, int64_t T, int64_t K,
                                                           uint16_t* __restrict__ out) {
    const int64_t per_row = K / 8, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= T * per_row) return;
    const uint4 q = reinterpret_cast<const uint4*>(h)[id];
    reinterpret_cast<uint4*>(out)[id] = targets[id / per_row] >= 0 ? q : make_uint4(0, 0, 0, 0);
}

typedef TileShape<8, 4, 2, 4, 2, 3> Shape256;
typedef TileShape<4, 4, 2, 4, 3, 3> Shape128;
typedef TileShape<4, 2, 1, 8, 2, 2> Shape64;
typedef TileShape<2, 2, 1, 8, 2, 2> Shape32;
typedef TileShape<1, 2, 1, 8, 2, 2> Shape16;
static int64_t rows_of_tile(int64_t T) { return T <= 16 ? 16 : T <= 32 ? 32 : T <= 64 ? 64 : T <= 128 ? 128 : 256; }

CePlan ce_plan(int64_t T, int64_t K, int64_t V, bool want_dh, bool want_dw) {
    CePlan p{};
    const int64_t kM = rows_of_tile(T);
    p.rows = kM;
    p.m_tiles = (T + kM - 1) / kM;
    p.tiles = (V + 255) / 256;
    const bool pieces = want_dh || want_dw;
    int64_t per = p.tiles;
    if (pieces) {
        const int64_t most = kCePieceBytes / (512 * (T > 0 ? T : 1)), cap = most > 1 ? most : 1, n = (p.tiles + cap - 1) / cap;
        per = n > 0 ? (p.tiles + n - 1) / n : 0;
    }
    p.piece_tiles = per;
    if (want_dh) {
        const int64_t tiles = p.m_tiles * ((K + 255) / 256);
        int64_t s = 1;
        while (tiles * s < 192 && s * 2 <= per) s *= 2;
        p.slices = s;
    }
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round_up_256(bytes);
        return here;
    };
    p.stats = take((size_t)p.tiles * T * sizeof(float2));
    p.running = take((size_t)T * sizeof(float2));
    p.rescale = take((size_t)T * 4);
    p.target_logit = take((size_t)T * 4);
    p.of_rows = take((size_t)T * sizeof(CeRow));
    if (pieces) p.e = take((size_t)T * per * 512);
    if (want_dh) p.sums = take((size_t)p.slices * T * K * 4);
    if (want_dw) p.h_live = take((size_t)T * K * 2);
    p.bytes = at;
    return p;
}

template <class Shape, int kMode>
static void launch_logits(const CeArgs& a, const CePlan& p, char* ws, int64_t tile0, int64_t tiles, const uint16_t* h) {
    const int64_t first = tile0 * 256, columns = a.V - first < tiles * 256 ? a.V - first : tiles * 256;
    hipLaunchKernelGGL((ce_logits_kernel<Shape, kMode>), dim3(product_grid(p.m_tiles * tiles)), dim3(Shape::kThreads), 0, a.stream, h, a.T, a.K, a.w + first * a.K,
                       columns, first, a.targets, (int)p.m_tiles, (int)tiles, reinterpret_cast<float2*>(ws + p.stats), reinterpret_cast<float*>(ws + p.target_logit),
                       reinterpret_cast<const CeRow*>(ws + p.of_rows), reinterpret_cast<uint16_t*>(ws + p.e), p.piece_tiles * 256);
}

template <class Shape>
static hipError_t launch_shape(const CeArgs& a, const CePlan& p, char* ws) {
    const int n_tiles = (int)((a.K + 255) / 256);
    uint16_t* e = reinterpret_cast<uint16_t*>(ws + p.e);
    const int64_t pitch = p.piece_tiles * 256;
    CeRow* rows = reinterpret_cast<CeRow*>(ws + p.of_rows);
    float* sums = reinterpret_cast<float*>(ws + p.sums);
    CeRowArgs r{};
    r.stats = reinterpret_cast<const float2*>(ws + p.stats);
    r.running = reinterpret_cast<float2*>(ws + p.running);
    r.rescale = reinterpret_cast<float*>(ws + p.rescale);
    r.target_logit = reinterpret_cast<const float*>(ws + p.target_logit);
    r.targets = a.targets, r.grad_loss = a.grad_loss, r.T = a.T, r.V = a.V, r.loss = a.loss, r.lse = a.lse, r.rows = rows;
    const dim3 row_grid((unsigned)((a.T + 63) / 64));
    const unsigned units = (unsigned)((a.T * (a.K / 8) + 255) / 256);
    const bool statistics_first = a.dw != nullptr || a.dh == nullptr;
    if (a.T > 0 && statistics_first) {
        launch_logits<Shape, kStatistics>(a, p, ws, 0, p.tiles, a.h);
        r.n_tiles = (int)p.tiles, r.first = r.last = true;
        hipLaunchKernelGGL(ce_rows_kernel, row_grid, dim3(1024), 0, a.stream, r);
    }
    if (a.dh == nullptr && a.dw == nullptr) return hipGetLastError();
    const uint16_t* h_live = a.h;
    if (a.dw != nullptr && units > 0) {
        uint16_t* to = reinterpret_cast<uint16_t*>(ws + p.h_live);
        hipLaunchKernelGGL(ce_live_rows_kernel, dim3(units), dim3(256), 0, a.stream, a.h, a.targets, a.T, a.K, to);
        h_live = to;
    }
    for (int64_t tile0 = 0; tile0 < p.tiles; tile0 += p.piece_tiles) {
        const int64_t tiles = p.tiles - tile0 < p.piece_tiles ? p.tiles - tile0 : p.piece_tiles, first = tile0 * 256;
        const int64_t columns = a.V - first < tiles * 256 ? a.V - first : tiles * 256;
        if (a.T > 0) {
            if (statistics_first) {
                launch_logits<Shape, kGradients>(a, p, ws, tile0, tiles, a.h);
            } else {
                launch_logits<Shape, kExponentials>(a, p, ws, tile0, tiles, a.h);
                r.n_tiles = (int)tiles, r.first = tile0 == 0, r.last = tile0 + tiles == p.tiles;
                r.e = e, r.pitch = pitch;
                hipLaunchKernelGGL(ce_rows_kernel, row_grid, dim3(1024), 0, a.stream, r);
            }
            if (a.dh != nullptr && n_tiles > 0) {
                const dim3 grid(product_grid(p.m_tiles * n_tiles * p.slices));
                hipLaunchKernelGGL(ce_dh_kernel<Shape>, grid, dim3(Shape::kThreads), 0, a.stream, e, a.T, pitch, a.w + first * a.K, columns, a.K, (int)p.m_tiles,
                                   n_tiles, (int)p.slices, statistics_first ? nullptr : r.rescale, tile0 == 0, sums);
            }
        }
        if (a.dw != nullptr && n_tiles > 0)
            hipLaunchKernelGGL(ce_dw_kernel<Shape256>, dim3(product_grid(tiles * n_tiles)), dim3(Shape256::kThreads), 0, a.stream, e, a.T, pitch, h_live, a.K, columns, (int)tiles,
                               n_tiles, a.dw + first * a.K);
    }
    if (a.dh != nullptr && units > 0) {
        if (statistics_first)
            hipLaunchKernelGGL(ce_dh_finish_kernel<true>, dim3(units), dim3(256), 0, a.stream, sums, (int)p.slices, a.T, a.K, rows, a.targets, a.V, a.w, a.dh);
        else
            hipLaunchKernelGGL(ce_dh_finish_kernel<false>, dim3(units), dim3(256), 0, a.stream, sums, (int)p.slices, a.T, a.K, rows, a.targets, a.V, a.w, a.dh);
    }
    return hipGetLastError();
}

hipError_t launch_cross_entropy(const CeArgs& a, void* workspace) {
    const CePlan p = ce_plan(a.T, a.K, a.V, a.dh != nullptr, a.dw != nullptr);
    char* ws = static_cast<char*>(workspace);
    switch (p.rows) {
        case 16: return launch_shape<Shape16>(a, p, ws);
        case 32: return launch_shape<Shape32>(a, p, ws);
        case 64: return launch_shape<Shape64>(a, p, ws);
        case 128: return launch_shape<Shape128>(a, p, ws);
        default: return launch_shape<Shape256>(a, p, ws);
    }
}

}  // namespace salr
