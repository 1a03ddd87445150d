// Layer norm of a row s of K values, s = x or the stored sum x + residual, and its gradient:
//
//   mean = sum s / K,  rstd = 1 / sqrt(sum (s - mean)^2 / K + eps),  xhat = (s - mean) rstd,  y = xhat w + b
//   g = dy w,  dx = rstd (g - sum g / K - xhat sum (g xhat) / K) + dsum,  dw = sum over rows of dy xhat,  db = sum over rows of dy
//
// What bounds both is memory: every matrix crosses it once.  A team of 1 to 16 waves holds a row in registers, as it lies in memory (8 or 16
// bytes of registers for four elements), each lane one to eight vectors of eight elements; sums go over the lanes in registers and over the
// team's waves through LDS.  The variance is summed from differences to the mean in a second pass over the registers: squares alone lose
// what a large mean hides.  Sums are fp32.
//
// dw and db: a workgroup of eight waves goes through rows, its lanes keep the sums of their columns; the teams of a workgroup are added in LDS,
// in order, and the workgroups' sums, at most kLayerNormParts of them, by a second launch: no atomics, the same bits every time.  Up to kLayerNormFewRows rows
// workgroups of their own read x and dy again beside those that form dx: one launch.
// Wide rows: above 16384 columns no form of the gradient has registers for what a lane holds, and above 8192 the one with dw and db has not.
// What does not fit goes to scratch memory and back (the compiler's report, in registers a lane: with dw and db 10 to 84 up to 16384 columns, 366 and 430 for rows of
// odd lengths, 682 to 1870 above; dx alone above 16384 107 to 198, 476 and 676 for odd ones).
//
// Measured: 4096 x 4096 bf16, with a residual 24.4 us (134 MB, 5.5 TB/s); its gradient with dsum, dw and db 28.8 us (4.7 TB/s, 4 us of them the second launch;
// with sixteen waves a workgroup, a row requested when it is needed and the weights read for each, 58 us); one row of 4096 3.1 us of kernel; 1111 x 2721 fp32
// with dw and db 17.6 us, where the launches' start and end are 10.  Wide rows, bf16, with dw and db and dx alone: 1024 x 14336 37.5 and 23.8 us, 4096 x 14336 93
// and 77 (254 and 114 at 14335), 4096 x 28672 1250 and 459 (1365 and 806 at 28671; its bytes take 135).
#include <type_traits>

#include "salr_eight.hpp"
#include "salr_internal.hpp"

namespace salr {

// Sum over the wave, in every lane: within rows of 16 lanes, then over the rows.
__device__ __forceinline__ float wave_sum(float v) {
    const auto add = [](float a, int b) { return a + __int_as_float(b); };
    v = add(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x111, 0xf, 0xf, false));
    v = add(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x112, 0xf, 0xf, false));
    v = add(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x114, 0xf, 0xf, false));
    v = add(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x118, 0xf, 0xf, false));
    v = add(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x142, 0xa, 0xf, false));
    v = add(v, __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x143, 0xc, 0xf, false));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), kWave - 1));
}

// Sum over a team of kTeam waves, every wave of the workgroup calling it.  `slots` (kSums floats a wave) are another set at every call until
// two barriers have passed.
template <int kTeam, int kSums>
__device__ __forceinline__ void team_sum(float (&v)[kSums], float* slots) {
#pragma unroll
    for (int i = 0; i < kSums; ++i) v[i] = wave_sum(v[i]);
    if constexpr (kTeam > 1) {
        const int wave = threadIdx.x >> 6, first = wave / kTeam * kTeam;
        if (lane_id() == 0)
#pragma unroll
            for (int i = 0; i < kSums; ++i) slots[wave * kSums + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kSums; ++i) {
            float s = 0.f;
#pragma unroll
            for (int t = 0; t < kTeam; ++t) s += slots[(first + t) * kSums + i];
            v[i] = s;
        }
    }
}

// Eight elements of a row from i on, of which `left` are there, in two steps: asked for, then as they are.  kWhole: all or none of them are there.
template <bool k32, bool kWhole>
__device__ __forceinline__ Eight<k32> row_request(const void* matrix, int64_t start, int i, int left, int64_t total) {
    if constexpr (kWhole) {
        Eight<k32> zero{};
        return left > 0 ? load_eight<k32, false, false>(static_cast<const char*>(matrix) + (start + i) * (k32 ? 4 : 2), 0, 8) : zero;
    } else {
        if (total < 8) return load_eight<k32, false, false>(static_cast<const char*>(matrix) + start * (k32 ? 4 : 2), i, left);   // the same for the launch
        return raw_eight<k32>(matrix, start + i, total);
    }
}
template <bool k32, bool kWhole>
__device__ __forceinline__ Eight<k32> row_values(const Eight<k32>& q, int64_t start, int i, int left, int64_t total) {
    if (kWhole || total < 8) return q;
    return true_eight<k32>(q, start + i, left, total);
}

// The same of weights, in fp32.
template <bool kWhole>
__device__ __forceinline__ void load_weights(const void* w, bool w32, int i, int K, float (&out)[8]) {
    const int left = K - i;
    if (w32) {
        const Eight<true> q = row_values<true, kWhole>(row_request<true, kWhole>(w, 0, i, left, K), 0, i, left, K);
#pragma unroll
        for (int j = 0; j < 8; ++j) out[j] = q.get(j);
    } else {
        const Eight<false> q = row_values<false, kWhole>(row_request<false, kWhole>(w, 0, i, left, K), 0, i, left, K);
#pragma unroll
        for (int j = 0; j < 8; ++j) out[j] = q.get(j);
    }
}

template <bool k32, int kTeam, int kUnits, bool kWhole>
__global__ __launch_bounds__(kTeam < 4 ? 256 : 64 * kTeam) void layer_norm_kernel(LayerNormArgs a) {
    constexpr int kWaves = kTeam < 4 ? 4 : kTeam, kTeams = kWaves / kTeam;
    __shared__ float slots[2][kWaves];
    const int team = threadIdx.x / (64 * kTeam), at = threadIdx.x % (64 * kTeam), K = a.K;
    const int64_t row = (int64_t)blockIdx.x * kTeams + team;
    const bool live = row < a.T;   // (the others go through the barriers)
    const int64_t start = (live ? row : 0) * K, total = a.T * K;
    char* y = static_cast<char*>(a.y) + start * (k32 ? 4 : 2);
    float s[kUnits][8], sums[1] = {0.f};
    Eight<k32> xq[kUnits], rq[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int i = 8 * (at + 64 * kTeam * u), left = live ? K - i : 0;
        xq[u] = row_request<k32, kWhole>(a.x, start, i, left, total);
    }
    if (a.residual != nullptr)
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int i = 8 * (at + 64 * kTeam * u), left = live ? K - i : 0;
            rq[u] = row_request<k32, kWhole>(a.residual, start, i, left, total);
        }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int i = 8 * (at + 64 * kTeam * u), left = live ? K - i : 0;
        const Eight<k32> q = row_values<k32, kWhole>(xq[u], start, i, left, total);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[u][j] = q.get(j);
    }
    if (a.residual != nullptr) {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int i = 8 * (at + 64 * kTeam * u), left = live ? K - i : 0;
            const Eight<k32> q = row_values<k32, kWhole>(rq[u], start, i, left, total);
            // the sum is rounded as it is stored, and the norm is of that: so is the gradient, which reads it back
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[u][j] += q.get(j);
                if constexpr (!k32) s[u][j] = (float)(__bf16)s[u][j];
            }
            if (left > 0) store_eight<k32, false>(static_cast<char*>(a.sum) + start * (k32 ? 4 : 2), i, kWhole ? 8 : left, s[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) sums[0] += s[u][j];
    team_sum<kTeam>(sums, slots[0]);
    const float mean = sums[0] / (float)K;
    sums[0] = 0.f;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int left = K - 8 * (at + 64 * kTeam * u);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = (kWhole ? 0 : j) < left ? s[u][j] - mean : 0.f;
            sums[0] = fmaf(d, d, sums[0]);
        }
    }
    team_sum<kTeam>(sums, slots[1]);
    const float rstd = 1.f / sqrtf(sums[0] / (float)K + a.eps);
    if (!live) return;
    if (at == 0) {
        if (a.mean != nullptr) a.mean[row] = mean;
        if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const int i = 8 * (at + 64 * kTeam * u), left = K - i;
        if (left <= 0) break;
        float w[8], b[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        load_weights<kWhole>(a.weight, a.w32, i, K, w);
        if (a.bias != nullptr) load_weights<kWhole>(a.bias, a.w32, i, K, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = fmaf((s[u][j] - mean) * rstd, w[j], b[j]);
        store_eight<k32, false>(y, i, kWhole ? 8 : left, w);
    }
}

// kWeights: dw and db too, the workgroup's sums of them as part[0][blockIdx.x][K] and part[1][..]; a row's requests are then out while the one before is
// worked on (kAhead; not for rows whose sums leave no registers for that), since a workgroup has its CU to itself.
template <int kTeam, bool kWeights>
constexpr int grad_waves() { return kWeights ? 8 : kTeam < 4 ? 4 : kTeam; }

template <bool k32, int kTeam, int kUnits, bool kWhole, bool kWeights, int kWaves>
__device__ __forceinline__ void backward_rows(const LayerNormGradArgs& a, int blocks) {
    constexpr int kTeams = kWaves / kTeam;
    constexpr bool kAhead = kWeights && kUnits <= 2;
    __shared__ float slots[2][kWaves * 2];
    __shared__ __align__(16) float totals[kTeams > 1 && kWeights ? 512 * kTeam * kUnits : 4];   // what the teams before have summed
    const int team = threadIdx.x / (64 * kTeam), at = threadIdx.x % (64 * kTeam), K = a.K;
    const bool want_dx = a.dx != nullptr, add = want_dx && a.dsum != nullptr;
    float dw[kWeights ? kUnits : 1][8] = {}, db[kWeights ? kUnits : 1][8] = {}, w[kUnits][8] = {};
    if (want_dx)
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int i = 8 * (at + 64 * kTeam * u);
            load_weights<kWhole>(a.weight, a.w32, i, K, w[u]);
        }
    const int64_t total = a.T * K;
    struct Row {
        Eight<k32> x[kUnits], dy[kUnits], ds[kUnits];
        float mean, rstd;
    };
    const auto request = [&](Row& r, int64_t row) {
        const bool live = row < a.T;
        const int64_t start = (live ? row : 0) * K;
        r.mean = live ? a.mean[row] : 0.f;
        r.rstd = live ? a.rstd[row] : 0.f;
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int i = 8 * (at + 64 * kTeam * u), left = live ? K - i : 0;
            r.x[u] = row_request<k32, kWhole>(a.x, start, i, left, total);
            r.dy[u] = row_request<k32, kWhole>(a.dy, start, i, left, total);
            if (add) r.ds[u] = row_request<k32, kWhole>(a.dsum, start, i, left, total);
        }
    };
    const int64_t stride = (int64_t)blocks * kTeams;
    Row next;
    if constexpr (kAhead) request(next, (int64_t)blockIdx.x * kTeams + team);
    int parity = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * kTeams; row0 < a.T; row0 += stride, parity ^= 1) {   // the same for the workgroup
        const int64_t row = row0 + team;
        const bool live = row < a.T;
        Row r;
        if constexpr (kAhead) {
            r = next;
            if (row0 + stride < a.T) request(next, row + stride);
        } else {
            request(r, row);
        }
        if constexpr (!kWhole) {
            const int64_t start = (live ? row : 0) * K;
#pragma unroll
            for (int u = 0; u < kUnits; ++u) {
                const int i = 8 * (at + 64 * kTeam * u), left = live ? K - i : 0;
                r.x[u] = row_values<k32, kWhole>(r.x[u], start, i, left, total);
                r.dy[u] = row_values<k32, kWhole>(r.dy[u], start, i, left, total);
                if (add) r.ds[u] = row_values<k32, kWhole>(r.ds[u], start, i, left, total);
            }
        }
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int left = live ? K - 8 * (at + 64 * kTeam * u) : 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = r.dy[u].get(j), xhat = (kWhole ? 0 : j) < left ? (r.x[u].get(j) - r.mean) * r.rstd : 0.f, g = d * w[u][j];
                sums[0] += g;
                sums[1] = fmaf(g, xhat, sums[1]);
                if constexpr (kWeights) {
                    dw[u][j] = fmaf(d, xhat, dw[u][j]);
                    db[u][j] += d;
                }
            }
        }
        if (!want_dx) continue;   // the same for the launch
        team_sum<kTeam>(sums, slots[parity]);
        const float g_mean = sums[0] / (float)K, along = sums[1] / (float)K;
        char* dx = static_cast<char*>(a.dx) + (live ? row : 0) * K * (k32 ? 4 : 2);
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int i = 8 * (at + 64 * kTeam * u), left = live ? K - i : 0;
            if (left <= 0) break;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float xhat = (r.x[u].get(j) - r.mean) * r.rstd;
                v[j] = r.rstd * (fmaf(-xhat, along, r.dy[u].get(j) * w[u][j] - g_mean));
                if (add) v[j] += r.ds[u].get(j);
            }
            store_eight<k32, false>(dx, i, kWhole ? 8 : left, v);
        }
    }
    if constexpr (kWeights) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            float* part = a.part + ((int64_t)which * blocks + blockIdx.x) * K;
            for (int t = 0; t < kTeams; ++t) {   // the teams one after the other
                if (t == team) {
#pragma unroll
                    for (int u = 0; u < kUnits; ++u) {
                        const int i = 8 * (at + 64 * kTeam * u), left = K - i;
                        float v[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = which == 0 ? dw[u][j] : db[u][j];
                        if (t > 0) {   // (totals has whole vectors of room)
                            const f32x4 lo = *reinterpret_cast<const f32x4*>(totals + i), hi = *reinterpret_cast<const f32x4*>(totals + i + 4);
#pragma unroll
                            for (int j = 0; j < 8; ++j) v[j] += j < 4 ? lo[j] : hi[j - 4];
                        }
                        if (t < kTeams - 1) {
                            *reinterpret_cast<f32x4*>(totals + i) = f32x4{v[0], v[1], v[2], v[3]};
                            *reinterpret_cast<f32x4*>(totals + i + 4) = f32x4{v[4], v[5], v[6], v[7]};
                        } else if (left > 0) {
                            store_eight<true, false>(part, i, kWhole ? 8 : left, v);
                        }
                    }
                }
                if constexpr (kTeams > 1) __syncthreads();
            }
        }
    }
}

template <bool k32, int kTeam, int kUnits, bool kWhole, bool kWeights>
__global__ __launch_bounds__((64 * grad_waves<kTeam, kWeights>())) void layer_norm_backward_kernel(LayerNormGradArgs a) {
    backward_rows<k32, kTeam, kUnits, kWhole, kWeights, grad_waves<kTeam, kWeights>()>(a, (int)gridDim.x);
}

// dw and db of 64 columns by one workgroup that goes through all rows, eight lanes a row and four rows a lane at a time: for few rows, beside the workgroups
// that form dx, instead of a launch behind them.  sums: 128 floats a wave.
template <bool k32, bool kWhole>
__device__ __forceinline__ void column_sums(const LayerNormGradArgs& a, int block, void* dw_out, void* db_out, float* sums) {
    constexpr int kRows = 4;
    const int K = a.K, c = 64 * block + 8 * (threadIdx.x & 7), left = K - c, waves = blockDim.x >> 6, wave = threadIdx.x >> 6, step = blockDim.x >> 3;
    const int T = (int)a.T;
    const int64_t total = a.T * K;
    float dw[8] = {}, db[8] = {};
    for (int t = threadIdx.x >> 3; t < T; t += kRows * step) {
        Eight<k32> xq[kRows], dyq[kRows];
        float mean[kRows], rstd[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {   // (rows behind the last: the last again, left out below)
            const int64_t at = min(t + r * step, T - 1), start = at * K;
            xq[r] = row_request<k32, kWhole>(a.x, start, c, left, total);
            dyq[r] = row_request<k32, kWhole>(a.dy, start, c, left, total);
            mean[r] = a.mean[at];
            rstd[r] = a.rstd[at];
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (t + r * step >= T) break;
            const int64_t start = (int64_t)(t + r * step) * K;
            const Eight<k32> x = row_values<k32, kWhole>(xq[r], start, c, left, total), dy = row_values<k32, kWhole>(dyq[r], start, c, left, total);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dw[j] = fmaf(dy.get(j), (x.get(j) - mean[r]) * rstd[r], dw[j]);
                db[j] += dy.get(j);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int apart = 8; apart < kWave; apart *= 2) {
            dw[j] += __shfl_xor(dw[j], apart);
            db[j] += __shfl_xor(db[j], apart);
        }
    if (lane_id() < 8)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sums[128 * wave + 8 * lane_id() + j] = dw[j];
            sums[128 * wave + 64 + 8 * lane_id() + j] = db[j];
        }
    __syncthreads();
    const int at = 64 * block + (threadIdx.x & 63);
    void* out = threadIdx.x < 64 ? dw_out : db_out;
    if (threadIdx.x >= 128 || at >= K || out == nullptr) return;
    float v = 0.f;
    for (int w = 0; w < waves; ++w) v += sums[128 * w + threadIdx.x];
    if (a.w32) static_cast<float*>(out)[at] = v;
    else static_cast<uint16_t*>(out)[at] = f32_to_bf16_rne(v);
}

template <int kTeam>
constexpr int few_waves() { return kTeam < 8 ? 8 : kTeam; }
template <bool k32, int kTeam, int kUnits, bool kWhole>
__global__ __launch_bounds__(64 * few_waves<kTeam>()) void layer_norm_backward_few_kernel(LayerNormGradArgs a, int row_blocks, void* dw, void* db) {
    __shared__ float sums[few_waves<kTeam>() * 128];
    if ((int)blockIdx.x < row_blocks) backward_rows<k32, kTeam, kUnits, kWhole, false, few_waves<kTeam>()>(a, row_blocks);
    else column_sums<k32, kWhole>(a, (int)blockIdx.x - row_blocks, dw, db, sums);
}

// dw (y 0) and db (y 1) from the workgroups' sums, 64 columns a workgroup, every sixteenth part a wave.  parts 0: zeros.
__global__ __launch_bounds__(1024) void layer_norm_parts_kernel(const float* part, int parts, int K, bool w32, void* dw, void* db) {
    __shared__ float sums[16][64];
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    void* out = blockIdx.y == 0 ? dw : db;
    if (out == nullptr) return;   // the same for the workgroup
    const int c = blockIdx.x * 64 + lane;
    const float* from = part + (int64_t)blockIdx.y * parts * K;
    float s = 0.f;
    if (c < K)
#pragma unroll 8
        for (int p = wave; p < parts; p += 16) s += from[(int64_t)p * K + c];
    sums[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || c >= K) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sums[w][lane];
    if (w32) static_cast<float*>(out)[c] = s;
    else static_cast<uint16_t*>(out)[c] = f32_to_bf16_rne(s);
}

// The team for rows of K: as few waves as hold a row with two vectors a lane.
template <typename Run>
void with_team_to_8192(int64_t K, Run run) {
    using std::integral_constant;
    if (K <= 512) run(integral_constant<int, 1>(), integral_constant<int, 1>());
    else if (K <= 1024) run(integral_constant<int, 1>(), integral_constant<int, 2>());
    else if (K <= 2048) run(integral_constant<int, 2>(), integral_constant<int, 2>());
    else if (K <= 4096) run(integral_constant<int, 4>(), integral_constant<int, 2>());
    else run(integral_constant<int, 8>(), integral_constant<int, 2>());
}
template <typename Run>
void with_team(int64_t K, Run run) {
    using std::integral_constant;
    if (K <= 8192) with_team_to_8192(K, run);
    else if (K <= 16384) run(integral_constant<int, 16>(), integral_constant<int, 2>());
    else run(integral_constant<int, 16>(), integral_constant<int, 4>());
}

// The team that sums dw and db too: eight waves at most, whose lanes have 256 registers each.  Enough for dw, db, the weights and a row up to two vectors a lane, not
// for four or eight (see above): those are for being there at all.
template <typename Run>
void with_grad_team(int64_t K, Run run) {
    using std::integral_constant;
    if (K <= 8192) with_team_to_8192(K, run);
    else if (K <= 16384) run(integral_constant<int, 8>(), integral_constant<int, 4>());
    else run(integral_constant<int, 8>(), integral_constant<int, 8>());
}

int64_t layer_norm_parts(int64_t T, int64_t K) {
    int team = 0;
    with_grad_team(K, [&](auto waves, auto) { team = waves; });
    const int64_t teams = 8 / team, groups = (T + teams - 1) / teams;
    return groups < kLayerNormParts ? groups : kLayerNormParts;
}

template <typename Run>
void with_whole(int64_t K, Run run) {   // rows of whole vectors
    if (K % 8 == 0) run(std::true_type());
    else run(std::false_type());
}

hipError_t launch_layer_norm(const LayerNormArgs& a, hipStream_t stream) {
    with_team(a.K, [&](auto waves, auto units) {
        with_whole(a.K, [&](auto whole) {
            constexpr int kTeam = waves, kUnits = units, kTeams = kTeam < 4 ? 4 / kTeam : 1;
            constexpr bool kWhole = decltype(whole)::value;
            const dim3 grid((unsigned)((a.T + kTeams - 1) / kTeams)), block(64 * kTeam * kTeams);
            if (a.f32) hipLaunchKernelGGL((layer_norm_kernel<true, kTeam, kUnits, kWhole>), grid, block, 0, stream, a);
            else hipLaunchKernelGGL((layer_norm_kernel<false, kTeam, kUnits, kWhole>), grid, block, 0, stream, a);
        });
    });
    return hipGetLastError();
}

hipError_t launch_layer_norm_backward(const LayerNormGradArgs& a, void* dw, void* db, hipStream_t stream) {
    const bool weights = dw != nullptr || db != nullptr;
    const int64_t parts = layer_norm_parts(a.T, a.K);
    const auto run = [&](auto kernel, int64_t groups, int threads) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3((unsigned)threads), 0, stream, a);
    };
    if (a.T > 0 && weights && a.T <= kLayerNormFewRows) {   // (leaves the workspace alone)
        with_team(a.K, [&](auto waves, auto units) {
            with_whole(a.K, [&](auto whole) {
                constexpr int kTeam = waves, kUnits = units, kThreads = 64 * few_waves<kTeam>(), kTeams = few_waves<kTeam>() / kTeam;
                constexpr bool kWhole = decltype(whole)::value;
                const int rows = a.dx != nullptr ? (int)((a.T + kTeams - 1) / kTeams) : 0, columns = (a.K + 63) / 64;
                const auto launch = [&](int row_blocks, int blocks) {
                    const dim3 grid((unsigned)blocks), block(kThreads);
                    if (a.f32) hipLaunchKernelGGL((layer_norm_backward_few_kernel<true, kTeam, kUnits, kWhole>), grid, block, 0, stream, a, row_blocks, dw, db);
                    else hipLaunchKernelGGL((layer_norm_backward_few_kernel<false, kTeam, kUnits, kWhole>), grid, block, 0, stream, a, row_blocks, dw, db);
                };
                if (a.dx != nullptr && (a.dx == a.dy || a.dx == a.x)) {   // in place: the rows are written once the columns' workgroups have read them
                    launch(0, columns);
                    launch(rows, rows);
                } else {
                    launch(rows, rows + columns);
                }
            });
        });
        return hipGetLastError();
    }
    if (a.T > 0 && weights)
        with_grad_team(a.K, [&](auto waves, auto units) {
            with_whole(a.K, [&](auto whole) {
                constexpr int kTeam = waves, kUnits = units;
                constexpr bool kWhole = decltype(whole)::value;
                if (a.f32) run(layer_norm_backward_kernel<true, kTeam, kUnits, kWhole, true>, parts, 512);
                else run(layer_norm_backward_kernel<false, kTeam, kUnits, kWhole, true>, parts, 512);
            });
        });
    else if (a.T > 0 && a.dx != nullptr)
        with_team(a.K, [&](auto waves, auto units) {
            with_whole(a.K, [&](auto whole) {
                constexpr int kTeam = waves, kUnits = units, kThreads = 64 * grad_waves<kTeam, false>(), kTeams = kThreads / 64 / kTeam;
                constexpr bool kWhole = decltype(whole)::value;
                if (a.f32) run(layer_norm_backward_kernel<true, kTeam, kUnits, kWhole, false>, (a.T + kTeams - 1) / kTeams, kThreads);
                else run(layer_norm_backward_kernel<false, kTeam, kUnits, kWhole, false>, (a.T + kTeams - 1) / kTeams, kThreads);
            });
        });
    if (weights)
        hipLaunchKernelGGL(layer_norm_parts_kernel, dim3((unsigned)((a.K + 63) / 64), 2), dim3(1024), 0, stream, a.part, (int)parts, a.K, a.w32, dw, db);
    return hipGetLastError();
}

}  // namespace salr
