// The optimiser's side of a fine-tuning step: AdamW over many tensors in one launch, with states in 32 or in 8 bits, and the norm
// of all gradients with the factor that clips them.  Both walk one list of chunks (salr_step_plan), a record of pointers each.
//
//   g = c grad;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2;
//   p = p (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Every product and sum above is rounded to fp32 on its own (no contraction), so that the 8-bit states do not depend on how a
// compiler pairs them.  States in 8 bits: 128 elements of a tensor share two fp32 scales, m and sqrt(v) are kept as values of
// the 8-bit type with four exponent and three mantissa bits, the block's largest magnitude at 448.  sqrt(v) and not v, for twice
// the range.  m is rounded to nearest (it moves by a tenth of the gradient a step, more than a value's spacing); sqrt(v) moves
// by a thousandth and less of itself, which nearest would undo step after step: it is rounded up with the probability of what is
// cut off, drawn from the element's position and the step's seed, and never to zero, which would make a step of any size out
// of a small m.
#include <cmath>
#include <type_traits>

#include "salr_device.hpp"
#include "salr_eight.hpp"
#include "salr_internal.hpp"
#include "salr_linear_common.hpp"

namespace salr {

constexpr float kFp8Most = 448.f;
constexpr float kFp8Tiny = 0x1p-100f;   // a block below this is stored as zeros: 448 times its inverse is still finite

__device__ __forceinline__ uint2 load_codes(const void* base, int i, int left) {
    const uint8_t* from = static_cast<const uint8_t*>(base) + i;
    if (left >= 8) return *reinterpret_cast<const uint2*>(from);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) w[j >> 2] |= (uint32_t)from[j] << (8 * (j & 3));
    return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ void store_codes(void* base, int i, int left, uint2 c) {
    uint8_t* to = static_cast<uint8_t*>(base) + i;
    if (left >= 8) {
        *reinterpret_cast<uint2*>(to) = c;
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < left) to[j] = (uint8_t)((j < 4 ? c.x : c.y) >> (8 * (j & 3)));
}

__device__ __forceinline__ void decode_codes(uint2 c, float (&x)[8]) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(c.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c.x, true);
    const f32x2 d = __builtin_amdgcn_cvt_pk_f32_fp8(c.y, false), e = __builtin_amdgcn_cvt_pk_f32_fp8(c.y, true);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = d[0], x[5] = d[1], x[6] = e[0], x[7] = e[1];
}

__device__ __forceinline__ uint2 encode_codes(const float (&x)[8]) {   // to nearest, ties to even
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], hi, true);
    return make_uint2((uint32_t)lo, (uint32_t)hi);
}

// The largest of a value over the sixteen lanes of a row, in all of them.
__device__ __forceinline__ float row_max(float x) {
    const auto turned = [](float v, auto by) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), decltype(by)::value, 0xf, 0xf, false));
    };
    x = fmaxf(x, turned(x, std::integral_constant<int, 0x128>{}));   // row_ror 8, 4, 2, 1
    x = fmaxf(x, turned(x, std::integral_constant<int, 0x124>{}));
    x = fmaxf(x, turned(x, std::integral_constant<int, 0x122>{}));
    return fmaxf(x, turned(x, std::integral_constant<int, 0x121>{}));
}

// Twenty random bits of a position: three rounds of a 32-bit product with an odd number (binary places of the golden ratio and of
// the roots of 2 and 3) and a shift down.
__device__ __forceinline__ uint32_t random20(uint32_t position, uint32_t key) {
    uint32_t x = position * 0x9E3779B1u + key;
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 13;
    x *= 0xBB67AE85u;
    return x >> 12;
}

// x in [0, 448 and a little] to a value of the 8-bit type, up with the probability of what is cut off.
__device__ __forceinline__ float random_round(float x, uint32_t bits20) {
#pragma clang fp contract(off)
    const float up = x < 0x1p-6f ? 0x1p-6f : 0.f;   // subnormal there, spacing 2^-9: as that of the values from 2^-6 on
    const float y = __uint_as_float((__float_as_uint(x + up) + bits20) & ~0xFFFFFu) - up;
    return x > 0.f ? __builtin_amdgcn_fmed3f(y, 0x1p-9f, kFp8Most) : x;   // (a NaN stays one)
}

struct StepScalars {
    float beta1, beta2, keep1, keep2;   // keep = 1 - beta
    float rate, shrink, root_scale, eps;   // lr / (1 - b1^t), 1 - lr decay, 1 / sqrt(1 - b2^t)
    uint32_t key;
};

// Workgroups to a record: one pass of 2048 elements each.  A workgroup that goes through all of a record has its requests out a quarter at a time:
// 132 M elements in 32 (8) bits 718 (424) us so, 685 (390) in four, 4.9 M in 8 bits 25 and 18.
constexpr int kStepParts = 4;

template <bool kParam32, bool kGrad32, bool k8>
__global__ __launch_bounds__(256) void adamw_kernel(const StepChunk* __restrict__ plan, StepScalars h, const float* __restrict__ grad_scale) {
#pragma clang fp contract(off)
    const float c = grad_scale != nullptr ? *grad_scale : 1.f;
    if (!(fabsf(c) < __builtin_inff())) return;   // the norm of the gradients was not finite: nothing changes
    const StepChunk t = plan[blockIdx.x / kStepParts];
    // (the sixteen lanes of a block of 128 stay together: lanes past the end hold zeros)
    const int end = k8 ? (t.count + (int)kStepBlock - 1) / (int)kStepBlock * (int)kStepBlock : t.count;
    const int i = (blockIdx.x % kStepParts) * 2048 + threadIdx.x * 8;
    if (i < end) {
        const int left = t.count - i;
        const Eight<kGrad32> grad = load_eight<kGrad32>(t.grad, i, left);
        const Eight<kParam32> param = load_eight<kParam32>(t.param, i, left);
        float m[8], v[8], p[8];
        if constexpr (k8) {
            const float2 scale = reinterpret_cast<const float2*>(t.scales)[i / kStepBlock];
            decode_codes(load_codes(t.exp_avg, i, left), m);
            decode_codes(load_codes(t.exp_avg_sq, i, left), v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                m[j] *= scale.x;
                v[j] *= scale.y;
                v[j] *= v[j];
            }
        } else {
            const Eight<true> m0 = load_eight<true>(t.exp_avg, i, left), v0 = load_eight<true>(t.exp_avg_sq, i, left);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                m[j] = m0.get(j);
                v[j] = v0.get(j);
            }
        }
        float root[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float g = grad_scale != nullptr ? grad.get(j) * c : grad.get(j);
            m[j] = m[j] * h.beta1 + g * h.keep1;
            v[j] = v[j] * h.beta2 + g * g * h.keep2;
            root[j] = sqrtf(v[j]);
            p[j] = param.get(j) * h.shrink - m[j] * h.rate / (root[j] * h.root_scale + h.eps);
        }
        store_eight<kParam32>(t.param, i, left, p);
        if (kParam32 && t.copy != nullptr) store_eight<false>(t.copy, i, left, p);
        if constexpr (k8) {
            float most_m = 0.f, most_r = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                most_m = fmaxf(most_m, fabsf(m[j]));
                most_r = fmaxf(most_r, root[j]);
            }
            most_m = row_max(most_m);
            most_r = row_max(most_r);
            const bool some_m = most_m >= kFp8Tiny, some_r = most_r >= kFp8Tiny;
            const float inv_m = some_m ? kFp8Most * (1.f / most_m) : 0.f, inv_r = some_r ? kFp8Most * (1.f / most_r) : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                m[j] *= inv_m;
                root[j] = random_round(root[j] * inv_r, random20(t.position + (uint32_t)(i + j), h.key));
            }
            store_codes(t.exp_avg, i, left, encode_codes(m));
            store_codes(t.exp_avg_sq, i, left, encode_codes(root));
            if ((threadIdx.x & 15) == 0)
                reinterpret_cast<float2*>(t.scales)[i / kStepBlock] = make_float2(some_m ? most_m * (1.f / kFp8Most) : 0.f, some_r ? most_r * (1.f / kFp8Most) : 0.f);
        } else {
            store_eight<true>(t.exp_avg, i, left, m);
            store_eight<true>(t.exp_avg_sq, i, left, v);
        }
    }
}

// Sum over a workgroup of kNormThreads, in a fixed order; every thread gets it.
constexpr int kNormThreads = 1024, kNormGroups = kNormThreads / 256;
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double part[kNormThreads / kWave];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    __syncthreads();   // (used twice)
    if (lane_id() == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < kNormThreads / kWave; ++w) x += part[w];
    return x;
}

template <bool kGrad32>
__device__ __forceinline__ double squares(const Eight<kGrad32>& grad) {
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const double g = grad.get(j);
        sum = fma(g, g, sum);
    }
    return sum;
}

// Squares are summed in fp64: those of gradients past 1e19 leave the range of fp32.  Four groups of 256 threads a workgroup, each with every
// fourth of its records; a record's loads are out together, and the next record's pointers before them.  The workgroup that ends last
// adds the partial sums up, in their order: they are written and read past the caches of one XCD, and the count of those that
// ended is left at zero for the next call.  A second launch for it costs 4 us more.
template <bool kGrad32>
__global__ __launch_bounds__(kNormThreads) void grad_norm_kernel(const StepChunk* __restrict__ plan, int64_t chunks, float max_norm, float* __restrict__ out,
                                                                 uint32_t* __restrict__ ended, double* __restrict__ partial) {
    __shared__ bool last;
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), thread = threadIdx.x & 255;
    const int64_t stride = (int64_t)gridDim.x * kNormGroups;
    double sum = 0.0;
    int64_t k = (int64_t)blockIdx.x * kNormGroups + group;
    StepChunk next{};
    if (k < chunks) next = plan[k];
    for (; k < chunks; k += stride) {
        const StepChunk t = next;
        if (k + stride < chunks) next = plan[k + stride];
        if (t.count == kStepChunk) {
            Eight<kGrad32> grad[kStepChunk / 2048];
#pragma unroll
            for (int u = 0; u < kStepChunk / 2048; ++u) grad[u] = load_eight<kGrad32, true>(t.grad, thread * 8 + 2048 * u, 8);
#pragma unroll
            for (int u = 0; u < kStepChunk / 2048; ++u) sum += squares<kGrad32>(grad[u]);
        } else {
            for (int i = thread * 8; i < t.count; i += 2048) sum += squares<kGrad32>(load_eight<kGrad32>(t.grad, i, t.count - i));
        }
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) {
        __hip_atomic_store(partial + blockIdx.x, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // it is in memory
        last = __hip_atomic_fetch_add(ended, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;   // the same for the whole workgroup
    sum = 0.0;
    if (threadIdx.x < gridDim.x) sum = __hip_atomic_load(partial + threadIdx.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sum = block_sum(sum);
    if (threadIdx.x == 0) {
        const float norm = (float)sqrt(sum);
        const float factor = max_norm / (norm + 1e-6f);
        out[0] = norm;
        out[1] = fabsf(norm) < __builtin_inff() ? (factor < 1.f ? factor : 1.f) : __builtin_nanf("");
        __hip_atomic_store(ended, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

int64_t step_chunks(const int64_t* counts, int64_t n) {
    int64_t chunks = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (counts[i] < 0 || counts[i] > kStepMaxCount) return -1;
        chunks += (counts[i] + kStepChunk - 1) / kStepChunk;
        if (chunks > kStepMaxChunks) return -1;
    }
    return chunks;
}

void write_step_plan(const salr_step_tensor_t* tensors, int64_t n, bool param32, bool grad32, int state_bits, StepChunk* out) {
    uint64_t position = 0;
    const auto moved = [](auto* p, int64_t bytes) { return p == nullptr ? nullptr : reinterpret_cast<decltype(p)>(reinterpret_cast<uintptr_t>(p) + bytes); };
    for (int64_t i = 0; i < n; ++i) {
        const salr_step_tensor_t& t = tensors[i];
        for (int64_t at = 0; at < t.count; at += kStepChunk) {
            StepChunk c{};
            c.grad = moved(t.grad, at * (grad32 ? 4 : 2));
            if (state_bits != 0) {
                c.param = moved(t.param, at * (param32 ? 4 : 2));
                c.copy = param32 ? moved(t.copy, at * 2) : nullptr;
                c.exp_avg = moved(t.exp_avg, at * (state_bits / 8));
                c.exp_avg_sq = moved(t.exp_avg_sq, at * (state_bits / 8));
                c.scales = state_bits == 8 ? moved(t.scales, at / kStepBlock * 8) : nullptr;
            }
            c.count = (int32_t)(t.count - at < kStepChunk ? t.count - at : kStepChunk);
            c.position = (uint32_t)(position + (uint64_t)at);
            *out++ = c;
        }
        position += (uint64_t)((t.count + kStepBlock - 1) / kStepBlock * kStepBlock);
    }
}

hipError_t launch_adamw(const StepChunk* plan, int64_t chunks, bool param32, bool grad32, bool eight, const AdamwArgs& a, hipStream_t stream) {
    if (chunks == 0) return hipSuccess;
    StepScalars h;
    h.beta1 = (float)a.beta1;
    h.beta2 = (float)a.beta2;
    h.keep1 = (float)(1.0 - a.beta1);
    h.keep2 = (float)(1.0 - a.beta2);
    h.rate = (float)(a.lr / (1.0 - std::pow(a.beta1, (double)a.step)));
    h.shrink = (float)(1.0 - a.lr * a.weight_decay);
    h.root_scale = (float)(1.0 / std::sqrt(1.0 - std::pow(a.beta2, (double)a.step)));
    h.eps = (float)a.eps;
    h.key = (uint32_t)a.seed * 0x85157AF5u;
    typedef void (*Kernel)(const StepChunk*, StepScalars, const float*);
    static_assert(kStepParts * 2048 == kStepChunk, "a record is covered");
    static constexpr Kernel kernels[2][2][2] = {{{adamw_kernel<false, false, false>, adamw_kernel<false, false, true>},
                                                 {adamw_kernel<false, true, false>, adamw_kernel<false, true, true>}},
                                                {{adamw_kernel<true, false, false>, adamw_kernel<true, false, true>},
                                                 {adamw_kernel<true, true, false>, adamw_kernel<true, true, true>}}};
    constexpr int64_t kAtOnce = kMostThreads / (kStepParts * 256);   // records: 34 G elements
    for (int64_t first = 0; first < chunks; first += kAtOnce) {
        const int64_t here = chunks - first < kAtOnce ? chunks - first : kAtOnce;
        hipLaunchKernelGGL(kernels[param32][grad32][eight], dim3((unsigned)(here * kStepParts)), dim3(256), 0, stream, plan + first, h, a.grad_scale);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_grad_norm(const StepChunk* plan, int64_t chunks, bool grad32, float max_norm, float* out, void* workspace, hipStream_t stream) {
    uint32_t* ended = static_cast<uint32_t*>(workspace);
    double* partial = reinterpret_cast<double*>(static_cast<char*>(workspace) + 256);
    const int64_t groups = (chunks + kNormGroups - 1) / kNormGroups;
    const int blocks = (int)(groups < 1 ? 1 : groups < kGradNormBlocks ? groups : kGradNormBlocks);
    if (grad32) hipLaunchKernelGGL(grad_norm_kernel<true>, dim3(blocks), dim3(kNormThreads), 0, stream, plan, chunks, max_norm, out, ended, partial);
    else hipLaunchKernelGGL(grad_norm_kernel<false>, dim3(blocks), dim3(kNormThreads), 0, stream, plan, chunks, max_norm, out, ended, partial);
    return hipGetLastError();
}

}  // namespace salr
