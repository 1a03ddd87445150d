// Dropout, with the residual that it is added to: y = residual + (keep ? x / (1 - p) : 0).  Which elements stay follows from their
// positions and a seed, so that the backward pass, the same call on the gradient, forms the mask anew and none is stored.
//
// Random bits: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011), the counter a block of
// eight elements and the caller's offset, the key the seed: a block's four words are 16 bits for each of its elements.  p is taken in steps
// of 2^-16 for that, and 1 / (1 - p) of the step that was taken, so that the mean is right.  32 bits an element would be twice the rounds,
// and with those the kernel is near to what the integer units can do: a round is two 32 x 32 bit products at a quarter of the rate and four
// xors, 24 cycles of a lane, so ten rounds over eight elements are 30 beside some 10 for the element itself.
#include "salr_eight.hpp"
#include "salr_internal.hpp"

namespace salr {

__device__ __forceinline__ uint4 philox(uint64_t counter, uint64_t offset, uint64_t seed) {
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// A thread takes a block of eight at a time, the grid strides.  y may be x or residual: a block is read before it is written, by its thread.
template <bool k32, bool kResidual>
__global__ __launch_bounds__(256) void dropout_kernel(const void* x, const void* residual, int64_t count, uint32_t cut, float scale, uint64_t seed,
                                                      const int64_t* seed_at, uint64_t offset, void* y) {
    constexpr int kBytes = 8 * (k32 ? 4 : 2);
    if (seed_at != nullptr) seed = (uint64_t)*seed_at;
    const int64_t blocks = (count + 7) >> 3, stride = (int64_t)gridDim.x * 256;
    for (int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x; b < blocks; b += stride) {
        const int left = count - 8 * b < 8 ? (int)(count - 8 * b) : 8;
        const Eight<k32> in = load_eight<k32, false, false>(static_cast<const char*>(x) + b * kBytes, 0, left);
        Eight<k32> r;
        if constexpr (kResidual) r = load_eight<k32, false, false>(static_cast<const char*>(residual) + b * kBytes, 0, left);
        const uint4 words = philox((uint64_t)b, offset, seed);
        float out[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t w = j < 2 ? words.x : j < 4 ? words.y : j < 6 ? words.z : words.w;
            const bool keep = ((j & 1) ? w >> 16 : w & 0xFFFFu) >= cut;
            const float v = in.get(j) * scale;
            out[j] = keep ? v : 0.f;   // (a selection: what is dropped may be infinite or NaN)
            if constexpr (kResidual) out[j] += r.get(j);
        }
        store_eight<k32, false>(static_cast<char*>(y) + b * kBytes, 0, left, out);
    }
}

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t stream) {
    const int64_t groups = (a.count + 2047) / 2048, most = 8192;
    const dim3 grid((unsigned)(groups < most ? groups : most));
    const float scale = 65536.f / (float)(65536 - a.cut);
    const auto run = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a.x, a.residual, a.count, a.cut, scale, (uint64_t)a.seed, a.seed_at, (uint64_t)a.offset, a.y);
    };
    if (a.f32) a.residual ? run(dropout_kernel<true, true>) : run(dropout_kernel<true, false>);
    else a.residual ? run(dropout_kernel<false, true>) : run(dropout_kernel<false, false>);
    return hipGetLastError();
}

}  // namespace salr
