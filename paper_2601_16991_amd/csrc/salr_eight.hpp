// Eight consecutive elements of a tensor in fp32 or bf16, as the elementwise kernels take them: one or two 16-byte vectors.
#pragma once

#include "salr_device.hpp"
#include "salr_linear_common.hpp"

namespace salr {

typedef uint32_t AlignedUint4 __attribute__((ext_vector_type(4)));
typedef AlignedUint4 AnyUint4 __attribute__((aligned(2)));   // at any element's address

template <bool k32>
struct Eight {   // eight elements as they are in memory
    uint4 q[k32 ? 2 : 1];
    __device__ __forceinline__ float get(int j) const {
        if constexpr (k32) {
            const uint4 v = q[j >> 2];
            return __uint_as_float((j & 3) == 0 ? v.x : (j & 3) == 1 ? v.y : (j & 3) == 2 ? v.z : v.w);
        } else {
            return bf16_bits_to_f32(unit_elem(q[0], j));
        }
    }
};

// Elements i .. i + 7 of a tensor of which `left` are there (zeros for the others).  kOnce: not kept in the caches, for a pass that only
// reads (132 M gradients in bf16 47 us so, 53 otherwise; where the pass writes them back it is the other way round, 712 and 685 us).
// kAligned: base is 16-byte aligned and i a multiple of eight; else of elements anywhere (rows of odd lengths: one request a vector all the same,
// which the memory pipeline takes at any address).
template <bool k32, bool kOnce = false, bool kAligned = true>
__device__ __forceinline__ Eight<k32> load_eight(const void* base, int i, int left) {
    Eight<k32> r;
    if (left >= 8) {
        if constexpr (!kAligned) {
            const AnyUint4* any = reinterpret_cast<const AnyUint4*>(static_cast<const char*>(base) + (int64_t)i * (k32 ? 4 : 2));
            r.q[0] = __builtin_bit_cast(uint4, any[0]);
            if constexpr (k32) r.q[1] = __builtin_bit_cast(uint4, any[1]);
            return r;
        }
        const uint4* from = reinterpret_cast<const uint4*>(static_cast<const char*>(base) + (int64_t)i * (k32 ? 4 : 2));
        if constexpr (kOnce) {
            typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
            const u32x4_t* q = reinterpret_cast<const u32x4_t*>(from);
            r.q[0] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(q));
            if constexpr (k32) r.q[1] = __builtin_bit_cast(uint4, __builtin_nontemporal_load(q + 1));
        } else {
            r.q[0] = from[0];
            if constexpr (k32) r.q[1] = from[1];
        }
    } else {
        uint32_t e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            e[j] = 0;
            if (j < left) e[j] = k32 ? static_cast<const uint32_t*>(base)[i + j] : static_cast<const uint16_t*>(base)[i + j];
        }
        if constexpr (k32) {
            r.q[0] = make_uint4(e[0], e[1], e[2], e[3]);
            r.q[1] = make_uint4(e[4], e[5], e[6], e[7]);
        } else {
            r.q[0] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
        }
    }
    return r;
}

// The same eight elements, from element `at` on of a matrix of `total` >= 8, of a row of any length, in two steps that hold no branch, so that many requests
// are under way at once (with load_eight a wave at the end of a row waits for each): raw_eight asks for them, pulled back from the
// matrix' end where they would leave it; true_eight shifts what came to its place and puts zeros behind the first `left`.
template <bool k32>
__device__ __forceinline__ Eight<k32> raw_eight(const void* matrix, int64_t at, int64_t total) {
    return load_eight<k32, false, false>(static_cast<const char*>(matrix) + (at < total - 8 ? at : total - 8) * (k32 ? 4 : 2), 0, 8);
}
template <bool k32>
__device__ __forceinline__ Eight<k32> true_eight(const Eight<k32>& q, int64_t at, int left, int64_t total) {
    Eight<k32> r = q;
    const int64_t past = at - (total - 8);
    const int by = past <= 0 ? 0 : past < 8 ? (int)past : 8;
    if (__any(by > 0 || left < 8)) {   // (a wave in the middle of a row has nothing to do)
        uint32_t e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (k32) {
                const uint4 v = q.q[j >> 2];
                e[j] = (j & 3) == 0 ? v.x : (j & 3) == 1 ? v.y : (j & 3) == 2 ? v.z : v.w;
            } else {
                e[j] = unit_elem(q.q[0], j);
            }
        }
#pragma unroll
        for (int step = 1; step < 8; step *= 2)
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = by & step ? (j + step < 8 ? e[j + step] : 0u) : e[j];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = j < left && by < 8 ? e[j] : 0u;
        if constexpr (k32) {
            r.q[0] = make_uint4(e[0], e[1], e[2], e[3]);
            r.q[1] = make_uint4(e[4], e[5], e[6], e[7]);
        } else {
            r.q[0] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
        }
    }
    return r;
}

template <bool k32, bool kAligned = true>
__device__ __forceinline__ void store_eight(void* base, int i, int left, const float (&x)[8]) {
    if (left >= 8) {
        AlignedUint4 q[k32 ? 2 : 1];
        if constexpr (k32) {
            q[0] = AlignedUint4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
            q[1] = AlignedUint4{__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])};
        } else {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));   // (rounded to nearest, ties to even)
            uint32_t e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x[2 * j], (__bf16)x[2 * j + 1]});
            q[0] = AlignedUint4{e[0], e[1], e[2], e[3]};
        }
        char* at = static_cast<char*>(base) + (int64_t)i * (k32 ? 4 : 2);
#pragma unroll
        for (int v = 0; v < (k32 ? 2 : 1); ++v) {
            if constexpr (kAligned) reinterpret_cast<AlignedUint4*>(at)[v] = q[v];
            else reinterpret_cast<AnyUint4*>(at)[v] = q[v];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j >= left) break;
            if constexpr (k32) static_cast<float*>(base)[i + j] = x[j];
            else static_cast<uint16_t*>(base)[i + j] = f32_to_bf16_rne(x[j]);
        }
    }
}

}  // namespace salr
