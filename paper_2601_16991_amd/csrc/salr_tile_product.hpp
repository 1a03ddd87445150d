// Tile of a matrix product on the matrix cores with both operands from row-major memory as it is, through LDS:
//
//   C[m][n] = sum_k P(m, k) Q(n, k)
//
// An operand lies in memory along k (P[m][k]: "rows" layout) or across it (P[k][m]: "columns" layout, transposed on its way from
// LDS to registers by ds_read_b64_tr_b16).  Workgroup: kWM x kWN waves, wave tile 16 kMI (m) x 16 kNI (n), steps of
// 64 along k.  Loads go straight to LDS (16 bytes a lane), each operand into a ring of its own; nothing is read past an
// operand's end: rows, columns and steps that are not there come out of the buffer load as zeros.
//
// LDS of one step.  Rows layout: [rows][64] with rows of 128 bytes, 16-byte piece c of row r at c ^ rows_swizzle(r).  Columns layout:
// [64][256] with rows of 512 bytes, 32-byte piece c of row k at c ^ columns_swizzle(k): the sixteen rows that one transposing read
// touches lie on different banks.
#pragma once

#include <type_traits>

#include "salr_device.hpp"

namespace salr {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kProductXcds = 8;

// c += a b, a: sixteen n, b: sixteen m; lane 16 g + i then holds n = 4 g .. 4 g + 3 of m = i.
__device__ __forceinline__ void product_mfma(f32x4& c, const bf16x8& a, const bf16x8& b) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

constexpr int kProductStep = 64;   // of k

__device__ __forceinline__ int rows_swizzle(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ int columns_swizzle(int k) { return (k & 3) | ((k >> 3) & 3) << 2; }

// One operand's tile: kRows wide (m or n), steps of k counted from its start.  All members but the lane's are uniform.
template <bool kColumns, int kRows, int kWaves>
struct TileSource {
    static_assert(!kColumns || kRows == 256, "columns layout: tiles of 256");
    static constexpr int kInstructions = kRows / 8;   // loads of 1 KB in a step, of all waves
    static constexpr int kLoads = kInstructions >= kWaves ? kInstructions / kWaves : 1;
    static constexpr bool kAllWaves = kInstructions >= kWaves;
    static constexpr uint32_t kOut = 0xFFFFFFF0u;   // past every buffer: zeros

    uint64_t base;      // of step 0
    int64_t bytes;      // from there to the end of the last row of the tile
    uint32_t advance;   // bytes a step
    uint32_t offset;    // this lane's place in load 0
    uint32_t stride;    // from load to load
    int32_t k_left;     // rows layout: columns from this lane's first one of step 0 to the end; columns layout: columns of the tile that exist

    // rows layout: `rows_left` rows from p on, each `k_end` long; columns layout: k_end rows, `rows_left` columns from p on
    __device__ __forceinline__ TileSource(const uint16_t* p, int64_t pitch_elems, int64_t rows_left, int64_t k_end, int wave, int lane) {
        base = reinterpret_cast<uint64_t>(p);
        const uint32_t pitch = (uint32_t)(pitch_elems * 2);
        const int64_t here = rows_left < kRows ? rows_left : kRows;
        if constexpr (!kColumns) {   // load j: rows 8 (wave + kWaves j) .. + 7, eight lanes each
            const int row = 8 * wave + (lane >> 3), piece = (lane & 7) ^ rows_swizzle(row);
            offset = row * pitch + piece * 16;
            stride = 8 * kWaves * pitch;
            advance = kProductStep * 2;
            bytes = here * (int64_t)pitch - (pitch - (int64_t)k_end * 2);
            k_left = (int32_t)(k_end - 8 * piece);
        } else {   // load j: k rows 2 (wave + kWaves j) and the next one, 32 lanes each
            offset = (2 * wave + (lane >> 5)) * pitch;
            stride = 2 * kWaves * pitch;
            advance = kProductStep * pitch;
            bytes = k_end * (int64_t)pitch - (pitch - here * 2);
            k_left = (int32_t)here;
        }
    }

    // Load j of step `s` to LDS at `lds` (uniform): all of it in assembly, so that the waits stay with the caller.  `live`: the step exists.
    __device__ __forceinline__ void fetch(int s, int j, uint32_t lds, bool live, int wave, int lane) const {
        if (!kAllWaves && wave >= kInstructions) return;
        const uint64_t at = base + (uint64_t)s * advance;
        const int64_t left = live ? bytes - (int64_t)s * advance : 0;
        const uint32_t room = left <= 0 ? 0u : left < 0x7FFFFFFF ? (uint32_t)left : 0x7FFFFFFFu;
        uint32_t v;
        if constexpr (!kColumns) {
            v = kProductStep * s < k_left ? offset + j * stride : kOut;
        } else {
            const int row = 2 * (wave + kWaves * j) + (lane >> 5), slot = lane & 31;
            const int piece = (((slot >> 1) ^ columns_swizzle(row)) << 1) | (slot & 1);
            v = 8 * piece < k_left ? offset + j * stride + piece * 16 : kOut;
        }
        const u32x4 buffer = {(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, room, 0x00020000u};
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (wave + kWaves * j) * 1024);
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(v), "s"(buffer), "s"(to) : "memory", "m0");
    }
};

// Sixteen rows (from `row0` on) by 32 of k (half of a step) of a tile, as an operand of the instruction.
template <bool kColumns>
__device__ __forceinline__ bf16x8 tile_operand(const char* tile, int row0, int half, int lane) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (!kColumns) {
        const int row = row0 + i;
        return *reinterpret_cast<const bf16x8*>(tile + row * 128 + (((4 * half + g) ^ rows_swizzle(row)) * 16));
    } else {
        // lane i of a group of sixteen names 8 bytes: k row (i / 4), columns 4 (i % 4) ..; it receives column i of the four rows
        typedef __attribute__((address_space(3))) bf16x4* LdsPtr;
        bf16x4 four[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = 32 * half + 8 * g + 4 * h + (i >> 2);
            four[h] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsPtr)(tile + k * 512 + ((row0 >> 4) ^ columns_swizzle(k)) * 32 + (i & 3) * 8));
        }
        return __builtin_shufflevector(four[0], four[1], 0, 1, 2, 3, 4, 5, 6, 7);
    }
}

// Which tile a workgroup takes.  Consecutive ids land on different XCDs, each with an L2 of its own: XCD c takes the c-th eighth of
// the work, ordered so that workgroups side by side on it share operands: k slice, groups of eight m-tiles, n, m.
struct TilePlace {
    int mt, nt, kz;
    bool any;
    __device__ __forceinline__ TilePlace(int m_tiles, int n_tiles, int slices) {
        const int per_k = m_tiles * n_tiles, total = per_k * slices, per_xcd = (total + kProductXcds - 1) / kProductXcds;
        const int id = (int)blockIdx.x % kProductXcds * per_xcd + (int)blockIdx.x / kProductXcds;
        any = id < total && (int)blockIdx.x / kProductXcds < per_xcd;
        kz = id / per_k;
        const int tile = id % per_k, mg = tile / (8 * n_tiles), in_group = tile - mg * 8 * n_tiles;
        const int group_rows = m_tiles - 8 * mg < 8 ? m_tiles - 8 * mg : 8;
        nt = in_group / group_rows;
        mt = 8 * mg + in_group % group_rows;
    }
};
inline unsigned product_grid(int64_t workgroups) { return (unsigned)((workgroups + kProductXcds - 1) / kProductXcds * kProductXcds); }

// Shape of a workgroup's tile: 16 kMI kWM (m) x 16 kNI kWN (n); steps of either operand that LDS holds.
template <int kMI_, int kNI_, int kWM_, int kWN_, int kPSlots_, int kQSlots_>
struct TileShape {
    static constexpr int kMI = kMI_, kNI = kNI_, kWM = kWM_, kWN = kWN_, kPSlots = kPSlots_, kQSlots = kQSlots_;
    static constexpr int kWaves = kWM * kWN, kThreads = 64 * kWaves;
    static constexpr int kM = 16 * kMI * kWM, kN = 16 * kNI * kWN;
    static constexpr int kPBytes = kM * 2 * kProductStep, kQBytes = kN * 2 * kProductStep;
    static constexpr int kLdsBytes = kPSlots * kPBytes + kQSlots * kQBytes;
    static_assert(kPSlots >= 2 && (kQSlots == kPSlots || kQSlots == 3), "see tile_product");
    static_assert(kN / 8 >= kWaves, "every wave has loads of Q");
};

// The k loop over steps [begin, end) of both sources; acc[i][j] += ... .  On return every wave has read its last operands and no load is
// under way.
//
// A step is two halves of 32 along k.  The operands of a half are read from LDS during the products of the half before.  The barrier
// between the halves says that the next step has landed, and that every wave holds the rest of this one in registers: its slots are free.
// Requests are spread over the products, because a burst of them holds the waves up (4 to 6 % of a call): P's into the slot just left, in
// the second half; Q's, where it has a slot more, in the first half of the next step (3 % of a call).
//
// On 256 x 256 tiles the chip's power is the limit: 4096 x 4096 x 32768 with Q transposed 777 us, 1415 TFLOP/s, at 1.8 GHz of 2.4 with the matrix cores busy 73 %
// of the cycles, LDS 27 %, no bank conflicts.  In a loop of nothing but products the instruction of 32 x 32 x 16 is 13 % slower than this one.  Of 1675 us (2048 x 4096 x 131072) 335 are the loads' (64 KB a step cross from an L2 to each CU), 125 the reads
// from LDS.  128 x 256 tiles: 0.9 us a step for 1.56, where they make a round of the CUs shorter.
// A workgroup makes one tile: going on to the next, its first steps requested before the stores, is 1 to 2 % slower, since loads and stores are waited for
// together, where those of a workgroup that has ended drain behind the next one's start.
// (Eight waves of 128 x 64, two a SIMD: four of 128 x 128 read a third less from LDS and are 5 to 7 % slower, a SIMD's one wave stands at every barrier.)
template <class Shape, bool kPColumns, bool kQColumns>
__device__ __forceinline__ void tile_product(const TileSource<kPColumns, Shape::kM, Shape::kWaves>& ps, const TileSource<kQColumns, Shape::kN, Shape::kWaves>& qs,
                                             int begin, int end, char* lds, f32x4 (&acc)[Shape::kMI][Shape::kNI]) {
    typedef TileSource<kPColumns, Shape::kM, Shape::kWaves> PSource;
    typedef TileSource<kQColumns, Shape::kN, Shape::kWaves> QSource;
    constexpr int SP = Shape::kPSlots, SQ = Shape::kQSlots, kMI = Shape::kMI, kNI = Shape::kNI, kLoads = PSource::kLoads + QSource::kLoads;
    // loads that every wave makes in a step (a wave that has one more waits for it earlier than it has to)
    constexpr int kSure = QSource::kLoads + (PSource::kAllWaves ? PSource::kLoads : 0);
    constexpr bool kApart = SQ > 2;
    constexpr int kSureP = PSource::kAllWaves ? PSource::kLoads : 0;
    // what may be under way when step s + 1 has to be there, by what was requested behind its two parts.  Apart: Q of step s + SQ - 1
    // during the half before, P of s + SP - 1 before that; else both of s + SP - 1 then.
    constexpr int kUnderWay = !kApart ? (SP - 2) * kSure : SP == 2 ? QSource::kLoads : (SQ - 3) * kSure + kSureP + QSource::kLoads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / Shape::kWN, wn = wave % Shape::kWN;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    constexpr int kQFirst = SP * Shape::kPBytes;   // Q's ring behind P's
    auto fetch_p = [&](int s, int slot, int c) { ps.fetch(s, c, lds0 + slot * Shape::kPBytes, s < end, wave, lane); };
    auto fetch_q = [&](int s, int slot, int c) { qs.fetch(s, c, lds0 + kQFirst + slot * Shape::kQBytes, s < end, wave, lane); };
    auto read = [&](int p_slot, int q_slot, int half, int c, bf16x8 (&q)[kNI], bf16x8 (&p)[kMI]) {
        if (c < kNI) q[c] = tile_operand<kQColumns>(lds + kQFirst + q_slot * Shape::kQBytes, 16 * (wn * kNI + c), half, lane);
        else p[c - kNI] = tile_operand<kPColumns>(lds + p_slot * Shape::kPBytes, 16 * (wm * kMI + c - kNI), half, lane);
    };
    constexpr int kQAhead = kApart ? SQ - 1 : SQ;   // steps of Q requested before the first
#pragma unroll
    for (int t = 0; t < (SP > kQAhead ? SP : kQAhead); ++t) {
#pragma unroll
        for (int c = 0; c < PSource::kLoads; ++c)
            if (t < SP) fetch_p(begin + t, t, c);
#pragma unroll
        for (int c = 0; c < QSource::kLoads; ++c)
            if (t < kQAhead) fetch_q(begin + t, t, c);
    }
    bf16x8 q0[kNI], p0[kMI], q1[kNI], p1[kMI];
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"((SP - 1) * kSureP + (kQAhead - 1) * QSource::kLoads) : "memory");
#pragma unroll
    for (int c = 0; c < kNI + kMI; ++c) read(0, 0, 0, c, q0, p0);
    // Products of one half, with the reads of the next (operands in the order in which its products want them) and `requests` spread over them.
    auto products = [&](const bf16x8 (&q)[kNI], const bf16x8 (&p)[kMI], auto&& read_next, auto requests, auto&& request) {
        constexpr int kRequests = decltype(requests)::value;
#pragma unroll
        for (int i = 0; i < kMI; ++i) {
#pragma unroll
            for (int c = (kNI + kMI) * i / kMI; c < (kNI + kMI) * (i + 1) / kMI; ++c) read_next(c);
#pragma unroll
            for (int c = kRequests * i / kMI; c < kRequests * (i + 1) / kMI; ++c) request(c);
#pragma unroll
            for (int t = 0; t < kNI; ++t) {
                const int j = i % 2 == 0 ? t : kNI - 1 - t;   // to and fro, one operand stays each time: 0.5 % of a call, in power
                product_mfma(acc[i][j], q[j], p[i]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    int p_slot = 0, q_slot = 0;
    for (int s = begin; s < end; ++s) {
        const int p_next = p_slot + 1 == SP ? 0 : p_slot + 1, q_next = q_slot + 1 == SQ ? 0 : q_slot + 1;
        const int q_before = q_slot == 0 ? SQ - 1 : q_slot - 1;
        products(q0, p0, [&](int c) { read(p_slot, q_slot, 1, c, q1, p1); }, std::integral_constant<int, kApart ? QSource::kLoads : 0>{},
                 [&](int c) { fetch_q(s + SQ - 1, q_before, c); });
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kUnderWay) : "memory");
        products(q1, p1, [&](int c) { read(p_next, q_next, 0, c, q0, p0); }, std::integral_constant<int, kApart ? PSource::kLoads : kLoads>{}, [&](int c) {
            if (c < PSource::kLoads) fetch_p(s + SP, p_slot, c);
            else fetch_q(s + SQ, q_slot, c - PSource::kLoads);
        });
        p_slot = p_next;
        q_slot = q_next;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

}  // namespace salr
