// Tile of a matrix product on the matrix cores with both operands from row-major memory as it is, through LDS:
//
//   C[m][n] = sum_k P(m, k) Q(n, k)
//
// An operand lies in memory along k (P[m][k]: "rows" layout) or across it (P[k][m]: "columns" layout, transposed on its way from
// LDS to registers by ds_read_b64_tr_b16).  Workgroup: kWM x kWN waves, wave tile 16 kMI (m) x 16 kNI (n), tile of n always 256
// wide, steps of 64 along k.  Loads go straight to LDS (16 bytes a lane) into a ring of kStages steps; nothing is read past an
// operand's end: rows, columns and steps that are not there come out of the buffer load as zeros.
//
// LDS of one step.  Rows layout: [rows][64] with rows of 128 bytes, 16-byte piece c of row r at c ^ ((r >> 1) & 7).  Columns layout:
// [64][256] with rows of 512 bytes, 32-byte piece c of row k at c ^ ((k & 3) | ((k >> 3) & 3) << 2): the sixteen rows that one
// transposing read touches lie on different banks.
#pragma once

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

// One operand's tile: kRows wide (m or n), k-steps [.., ..) of `steps` from `k0` on.  All members but the lane's are uniform.
template <bool kColumns, int kRows, int kWaves>
struct TileSource {
    static_assert(!kColumns || kRows == 256, "columns layout: tiles of 256");
    static constexpr int kLoads = kRows / 8 / kWaves > 0 ? kRows / 8 / kWaves : 1;   // 1 KB each, per wave and step
    static constexpr int kBytes = kRows * 128;
    static constexpr uint32_t kOut = 0xFFFFFFF0u;   // past every buffer: zeros

    uint64_t base;      // of step 0
    int64_t bytes;      // from there to the end of the last row of the tile
    uint32_t advance;   // bytes a step
    uint32_t pitch;     // bytes a row
    uint32_t offset;    // this lane's place in load 0
    uint32_t stride;    // from load to load
    uint32_t loads_here;   // loads of this wave (rows layout with fewer rows than waves * 8: 0 or 1)
    int32_t k_left;     // rows layout: columns from this lane's first one of step 0 to the end

    // rows layout: `rows_left` rows from p on, each `k_end` long; columns layout: k_end rows, `rows_left` columns from p on
    __device__ __forceinline__ TileSource(const uint16_t* p, int64_t pitch_elems, int64_t rows_left, int64_t k_end, int wave, int lane) {
        base = reinterpret_cast<uint64_t>(p);
        pitch = (uint32_t)(pitch_elems * 2);
        loads_here = kRows / 8 >= kWaves ? kLoads : (wave < kRows / 8 ? 1 : 0);
        if constexpr (!kColumns) {
            const int row = 8 * wave + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
            offset = row * pitch + piece * 16;
            stride = 8 * kWaves * pitch;
            advance = 128;
            bytes = (rows_left < kRows ? rows_left : kRows) * (int64_t)pitch - (pitch - (int64_t)k_end * 2);
            k_left = (int32_t)(k_end - 8 * piece);
        } else {
            // load j: step rows 2 (wave + kWaves j) and the next one; with 8 waves the swizzle of row + 16 j differs, so the piece
            // is worked out per load
            const int row = 2 * wave + (lane >> 5);
            offset = row * pitch;
            stride = 2 * kWaves * pitch;
            advance = 64 * pitch;
            bytes = k_end * (int64_t)pitch - (pitch - (rows_left < kRows ? rows_left : kRows) * 2);
            k_left = (int32_t)(rows_left < kRows ? rows_left : kRows);   // columns of the tile that are there
        }
    }

    // Load j of step `s` to LDS at `lds` (uniform): all of it in assembly, so that the waits stay with the caller.  `live`: the step exists.
    __device__ __forceinline__ void fetch(int s, int j, uint32_t lds, bool live, int wave, int lane) const {
        if (kRows / 8 < kWaves && loads_here == 0) return;
        const uint64_t at = base + (uint64_t)s * advance;
        const int64_t left = live ? bytes - (int64_t)s * advance : 0;
        const uint32_t room = left <= 0 ? 0u : left < 0x7FFFFFFF ? (uint32_t)left : 0x7FFFFFFFu;
        uint32_t v;
        if constexpr (!kColumns) {
            v = 64 * s < k_left ? offset + j * stride : kOut;
        } else {
            const int row = 2 * (wave + kWaves * j) + (lane >> 5), slot = lane & 31;
            const int piece = (((slot >> 1) ^ ((row & 3) | ((row >> 3) & 3) << 2)) << 1) | (slot & 1);
            v = 8 * piece < k_left ? offset + j * stride + piece * 16 : kOut;
        }
        const u32x4 buffer = {(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, room, 0x00020000u};
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (wave + kWaves * j) * 1024);
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(v), "s"(buffer), "s"(to) : "memory", "m0");
    }
};

// Sixteen rows (from `row0` on) by 32 k (half `s` of the step) of a tile, as an operand of the instruction.
template <bool kColumns>
__device__ __forceinline__ bf16x8 tile_operand(const char* tile, int row0, int s, int lane) {
    const int i = lane & 15, g = lane >> 4;
    if constexpr (!kColumns) {
        const int row = row0 + i;
        return *reinterpret_cast<const bf16x8*>(tile + row * 128 + (((4 * s + g) ^ ((row >> 1) & 7)) * 16));
    } else {
        // lane i of a group of sixteen names 8 bytes: k row (i / 4), columns 4 (i % 4) ..; it receives column i of the four rows
        typedef __attribute__((address_space(3))) bf16x4* LdsPtr;
        bf16x4 half[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = 32 * s + 8 * g + 4 * h + (i >> 2);
            const int piece = (row0 >> 4) ^ ((k & 3) | ((k >> 3) & 3) << 2);
            half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((LdsPtr)(tile + k * 512 + piece * 32 + (i & 3) * 8));
        }
        return __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
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

// Shape of a workgroup's tile: 16 kMI kWM x 256.
template <int kMI_, int kWM_, int kStages_>
struct TileShape {
    static constexpr int kMI = kMI_, kWM = kWM_, kStages = kStages_;
    static constexpr int kWN = 8 / kWM, kNI = 16 / kWN, kWaves = 8, kThreads = 512;
    static constexpr int kM = 16 * kMI * kWM, kN = 256;
    static constexpr int kStageBytes = (kM + kN) * 128;
    static constexpr int kLdsBytes = kStages * kStageBytes;
};

// The k loop over steps [begin, end) of both sources; acc[i][j] += ... .  `adjust(p, s, half, i)` may change the operand of P (m).
// On return every wave has read its last operands and no load is under way.
template <class Shape, bool kPColumns, bool kQColumns, class Adjust>
__device__ __forceinline__ void tile_product(const TileSource<kPColumns, Shape::kM, 8>& ps, const TileSource<kQColumns, 256, 8>& qs, int begin, int end,
                                             char* lds, f32x4 (&acc)[Shape::kMI][Shape::kNI], Adjust&& adjust) {
    constexpr int S = Shape::kStages, kMI = Shape::kMI, kNI = Shape::kNI;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / Shape::kWN, wn = wave % Shape::kWN;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
    constexpr int kPLoads = TileSource<kPColumns, Shape::kM, 8>::kLoads, kQLoads = TileSource<kQColumns, 256, 8>::kLoads;
    auto fetch = [&](int s, int slot) {
        const uint32_t to = lds0 + slot * Shape::kStageBytes;
#pragma unroll
        for (int j = 0; j < kQLoads; ++j) qs.fetch(s, j, to + Shape::kM * 128, s < end, wave, lane);
#pragma unroll
        for (int j = 0; j < kPLoads; ++j) ps.fetch(s, j, to, s < end, wave, lane);
    };
#pragma unroll
    for (int p = 0; p < S - 1; ++p) fetch(begin + p, p);
    int slot = 0;
    for (int s = begin; s < end; ++s) {
        // step s has landed (at most the loads of the S - 2 steps after it are under way; a wave that has none of P's waits longer), and
        // every wave is through with step s - 1, whose slot the next request fills
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((S - 2) * (kQLoads + (Shape::kM >= 64 ? kPLoads : 0))) : "memory");
        const int last = slot == 0 ? S - 1 : slot - 1;
        fetch(s + S - 1, last);
        const char* pt = lds + slot * Shape::kStageBytes;
        const char* qt = pt + Shape::kM * 128;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            bf16x8 q[kNI], p[kMI];
#pragma unroll
            for (int j = 0; j < kNI; ++j) q[j] = tile_operand<kQColumns>(qt, 16 * (wn * kNI + j), half, lane);
#pragma unroll
            for (int i = 0; i < kMI; ++i) p[i] = adjust(tile_operand<kPColumns>(pt, 16 * (wm * kMI + i), half, lane), s, i);
#pragma unroll
            for (int i = 0; i < kMI; ++i)
#pragma unroll
                for (int j = 0; j < kNI; ++j) product_mfma(acc[i][j], q[j], p[i]);
        }
        slot = slot + 1 == S ? 0 : slot + 1;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

}  // namespace salr
