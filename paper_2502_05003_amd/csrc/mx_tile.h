// y = a b^T on microscaled operands (see mx_gemm.hip) for outputs of many tiles.  A workgroup of four waves works through tiles
// of 64 WI x 64 WJ outputs, each wave 32 WI x 32 WJ of them in accumulation registers, as one stream of stages: 128 bytes of
// each activation row (256 elements in E2M1, 128 in E4M3), whole cache lines, and the same elements of the weights.  Two stages
// of LDS, filled by direct transfers.
//
// A stage is multiplied block of 32 rows by block: the wave's weight fragments of the whole stage stay in registers, the
// activations' come one block ahead.  The last block of a stage runs behind the barrier that announces the next one:
//   barrier: the stage has landed, the other buffer has been left by all waves
//   phase 1   multiply block WI - 1 of the stage before; each weight fragment that is done with is replaced by the new stage's
//   phase 2   block 0 of the stage;  phase 3 ..  blocks 1 .. WI - 2
//   wait for the reads of block WI - 1 and for the next stage's transfers, which the first phases have issued; barrier
// Nothing but the waits for these two interrupts the matrix instructions, tile ends included: the transfers run on into the
// workgroup's next tile, whose first products start from zero (C = 0, no accumulator is cleared), and block b of a finished
// tile is rounded, parked in the wave's corner of LDS and stored as whole row segments while block b + 1 is multiplied.  The stores
// are issued behind their stage's transfers and counted, so that nothing waits for them before the end of the stage that follows
// (16384 x 5632 x 2048 132 -> 124 us, 16384 x 4096 x 1024 67 -> 62).
//
// What bounds it: with large contractions the chip's power (4096 x 4096 x 16640 in E2M1 139 to 148 us, 3.8 to 4.0 PFLOP/s; with
// operands of zeros 103, where the wave's instructions are the bound, one in 8 cycles; the matrix instructions alone, from
// registers, sustain 6.5), with short ones the tiles' ends on top (16384 x 5632 x 2048 119 us, 36 of them the output at the rate of
// a large copy; matrix pipes 0.33 busy).  Tried and dropped: each stage in two groups of transfers with a whole stage's time each, for a
// second barrier per stage (4096 x 4096 x 4096 41 -> 45 us); lines asked for two stages ahead (120 -> 140); all transfers in
// phase 1 or spread over all phases (the same within 2 %).
#pragma once

#include <algorithm>

#include "mx_formats.h"
#include "mx_stages.h"
#include "quest_internal.h"

namespace quest {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

constexpr int kF4 = 4, kF8 = 0;            // its codes for E2M1 and E4M3
constexpr int kTileThreads = 256;
constexpr int kParkBytes = 32 * 128;       // 32 rows by 64 columns in bf16

template <int FORMAT, int WI, int WJ>
struct MxTile {
    static constexpr bool kE4M3 = FORMAT == QUEST_MX_E4M3;
    static constexpr int kRows = 64 * WI, kCols = 64 * WJ;
    static constexpr int kSteps = kE4M3 ? 1 : 2;                 // matrix instructions along a stage
    typedef MxStages<kSteps> Stages;
    static constexpr int kRowA = 128, kRowB = 64 * kSteps;       // bytes of a row in a stage
    static constexpr int kBytesA = kRows * kRowA, kStage = kBytesA + kCols * kRowB;
    static constexpr int kScales = (kRows + kCols) * 16;
    static constexpr int kLds = 2 * kStage + 2 * kScales + 4 * kParkBytes;
    static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
};

// a range of memory for buffer instructions, which leave out what lies beyond it
__device__ __forceinline__ quest_v4u buffer_of(const void *p, uint32_t bytes)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    return quest_v4u{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, bytes, 0x00027000u};
}

// 16 bytes per lane from a buffer into LDS: lane l lands at lds_base + LDS_IMM + 16 l (see lds_dma16_at)
template <int LDS_IMM>
__device__ __forceinline__ void lds_buffer16_at(const quest_v4u &buffer, uint32_t lane_offset, uint32_t lds_base)
{
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                 :
                 : "v"(lane_offset), "s"(buffer), "s"(lds_base), "n"(LDS_IMM)
                 : "memory", "scc");
}

// The same IMM bytes further on in the buffer and in LDS, with M0 as it was left
template <int IMM>
__device__ __forceinline__ void lds_buffer16_next(const quest_v4u &buffer, uint32_t lane_offset)
{
    static_assert(IMM >= 0 && IMM < 4096, "the instruction's offset field");
    asm volatile("buffer_load_dwordx4 %0, %1, 0 offen offset:%2 lds" : : "v"(lane_offset), "s"(buffer), "n"(IMM) : "memory");
}

// what an iteration (a stage) of the stream is
enum {
    kStageFirst = 1,      // the first of its tile: the tile before ends in phase 1
    kAfterFirst = 2,      // the one behind it
    kStageLast = 4        // the last of its tile
};

// what a kernel stores
enum {
    kWholePieces = 0,     // y in 16-byte pieces: rows and columns that fit them
    kAnyRows = 1,         // y of any width, pitch and start
    kRawSums = 2          // the fp32 sums, and y as above, if it is wanted.  (Its three predicated stores for each four sums, beside
                          // all accumulators, do not fit the registers: 4096 x 4096 x 1024 in E2M1 50 us, y alone 19.)
};

// TWO: tiles of two stages (else more)
template <int FORMAT, int WI, int WJ, bool TWO, int OUT>
__global__ __launch_bounds__(kTileThreads, 1) void mx_tile_kernel(
    const uint8_t *__restrict__ a_codes, const uint8_t *__restrict__ a_scales, const uint8_t *__restrict__ b_codes,
    const uint8_t *__restrict__ b_scales, int M, int N, int K, int tiles_m, int tiles_n, uint16_t *__restrict__ y, int64_t ld_y,
    float *__restrict__ acc_out)
{
    typedef MxTile<FORMAT, WI, WJ> T;
    constexpr bool kE4M3 = T::kE4M3;
    constexpr int NJ = 2 * WJ, kFragB = T::kSteps * NJ;  // 16-column fragments of a wave; of a whole stage
    constexpr int nA = 2 * WI, nB = T::kCols * T::kRowB / 4096, kDma = nA + nB;   // transfers of a wave and stage
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];

    // Tiles of this workgroup: each XCD (workgroup ids go to the eight in turn) has one contiguous run of tiles, ordered four
    // tile-rows deep, of which its workgroups take every (number of workgroups)-th.
    const int total = tiles_m * tiles_n, per_xcd = (total + 7) / 8, peers = gridDim.x / 8;
    const int xcd = blockIdx.x & 7, run_end = min((xcd + 1) * per_xcd, total);
    int tile = xcd * per_xcd + (blockIdx.x >> 3);
    if (tile >= run_end)
        return;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = wave >> 1, wc = wave & 1;
    const int l16 = lane & 15, quarter = lane >> 4;
    const uint32_t smem_addr = lds_address(smem);
    const int64_t row_a = kE4M3 ? K : K / 2, row_b = K / 2;
    const int row_scales = K / 32;                       // bytes
    const int stages = T::Stages::count(K);
    const bool half_stage = T::Stages::ends_in_half(K);  // E2M1: the last stage of a tile holds 128 elements

    // ---- transfers, one stage ahead of the multiplication.  One moves 1 KiB: lane l lands at 16 l, so it fetches the chunk that
    // belongs there (see the reads below).  The rows of a tile are a buffer that ends with the operand: transfers of rows beyond
    // it bring nothing that is used or stored.
    quest_v4u fetch_a, fetch_b;
    const uint8_t *fetch_as, *fetch_bs;
    uint32_t fetch_rows_a, fetch_rows_b;
    auto set_fetch_tile = [&](int at, int &m0, int &n0) __attribute__((always_inline)) {
        const int band = at / (4 * tiles_n), band_rows = min(4, tiles_m - band * 4), in_band = at - band * 4 * tiles_n;
        m0 = __builtin_amdgcn_readfirstlane((band * 4 + in_band % band_rows) * T::kRows);
        n0 = __builtin_amdgcn_readfirstlane(in_band / band_rows * T::kCols);
        fetch_rows_a = min(T::kRows, M - m0);
        fetch_rows_b = min(T::kCols, N - n0);
        fetch_a = buffer_of(a_codes + m0 * row_a, fetch_rows_a * (uint32_t)row_a);
        fetch_b = buffer_of(b_codes + n0 * row_b, fetch_rows_b * (uint32_t)row_b);
        fetch_as = a_scales + (int64_t)m0 * row_scales;
        fetch_bs = b_scales + (int64_t)n0 * row_scales;
    };
    // Lanes' byte offsets, for rows of eight with an even and with an odd number, and what a half stage takes back of them: it
    // has no second half of a row's 128 bytes, whose lanes fetch the first again.
    uint32_t a_at[2], b_at[2];
    const uint32_t back[2] = {(lane & 4) ? 64u : 0u, (lane & 4) ? 0u : 64u};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int chunk = (lane & 7) ^ (4 * h + (lane >> 4));
        a_at[h] = (uint32_t)(wave * nA * 8 + (lane >> 3)) * (uint32_t)row_a + 16u * chunk;
        b_at[h] = T::kRowB == 128 ? (uint32_t)(wave * nB * 8 + (lane >> 3)) * (uint32_t)row_b + 16u * chunk
                                  : (uint32_t)(wave * nB * 16 + (lane >> 2)) * (uint32_t)row_b + 16u * ((lane & 3) ^ (lane >> 4));
    }
    auto transfer = [&](auto pc, uint32_t stage, int at, bool half) __attribute__((always_inline)) {
        constexpr int p = decltype(pc)::value, h = p & 1, q = p - nA;
        const uint32_t less = !kE4M3 && half ? back[h] : 0u;
        // (M0 for four at a time: the others differ in the instruction's offset, which moves both ends; rows are 128 bytes or more
        // apart, so the offset in memory that makes up for it is not negative)
        if constexpr (p < nA) {
            constexpr int more = 1024 * (p % 4);
            const uint32_t from = a_at[h] + (uint32_t)(8 * p * (int)row_a + at * T::kRowA - more) - less;
            if constexpr (more == 0)
                lds_buffer16_at<1024 * p>(fetch_a, from, stage + wave * (nA * 1024));
            else
                lds_buffer16_next<more>(fetch_a, from);
        } else {
            constexpr int more = 1024 * (q % 4);
            const uint32_t from = b_at[h] + (uint32_t)((T::kRowB == 128 ? 8 : 16) * q * (int)row_b + at * T::kRowB - more) - less;
            if constexpr (more == 0)
                lds_buffer16_at<T::kBytesA + 1024 * q>(fetch_b, from, stage + wave * (nB * 1024));
            else
                lds_buffer16_next<more>(fetch_b, from);
        }
    };
    const uint32_t scale_at = (uint32_t)lane * (uint32_t)row_scales;
    const uint32_t scale_addr = smem_addr + 2 * T::kStage;
    auto transfer_scales = [&](int buffer, int at) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < (WI + WJ + 3) / 4; ++h) {
            const int piece = wave + 4 * h;
            const bool left = piece < WI;
            if (piece >= WI + WJ)
                continue;
            lds_buffer16_at<0>(buffer_of(left ? fetch_as : fetch_bs, (left ? fetch_rows_a : fetch_rows_b) * (uint32_t)row_scales),
                               scale_at + (uint32_t)(64 * (left ? piece : piece - WI) * row_scales + 4 * T::Stages::chunk(at)),
                               scale_addr + buffer * T::kScales + piece * 1024);
        }
    };

    // ---- fragments.  Chunk c of row r of 128 bytes sits at c ^ ((r >> 1) & 7) (64 bytes: c ^ ((r >> 2) & 3)): sixteen
    // consecutive rows then meet sixteen different 16-byte slots modulo 256 bytes.
    //   E2M1, step t: chunk 4 t + quarter;  E4M3: chunks quarter and 4 + quarter
    uint4 af[2][2][2], bf[kFragB];         // activations: [block & 1][upper or lower 16 rows][chunk]
    uint32_t sa[WI][2], sb[NJ];            // scale bytes of the lane's row: byte t for step t
    const uint32_t a_lane = (wr * 32 * WI + l16) * T::kRowA + ((quarter ^ ((l16 >> 1) & 7)) << 4);
    const uint32_t b_lane = T::kBytesA + (wc * 32 * WJ + l16) * T::kRowB +
                            ((T::kRowB == 128 ? quarter ^ ((l16 >> 1) & 7) : quarter ^ ((l16 >> 2) & 3)) << 4);
    auto read_a = [&](const uint8_t *stage, auto block, auto number) __attribute__((always_inline)) {
        constexpr int i = decltype(block)::value, u = decltype(number)::value & 1, c = decltype(number)::value >> 1;
        af[i & 1][u][c] = *reinterpret_cast<const uint4 *>(stage + (a_lane ^ (c << 6)) + (32 * i + 16 * u) * T::kRowA);
    };
    auto read_b = [&](const uint8_t *stage, auto frag) __attribute__((always_inline)) {
        constexpr int f = decltype(frag)::value, t = f / NJ, j = f % NJ;
        bf[f] = *reinterpret_cast<const uint4 *>(stage + (b_lane ^ (t << 6)) + 16 * j * T::kRowB);
    };
    // A row's scales of a stage begin at dword `word` of its chunk (E2M1: a pair); the lane's byte is that of its quarter
    const uint32_t pick_pair = 0x0c0c0000u | (uint32_t)(4 + quarter) << 8 | (uint32_t)quarter;
    const uint32_t pick_first = 0x0c0c0c00u | (uint32_t)quarter;
    auto read_scale = [&](int buffer, int word, int row) __attribute__((always_inline)) {
        const uint8_t *at = smem + 2 * T::kStage + buffer * T::kScales + row * 16;
        if constexpr (T::kSteps == 2)
            return *reinterpret_cast<const uint2 *>(at + word * 4);
        else
            return *reinterpret_cast<const uint32_t *>(at + word * 4);
    };
    auto picked = [&](auto raw, uint32_t by) __attribute__((always_inline)) {
        if constexpr (T::kSteps == 2)
            return __builtin_amdgcn_perm(raw.y, raw.x, by);
        else
            return raw >> by;
    };

    v4f acc[2 * WI][NJ];
    // The two products of block i with weight fragment f: the weights are the row operand, so a lane's sums are four consecutive
    // outputs of a row.  (Of the two forms of the instruction this one does more under the chip's power limit, from
    // registers with random codes 6.5 against 6.0 PFLOP/s in E2M1 and 4.2 against 3.8 with E4M3: a sum is read and written
    // once for 128 elements, not for 64.)
    auto multiply = [&](auto block, auto frag, auto from_zero, const uint32_t (&scale_a)[2]) __attribute__((always_inline)) {
        constexpr int i = decltype(block)::value, f = decltype(frag)::value, t = f / NJ, j = f % NJ;
        constexpr bool zero = decltype(from_zero)::value && t == 0;
        const v8i b = v8i{(int)bf[f].x, (int)bf[f].y, (int)bf[f].z, (int)bf[f].w, 0, 0, 0, 0};
        static_for<2>([&](auto uc) {
            constexpr int u = decltype(uc)::value;
            const uint4 &lo = af[i & 1][u][kE4M3 ? 0 : t], &hi = af[i & 1][u][1];
            const v8i a = kE4M3 ? v8i{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, (int)hi.x, (int)hi.y, (int)hi.z, (int)hi.w}
                                : v8i{(int)lo.x, (int)lo.y, (int)lo.z, (int)lo.w, 0, 0, 0, 0};
            v4f &sum = acc[2 * i + u][j];
            sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, zero ? v4f{0, 0, 0, 0} : sum, kF4, kE4M3 ? kF8 : kF4, t,
                                                                   (int)sb[j], t, (int)scale_a[u]);
        });
    };

    // ---- the output of a finished tile
    int out_m = 0, out_n = 0;              // this wave's part of it
    uint8_t *const park = smem + 2 * T::kStage + 2 * T::kScales + wave * kParkBytes;
    const uint32_t y_lane = (uint32_t)(lane >> 3) * (uint32_t)ld_y * 2u + 16u * (lane & 7);
    quest_v4u out_reg[4];
    // Part n of kOutParts of storing block i; the block has WJ / 2 pieces of 64 columns, a piece four writes, one read, one store.
    constexpr int kOutParts = (WJ / 2) * 6;
    auto store_part = [&](auto block, auto part) __attribute__((always_inline)) {
        constexpr int i = decltype(block)::value, piece = decltype(part)::value / 6, n = decltype(part)::value % 6;
        // rows and columns that do not exist lie outside of the buffers
        const int rows = min(max(M - out_m - 32 * i, 0), 32);
        constexpr uint32_t kNowhere = 0x80000000u;
        if constexpr (OUT == kRawSums && n == 0 && piece == 0) {
            const auto buffer = __builtin_amdgcn_make_buffer_rsrc(acc_out + (int64_t)(out_m + 32 * i) * N + out_n, 0, rows * N * 4,
                                                                  0x00027000);
            static_for<2 * NJ>([&](auto tc) {
                constexpr int u = decltype(tc)::value / NJ, j = decltype(tc)::value % NJ;
                const int left = N - out_n - 16 * j - 4 * quarter, tail = left > 0 && left < 4 ? left : 0;
                const uint32_t at = ((uint32_t)(16 * u + l16) * (uint32_t)N + 16u * j + 4u * quarter) * 4u;
                const auto sum = __builtin_bit_cast(quest_v4u, acc[2 * i + u][j]);
                __builtin_amdgcn_raw_buffer_store_b128(sum, buffer, (int)(left >= 4 ? at : kNowhere), 0, 0);
                __builtin_amdgcn_raw_buffer_store_b64(v2u{sum[0], sum[1]}, buffer, (int)(tail & 2 ? at : kNowhere), 0, 0);
                __builtin_amdgcn_raw_buffer_store_b32(tail & 2 ? sum[2] : sum[0], buffer,
                                                      (int)(tail & 1 ? at + 4u * (tail & 2) : kNowhere), 0, 0);
            });
        }
        if constexpr (n < 4) {             // columns 16 n .. + 16 of the piece
            static_for<2>([&](auto uc) {
                constexpr int u = decltype(uc)::value;
                const v4f &sum = acc[2 * i + u][4 * piece + n];
                *reinterpret_cast<uint2 *>(park + (16 * u + l16) * 128 + (((2 * n + (quarter >> 1)) ^ (l16 & 7)) << 4) + 8 * (quarter & 1)) =
                    make_uint2(pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]));
            });
        } else if constexpr (n == 4) {
#pragma unroll
            for (int pass = 0; pass < 4; ++pass) {
                const int row = 8 * pass + (lane >> 3);
                out_reg[pass] = *reinterpret_cast<const quest_v4u *>(park + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
            }
        } else {
            // (any two-byte boundary will do for these stores; the buffer itself begins at a dword)
            const uint64_t place = reinterpret_cast<uint64_t>(y + (int64_t)(out_m + 32 * i) * ld_y + out_n + 64 * piece);
            const uint32_t odd = OUT == kWholePieces ? 0u : (uint32_t)place & 2u;
            const auto buffer = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(place - odd), 0,
                                                                  OUT == kWholePieces || y ? rows * (int)ld_y * 2 + (int)odd : 0, 0x00027000);
            const int left = N - out_n - 64 * piece - 8 * (lane & 7), tail = left > 0 && left < 8 ? left : 0;
            const uint32_t at = y_lane + odd;
#pragma unroll
            for (int pass = 0; pass < 4; ++pass) {
                const uint32_t down = (uint32_t)(8 * pass) * (uint32_t)ld_y * 2u;
                const quest_v4u &v = out_reg[pass];
                __builtin_amdgcn_raw_buffer_store_b128(v, buffer, (int)((left >= 8 || (OUT == kWholePieces && left > 0) ? at : kNowhere) + down), 0, 0);
                if constexpr (OUT != kWholePieces) {   // four, two and one of a row's last columns
                    __builtin_amdgcn_raw_buffer_store_b64(v2u{v[0], v[1]}, buffer, (int)((tail & 4 ? at : kNowhere) + down), 0, 0);
                    __builtin_amdgcn_raw_buffer_store_b32(tail & 4 ? v[2] : v[0], buffer,
                                                          (int)((tail & 2 ? at + 2u * (tail & 4) : kNowhere) + down), 0, 0);
                    const uint32_t last = tail & 4 ? (tail & 2 ? v[3] : v[2]) : tail & 2 ? v[1] : v[0];
                    __builtin_amdgcn_raw_buffer_store_b16((short)last, buffer,
                                                          (int)((tail & 1 ? at + 2u * (tail & 6) : kNowhere) + down), 0, 0);
                }
            }
        }
    };

    int cur = 0, scale_buffer = 0;         // where the stage being multiplied is
    int m0, n0, next_m0 = 0, next_n0 = 0;
    // One stage: number `at` of the tile; the stage behind it is fetched
    auto iteration = [&](auto kind, int at) __attribute__((always_inline)) {
        constexpr int k = decltype(kind)::value;
        constexpr bool last = (k & kStageLast) != 0, boundary = (k & kStageFirst) != 0;
        const uint8_t *stage = smem + cur * T::kStage;
        const uint32_t refill = smem_addr + (cur ^ 1) * T::kStage;
        if constexpr (last) {
            if (tile + peers < run_end)    // else the tile's first stage again, not used
                set_fetch_tile(tile + peers, next_m0, next_n0);
        }
        const int fetched = last ? 0 : at + 1;
        const bool fetched_half = !kE4M3 && half_stage && fetched == stages - 1;
        const bool new_scales = T::Stages::opens_chunk(fetched);
        if (new_scales)
            transfer_scales(scale_buffer ^ 1, fetched);
        // This stage's scales: read during phase 1, whose products need those of the stage before
        uint32_t sb_new[NJ];
        const uint32_t sa_before[2] = {sa[WI - 1][0], sa[WI - 1][1]};
        const int word = T::Stages::word(at);
        constexpr int kRowScales = 2 * WI + NJ, kPerSlot = (kRowScales + kFragB - 1) / kFragB, kBehind = 4 / kPerSlot;
        decltype(read_scale(0, 0, 0)) raw[kRowScales];
        // The second half of a half stage holds the first one's codes again: with scales of 2^-127 on both sides their products
        // (below 2^-240) leave the fp32 sums as they are.
        uint32_t pick = T::kSteps == 2 ? pick_pair : 8u * quarter;
        if constexpr (last && !kE4M3)
            pick = half_stage ? pick_first : pick;
        auto scale_slot = [&](auto slot) __attribute__((always_inline)) {
            static_for<kPerSlot>([&](auto more) {
                constexpr int now = decltype(slot)::value * kPerSlot + decltype(more)::value, then = now - kBehind * kPerSlot;
                if constexpr (now < kRowScales)
                    raw[now] = read_scale(scale_buffer, word, now < 2 * WI ? wr * 32 * WI + 16 * now + l16
                                                                           : T::kRows + wc * 32 * WJ + 16 * (now - 2 * WI) + l16);
                if constexpr (then >= 0 && then < kRowScales) {
                    if constexpr (then < 2 * WI)
                        sa[then / 2][then % 2] = picked(raw[then], pick);
                    else
                        sb_new[then - 2 * WI] = picked(raw[then], pick);
                }
            });
        };
        // transfers spread over phases 1 and 2, in E2M1, which has more of them, over 3 (4096 x 4096 x 16640: 143 -> 139 us);
        // where a tile before ends, all of them ahead of its stores
        constexpr int kDmaSlots = boundary ? 5 * kFragB / kOutParts + 1 : (kE4M3 || WI < 4 ? 2 : 3) * kFragB;
        constexpr int kStoresBehind = [] {   // the last of them, at least
            int count = 0;
            for (int number = boundary ? 0 : 2; number < (boundary ? 2 : last ? WI : 0); ++number)
                for (int piece = 0; piece < WJ / 2; ++piece)
                    if (number * kFragB + (6 * piece + 5) * kFragB / kOutParts >= (kDma - 1) * kDmaSlots / kDma)
                        count += 4;
            return count;
        }();
        auto phase = [&](auto blockc, auto numberc) __attribute__((always_inline)) {
            constexpr int block = decltype(blockc)::value, number = decltype(numberc)::value;   // number: 0 = phase 1
            constexpr bool before = number == 0;
            constexpr bool from_zero = before ? (k & kAfterFirst) != 0 : (k & kStageFirst) != 0;
            // the block whose output is stored meanwhile
            constexpr int storing = boundary && number == 0 ? WI - 2 : boundary && number == 1 ? WI - 1
                                    : last && number >= 2   ? block - 1
                                                            : -1;
            static_for<kFragB>([&](auto fc) {
                constexpr int f = decltype(fc)::value;
                multiply(blockc, fc, std::integral_constant<bool, from_zero>{}, before ? sa_before : sa[block]);
                if constexpr (before)
                    read_b(stage, fc);
                if constexpr (before)
                    scale_slot(fc);
                // the next block's activations: four reads, as early as their registers are free
                constexpr int next = before ? 0 : block + 1;
                static_for<4>([&](auto c) {
                    if constexpr (decltype(c)::value / 2 == f)
                        read_a(stage, std::integral_constant<int, next>{}, c);
                });
                if constexpr (number * kFragB + f < kDmaSlots)
                    static_for<kDma>([&](auto p) {
                        if constexpr (decltype(p)::value * kDmaSlots / kDma == number * kFragB + f)
                            transfer(p, refill, fetched, fetched_half);
                    });
                if constexpr (storing >= 0)
                    static_for<kOutParts>([&](auto n) {
                        if constexpr (decltype(n)::value * kFragB / kOutParts == f)
                            store_part(std::integral_constant<int, storing>{}, n);
                    });
                __builtin_amdgcn_sched_barrier(0);
            });
            if constexpr (before) {
                static_for<kBehind>([&](auto more) { scale_slot(std::integral_constant<int, kFragB + decltype(more)::value>{}); });
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    sb[j] = sb_new[j];
            }
        };
        phase(std::integral_constant<int, WI - 1>{}, std::integral_constant<int, 0>{});
        static_for<WI - 1>([&](auto i) { phase(i, std::integral_constant<int, decltype(i)::value + 1>{}); });
        // The reads of block WI - 1 are back, the next stage has landed.  Stores, which were issued behind its transfers, may be on
        // their way until the stage behind it has landed.
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
        wait_vmcnt<kStoresBehind>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");        // no read of the new stage ahead of it
        cur ^= 1;
        scale_buffer ^= new_scales ? 1 : 0;
    };
    auto wave_part = [&]() {
        out_m = m0 + wr * 32 * WI;
        out_n = n0 + wc * 32 * WJ;
    };

    set_fetch_tile(tile, m0, n0);
    next_m0 = m0;
    next_n0 = n0;
    transfer_scales(0, 0);
    static_for<kDma>([&](auto p) { transfer(p, smem_addr, 0, false); });
    wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    // before the first tile: products of zeros, stored nowhere
    out_m = M;
    static_for<kFragB>([&](auto f) { bf[decltype(f)::value] = make_uint4(0, 0, 0, 0); });
    static_for<4>([&](auto c) {
        constexpr int u = decltype(c)::value & 1, h = decltype(c)::value >> 1;
        af[0][u][h] = af[1][u][h] = make_uint4(0, 0, 0, 0);
    });
    static_for<WI>([&](auto i) { sa[decltype(i)::value][0] = sa[decltype(i)::value][1] = 0; });
    static_for<NJ>([&](auto j) { sb[decltype(j)::value] = 0; });
    static_for<2 * WI>([&](auto i) { static_for<NJ>([&](auto j) { acc[decltype(i)::value][decltype(j)::value] = v4f{0, 0, 0, 0}; }); });
    for (; tile < run_end; tile += peers) {
        iteration(std::integral_constant<int, kStageFirst>{}, 0);
        m0 = next_m0;
        n0 = next_n0;
        wave_part();
        if constexpr (TWO) {
            iteration(std::integral_constant<int, kAfterFirst | kStageLast>{}, 1);
        } else {
            iteration(std::integral_constant<int, kAfterFirst>{}, 1);
            for (int at = 2; at < stages - 1; ++at)
                iteration(std::integral_constant<int, 0>{}, at);
            iteration(std::integral_constant<int, kStageLast>{}, stages - 1);
        }
    }
    // the last block of the last tile
    static_for<kFragB>([&](auto fc) { multiply(std::integral_constant<int, WI - 1>{}, fc, std::false_type{}, sa[WI - 1]); });
    static_for<2>([&](auto b) {
        static_for<kOutParts>([&](auto n) { store_part(std::integral_constant<int, WI - 2 + decltype(b)::value>{}, n); });
    });
}

template <int FORMAT, int WI, int WJ>
hipError_t launch_tiles(const MxGemmArgs &a, hipStream_t stream)
{
    typedef MxTile<FORMAT, WI, WJ> T;
    const int tiles_m = (int)((a.M + T::kRows - 1) / T::kRows), tiles_n = (int)((a.N + T::kCols - 1) / T::kCols);
    const int per_xcd = (int)(((int64_t)tiles_m * tiles_n + 7) / 8), peers = std::min(per_xcd, device_compute_units() / 8);
    const bool whole = (a.ld_y & 7) == 0 && (a.N & 7) == 0 && (reinterpret_cast<uintptr_t>(a.y) & 15) == 0;
    auto kernel = a.acc_out ? mx_tile_kernel<FORMAT, WI, WJ, false, kRawSums>
                  : whole   ? mx_tile_kernel<FORMAT, WI, WJ, false, kWholePieces>
                            : mx_tile_kernel<FORMAT, WI, WJ, false, kAnyRows>;
    if constexpr (!T::kE4M3) {   // (in E4M3 the shortest contraction has three)
        if (T::Stages::count((int)a.K) == 2)
            kernel = a.acc_out ? mx_tile_kernel<FORMAT, WI, WJ, true, kRawSums>
                     : whole   ? mx_tile_kernel<FORMAT, WI, WJ, true, kWholePieces>
                               : mx_tile_kernel<FORMAT, WI, WJ, true, kAnyRows>;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)(8 * peers)), dim3(kTileThreads), T::kLds, stream, a.a_codes, a.a_scales, a.b_codes,
                       a.b_scales, (int)a.M, (int)a.N, (int)a.K, tiles_m, tiles_n, static_cast<uint16_t *>(a.y), a.ld_y, a.acc_out);
    return hipGetLastError();
}

template <int FORMAT, int WI, int WJ>
hipError_t prepare_tiles()
{
    constexpr int kLds = MxTile<FORMAT, WI, WJ>::kLds;
    hipError_t err = hipSuccess;
    auto allow = [&](auto kernel) {
        if (err == hipSuccess)
            err = allow_dynamic_lds(reinterpret_cast<const void *>(kernel), kLds);
    };
    allow(mx_tile_kernel<FORMAT, WI, WJ, false, kWholePieces>);
    allow(mx_tile_kernel<FORMAT, WI, WJ, false, kAnyRows>);
    allow(mx_tile_kernel<FORMAT, WI, WJ, false, kRawSums>);
    if constexpr (!MxTile<FORMAT, WI, WJ>::kE4M3) {
        allow(mx_tile_kernel<FORMAT, WI, WJ, true, kWholePieces>);
        allow(mx_tile_kernel<FORMAT, WI, WJ, true, kAnyRows>);
        allow(mx_tile_kernel<FORMAT, WI, WJ, true, kRawSums>);
    }
    return err;
}

// a.M, a.N of any size, a.K >= 384, which are two stages or more, rows of y less than 2^24 elements
// apart; tiles of `block` x `block`: 256 or 128
template <int FORMAT>
hipError_t launch_mx_tiles(const MxGemmArgs &a, int block, hipStream_t stream)
{
    return block == 256 ? launch_tiles<FORMAT, 4, 4>(a, stream) : launch_tiles<FORMAT, 2, 2>(a, stream);
}

template <int FORMAT>
hipError_t prepare_mx_tiles()
{
    const hipError_t err = prepare_tiles<FORMAT, 4, 4>();
    return err != hipSuccess ? err : prepare_tiles<FORMAT, 2, 2>();
}

}  // namespace
}  // namespace quest
