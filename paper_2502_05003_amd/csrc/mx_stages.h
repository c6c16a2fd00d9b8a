// Where a stage of the tile kernel for microscaled operands (mx_tile.h) finds its scales.  A row has a dword of four scales for each
// 128 elements (a unit, what one matrix instruction takes); a transfer brings a chunk of four dwords of each row into LDS, which serves
// the stages of 512 elements.  Chunks begin at multiples of four dwords from the row's start, also where the row ends inside one (its
// last dwords are then the next row's, or nothing at the operand's end, and belong to no stage): so the two dwords of a stage of two
// units lie in one aligned pair, and that of half a stage is the first of its pair.
#pragma once

#include <hip/hip_runtime.h>

namespace quest {

// STEPS: units of a stage; K a multiple of 128
template <int STEPS>
struct MxStages {
    static_assert(STEPS == 1 || STEPS == 2, "");
    static constexpr int kUnit = 128, kStageK = kUnit * STEPS, kChunk = 4;

    static __host__ __device__ constexpr int count(int K) { return (K + kStageK - 1) / kStageK; }
    // whether the last stage holds one unit of two
    static __host__ __device__ constexpr bool ends_in_half(int K) { return K % kStageK != 0; }
    // whether stage `at` is the first that its chunk serves
    static __host__ __device__ constexpr bool opens_chunk(int at) { return (at * STEPS & (kChunk - 1)) == 0; }
    // the dword of the row with which the stage's chunk begins
    static __host__ __device__ constexpr int chunk(int at) { return at * STEPS & ~(kChunk - 1); }
    // the dword of the chunk with which the stage's begin
    static __host__ __device__ constexpr int word(int at) { return at * STEPS & (kChunk - 1); }
};

}  // namespace quest
