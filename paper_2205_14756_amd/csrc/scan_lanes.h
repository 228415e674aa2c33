// Lanes that share a channel of the selective scan: 8 or 16 neighbours of a wave (4 of a step for single tokens), each with some of its states.
#pragma once
#include "msla_device.h"

namespace msla {
namespace {

template <int CTRL>
__device__ __forceinline__ float moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// the value of lane ^ 1, ^ 2, ^ 8
__device__ __forceinline__ float across1(float v) { return moved<0xB1>(v); }
__device__ __forceinline__ float across2(float v) { return moved<0x4E>(v); }
__device__ __forceinline__ float across8(float v) { return moved<0x128>(v); }

// The sum of p[j] over the L lanes that share a channel, to lane j of them: each step leaves half of the numbers, of twice as many lanes.
template <int L>
__device__ __forceinline__ float deal(const float (&p)[L], int lane);

template <>
__device__ __forceinline__ float deal<4>(const float (&p)[4], int lane) {
    const bool b2 = lane & 2, b1 = lane & 1;
    const float r0 = (b2 ? p[2] : p[0]) + across2(b2 ? p[0] : p[2]), r1 = (b2 ? p[3] : p[1]) + across2(b2 ? p[1] : p[3]);
    return (b1 ? r1 : r0) + across1(b1 ? r0 : r1);
}

// r[i]: in lanes without the 4 q[i], in the others q[i + 4], each with that of lane ^ 4.  Written out, here and below, as the compiler selects first and
// adds then, three instructions for these two.  (A data-parallel move reads a register two wait states after it was written, at the earliest.)
template <>
__device__ __forceinline__ float deal<8>(const float (&q)[8], int lane) {
    float r[4];
    asm("s_nop 1\n"
        "v_add_f32_dpp %0, %4, %4 row_shl:4 row_mask:0xf bank_mask:0x5\n"
        "v_add_f32_dpp %1, %5, %5 row_shl:4 row_mask:0xf bank_mask:0x5\n"
        "v_add_f32_dpp %2, %6, %6 row_shl:4 row_mask:0xf bank_mask:0x5\n"
        "v_add_f32_dpp %3, %7, %7 row_shl:4 row_mask:0xf bank_mask:0x5\n"
        "v_add_f32_dpp %0, %8, %8 row_shr:4 row_mask:0xf bank_mask:0xa\n"
        "v_add_f32_dpp %1, %9, %9 row_shr:4 row_mask:0xf bank_mask:0xa\n"
        "v_add_f32_dpp %2, %10, %10 row_shr:4 row_mask:0xf bank_mask:0xa\n"
        "v_add_f32_dpp %3, %11, %11 row_shr:4 row_mask:0xf bank_mask:0xa\n"
        "s_nop 1"
        : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
        : "v"(q[0]), "v"(q[1]), "v"(q[2]), "v"(q[3]), "v"(q[4]), "v"(q[5]), "v"(q[6]), "v"(q[7]));
    return deal<4>(r, lane);
}

template <>
__device__ __forceinline__ float deal<16>(const float (&p)[16], int lane) {
    float q[8];
    asm("s_nop 1\n"
        "v_add_f32_dpp %0, %8, %8 row_ror:8 row_mask:0xf bank_mask:0xf\n"
        "v_add_f32_dpp %1, %9, %9 row_ror:8 row_mask:0xf bank_mask:0xf\n"
        "v_add_f32_dpp %2, %10, %10 row_ror:8 row_mask:0xf bank_mask:0xf\n"
        "v_add_f32_dpp %3, %11, %11 row_ror:8 row_mask:0xf bank_mask:0xf\n"
        "v_add_f32_dpp %4, %12, %12 row_ror:8 row_mask:0xf bank_mask:0xf\n"
        "v_add_f32_dpp %5, %13, %13 row_ror:8 row_mask:0xf bank_mask:0xf\n"
        "v_add_f32_dpp %6, %14, %14 row_ror:8 row_mask:0xf bank_mask:0xf\n"
        "v_add_f32_dpp %7, %15, %15 row_ror:8 row_mask:0xf bank_mask:0xf\n"
        "v_add_f32_dpp %0, %16, %16 row_ror:8 row_mask:0xf bank_mask:0xc\n"
        "v_add_f32_dpp %1, %17, %17 row_ror:8 row_mask:0xf bank_mask:0xc\n"
        "v_add_f32_dpp %2, %18, %18 row_ror:8 row_mask:0xf bank_mask:0xc\n"
        "v_add_f32_dpp %3, %19, %19 row_ror:8 row_mask:0xf bank_mask:0xc\n"
        "v_add_f32_dpp %4, %20, %20 row_ror:8 row_mask:0xf bank_mask:0xc\n"
        "v_add_f32_dpp %5, %21, %21 row_ror:8 row_mask:0xf bank_mask:0xc\n"
        "v_add_f32_dpp %6, %22, %22 row_ror:8 row_mask:0xf bank_mask:0xc\n"
        "v_add_f32_dpp %7, %23, %23 row_ror:8 row_mask:0xf bank_mask:0xc"
        : "=&v"(q[0]), "=&v"(q[1]), "=&v"(q[2]), "=&v"(q[3]), "=&v"(q[4]), "=&v"(q[5]), "=&v"(q[6]), "=&v"(q[7])
        : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "v"(p[4]), "v"(p[5]), "v"(p[6]), "v"(p[7]), "v"(p[8]), "v"(p[9]), "v"(p[10]), "v"(p[11]),
          "v"(p[12]), "v"(p[13]), "v"(p[14]), "v"(p[15]));
    return deal<8>(q, lane);
}

// the sum of v over four neighbours, to all of them
__device__ __forceinline__ float sum_of_four(float v) {
    v += across1(v);
    v += across2(v);
    return v;
}

// lanes below 32 get a's sum over lane ^ 32, the others b's
__device__ __forceinline__ float halve32(float a, float b) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned first = r[0], second = r[1];        // (bit_cast of a vector's element itself reads element 0)
    return __builtin_bit_cast(float, first) + __builtin_bit_cast(float, second);
}
// even rows of 16 lanes get a's sum over lane ^ 16, odd ones b's
__device__ __forceinline__ float halve16(float a, float b) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned first = r[0], second = r[1];
    return __builtin_bit_cast(float, first) + __builtin_bit_cast(float, second);
}
// lanes without the 8 get a's sum over lane ^ 8, the others b's
__device__ __forceinline__ float halve8(float a, float b, int lane) {
    const bool mine_b = lane & 8;
    return (mine_b ? b : a) + across8(mine_b ? a : b);
}

}  // namespace
}  // namespace msla
