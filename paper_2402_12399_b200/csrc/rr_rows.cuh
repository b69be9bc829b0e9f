// Rows of the router's scores [T,E] spread over groups of lanes: a token is handled by a group of GS lanes (a
// power of two, 1..32), each keeping up to eight columns in registers.  Shared by the kernels that take the
// softmax of every row (load-balance losses).
#pragma once
#include "rr_common.cuh"

namespace rr {

template <int GS>
__device__ __forceinline__ float group_max(float v)
{
#pragma unroll
    for (int o = GS / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
template <int GS>
__device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = GS / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Which columns a lane keeps.  Vector layout (E a multiple of 4): float4 pieces, piece q of lane gl
// covers columns q*4*GS + 4*gl .. + 3, so one load instruction of a group reads 16*GS contiguous bytes.
// Scalar layout (any E): element c is column c*GS + gl.
template <int GS, bool VEC>
__device__ __forceinline__ int column_of(int c, int gl)
{
    return VEC ? (c >> 2) * (4 * GS) + 4 * gl + (c & 3) : c * GS + gl;
}

// Lane layout for E experts: with E a multiple of 4 a lane keeps up to eight columns as float4 pieces
// and the group is as small as that allows (few shuffle steps: the reductions over the group, not the
// loads, bound these kernels otherwise); any other E takes scalar columns over up to 32 lanes.
struct Layout {
    bool vec;
    int gs, cpl;
};
inline Layout layout_of(int E)
{
    int epad = 1;
    while (epad < E) epad <<= 1;
    if (E % 4 == 0) {
        const int cpl = epad < 8 ? 4 : 8;
        return {true, epad / cpl, cpl};
    }
    return {false, epad < 32 ? epad : 32, epad <= 32 ? 1 : epad / 32};
}

// executes `CALL<GS, CPL, VEC>(args...);` for the layout of E (CALL may start with an assignment or `return`)
#define RR_ROWS_DISPATCH(CALL, E, ...)                                             \
    do {                                                                           \
        const ::rr::Layout rows_layout_ = ::rr::layout_of(E);                      \
        const int rows_gs_ = rows_layout_.gs;                                      \
        if (rows_layout_.vec) {                                                    \
            if (rows_layout_.cpl == 4) { CALL<1, 4, true>(__VA_ARGS__); break; }   \
            if (rows_gs_ == 1) { CALL<1, 8, true>(__VA_ARGS__); break; }           \
            if (rows_gs_ == 2) { CALL<2, 8, true>(__VA_ARGS__); break; }           \
            if (rows_gs_ == 4) { CALL<4, 8, true>(__VA_ARGS__); break; }           \
            if (rows_gs_ == 8) { CALL<8, 8, true>(__VA_ARGS__); break; }           \
            if (rows_gs_ == 16) { CALL<16, 8, true>(__VA_ARGS__); break; }         \
            CALL<32, 8, true>(__VA_ARGS__);                                        \
            break;                                                                 \
        }                                                                          \
        if (rows_layout_.cpl == 2) { CALL<32, 2, false>(__VA_ARGS__); break; }     \
        if (rows_layout_.cpl == 4) { CALL<32, 4, false>(__VA_ARGS__); break; }     \
        if (rows_layout_.cpl == 8) { CALL<32, 8, false>(__VA_ARGS__); break; }     \
        if (rows_gs_ == 1) { CALL<1, 1, false>(__VA_ARGS__); break; }              \
        if (rows_gs_ == 2) { CALL<2, 1, false>(__VA_ARGS__); break; }              \
        if (rows_gs_ == 4) { CALL<4, 1, false>(__VA_ARGS__); break; }              \
        if (rows_gs_ == 8) { CALL<8, 1, false>(__VA_ARGS__); break; }              \
        if (rows_gs_ == 16) { CALL<16, 1, false>(__VA_ARGS__); break; }            \
        CALL<32, 1, false>(__VA_ARGS__);                                           \
    } while (0)

}  // namespace rr
