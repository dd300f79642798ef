// Of the gated linear recurrence, forwards and backwards: its gates, and how runs of positions are joined.
//
// A position takes the state h to a h + u, and a run of positions, one after the other, to A h + H, so that runs join as positions do:
// (A, H) then (A', H') is (A A', A' H + H').  A lane goes through P positions side by side, the LANES lanes of a block of channels are joined within
// their row of 16 by DPP, the waves of a workgroup through LDS.  All a are at most 1, so that no product leaves fp32's range upwards.
#pragma once

#include "seq_internal.h"

namespace convmi {
namespace {

constexpr int kRecWaves = 16;  // of a workgroup, at most

// A channel's A and biases as the gates take them.
template <int V>
struct RecParams {
    float A[V], f[V], i[V];
    __device__ __forceinline__ RecParams(const SeqRecArgs &a, int cb)
    {
#pragma unroll
        for (int k = 0; k < V; ++k) f[k] = i[k] = 0;
        seq_vector<V>(a.A, cb, A);
        if (a.f_bias) seq_vector<V>(a.f_bias, cb, f);
        if (a.i_bias) seq_vector<V>(a.i_bias, cb, i);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            A[k] = seq_decay(A[k] > 0 ? 0.0f : A[k]);
            f[k] *= -kLog2e;
            i[k] *= -kLog2e;
        }
    }
};

// 1 / (1 + exp(-(x + bias))); `bias` comes times -log2(e).
static __device__ __forceinline__ float rec_gate(float x, float bias) { return __builtin_amdgcn_rcpf(1.0f + seq_exp2(fmaf(-kLog2e, x, bias))); }

// 1 - a^2 for a = 2^t, t <= 0.  Near zero, where the difference would lose what a has rounded away, -t times a polynomial of t through the values at
// Chebyshev's points of (-0.36, 0): 1e-7 off at most; beyond, a^2 is at most 0.61.
static __device__ __forceinline__ float rec_rest(float t, float a)
{
    float p = -0.0347420424f;
    p = fmaf(p, t, -0.151484966f);
    p = fmaf(p, t, -0.443728805f);
    p = fmaf(p, t, -0.960892439f);
    p = fmaf(p, t, -1.38629425f);
    return t > -0.36f ? t * p : fmaf(-a, a, 1.0f);
}

// x of the lane D places before (BACK: behind) in a row of 16, `none` where that lies outside.
template <int D, bool BACK>
static __device__ __forceinline__ float rec_near(float none, float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(x), (BACK ? 0x100 : 0x110) + D, 0xf, 0xf, false));
}
// The same with zeros outside.
template <int D, bool BACK>
static __device__ __forceinline__ float rec_near0(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), (BACK ? 0x100 : 0x110) + D, 0xf, 0xf, true));
}

// Joins each lane's run with those of all lanes before (BACK: behind) it among LANES, `at` its place there.
template <int LANES, int D, bool BACK>
static __device__ __forceinline__ void rec_join(float &A, float &H, int at)
{
    if constexpr (D < LANES) {
        float a = rec_near<D, BACK>(1.0f, A), h = rec_near0<D, BACK>(H);
        if (LANES < 16 && (BACK ? at + D >= LANES : at < D)) a = 1, h = 0;
        H = fmaf(A, h, H);
        A *= a;
        rec_join<LANES, 2 * D, BACK>(A, H, at);
    }
}

}  // namespace
}  // namespace convmi
