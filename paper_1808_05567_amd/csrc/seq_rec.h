// Of the gated linear recurrence, forwards and backwards: its gates, and how runs of positions are joined.
//
// A position takes the state h to a h + u, and a run of positions, one after the other, to A h + H, so that runs join as positions do:
// (A, H) then (A', H') is (A A', A' H + H').  A lane goes through P positions side by side of four channels, the lanes of a wave that have the same channels are
// joined by moves between lanes, the waves of a workgroup through LDS.  All a are at most 1, so that no product leaves fp32's range upwards.
#pragma once

#include "seq_internal.h"

namespace convmi {
namespace {

constexpr int kRecE = 4;  // channels of a lane

// Which channels and positions a lane has.  Where a block's positions follow one another a wave has one block, else 128 bytes of channels side by side, so that
// a wave's accesses are whole lines in both.
template <typename T, bool ROWS>
struct RecLanes {
    static constexpr int V = SeqElem<T>::V;
    static constexpr int UNITS = ROWS ? 2 * V : V / kRecE;  // fours of channels of a wave
    static constexpr int LANES = 64 / UNITS;             // that have the same ones
    static constexpr int COLS = UNITS * kRecE;
    static __device__ __forceinline__ int unit(int lane) { return ROWS ? lane % UNITS : lane / LANES; }
    static __device__ __forceinline__ int at(int lane) { return ROWS ? lane / UNITS : lane % LANES; }
    static constexpr int STEP = ROWS ? UNITS : 1;  // from one to the next
};

// Four channels.
static __device__ __forceinline__ void rec_unpack(const seq_f32x4 &b, float (&f)[kRecE])
{
#pragma unroll
    for (int k = 0; k < kRecE; ++k) f[k] = b[k];
}
static __device__ __forceinline__ void rec_unpack(const seq_u32x2 &b, float (&f)[kRecE])
{
#pragma unroll
    for (int k = 0; k < kRecE; k += 2) {
        f[k] = __uint_as_float(b[k / 2] << 16);
        f[k + 1] = __uint_as_float(b[k / 2] & 0xFFFF0000u);
    }
}
template <typename T>
struct RecFour;
template <>
struct RecFour<float> {
    typedef seq_f32x4 type;
    static __device__ __forceinline__ type pack(const float (&f)[kRecE]) { return type{f[0], f[1], f[2], f[3]}; }
};
template <>
struct RecFour<unsigned short> {
    typedef seq_u32x2 type;
    static __device__ __forceinline__ type pack(const float (&f)[kRecE]) { return type{seq_pack_bf16(f[0], f[1]), seq_pack_bf16(f[2], f[3])}; }
};

// A tensor as a wave takes it: where its first block and a sequence begin, the same for all lanes, and the bytes from there to a lane's channels and
// first position, which 32 bits hold (a plan's views see to that).
template <typename T>
struct RecTensor {
    typedef typename RecFour<T>::type Four;
    char *base;
    long long pitch;  // bytes from position to position
    unsigned lane;
    template <typename L, int P>
    static __device__ __forceinline__ RecTensor of(const void *p, const SeqView &v, int n, int c0, int c, int at)
    {
        const int b0 = c0 / L::V;
        RecTensor t;
        t.base = static_cast<char *>(const_cast<void *>(p)) + (n * v.n + b0 * v.c) * (long long)sizeof(T);
        t.pitch = v.l * (long long)sizeof(T);
        t.lane = ((unsigned)(c / L::V - b0) * (unsigned)v.c + (unsigned)(at * P) * (unsigned)v.l + (unsigned)(c % L::V)) * (unsigned)sizeof(T);
        return t;
    }
    // l: position of the wave's first lane, the same for all lanes.  (An address in scalar registers and a lane's distance are one instruction; the compiler,
    // left alone, adds the distance to `base` once and to that, in vector registers, the rest.)
    template <typename B>
    __device__ __forceinline__ __attribute__((address_space(1))) B *at(int l, unsigned distance) const
    {
        auto *p = (__attribute__((address_space(1))) char *)(base + l * pitch);
        asm("" : "+s"(p), "+v"(distance));
        return (__attribute__((address_space(1))) B *)(p + distance);
    }
    __device__ __forceinline__ Four load(int l) const { return *at<Four>(l, lane); }
    template <bool PAST, typename B>
    __device__ __forceinline__ void store(int l, unsigned distance, const B &b) const
    {
        if constexpr (PAST)
            __builtin_nontemporal_store(b, at<B>(l, distance));
        else
            *at<B>(l, distance) = b;
    }
};

// A wave's results on their way out.  Where the wave has one block, a lane's P positions are 16 P bytes, of which it may have 8, and stores of them would touch
// every line 2 P times (forwards, 8 x 2048 x 2048 bf16: 97 us where whole lines take 78); they go through LDS, in 16 bytes a position, and out by 64 positions an
// instruction.  Position P at + j lies at LANES j + at.
template <typename T, bool ROWS, int P, bool PAST>
struct RecOut {
    typedef RecLanes<T, ROWS> L;
    typedef typename RecFour<T>::type Four;
    static constexpr int SLOTS = ROWS ? 1 : L::LANES * P;
    seq_u32x4 *lds;  // of the wave
    RecTensor<T> to;
    __device__ __forceinline__ void put(int w0, int j, bool ok, int lane, const Four &b) const
    {
        if constexpr (ROWS) {
            if (ok) to.template store<PAST>(w0 + j, to.lane, b);
        } else
            *reinterpret_cast<Four *>(reinterpret_cast<T *>(lds + L::LANES * j + L::at(lane)) + L::unit(lane) * kRecE) = b;
    }
    // ends: behind the last position that there is
    __device__ __forceinline__ void out(int w0, int ends, int lane) const
    {
        if constexpr (!ROWS) blocks(w0, ends, lane, [&](int q) { return lds[L::LANES * (lane % P) + (64 * q + lane) / P]; });
    }
    // zeros at all positions
    __device__ __forceinline__ void clear(int w0, int ends, bool live, int lane) const
    {
        if constexpr (ROWS) {
#pragma unroll
            for (int j = 0; j < P; ++j)
                if (live && w0 + L::at(lane) * P + j < ends) to.template store<PAST>(w0 + j, to.lane, Four{});
        } else
            blocks(w0, ends, lane, [](int) { return seq_u32x4{}; });
    }
    template <typename F>
    __device__ __forceinline__ void blocks(int w0, int ends, int lane, F &&block) const
    {
#pragma unroll
        for (int q = 0; q < SLOTS / 64; ++q)
            if (w0 + 64 * q + lane < ends) to.template store<PAST>(w0 + 64 * q, (unsigned)lane * (unsigned)to.pitch, block(q));
    }
};

// A lane's A and biases as the gates take them; c: its first channel.
struct RecParams {
    float A[kRecE], f[kRecE], i[kRecE];
    __device__ __forceinline__ RecParams(const SeqRecArgs &a, int c)
    {
#pragma unroll
        for (int k = 0; k < kRecE; ++k) f[k] = i[k] = 0;
        seq_vector<kRecE>(a.A + c, 0, A);
        if (a.f_bias) seq_vector<kRecE>(a.f_bias + c, 0, f);
        if (a.i_bias) seq_vector<kRecE>(a.i_bias + c, 0, i);
#pragma unroll
        for (int k = 0; k < kRecE; ++k) {
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

// x of the lane that CTRL names, `none` where there is none.
template <int CTRL>
static __device__ __forceinline__ float rec_dpp(float none, float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(x), CTRL, 0xf, 0xf, false));
}
static __device__ __forceinline__ float rec_lane(float x, int lane) { return __int_as_float(__builtin_amdgcn_ds_bpermute(lane * 4, __float_as_int(x))); }

// (A, H) after what `a, h` bring: of positions before it (BACK: behind).
static __device__ __forceinline__ void rec_after(float &A, float &H, float a, float h)
{
    H = fmaf(A, h, H);
    A *= a;
}

// Joins each lane's four runs with those of the lane that `how` names.  A lane that has none, or whose row `how` leaves out, keeps its own: the instruction does not
// write there.  (As moves, with 1 and 0 where there is no lane, a product and a sum: 5 instructions a channel for these 2.)  What a move between lanes reads has to be
// written two instructions before: four channels in turn are that far apart, and the first and the last wait.
#define REC_STEP(how)                                  \
    "v_fmac_f32_dpp %4, %4, %0 " how " bank_mask:0xf\n" \
    "v_fmac_f32_dpp %5, %5, %1 " how " bank_mask:0xf\n" \
    "v_fmac_f32_dpp %6, %6, %2 " how " bank_mask:0xf\n" \
    "v_fmac_f32_dpp %7, %7, %3 " how " bank_mask:0xf\n" \
    "v_mul_f32_dpp %0, %0, %0 " how " bank_mask:0xf\n"  \
    "v_mul_f32_dpp %1, %1, %1 " how " bank_mask:0xf\n"  \
    "v_mul_f32_dpp %2, %2, %2 " how " bank_mask:0xf\n"  \
    "v_mul_f32_dpp %3, %3, %3 " how " bank_mask:0xf\n"
#define REC_STEPS(A, H, text)            \
    asm volatile("s_nop 4\n" text "s_nop 1" \
                 : "+v"(A[0]), "+v"(A[1]), "+v"(A[2]), "+v"(A[3]), "+v"(H[0]), "+v"(H[1]), "+v"(H[2]), "+v"(H[3]))

// Joins each lane's runs with those of all lanes before (BACK: behind) it that have its channels.
template <typename T, bool ROWS, bool BACK>
static __device__ __forceinline__ void rec_join(float (&A)[kRecE], float (&H)[kRecE], int lane)
{
    typedef RecLanes<T, ROWS> L;
    const auto across = [&](int from, bool ok) {
#pragma unroll
        for (int k = 0; k < kRecE; ++k) {
            float a = rec_lane(A[k], from), h = rec_lane(H[k], from);
            if (!ok) a = 1, h = 0;
            rec_after(A[k], H[k], a, h);
        }
    };
    if constexpr (ROWS) {
#pragma unroll
        for (int d = 1; d < L::LANES; d *= 2) {
            const int from = BACK ? lane + d * L::STEP : lane - d * L::STEP;
            across(from & 63, from >= 0 && from < 64);
        }
    } else if constexpr (!BACK) {
        // within rows of 16, then the last lane of a row to the next row, then that of the lower half to the upper one
        if constexpr (L::LANES == 64)
            REC_STEPS(A, H, REC_STEP("row_shr:1 row_mask:0xf") REC_STEP("row_shr:2 row_mask:0xf") REC_STEP("row_shr:4 row_mask:0xf") REC_STEP("row_shr:8 row_mask:0xf")
                                REC_STEP("row_bcast:15 row_mask:0xa") REC_STEP("row_bcast:31 row_mask:0xc"));
        else
            REC_STEPS(A, H, REC_STEP("row_shr:1 row_mask:0xf") REC_STEP("row_shr:2 row_mask:0xf") REC_STEP("row_shr:4 row_mask:0xf") REC_STEP("row_shr:8 row_mask:0xf")
                                REC_STEP("row_bcast:15 row_mask:0xa"));
    } else {
        REC_STEPS(A, H, REC_STEP("row_shl:1 row_mask:0xf") REC_STEP("row_shl:2 row_mask:0xf") REC_STEP("row_shl:4 row_mask:0xf") REC_STEP("row_shl:8 row_mask:0xf"));
        across(((lane | 15) + 1) & 63, !(lane & 16));
        if constexpr (L::LANES == 64) across(32, !(lane & 32));
    }
}
// What all lanes before (BACK: behind) it make of x, from the joined runs: what the nearest of them, with the others, does.
template <typename T, bool ROWS, bool BACK>
static __device__ __forceinline__ float rec_until(float A, float H, float x, int lane)
{
    typedef RecLanes<T, ROWS> L;
    const float own = fmaf(A, x, H);
    float near;
    if constexpr (ROWS)
        near = rec_lane(own, (BACK ? lane + L::STEP : lane - L::STEP) & 63);
    else
        near = rec_dpp<BACK ? 0x130 : 0x138>(x, own);  // by a lane, over the whole wave
    if constexpr (L::LANES == 64) return near;
    return L::at(lane) == (BACK ? L::LANES - 1 : 0) ? x : near;
}

// x after n runs, `step` numbers apart, with their A and H: eight at a time, so that one trip to memory brings them.
static __device__ __forceinline__ float rec_through(const float *A, const float *H, long long step, int n, float x)
{
    constexpr int TOGETHER = 8;
    for (int r = 0; r < n; r += TOGETHER) {
        float a[TOGETHER], h[TOGETHER];
#pragma unroll
        for (int i = 0; i < TOGETHER; ++i) {
            const long long at = min(r + i, n - 1) * step;
            a[i] = A[at];
            h[i] = H[at];
        }
#pragma unroll
        for (int i = 0; i < TOGETHER; ++i)
            if (r + i < n) x = fmaf(a[i], x, h[i]);
    }
    return x;
}

}  // namespace
}  // namespace convmi
