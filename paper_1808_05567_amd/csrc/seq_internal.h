// Shared by the translation units of the sequence operators (include/seq_mi355x.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "seq_mi355x.h"

namespace convmi {

typedef unsigned seq_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned seq_u32x2 __attribute__((ext_vector_type(2)));
typedef float seq_f32x2 __attribute__((ext_vector_type(2)));
typedef float seq_f32x4 __attribute__((ext_vector_type(4)));

// A sequence tensor: element (n, c, l) lies n * .n + (c / V) * .c + l * .l + c % V elements behind the base.
// 64-bit distances: a tensor may have more than 2^32 elements.
struct SeqView {
    long long n, c, l;
};

struct SeqConvArgs {
    const void *x, *dy, *state_in;
    void *y, *dx, *state_out;
    const float *w, *bias;
    const int *lengths, *slots;
    float *part;  // [parts][W + 1][Cp]: partial sums of dw and dbias
    float *dw, *dbias;
    SeqView vx, vy, vdy, vdx;
    int N, Cb, Cp, L, silu, n_slots;
    int past;                    // results go past the caches
    int cgroups, ranges, range;  // groups of 8 blocks; runs of positions and their length
};

struct SeqScanArgs {
    const void *x, *dt, *B, *C, *z, *dy;
    const float *A, *D, *dt_bias, *state_in;
    void *y, *dx, *ddt, *dB, *dC, *dz;
    float *state_out, *dA, *dD, *ddt_bias;
    const int *lengths, *slots;
    SeqView vx, vdt, vB, vC, vz, vy, vdy, vdx, vddt, vdB, vdC, vdz;
    int N, Ch, Cp, L, S, G, CG;  // Ch channels, CG of them a group
    int softplus, n_slots;
    int tiles;          // tiles of channels a group
    int chunks, chunk;  // runs of positions and their length, a multiple of 8
    float *hl;          // [N][chunks][S][Cp]: state at the end of a chunk from zeros, then at its start
    float *gl;          // the same for the gradient, back to front
    float *sd;          // [N][chunks][Cp]: sum of d over a chunk
    int notes;          // chunk / 8 - 1
    float *marks;       // [N][chunks][notes][S][Cp]: state from zeros at the start of a chunk's eights but the first
    float *md;          // [N][chunks][notes][Cp]: sum of d up to there
    float *vec;         // [N][chunks][2][Cp]: partial dD, ddt_bias
    float *bc;          // [N][L][G * btiles][2][S]: partial dB, dC
    int btiles;         // workgroups' shares of a group's channels in the backward kernel
};

// f and i: what goes into the gates of the old state and of the input.
struct SeqRecArgs {
    const void *x, *f, *i, *z, *dy;
    void *y, *dx, *df, *di, *dz;
    const float *A, *f_bias, *i_bias, *state_in;
    float *state_out, *dA, *df_bias, *di_bias;
    const int *lengths, *slots;
    SeqView vx, vf, vi, vz, vy, vdy, vdx, vdf, vdi, vdz;
    int N, Cb, Cp, L, n_slots;
    int past;                // results go past the caches
    int rows;                // a position's blocks follow one another
    int few;                 // workgroups: fewer than two a compute unit
    int waves;               // of a workgroup
    int runs, run;           // runs of positions that workgroups share a sequence in, and their length
    int rounds;              // backwards: times that a workgroup has all of its waves' positions
    float *totals;  // where there are several runs, forwards [N][runs][2][Cp]: 0 and the state before the first run, then what runs make of a state; backwards
                    // [N][runs][3][Cp]: what they make of a state, from the front and from the back
    float *marks;   // [N][runs][rounds][Cp]: what reaches the last position of each from behind it
    float *part;    // [N][runs][3][Cp]: sums of dA, df_bias and di_bias over a run
};

struct SeqNormArgs {
    const void *x, *res, *dy, *dr;
    const float *w;
    void *r, *y, *dx;
    int8_t *q;
    float *scale, *part, *dw;
    SeqView vx, vres, vr, vy, vq, vdy, vdr, vdx;
    int N, C, Cb, Cp, L;
    long long rows;  // N * L
    float eps;
    int parts;
    int past;  // results go past the caches
    // the layer norm's
    const float *b;
    float *db;
    const int *lengths;
};

constexpr int kSeqAdamwBlock = 256, kSeqAdamwTensors = 80;  // numbers with a scale of their own; tensors of a launch
constexpr int kSeqAdamwShare = 4096;                        // numbers of a workgroup

struct SeqAdamwTensor {
    float *p;
    const void *g;
    unsigned short *copy;
    int64_t size;
    unsigned block;  // of the states, where the tensor's begin
    float decay;
};
// A launch's tensors (4 KB hold the arguments of one).
struct SeqAdamwArgs {
    void *m, *v;
    float *scales;  // [2][blocks]
    const float *now;  // rate, step, factor; NULL: what follows
    float rate, by_m, by_v, factor;  // rate / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    double log1, log2;  // of the betas
    float beta1, rest1, beta2, rest2, eps;  // rest: 1 - beta
    unsigned blocks;
    int count;
    unsigned first[kSeqAdamwTensors];  // of a tensor's workgroups
    SeqAdamwTensor tensor[kSeqAdamwTensors];
};

struct SeqMv4Args {
    const void *x, *wt;
    const float *xscale, *scale, *bias;
    void *y;
    int M, C, K, Cx, Cs, Kp, Ky, group;  // Cs: runs of 128 channels
};

hipError_t launch_seq_conv_fwd(int dtype, int W, const SeqConvArgs &a, hipStream_t s);
hipError_t launch_seq_conv_step(int dtype, int W, const SeqConvArgs &a, hipStream_t s);
hipError_t launch_seq_conv_bwd(int dtype, int W, const SeqConvArgs &a, hipStream_t s);
hipError_t launch_seq_scan_fwd(int dtype, const SeqScanArgs &a, hipStream_t s);
hipError_t launch_seq_scan_step(int dtype, const SeqScanArgs &a, hipStream_t s);
hipError_t launch_seq_scan_ends(int dtype, const SeqScanArgs &a, hipStream_t s);
hipError_t launch_seq_scan_bwd(int dtype, const SeqScanArgs &a, hipStream_t s);
hipError_t launch_seq_rec_fwd(int dtype, const SeqRecArgs &a, hipStream_t s);
hipError_t launch_seq_rec_step(int dtype, const SeqRecArgs &a, hipStream_t s);
hipError_t launch_seq_rec_totals(int dtype, bool back, const SeqRecArgs &a, hipStream_t s);
hipError_t launch_seq_rec_bwd(int dtype, const SeqRecArgs &a, hipStream_t s);
hipError_t launch_seq_norm_fwd(int dtype, const SeqNormArgs &a, hipStream_t s);
hipError_t launch_seq_norm_bwd(int dtype, const SeqNormArgs &a, hipStream_t s);
hipError_t launch_seq_lnorm_fwd(int dtype, const SeqNormArgs &a, hipStream_t s);
hipError_t launch_seq_lnorm_bwd(int dtype, const SeqNormArgs &a, hipStream_t s);
hipError_t launch_seq_adamw(int dtype, int bits, const SeqAdamwArgs &a, unsigned workgroups, hipStream_t s);
hipError_t launch_seq_mv4(int dtype, const SeqMv4Args &a, hipStream_t s);
hipError_t launch_seq_mv4_quant(const SeqMv4Args &a, const float *w, void *wt, float *scale, hipStream_t s);
hipError_t launch_seq_mv4_unquant(const SeqMv4Args &a, float *w, hipStream_t s);

// States a scan kernel is built for; channels of a wave of the backward kernel, whose lanes take 2 channels x 4 states, and its waves,
// which take tiles side by side.
constexpr int seq_scan_states(int S) { return S <= 8 ? 8 : S <= 16 ? 16 : S <= 32 ? 32 : 64; }
constexpr int seq_scan_bwd_channels(int SP) { return 512 / SP; }
constexpr int kSeqBwdWaves = 4;

// The scan's launches, as they are made and as a plan's are counted.  Those over runs: waves of 64 channels, kSeqScanWaves a workgroup, more than
// 32 states by two waves where no sum over them is formed.  That which joins runs: workgroups of 64 columns, a wave per 16 runs, up to 16.
constexpr int kSeqScanWaves = 4, kSeqJoinWaves = 16;
inline int64_t seq_scan_waves(const SeqScanArgs &a, bool sums) { return (int64_t)a.N * a.G * a.tiles * a.chunks * (sums || a.S <= 32 ? 1 : 2); }
inline int64_t seq_join_groups(const SeqScanArgs &a) { return a.N * (((int64_t)a.S * a.Cp + 63) / 64); }
inline int seq_join_waves(int chunks) { return chunks <= 16 * kSeqJoinWaves ? (chunks + 15) / 16 : kSeqJoinWaves; }

// The recurrence's waves have one block of channels where a block's positions follow one another, and 128 bytes of them where a position's blocks do; the lanes
// that have the same four channels take some positions side by side each at a time.
inline int seq_rec_cols(bool rows, int vlen) { return rows ? 8 * vlen : vlen; }
inline int64_t seq_rec_groups(int64_t Cp, bool rows, int vlen) { return (Cp + seq_rec_cols(rows, vlen) - 1) / seq_rec_cols(rows, vlen); }
inline int seq_rec_lanes(bool rows, int vlen) { return 64 / (seq_rec_cols(rows, vlen) / 4); }
constexpr int seq_rec_positions(bool rows) { return rows ? 4 : 2; }
constexpr int kSeqRecBwdPositions = 2, kSeqRecWaves = 16, kSeqRecBwdWaves = 8, kSeqRecTotalsWaves = 8;  // of a lane; of a workgroup at most

// Results of more bytes than this go past the caches (the L2s hold 32 MB together).
constexpr long long kSeqPastBytes = 16LL << 20;

#ifdef __HIPCC__
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

static __device__ __forceinline__ unsigned seq_pack_bf16(float lo, float hi)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 p = {(__bf16)lo, (__bf16)hi};  // to nearest even
    return __builtin_bit_cast(unsigned, p);
}

// T: float, or unsigned short for bf16.  A block of V numbers is one 16-byte access.
template <typename T>
struct SeqElem;
template <>
struct SeqElem<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ float get(float x) { return x; }
    static __device__ __forceinline__ float put(float x) { return x; }
    static __device__ __forceinline__ void unpack(const seq_u32x4 &b, float (&f)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(b[i]);
    }
    static __device__ __forceinline__ seq_u32x4 pack(const float (&f)[4])
    {
        seq_u32x4 b;
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(f[i]);
        return b;
    }
};
template <>
struct SeqElem<unsigned short> {
    static constexpr int V = 8;
    static __device__ __forceinline__ float get(unsigned short x) { return __uint_as_float((unsigned)x << 16); }
    static __device__ __forceinline__ unsigned short put(float x) { return (unsigned short)seq_pack_bf16(x, x); }
    static __device__ __forceinline__ void unpack(const seq_u32x4 &b, float (&f)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(b[i] << 16);
            f[2 * i + 1] = __uint_as_float(b[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ seq_u32x4 pack(const float (&f)[8])
    {
        seq_u32x4 b;
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = seq_pack_bf16(f[2 * i], f[2 * i + 1]);
        return b;
    }
};

template <typename T>
static __device__ __forceinline__ seq_u32x4 seq_load(const T *p)
{
    return *reinterpret_cast<const seq_u32x4 *>(p);
}
template <typename T>
static __device__ __forceinline__ void seq_store(T *p, const seq_u32x4 &b)
{
    *reinterpret_cast<seq_u32x4 *>(p) = b;
}

// PAST: past the caches, for results that they would not hold until someone reads them, and that push out what is read again.
template <bool PAST, typename T>
static __device__ __forceinline__ void seq_store_result(T *p, const seq_u32x4 &b)
{
    if constexpr (PAST)
        __builtin_nontemporal_store(b, reinterpret_cast<seq_u32x4 *>(p));
    else
        seq_store(p, b);
}

// V floats of an fp32 vector from block b on.
template <int V>
static __device__ __forceinline__ void seq_vector(const float *p, int b, float (&f)[V])
{
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        const seq_f32x4 q = *reinterpret_cast<const seq_f32x4 *>(p + (long long)b * V + i);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[i + j] = q[j];
    }
}

static __device__ __forceinline__ int seq_length(const int *lengths, int n, int L)
{
    return lengths ? min(max(lengths[n], 0), L) : L;
}

static __device__ __forceinline__ float seq_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
// A state's A for the binary exponential.  Minus infinity goes as the lowest number: what fills up an eight of positions has steps of zero, which
// times infinity are no numbers.
static __device__ __forceinline__ float seq_decay(float A)
{
    const float a = A * kLog2e;
    return a == -INFINITY ? -3.40282347e38f : a;
}
// What a run makes of the state h before it: `own` from zeros, and h times 2^e.  Zero stays zero, whatever it would grow by.
static __device__ __forceinline__ float seq_carry(float e, float h, float own) { return h == 0 ? own : fmaf(seq_exp2(e), h, own); }
// 1 / (1 + exp(-x)); the hardware's exponential and reciprocal are good to an ulp
static __device__ __forceinline__ float seq_sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + seq_exp2(-kLog2e * x)); }

// log(1 + exp(x)) = max(x, 0) + log(1 + e), e = exp(-|x|) <= 1, and log(1 + e) = 2 atanh(t), t = e / (2 + e) <= 1/3.  atanh(t) / t is
// 1 + t^2 times a cubic in t^2, through its values at Chebyshev's points: 1.6e-8 off at most.  (The logarithm of 1 + e itself loses what e
// has below 2^-24: steps of 1e-3 would be good to 6e-5.  The series to the same error takes eight terms.)
static __device__ __forceinline__ float seq_softplus(float x, float *slope = nullptr)
{
    const float e = seq_exp2(-kLog2e * fabsf(x));
    if (slope) {  // its derivative, 1 / (1 + exp(-x))
        const float r = __builtin_amdgcn_rcpf(1.0f + e);
        *slope = x < 0 ? e * r : r;
    }
    const float t = e * __builtin_amdgcn_rcpf(2.0f + e), u = t * t;
    float p = 0.134337744f;
    p = fmaf(p, u, 0.141169779f);
    p = fmaf(p, u, 0.200038355f);
    p = fmaf(p, u, 0.333333197f);
    p = fmaf(p * u, t, t);
    return fmaf(2.0f, p, x != x ? x : fmaxf(x, 0.0f));
}

// Between writes and reads of LDS by lanes of one wave: its LDS operations are done in order, the compiler has to keep them so.
static __device__ __forceinline__ void seq_wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Sum of parts of one column in a fixed order: 32 strands of them, each in turn, then the strands pairwise.  1024 threads a
// workgroup, 32 columns: the result is in those of strand 0.  (512 parts of 2048 columns: 4 strands and one load at a time take 20 us.)
constexpr int kSumColumns = 32, kSumStrands = 32;
static __device__ __forceinline__ float seq_sum_parts(const float *p, long long pitch, int parts, bool ok)
{
    __shared__ float lds[kSumStrands][kSumColumns];
    const int col = threadIdx.x % kSumColumns, strand = threadIdx.x / kSumColumns;
    float s = 0;
    if (ok) {
        int k = strand;
        for (; k + 7 * kSumStrands < parts; k += 8 * kSumStrands) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = p[(k + i * kSumStrands) * pitch];
#pragma unroll
            for (int i = 0; i < 8; ++i) s += f[i];
        }
        for (; k < parts; k += kSumStrands) s += p[k * pitch];
    }
    lds[strand][col] = s;
    __syncthreads();
#pragma unroll
    for (int d = kSumStrands / 2; d > 0; d /= 2) {
        if (strand < d) lds[strand][col] += lds[strand + d][col];
        __syncthreads();
    }
    return lds[0][col];
}

// Lane i of every row of 16 lanes, in all lanes of that row.
template <int I>
static __device__ __forceinline__ float seq_row_lane(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x150 + I, 0xf, 0xf, true));
}
// x + x of the lane that `CTRL` names.
template <int CTRL>
static __device__ __forceinline__ float seq_add_lane(float x)
{
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
#endif

}  // namespace convmi
