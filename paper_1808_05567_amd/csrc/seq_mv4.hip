// Products of a few rows with weights of 4 bits and a scale for each group of channels:
//
//   y[m,k] = xscale[m] sum_groups scale[g][k] sum_{c in g} q[k,c] x[m,c] + bias[k]
//
// On the matrix instructions, weights as the rows: 16 weight rows x 16 tokens x 32 channels.  The inner sums are exact for
// 8-bit activations (integers) and sums of exact products in fp32 for bf16 ones: a whole number from -8 to 7 is exact in both types.
// fp32 activations go as three bf16 numbers whose sum they are.  Scales are applied to the fp32 sums.
//
// A lane's 16 bytes of weights are 8 channels of each of 4 runs of 32, so that one instruction takes one run of 32 whole and
// a group of 32, 64 or 128 channels is one, two or four of them, whatever its scale.
//
// Bound by the weights' bytes for few rows.  The kernel under the profiler, three sets of tensors in turn: 4096 x 8192 for one token in 8 bits 6.8 us
// (18 MB, 2.6 TB/s, of which a launch and a first trip to memory are some 4 us), in bf16 7.7, in fp32 12.6; for 32 tokens 8.1, 10.2 and 20.8; for 64
// 11.0, 15.0 and 39.  (A call among others takes as long or up to 0.7 us less.)
#include "seq_internal.h"

namespace convmi {
namespace {

constexpr int kMaxWaves = 8;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// Activations of one lane: 8 channels of one token.
template <int DT>
struct Act;
template <>
struct Act<SEQ_I8> {
    typedef int8_t T;
    typedef i32x4 Acc;
    typedef seq_u32x2 Raw;
    seq_u32x2 x;
    // eight channels, of which `left` there are
    static __device__ __forceinline__ Raw fetch(const int8_t *p, int left) { return left >= 8 ? *reinterpret_cast<const seq_u32x2 *>(p) : seq_u32x2{}; }
    __device__ __forceinline__ explicit Act(const Raw &r) : x(r) {}
    // eight weights from a word: sixteen times their values, in the upper halves of bytes (low ones of each byte first)
    struct Wt {
        long lo_hi;
    };
    static __device__ __forceinline__ Wt unpack(unsigned w)
    {
        const unsigned even = w << 4 & 0xF0F0F0F0u, odd = w & 0xF0F0F0F0u;
        // bytes 0 2 4 6 and 1 3 5 7 to 0 1 2 3 4 5 6 7
        const unsigned a = __builtin_amdgcn_perm(odd, even, 0x05010400), b = __builtin_amdgcn_perm(odd, even, 0x07030602);
        return {(long)((unsigned long)b << 32 | a)};
    }
    static constexpr float unit = 1.0f / 16;
    static __device__ __forceinline__ Acc mma(const Wt &w, const Act &a, const Acc &c)
    {
        return __builtin_amdgcn_mfma_i32_16x16x32_i8(w.lo_hi, (long)((unsigned long)a.x[1] << 32 | a.x[0]), c, 0, 0, 0);
    }
};
struct WtBf16 {
    seq_u32x4 b;
    // eight weights from a word as bf16 numbers
    static __device__ __forceinline__ WtBf16 of(unsigned w)
    {
        WtBf16 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int lo = (int)(w << (28 - 8 * i)) >> 28, hi = (int)(w << (24 - 8 * i)) >> 28;
            r.b[i] = seq_pack_bf16((float)lo, (float)hi);
        }
        return r;
    }
};
template <>
struct Act<SEQ_BF16> {
    typedef unsigned short T;
    typedef seq_f32x4 Acc;
    typedef seq_u32x4 Raw;
    seq_u32x4 x;
    static __device__ __forceinline__ Raw fetch(const unsigned short *p, int left) { return left >= 8 ? seq_load(p) : seq_u32x4{}; }
    __device__ __forceinline__ explicit Act(const Raw &r) : x(r) {}
    typedef WtBf16 Wt;
    static __device__ __forceinline__ Wt unpack(unsigned w) { return WtBf16::of(w); }
    static constexpr float unit = 1.0f;
    static __device__ __forceinline__ Acc mma(const Wt &w, const Act &a, const Acc &c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.b), __builtin_bit_cast(bf16x8, a.x), c, 0, 0, 0);
    }
};
template <>
struct Act<SEQ_F32> {
    typedef float T;
    typedef seq_f32x4 Acc;
    struct Raw {
        seq_f32x4 lo, hi;
    };
    seq_u32x4 h, m, l;
    static __device__ __forceinline__ Raw fetch(const float *p, int left)
    {
        return {left >= 4 ? *reinterpret_cast<const seq_f32x4 *>(p) : seq_f32x4{}, left >= 8 ? *reinterpret_cast<const seq_f32x4 *>(p + 4) : seq_f32x4{}};
    }
    __device__ __forceinline__ explicit Act(const Raw &r)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p0 = i < 2 ? r.lo[2 * i] : r.hi[2 * i - 4], p1 = i < 2 ? r.lo[2 * i + 1] : r.hi[2 * i - 3];
            h[i] = seq_pack_bf16(p0, p1);
            // (of infinities and numbers that round to them, from 3.39e38 on, nothing is left)
            float r0 = p0 - __uint_as_float(h[i] << 16), r1 = p1 - __uint_as_float(h[i] & 0xFFFF0000u);
            r0 = fabsf(r0) < INFINITY ? r0 : 0.0f;
            r1 = fabsf(r1) < INFINITY ? r1 : 0.0f;
            m[i] = seq_pack_bf16(r0, r1);
            l[i] = seq_pack_bf16(r0 - __uint_as_float(m[i] << 16), r1 - __uint_as_float(m[i] & 0xFFFF0000u));
        }
    }
    typedef WtBf16 Wt;
    static __device__ __forceinline__ Wt unpack(unsigned w) { return WtBf16::of(w); }
    static constexpr float unit = 1.0f;
    static __device__ __forceinline__ Acc mma(const Wt &w, const Act &a, Acc c)
    {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.b), __builtin_bit_cast(bf16x8, a.l), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.b), __builtin_bit_cast(bf16x8, a.m), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.b), __builtin_bit_cast(bf16x8, a.h), c, 0, 0, 0);
    }
};

// A workgroup: 16 * KT weight rows, 16 * NT tokens, all channels, the runs of 128 dealt to its waves in turn.  A wave has the loads of U runs on
// their way at a time: there are few, and each is a trip to memory.  The activations come from the caches, once for all KT tiles of weights.
//
// STAGE: several tokens.  Loaded as the instructions want them a token's 128 channels are four loads of a quarter (8 bits) or half of each of its
// cache lines, 16 tokens' lines at a time, and the caches take longer to look these up than to deliver them.  So a wave loads whole lines and
// turns them in an LDS area of its own.
template <int DT, int KT, int NT, int GROUP, int U, bool STAGE>
__global__ __launch_bounds__(64 * kMaxWaves) void seq_mv4_kernel(const SeqMv4Args a)
{
    typedef Act<DT> A;
    typedef typename A::T T;
    // (a token's rows, or channels, and 16 bytes more: sixteen tokens' blocks of 16 bytes go to different banks)
    constexpr int ROWS = 16 * KT, PITCH = ROWS + 4, LINE = 128 * sizeof(T) + 16, TOKEN = STAGE && LINE > PITCH * 4 ? LINE / 4 : PITCH, AREA = NT * 16 * TOKEN;
    constexpr int PIECES = 128 * sizeof(T) / 16, PART = 16 / sizeof(T), LOADS = NT * 16 * PIECES / 64;  // of 16 bytes a token; channels of one
    __shared__ __align__(16) float lds[kMaxWaves * AREA];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
    const int j = lane / 16, col = lane % 16;  // operands: row or token `col`, channels 8 j ... + 7 of a run of 32
    const int k0 = blockIdx.x * 16 * KT, m0 = blockIdx.y * 16 * NT;
    const seq_u32x4 *wt[KT];
    const float *scale[KT];  // results: rows 4 j ... + 3 of a tile, token `col`
#pragma unroll
    for (int q = 0; q < KT; ++q) {
        const int k = min(k0 + 16 * q, a.Kp - 16);  // (a tile past the last one is the last one, and is not stored)
        wt[q] = static_cast<const seq_u32x4 *>(a.wt) + (long long)(k + col) * 4 + j;
        scale[q] = a.scale + k + 4 * j;
    }
    const T *x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) x[t] = static_cast<const T *>(a.x) + (long long)min(m0 + t * 16 + col, a.M - 1) * a.Cx + 8 * j;
    // staged: load r is piece lane % PIECES of token (lane + 64 r) / PIECES
    const int piece = lane % PIECES * PART;
    char *const mine = reinterpret_cast<char *>(lds + wave * AREA), *const to = mine + lane / PIECES * LINE + lane % PIECES * 16;
    const char *const from = mine + col * LINE + 8 * j * sizeof(T);
    const T *xs[STAGE ? LOADS : 1];
    if (STAGE)
#pragma unroll
        for (int r = 0; r < LOADS; ++r) xs[r] = static_cast<const T *>(a.x) + (long long)min(m0 + (lane + 64 * r) / PIECES, a.M - 1) * a.Cx + piece;
    seq_f32x4 sum[KT][NT] = {};
    constexpr int per = GROUP / 32, groups = 4 / per;  // runs of 32 a group, groups a run of 128
    for (int first = wave; first < a.Cs; first += waves * U) {
        seq_u32x4 w[U][KT];
        seq_f32x4 sc[U][KT][groups];
        typename A::Raw raw[STAGE ? 1 : U][NT][4];
        seq_u32x4 whole[STAGE ? U : 1][STAGE ? LOADS : 1];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = first + u * waves;
            if (c >= a.Cs) break;
#pragma unroll
            for (int q = 0; q < KT; ++q) {
                w[u][q] = wt[q][(long long)c * a.Kp * 4];
#pragma unroll
                for (int i = 0; i < groups; ++i)
                    if (c * 128 + i * GROUP < a.C) sc[u][q][i] = *reinterpret_cast<const seq_f32x4 *>(scale[q] + (long long)(c * groups + i) * a.Kp);
            }
            // (x ends at Cx, the weights go on with zeros to the end of the run of 128)
            if constexpr (STAGE) {
#pragma unroll
                for (int r = 0; r < LOADS; ++r) {
                    whole[u][r] = seq_u32x4{};
                    if (c * 128 + piece < a.Cx) whole[u][r] = seq_load(xs[r] + c * 128);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int t = 0; t < NT; ++t) raw[u][t][i] = A::fetch(x[t] + c * 128 + i * 32, a.Cx - c * 128 - i * 32 - 8 * j);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = first + u * waves;
            if (c >= a.Cs) break;
            if constexpr (STAGE) {
                seq_wave_sync();
#pragma unroll
                for (int r = 0; r < LOADS; ++r) *reinterpret_cast<seq_u32x4 *>(to + r * (64 / PIECES) * LINE) = whole[u][r];
                seq_wave_sync();
            }
            typename A::Acc acc[KT][NT];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i % per == 0)
#pragma unroll
                    for (int q = 0; q < KT; ++q)
#pragma unroll
                        for (int t = 0; t < NT; ++t) acc[q][t] = typename A::Acc{};
                typename A::Wt wi[KT];
#pragma unroll
                for (int q = 0; q < KT; ++q) wi[q] = A::unpack(w[u][q][i]);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    if constexpr (STAGE) raw[0][t][i] = A::fetch(reinterpret_cast<const T *>(from + t * 16 * LINE) + 32 * i, 8);
                    const A act(raw[STAGE ? 0 : u][t][i]);
#pragma unroll
                    for (int q = 0; q < KT; ++q) acc[q][t] = A::mma(wi[q], act, acc[q][t]);
                }
                if (i % per == per - 1 && c * 128 + i / per * GROUP < a.C) {
#pragma unroll
                    for (int q = 0; q < KT; ++q)
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e) sum[q][t][e] = fmaf(sc[u][q][i / per][e], (float)acc[q][t][e], sum[q][t][e]);
                }
            }
        }
    }
    // [wave][token][row]: the waves' parts are added in order, one result a thread
    if (STAGE) seq_wave_sync();
#pragma unroll
    for (int q = 0; q < KT; ++q)
#pragma unroll
        for (int t = 0; t < NT; ++t)
            *reinterpret_cast<seq_f32x4 *>(&lds[wave * AREA + (t * 16 + col) * PITCH + q * 16 + 4 * j]) = sum[q][t];
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 16 * ROWS; i += blockDim.x) {
        float s = 0;
        for (int v = 0; v < waves; ++v) s += lds[v * AREA + i / ROWS * PITCH + i % ROWS];
        const int m = m0 + i / ROWS, k = k0 + i % ROWS;
        if (m >= a.M || k >= a.Ky) continue;
        s *= A::unit;
        if (a.xscale) s *= a.xscale[m];
        if (a.bias && k < a.K) s += a.bias[k];
        if (k >= a.K) s = 0;
        if constexpr (DT == SEQ_F32)
            static_cast<float *>(a.y)[(long long)m * a.Ky + k] = s;
        else
            static_cast<unsigned short *>(a.y)[(long long)m * a.Ky + k] = SeqElem<unsigned short>::put(s);
    }
}

// One thread a word of eight weights; the 16, 8 or 4 threads of one group's words stand side by side.
__global__ __launch_bounds__(256) void seq_mv4_quant_kernel(const SeqMv4Args a, const float *w, unsigned *wt, float *scale)
{
    const long long total = (long long)a.Cs * 16 * a.Kp;
    for (long long base = (long long)blockIdx.x * 256; base < total; base += (long long)gridDim.x * 256) {
        // (total is a multiple of 256: Kp is one of 16)
        const long long t = base + threadIdx.x;
        const int u = (int)(t % 16), k = (int)(t / 16 % a.Kp), cs = (int)(t / 16 / a.Kp);
        const int c0 = cs * 128 + u * 8;  // word i = u / 4 of the bytes j = u % 4
        float f[8];
        unsigned m = 0;  // (as unsigned numbers NaN is the largest)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            f[e] = k < a.K && c0 + e < a.C ? w[(long long)k * a.C + c0 + e] : 0.0f;
            m = max(m, __float_as_uint(fabsf(f[e])));
        }
        for (int d = 1; d < a.group / 8; d *= 2) m = max(m, (unsigned)__shfl_xor((int)m, d));
        // (no scale holds a group with an infinity: its products are no numbers, rather than wrong ones)
        const float s = m < 0x7F800000u ? __uint_as_float(m) / 7.0f : __builtin_nanf("");
        unsigned word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) word |= ((unsigned)(int)rintf(fminf(fmaxf(s > 0 ? f[e] / s : 0.0f, -8.0f), 7.0f)) & 15u) << 4 * e;
        wt[(((long long)cs * a.Kp + k) * 4 + u % 4) * 4 + u / 4] = word;
        if (c0 % a.group == 0 && c0 < a.C) scale[(long long)(c0 / a.group) * a.Kp + k] = s;
    }
}

__global__ __launch_bounds__(256) void seq_mv4_unquant_kernel(const SeqMv4Args a, float *w)
{
    const long long total = (long long)a.K * a.C;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < total; t += (long long)gridDim.x * 256) {
        const int k = (int)(t / a.C), c = (int)(t % a.C);
        const unsigned word = static_cast<const unsigned *>(a.wt)[(((long long)(c / 128) * a.Kp + k) * 4 + c % 32 / 8) * 4 + c % 128 / 32];
        w[t] = (float)((int)(word << (28 - 4 * (c % 8))) >> 28) * a.scale[(long long)(c / a.group) * a.Kp + k];
    }
}

template <int DT, int GROUP, int KT, int NT, int U, bool STAGE>
hipError_t launch_nt(const SeqMv4Args &a, hipStream_t s)
{
    const int threads = (a.Cs < kMaxWaves ? a.Cs : kMaxWaves) * 64;
    seq_mv4_kernel<DT, KT, NT, GROUP, U, STAGE><<<dim3((a.Kp / 16 + KT - 1) / KT, (a.M + 16 * NT - 1) / (16 * NT)), threads, 0, s>>>(a);
    return hipGetLastError();
}
template <int DT, int GROUP, int KT>
hipError_t launch_kt(const SeqMv4Args &a, hipStream_t s)
{
    // Staged from five tokens on; not fp32, of which a token's quarter of a run is a whole line (48 tokens of 4096 x 8192 44 us both).
    constexpr bool STAGE = DT != SEQ_F32;
    constexpr int U = STAGE && !(DT == SEQ_BF16 && GROUP == 32 && KT == 2) ? 4 : 2;  // (as many as the registers hold)
    if (a.M <= 4) return launch_nt<DT, GROUP, KT, 1, U, false>(a, s);
    if (a.M <= 16) return launch_nt<DT, GROUP, KT, 1, U, STAGE>(a, s);
    if constexpr (KT > 1) {
        // The tokens by up to four tiles of 16 a workgroup (fp32 three: 64 tokens 42 and 40 us), evenly: for each share the weights come again.  (48 tokens of 4096 x 8192, by
        // twos and by threes: 8 bits 14.2 and 9.9 us, fp32 43 and 31.  Few weights want the workgroups: 1024 x 2048 in 8 bits 3.5 and 4.2.)
        constexpr int most = STAGE ? 4 : 3;
        const int tiles = (a.M + 15) / 16, rows = (tiles + most - 1) / most, each = (tiles + rows - 1) / rows;
        if (each == 3) return launch_nt<DT, GROUP, KT, 3, 1, STAGE>(a, s);
        if constexpr (STAGE)
            if (each == 4) return launch_nt<DT, GROUP, KT, 4, 1, STAGE>(a, s);
    }
    return launch_nt<DT, GROUP, KT, 2, STAGE ? 2 : 1, STAGE>(a, s);
}
template <int DT, int GROUP>
hipError_t launch(const SeqMv4Args &a, hipStream_t s)
{
    // Two tiles of weights a workgroup where there are workgroups for all compute units (256) even so; for half of them already where there
    // are two tiles of tokens, whose turns through LDS otherwise take longer than the weights.  (One tile and two: 4096 x 8192, 32 tokens bf16 12.9
    // and 10.8 us, 48 fp32 63 and 32, one 8.2 both; 24 tokens 2048 x 4100 8.4 and 6.8, 2048 x 2048 5.5 and 6.6; 16 in 8 bits 4096 x 4096
    // 5.7 and 6.7; 8 bf16 1024 x 1024 3.6 and 4.0.  Four tiles: 24 tokens 2048 x 4100 11.6.)
    return a.Kp / 32 >= (a.M > 16 ? 128 : 256) ? launch_kt<DT, GROUP, 2>(a, s) : launch_kt<DT, GROUP, 1>(a, s);
}
template <int DT>
hipError_t launch_group(const SeqMv4Args &a, hipStream_t s)
{
    return a.group == 32 ? launch<DT, 32>(a, s) : a.group == 64 ? launch<DT, 64>(a, s) : launch<DT, 128>(a, s);
}
}  // namespace

hipError_t launch_seq_mv4(int dtype, const SeqMv4Args &a, hipStream_t s)
{
    return dtype == SEQ_I8 ? launch_group<SEQ_I8>(a, s) : dtype == SEQ_BF16 ? launch_group<SEQ_BF16>(a, s) : launch_group<SEQ_F32>(a, s);
}
hipError_t launch_seq_mv4_quant(const SeqMv4Args &a, const float *w, void *wt, float *scale, hipStream_t s)
{
    const long long blocks = (long long)a.Cs * a.Kp / 16;
    seq_mv4_quant_kernel<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(a, w, static_cast<unsigned *>(wt), scale);
    return hipGetLastError();
}
hipError_t launch_seq_mv4_unquant(const SeqMv4Args &a, float *w, hipStream_t s)
{
    const long long blocks = ((long long)a.K * a.C + 255) / 256;
    seq_mv4_unquant_kernel<<<(unsigned)(blocks < 65536 ? blocks : 65536), 256, 0, s>>>(a, w);
    return hipGetLastError();
}

}  // namespace convmi
