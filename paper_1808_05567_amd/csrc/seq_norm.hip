// Root-mean-square norm with the residual's addition, forward (result in the tensors' type or in 8 bits) and backward.
//
//   r = x + res,   y = w r rstd,  rstd = 1 / sqrt(mean r^2 + eps)
//   dx = dr + rstd (w dy - r rstd^2 mean(w dy r)),   dw = sum dy r rstd
//
// A few operations an element: bound by memory.  A workgroup holds whole positions in registers between the sums over
// their channels and the result, so that each tensor is read once.  Measured, 8 x 2048 positions of 2048 channels in bf16, 268 MB: forward 54 us
// (5.0 TB/s; positions side by side 48), backward 78 (66) and 5 for the sums of dw; 2 x 1024 positions in fp32, 67 MB, backward 18 and 4.
#include <type_traits>

#include "seq_internal.h"

namespace convmi {
namespace {

constexpr int kMaxThreads = 512;

// Sums (or largest unsigned) of v over the threads with the same place in the tile of LT positions, in all of them: by turns of
// rows of 16 lanes, then between rows and halves of a wave, then in LDS (ALONE: each wave has a position of its own).  Within rows a lane
// starts from its own number: sums of one position may differ by a unit between its lanes, the same way on every run.
template <int LT, bool MAX, bool ALONE = false>
static __device__ __forceinline__ float row_sum(float v, float *lds)
{
    auto join = [](float p, float q) { return MAX ? __uint_as_float(max(__float_as_uint(p), __float_as_uint(q))) : p + q; };
    auto turn = [](float p, auto by) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(p), 0x120 + decltype(by)::value, 0xf, 0xf, true)); };
    if constexpr (LT <= 1) v = join(v, turn(v, std::integral_constant<int, 1>()));
    if constexpr (LT <= 2) v = join(v, turn(v, std::integral_constant<int, 2>()));
    if constexpr (LT <= 4) v = join(v, turn(v, std::integral_constant<int, 4>()));
    if constexpr (LT <= 8) v = join(v, turn(v, std::integral_constant<int, 8>()));
    const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = join(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
    const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = join(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
    const int waves = blockDim.x / 64;
    if (ALONE || waves == 1) return v;
    if (threadIdx.x % 64 < LT) lds[threadIdx.x / 64 * LT + threadIdx.x % 64] = v;
    __syncthreads();
    v = lds[threadIdx.x % LT];
    for (int w = 1; w < waves; ++w) v = join(v, lds[w * LT + threadIdx.x % LT]);
    __syncthreads();
    return v;
}

// LT positions at a time, 64 / LT blocks a wave side by side: 8 x 8 where a block's positions follow one another (128 bytes),
// 1 x 64 where a position's blocks do.  NV: blocks a thread holds; 0: more than fit, each read twice.
template <typename T, int LT, int NV, bool Q8, bool PAST>
__global__ __launch_bounds__(kMaxThreads) void seq_norm_fwd_kernel(const SeqNormArgs a)
{
    constexpr int V = SeqElem<T>::V;
    __shared__ float lds[kMaxThreads / 64 * LT];
    // (a launch has at most 2^32 work-items)
    for (long long tile = blockIdx.x; tile * LT < a.rows; tile += gridDim.x) {
        const long long row = tile * LT + threadIdx.x % LT;
        const bool live = row < a.rows;
        const int n = live ? (int)(row / a.L) : 0, l = live ? (int)(row % a.L) : 0;
        const int first = threadIdx.x / LT, step = blockDim.x / LT;
        const T *x = static_cast<const T *>(a.x) + n * a.vx.n + l * a.vx.l;
        const T *res = a.res ? static_cast<const T *>(a.res) + n * a.vres.n + l * a.vres.l : nullptr;
        T *r = a.r ? static_cast<T *>(a.r) + n * a.vr.n + l * a.vr.l : nullptr;
        auto sum_of = [&](int b) {
            seq_u32x4 p = seq_load(x + b * a.vx.c);
            if (res) {
                float f[V], g[V];
                SeqElem<T>::unpack(p, f);
                SeqElem<T>::unpack(seq_load(res + b * a.vres.c), g);
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] += g[i];
                p = SeqElem<T>::pack(f);
            }
            if (r) seq_store_result<PAST && NV != 0>(r + b * a.vr.c, p);
            return p;
        };
        auto squares = [](const seq_u32x4 &p, float s) {
            float f[V];
            SeqElem<T>::unpack(p, f);
#pragma unroll
            for (int i = 0; i < V; ++i) s = fmaf(f[i], f[i], s);
            return s;
        };
        seq_u32x4 keep[NV ? NV : 1];
        float s = 0;
        if constexpr (NV > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int b = first + j * step;
                keep[j] = seq_u32x4{};
                if (live && b < a.Cb) keep[j] = sum_of(b);
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) s = squares(keep[j], s);
        } else if (live) {
            for (int b = first; b < a.Cb; b += step) s = squares(sum_of(b), s);
        }
        const float rstd = 1.0f / sqrtf(row_sum<LT, false>(s, lds) / a.C + a.eps);
        // (the second time from where the first left it: r may lie in x's or res's place)
        auto again = [&](int j, int b) {
            if constexpr (NV > 0) return keep[j];
            if (r) return seq_load(r + b * a.vr.c);
            seq_u32x4 p = seq_load(x + b * a.vx.c);
            if (res) {
                float f[V], g[V];
                SeqElem<T>::unpack(p, f);
                SeqElem<T>::unpack(seq_load(res + b * a.vres.c), g);
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] += g[i];
                p = SeqElem<T>::pack(f);
            }
            return p;
        };
        auto norm = [&](const seq_u32x4 &p, int b, float (&f)[V]) {
            float w[V];
            SeqElem<T>::unpack(p, f);
            seq_vector<V>(a.w, b, w);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = f[i] * rstd * w[i];
        };
        if constexpr (!Q8) {
            if (!live) continue;
            T *y = static_cast<T *>(a.y) + n * a.vy.n + l * a.vy.l;
            auto put = [&](int j, int b) {
                float f[V];
                norm(again(j, b), b, f);
                seq_store_result<PAST>(y + b * a.vy.c, SeqElem<T>::pack(f));
            };
            if constexpr (NV > 0) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (first + j * step < a.Cb) put(j, first + j * step);
            } else
                for (int b = first; b < a.Cb; b += step) put(0, b);
        } else {
            // (as unsigned numbers NaN is the largest: one in a position makes its scale NaN)
            float m = 0;
            auto largest = [&](int j, int b) {
                float f[V];
                norm(again(j, b), b, f);
#pragma unroll
                for (int i = 0; i < V; ++i) m = __uint_as_float(max(__float_as_uint(m), __float_as_uint(fabsf(f[i]))));
            };
            if constexpr (NV > 0) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (live && first + j * step < a.Cb) largest(j, first + j * step);
            } else if (live)
                for (int b = first; b < a.Cb; b += step) largest(0, b);
            m = row_sum<LT, true>(m, lds);
            if (!live) continue;
            float scale = m / 127.0f;
            if (scale < 1.17549435e-38f) scale = 0;  // (its reciprocal would be infinite)
            if (first == 0) a.scale[row] = scale;
            const float inv = scale == 0 ? 0 : 1.0f / scale;
            int8_t *q = a.q + n * a.vq.n + l * a.vq.l;
            auto put = [&](int j, int b) {
                unsigned word[V / 4] = {};
                if (b < a.Cb) {
                    float f[V];
                    norm(again(j, b), b, f);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int v = (int)rintf(fminf(fmaxf(f[i] * inv, -127.0f), 127.0f));
                        word[i / 4] |= (unsigned)(v & 255) << i % 4 * 8;
                    }
                }
                unsigned *at = reinterpret_cast<unsigned *>(q + b * V / 16 * a.vq.c + b * V % 16);
#pragma unroll
                for (int i = 0; i < V / 4; ++i) at[i] = word[i];
            };
            const int blocks = (a.Cb * V + 15) / 16 * (16 / V);  // (up to the end of the last 16 channels)
            if constexpr (NV > 0) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (first + j * step < a.Cb) put(j, first + j * step);
                for (int b = a.Cb + first; b < blocks; b += step) put(0, b);
            } else
                for (int b = first; b < blocks; b += step) put(0, b);
        }
    }
}

// ALONE: each wave has positions of its own, and waits for no other until their parts of dw are added.
template <typename T, int LT, int NV, bool ALONE>
__global__ __launch_bounds__(kMaxThreads) void seq_norm_bwd_kernel(const SeqNormArgs a)
{
    static_assert(!ALONE || LT == 1, "one position a wave");
    constexpr int V = SeqElem<T>::V;
    constexpr int NK = NV ? NV : 1;
    __shared__ float lds[kMaxThreads / 64 * LT];
    const int first = ALONE ? threadIdx.x % 64 : threadIdx.x / LT, step = ALONE ? 64 : blockDim.x / LT;
    const int waves = blockDim.x / 64, each = ALONE ? waves : LT;  // positions of a workgroup at a time
    float dw[NK][V] = {};
    for (long long tile = blockIdx.x; tile * each < a.rows; tile += gridDim.x) {
        const long long row = tile * each + (ALONE ? threadIdx.x / 64 : threadIdx.x % LT);
        const bool live = row < a.rows;
        const int n = live ? (int)(row / a.L) : 0, l = live ? (int)(row % a.L) : 0;
        const T *r = static_cast<const T *>(a.r) + n * a.vr.n + l * a.vr.l;
        const T *dy = static_cast<const T *>(a.dy) + n * a.vdy.n + l * a.vdy.l;
        const T *dr = a.dr ? static_cast<const T *>(a.dr) + n * a.vdr.n + l * a.vdr.l : nullptr;
        T *dx = static_cast<T *>(a.dx) + n * a.vdx.n + l * a.vdx.l;
        seq_u32x4 kr[NK], ky[NK];
        float ss = 0, dot = 0;
        auto sums = [&](const seq_u32x4 &p, const seq_u32x4 &q, int b) {
            float f[V], g[V], w[V];
            SeqElem<T>::unpack(p, f);
            SeqElem<T>::unpack(q, g);
            seq_vector<V>(a.w, b, w);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                ss = fmaf(f[i], f[i], ss);
                dot = fmaf(f[i], g[i] * w[i], dot);
            }
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int b = first + j * step;
                kr[j] = ky[j] = seq_u32x4{};
                if (live && b < a.Cb) {
                    kr[j] = seq_load(r + b * a.vr.c);
                    ky[j] = seq_load(dy + b * a.vdy.c);
                }
            }
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (first + j * step < a.Cb) sums(kr[j], ky[j], first + j * step);
        } else if (live)
            for (int b = first; b < a.Cb; b += step) sums(seq_load(r + b * a.vr.c), seq_load(dy + b * a.vdy.c), b);
        ss = row_sum<LT, false, ALONE>(ss, lds);
        dot = row_sum<LT, false, ALONE>(dot, lds);
        const float rstd = 1.0f / sqrtf(ss / a.C + a.eps);
        const float mean = dot / a.C * rstd * rstd;
        auto put = [&](const seq_u32x4 &p, const seq_u32x4 &q, int j, int b) {
            float f[V], g[V], w[V], d[V] = {};
            SeqElem<T>::unpack(p, f);
            SeqElem<T>::unpack(q, g);
            seq_vector<V>(a.w, b, w);
            if (dr) SeqElem<T>::unpack(seq_load(dr + b * a.vdr.c), d);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                d[i] = fmaf(rstd, fmaf(-mean, f[i], g[i] * w[i]), d[i]);
                dw[j][i] = fmaf(g[i], f[i] * rstd, dw[j][i]);
            }
            seq_store(dx + b * a.vdx.c, SeqElem<T>::pack(d));
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (live && first + j * step < a.Cb) put(kr[j], ky[j], j, first + j * step);
        } else {
            // (the positions of one workgroup in turn: its part of dw is summed where it is stored)
            float *part = a.part + (long long)blockIdx.x * a.Cp;
            for (int b = first; b < a.Cb; b += step) {
#pragma unroll
                for (int i = 0; i < V; ++i) dw[0][i] = 0;
                if (live) put(seq_load(r + b * a.vr.c), seq_load(dy + b * a.vdy.c), 0, b);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float s = dw[0][i];
#pragma unroll
                    for (int d = 1; d < LT; d *= 2) s += __shfl_xor(s, d);
                    if (threadIdx.x % LT == 0) {
                        float *at = part + (long long)b * V + i;
                        *at = tile == blockIdx.x ? s : *at + s;
                    }
                }
            }
        }
    }
    if constexpr (ALONE) {
        // the waves' sums in order, a block a lane at a time
        __shared__ float sums[kMaxThreads / 64][64 * V];
        float *part = a.part + (long long)blockIdx.x * a.Cp;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) sums[threadIdx.x / 64][i * 64 + first] = dw[j][i];
            __syncthreads();
            for (int e = threadIdx.x; e < 64 * V; e += blockDim.x) {
                const int b = j * 64 + e % 64;
                float s = 0;
                for (int w = 0; w < waves; ++w) s += sums[w][e];
                if (b < a.Cb) part[(long long)b * V + e / 64] = s;
            }
            __syncthreads();
        }
    } else if constexpr (NV > 0) {
        float *part = a.part + (long long)blockIdx.x * a.Cp;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int b = first + j * step;
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int d = 1; d < LT; d *= 2) dw[j][i] += __shfl_xor(dw[j][i], d);
            if (b < a.Cb && threadIdx.x % LT == 0)
#pragma unroll
                for (int i = 0; i < V; ++i) part[(long long)b * V + i] = dw[j][i];
        }
    }
}

// dw: the workgroups' sums in order.
__global__ __launch_bounds__(1024) void seq_norm_reduce_kernel(const float *part, float *dw, int parts, int Cp)
{
    const int c = blockIdx.x * kSumColumns + threadIdx.x % kSumColumns;
    const float s = seq_sum_parts(part + c, Cp, parts, c < Cp);
    if (threadIdx.x < kSumColumns && c < Cp) dw[c] = s;
}

hipError_t reduce(const SeqNormArgs &a, unsigned parts, hipStream_t s)
{
    seq_norm_reduce_kernel<<<(a.Cp + kSumColumns - 1) / kSumColumns, 1024, 0, s>>>(a.part, a.dw, (int)parts, a.Cp);
    return hipGetLastError();
}

template <typename T, int LT, int NV>
hipError_t launch_nv(bool bwd, const SeqNormArgs &a, int threads, hipStream_t s)
{
    const long long tiles = (a.rows + LT - 1) / LT;
    const unsigned grid = (unsigned)(tiles < 1 << 22 ? tiles : 1 << 22);
    if constexpr (LT == 16) {
        if (bwd) return hipErrorInvalidValue;  // (goes by eight)
    } else if (bwd) {
        const unsigned parts = grid < (unsigned)a.parts ? grid : (unsigned)a.parts;
        seq_norm_bwd_kernel<T, LT, NV, false><<<parts, threads, 0, s>>>(a);
        return reduce(a, parts, s);
    }
    if (a.q)
        seq_norm_fwd_kernel<T, LT, NV, true, false><<<grid, threads, 0, s>>>(a);
    else if (a.past)
        seq_norm_fwd_kernel<T, LT, NV, false, true><<<grid, threads, 0, s>>>(a);
    else
        seq_norm_fwd_kernel<T, LT, NV, false, false><<<grid, threads, 0, s>>>(a);
    return hipGetLastError();
}

// Threads of a workgroup and blocks that each holds: 256 threads with up to 8 blocks, then up to 512.  LT positions that do not fit
// that go as fewer at a time, in shorter pieces; what one position does not fit is read twice.
template <typename T, int LT>
hipError_t launch_lt(bool bwd, const SeqNormArgs &a, hipStream_t s)
{
    const long long lanes = (long long)a.Cb * LT;
    int threads = 64;
    while (threads < 256 && threads < lanes) threads *= 2;
    if (threads * 8 < lanes) threads = kMaxThreads;
    const long long nv = (lanes + threads - 1) / threads;
    if constexpr (LT >= 8 || LT == 1) {  // (what comes to 4 and 2 has more)
        if (nv <= 1) return launch_nv<T, LT, 1>(bwd, a, threads, s);
        if (nv <= 2) return launch_nv<T, LT, 2>(bwd, a, threads, s);
        if (nv <= 4) return launch_nv<T, LT, 4>(bwd, a, threads, s);
    }
    if (nv <= 8) return launch_nv<T, LT, 8>(bwd, a, threads, s);
    if constexpr (LT > 1)
        return launch_lt<T, LT / 2>(bwd, a, s);
    else
        return launch_nv<T, LT, 0>(bwd, a, threads, s);
}
template <typename T, int NV>
hipError_t launch_alone(const SeqNormArgs &a, hipStream_t s)
{
    seq_norm_bwd_kernel<T, 1, NV, true><<<(unsigned)a.parts, 256, 0, s>>>(a);
    return reduce(a, (unsigned)a.parts, s);
}
template <typename T>
hipError_t launch_t(bool bwd, const SeqNormArgs &a, hipStream_t s)
{
    // one position at a time where its blocks follow one another in what is read; else eight, forwards sixteen where that leaves two
    // workgroups for each compute unit (8 x 2048 x 2048 bf16 61 -> 55 us; backwards, with fewer registers left, 78 -> 86)
    constexpr int V = SeqElem<T>::V;
    const SeqView &v = bwd ? a.vr : a.vx;
    if (v.c == V || a.L == 1) {
        // a wave each where that leaves every workgroup two for each of its waves (8 x 2048 x 2048 bf16, workgroups of one position: 85 us)
        if (bwd && a.rows >= 8LL * a.parts && a.Cb <= 8 * 64)
            return a.Cb <= 64 ? launch_alone<T, 1>(a, s) : a.Cb <= 2 * 64 ? launch_alone<T, 2>(a, s) : a.Cb <= 4 * 64 ? launch_alone<T, 4>(a, s) : launch_alone<T, 8>(a, s);
        return launch_lt<T, 1>(bwd, a, s);
    }
    return bwd || a.rows < 16 * 512 ? launch_lt<T, 8>(bwd, a, s) : launch_lt<T, 16>(bwd, a, s);
}
}  // namespace

hipError_t launch_seq_norm_fwd(int dtype, const SeqNormArgs &a, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch_t<unsigned short>(false, a, s) : launch_t<float>(false, a, s);
}
hipError_t launch_seq_norm_bwd(int dtype, const SeqNormArgs &a, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch_t<unsigned short>(true, a, s) : launch_t<float>(true, a, s);
}

}  // namespace convmi
