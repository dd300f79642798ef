// Layer norm with the residual's addition, forward (result in the tensors' type or in 8 bits) and backward.
//
//   r = x + res,   u = (r - mean r) rstd,   y = u w + b,   rstd = 1 / sqrt(mean (r - mean r)^2 + eps)
//   dx = dr + rstd (w dy - mean(w dy) - u mean(w dy u)),   dw = sum dy u,   db = sum dy
//
// As the root-mean-square norm: a workgroup holds whole positions in registers between the sums over their channels and the result.  The squares are
// of the differences from the mean, formed after it is known: a mean far from zero costs nothing of the variance.
#include <type_traits>

#include "seq_internal.h"

namespace convmi {
namespace {

constexpr int kMaxThreads = 512;

// Sums (MAX: largest unsigned) of K numbers over the threads with the same place in a tile of LT positions, in all of them, in an order that goes by
// the threads' places alone.  ALONE: each wave has positions of its own.
template <int LT, bool MAX, bool ALONE, int K>
static __device__ __forceinline__ void row_sums(float (&v)[K], float *lds)
{
    auto join = [](float p, float q) { return MAX ? __uint_as_float(max(__float_as_uint(p), __float_as_uint(q))) : p + q; };
    auto turn = [](float p, auto by) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(p), 0x120 + decltype(by)::value, 0xf, 0xf, true)); };
    const int waves = blockDim.x / 64, wave = threadIdx.x / 64, at = threadIdx.x % LT;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if constexpr (LT <= 1) v[k] = join(v[k], turn(v[k], std::integral_constant<int, 1>()));
        if constexpr (LT <= 2) v[k] = join(v[k], turn(v[k], std::integral_constant<int, 2>()));
        if constexpr (LT <= 4) v[k] = join(v[k], turn(v[k], std::integral_constant<int, 4>()));
        if constexpr (LT <= 8) v[k] = join(v[k], turn(v[k], std::integral_constant<int, 8>()));
        const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[k]), __float_as_uint(v[k]), false, false);
        v[k] = join(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
        const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[k]), __float_as_uint(v[k]), false, false);
        v[k] = join(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
    }
    if (ALONE || waves == 1) return;
    if (threadIdx.x % 64 < LT)
#pragma unroll
        for (int k = 0; k < K; ++k) lds[(wave * K + k) * LT + at] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        v[k] = lds[k * LT + at];
        for (int w = 1; w < waves; ++w) v[k] = join(v[k], lds[(w * K + k) * LT + at]);
    }
    __syncthreads();
}

// Where a position lies, and whether it is inside its sequence; what is behind its end comes out as zero.
template <typename T>
struct Place {
    bool live, inside;
    int n, l;
    __device__ __forceinline__ Place(const SeqNormArgs &a, long long row)
    {
        live = row < a.rows;
        n = live ? (int)(row / a.L) : 0;
        l = live ? (int)(row % a.L) : 0;
        inside = live && (!a.lengths || l < seq_length(a.lengths, n, a.L));
    }
};

// The slots of the last block beyond C, which count in no sum and come out as zero.
template <int V>
static __device__ __forceinline__ void clear_beyond(const SeqNormArgs &a, int b, float (&f)[V])
{
    if (a.C == a.Cp || b != a.Cb - 1) return;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (b * V + i >= a.C) f[i] = 0;
}

// LT positions at a time, 64 / LT blocks a wave side by side, as in the root-mean-square norm.  NV: blocks a thread holds; 0: more than fit, read again.
template <typename T, int LT, int NV, bool Q8, bool PAST>
__global__ __launch_bounds__(kMaxThreads) void seq_lnorm_fwd_kernel(const SeqNormArgs a)
{
    constexpr int V = SeqElem<T>::V;
    __shared__ float lds[kMaxThreads / 64 * LT];
    for (long long tile = blockIdx.x; tile * LT < a.rows; tile += gridDim.x) {
        const long long row = tile * LT + threadIdx.x % LT;
        const Place<T> at(a, row);
        const int first = threadIdx.x / LT, step = blockDim.x / LT;
        const T *x = static_cast<const T *>(a.x) + at.n * a.vx.n + at.l * a.vx.l;
        const T *res = a.res ? static_cast<const T *>(a.res) + at.n * a.vres.n + at.l * a.vres.l : nullptr;
        T *r = a.r ? static_cast<T *>(a.r) + at.n * a.vr.n + at.l * a.vr.l : nullptr;
        // (a position behind its sequence's end: zeros, whatever x and res hold)
        auto sum_of = [&](int b) {
            if (!at.inside) return seq_u32x4{};
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
        auto first_time = [&](int b) {
            const seq_u32x4 p = sum_of(b);
            if (r) seq_store_result<PAST && NV != 0>(r + b * a.vr.c, p);
            return p;
        };
        seq_u32x4 keep[NV ? NV : 1];
        // (again from where the first time left it: r may lie in x's or res's place)
        auto again = [&](int j, int b) {
            if constexpr (NV > 0) return keep[j];
            return r ? seq_load(r + b * a.vr.c) : sum_of(b);
        };
        auto over = [&](auto &&each) {
            if constexpr (NV > 0) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (at.live && first + j * step < a.Cb) each(j, first + j * step);
            } else if (at.live)
                for (int b = first; b < a.Cb; b += step) each(0, b);
        };
        float s[1] = {};
        if constexpr (NV > 0) over([&](int j, int b) { keep[j] = first_time(b); });
        over([&](int j, int b) {
            float f[V];
            if constexpr (NV > 0)
                SeqElem<T>::unpack(keep[j], f);
            else
                SeqElem<T>::unpack(first_time(b), f);
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += f[i];
        });
        row_sums<LT, false, false>(s, lds);
        const float mean = s[0] / a.C;
        s[0] = 0;
        auto difference = [&](int j, int b, float (&f)[V]) {
            SeqElem<T>::unpack(again(j, b), f);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] -= mean;
            clear_beyond<V>(a, b, f);
        };
        over([&](int j, int b) {
            float f[V];
            difference(j, b, f);
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] = fmaf(f[i], f[i], s[0]);
        });
        row_sums<LT, false, false>(s, lds);
        const float rstd = 1.0f / sqrtf(s[0] / a.C + a.eps);
        auto norm = [&](int j, int b, float (&f)[V]) {
            float w[V], c[V] = {};
            difference(j, b, f);
            seq_vector<V>(a.w, b, w);
            if (a.b) seq_vector<V>(a.b, b, c);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = at.inside ? fmaf(f[i] * rstd, w[i], c[i]) : 0.0f;
            clear_beyond<V>(a, b, f);
        };
        if constexpr (!Q8) {
            T *y = static_cast<T *>(a.y) + at.n * a.vy.n + at.l * a.vy.l;
            over([&](int j, int b) {
                float f[V];
                norm(j, b, f);
                seq_store_result<PAST>(y + b * a.vy.c, SeqElem<T>::pack(f));
            });
        } else {
            // (as unsigned numbers NaN is the largest: one in a position makes its scale NaN)
            float m[1] = {};
            over([&](int j, int b) {
                float f[V];
                norm(j, b, f);
#pragma unroll
                for (int i = 0; i < V; ++i) m[0] = __uint_as_float(max(__float_as_uint(m[0]), __float_as_uint(fabsf(f[i]))));
            });
            row_sums<LT, true, false>(m, lds);
            if (!at.live) continue;
            float scale = m[0] / 127.0f;
            if (scale < 1.17549435e-38f) scale = 0;  // (its reciprocal would be infinite)
            if (first == 0) a.scale[row] = scale;
            const float inv = scale == 0 ? 0 : 1.0f / scale;
            int8_t *q = a.q + at.n * a.vq.n + at.l * a.vq.l;
            auto put = [&](int j, int b) {
                unsigned word[V / 4] = {};
                if (b < a.Cb) {
                    float f[V];
                    norm(j, b, f);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int v = (int)rintf(fminf(fmaxf(f[i] * inv, -127.0f), 127.0f));
                        word[i / 4] |= (unsigned)(v & 255) << i % 4 * 8;
                    }
                }
                unsigned *to = reinterpret_cast<unsigned *>(q + b * V / 16 * a.vq.c + b * V % 16);
#pragma unroll
                for (int i = 0; i < V / 4; ++i) to[i] = word[i];
            };
            over(put);
            const int blocks = (a.Cb * V + 15) / 16 * (16 / V);  // (up to the end of the last 16 channels)
            if (first == 0)
                for (int b = a.Cb; b < blocks; ++b) put(0, b);
        }
    }
}

// ALONE: each wave has positions of its own, and waits for no other until their parts of dw and db are added.
template <typename T, int LT, int NV, bool ALONE>
__global__ __launch_bounds__(kMaxThreads) void seq_lnorm_bwd_kernel(const SeqNormArgs a)
{
    static_assert(!ALONE || LT == 1, "one position a wave");
    constexpr int V = SeqElem<T>::V, NK = NV ? NV : 1;
    __shared__ float lds[kMaxThreads / 64 * LT * 2];
    const int first = ALONE ? threadIdx.x % 64 : threadIdx.x / LT, step = ALONE ? 64 : blockDim.x / LT;
    const int waves = blockDim.x / 64, each = ALONE ? waves : LT;  // positions of a workgroup at a time
    float *part = a.part + (long long)blockIdx.x * 2 * a.Cp;
    float dw[NK][V] = {}, db[NK][V] = {};
    for (long long tile = blockIdx.x; tile * each < a.rows; tile += gridDim.x) {
        const Place<T> at(a, tile * each + (ALONE ? threadIdx.x / 64 : threadIdx.x % LT));
        const T *r = static_cast<const T *>(a.r) + at.n * a.vr.n + at.l * a.vr.l;
        const T *dy = static_cast<const T *>(a.dy) + at.n * a.vdy.n + at.l * a.vdy.l;
        const T *dr = a.dr ? static_cast<const T *>(a.dr) + at.n * a.vdr.n + at.l * a.vdr.l : nullptr;
        T *dx = static_cast<T *>(a.dx) + at.n * a.vdx.n + at.l * a.vdx.l;
        seq_u32x4 kr[NK], ky[NK];
        auto load = [&](int j, int b) {
            kr[j] = ky[j] = seq_u32x4{};
            if (at.inside) {
                kr[j] = seq_load(r + b * a.vr.c);
                ky[j] = seq_load(dy + b * a.vdy.c);
            }
        };
        auto over = [&](auto &&body) {
            if constexpr (NV > 0) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (at.live && first + j * step < a.Cb) body(j, first + j * step);
            } else if (at.live)
                for (int b = first; b < a.Cb; b += step) {
                    load(0, b);
                    body(0, b);
                }
        };
        if constexpr (NV > 0) over(load);
        float s[2] = {};
        over([&](int j, int b) {
            float f[V], g[V], w[V];
            SeqElem<T>::unpack(kr[j], f);
            SeqElem<T>::unpack(ky[j], g);
            seq_vector<V>(a.w, b, w);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[0] += f[i];
                s[1] = fmaf(g[i], w[i], s[1]);
            }
        });
        row_sums<LT, false, ALONE>(s, lds);
        const float mean = s[0] / a.C, through = s[1] / a.C;
        s[0] = s[1] = 0;
        auto difference = [&](int j, int b, float (&f)[V], float (&g)[V]) {
            SeqElem<T>::unpack(kr[j], f);
            SeqElem<T>::unpack(ky[j], g);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] -= mean;
            clear_beyond<V>(a, b, f);
        };
        over([&](int j, int b) {
            float f[V], g[V], w[V];
            difference(j, b, f, g);
            seq_vector<V>(a.w, b, w);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[0] = fmaf(f[i], f[i], s[0]);
                s[1] = fmaf(f[i], g[i] * w[i], s[1]);
            }
        });
        row_sums<LT, false, ALONE>(s, lds);
        const float rstd = 1.0f / sqrtf(s[0] / a.C + a.eps);
        const float along = s[1] / a.C * rstd * rstd;
        over([&](int j, int b) {
            float f[V], g[V], w[V], d[V] = {};
            difference(j, b, f, g);
            seq_vector<V>(a.w, b, w);
            if (dr && at.inside) SeqElem<T>::unpack(seq_load(dr + b * a.vdr.c), d);
            if constexpr (NV == 0) {
#pragma unroll
                for (int i = 0; i < V; ++i) dw[0][i] = db[0][i] = 0;
            }
            if (at.inside) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    d[i] = fmaf(rstd, fmaf(-along, f[i], fmaf(g[i], w[i], -through)), d[i]);
                    dw[j][i] = fmaf(g[i], f[i] * rstd, dw[j][i]);
                    db[j][i] += g[i];
                }
                clear_beyond<V>(a, b, d);
            }
            seq_store(dx + b * a.vdx.c, SeqElem<T>::pack(d));
            if constexpr (NV == 0) {
                // (the positions of one workgroup in turn, one at a time: its part is summed where it is stored)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float *to = part + (long long)b * V + i;
                    *to = tile == blockIdx.x ? dw[0][i] : *to + dw[0][i];
                    to += a.Cp;
                    *to = tile == blockIdx.x ? db[0][i] : *to + db[0][i];
                }
            }
        });
    }
    if constexpr (ALONE) {
        // the waves' sums in order, a block a lane at a time
        __shared__ float sums[kMaxThreads / 64][64 * V];
#pragma unroll
        for (int j = 0; j < 2 * NV; ++j) {
#pragma unroll
            for (int i = 0; i < V; ++i) sums[threadIdx.x / 64][i * 64 + first] = j < NV ? dw[j % NV][i] : db[j % NV][i];
            __syncthreads();
            for (int e = threadIdx.x; e < 64 * V; e += blockDim.x) {
                const int b = j % NV * 64 + e % 64;
                float s = 0;
                for (int w = 0; w < waves; ++w) s += sums[w][e];
                if (b < a.Cb) part[(j < NV ? 0 : a.Cp) + (long long)b * V + e / 64] = s;
            }
            __syncthreads();
        }
    } else if constexpr (NV > 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int b = first + j * step;
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int d = 1; d < LT; d *= 2) {
                    dw[j][i] += __shfl_xor(dw[j][i], d);
                    db[j][i] += __shfl_xor(db[j][i], d);
                }
            if (b < a.Cb && threadIdx.x % LT == 0)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    part[(long long)b * V + i] = dw[j][i];
                    part[a.Cp + (long long)b * V + i] = db[j][i];
                }
        }
    }
}

// dw and db: the workgroups' sums in order.
__global__ __launch_bounds__(1024) void seq_lnorm_reduce_kernel(const float *part, float *dw, float *db, int parts, int Cp)
{
    const int c = blockIdx.x * kSumColumns + threadIdx.x % kSumColumns;
    const float s = seq_sum_parts(part + c, 2LL * Cp, parts, c < 2 * Cp);
    if (threadIdx.x >= kSumColumns || c >= 2 * Cp) return;
    if (c < Cp)
        dw[c] = s;
    else if (db)
        db[c - Cp] = s;
}

hipError_t reduce(const SeqNormArgs &a, unsigned parts, hipStream_t s)
{
    seq_lnorm_reduce_kernel<<<(2 * a.Cp + kSumColumns - 1) / kSumColumns, 1024, 0, s>>>(a.part, a.dw, a.db, (int)parts, a.Cp);
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
        seq_lnorm_bwd_kernel<T, LT, NV, false><<<parts, threads, 0, s>>>(a);
        return reduce(a, parts, s);
    }
    if (a.q)
        seq_lnorm_fwd_kernel<T, LT, NV, true, false><<<grid, threads, 0, s>>>(a);
    else if (a.past)
        seq_lnorm_fwd_kernel<T, LT, NV, false, true><<<grid, threads, 0, s>>>(a);
    else
        seq_lnorm_fwd_kernel<T, LT, NV, false, false><<<grid, threads, 0, s>>>(a);
    return hipGetLastError();
}

// Threads of a workgroup and blocks that each holds: 256 threads with up to 8 blocks, then up to 512.  LT positions that do not fit
// that go as fewer at a time; what one position does not fit is read again.
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
    seq_lnorm_bwd_kernel<T, 1, NV, true><<<(unsigned)a.parts, 256, 0, s>>>(a);
    return reduce(a, (unsigned)a.parts, s);
}
template <typename T>
hipError_t launch_t(bool bwd, const SeqNormArgs &a, hipStream_t s)
{
    constexpr int V = SeqElem<T>::V;
    const SeqView &v = bwd ? a.vr : a.vx;
    if (v.c == V || a.L == 1) {
        if (bwd && a.rows >= 8LL * a.parts && a.Cb <= 8 * 64)
            return a.Cb <= 64 ? launch_alone<T, 1>(a, s) : a.Cb <= 2 * 64 ? launch_alone<T, 2>(a, s) : a.Cb <= 4 * 64 ? launch_alone<T, 4>(a, s) : launch_alone<T, 8>(a, s);
        return launch_lt<T, 1>(bwd, a, s);
    }
    return bwd || a.rows < 16 * 512 ? launch_lt<T, 8>(bwd, a, s) : launch_lt<T, 16>(bwd, a, s);
}
}  // namespace

hipError_t launch_seq_lnorm_fwd(int dtype, const SeqNormArgs &a, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch_t<unsigned short>(false, a, s) : launch_t<float>(false, a, s);
}
hipError_t launch_seq_lnorm_bwd(int dtype, const SeqNormArgs &a, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch_t<unsigned short>(true, a, s) : launch_t<float>(true, a, s);
}

}  // namespace convmi
