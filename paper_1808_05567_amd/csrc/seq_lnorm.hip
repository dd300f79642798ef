// Layer norm with the residual's addition, forward (result in the tensors' type or in 8 bits) and backward.
//
//   r = x + res,   u = (r - mean r) rstd,   y = u w + b,   rstd = 1 / sqrt(mean (r - mean r)^2 + eps)
//   dx = dr + rstd (w dy - mean(w dy) - u mean(w dy u)),   dw = sum dy u,   db = sum dy
//
// As the root-mean-square norm: a workgroup holds whole positions in registers between the sums over their channels and the result.  Squares are of
// differences from a mean, so that one far from zero costs nothing of the variance: each wave has the mean m_w of its own n_w channels and sums about that,
//   q_w = sum (r - m_w)^2,  and backwards  G_w = sum w dy,  p_w = sum w dy (r - m_w),
// which the workgroup joins in one exchange:  mean = sum n_w m_w / C,  sum (r - mean)^2 = sum q_w + n_w (m_w - mean)^2,
//   sum w dy (r - mean) = sum p_w + G_w (m_w - mean).
// A few operations an element: bound by memory.  Measured, 8 x 2048 positions of 2048 channels in bf16, 268 MB: forward 58 us (4.6 TB/s; positions side by side 51),
// backward 70 (3.8 TB/s; 71), of which 5 are the sums of dw and db over the workgroups; 3 x 333 positions of 1000 fp32 channels side by side, 12 MB: backward 9 and 4;
// 16 x 4096 to 8 bits 5.4.
#include <algorithm>
#include <type_traits>

#include "seq_internal.h"

namespace convmi {
namespace {

constexpr int kMaxThreads = 1024, kAloneWaves = 4, kParts = 512;
// Forwards, inputs of more bytes than this are read past the caches, as results are written: with their results they are more than the last one of 256 MB holds (positions of 2048 bf16
// channels, three sets of tensors in turn: 67 MB 61.5 -> 58.5 us, 50 MB 48.4 -> 46.8, but 42 MB 36.5 -> 41.9).  Backwards they are wherever results are (67 MB 73 -> 70.6, 42 MB 49.5 -> 46.9,
// 33 MB 37.0 -> 36.7).
constexpr long long kOnceBytes = 48LL << 20;

// Sums (MAX: largest unsigned) of K numbers over the lanes of a wave with the same place in a tile of LT positions, in all of them.
template <int LT, bool MAX, int K>
static __device__ __forceinline__ void wave_sums(float (&v)[K])
{
    auto join = [](float p, float q) { return MAX ? __uint_as_float(max(__float_as_uint(p), __float_as_uint(q))) : p + q; };
    auto turn = [](float p, auto by) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(p), 0x120 + decltype(by)::value, 0xf, 0xf, true)); };
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
}

// Channels of a position that wave w has: of blocks w * 64 / LT ... and of those `step` blocks on, and so forth.
template <int LT, int V>
static __device__ __forceinline__ float channels_of(const SeqNormArgs &a, int w, int step)
{
    int n = 0;
    for (int b = w * (64 / LT); b < a.Cb; b += step) n += min(max(a.C - b * V, 0), 64 / LT * V);
    return (float)n;
}

// A position's sums from those of its waves, all four of them in each wave's lanes in the same order.  lds: not that of the exchange before, which some wave may
// still read.  in: mean, q and, backwards, G, p; out: mean, sum of squares and, backwards, sum of w dy, sum of w dy (r - mean).
template <int LT, bool BWD, int V>
static __device__ __forceinline__ void join_waves(const SeqNormArgs &a, seq_f32x4 &sums, seq_f32x4 *lds)
{
    constexpr int EACH = (kMaxThreads / 64 + 64 / LT - 1) / (64 / LT), K = BWD ? 2 : 1;
    const int waves = blockDim.x / 64, wave = threadIdx.x / 64, at = threadIdx.x % LT, bl = threadIdx.x % 64 / LT, step = blockDim.x / LT;
    if (threadIdx.x % 64 < LT) lds[wave * LT + at] = sums;
    __syncthreads();
    seq_f32x4 e[EACH];
    float n[EACH], t[K] = {}, u[K] = {};
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int w = bl + i * (64 / LT);
        e[i] = seq_f32x4{};
        n[i] = 0;
        if (w < waves) {
            e[i] = lds[w * LT + at];
            n[i] = channels_of<LT, V>(a, w, step);
        }
        t[0] = fmaf(n[i], e[i][0], t[0]);
        if constexpr (BWD) t[1] += e[i][2];
    }
    wave_sums<LT, false>(t);
    const float mean = t[0] / a.C;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const float d = e[i][0] - mean;
        u[0] += n[i] == 0 ? 0.0f : fmaf(n[i] * d, d, e[i][1]);
        if constexpr (BWD) u[1] += n[i] == 0 ? 0.0f : fmaf(e[i][2], d, e[i][3]);
    }
    wave_sums<LT, false>(u);
    sums = seq_f32x4{mean, u[0], BWD ? t[1] : 0.0f, BWD ? u[1] : 0.0f};
}

// ONCE: what no one reads again does not stay in the caches.
template <bool ONCE, typename T>
static __device__ __forceinline__ seq_u32x4 load_once(const T *p)
{
    if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const seq_u32x4 *>(p));
    return seq_load(p);
}

// What is unpacked from b behind this is unpacked again, rather than kept in registers from before, where it takes twice as many.
static __device__ __forceinline__ void again_from(seq_u32x4 &b) { asm volatile("" : "+v"(b)); }

// Where a position lies, and whether it is inside its sequence; what is behind its end comes out as zero.
template <typename T>
struct Place {
    bool live, inside;
    int n, l;
    __device__ __forceinline__ Place(const SeqNormArgs &a, long long row)
    {
        live = row < a.rows;  // (which 31 bits hold)
        n = live ? (int)((unsigned)row / (unsigned)a.L) : 0;
        l = live ? (int)((unsigned)row - (unsigned)n * (unsigned)a.L) : 0;
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
template <typename T, int LT, int NV, bool Q8, bool PAST, bool ONCE>
__global__ __launch_bounds__(kMaxThreads) void seq_lnorm_fwd_kernel(const SeqNormArgs a)
{
    constexpr int V = SeqElem<T>::V;
    __shared__ seq_f32x4 lds[2][kMaxThreads / 64 * LT];
    __shared__ float largest_of[Q8 ? kMaxThreads / 64 * LT : 1];
    const float channels = channels_of<LT, V>(a, threadIdx.x / 64, blockDim.x / LT);
    int turn = 0;
    for (long long tile = blockIdx.x; tile * LT < a.rows; tile += gridDim.x) {
        const long long row = tile * LT + threadIdx.x % LT;
        const Place<T> at(a, row);
        const int first = threadIdx.x / LT, step = blockDim.x / LT;
        const T *x = static_cast<const T *>(a.x) + at.n * a.vx.n + at.l * a.vx.l;
        const T *res = a.res ? static_cast<const T *>(a.res) + at.n * a.vres.n + at.l * a.vres.l : nullptr;
        T *r = a.r ? static_cast<T *>(a.r) + at.n * a.vr.n + at.l * a.vr.l : nullptr;
        auto added = [](const seq_u32x4 &p, const seq_u32x4 &q) {
            float f[V], g[V];
            SeqElem<T>::unpack(p, f);
            SeqElem<T>::unpack(q, g);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] += g[i];
            return SeqElem<T>::pack(f);
        };
        // (a position behind its sequence's end: zeros, whatever x and res hold)
        auto sum_of = [&](int b) {
            if (!at.inside) return seq_u32x4{};
            const seq_u32x4 p = seq_load(x + b * a.vx.c);
            return res ? added(p, seq_load(res + b * a.vres.c)) : p;
        };
        auto first_time = [&](int b) {
            const seq_u32x4 p = sum_of(b);
            if (r) seq_store(r + b * a.vr.c, p);
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
        if constexpr (NV > 0) {
            // all of it is asked for before any r is stored, which may lie in x's or res's place
            seq_u32x4 more[NV];
            over([&](int j, int b) {
                keep[j] = more[j] = seq_u32x4{};
                if (!at.inside) return;
                keep[j] = load_once<ONCE>(x + b * a.vx.c);
                if (res) more[j] = load_once<ONCE>(res + b * a.vres.c);
            });
            over([&](int j, int b) {
                if (res) keep[j] = added(keep[j], more[j]);
                if (r) seq_store_result<PAST>(r + b * a.vr.c, keep[j]);
            });
        }
        over([&](int j, int b) {
            float f[V];
            if constexpr (NV > 0)
                SeqElem<T>::unpack(keep[j], f);
            else
                SeqElem<T>::unpack(first_time(b), f);
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += f[i];
        });
        wave_sums<LT, false>(s);
        const float own = s[0] / fmaxf(channels, 1.0f);
        s[0] = 0;
        auto difference = [&](int j, int b, float mean, float (&f)[V]) {
            if constexpr (NV > 0) again_from(keep[j]);
            SeqElem<T>::unpack(again(j, b), f);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] -= mean;
            clear_beyond<V>(a, b, f);
        };
        over([&](int j, int b) {
            float f[V];
            difference(j, b, own, f);
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] = fmaf(f[i], f[i], s[0]);
        });
        wave_sums<LT, false>(s);
        seq_f32x4 sums = {own, s[0], 0, 0};
        if (blockDim.x > 64) join_waves<LT, false, V>(a, sums, lds[turn]);
        turn ^= 1;
        const float mean = sums[0], rstd = 1.0f / sqrtf(sums[1] / a.C + a.eps);
        auto norm = [&](int j, int b, float (&f)[V]) {
            float w[V], c[V] = {};
            difference(j, b, mean, f);
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
            wave_sums<LT, true>(m);
            if (blockDim.x > 64) {
                // (between two of these lies the exchange of the sums)
                if (threadIdx.x % 64 < LT) largest_of[threadIdx.x / 64 * LT + threadIdx.x % LT] = m[0];
                __syncthreads();
                for (int w = 0; w < (int)blockDim.x / 64; ++w) m[0] = __uint_as_float(max(__float_as_uint(m[0]), __float_as_uint(largest_of[w * LT + threadIdx.x % LT])));
            }
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
// What the next positions need is asked for before these are worked on: a compute unit holds one workgroup of 16 waves.
template <typename T, int LT, int NV, bool ALONE, bool PAST>
__global__ __launch_bounds__(ALONE ? 64 * kAloneWaves : kMaxThreads) void seq_lnorm_bwd_kernel(const SeqNormArgs a)
{
    static_assert(!ALONE || LT == 1, "one position a wave");
    constexpr int V = SeqElem<T>::V, NK = NV ? NV : 1;
    __shared__ seq_f32x4 lds[2][kMaxThreads / 64 * LT];
    constexpr bool SHARED = LT > 1 && NV > 0;  // w lies in LDS, where lanes share it
    __shared__ __align__(16) float lw[SHARED ? kMaxThreads / LT * NV * V : 4];
    const int first = ALONE ? threadIdx.x % 64 : threadIdx.x / LT, step = ALONE ? 64 : blockDim.x / LT;
    const int waves = blockDim.x / 64, each = ALONE ? waves : LT;  // positions of a workgroup at a time
    float *part = a.part + (long long)blockIdx.x * 2 * a.Cp;
    float dw[NK][V] = {}, db[NK][V] = {}, kw[SHARED ? 1 : NK][V];
    if constexpr (SHARED) {
        for (int c = threadIdx.x; c < a.Cp; c += blockDim.x) lw[c] = a.w[c];
        __syncthreads();
    } else if constexpr (NV > 0) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (first + j * step < a.Cb) seq_vector<V>(a.w, first + j * step, kw[j]);
    }
    auto weights = [&](int j, int b, float (&w)[V]) {
        if constexpr (SHARED)
            seq_vector<V>(lw, b, w);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] = kw[j][i];
    };
    const float channels = channels_of<LT, V>(a, ALONE ? 0 : threadIdx.x / 64, step);
    int turn = 0;
    struct Blocks {
        seq_u32x4 r[NK], dy[NK];
    } now, next;
    seq_u32x4 now_dr[NK];
    auto place = [&](long long tile) { return Place<T>(a, tile * each + (ALONE ? threadIdx.x / 64 : threadIdx.x % LT)); };
    // where a position's first block of a thread lies; the others are the same distances on for all threads
    auto where = [&](const void *p, const SeqView &v, const Place<T> &at) { return static_cast<const T *>(p) + at.n * v.n + at.l * v.l + first * v.c; };
    auto load_all = [&](const Place<T> &at, Blocks &k) {
        const T *r = where(a.r, a.vr, at), *dy = where(a.dy, a.vdy, at);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            k.r[j] = k.dy[j] = seq_u32x4{};
            if (!at.inside || first + j * step >= a.Cb) continue;
            k.r[j] = load_once<PAST>(r + j * (step * a.vr.c));
            k.dy[j] = load_once<PAST>(dy + j * (step * a.vdy.c));
        }
    };
    // (dr is needed last: it is asked for when these positions' sums begin)
    auto load_dr = [&](const Place<T> &at) {
        const T *dr = a.dr ? where(a.dr, a.vdr, at) : nullptr;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            now_dr[j] = seq_u32x4{};
            if (dr && at.inside && first + j * step < a.Cb) now_dr[j] = load_once<PAST>(dr + j * (step * a.vdr.c));
        }
    };
    if constexpr (NV > 0) load_all(place(blockIdx.x), next);
    for (long long tile = blockIdx.x; tile * each < a.rows; tile += gridDim.x) {
        const Place<T> at = place(tile);
        auto over = [&](auto &&body) {
            if constexpr (NV > 0) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (at.live && first + j * step < a.Cb) body(j, first + j * step);
            } else if (at.live)
                for (int b = first; b < a.Cb; b += step) {
                    now.r[0] = now.dy[0] = now_dr[0] = seq_u32x4{};
                    if (at.inside) {
                        now.r[0] = seq_load(static_cast<const T *>(a.r) + at.n * a.vr.n + at.l * a.vr.l + b * a.vr.c);
                        now.dy[0] = seq_load(static_cast<const T *>(a.dy) + at.n * a.vdy.n + at.l * a.vdy.l + b * a.vdy.c);
                        if (a.dr) now_dr[0] = seq_load(static_cast<const T *>(a.dr) + at.n * a.vdr.n + at.l * a.vdr.l + b * a.vdr.c);
                    }
                    seq_vector<V>(a.w, b, kw[0]);
                    body(0, b);
                }
        };
        if constexpr (NV > 0) {
            now = next;
            load_dr(at);
            load_all(place(tile + gridDim.x), next);
        }
        float s[2] = {};
        over([&](int j, int b) {
            float f[V], g[V], w[V];
            SeqElem<T>::unpack(now.r[j], f);
            SeqElem<T>::unpack(now.dy[j], g);
            weights(j, b, w);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[0] += f[i];
                s[1] = fmaf(g[i], w[i], s[1]);
            }
        });
        wave_sums<LT, false>(s);
        const float own = s[0] / fmaxf(channels, 1.0f), own_dy = s[1];
        s[0] = s[1] = 0;
        auto difference = [&](int j, int b, float mean, float (&f)[V], float (&g)[V]) {
            again_from(now.r[j]);
            again_from(now.dy[j]);
            SeqElem<T>::unpack(now.r[j], f);
            SeqElem<T>::unpack(now.dy[j], g);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] -= mean;
            clear_beyond<V>(a, b, f);
        };
        over([&](int j, int b) {
            float f[V], g[V], w[V];
            difference(j, b, own, f, g);
            weights(j, b, w);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[0] = fmaf(f[i], f[i], s[0]);
                s[1] = fmaf(f[i], g[i] * w[i], s[1]);
            }
        });
        wave_sums<LT, false>(s);
        seq_f32x4 sums = {own, s[0], own_dy, s[1]};
        if (!ALONE && blockDim.x > 64) join_waves<LT, true, V>(a, sums, lds[turn]);
        turn ^= 1;
        const float mean = sums[0], rstd = 1.0f / sqrtf(sums[1] / a.C + a.eps), through = sums[2] / a.C, along = sums[3] / a.C * rstd * rstd;
        T *dx = const_cast<T *>(where(a.dx, a.vdx, at));
        over([&](int j, int b) {
            float f[V], g[V], d[V], w[V];
            difference(j, b, mean, f, g);
            SeqElem<T>::unpack(now_dr[j], d);
            weights(j, b, w);
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
            seq_store_result<PAST>(NV > 0 ? dx + j * (step * a.vdx.c) : dx + (b - first) * a.vdx.c, SeqElem<T>::pack(d));
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
        __shared__ float sums[kAloneWaves][64 * V];
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

template <typename T, int LT, int NV>
hipError_t launch_fwd(const SeqNormArgs &a, int threads, hipStream_t s)
{
    const long long tiles = (a.rows + LT - 1) / LT;
    const unsigned grid = (unsigned)(tiles < 1 << 21 ? tiles : 1 << 21);  // (of 1024 threads: a launch has less than 2^32)
    if (a.q)
        seq_lnorm_fwd_kernel<T, LT, NV, true, false, false><<<grid, threads, 0, s>>>(a);
    else if (a.rows * a.Cb * 16 > kOnceBytes)
        seq_lnorm_fwd_kernel<T, LT, NV, false, true, true><<<grid, threads, 0, s>>>(a);
    else if (a.past)
        seq_lnorm_fwd_kernel<T, LT, NV, false, true, false><<<grid, threads, 0, s>>>(a);
    else
        seq_lnorm_fwd_kernel<T, LT, NV, false, false, false><<<grid, threads, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, int LT, int NV, bool ALONE>
hipError_t launch_bwd(const SeqNormArgs &a, int threads, hipStream_t s)
{
    // parts of dw and db: as many as there are workgroups at a time, but 512 where each of 1024 would have less than 8 tiles (8 x 2048 positions of 2048 bf16 channels side by
    // side: 512 of them 85 us, 1024 71; 8 x 8000 of 300 fp32, a wave each, 92 and 72; 3 x 333 of 1000 fp32 11.3 and 14.0)
    const long long each = ALONE ? kAloneWaves : LT, tiles = (a.rows + each - 1) / each;
    const long long most = threads > 512 ? kParts / 2 : threads <= 256 && tiles >= 16LL * kParts ? 2 * kParts : kParts;
    const unsigned parts = (unsigned)std::min<long long>(std::min<long long>(most, a.parts), tiles);
    if (a.past)
        seq_lnorm_bwd_kernel<T, LT, NV, ALONE, true><<<parts, threads, 0, s>>>(a);
    else
        seq_lnorm_bwd_kernel<T, LT, NV, ALONE, false><<<parts, threads, 0, s>>>(a);
    seq_lnorm_reduce_kernel<<<(2 * a.Cp + kSumColumns - 1) / kSumColumns, 1024, 0, s>>>(a.part, a.dw, a.db, (int)parts, a.Cp);
    return hipGetLastError();
}

// Threads of a workgroup and blocks that each holds: up to 4 forwards, 2 backwards, whose sums of dw and db take 16 registers a bf16 block, so that
// four waves a SIMD have their registers; from 256 threads on if that takes fewer blocks, and a block each where positions are few (16 x 4096 bf16 to 8 bits: 6.5 -> 5.4 us).  LT positions that do not fit 1024 threads go as fewer at a time; what one
// position does not fit is read again.
template <typename T, int LT, bool BWD>
hipError_t launch_lt(const SeqNormArgs &a, hipStream_t s)
{
    constexpr int MOST = BWD ? 2 : 4;
    const long long lanes = (long long)a.Cb * LT;
    int threads = 64;
    while (threads < (a.rows <= 512 ? kMaxThreads : 256) && threads < lanes) threads *= 2;
    while (threads < kMaxThreads && threads * MOST < lanes) threads *= 2;
    const long long nv = (lanes + threads - 1) / threads;
    if constexpr (BWD) {
        if (nv <= 1) return launch_bwd<T, LT, 1, false>(a, threads, s);
        if (nv <= 2) return launch_bwd<T, LT, 2, false>(a, threads, s);
    } else {
        if (nv <= 1) return launch_fwd<T, LT, 1>(a, threads, s);
        if (nv <= 2) return launch_fwd<T, LT, 2>(a, threads, s);
        if (nv <= 4) return launch_fwd<T, LT, 4>(a, threads, s);
    }
    if constexpr (LT > 1)
        return launch_lt<T, LT / 2, BWD>(a, s);
    else if constexpr (BWD)
        return launch_bwd<T, 1, 0, false>(a, threads, s);
    else
        return launch_fwd<T, 1, 0>(a, threads, s);
}
template <typename T, bool BWD>
hipError_t launch_t(const SeqNormArgs &a, hipStream_t s)
{
    // one position at a time where its blocks follow one another in what is read; else eight, forwards sixteen where that leaves two
    // workgroups for each compute unit
    constexpr int V = SeqElem<T>::V;
    const SeqView &v = BWD ? a.vr : a.vx;
    if (v.c == V || a.L == 1) {
        // a wave each where that leaves every workgroup two for each of its waves and 16 channels a lane do (8 x 1024 x 1024 fp32, workgroups of one position:
        // 35 us, this 27; 999 x 1000 take 13 either way)
        if constexpr (BWD) {
            if (a.rows >= 2LL * kAloneWaves * kParts && a.Cb <= 64 * 16 / V) {
                if (a.Cb <= 64) return launch_bwd<T, 1, 1, true>(a, 64 * kAloneWaves, s);
                if (a.Cb <= 2 * 64) return launch_bwd<T, 1, 2, true>(a, 64 * kAloneWaves, s);
                if constexpr (V == 4) return launch_bwd<T, 1, 4, true>(a, 64 * kAloneWaves, s);
            }
        }
        return launch_lt<T, 1, BWD>(a, s);
    }
    if constexpr (!BWD) {
        if (a.rows >= 16 * 512) return launch_lt<T, 16, false>(a, s);
    }
    return launch_lt<T, 8, BWD>(a, s);
}
}  // namespace

hipError_t launch_seq_lnorm_fwd(int dtype, const SeqNormArgs &a, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch_t<unsigned short, false>(a, s) : launch_t<float, false>(a, s);
}
hipError_t launch_seq_lnorm_bwd(int dtype, const SeqNormArgs &a, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch_t<unsigned short, true>(a, s) : launch_t<float, true>(a, s);
}

}  // namespace convmi
