// Gradients of the selective scan.  With g[l] the gradient of the state after position l, back to front,
//
//   g[l] = C dy + exp(d+ A) g+,   dC = sum_c dy h,   dB = sum_c g d x,   dx = D dy + d sum_s g B,
//   dd = sum_s (A t + g B x),   dA = sum d t,   t = g exp(d A) h[l-1]
//
// (dy that of y before the gate.)  The states are formed again rather than kept: positions go in runs of 64.  A first launch finds
// what each run does to a state and to a gradient, a second puts these together, so that a run knows the state before it and the gradient
// behind it.  A wave then goes through its run forwards, noting the state in LDS every 8 positions, and through these
// eights from the back: forwards again with the 8 states in registers, then backwards.
//
// A thread takes 4 channels x 4 states: half of the sums over states and over channels stay inside it; those over states end in
// a quad of lanes, those over channels in exchanges that halve what is left each time.
// Some 20 operations and three exponentials a state and position: bound by the vector units.
#include "seq_internal.h"

namespace convmi {
namespace {

constexpr int kT = 8;  // positions held at a time

// Which way an eight is staged for.
struct Forward {
    static constexpr bool value = false;
};
struct Back {
    static constexpr bool value = true;
};

// Sum over the NL lanes that hold the states of the same channels.
template <int NL>
static __device__ __forceinline__ float sum_states(float x)
{
    x = seq_add_lane<0xB1>(x);                         // lane ^ 1
    if constexpr (NL >= 4) x = seq_add_lane<0x4E>(x);  // lane ^ 2
    if constexpr (NL >= 8) x = seq_add_lane<0x141>(x); // 7 - lane, within eights
    if constexpr (NL >= 16) x = seq_add_lane<0x140>(x);  // 15 - lane, within sixteens
    return x;
}
// p: sums over halves of the wave, those of p in the lower half, of q in the upper one.
static __device__ __forceinline__ float swap32(float p, float q)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(p), __float_as_uint(q), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// ... over pairs of rows of 16, those of p in the even one, of q in the odd one.
static __device__ __forceinline__ float swap16(float p, float q)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(p), __float_as_uint(q), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Sum over the lanes of a row that hold the same states of different channels.
template <int NL>
static __device__ __forceinline__ float sum_row(float x)
{
    if constexpr (NL <= 8) x = seq_add_lane<0x128>(x);  // 8 lanes on
    if constexpr (NL <= 4) x = seq_add_lane<0x124>(x);
    if constexpr (NL <= 2) x = seq_add_lane<0x122>(x);
    return x;
}

template <typename T, int SP>
__global__ __launch_bounds__(64) void seq_scan_bwd_kernel(const SeqScanArgs a)
{
    constexpr int V = SeqElem<T>::V, NL = SP / 4, WC = seq_scan_bwd_channels(SP), NSUB = kSeqBwdChunk / kT;
    constexpr int VEC = WC / V * kT, NV = (VEC + 63) / 64;
    __shared__ __align__(16) float marks[NSUB - 1][4][64][4];  // the states at the start of eights 1 ... 7
    // d, x, dy of the eight; once used, what the sums over states were: A t, g B, C h
    __shared__ __align__(16) float sd[kT][WC], sx[kT][WC], sg[kT][WC];
    __shared__ __align__(16) float sB[kT][SP], sC[kT][SP];
    const int lane = threadIdx.x, sl = lane % NL, cl = lane / NL;
    int t = blockIdx.x;
    const int chunk = t % a.chunks;
    t /= a.chunks;
    const int g = t % a.G, tl = t / a.G % a.btiles, n = t / a.G / a.btiles;
    const int c0 = g * a.CG + tl * WC, c_end = min(c0 + WC, (g + 1) * a.CG);
    const int len = seq_length(a.lengths, n, a.L);
    const int begin = chunk * kSeqBwdChunk, end = min(begin + kSeqBwdChunk, a.L), stop = min(end, len);
    const int eights = stop > begin ? (stop - begin + kT - 1) / kT : 0;

    // element-wise: block cbl, position ll of an eight
    bool in[NV];
    int ll[NV], cb[NV], to[NV];
    float D[NV][V], bias[NV][V], aD[NV][V] = {}, ab[NV][V] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = lane + 64 * i, cbl = e / kT;
        ll[i] = e % kT;
        in[i] = e < VEC && c0 + cbl * V < c_end;
        cb[i] = c0 / V + (in[i] ? cbl : 0);
        to[i] = e < VEC ? cbl * V : 0;
#pragma unroll
        for (int j = 0; j < V; ++j) D[i][j] = bias[i][j] = 0;
        if (a.D) seq_vector<V>(a.D, cb[i], D[i]);
        if (a.dt_bias) seq_vector<V>(a.dt_bias, cb[i], bias[i]);
    }
    auto block = [&](const void *p, const SeqView &v, int i, int l) {
        return seq_load(static_cast<const T *>(p) + n * v.n + cb[i] * v.c + l * v.l);
    };
    auto put = [&](void *p, const SeqView &v, int i, int l, const float (&f)[V]) {
        seq_store(static_cast<T *>(p) + n * v.n + cb[i] * v.c + l * v.l, SeqElem<T>::pack(f));
    };

    // scan-wise: channels c ... + 3, states s ... + 3
    const int c = c0 + cl * 4, s = sl * 4;
    const bool live = c < c_end;
    const long long at = ((long long)n * a.chunks + chunk) * a.S * a.Cp + (live ? c : c0);
    float A[4][4], h[4][4], carry[4][4], dA[4][4] = {};  // [state][channel]
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        seq_f32x4 q = {}, p = {}, r = {};
        if (live && s + j < a.S) {
            q = *reinterpret_cast<const seq_f32x4 *>(a.A + (long long)(s + j) * a.Cp + c);
            if (a.chunks > 1) {
                p = *reinterpret_cast<const seq_f32x4 *>(a.hl + at + (long long)(s + j) * a.Cp);
                r = *reinterpret_cast<const seq_f32x4 *>(a.gl + at + (long long)(s + j) * a.Cp);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // (channels beyond the last one take no part, whatever their parameters hold)
            const bool ok = c + i < c_end;
            A[j][i] = ok ? q[i] * kLog2e : 0.0f;
            h[j][i] = ok ? p[i] : 0.0f;
            carry[j][i] = ok ? r[i] : 0.0f;
        }
    }

    float kx[NV][V], kd[NV][V], ksig[NV][V], kg[NV][V], kz[NV][V];
    // loads the eight at l0 and puts it in LDS; BACK: with all that the way back needs
    auto stage = [&](int l0, auto back) {
        constexpr bool BACK = decltype(back)::value;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int l = l0 + ll[i];
#pragma unroll
            for (int j = 0; j < V; ++j) kx[i][j] = kd[i][j] = ksig[i][j] = kg[i][j] = kz[i][j] = 0;
            if (in[i] && l < stop) {
                float raw[V], gate[V], z[V];
                SeqElem<T>::unpack(block(a.x, a.vx, i, l), kx[i]);
                SeqElem<T>::unpack(block(a.dt, a.vdt, i, l), raw);
                if (BACK) {
                    SeqElem<T>::unpack(block(a.dy, a.vdy, i, l), kg[i]);
                    if (a.z) SeqElem<T>::unpack(block(a.z, a.vz, i, l), z);
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float r = raw[j] + bias[i][j];
                    kd[i][j] = a.softplus ? seq_softplus(r) : r;
                    if (BACK) {
                        ksig[i][j] = a.softplus ? seq_sigmoid(r) : 1.0f;
                        if (a.z) {
                            const float p = seq_sigmoid(z[j]);
                            kz[i][j] = kg[i][j] * p * (1.0f + z[j] * (1.0f - p));
                            kg[i][j] *= z[j] * p;
                        }
                    }
                    if (cb[i] * V + j >= a.Ch) kx[i][j] = kd[i][j] = kg[i][j] = kz[i][j] = 0;
                }
            }
            if (lane + 64 * i < VEC)
#pragma unroll
                for (int j = 0; j < V; j += 4) {
                    *reinterpret_cast<seq_f32x4 *>(&sd[ll[i]][to[i] + j]) = seq_f32x4{kd[i][j], kd[i][j + 1], kd[i][j + 2], kd[i][j + 3]};
                    *reinterpret_cast<seq_f32x4 *>(&sx[ll[i]][to[i] + j]) = seq_f32x4{kx[i][j], kx[i][j + 1], kx[i][j + 2], kx[i][j + 3]};
                    if (BACK) *reinterpret_cast<seq_f32x4 *>(&sg[ll[i]][to[i] + j]) = seq_f32x4{kg[i][j], kg[i][j + 1], kg[i][j + 2], kg[i][j + 3]};
                }
        }
#pragma unroll
        for (int i = lane; i < kT * SP; i += 64) {
            const int l = l0 + i / SP, st = i % SP, e = g * a.S + st;
            const bool ok = l < stop && st < a.S;
            sB[i / SP][st] = ok ? SeqElem<T>::get(static_cast<const T *>(a.B)[n * a.vB.n + e / V * a.vB.c + l * a.vB.l + e % V]) : 0.0f;
            if (BACK) sC[i / SP][st] = ok ? SeqElem<T>::get(static_cast<const T *>(a.C)[n * a.vC.n + e / V * a.vC.c + l * a.vC.l + e % V]) : 0.0f;
        }
        __syncthreads();
    };
    for (int e = 0; e + 1 < eights; ++e) {
        stage(begin + e * kT, Forward());
#pragma unroll
        for (int l = 0; l < kT; ++l) {
            const seq_f32x4 d = *reinterpret_cast<const seq_f32x4 *>(&sd[l][cl * 4]), x = *reinterpret_cast<const seq_f32x4 *>(&sx[l][cl * 4]);
            const seq_f32x4 B = *reinterpret_cast<const seq_f32x4 *>(&sB[l][s]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float dx = d[i] * x[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) h[j][i] = fmaf(seq_exp2(d[i] * A[j][i]), h[j][i], B[j] * dx);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) *reinterpret_cast<seq_f32x4 *>(marks[e][j][lane]) = seq_f32x4{h[j][0], h[j][1], h[j][2], h[j][3]};
    }

    for (int e = eights - 1; e >= 0; --e) {
        const int l0 = begin + e * kT;
        stage(l0, Back());
        float hs[kT + 1][4][4], as[kT][4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            seq_f32x4 p = {};
            if (e > 0)
                p = *reinterpret_cast<const seq_f32x4 *>(marks[e - 1][j][lane]);
            else if (live && s + j < a.S && a.chunks > 1)
                p = *reinterpret_cast<const seq_f32x4 *>(a.hl + at + (long long)(s + j) * a.Cp);
#pragma unroll
            for (int i = 0; i < 4; ++i) hs[0][j][i] = c + i < c_end ? p[i] : 0.0f;
        }
#pragma unroll
        for (int l = 0; l < kT; ++l) {
            const seq_f32x4 d = *reinterpret_cast<const seq_f32x4 *>(&sd[l][cl * 4]), x = *reinterpret_cast<const seq_f32x4 *>(&sx[l][cl * 4]);
            const seq_f32x4 B = *reinterpret_cast<const seq_f32x4 *>(&sB[l][s]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float dx = d[i] * x[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    as[l][j][i] = seq_exp2(d[i] * A[j][i]);
                    hs[l + 1][j][i] = fmaf(as[l][j][i], hs[l][j][i], B[j] * dx);
                }
            }
        }
#pragma unroll
        for (int l = kT - 1; l >= 0; --l) {
            const seq_f32x4 d = *reinterpret_cast<const seq_f32x4 *>(&sd[l][cl * 4]), x = *reinterpret_cast<const seq_f32x4 *>(&sx[l][cl * 4]);
            const seq_f32x4 dy = *reinterpret_cast<const seq_f32x4 *>(&sg[l][cl * 4]);
            const seq_f32x4 B = *reinterpret_cast<const seq_f32x4 *>(&sB[l][s]), C = *reinterpret_cast<const seq_f32x4 *>(&sC[l][s]);
            float bc[8] = {};  // dB, dC of the four states
            seq_f32x4 gB = {}, At = {}, Ch = {};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float dx = d[i] * x[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float gr = fmaf(dy[i], C[j], carry[j][i]);
                    bc[4 + j] = fmaf(dy[i], hs[l + 1][j][i], bc[4 + j]);
                    bc[j] = fmaf(gr, dx, bc[j]);
                    gB[i] = fmaf(gr, B[j], gB[i]);
                    Ch[i] = fmaf(C[j], hs[l + 1][j][i], Ch[i]);
                    carry[j][i] = gr * as[l][j][i];
                    const float th = carry[j][i] * hs[l][j][i];
                    dA[j][i] = fmaf(th, d[i], dA[j][i]);
                    At[i] = fmaf(th, A[j][i], At[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                gB[i] = sum_states<NL>(gB[i]);
                At[i] = sum_states<NL>(At[i]);
                if (a.z) Ch[i] = sum_states<NL>(Ch[i]);
            }
            if (sl == 0) {
                *reinterpret_cast<seq_f32x4 *>(&sd[l][cl * 4]) = At;
                *reinterpret_cast<seq_f32x4 *>(&sx[l][cl * 4]) = gB;
                if (a.z) *reinterpret_cast<seq_f32x4 *>(&sg[l][cl * 4]) = Ch;
            }
            float u[4], v[2];
#pragma unroll
            for (int j = 0; j < 4; ++j) u[j] = swap32(bc[j], bc[j + 4]);
#pragma unroll
            for (int j = 0; j < 2; ++j) v[j] = sum_row<NL>(swap16(u[j], u[j + 2]));
            // the lower half of the wave has dB, the upper one dC; even rows states s, s + 1, odd ones s + 2, s + 3
            if (lane % 16 < NL && l0 + l < stop) {
                const int st = lane % 16 * 4 + lane / 16 % 2 * 2;
                float *bp = a.bc + (((long long)n * a.L + l0 + l) * (a.G * a.btiles) + g * a.btiles + tl) * 2 * a.S + lane / 32 * a.S + st;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (st + j < a.S) bp[j] = v[j];
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int l = l0 + ll[i];
            if (!in[i] || l >= end) continue;
            float dx[V], ddt[V], dz[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float At = sd[ll[i]][to[i] + j], gB = sx[ll[i]][to[i] + j];
                dx[j] = fmaf(D[i][j], kg[i][j], kd[i][j] * gB);
                ddt[j] = fmaf(kLn2, At, kx[i][j] * gB) * ksig[i][j];
                if (a.z) dz[j] = kz[i][j] * fmaf(D[i][j], kx[i][j], sg[ll[i]][to[i] + j]);
                if (cb[i] * V + j >= a.Ch) ddt[j] = dx[j] = dz[j] = 0;
                aD[i][j] = fmaf(kg[i][j], kx[i][j], aD[i][j]);
                ab[i][j] += ddt[j];
            }
            put(a.dx, a.vdx, i, l, dx);
            put(a.ddt, a.vddt, i, l, ddt);
            if (a.z) put(a.dz, a.vdz, i, l, dz);
        }
    }
    // zeros past the end
    const float zero[V] = {};
    for (int l0 = begin + eights * kT; l0 < end; l0 += kT)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!in[i] || l0 + ll[i] >= end) continue;
            put(a.dx, a.vdx, i, l0 + ll[i], zero);
            put(a.ddt, a.vddt, i, l0 + ll[i], zero);
            if (a.z) put(a.dz, a.vdz, i, l0 + ll[i], zero);
        }
    // this run's part of the parameters' gradients; that of A where its state was
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (live && s + j < a.S) *reinterpret_cast<seq_f32x4 *>(a.hl + at + (long long)(s + j) * a.Cp) = seq_f32x4{dA[j][0], dA[j][1], dA[j][2], dA[j][3]};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float p = aD[i][j], q = ab[i][j];
#pragma unroll
            for (int d = 1; d < kT; d *= 2) {
                p += __shfl_xor(p, d);
                q += __shfl_xor(q, d);
            }
            if (in[i] && ll[i] == 0) {
                float *v = a.vec + ((long long)n * a.chunks + chunk) * 2 * a.Cp + cb[i] * V + j;
                v[0] = p;
                v[a.Cp] = q;
            }
        }
}

// dB and dC: the tiles' parts of a position in order; one thread a result.
template <typename T>
__global__ __launch_bounds__(256) void seq_scan_bc_kernel(const SeqScanArgs a)
{
    constexpr int V = SeqElem<T>::V;
    const int Sp = (a.G * a.S + V - 1) / V * V;
    const long long total = (long long)a.N * a.L * 2 * Sp;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < total; t += (long long)gridDim.x * 256) {
        const int e = (int)(t % Sp), which = (int)(t / Sp % 2);
        const long long row = t / Sp / 2;
        const int n = (int)(row / a.L), l = (int)(row % a.L);
        float sum = 0;
        if (e < a.G * a.S && l < seq_length(a.lengths, n, a.L)) {
            const int g = e / a.S, s = e % a.S;
            const float *p = a.bc + ((row * a.G + g) * a.btiles * 2 + which) * a.S + s;
            for (int k = 0; k < a.btiles; ++k) sum += p[(long long)k * 2 * a.S];
        }
        const SeqView &v = which ? a.vdC : a.vdB;
        static_cast<T *>(which ? a.dC : a.dB)[n * v.n + e / V * v.c + l * v.l + e % V] = SeqElem<T>::put(sum);
    }
}

// dA, dD, ddt_bias: the runs' parts in order.
__global__ __launch_bounds__(1024) void seq_scan_params_kernel(const SeqScanArgs a)
{
    const long long state = (long long)a.S * a.Cp, col = (long long)blockIdx.x * kSumColumns + threadIdx.x % kSumColumns;
    const bool of_A = col < state;
    const long long e = of_A ? col : col - state, pitch = of_A ? state : 2LL * a.Cp;
    // (results of channels beyond the last one are zero)
    const float s = seq_sum_parts((of_A ? a.hl : a.vec) + e, pitch, a.N * a.chunks, e < pitch && e % a.Cp < a.Ch);
    if (threadIdx.x >= kSumColumns || e >= pitch) return;
    float *out = of_A ? a.dA + e : e < a.Cp ? (a.dD ? a.dD + e : nullptr) : a.ddt_bias ? a.ddt_bias + (e - a.Cp) : nullptr;
    if (out) *out = s;
}

template <typename T, int SP>
hipError_t launch(int dtype, const SeqScanArgs &a, hipStream_t s)
{
    if (a.chunks > 1) {
        const hipError_t e = launch_seq_scan_ends(dtype, a, s);
        if (e != hipSuccess) return e;
    }
    seq_scan_bwd_kernel<T, SP><<<(unsigned)((long long)a.N * a.G * a.btiles * a.chunks), 64, 0, s>>>(a);
    const long long results = ((long long)a.N * a.L * 2 * (a.G * a.S + 7) + 255) / 256;
    seq_scan_bc_kernel<T><<<(unsigned)(results < (1 << 20) ? results : 1 << 20), 256, 0, s>>>(a);
    seq_scan_params_kernel<<<(unsigned)(((a.S + 2LL) * a.Cp + kSumColumns - 1) / kSumColumns), 1024, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_t(int dtype, const SeqScanArgs &a, hipStream_t s)
{
    switch (seq_scan_states(a.S)) {
        case 8: return launch<T, 8>(dtype, a, s);
        case 16: return launch<T, 16>(dtype, a, s);
        case 32: return launch<T, 32>(dtype, a, s);
    }
    return launch<T, 64>(dtype, a, s);
}
}  // namespace

hipError_t launch_seq_scan_bwd(int dtype, const SeqScanArgs &a, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch_t<unsigned short>(dtype, a, s) : launch_t<float>(dtype, a, s);
}

}  // namespace convmi
