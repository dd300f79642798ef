// Gradients of the gated linear recurrence.
//
//   a = exp(t), t = A s, k = sqrt(1 - a^2), h[l] = a h[l-1] + k g x;   dh[l] = dy z sigmoid(z) + a[l+1] dh[l+1]
//   dx = dh k g,   di = dh k x g (1 - g),   dt = a dh (h[l-1] - g x a / k),   df = dt A s (1 - s),   dA = sum dt s,
//   dz = dy h sigmoid(z) (1 + z (1 - sigmoid(z))),   df_bias = sum df,   di_bias = sum di
#include "seq_rec.h"

namespace convmi {
namespace {

// A workgroup takes 64 / LANES blocks of channels of one sequence through all of its positions, as forwards: first from the front for the states before
// each round of its waves, where there are several, then from the back.
template <typename T, int LANES, int P>
__global__ __launch_bounds__(64 * kRecWaves) void seq_rec_bwd_kernel(const SeqRecArgs a)
{
    constexpr int V = SeqElem<T>::V, BLOCKS = 64 / LANES;
    __shared__ float runs[2][kRecWaves][BLOCKS][3][V];
    const int waves = blockDim.x / 64, wave = threadIdx.x / 64, at = threadIdx.x % LANES, bl = threadIdx.x % 64 / LANES;
    const int groups = (a.Cb + BLOCKS - 1) / BLOCKS, n = blockIdx.x / groups;
    const bool live = blockIdx.x % groups * BLOCKS + bl < a.Cb;
    const int cb = live ? blockIdx.x % groups * BLOCKS + bl : a.Cb - 1;
    const int len = seq_length(a.lengths, n, a.L);
    const T *x = static_cast<const T *>(a.x) + n * a.vx.n + cb * a.vx.c;
    const T *f = static_cast<const T *>(a.f) + n * a.vf.n + cb * a.vf.c;
    const T *i = static_cast<const T *>(a.i) + n * a.vi.n + cb * a.vi.c;
    const T *z = a.z ? static_cast<const T *>(a.z) + n * a.vz.n + cb * a.vz.c : nullptr;
    const T *dy = static_cast<const T *>(a.dy) + n * a.vdy.n + cb * a.vdy.c;
    T *dx = static_cast<T *>(a.dx) + n * a.vdx.n + cb * a.vdx.c;
    T *df = static_cast<T *>(a.df) + n * a.vdf.n + cb * a.vdf.c;
    T *di = static_cast<T *>(a.di) + n * a.vdi.n + cb * a.vdi.c;
    T *dz = a.z ? static_cast<T *>(a.dz) + n * a.vdz.n + cb * a.vdz.c : nullptr;
    const RecParams<V> par(a, cb);
    const int each = waves * LANES * P;
    float state[V] = {};
    int turn = 0;
    if (a.rounds > 1) {
        for (int round = 0; round < a.rounds; ++round, turn ^= 1) {
            float *mark = a.marks + ((long long)n * a.rounds + round) * a.Cp + (long long)cb * V;
            if (live && wave == 0 && at == 0)
#pragma unroll
                for (int k = 0; k < V; ++k) mark[k] = state[k];
            const long long l0 = (long long)round * each + (wave * LANES + at) * P;
            float A[V], H[V];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                A[k] = 1;
                H[k] = 0;
            }
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const long long l = l0 + j;
                if (l < len) {
                    float fx[V], ff[V], fi[V];
                    SeqElem<T>::unpack(seq_load(x + l * a.vx.l), fx);
                    SeqElem<T>::unpack(seq_load(f + l * a.vf.l), ff);
                    SeqElem<T>::unpack(seq_load(i + l * a.vi.l), fi);
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        const float t = par.A[k] * rec_gate(ff[k], par.f[k]), pa = seq_exp2(t);
                        H[k] = fmaf(pa, H[k], __builtin_amdgcn_sqrtf(rec_rest(t, pa)) * rec_gate(fi[k], par.i[k]) * fx[k]);
                        A[k] *= pa;
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < V; ++k) rec_join<LANES, 1, false>(A[k], H[k], at);
            if (at == LANES - 1)
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    runs[turn][wave][bl][0][k] = A[k];
                    runs[turn][wave][bl][1][k] = H[k];
                }
            __syncthreads();
            for (int w = 0; w < waves; ++w)
#pragma unroll
                for (int k = 0; k < V; ++k) state[k] = fmaf(runs[turn][w][bl][0][k], state[k], runs[turn][w][bl][1][k]);
        }
        __syncthreads();  // (the states before the rounds are there for all waves)
    }
    float back[V] = {};  // a dh of the position behind a round
    float sums[3][V] = {};
    for (int round = a.rounds - 1; round >= 0; --round, turn ^= 1) {
        if (a.rounds > 1) seq_vector<V>(a.marks + ((long long)n * a.rounds + round) * a.Cp, cb, state);
        const long long l0 = (long long)round * each + (wave * LANES + at) * P;
        seq_u32x4 bx[P], bf[P], bi[P], bz[P], bdy[P];
        float pa[P][V], ph[P][V], up[P][V];  // a; k g x, then the state before; what reaches h from y
        float A[V], H[V], B[V];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const long long l = l0 + j;
            bx[j] = bf[j] = bi[j] = bz[j] = bdy[j] = seq_u32x4{};
            if (l < len) {
                bx[j] = seq_load(x + l * a.vx.l);
                bf[j] = seq_load(f + l * a.vf.l);
                bi[j] = seq_load(i + l * a.vi.l);
                bdy[j] = seq_load(dy + l * a.vdy.l);
                if (z) bz[j] = seq_load(z + l * a.vz.l);
            }
        }
#pragma unroll
        for (int j = 0; j < P; ++j) {
            float fx[V], ff[V], fi[V], fz[V];
            SeqElem<T>::unpack(bx[j], fx);
            SeqElem<T>::unpack(bf[j], ff);
            SeqElem<T>::unpack(bi[j], fi);
            SeqElem<T>::unpack(bz[j], fz);
            SeqElem<T>::unpack(bdy[j], up[j]);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if (l0 + j < len) {
                    const float t = par.A[k] * rec_gate(ff[k], par.f[k]);
                    pa[j][k] = seq_exp2(t);
                    ph[j][k] = __builtin_amdgcn_sqrtf(rec_rest(t, pa[j][k])) * rec_gate(fi[k], par.i[k]) * fx[k];
                    if (z) up[j][k] *= fz[k] * seq_sigmoid(fz[k]);
                } else {
                    pa[j][k] = 1;
                    ph[j][k] = up[j][k] = 0;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < V; ++k) {
            A[k] = 1;
            H[k] = B[k] = 0;
#pragma unroll
            for (int j = 0; j < P; ++j) {
                H[k] = fmaf(pa[j][k], H[k], ph[j][k]);
                A[k] *= pa[j][k];
            }
#pragma unroll
            for (int j = P - 1; j >= 0; --j) B[k] = pa[j][k] * (up[j][k] + B[k]);
        }
        float Ab[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            Ab[k] = A[k];
            rec_join<LANES, 1, false>(A[k], H[k], at);
            rec_join<LANES, 1, true>(Ab[k], B[k], at);
        }
        if (at == LANES - 1)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                runs[turn][wave][bl][0][k] = A[k];
                runs[turn][wave][bl][1][k] = H[k];
            }
        if (at == 0)
#pragma unroll
            for (int k = 0; k < V; ++k) runs[turn][wave][bl][2][k] = B[k];
        __syncthreads();
        float h[V], d[V];  // before and behind the wave's positions
        for (int w = 0; w < waves; ++w)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if (w == wave) h[k] = state[k];
                state[k] = fmaf(runs[turn][w][bl][0][k], state[k], runs[turn][w][bl][1][k]);
            }
        for (int w = waves - 1; w >= 0; --w)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if (w == wave) d[k] = back[k];
                back[k] = fmaf(runs[turn][w][bl][0][k], back[k], runs[turn][w][bl][2][k]);
            }
#pragma unroll
        for (int k = 0; k < V; ++k) {  // the lane's
            float la = rec_near<1, false>(1.0f, A[k]), lh = rec_near0<1, false>(H[k]);
            if (at == 0) la = 1, lh = 0;
            h[k] = fmaf(la, h[k], lh);
            la = rec_near<1, true>(1.0f, Ab[k]), lh = rec_near0<1, true>(B[k]);
            if (at == LANES - 1) la = 1, lh = 0;
            d[k] = fmaf(la, d[k], lh);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const float before = h[k];
                h[k] = fmaf(pa[j][k], h[k], ph[j][k]);
                ph[j][k] = before;
            }
        }
#pragma unroll
        for (int j = P - 1; j >= 0; --j) {
            const long long l = l0 + j;
            if (l >= a.L || !live) continue;
            seq_u32x4 ox = {}, of = {}, oi = {}, oz = {};
            if (l < len) {
                float fx[V], ff[V], fi[V], fz[V], fdy[V];
                SeqElem<T>::unpack(bx[j], fx);
                SeqElem<T>::unpack(bf[j], ff);
                SeqElem<T>::unpack(bi[j], fi);
                SeqElem<T>::unpack(bz[j], fz);
                SeqElem<T>::unpack(bdy[j], fdy);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float s = rec_gate(ff[k], par.f[k]), g = rec_gate(fi[k], par.i[k]), t = par.A[k] * s, rest = rec_rest(t, pa[j][k]);
                    // (what is too small for a normal number is none: the hardware's root takes it for zero)
                    const float inv = rest >= 1.17549435e-38f ? __builtin_amdgcn_rsqf(rest) : 0.0f, root = rest * inv;
                    const float dh = up[j][k] + d[k], dhg = dh * g, gx = g * fx[k];
                    const float dt = dh * pa[j][k] * fmaf(-gx * pa[j][k], inv, ph[j][k]);
                    if (z) {
                        const float p = seq_sigmoid(fz[k]);
                        fz[k] = fdy[k] * fmaf(pa[j][k], ph[j][k], root * gx) * p * fmaf(fz[k], 1.0f - p, 1.0f);
                    }
                    fi[k] = dhg * root * fx[k] * (1.0f - g);
                    fx[k] = dhg * root;
                    ff[k] = dt * (t * kLn2) * (1.0f - s);
                    sums[0][k] = fmaf(dt, s, sums[0][k]);
                    sums[1][k] += ff[k];
                    sums[2][k] += fi[k];
                    d[k] = pa[j][k] * dh;
                }
                ox = SeqElem<T>::pack(fx);
                of = SeqElem<T>::pack(ff);
                oi = SeqElem<T>::pack(fi);
                oz = SeqElem<T>::pack(fz);
            }
            seq_store(dx + l * a.vdx.l, ox);
            seq_store(df + l * a.vdf.l, of);
            seq_store(di + l * a.vdi.l, oi);
            if (z) seq_store(dz + l * a.vdz.l, oz);
        }
    }
    // the sums of a sequence: over a block's lanes, then over the waves in order
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int k = 0; k < V; ++k) {
            float s = sums[q][k];
#pragma unroll
            for (int d = 1; d < LANES; d *= 2) s += __shfl_xor(s, d);
            if (at == 0) runs[0][wave][bl][q][k] = s;
        }
    __syncthreads();
    if (wave == 0 && at == 0 && live)
#pragma unroll
        for (int q = 0; q < 3; ++q)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float s = 0;
                for (int w = 0; w < waves; ++w) s += runs[0][w][bl][q][k];
                a.part[((long long)n * 3 + q) * a.Cp + (long long)cb * V + k] = s;
            }
}

// dA, df_bias and di_bias: the sequences' sums in order.
__global__ __launch_bounds__(1024) void seq_rec_reduce_kernel(const float *part, float *dA, float *df_bias, float *di_bias, int N, int Cp)
{
    const int col = blockIdx.x * kSumColumns + threadIdx.x % kSumColumns, q = blockIdx.y;
    const float s = seq_sum_parts(part + (long long)q * Cp + col, 3LL * Cp, N, col < Cp);
    float *to = q == 0 ? dA : q == 1 ? df_bias : di_bias;
    if (threadIdx.x < kSumColumns && col < Cp && to) to[col] = s;
}

template <typename T>
hipError_t launch_t(const SeqRecArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)((long long)a.N * seq_rec_groups(a.Cb, a.lanes));
    if (a.lanes == 16)
        seq_rec_bwd_kernel<T, 16, kSeqRecPositions><<<grid, 64 * a.waves, 0, s>>>(a);
    else
        seq_rec_bwd_kernel<T, 4, kSeqRecPositions><<<grid, 64 * a.waves, 0, s>>>(a);
    seq_rec_reduce_kernel<<<dim3((a.Cp + kSumColumns - 1) / kSumColumns, 3), 1024, 0, s>>>(a.part, a.dA, a.df_bias, a.di_bias, a.N, a.Cp);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_seq_rec_bwd(int dtype, const SeqRecArgs &a, hipStream_t s) { return dtype == SEQ_BF16 ? launch_t<unsigned short>(a, s) : launch_t<float>(a, s); }

}  // namespace convmi
