// Gradients of the gated linear recurrence.
//
//   a = exp(t), t = A s, k = sqrt(1 - a^2), h[l] = a h[l-1] + k g x;   dh[l] = dy z sigmoid(z) + a[l+1] dh[l+1]
//   dx = dh k g,   di = dh k x g (1 - g),   dt = a dh (h[l-1] - g x a / k),   df = dt A s (1 - s),   dA = sum dt s,
//   dz = dy h sigmoid(z) (1 + z (1 - sigmoid(z))),   df_bias = sum df,   di_bias = sum di
#include "seq_rec.h"

namespace convmi {
namespace {

// A workgroup takes a wave's channels of one sequence through all of its positions, as forwards: first from the front for the states before each round of
// its waves, where there are several, then from the back.
template <typename T, bool ROWS, int P, bool GATE, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void seq_rec_bwd_kernel(const SeqRecArgs a)
{
    typedef RecLanes<T, ROWS> L;
    typedef typename RecFour<T>::type Four;
    constexpr int E = kRecE;
    __shared__ __align__(16) float runs[2][WAVES][L::COLS][4];  // A, H and, backwards, B
    __shared__ __align__(16) float begin[2][WAVES][L::COLS];
    typedef RecOut<T, ROWS, P, false> Out;
    __shared__ seq_u32x4 results[WAVES][4][Out::SLOTS];
    const int waves = blockDim.x / 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, unit = L::unit(lane), at = L::at(lane);
    const int groups = (a.Cp + L::COLS - 1) / L::COLS, n = blockIdx.x / groups, c0 = blockIdx.x % groups * L::COLS;
    const bool live = c0 + unit * E < a.Cp;
    const int c = live ? c0 + unit * E : c0;
    const int len = seq_length(a.lengths, n, a.L);
    const auto tensor = [&](const void *p, const SeqView &v) { return RecTensor<T>::template of<L, P>(p, v, n, c0, c, at); };
    const RecTensor<T> x = tensor(a.x, a.vx), f = tensor(a.f, a.vf), i = tensor(a.i, a.vi), z = tensor(a.z, a.vz), dy = tensor(a.dy, a.vdy);
    const Out dx = {results[wave][0], tensor(a.dx, a.vdx)}, df = {results[wave][1], tensor(a.df, a.vdf)}, di = {results[wave][2], tensor(a.di, a.vdi)},
              dz = {results[wave][3], tensor(a.dz, a.vdz)};
    const RecParams par(a, c);
    // between waves each lane has one channel
    const int col = lane % L::COLS;
    const bool kept = c0 + col < a.Cp;
    float *marks = a.marks + (long long)n * a.rounds * a.Cp + (kept ? c0 + col : 0);
    const int each = waves * L::LANES * P;
    int turn = 0;
    float state = 0;
    for (int round = 0; round < a.rounds - 1; ++round, turn ^= 1) {
        if (kept && threadIdx.x < L::COLS) marks[(long long)round * a.Cp] = state;
        const long long w0 = (long long)round * each + wave * L::LANES * P, l0 = w0 + at * P;
        Four bx[P], bf[P], bi[P];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            bx[j] = bf[j] = bi[j] = Four{};
            if (l0 + j < len) {
                bx[j] = x.load(w0 + j);
                bf[j] = f.load(w0 + j);
                bi[j] = i.load(w0 + j);
            }
        }
        float A[E], H[E];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            float fx[E], ff[E], fi[E];
            rec_unpack(bx[j], fx);
            rec_unpack(bf[j], ff);
            rec_unpack(bi[j], fi);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const float t = par.A[k] * rec_gate(ff[k], par.f[k]), e = seq_exp2(t), p = l0 + j < len ? e : 1.0f;
                const float u = __builtin_amdgcn_sqrtf(rec_rest(t, e)) * rec_gate(fi[k], par.i[k]) * fx[k];
                H[k] = j == 0 ? u : fmaf(p, H[k], u);
                A[k] = j == 0 ? p : A[k] * p;
            }
        }
        rec_join<T, ROWS, false>(A, H, lane);
        if (at == L::LANES - 1)
#pragma unroll
            for (int k = 0; k < E; ++k) *reinterpret_cast<seq_f32x2 *>(&runs[turn][wave][unit * E + k][0]) = seq_f32x2{A[k], H[k]};
        __syncthreads();
        for (int w = 0; w < waves; ++w) state = fmaf(runs[turn][w][col][0], state, runs[turn][w][col][1]);
    }
    float back = 0;  // a dh of the position behind a round
    float sums[3][E] = {};
    for (int round = a.rounds - 1; round >= 0; --round, turn ^= 1) {
        // (the lanes of each wave that a mark comes from, or the first one's, which has passed a barrier since it stored it)
        if (round < a.rounds - 1) state = marks[(long long)round * a.Cp];
        const long long w0 = (long long)round * each + wave * L::LANES * P, l0 = w0 + at * P;
        Four bx[P], bf[P], bi[P], bz[P], bdy[P];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            bx[j] = bf[j] = bi[j] = bz[j] = bdy[j] = Four{};
            if (l0 + j < len) {
                bx[j] = x.load(w0 + j);
                bf[j] = f.load(w0 + j);
                bi[j] = i.load(w0 + j);
                bdy[j] = dy.load(w0 + j);
                if (GATE) bz[j] = z.load(w0 + j);
            }
        }
        float pa[P][E], ph[P][E], up[P][E];  // a; k g x, then the state before; what reaches h from y
        float A[E], H[E], Ab[E], B[E];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            float fx[E], ff[E], fi[E], fz[E];
            rec_unpack(bx[j], fx);
            rec_unpack(bf[j], ff);
            rec_unpack(bi[j], fi);
            rec_unpack(bz[j], fz);
            rec_unpack(bdy[j], up[j]);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const float t = par.A[k] * rec_gate(ff[k], par.f[k]), p = seq_exp2(t);
                pa[j][k] = l0 + j < len ? p : 1.0f;
                ph[j][k] = __builtin_amdgcn_sqrtf(rec_rest(t, p)) * rec_gate(fi[k], par.i[k]) * fx[k];
                if (GATE) up[j][k] *= fz[k] * seq_sigmoid(fz[k]);
                H[k] = j == 0 ? ph[j][k] : fmaf(pa[j][k], H[k], ph[j][k]);
                A[k] = j == 0 ? pa[j][k] : A[k] * pa[j][k];
            }
        }
#pragma unroll
        for (int k = 0; k < E; ++k) {
            B[k] = 0;
#pragma unroll
            for (int j = P - 1; j >= 0; --j) B[k] = pa[j][k] * (up[j][k] + B[k]);
            Ab[k] = A[k];
        }
        rec_join<T, ROWS, false>(A, H, lane);
        rec_join<T, ROWS, true>(Ab, B, lane);
        if (at == L::LANES - 1)
#pragma unroll
            for (int k = 0; k < E; ++k) *reinterpret_cast<seq_f32x2 *>(&runs[turn][wave][unit * E + k][0]) = seq_f32x2{A[k], H[k]};
        if (at == 0)
#pragma unroll
            for (int k = 0; k < E; ++k) runs[turn][wave][unit * E + k][2] = B[k];
        __syncthreads();
        float before = 0, behind = 0;
        for (int w = 0; w < wave; ++w) state = fmaf(runs[turn][w][col][0], state, runs[turn][w][col][1]);
        before = state;
        for (int w = waves - 1; w >= 0; --w) {
            if (w == wave) behind = back;
            back = fmaf(runs[turn][w][col][0], back, runs[turn][w][col][2]);
        }
        begin[0][wave][col] = before;  // (the lanes that have a channel twice write the same)
        begin[1][wave][col] = behind;
        seq_wave_sync();
        float h[E], d[E];
        rec_unpack(*reinterpret_cast<const seq_f32x4 *>(&begin[0][wave][unit * E]), h);
        rec_unpack(*reinterpret_cast<const seq_f32x4 *>(&begin[1][wave][unit * E]), d);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            h[k] = rec_until<T, ROWS, false>(A[k], H[k], h[k], lane);
            d[k] = rec_until<T, ROWS, true>(Ab[k], B[k], d[k], lane);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const float old = h[k];
                h[k] = fmaf(pa[j][k], h[k], ph[j][k]);
                ph[j][k] = old;
            }
        }
#pragma unroll
        for (int j = P - 1; j >= 0; --j) {
            float fx[E], ff[E], fi[E], fz[E], fdy[E];
            rec_again(bx[j]);
            rec_again(bf[j]);
            rec_again(bi[j]);
            rec_again(bz[j]);
            rec_again(bdy[j]);
            rec_unpack(bx[j], fx);
            rec_unpack(bf[j], ff);
            rec_unpack(bi[j], fi);
            rec_unpack(bz[j], fz);
            rec_unpack(bdy[j], fdy);
            const bool inside = l0 + j < len;
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const float s = rec_gate(ff[k], par.f[k]), g = rec_gate(fi[k], par.i[k]), t = par.A[k] * s, rest = rec_rest(t, pa[j][k]);
                // (what is too small for a normal number is none: the hardware's root takes it for zero)
                const float inv = rest >= 1.17549435e-38f ? __builtin_amdgcn_rsqf(rest) : 0.0f, root = rest * inv;
                const float dh = up[j][k] + d[k], dhg = dh * g, gx = g * fx[k];
                const float dt = dh * pa[j][k] * fmaf(-gx * pa[j][k], inv, ph[j][k]);
                if (GATE) {
                    const float p = seq_sigmoid(fz[k]);
                    fz[k] = fdy[k] * fmaf(pa[j][k], ph[j][k], root * gx) * p * fmaf(fz[k], 1.0f - p, 1.0f);
                }
                fi[k] = dhg * root * fx[k] * (1.0f - g);
                fx[k] = dhg * root;
                ff[k] = dt * (t * kLn2) * (1.0f - s);
                d[k] = pa[j][k] * dh;
                if (inside) {
                    sums[0][k] = fmaf(dt, s, sums[0][k]);
                    sums[1][k] += ff[k];
                    sums[2][k] += fi[k];
                }
            }
            const bool ok = live && l0 + j < a.L;
            dx.put(w0, j, ok, lane, inside ? RecFour<T>::pack(fx) : Four{});
            df.put(w0, j, ok, lane, inside ? RecFour<T>::pack(ff) : Four{});
            di.put(w0, j, ok, lane, inside ? RecFour<T>::pack(fi) : Four{});
            if (GATE) dz.put(w0, j, ok, lane, inside ? RecFour<T>::pack(fz) : Four{});
        }
        seq_wave_sync();
        dx.out(w0, a.L, lane);
        df.out(w0, a.L, lane);
        di.out(w0, a.L, lane);
        if (GATE) dz.out(w0, a.L, lane);
        seq_wave_sync();
    }
    // the sums of a sequence: over the lanes that have a channel, then over the waves in order
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int k = 0; k < E; ++k) {
            float s = sums[q][k];
#pragma unroll
            for (int d = 1; d < L::LANES; d *= 2) s += __shfl_xor(s, d * L::STEP);
            if (at == 0) runs[0][wave][unit * E + k][q] = s;
        }
    __syncthreads();
    if (threadIdx.x < L::COLS && kept)
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            float s = 0;
            for (int w = 0; w < waves; ++w) s += runs[0][w][col][q];
            a.part[((long long)n * 3 + q) * a.Cp + c0 + col] = s;
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

template <typename T, bool ROWS>
void launch_rows(const SeqRecArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)(a.N * seq_rec_groups(a.Cp, a.rows, SeqElem<T>::V));
    if (a.z)
        seq_rec_bwd_kernel<T, ROWS, kSeqRecBwdPositions, true, kSeqRecBwdWaves><<<grid, 64 * a.waves, 0, s>>>(a);
    else
        seq_rec_bwd_kernel<T, ROWS, kSeqRecBwdPositions, false, kSeqRecBwdWaves><<<grid, 64 * a.waves, 0, s>>>(a);
}
template <typename T>
hipError_t launch_t(const SeqRecArgs &a, hipStream_t s)
{
    if (a.rows)
        launch_rows<T, true>(a, s);
    else
        launch_rows<T, false>(a, s);
    seq_rec_reduce_kernel<<<dim3((a.Cp + kSumColumns - 1) / kSumColumns, 3), 1024, 0, s>>>(a.part, a.dA, a.df_bias, a.di_bias, a.N, a.Cp);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_seq_rec_bwd(int dtype, const SeqRecArgs &a, hipStream_t s) { return dtype == SEQ_BF16 ? launch_t<unsigned short>(a, s) : launch_t<float>(a, s); }

}  // namespace convmi
