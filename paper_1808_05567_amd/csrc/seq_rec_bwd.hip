// Gradients of the gated linear recurrence.
//
//   a = exp(t), t = A s, k = sqrt(1 - a^2), h[l] = a h[l-1] + k g x;   dh[l] = dy z sigmoid(z) + a[l+1] dh[l+1]
//   dx = dh k g,   di = dh k x g (1 - g),   dt = a dh (h[l-1] - g x a / k),   df = dt A s (1 - s),   dA = sum dt s,
//   dz = dy h sigmoid(z) (1 + z (1 - sigmoid(z))),   df_bias = sum df,   di_bias = sum di
//
// States go forwards and their gradients backwards, so that what a run of positions makes of either is found before both are known.  Some 120 operations an element, 14 of them
// exponentials, reciprocals or roots, and f, dy and z are read a second time, but for the first round, where a sequence is longer than a workgroup takes at a time.  Measured, bf16 with z:
// 8 x 2048 positions of 2048 channels, 604 MB and 176 of them again, of which the last cache may hold a part, 162 us (3.7 TB/s without those; vector units 0.4 to 0.7 busy; without z 128;
// positions side by side, 256 workgroups, 207), of which 5 are the sums over the workgroups; 1 x 8192 104 us; fp32, 1024 channels, 141 and without z 105.
#include "seq_rec.h"

namespace convmi {
namespace {

// A workgroup takes a wave's channels of one sequence through all of its positions, or of a run of them: where they are more than its waves have at a time, first from the back for what
// reaches the last position of each round from behind it (which takes f, dy and z; the states before the rounds would take x, f and i and half as much again), then from
// the front.
template <typename T, bool ROWS, int P, bool GATE, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 3) void seq_rec_bwd_kernel(const SeqRecArgs a)
{
    typedef RecLanes<T, ROWS> L;
    typedef typename RecFour<T>::type Four;
    constexpr int E = kRecE;
    __shared__ __align__(16) float runs[2][WAVES][L::COLS][4];  // A, H and, from the back, B
    __shared__ __align__(16) float begin[2][WAVES][L::COLS];
    // of each lane, from the gates to the gradients: s, g, k and what h is multiplied by in dz, in LDS rather than computed again (20 operations of some 110) or in registers,
    // of which four waves a SIMD have 128
    constexpr int KEPT = GATE ? 4 : 3;
    __shared__ seq_u32x4 kept[WAVES][KEPT][P * 64];
    typedef RecOut<T, ROWS, P, false> Out;
    // (the results go out through the place of the last position's, or of the same lane's, which have been read by then)
    static_assert(ROWS || Out::SLOTS == 64 * P || (Out::SLOTS <= 64 && P > 1), "results in the place of what was kept");
    constexpr int RESULTS = ROWS || Out::SLOTS == 64 * P ? 0 : 64 * (P - 1);
    const int waves = blockDim.x / 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, unit = L::unit(lane), at = L::at(lane);
    const int groups = (a.Cp + L::COLS - 1) / L::COLS, run = blockIdx.x / groups % a.runs, n = blockIdx.x / groups / a.runs, c0 = blockIdx.x % groups * L::COLS;
    const bool live = c0 + unit * E < a.Cp;
    const int c = live ? c0 + unit * E : c0;
    const int len = seq_length(a.lengths, n, a.L);
    const auto tensor = [&](const void *p, const SeqView &v) { return RecTensor<T>::template of<L, P>(p, v, n, c0, c, at); };
    const RecTensor<T> x = tensor(a.x, a.vx), f = tensor(a.f, a.vf), i = tensor(a.i, a.vi), z = tensor(a.z, a.vz), dy = tensor(a.dy, a.vdy);
    const Out dx = {kept[wave][0] + RESULTS, tensor(a.dx, a.vdx)}, df = {kept[wave][1] + RESULTS, tensor(a.df, a.vdf)},
              di = {kept[wave][2] + RESULTS, tensor(a.di, a.vdi)}, dz = {kept[wave][KEPT - 1] + RESULTS, tensor(a.dz, a.vdz)};
    // A and the biases, in LDS rather than in 12 registers between their uses (8 x 2048 x 2048 bf16 without z: 141 -> 131 us)
    __shared__ seq_f32x4 params[3][L::UNITS];
    if (wave == 0 && at == 0) {
        const RecParams p(a, c);
        params[0][unit] = RecFour<float>::pack(p.A);
        params[1][unit] = RecFour<float>::pack(p.f);
        params[2][unit] = RecFour<float>::pack(p.i);
    }
    __syncthreads();
    // between waves each lane has one channel
    const int col = lane % L::COLS;
    const bool mine = c0 + col < a.Cp;
    float *marks = a.marks + ((long long)n * a.runs + run) * a.rounds * a.Cp + (mine ? c0 + col : 0);
    const int each = waves * L::LANES * P;
    // What is behind a sequence's end is loaded as zeros: nothing comes from there.
    const auto load = [&](const RecTensor<T> &t, int w0, Four (&b)[P]) {
        const int l0 = w0 + at * P;
        if (w0 + L::LANES * P <= len) {
#pragma unroll
            for (int j = 0; j < P; ++j) b[j] = t.load(w0 + j);
        } else {
#pragma unroll
            for (int j = 0; j < P; ++j) {
                b[j] = Four{};
                if (l0 + j < len) b[j] = t.load(w0 + j);
            }
        }
    };
    const int from = run * a.run, first = from + wave * L::LANES * P, to = min(a.L, from + a.run);  // (a.L is at most 2^30)
    const int rounds = min(a.rounds, (max(len - from, 0) + each - 1) / each);  // that the sequence reaches
    int turn = 0;
    float state = 0, back = 0;  // before the run, and a dh of the position behind it, then behind its rounds
    if (a.runs > 1) {
        const long long step = 3LL * a.Cp;
        const float *t = a.totals + n * a.runs * step + (mine ? c0 + col : 0), *last = t + (a.runs - 1) * step;
        state = rec_through(t, t + a.Cp, step, run, state);
        back = rec_through(last, last + 2 * a.Cp, -step, a.runs - 1 - run, back);
    }
    if (mine && threadIdx.x < L::COLS) marks[max(rounds - 1, 0) * (long long)a.Cp] = back;
    // (what the next round needs is asked for when this one's has come)
    Four bx[P], bf[P], bi[P], bz[P], bdy[P];
    const auto load_back = [&](int round) {
        const int w0 = round * each + first;
        load(f, w0, bf);
        load(dy, w0, bdy);
        if constexpr (GATE) load(z, w0, bz);
    };
    if (rounds > 1) load_back(rounds - 1);
    for (int round = rounds - 1; round > 0; --round, turn ^= 1) {
        float A[E], B[E], pA[E], pf[E];
        rec_unpack(params[0][unit], pA);
        rec_unpack(params[1][unit], pf);
#pragma unroll
        for (int j = P - 1; j >= 0; --j) {
            float ff[E], fz[E], up[E];
            rec_unpack(bf[j], ff);
            rec_unpack(bdy[j], up);
            if constexpr (GATE) rec_unpack(bz[j], fz);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const float p = seq_exp2(pA[k] * rec_gate(ff[k], pf[k]));
                if constexpr (GATE) up[k] *= fz[k] * seq_sigmoid(fz[k]);
                B[k] = p * (j == P - 1 ? up[k] : up[k] + B[k]);
                A[k] = j == P - 1 ? p : A[k] * p;
            }
        }
        if (round > 1) load_back(round - 1);
        rec_join<T, ROWS, true>(A, B, lane);
        if (at == 0)
#pragma unroll
            for (int k = 0; k < E; ++k) *reinterpret_cast<seq_f32x2 *>(&runs[turn][wave][unit * E + k][0]) = seq_f32x2{A[k], B[k]};
        __syncthreads();
        for (int w = waves - 1; w >= 0; --w) back = fmaf(runs[turn][w][col][0], back, runs[turn][w][col][1]);
        if (mine && threadIdx.x < L::COLS) marks[(long long)(round - 1) * a.Cp] = back;
    }
    __syncthreads();  // (the marks are there for all waves)
    float sums[3][E] = {};
    // What a round needs is asked for when the one before has come: all of it, or f and i, which it needs first, where that leaves registers for a fourth workgroup a compute unit
    // (8 x 2048 x 2048 bf16: all 171 us, those 164; but rows of 8 x 2048 x 2048, one workgroup a compute unit, 207 and 226, of 16 x 1024 x 2048, two, 214 and 216, without z 182 and 203).
    constexpr bool ALL = ROWS || WAVES > kSeqRecBwdWaves / 2;
    const auto load_rest = [&](int round) {
        const int w0 = round * each + first;
        load(x, w0, bx);
        load(dy, w0, bdy);
        if constexpr (GATE) load(z, w0, bz);
    };
    const auto load_ahead = [&](int round) {
        const int w0 = round * each + first;
        load(f, w0, bf);
        load(i, w0, bi);
        if constexpr (ALL) load_rest(round);
    };
    load_ahead(0);
    for (int round = 0; round < rounds; ++round, turn ^= 1) {
        back = marks[(long long)round * a.Cp];
        const int w0 = round * each + first, l0 = w0 + at * P;
        Four kx[P];
        if constexpr (!ALL) load_rest(round);
        float pa[P][E], ph[P][E], up[P][E];  // a; k g x, then the state before; what reaches h from y
        float A[E], H[E], Ab[E], B[E], pA[E], pf[E], pi[E];
        rec_unpack(params[0][unit], pA);
        rec_unpack(params[1][unit], pf);
        rec_unpack(params[2][unit], pi);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            float fx[E], ff[E], fi[E], fz[E], root[E];
            rec_unpack(bx[j], fx);
            rec_unpack(bf[j], ff);
            rec_unpack(bi[j], fi);
            rec_unpack(bdy[j], up[j]);
            if constexpr (GATE) rec_unpack(bz[j], fz);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                ff[k] = rec_gate(ff[k], pf[k]);
                fi[k] = rec_gate(fi[k], pi[k]);
                const float t = pA[k] * ff[k];
                pa[j][k] = seq_exp2(t);
                root[k] = __builtin_amdgcn_sqrtf(rec_rest(t, pa[j][k]));
                ph[j][k] = root[k] * fi[k] * fx[k];
                if constexpr (GATE) {
                    const float p = seq_sigmoid(fz[k]), y = up[j][k];
                    up[j][k] *= fz[k] * p;
                    fz[k] = y * p * fmaf(fz[k], 1.0f - p, 1.0f);
                }
                H[k] = j == 0 ? ph[j][k] : fmaf(pa[j][k], H[k], ph[j][k]);
                A[k] = j == 0 ? pa[j][k] : A[k] * pa[j][k];
            }
            kept[wave][0][j * 64 + lane] = SeqElem<float>::pack(ff);
            kept[wave][1][j * 64 + lane] = SeqElem<float>::pack(fi);
            kept[wave][2][j * 64 + lane] = SeqElem<float>::pack(root);
            if constexpr (GATE) kept[wave][3][j * 64 + lane] = SeqElem<float>::pack(fz);
        }
#pragma unroll
        for (int j = 0; j < P; ++j) {
            kx[j] = bx[j];
        }
        if (round < rounds - 1) load_ahead(round + 1);
#pragma unroll
        for (int k = 0; k < E; ++k) {
#pragma unroll
            for (int j = P - 1; j >= 0; --j) B[k] = pa[j][k] * (j == P - 1 ? up[j][k] : up[j][k] + B[k]);
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
        float before = 0;
        for (int w = 0; w < waves; ++w) {
            if (w == wave) before = state;
            state = fmaf(runs[turn][w][col][0], state, runs[turn][w][col][1]);
        }
        for (int w = waves - 1; w > wave; --w) back = fmaf(runs[turn][w][col][0], back, runs[turn][w][col][2]);
        begin[0][wave][col] = before;  // (the lanes that have a channel twice write the same)
        begin[1][wave][col] = back;
        seq_wave_sync();
        float h[E], d[E];
        rec_unpack(params[0][unit], pA);
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
            float fx[E], ff[E], fi[E], fz[E], s[E], g[E], root[E], p[E];
            rec_unpack(kx[j], fx);
            SeqElem<float>::unpack(kept[wave][0][j * 64 + lane], s);
            SeqElem<float>::unpack(kept[wave][1][j * 64 + lane], g);
            SeqElem<float>::unpack(kept[wave][2][j * 64 + lane], root);
            if constexpr (GATE) {
                SeqElem<float>::unpack(kept[wave][3][j * 64 + lane], p);
            }
            seq_wave_sync();
            const bool inside = l0 + j < len;
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const float dh = up[j][k] + d[k], dhk = dh * root[k], gx = g[k] * fx[k], back = pa[j][k] * dh;
                // (a pays for what k lets in; k of zero lets nothing in)
                const float inv = root[k] > 0 ? __builtin_amdgcn_rcpf(root[k]) : 0.0f;
                const float dt = back * fmaf(-gx * pa[j][k], inv, ph[j][k]);
                if constexpr (GATE) fz[k] = p[k] * fmaf(pa[j][k], ph[j][k], root[k] * gx);
                fi[k] = dhk * gx * (1.0f - g[k]);
                fx[k] = dhk * g[k];
                const float dts = dt * s[k];
                ff[k] = dts * (pA[k] * kLn2) * (1.0f - s[k]);
                d[k] = back;
                sums[0][k] += dts;
                sums[1][k] += ff[k];
                sums[2][k] += fi[k];
            }
            const bool ok = live && l0 + j < to;
            dx.put(w0, j, ok, lane, inside ? RecFour<T>::pack(fx) : Four{});
            df.put(w0, j, ok, lane, inside ? RecFour<T>::pack(ff) : Four{});
            di.put(w0, j, ok, lane, inside ? RecFour<T>::pack(fi) : Four{});
            if constexpr (GATE) dz.put(w0, j, ok, lane, inside ? RecFour<T>::pack(fz) : Four{});
        }
        seq_wave_sync();
        dx.out(w0, to, lane);
        df.out(w0, to, lane);
        di.out(w0, to, lane);
        if constexpr (GATE) dz.out(w0, to, lane);
        seq_wave_sync();
    }
    for (int round = rounds; round < a.rounds; ++round) {
        const int w0 = round * each + first;
        dx.clear(w0, to, live, lane);
        df.clear(w0, to, live, lane);
        di.clear(w0, to, live, lane);
        if constexpr (GATE) dz.clear(w0, to, live, lane);
    }
    // the sums of a run: over the lanes that have a channel, then over the waves in order
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
    if (threadIdx.x < L::COLS && mine)
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            float s = 0;
            for (int w = 0; w < waves; ++w) s += runs[0][w][col][q];
            a.part[(((long long)n * a.runs + run) * 3 + q) * a.Cp + c0 + col] = s;
        }
}

// dA, df_bias and di_bias: the runs' sums in order.
__global__ __launch_bounds__(1024) void seq_rec_reduce_kernel(const float *part, float *dA, float *df_bias, float *di_bias, int parts, int Cp)
{
    const int col = blockIdx.x * kSumColumns + threadIdx.x % kSumColumns, q = blockIdx.y;
    const float s = seq_sum_parts(part + (long long)q * Cp + col, 3LL * Cp, parts, col < Cp);
    float *to = q == 0 ? dA : q == 1 ? df_bias : di_bias;
    if (threadIdx.x < kSumColumns && col < Cp && to) to[col] = s;
}

template <typename T, bool ROWS, bool GATE>
void launch_gate(const SeqRecArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)(a.N * a.runs * seq_rec_groups(a.Cp, a.rows, SeqElem<T>::V));
    constexpr int P = kSeqRecBwdPositions;
    if (a.waves > kSeqRecBwdWaves / 2)
        seq_rec_bwd_kernel<T, ROWS, P, GATE, kSeqRecBwdWaves><<<grid, 64 * a.waves, 0, s>>>(a);
    else
        seq_rec_bwd_kernel<T, ROWS, P, GATE, kSeqRecBwdWaves / 2><<<grid, 64 * a.waves, 0, s>>>(a);
}
template <typename T, bool ROWS>
void launch_rows(const SeqRecArgs &a, hipStream_t s)
{
    if (a.z)
        launch_gate<T, ROWS, true>(a, s);
    else
        launch_gate<T, ROWS, false>(a, s);
}
template <typename T>
hipError_t launch_t(int dtype, const SeqRecArgs &a, hipStream_t s)
{
    if (a.runs > 1) {
        const hipError_t e = launch_seq_rec_totals(dtype, true, a, s);
        if (e != hipSuccess) return e;
    }
    if (a.rows)
        launch_rows<T, true>(a, s);
    else
        launch_rows<T, false>(a, s);
    seq_rec_reduce_kernel<<<dim3((a.Cp + kSumColumns - 1) / kSumColumns, 3), 1024, 0, s>>>(a.part, a.dA, a.df_bias, a.di_bias, a.N * a.runs, a.Cp);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_seq_rec_bwd(int dtype, const SeqRecArgs &a, hipStream_t s) { return dtype == SEQ_BF16 ? launch_t<unsigned short>(dtype, a, s) : launch_t<float>(dtype, a, s); }

}  // namespace convmi
