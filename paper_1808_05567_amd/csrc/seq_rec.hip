// Gated linear recurrence of every channel, forward and over one new position.
//
//   s = sigmoid(f + f_bias), g = sigmoid(i + i_bias), a = exp(A s), h[l] = a h[l-1] + sqrt(1 - a^2) g x[l], y = h z sigmoid(z)
//
// Each tensor is read once: what positions make of a state is kept in registers until the state before them is known.  Some 50 operations an element,
// four of them exponentials, three reciprocals, one a root: bound by memory, the vector units 0.4 to 0.7 busy (counters do not tell operations of 2 clocks from those of 4).
// Measured, bf16 with z: 8 x 2048 positions of 2048 channels, 336 MB, 73.5 us (4.5 TB/s; positions side by side 79; without z, 268 MB, 71.5; fp32, 1024 channels, 65.7 and
// without z 66.4), 1 x 8192, 168 MB, 40 us (4.2 TB/s); fp32 without z, 5 sequences of up to 777, 1000 channels side by side, 62 MB: 20.7 us;
// one position of 32 sequences, 4096 channels: 3.7 us, a trip to memory and the launch.
#include "seq_rec.h"

namespace convmi {
namespace {

// A workgroup takes a wave's channels of one sequence through all of its positions, or of a run of them, waves * LANES * P at a time.  P: two positions a lane where a block's
// positions follow one another, whose results go out in 16 bytes each (8 x 2048 x 2048 bf16: four 98 us, one 96, two 89, before results went through LDS); four where they do
// not, since moves between lanes go through LDS there (5 ragged fp32 sequences: two 25.6 us, four 21.3).
// GATE: there is a z.  AHEAD: what the next round needs is asked for when this one's has come (where a compute unit has one workgroup: 1 x 8192 x 2048 bf16 45 -> 43 us,
// ragged rows 26 -> 21; where its registers cost a third workgroup it does not pay: 8 x 2048 x 2048 72 -> 77).
// Without that, dense blocks have 64 registers but in fp32 with z, so that four workgroups of 8 waves share a compute unit (8 x 2048 x 2048 bf16, one register spilled, 75.0 -> 74.1 us,
// without z 77.6 -> 72.6; 16 x 300 x 2048 30.5 -> 27.9; 4 x 2048 x 2048 fp32, 5 registers spilled, 64.9 -> 71.4).  Positions side by side take 79 to 110, with AHEAD up to 128, all there
// are (fp32 without z: one spilled).  All builds without z keep some of what they have loaded in scratch memory, 24 bytes a lane in bf16 and 48 in fp32: they move a fifth less
// than those with z and take as long.
template <typename T, bool ROWS, int P, bool GATE, bool PAST, bool AHEAD>
__global__ __launch_bounds__(64 * kSeqRecWaves, AHEAD || ROWS || (GATE && sizeof(T) == 4) ? 4 : 8) void seq_rec_fwd_kernel(const SeqRecArgs a)
{
    typedef RecLanes<T, ROWS> L;
    typedef typename RecFour<T>::type Four;
    constexpr int E = kRecE;
    __shared__ __align__(16) float runs[2][kSeqRecWaves][L::COLS][2];
    __shared__ __align__(16) float begin[kSeqRecWaves][L::COLS];
    typedef RecOut<T, ROWS, P, PAST> Out;
    __shared__ seq_u32x4 results[kSeqRecWaves][Out::SLOTS];
    const int waves = blockDim.x / 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, unit = L::unit(lane), at = L::at(lane);
    const int groups = (a.Cp + L::COLS - 1) / L::COLS, run = blockIdx.x / groups % a.runs, n = blockIdx.x / groups / a.runs, c0 = blockIdx.x % groups * L::COLS;
    const bool live = c0 + unit * E < a.Cp;
    const int c = live ? c0 + unit * E : c0;
    const int len = seq_length(a.lengths, n, a.L);
    const auto tensor = [&](const void *p, const SeqView &v) { return RecTensor<T>::template of<L, P>(p, v, n, c0, c, at); };
    const RecTensor<T> x = tensor(a.x, a.vx), f = tensor(a.f, a.vf), i = tensor(a.i, a.vi), z = tensor(a.z, a.vz);
    const Out y = {results[wave], tensor(a.y, a.vy)};
    const int slot = a.slots ? a.slots[n] : n;
    const bool has_slot = slot >= 0 && slot < a.n_slots;
    __shared__ seq_f32x4 params[3][L::UNITS];  // A and the biases: not in registers between their uses
    if (wave == 0 && at == 0) {
        const RecParams p(a, c);
        params[0][unit] = RecFour<float>::pack(p.A);
        params[1][unit] = RecFour<float>::pack(p.f);
        params[2][unit] = RecFour<float>::pack(p.i);
    }
    __syncthreads();
    // between waves each lane has one channel
    const int col = lane % L::COLS;
    const bool kept = has_slot && c0 + col < a.Cp;
    float state = 0;
    if (a.runs == 1)
        state = a.state_in && kept ? a.state_in[(long long)slot * a.Cp + c0 + col] : 0.0f;
    else if (c0 + col < a.Cp) {
        const float *t = a.totals + (long long)n * a.runs * 2 * a.Cp + c0 + col;
        state = rec_through(t, t + a.Cp, 2LL * a.Cp, run + 1, state);
    }
    const int from = run * a.run, to = min(a.L, from + a.run);  // (a.L is at most 2^30)
    const int each = waves * L::LANES * P;
    int turn = 0;
    Four bx[P], bf[P], bi[P], bz[P], kz[P];
    const auto load = [&](int w0) {
        const int l0 = w0 + at * P;
        if (w0 + L::LANES * P <= len) {
#pragma unroll
            for (int j = 0; j < P; ++j) {
                bf[j] = f.load(w0 + j);
                bi[j] = i.load(w0 + j);
                bx[j] = x.load(w0 + j);
                if (GATE) bz[j] = z.load(w0 + j);
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < P; ++j) {
            bx[j] = bf[j] = bi[j] = bz[j] = Four{};
            if (l0 + j < len) {
                bx[j] = x.load(w0 + j);
                bf[j] = f.load(w0 + j);
                bi[j] = i.load(w0 + j);
                if (GATE) bz[j] = z.load(w0 + j);
            }
        }
    };
    if constexpr (AHEAD) load(from + wave * L::LANES * P);
    int base = from;
    for (; base < min(to, len); base += each, turn ^= 1) {
        const int w0 = base + wave * L::LANES * P, l0 = w0 + at * P;
        if constexpr (!AHEAD) load(w0);
        float A[E], H[E], pa[P][E], ph[P][E], pA[E], pf[E], pi[E];
        rec_unpack(params[0][unit], pA);
        rec_unpack(params[1][unit], pf);
        rec_unpack(params[2][unit], pi);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            float fx[E], ff[E], fi[E];
            rec_unpack(bx[j], fx);
            rec_unpack(bf[j], ff);
            rec_unpack(bi[j], fi);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const float t = pA[k] * rec_gate(ff[k], pf[k]), p = seq_exp2(t);
                pa[j][k] = l0 + j < len ? p : 1.0f;
                // (what is behind the end was loaded as zero)
                ph[j][k] = __builtin_amdgcn_sqrtf(rec_rest(t, p)) * rec_gate(fi[k], pi[k]) * fx[k];
                H[k] = j == 0 ? ph[j][k] : fmaf(pa[j][k], H[k], ph[j][k]);
                A[k] = j == 0 ? pa[j][k] : A[k] * pa[j][k];
            }
        }
#pragma unroll
        for (int j = 0; j < P; ++j) kz[j] = bz[j];
        if (AHEAD && base + each < min(to, len)) load(w0 + each);
        rec_join<T, ROWS, false>(A, H, lane);
        if (at == L::LANES - 1)
#pragma unroll
            for (int k = 0; k < E; k += 2)
                *reinterpret_cast<seq_f32x4 *>(&runs[turn][wave][unit * E + k][0]) = seq_f32x4{A[k], H[k], A[k + 1], H[k + 1]};
        __syncthreads();
        float before = 0;
        for (int w = 0; w < waves; ++w) {
            if (w == wave) before = state;
            state = fmaf(runs[turn][w][col][0], state, runs[turn][w][col][1]);
        }
        begin[wave][col] = before;  // (the lanes that have a channel twice write the same)
        seq_wave_sync();
        float h[E];
        rec_unpack(*reinterpret_cast<const seq_f32x4 *>(&begin[wave][unit * E]), h);
#pragma unroll
        for (int k = 0; k < E; ++k) h[k] = rec_until<T, ROWS, false>(A[k], H[k], h[k], lane);
#pragma unroll
        for (int j = 0; j < P; ++j) {
            float o[E], fz[E];
            rec_unpack(kz[j], fz);
#pragma unroll
            for (int k = 0; k < E; ++k) {
                h[k] = fmaf(pa[j][k], h[k], ph[j][k]);
                o[k] = GATE ? h[k] * fz[k] * seq_sigmoid(fz[k]) : h[k];
            }
            y.put(w0, j, live && l0 + j < a.L, lane, l0 + j < len ? RecFour<T>::pack(o) : Four{});
        }
        seq_wave_sync();
        y.out(w0, a.L, lane);
        seq_wave_sync();
    }
    for (; base < to; base += each) y.clear(base + wave * L::LANES * P, a.L, live, lane);
    if (a.state_out && kept && run == a.runs - 1 && threadIdx.x < L::COLS) a.state_out[(long long)slot * a.Cp + c0 + col] = state;
}

// What the runs of a sequence make of a state, for those that come after them: forwards of all but the last, and the state before the first.  BACK: of all, from the
// front and from the back.
template <typename T, bool ROWS, int P, bool BACK>
__global__ __launch_bounds__(64 * kSeqRecTotalsWaves) void seq_rec_totals_kernel(const SeqRecArgs a)
{
    typedef RecLanes<T, ROWS> L;
    typedef typename RecFour<T>::type Four;
    constexpr int E = kRecE;
    __shared__ __align__(16) float runs[2][kSeqRecTotalsWaves][L::COLS][4];
    const int waves = blockDim.x / 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, unit = L::unit(lane), at = L::at(lane);
    const int groups = (a.Cp + L::COLS - 1) / L::COLS, here = BACK ? a.runs : a.runs - 1;
    const int run = blockIdx.x / groups % here, n = blockIdx.x / groups / here, c0 = blockIdx.x % groups * L::COLS;
    const int c = c0 + unit * E < a.Cp ? c0 + unit * E : c0;
    const int len = seq_length(a.lengths, n, a.L);
    const auto tensor = [&](const void *p, const SeqView &v) { return RecTensor<T>::template of<L, P>(p, v, n, c0, c, at); };
    const RecTensor<T> x = tensor(a.x, a.vx), f = tensor(a.f, a.vf), i = tensor(a.i, a.vi), z = tensor(a.z, a.vz), dy = tensor(a.dy, a.vdy);
    const RecParams par(a, c);
    const int col = lane % L::COLS;
    const bool mine = c0 + col < a.Cp;
    const int from = run * a.run, to = min(len, from + a.run);
    const int each = waves * L::LANES * P;
    float sumA = 1, sumH = 0, sumB = 0;
    int turn = 0;
    // (behind a sequence's end nothing changes)
    for (int base = from; base < to; base += each, turn ^= 1) {
        const int w0 = base + wave * L::LANES * P, l0 = w0 + at * P;
        Four bx[P], bf[P], bi[P], bz[P], bdy[P];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            bx[j] = bf[j] = bi[j] = bz[j] = bdy[j] = Four{};
            if (l0 + j < to) {
                bx[j] = x.load(w0 + j);
                bf[j] = f.load(w0 + j);
                bi[j] = i.load(w0 + j);
                if (BACK) bdy[j] = dy.load(w0 + j);
                if (BACK && a.z) bz[j] = z.load(w0 + j);
            }
        }
        float A[E], H[E], Ab[E], B[E], pa[P][E], up[P][E];
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
                pa[j][k] = l0 + j < to ? p : 1.0f;
                const float u = __builtin_amdgcn_sqrtf(rec_rest(t, p)) * rec_gate(fi[k], par.i[k]) * fx[k];
                H[k] = j == 0 ? u : fmaf(pa[j][k], H[k], u);
                A[k] = j == 0 ? pa[j][k] : A[k] * pa[j][k];
            }
            if (BACK && a.z)
#pragma unroll
                for (int k = 0; k < E; ++k) up[j][k] *= fz[k] * seq_sigmoid(fz[k]);
        }
        if constexpr (BACK) {
#pragma unroll
            for (int k = 0; k < E; ++k) {
#pragma unroll
                for (int j = P - 1; j >= 0; --j) B[k] = pa[j][k] * (j == P - 1 ? up[j][k] : up[j][k] + B[k]);
                Ab[k] = A[k];
            }
            rec_join<T, ROWS, true>(Ab, B, lane);
            if (at == 0)
#pragma unroll
                for (int k = 0; k < E; ++k) runs[turn][wave][unit * E + k][2] = B[k];
        }
        rec_join<T, ROWS, false>(A, H, lane);
        if (at == L::LANES - 1)
#pragma unroll
            for (int k = 0; k < E; ++k) *reinterpret_cast<seq_f32x2 *>(&runs[turn][wave][unit * E + k][0]) = seq_f32x2{A[k], H[k]};
        __syncthreads();
        for (int w = 0; w < waves; ++w) {
            const float *r = runs[turn][w][col];
            if (BACK) sumB = fmaf(sumA, r[2], sumB);
            sumH = fmaf(r[0], sumH, r[1]);
            sumA *= r[0];
        }
    }
    if (threadIdx.x >= L::COLS || !mine) return;
    float *t = a.totals + ((long long)n * a.runs + run + (BACK ? 0 : 1)) * (BACK ? 3 : 2) * a.Cp + c0 + col;
    t[0] = sumA;
    t[a.Cp] = sumH;
    if (BACK) t[2 * a.Cp] = sumB;
    if (!BACK && run == 0) {
        const int slot = a.slots ? a.slots[n] : n;
        t -= 2 * a.Cp;
        t[0] = 0;
        t[a.Cp] = a.state_in && slot >= 0 && slot < a.n_slots ? a.state_in[(long long)slot * a.Cp + c0 + col] : 0.0f;
    }
}

template <typename T>
__global__ __launch_bounds__(64) void seq_rec_step_kernel(const SeqRecArgs a)
{
    constexpr int V = SeqElem<T>::V, E = kRecE;
    const long long t = (long long)blockIdx.x * 64 + threadIdx.x;
    if (t >= (long long)a.N * (a.Cp / E)) return;
    const int n = (int)(t / (a.Cp / E)), c = (int)(t % (a.Cp / E)) * E, cb = c / V;
    const int slot = a.slots ? a.slots[n] : n;
    typedef typename RecFour<T>::type Four;
    const auto four = [&](const void *p, const SeqView &v) { return reinterpret_cast<const Four *>(static_cast<const T *>(p) + n * v.n + cb * v.c + c % V); };
    Four *y = const_cast<Four *>(four(a.y, a.vy));
    if (slot < 0 || slot >= a.n_slots) {
        *y = Four{};
        return;
    }
    float *to = a.state_out + (long long)slot * a.Cp + c;
    float h[E], fx[E], ff[E], fi[E], fz[E], o[E];
    seq_vector<E>(to, 0, h);
    rec_unpack(*four(a.x, a.vx), fx);
    rec_unpack(*four(a.f, a.vf), ff);
    rec_unpack(*four(a.i, a.vi), fi);
    if (a.z) rec_unpack(*four(a.z, a.vz), fz);
    const RecParams par(a, c);
#pragma unroll
    for (int k = 0; k < E; ++k) {
        const float e = par.A[k] * rec_gate(ff[k], par.f[k]), d = seq_exp2(e);
        h[k] = fmaf(d, h[k], __builtin_amdgcn_sqrtf(rec_rest(e, d)) * rec_gate(fi[k], par.i[k]) * fx[k]);
        o[k] = a.z ? h[k] * fz[k] * seq_sigmoid(fz[k]) : h[k];
    }
    *y = RecFour<T>::pack(o);
    *reinterpret_cast<seq_f32x4 *>(to) = seq_f32x4{h[0], h[1], h[2], h[3]};
}

template <typename T, bool ROWS, bool GATE, bool AHEAD>
hipError_t launch_ahead(const SeqRecArgs &a, hipStream_t s)
{
    constexpr int P = seq_rec_positions(ROWS);
    const unsigned grid = (unsigned)(a.N * a.runs * seq_rec_groups(a.Cp, a.rows, SeqElem<T>::V));
    if (a.past)
        seq_rec_fwd_kernel<T, ROWS, P, GATE, true, AHEAD><<<grid, 64 * a.waves, 0, s>>>(a);
    else
        seq_rec_fwd_kernel<T, ROWS, P, GATE, false, AHEAD><<<grid, 64 * a.waves, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, bool ROWS, bool GATE>
hipError_t launch_gate(const SeqRecArgs &a, hipStream_t s)
{
    constexpr bool REGISTERS = sizeof(T) == 2 || !ROWS || !GATE;  // (there are enough of)
    if constexpr (REGISTERS) {
        if (a.few) return launch_ahead<T, ROWS, GATE, true>(a, s);
    }
    return launch_ahead<T, ROWS, GATE, false>(a, s);
}
template <typename T, bool ROWS>
hipError_t launch_rows(const SeqRecArgs &a, hipStream_t s)
{
    return a.z ? launch_gate<T, ROWS, true>(a, s) : launch_gate<T, ROWS, false>(a, s);
}
template <typename T, bool ROWS>
hipError_t launch_totals(bool back, const SeqRecArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)(a.N * (a.runs - !back) * seq_rec_groups(a.Cp, a.rows, SeqElem<T>::V));
    constexpr int P = seq_rec_positions(ROWS);
    if (back)
        seq_rec_totals_kernel<T, ROWS, P, true><<<grid, 64 * kSeqRecTotalsWaves, 0, s>>>(a);
    else
        seq_rec_totals_kernel<T, ROWS, P, false><<<grid, 64 * kSeqRecTotalsWaves, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_totals_t(bool back, const SeqRecArgs &a, hipStream_t s)
{
    return a.rows ? launch_totals<T, true>(back, a, s) : launch_totals<T, false>(back, a, s);
}
template <typename T>
hipError_t launch_t(const SeqRecArgs &a, hipStream_t s)
{
    if (a.runs > 1) {
        const hipError_t e = launch_totals_t<T>(false, a, s);
        if (e != hipSuccess) return e;
    }
    return a.rows ? launch_rows<T, true>(a, s) : launch_rows<T, false>(a, s);
}
template <typename T>
hipError_t launch_step(const SeqRecArgs &a, hipStream_t s)
{
    seq_rec_step_kernel<T><<<(unsigned)(((long long)a.N * (a.Cp / kRecE) + 63) / 64), 64, 0, s>>>(a);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_seq_rec_fwd(int dtype, const SeqRecArgs &a, hipStream_t s) { return dtype == SEQ_BF16 ? launch_t<unsigned short>(a, s) : launch_t<float>(a, s); }
hipError_t launch_seq_rec_totals(int dtype, bool back, const SeqRecArgs &a, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch_totals_t<unsigned short>(back, a, s) : launch_totals_t<float>(back, a, s);
}
hipError_t launch_seq_rec_step(int dtype, const SeqRecArgs &a, hipStream_t s) { return dtype == SEQ_BF16 ? launch_step<unsigned short>(a, s) : launch_step<float>(a, s); }

}  // namespace convmi
