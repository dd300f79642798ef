// Gated linear recurrence of every channel, forward and over one new position.
//
//   s = sigmoid(f + f_bias), g = sigmoid(i + i_bias), a = exp(A s), h[l] = a h[l-1] + sqrt(1 - a^2) g x[l], y = h z sigmoid(z)
#include "seq_rec.h"

namespace convmi {
namespace {

// A workgroup takes 64 / LANES blocks of channels of one sequence through all of its positions, waves * LANES * P of them at a time.
template <typename T, int LANES, int P, bool PAST>
__global__ __launch_bounds__(64 * kRecWaves) void seq_rec_fwd_kernel(const SeqRecArgs a)
{
    constexpr int V = SeqElem<T>::V, BLOCKS = 64 / LANES;
    __shared__ float runs[2][kRecWaves][BLOCKS][2][V];
    const int waves = blockDim.x / 64, wave = threadIdx.x / 64, at = threadIdx.x % LANES, bl = threadIdx.x % 64 / LANES;
    const int groups = (a.Cb + BLOCKS - 1) / BLOCKS, n = blockIdx.x / groups;
    const bool live = blockIdx.x % groups * BLOCKS + bl < a.Cb;
    const int cb = live ? blockIdx.x % groups * BLOCKS + bl : a.Cb - 1;
    const int len = seq_length(a.lengths, n, a.L);
    const T *x = static_cast<const T *>(a.x) + n * a.vx.n + cb * a.vx.c;
    const T *f = static_cast<const T *>(a.f) + n * a.vf.n + cb * a.vf.c;
    const T *i = static_cast<const T *>(a.i) + n * a.vi.n + cb * a.vi.c;
    const T *z = a.z ? static_cast<const T *>(a.z) + n * a.vz.n + cb * a.vz.c : nullptr;
    T *y = static_cast<T *>(a.y) + n * a.vy.n + cb * a.vy.c;
    const int slot = a.slots ? a.slots[n] : n;
    const bool has_slot = slot >= 0 && slot < a.n_slots;
    const RecParams<V> par(a, cb);
    float state[V] = {};
    if (a.state_in && has_slot) seq_vector<V>(a.state_in + (long long)slot * a.Cp, cb, state);
    const int each = waves * LANES * P;
    int turn = 0;
    for (long long base = 0; base < a.L; base += each, turn ^= 1) {
        const long long l0 = base + (wave * LANES + at) * P;
        float A[V], H[V], pa[P][V], ph[P][V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            A[k] = 1;
            H[k] = 0;
        }
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const long long l = l0 + j;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                pa[j][k] = 1;
                ph[j][k] = 0;
            }
            if (l < len) {
                float fx[V], ff[V], fi[V];
                SeqElem<T>::unpack(seq_load(x + l * a.vx.l), fx);
                SeqElem<T>::unpack(seq_load(f + l * a.vf.l), ff);
                SeqElem<T>::unpack(seq_load(i + l * a.vi.l), fi);
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const float t = par.A[k] * rec_gate(ff[k], par.f[k]);
                    pa[j][k] = seq_exp2(t);
                    ph[j][k] = __builtin_amdgcn_sqrtf(rec_rest(t, pa[j][k])) * rec_gate(fi[k], par.i[k]) * fx[k];
                }
            }
#pragma unroll
            for (int k = 0; k < V; ++k) {
                H[k] = fmaf(pa[j][k], H[k], ph[j][k]);
                A[k] *= pa[j][k];
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
        float h[V];  // before the wave's positions
        for (int w = 0; w < waves; ++w)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if (w == wave) h[k] = state[k];
                state[k] = fmaf(runs[turn][w][bl][0][k], state[k], runs[turn][w][bl][1][k]);
            }
#pragma unroll
        for (int k = 0; k < V; ++k) {  // before the lane's
            float la = rec_near<1, false>(1.0f, A[k]), lh = rec_near0<1, false>(H[k]);
            if (at == 0) la = 1, lh = 0;
            h[k] = fmaf(la, h[k], lh);
        }
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const long long l = l0 + j;
            seq_u32x4 out = {};
#pragma unroll
            for (int k = 0; k < V; ++k) h[k] = fmaf(pa[j][k], h[k], ph[j][k]);
            if (l < len) {
                float o[V], fz[V];
                if (z) SeqElem<T>::unpack(seq_load(z + l * a.vz.l), fz);
#pragma unroll
                for (int k = 0; k < V; ++k) o[k] = z ? h[k] * fz[k] * seq_sigmoid(fz[k]) : h[k];
                out = SeqElem<T>::pack(o);
            }
            if (live && l < a.L) seq_store_result<PAST>(y + l * a.vy.l, out);
        }
    }
    if (a.state_out && has_slot && live && wave == 0 && at == 0) {
        float *to = a.state_out + (long long)slot * a.Cp + (long long)cb * V;
#pragma unroll
        for (int k = 0; k < V; k += 4) *reinterpret_cast<seq_f32x4 *>(to + k) = seq_f32x4{state[k], state[k + 1], state[k + 2], state[k + 3]};
    }
}

template <typename T>
__global__ __launch_bounds__(64) void seq_rec_step_kernel(const SeqRecArgs a)
{
    constexpr int V = SeqElem<T>::V;
    const long long t = (long long)blockIdx.x * 64 + threadIdx.x;
    if (t >= (long long)a.N * a.Cb) return;
    const int n = (int)(t / a.Cb), cb = (int)(t % a.Cb);
    const int slot = a.slots ? a.slots[n] : n;
    T *y = static_cast<T *>(a.y) + n * a.vy.n + cb * a.vy.c;
    if (slot < 0 || slot >= a.n_slots) {
        seq_store(y, seq_u32x4{});
        return;
    }
    float *to = a.state_out + (long long)slot * a.Cp + (long long)cb * V;
    float h[V], fx[V], ff[V], fi[V], fz[V];
    seq_vector<V>(to, 0, h);
    SeqElem<T>::unpack(seq_load(static_cast<const T *>(a.x) + n * a.vx.n + cb * a.vx.c), fx);
    SeqElem<T>::unpack(seq_load(static_cast<const T *>(a.f) + n * a.vf.n + cb * a.vf.c), ff);
    SeqElem<T>::unpack(seq_load(static_cast<const T *>(a.i) + n * a.vi.n + cb * a.vi.c), fi);
    if (a.z) SeqElem<T>::unpack(seq_load(static_cast<const T *>(a.z) + n * a.vz.n + cb * a.vz.c), fz);
    const RecParams<V> par(a, cb);
    float o[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const float e = par.A[k] * rec_gate(ff[k], par.f[k]), d = seq_exp2(e);
        h[k] = fmaf(d, h[k], __builtin_amdgcn_sqrtf(rec_rest(e, d)) * rec_gate(fi[k], par.i[k]) * fx[k]);
        o[k] = a.z ? h[k] * fz[k] * seq_sigmoid(fz[k]) : h[k];
    }
    seq_store(y, SeqElem<T>::pack(o));
#pragma unroll
    for (int k = 0; k < V; k += 4) *reinterpret_cast<seq_f32x4 *>(to + k) = seq_f32x4{h[k], h[k + 1], h[k + 2], h[k + 3]};
}

template <typename T, int LANES>
hipError_t launch_lanes(const SeqRecArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)((long long)a.N * seq_rec_groups(a.Cb, LANES));
    if (a.past)
        seq_rec_fwd_kernel<T, LANES, kSeqRecPositions, true><<<grid, 64 * a.waves, 0, s>>>(a);
    else
        seq_rec_fwd_kernel<T, LANES, kSeqRecPositions, false><<<grid, 64 * a.waves, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_t(const SeqRecArgs &a, hipStream_t s)
{
    return a.lanes == 16 ? launch_lanes<T, 16>(a, s) : launch_lanes<T, 4>(a, s);
}
template <typename T>
hipError_t launch_step(const SeqRecArgs &a, hipStream_t s)
{
    seq_rec_step_kernel<T><<<(unsigned)(((long long)a.N * a.Cb + 63) / 64), 64, 0, s>>>(a);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_seq_rec_fwd(int dtype, const SeqRecArgs &a, hipStream_t s) { return dtype == SEQ_BF16 ? launch_t<unsigned short>(a, s) : launch_t<float>(a, s); }
hipError_t launch_seq_rec_step(int dtype, const SeqRecArgs &a, hipStream_t s) { return dtype == SEQ_BF16 ? launch_step<unsigned short>(a, s) : launch_step<float>(a, s); }

}  // namespace convmi
