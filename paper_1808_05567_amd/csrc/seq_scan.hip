// Selective state space scan, forward and over one new position.
//
//   h[s] = exp(d A[s]) h[s] + d x B[s],   y = sum_s C[s] h[s] + D x,   y *= z sigmoid(z)
//
// One lane a channel, its states in registers, one position after the other.  B and C are the same for all channels of a
// group: lane i of each row of 16 holds state i, and an instruction takes it from there (row_newbcast) at no cost.
//
// Five operations and an exponential a state and position against 2 to 8 bytes a position: bound by the vector units.  Too few
// channels to fill the machine are split along the positions too: a first launch takes each run of positions from a state of
// zeros and notes the state it ends in and the sum of d, from which what the run does to any state follows:
// exp(A sum d) h + that; a second puts these together in order; a third goes through each run from the right state.
#include "seq_internal.h"

namespace convmi {
namespace {

constexpr int kWaves = 4;  // a workgroup

template <int SP>
struct States {
    static constexpr int R = (SP + 15) / 16;  // registers that hold SP states of B or C, 16 lanes each
};

template <int I, int SP, bool OUT>
static __device__ __forceinline__ void seq_step(float (&h)[SP], const float (&A)[SP], float d, float dx, const float (&B)[States<SP>::R],
                                                const float (&C)[States<SP>::R], float (&y)[4])
{
    if constexpr (I < SP) {
        const float a = seq_exp2(d * A[I]);
        h[I] = fmaf(a, h[I], seq_row_lane<I % 16>(B[I / 16]) * dx);
        if constexpr (OUT) y[I % 4] = fmaf(seq_row_lane<I % 16>(C[I / 16]), h[I], y[I % 4]);
        seq_step<I + 1, SP, OUT>(h, A, d, dx, B, C, y);
    }
}

// The same for the ends of a run, in both directions: h from zeros, and the gradient g of the state before the run where none comes
// from behind it, the sum over its positions of C dy times the product P of all decays up to there.
template <int I, int SP>
static __device__ __forceinline__ void seq_step_ends(float (&h)[SP], float (&g)[SP], float (&P)[SP], const float (&A)[SP], float d, float dx, float dy,
                                                     const float (&B)[States<SP>::R], const float (&C)[States<SP>::R])
{
    if constexpr (I < SP) {
        const float a = seq_exp2(d * A[I]);
        h[I] = fmaf(a, h[I], seq_row_lane<I % 16>(B[I / 16]) * dx);
        P[I] *= a;
        g[I] = fmaf(P[I], seq_row_lane<I % 16>(C[I / 16]) * dy, g[I]);
        seq_step_ends<I + 1, SP>(h, g, P, A, d, dx, dy, B, C);
    }
}

// MODE 0: the state a run ends in from zeros; 1: results (chunks == 1: the whole sequence); 2: the ends for the gradients.
template <typename T, int SP, int MODE>
__global__ __launch_bounds__(64 * kWaves) void seq_scan_kernel(const SeqScanArgs a)
{
    constexpr int V = SeqElem<T>::V, R = States<SP>::R, CB = 64 / V, NV = CB * 8 / 64;
    constexpr bool OUT = MODE == 1, ENDS = MODE == 2, ALL = OUT || ENDS;
    constexpr int SG = ENDS ? SP : 1;
    constexpr int E = SP / 8, BL = SP < 16 ? SP : 16;  // elements of B of 8 positions a lane loads; lanes of a row that hold states
    __shared__ float bcs[kWaves][ALL ? 2 : 1][8 * SP];
    __shared__ __align__(16) T tiles[kWaves][ALL ? 4 : 2][8 * 64];  // x, dt, z, y (ENDS: dy) of 8 positions x 64 channels
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    auto &tile = tiles[wave];
    auto &bc = bcs[wave];
    // (waves share nothing: four a workgroup are one on each SIMD)
    long long t = (long long)blockIdx.x * kWaves + wave;
    const int tl = (int)(t % a.tiles);
    t /= a.tiles;
    const int g = (int)(t % a.G);
    t /= a.G;
    const int chunk = (int)(t % a.chunks), n = (int)(t / a.chunks);
    if (n >= a.N) return;
    const int c0 = g * a.CG + tl * 64, c_end = min(c0 + 64, (g + 1) * a.CG);
    const int c = c0 + lane;
    const bool live = c < c_end;
    const int cs = live ? c : c0;
    const int len = seq_length(a.lengths, n, a.L);
    const int begin = chunk * a.chunk, end = min(begin + a.chunk, a.L), stop = min(end, len);

    float A[SP], h[SP], gr[SG], P[SG];
#pragma unroll
    for (int s = 0; s < SP; ++s) {
        A[s] = s < a.S ? a.A[(long long)s * a.Cp + cs] * kLog2e : 0.0f;
        h[s] = 0;
        if (ENDS) gr[s % SG] = 0, P[s % SG] = 1;
    }
    const float bias = a.dt_bias ? a.dt_bias[cs] : 0.0f, D = OUT && a.D ? a.D[cs] : 0.0f;
    const int slot = a.slots ? a.slots[n] : n;
    const bool has_slot = slot >= 0 && slot < a.n_slots;
    const long long at = ((long long)n * a.chunks + chunk) * a.S * a.Cp + cs;
    if (OUT) {
        if (a.chunks > 1) {
#pragma unroll
            for (int s = 0; s < SP; ++s)
                if (s < a.S) h[s] = a.hl[at + (long long)s * a.Cp];
        } else if (a.state_in && has_slot) {
#pragma unroll
            for (int s = 0; s < SP; ++s)
                if (s < a.S) h[s] = a.state_in[((long long)slot * a.S + s) * a.Cp + cs];
        }
    }

    // what a lane loads and stores: block cbl of the tile's, position ll of 8
    const T *px[NV], *pd[NV], *pz[NV];
    const T *pg[NV];
    T *py[NV];
    bool in[NV];
    int ll[NV], to[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int e = lane + 64 * i, cbl = e / 8;
        ll[i] = e % 8;
        to[i] = ll[i] * 64 + cbl * V;
        in[i] = c0 + cbl * V < c_end;
        const int cb = c0 / V + (in[i] ? cbl : 0);
        px[i] = static_cast<const T *>(a.x) + n * a.vx.n + cb * a.vx.c;
        pd[i] = static_cast<const T *>(a.dt) + n * a.vdt.n + cb * a.vdt.c;
        if (ALL) pz[i] = a.z ? static_cast<const T *>(a.z) + n * a.vz.n + cb * a.vz.c : nullptr;
        if (ENDS) pg[i] = static_cast<const T *>(a.dy) + n * a.vdy.n + cb * a.vdy.c;
        if (OUT) {
            py[i] = static_cast<T *>(a.y) + n * a.vy.n + cb * a.vy.c;
        }
    }
    // B and C: positions and states of the elements that a lane loads
    const T *pB[E], *pC[E];
    bool has[E];
#pragma unroll
    for (int r = 0; r < E; ++r) {
        const int s = (lane + 64 * r) % SP;
        has[r] = s < a.S;
        const int e = g * a.S + (has[r] ? s : 0);
        pB[r] = static_cast<const T *>(a.B) + n * a.vB.n + e / V * a.vB.c + e % V;
        if (ALL) pC[r] = static_cast<const T *>(a.C) + n * a.vC.n + e / V * a.vC.c + e % V;
    }

    seq_u32x4 nx[NV], nd[NV], nz[NV], ng[NV];
    T nB[E], nC[E];
    auto fetch = [&](int l0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int l = l0 + ll[i];
            const bool ok = in[i] && l < stop;
            nx[i] = nd[i] = nz[i] = ng[i] = seq_u32x4{};
            if (ok) {
                nx[i] = seq_load(px[i] + l * a.vx.l);
                nd[i] = seq_load(pd[i] + l * a.vdt.l);
                if (ALL && a.z) nz[i] = seq_load(pz[i] + l * a.vz.l);
                if (ENDS) ng[i] = seq_load(pg[i] + l * a.vdy.l);
            }
        }
#pragma unroll
        for (int r = 0; r < E; ++r) {
            const int l = l0 + (lane + 64 * r) / SP;
            const bool ok = has[r] && l < stop;
            nB[r] = ok ? pB[r][l * a.vB.l] : T(0);
            if (ALL) nC[r] = ok ? pC[r][l * a.vC.l] : T(0);
        }
    };
    float sum_d = 0;
    if (begin < stop) fetch(begin);
    for (int l0 = begin; l0 < stop; l0 += 8) {
        seq_wave_sync();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            seq_store(tile[0] + to[i], nx[i]);
            seq_store(tile[1] + to[i], nd[i]);
            if (ALL) seq_store(tile[ALL ? 2 : 0] + to[i], nz[i]);
            if (ENDS) seq_store(tile[ALL ? 3 : 0] + to[i], ng[i]);
        }
#pragma unroll
        for (int r = 0; r < E; ++r) {
            bc[0][lane + 64 * r] = SeqElem<T>::get(nB[r]);
            if (ALL) bc[ALL ? 1 : 0][lane + 64 * r] = SeqElem<T>::get(nC[r]);
        }
        seq_wave_sync();
        if (l0 + 8 < stop) fetch(l0 + 8);
        if (ENDS && l0 > begin && live) {
            const long long m = ((long long)n * a.chunks + chunk) * kSeqMarks + (l0 - begin) / 8 - 1;
#pragma unroll
            for (int s = 0; s < SP; ++s)
                if (s < a.S) a.marks[(m * a.S + s) * a.Cp + c] = h[s];
            a.md[m * a.Cp + c] = sum_d;
        }
        // one position after the other, its numbers read from LDS during the one before.  (Left to itself the compiler spreads the
        // eight over each other, in all registers there are.)
        struct Position {
            T x, d, z, dy;
            float B[R], C[R];
        };
        const auto read = [&](int j) {
            Position p = {};
            p.x = tile[0][j * 64 + lane];
            p.d = tile[1][j * 64 + lane];
            if (ALL) p.z = tile[ALL ? 2 : 0][j * 64 + lane];
            if (ENDS) p.dy = tile[ALL ? 3 : 0][j * 64 + lane];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                p.B[r] = bc[0][j * SP + lane % BL + 16 * r];
                if (ALL) p.C[r] = bc[ALL ? 1 : 0][j * SP + lane % BL + 16 * r];
            }
            return p;
        };
        Position now = read(0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            Position next = {};
            if (j < 7) next = read(j + 1);
            const float x = SeqElem<T>::get(now.x), raw = SeqElem<T>::get(now.d) + bias, soft = seq_softplus(raw);
            float d = a.softplus ? soft : raw;
            if (l0 + j >= stop) d = 0;  // (what follows the end changes nothing: x, B, C and z are zero there)
            float gate = 1;
            if (ALL) {
                const float z = SeqElem<T>::get(now.z), of_z = z * seq_sigmoid(z);
                gate = a.z ? of_z : 1.0f;
            }
            float y[4] = {};
            if constexpr (ENDS)
                seq_step_ends<0, SP>(h, gr, P, A, d, d * x, SeqElem<T>::get(now.dy) * gate, now.B, now.C);
            else
                seq_step<0, SP, OUT>(h, A, d, d * x, now.B, now.C, y);
            sum_d += d;
            if (OUT) {
                const float o = fmaf(D, x, (y[0] + y[1]) + (y[2] + y[3])) * gate;
                tile[OUT ? 3 : 0][j * 64 + lane] = SeqElem<T>::put(live ? o : 0.0f);
            }
            now = next;
            __builtin_amdgcn_sched_barrier(0);
        }
        if (OUT) {
            seq_wave_sync();
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (in[i] && l0 + ll[i] < end)
                    seq_store(py[i] + (l0 + ll[i]) * a.vy.l, l0 + ll[i] < stop ? seq_load(tile[OUT ? 3 : 0] + to[i]) : seq_u32x4{});
        }
    }
    if (OUT) {
        // zeros past the end, from where the last eight positions stopped
        for (int l0 = begin + (max(stop - begin, 0) + 7) / 8 * 8; l0 < end; l0 += 8)
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (in[i] && l0 + ll[i] < end) seq_store(py[i] + (l0 + ll[i]) * a.vy.l, seq_u32x4{});
        // the run that the last position is in stores the state, the first one that of an empty sequence
        const bool last = len == 0 ? chunk == 0 : begin < len && len <= begin + a.chunk;
        if (a.state_out && has_slot && last && live)
#pragma unroll
            for (int s = 0; s < SP; ++s)
                if (s < a.S) a.state_out[((long long)slot * a.S + s) * a.Cp + c] = h[s];
    } else if (live) {
#pragma unroll
        for (int s = 0; s < SP; ++s)
            if (s < a.S) {
                a.hl[at + (long long)s * a.Cp] = h[s];
                if (ENDS) a.gl[at + (long long)s * a.Cp] = gr[s % SG];
            }
        a.sd[((long long)n * a.chunks + chunk) * a.Cp + c] = sum_d;
    }
}

// The state at the start of each run from those the runs end in, in place; the gradient at the end of each the same way, from the back.
__global__ __launch_bounds__(256) void seq_scan_join_kernel(const SeqScanArgs a)
{
    const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
    const long long state = (long long)a.S * a.Cp;
    if (t >= a.N * state) return;
    const int n = (int)(t / state), c = (int)(t % a.Cp);
    const long long e = t % state;
    if (c >= a.Ch) return;
    const int slot = a.slots ? a.slots[n] : n;
    const float A = a.A[e] * kLog2e;
    const float first = a.state_in && slot >= 0 && slot < a.n_slots ? a.state_in[slot * state + e] : 0.0f;
    const float *sd = a.sd + (long long)n * a.chunks * a.Cp + c;
    // what a run adds and the sum of its d come 16 runs at a time, ahead of the chain that they go into
    const auto chain = [&](float *ends, float h, bool back) {
        ends += (long long)n * a.chunks * state + e;
        for (int k0 = 0; k0 < a.chunks; k0 += 16) {
            float own[16], d[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int k = back ? a.chunks - 1 - k0 - i : k0 + i;
                const bool ok = k0 + i < a.chunks;
                own[i] = ok ? ends[k * state] : 0.0f;
                d[i] = ok ? sd[(long long)k * a.Cp] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int k = back ? a.chunks - 1 - k0 - i : k0 + i;
                if (k0 + i < a.chunks) ends[k * state] = h;
                h = fmaf(seq_exp2(A * d[i]), h, own[i]);
            }
        }
    };
    chain(a.hl, first, false);
    if (a.gl) chain(a.gl, 0.0f, true);
}

// One new position: 64 channels a workgroup, its four waves taking every fourth state.
template <typename T>
__global__ __launch_bounds__(256) void seq_scan_step_kernel(const SeqScanArgs a)
{
    constexpr int V = SeqElem<T>::V;
    __shared__ float lds[256];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int ct = (a.Cp + 63) / 64, n = blockIdx.x / ct, c = blockIdx.x % ct * 64 + lane;
    const int slot = a.slots ? a.slots[n] : n;
    const bool has_slot = slot >= 0 && slot < a.n_slots;
    const bool live = c < a.Ch;
    auto at = [&](const SeqView &v, int e) { return n * v.n + e / V * v.c + e % V; };
    float x = 0, y = 0;
    if (live && has_slot) {
        const int g = c / a.CG;
        x = SeqElem<T>::get(static_cast<const T *>(a.x)[at(a.vx, c)]);
        float d = SeqElem<T>::get(static_cast<const T *>(a.dt)[at(a.vdt, c)]) + (a.dt_bias ? a.dt_bias[c] : 0.0f);
        if (a.softplus) d = seq_softplus(d);
        float *h = a.state_out + (long long)slot * a.S * a.Cp + c;
#pragma unroll 4
        for (int s = wave; s < a.S; s += 4) {
            const float B = SeqElem<T>::get(static_cast<const T *>(a.B)[at(a.vB, g * a.S + s)]);
            const float C = SeqElem<T>::get(static_cast<const T *>(a.C)[at(a.vC, g * a.S + s)]);
            const float next = fmaf(seq_exp2(d * (a.A[(long long)s * a.Cp + c] * kLog2e)), h[(long long)s * a.Cp], d * x * B);
            h[(long long)s * a.Cp] = next;
            y = fmaf(C, next, y);
        }
    }
    lds[threadIdx.x] = y;
    __syncthreads();
    if (wave != 0 || c >= a.Cp) return;
    y = (lds[lane] + lds[lane + 64]) + (lds[lane + 128] + lds[lane + 192]);
    if (live && has_slot) {
        if (a.D) y = fmaf(a.D[c], x, y);
        if (a.z) {
            const float z = SeqElem<T>::get(static_cast<const T *>(a.z)[at(a.vz, c)]);
            y *= z * seq_sigmoid(z);
        }
    }
    static_cast<T *>(a.y)[at(a.vy, c)] = SeqElem<T>::put(y);
}

template <typename T, int SP>
hipError_t launch(const SeqScanArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)(((long long)a.N * a.G * a.tiles * a.chunks + kWaves - 1) / kWaves);
    if (a.chunks > 1) {
        seq_scan_kernel<T, SP, 0><<<grid, 64 * kWaves, 0, s>>>(a);
        seq_scan_join_kernel<<<(unsigned)(((long long)a.N * a.S * a.Cp + 255) / 256), 256, 0, s>>>(a);
    }
    seq_scan_kernel<T, SP, 1><<<grid, 64 * kWaves, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, int SP>
hipError_t launch_ends(const SeqScanArgs &a, hipStream_t s)
{
    seq_scan_kernel<T, SP, 2><<<(unsigned)(((long long)a.N * a.G * a.tiles * a.chunks + kWaves - 1) / kWaves), 64 * kWaves, 0, s>>>(a);
    if (a.chunks > 1) seq_scan_join_kernel<<<(unsigned)(((long long)a.N * a.S * a.Cp + 255) / 256), 256, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_t(bool ends, const SeqScanArgs &a, hipStream_t s)
{
    switch (seq_scan_states(a.S)) {
        case 8: return ends ? launch_ends<T, 8>(a, s) : launch<T, 8>(a, s);
        case 16: return ends ? launch_ends<T, 16>(a, s) : launch<T, 16>(a, s);
        case 32: return ends ? launch_ends<T, 32>(a, s) : launch<T, 32>(a, s);
    }
    return ends ? launch_ends<T, 64>(a, s) : launch<T, 64>(a, s);
}
}  // namespace

hipError_t launch_seq_scan_fwd(int dtype, const SeqScanArgs &a, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch_t<unsigned short>(false, a, s) : launch_t<float>(false, a, s);
}
hipError_t launch_seq_scan_ends(int dtype, const SeqScanArgs &a, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch_t<unsigned short>(true, a, s) : launch_t<float>(true, a, s);
}
hipError_t launch_seq_scan_step(int dtype, const SeqScanArgs &a, hipStream_t s)
{
    const unsigned grid = (unsigned)((long long)a.N * ((a.Cp + 63) / 64));
    if (dtype == SEQ_BF16)
        seq_scan_step_kernel<unsigned short><<<grid, 256, 0, s>>>(a);
    else
        seq_scan_step_kernel<float><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace convmi
