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
//
// Measured, one sequence of 4096 positions, 2048 channels, 16 states, bf16, 64 runs: 35, 7 and 49 us.  A position of 16 states takes the first launch
// some 350 clocks where its operations take 320; the step's softplus and the loads of a position another 130 each, and what is left is the
// launches and the waves' first trips to memory.
#include "seq_internal.h"

namespace convmi {
namespace {

constexpr int kWaves = kSeqScanWaves;  // a workgroup

template <int SP>
struct States {
    static constexpr int R = (SP + 15) / 16;  // registers that hold SP states of B or C, 16 lanes each
};

// One position of states 16 Q ... + 15.  In steps whose operations do not wait for each other, held apart: left to itself the compiler
// puts each exponential right before its use, and a wave waits for every one.
template <int I, int N>
static __device__ __forceinline__ void seq_spread(float B, float dx, float (&to)[16])
{
    if constexpr (I < N) {
        to[I] = seq_row_lane<I>(B) * dx;
        seq_spread<I + 1, N>(B, dx, to);
    }
}
template <int I, int N>
static __device__ __forceinline__ void seq_spread(float C, float (&to)[16])
{
    if constexpr (I < N) {
        to[I] = seq_row_lane<I>(C);
        seq_spread<I + 1, N>(C, to);
    }
}
template <int Q, int SP, bool OUT, bool ENDS>
static __device__ __forceinline__ void seq_step(float (&h)[SP], const float (&A)[SP], float (&g)[ENDS ? SP : 1], float (&P)[ENDS ? SP : 1], float d, float dx,
                                                float dy, const float (&B)[States<SP>::R], const float (&C)[States<SP>::R], float (&y)[4])
{
    if constexpr (Q < States<SP>::R) {
        constexpr int N = SP < 16 ? SP : 16, S0 = 16 * Q;
        float a[16], b[16], c[16];
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] = d * A[S0 + i];
        if constexpr (OUT) seq_spread<0, N>(C[Q], c);
        if constexpr (ENDS) seq_spread<0, N>(C[Q], dy, c);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] = seq_exp2(a[i]);
        seq_spread<0, N>(B[Q], dx, b);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < N; ++i) h[S0 + i] = fmaf(a[i], h[S0 + i], b[i]);
        if constexpr (ENDS)
#pragma unroll
            for (int i = 0; i < N; ++i) P[S0 + i] *= a[i];
        if constexpr (ENDS)
#pragma unroll
            for (int i = 0; i < N; ++i) g[S0 + i] = fmaf(P[S0 + i], c[i], g[S0 + i]);
        if constexpr (OUT)
#pragma unroll
            for (int i = 0; i < N; ++i) y[i % 4] = fmaf(c[i], h[S0 + i], y[i % 4]);
        __builtin_amdgcn_sched_barrier(0);
        seq_step<Q + 1, SP, OUT, ENDS>(h, A, g, P, d, dx, dy, B, C, y);
    }
}

// MODE 0: the state a run ends in from zeros; 1: results (chunks == 1: the whole sequence); 2: the ends for the gradients: h from zeros,
// noted every 8 positions, and the gradient g of the state before the run where none comes from behind it, the sum over its
// positions of C dy times the product P of all decays up to there.
//
// What concerns single numbers of the tensors (the step's softplus, the gate) is done to the blocks that a lane loads, eight positions at a time;
// LDS turns blocks into channels and back.
template <typename T, int SP, int MODE>
__global__ __launch_bounds__(64 * kWaves) void seq_scan_kernel(const SeqScanArgs a)
{
    constexpr int V = SeqElem<T>::V, R = States<SP>::R, CB = 64 / V, NV = CB * 8 / 64;
    constexpr bool OUT = MODE == 1, ENDS = MODE == 2, ALL = OUT || ENDS;
    constexpr int SG = ENDS ? SP : 1;
    constexpr int E = SP / 8, BL = SP < 16 ? SP : 16;  // elements of B of 8 positions a lane loads; lanes of a row that hold states
    constexpr int W = 64 + 4;                          // (rows a block apart: the eight lanes with the same block write to different banks)
    struct __align__(16) Lds {
        float d[8][W], dx[8][W], dy[ENDS ? 8 : 1][W];  // d's rows take y once they are done with
        float B[8 * SP], C[ALL ? 8 * SP : 1];
    };
    __shared__ __align__(16) Lds all[kWaves];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    Lds &my = all[wave];
    // (waves share nothing: four a workgroup are one on each SIMD)
    unsigned t = blockIdx.x * kWaves + wave;  // (of at most 2^26 waves)
    // (more than 32 states in two waves where no sum over them is formed: one has not the registers)
    const int parts = OUT ? 1 : (a.S + SP - 1) / SP, s0 = OUT ? 0 : t % (unsigned)parts * SP, S = min(a.S - s0, SP);
    if (!OUT) t /= (unsigned)parts;
    const int tl = t % (unsigned)a.tiles;
    t /= (unsigned)a.tiles;
    const int g = t % (unsigned)a.G;
    t /= (unsigned)a.G;
    const int chunk = t % (unsigned)a.chunks, n = t / (unsigned)a.chunks;
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
        A[s] = s < S ? seq_decay(a.A[(long long)(s0 + s) * a.Cp + cs]) : 0.0f;
        h[s] = 0;
        if (ENDS) gr[s % SG] = 0, P[s % SG] = 1;
    }
    const int slot = a.slots ? a.slots[n] : n;
    const bool has_slot = slot >= 0 && slot < a.n_slots;
    const long long run = (long long)n * a.chunks + chunk, at = (run * a.S + s0) * a.Cp + cs;
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

    // A lane's blocks: block cbl of the tile's, position ll of 8.  Its places in the tensors move on by eight positions at a time: formed
    // anew, they would wait for the kernel's arguments each time.
    const int ll = lane % 8;
    bool in[NV];
    int to[NV];
    float bias[NV][V] = {}, D[NV][V] = {};
    const T *px[NV], *pd[NV], *pz[NV], *pg[NV];
    T *py[NV];
    auto place = [&](const void *p, const SeqView &v, int cb) { return static_cast<const T *>(p) + n * v.n + cb * v.c + (begin + ll) * v.l; };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int cbl = (lane + 64 * i) / 8;
        to[i] = cbl * V;
        in[i] = c0 + cbl * V < c_end;
        const int cb = c0 / V + (in[i] ? cbl : 0);
        if (a.dt_bias) seq_vector<V>(a.dt_bias, cb, bias[i]);
        if (OUT && a.D) seq_vector<V>(a.D, cb, D[i]);
        px[i] = place(a.x, a.vx, cb);
        pd[i] = place(a.dt, a.vdt, cb);
        if (ALL && a.z) pz[i] = place(a.z, a.vz, cb);
        if (ENDS) pg[i] = place(a.dy, a.vdy, cb);
        if (OUT) py[i] = const_cast<T *>(place(a.y, a.vy, cb));
    }
    const long long on_x = 8 * a.vx.l, on_d = 8 * a.vdt.l, on_z = 8 * a.vz.l, on_g = 8 * a.vdy.l, on_y = 8 * a.vy.l;
    // B and C: element r of a lane is state lane % SP of position (lane + 64 r) / SP
    const int e_of = g * a.S + s0 + (lane % SP < S ? lane % SP : 0), l_of = lane / SP;
    const bool has = lane % SP < S;
    const T *pB = static_cast<const T *>(a.B) + n * a.vB.n + e_of / V * a.vB.c + e_of % V + (begin + l_of) * a.vB.l;
    const T *pC = ALL ? static_cast<const T *>(a.C) + n * a.vC.n + e_of / V * a.vC.c + e_of % V + (begin + l_of) * a.vC.l : nullptr;
    const long long on_B = 64 / SP * a.vB.l, on_C = 64 / SP * a.vC.l;  // (64 / SP positions an element: E elements are eight)

    seq_u32x4 nx[NV], nd[NV], nz[NV], ng[NV];
    T nB[E], nC[E];
    const bool gated = ALL && a.z;
    auto fetch = [&](int l0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            nx[i] = nd[i] = nz[i] = ng[i] = seq_u32x4{};
            if (in[i] && l0 + ll < stop) {
                nx[i] = seq_load(px[i]);
                nd[i] = seq_load(pd[i]);
                if (gated) nz[i] = seq_load(pz[i]);
                if (ENDS) ng[i] = seq_load(pg[i]);
            }
            px[i] += on_x;
            pd[i] += on_d;
            if (gated) pz[i] += on_z;
            if (ENDS) pg[i] += on_g;
        }
#pragma unroll
        for (int r = 0; r < E; ++r) {
            const bool ok = has && l0 + l_of + r * (64 / SP) < stop;
            nB[r] = ok ? *pB : T(0);
            pB += on_B;
            if (ALL) {
                nC[r] = ok ? *pC : T(0);
                pC += on_C;
            }
        }
    };
    float sum_d = 0;
    if (begin < stop) fetch(begin);
    for (int l0 = begin; l0 < stop; l0 += 8) {
        float x[NV][V], gate[NV][V];
        const bool inside = l0 + ll < stop;
        seq_wave_sync();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float d[V], z[V], dy[V], dx[V];
            SeqElem<T>::unpack(nx[i], x[i]);
            SeqElem<T>::unpack(nd[i], d);
            SeqElem<T>::unpack(nz[i], z);
            SeqElem<T>::unpack(ng[i], dy);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float raw = d[j] + bias[i][j], soft = seq_softplus(raw);
                // (what follows the end changes nothing: x, B, C, dy are zero there too)
                d[j] = !inside ? 0.0f : a.softplus ? soft : raw;
                dx[j] = d[j] * x[i][j];
                gate[i][j] = 1;
                if (ALL) gate[i][j] = gated ? z[j] * seq_sigmoid(z[j]) : 1.0f;
                if (ENDS) dy[j] *= gate[i][j];
            }
#pragma unroll
            for (int j = 0; j < V; j += 4) {
                *reinterpret_cast<seq_f32x4 *>(&my.d[ll][to[i] + j]) = seq_f32x4{d[j], d[j + 1], d[j + 2], d[j + 3]};
                *reinterpret_cast<seq_f32x4 *>(&my.dx[ll][to[i] + j]) = seq_f32x4{dx[j], dx[j + 1], dx[j + 2], dx[j + 3]};
                if (ENDS) *reinterpret_cast<seq_f32x4 *>(&my.dy[ENDS ? ll : 0][to[i] + j]) = seq_f32x4{dy[j], dy[j + 1], dy[j + 2], dy[j + 3]};
            }
        }
#pragma unroll
        for (int r = 0; r < E; ++r) {
            my.B[lane + 64 * r] = SeqElem<T>::get(nB[r]);
            if (ALL) my.C[ALL ? lane + 64 * r : 0] = SeqElem<T>::get(nC[r]);
        }
        seq_wave_sync();
        if (l0 + 8 < stop) fetch(l0 + 8);
        if (ENDS && l0 > begin && live) {
            const long long m = run * a.notes + (l0 - begin) / 8 - 1;
#pragma unroll
            for (int s = 0; s < SP; ++s)
                if (s < S) a.marks[(m * a.S + s0 + s) * a.Cp + c] = h[s];
            if (s0 == 0) a.md[m * a.Cp + c] = sum_d;
        }
        // one position after the other, its numbers read from LDS during the one before
        struct Position {
            float d, dx, dy, B[R], C[R];
        };
        const auto read = [&](int j) {
            Position p = {};
            p.d = my.d[j][lane];
            p.dx = my.dx[j][lane];
            if (ENDS) p.dy = my.dy[ENDS ? j : 0][lane];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                p.B[r] = my.B[j * SP + lane % BL + 16 * r];
                if (ALL) p.C[r] = my.C[ALL ? j * SP + lane % BL + 16 * r : 0];
            }
            return p;
        };
        Position now = read(0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            Position next = {};
            if (j < 7) next = read(j + 1);
            float y[4] = {};
            seq_step<0, SP, OUT, ENDS>(h, A, gr, P, now.d, now.dx, now.dy, now.B, now.C, y);
            sum_d += now.d;
            if (OUT) my.d[j][lane] = (y[0] + y[1]) + (y[2] + y[3]);
            now = next;
        }
        if (OUT) {
            seq_wave_sync();
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (!in[i] || l0 + ll >= end) continue;
                float y[V];
#pragma unroll
                for (int j = 0; j < V; j += 4) {
                    const seq_f32x4 q = *reinterpret_cast<const seq_f32x4 *>(&my.d[ll][to[i] + j]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[j + k] = q[k];
                }
#pragma unroll
                for (int j = 0; j < V; ++j) y[j] = inside && c0 + to[i] + j < c_end ? fmaf(D[i][j], x[i][j], y[j]) * gate[i][j] : 0.0f;
                seq_store(py[i], SeqElem<T>::pack(y));
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) py[i] += on_y;
        }
    }
    if (OUT) {
        // zeros past the end, from where the last eight positions stopped
        for (int l0 = begin + (max(stop - begin, 0) + 7) / 8 * 8; l0 < end; l0 += 8)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (in[i] && l0 + ll < end) seq_store(py[i], seq_u32x4{});
                py[i] += on_y;
            }
        // the run that the last position is in stores the state, the first one that of an empty sequence
        const bool last = len == 0 ? chunk == 0 : begin < len && len <= begin + a.chunk;
        if (a.state_out && has_slot && last && live)
#pragma unroll
            for (int s = 0; s < SP; ++s)
                if (s < a.S) a.state_out[((long long)slot * a.S + s) * a.Cp + c] = h[s];
    } else if (live) {
#pragma unroll
        for (int s = 0; s < SP; ++s)
            if (s < S) {
                a.hl[at + (long long)s * a.Cp] = h[s];
                if (ENDS) a.gl[at + (long long)s * a.Cp] = gr[s % SG];
            }
        if (s0 == 0) a.sd[run * a.Cp + c] = sum_d;
    }
}

// The state at the start of each run from those the runs end in, in place; the gradient at the end of each the same way, from the back.  The
// waves of a workgroup (one per 16 runs, up to 16) take a part each of the runs of 64 columns: what a part does to a state is put
// together first, then it is gone through again from the right one.  (One thread for all runs: 2 x 174 of them, both ways, 256 channels, 16 states, 30 us; so 11.)
__global__ __launch_bounds__(64 * kSeqJoinWaves) void seq_scan_join_kernel(const SeqScanArgs a)
{
    __shared__ float of_zero[kSeqJoinWaves][64], of_d[kSeqJoinWaves][64];
    const int lane = threadIdx.x % 64, part = threadIdx.x / 64, parts = blockDim.x / 64;
    const long long state = (long long)a.S * a.Cp, columns = (state + 63) / 64;
    const int n = (int)(blockIdx.x / columns);
    const long long e = blockIdx.x % columns * 64 + lane;
    const int c = (int)(e % a.Cp);
    const bool live = e < state && c < a.Ch;
    const int slot = a.slots ? a.slots[n] : n;
    const float A = live ? seq_decay(a.A[e]) : 0.0f;
    const int each = (a.chunks + parts - 1) / parts, begin = min(part * each, a.chunks), end = min(begin + each, a.chunks);
    const float *sd = a.sd + (long long)n * a.chunks * a.Cp + c;
    const auto chain = [&](float *ends, float first, bool back) {
        ends += (long long)n * a.chunks * state + e;
        // what a run adds and the sum of its d come 16 runs at a time, ahead of the chain that they go into
        float own[16], d[16];
        const auto load = [&](int k0) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int k = back ? a.chunks - 1 - k0 - i : k0 + i;
                const bool ok = live && k0 + i < end;
                own[i] = ok ? ends[k * state] : 0.0f;
                d[i] = ok ? sd[(long long)k * a.Cp] : 0.0f;
            }
        };
        float h = 0, sum = 0;
        for (int k0 = begin; k0 < end; k0 += 16) {
            load(k0);
            if (part == parts - 1) break;  // (no part is after it; up to 16 runs are in registers now)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                h = seq_carry(A * d[i], h, own[i]);
                sum += d[i];
            }
        }
        of_zero[part][lane] = h;
        of_d[part][lane] = sum;
        __syncthreads();
        h = first;
        for (int p = 0; p < part; ++p) h = seq_carry(A * of_d[p][lane], h, of_zero[p][lane]);
        for (int k0 = begin; k0 < end; k0 += 16) {
            if (each > 16) load(k0);  // (or still there)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int k = back ? a.chunks - 1 - k0 - i : k0 + i;
                if (live && k0 + i < end) ends[k * state] = h;
                h = seq_carry(A * d[i], h, own[i]);
            }
        }
        __syncthreads();
    };
    chain(a.hl, live && a.state_in && slot >= 0 && slot < a.n_slots ? a.state_in[slot * state + e] : 0.0f, false);
    if (a.gl) chain(a.gl, 0.0f, true);
}

// One new position: 128 channels a workgroup, two a lane, its four waves each taking four states at a time, all loads of which go ahead of the
// first store.  (One channel a lane, a state at a time: 64 sequences of 4096 channels, 16 states, bf16 13.9 us.)
template <typename T>
__global__ __launch_bounds__(256) void seq_scan_step_kernel(const SeqScanArgs a)
{
    constexpr int V = SeqElem<T>::V;
    __shared__ seq_f32x2 lds[256];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int ct = (a.Cp + 127) / 128, n = blockIdx.x / ct, c = blockIdx.x % ct * 128 + lane * 2;
    const int slot = a.slots ? a.slots[n] : n;
    const bool has_slot = slot >= 0 && slot < a.n_slots;
    struct Two {
        T v[2];
    };
    auto at = [&](const SeqView &v, int e) { return n * v.n + e / V * v.c + e % V; };
    auto two = [&](const void *p, const SeqView &v, float (&f)[2]) {
        const Two t = *reinterpret_cast<const Two *>(static_cast<const T *>(p) + at(v, c));
        f[0] = SeqElem<T>::get(t.v[0]);
        f[1] = SeqElem<T>::get(t.v[1]);
    };
    float x[2] = {}, y[2] = {};
    if (c < a.Ch && has_slot) {
        const int g = c / a.CG;  // (of both: a group is a whole number of blocks)
        float d[2];
        two(a.x, a.vx, x);
        two(a.dt, a.vdt, d);
        const T *B = static_cast<const T *>(a.B) + n * a.vB.n, *C = static_cast<const T *>(a.C) + n * a.vC.n;
        const float *A = a.A + c;
        float *h = a.state_out + (long long)slot * a.S * a.Cp + c;
        for (int s0 = wave * 4; s0 < a.S; s0 += 16) {
            seq_f32x2 was[4], As[4];
            T Bs[4], Cs[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int s = min(s0 + j, a.S - 1), e = g * a.S + s;
                was[j] = *reinterpret_cast<const seq_f32x2 *>(h + (long long)s * a.Cp);
                As[j] = *reinterpret_cast<const seq_f32x2 *>(A + (long long)s * a.Cp);
                Bs[j] = B[e / V * a.vB.c + e % V];
                Cs[j] = C[e / V * a.vC.c + e % V];
            }
            if (s0 == wave * 4)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    d[i] += a.dt_bias ? a.dt_bias[c + i] : 0.0f;
                    if (a.softplus) d[i] = seq_softplus(d[i]);
                    d[i] = c + i < a.Ch ? d[i] : 0.0f;
                }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (s0 + j >= a.S) break;
                seq_f32x2 next;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    next[i] = fmaf(seq_exp2(d[i] * (As[j][i] * kLog2e)), was[j][i], d[i] * x[i] * SeqElem<T>::get(Bs[j]));
                    y[i] = fmaf(SeqElem<T>::get(Cs[j]), next[i], y[i]);
                }
                *reinterpret_cast<seq_f32x2 *>(h + (long long)(s0 + j) * a.Cp) = next;
            }
        }
    }
    lds[threadIdx.x] = seq_f32x2{y[0], y[1]};
    __syncthreads();
    if (wave != 0 || c >= a.Cp) return;
    float z[2] = {};
    if (c < a.Ch && has_slot && a.z) two(a.z, a.vz, z);
    Two out;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float o = (lds[lane][i] + lds[lane + 64][i]) + (lds[lane + 128][i] + lds[lane + 192][i]);
        const bool live = c + i < a.Ch && has_slot;
        if (live && a.D) o = fmaf(a.D[c + i], x[i], o);
        if (live && a.z) o *= z[i] * seq_sigmoid(z[i]);
        out.v[i] = SeqElem<T>::put(live ? o : 0.0f);
    }
    *reinterpret_cast<Two *>(static_cast<T *>(a.y) + at(a.vy, c)) = out;
}

hipError_t join(const SeqScanArgs &a, hipStream_t s)
{
    seq_scan_join_kernel<<<(unsigned)seq_join_groups(a), 64 * seq_join_waves(a.chunks), 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, int SP, int MODE>
hipError_t launch_mode(const SeqScanArgs &a, hipStream_t s)
{
    const int64_t waves = seq_scan_waves(a, MODE == 1);
    seq_scan_kernel<T, SP, MODE><<<(unsigned)((waves + kWaves - 1) / kWaves), 64 * kWaves, 0, s>>>(a);
    return hipGetLastError();
}
template <typename T, int MODE>
hipError_t launch_ends(const SeqScanArgs &a, hipStream_t s)
{
    return a.S <= 8 ? launch_mode<T, 8, MODE>(a, s) : a.S <= 16 ? launch_mode<T, 16, MODE>(a, s) : launch_mode<T, 32, MODE>(a, s);
}
template <typename T>
hipError_t launch_t(bool ends, const SeqScanArgs &a, hipStream_t s)
{
    if (ends || a.chunks > 1) {
        hipError_t e = ends ? launch_ends<T, 2>(a, s) : launch_ends<T, 0>(a, s);
        if (e == hipSuccess && a.chunks > 1) e = join(a, s);
        if (ends || e != hipSuccess) return e;
    }
    switch (seq_scan_states(a.S)) {
        case 8: return launch_mode<T, 8, 1>(a, s);
        case 16: return launch_mode<T, 16, 1>(a, s);
        case 32: return launch_mode<T, 32, 1>(a, s);
    }
    return launch_mode<T, 64, 1>(a, s);
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
    const unsigned grid = (unsigned)((long long)a.N * ((a.Cp + 127) / 128));
    if (dtype == SEQ_BF16)
        seq_scan_step_kernel<unsigned short><<<grid, 256, 0, s>>>(a);
    else
        seq_scan_step_kernel<float><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace convmi
