// Gradients of the selective scan.  With g[l] the gradient of the state after position l, back to front,
//
//   g[l] = C dy + exp(d+ A) g+,   dC = sum_c dy h,   dB = sum_c g d x,   dx = D dy + d sum_s g B,
//   dd = sum_s (A t + g B x),   dA = sum d t,   t = g exp(d A) h[l-1]
//
// (dy that of y before the gate.)  The states are formed again rather than kept: positions go in runs of 64 (16 or 32 of short tensors).  A first launch finds
// what each run does to a state and to a gradient and notes the state it reaches every 8 positions, all from zeros; a second puts
// the runs together, so that a run knows the state before it and the gradient behind it, and with the sum of d the state at each note:
// that from zeros plus exp(A sum d) times the one before the run.  A wave then goes through the eights of its run from the back,
// forwards with the 8 states in registers, then backwards.
//
// A lane takes 2 channels x 4 states: the sums over states end in a quad of lanes, those over channels in exchanges that halve what
// is left each time, then over the four waves of a workgroup in LDS.  (4 x 4 need fewer exchanges but more than 256 registers, and one
// wave a SIMD gets an operation into the vector units every 6 clocks, two in turn every 4: 2 x 2048 positions of 2048 channels 214 us.)
// Some 20 operations and two exponentials a state and position: bound by the vector units.
#include "seq_internal.h"

namespace convmi {
namespace {

constexpr int kT = 8;  // positions held at a time

constexpr int kWaves = kSeqBwdWaves;

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

template <typename T, int SP, bool GATE>
__global__ __launch_bounds__(64 * kWaves, 2) void seq_scan_bwd_kernel(const SeqScanArgs a)
{
    constexpr int V = SeqElem<T>::V, NL = SP / 4, WC = seq_scan_bwd_channels(SP);
    constexpr int PT = WC / V >= 8 ? 8 : 16;  // positions staged at a time: a block of one for each lane, where B and C leave room for them
    constexpr int VEC = WC / V * PT, NV = (VEC + 63) / 64, E = PT * SP / 64;
    struct __align__(16) Lds {
        // d, x, dy before the gate, what dz and ddt are multiplied with; the sums over states: A t, g B, C h
        float d[PT][WC], x[PT][WC], dy[PT][WC], slope[PT][WC], At[PT][WC], gB[PT][WC];
        float dgate[GATE ? PT : 1][WC], Ch[GATE ? PT : 1][WC];
        float B[PT][SP], C[PT][SP];  // once a position is done with: dB, dC of the wave's channels
    };
    __shared__ __align__(16) Lds all[kWaves];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), sl = lane % NL, cl = lane / NL;
    Lds &my = all[wave];
    int t = blockIdx.x;
    const int share = t % a.btiles;
    t /= a.btiles;
    const int g = t % a.G;
    t /= a.G;
    const int chunk = t % a.chunks, n = t / a.chunks;
    // (the last share's waves may have no channels: they go along for the barriers)
    const int c0 = g * a.CG + (share * kWaves + wave) * WC, c_end = min(c0 + WC, (g + 1) * a.CG);
    const int len = seq_length(a.lengths, n, a.L);
    const int begin = chunk * a.chunk, end = min(begin + a.chunk, a.L), stop = min(end, len);

    // element-wise: a lane's block and position of what is staged.  Formed anew each time, as its addresses are: kept, they cost registers.
    struct Place {
        bool in;
        int cb, to, l;
        unsigned blocks;
    };
    auto place = [&](int i) {
        int e = lane + 64 * i;
        asm volatile("" : "+v"(e));
        const int cbl = e / PT;
        const bool in = e < VEC && c0 + cbl * V < c_end;
        return Place{in, in ? c0 / V + cbl : 0, e < VEC ? cbl * V : 0, e % PT, (unsigned)cbl};
    };
    // (what lies between a tile's elements fits 32 bits)
    auto address = [&](const void *p, const SeqView &v, const Place &at, int p0) {
        const T *base = static_cast<const T *>(p) + n * v.n + c0 / V * v.c + p0 * v.l;
        return base + (at.blocks * (unsigned)v.c + (unsigned)at.l * (unsigned)v.l);
    };
    auto put = [&](void *p, const SeqView &v, const Place &at, int p0, const float (&f)[V]) {
        seq_store(const_cast<T *>(address(p, v, at, p0)), SeqElem<T>::pack(f));
    };
    // Column of a row in LDS: the fours of a row change places with the row, or the rows of one block would lie in the same banks.
    constexpr int FOURS = WC / 4 < 8 ? WC / 4 : 8;
    auto column = [](int l, int c) { return c ^ (l % FOURS * 4); };
    auto to_lds = [&](float (&row)[WC], const Place &at, const float (&f)[V]) {
#pragma unroll
        for (int j = 0; j < V; j += 4) *reinterpret_cast<seq_f32x4 *>(&row[column(at.l, at.to + j)]) = seq_f32x4{f[j], f[j + 1], f[j + 2], f[j + 3]};
    };
    auto from_lds = [&](const float (&row)[WC], const Place &at, float (&f)[V]) {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const seq_f32x4 q = *reinterpret_cast<const seq_f32x4 *>(&row[column(at.l, at.to + j)]);
#pragma unroll
            for (int k = 0; k < 4; ++k) f[j + k] = q[k];
        }
    };
    float aD[NV], ab[NV];  // sums of dy x and ddt over the run's positions of one channel: lane ll of eight's, ll < V
#pragma unroll
    for (int i = 0; i < NV; ++i) aD[i] = ab[i] = 0;

    // scan-wise: channels c, c + 1, states s ... + 3
    const int c = c0 + cl * 2, s = sl * 4;
    const bool live = c < c_end;
    const long long run = (long long)n * a.chunks + chunk, state = (long long)a.S * a.Cp;
    // this lane's row j of a state.  States and channels that there are not read another's: with B, C, x, dy and the gradient from behind
    // zero they add nothing, as long as their state is a number.
    unsigned at[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) at[j] = (unsigned)(min(s + j, a.S - 1) * a.Cp + (live ? c : g * a.CG));
    const bool there[2] = {live, c + 1 < c_end};
    auto two = [&](const float *p, int j) { return *reinterpret_cast<const seq_f32x2 *>(p + at[j]); };
    float A[4][2], carry[4][2], dA[4][2] = {};  // [state][channel]
    seq_f32x2 before[4];                        // the state before the run
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const seq_f32x2 q = two(a.A, j);
        seq_f32x2 r = {};
        before[j] = seq_f32x2{};
        if (a.chunks > 1) {
            r = two(a.gl + run * state, j);
            before[j] = two(a.hl + run * state, j);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            A[j][i] = there[i] ? seq_decay(q[i]) : 0.0f;
            carry[j][i] = there[i] && s + j < a.S ? r[i] : 0.0f;
        }
    }

    // what is needed next from memory, on its way meanwhile: positions to stage, the note at the start of an eight
    seq_u32x4 nx[NV], nd[NV], ng[NV], nz[NV];
    T nB[E], nC[E];
    // element r of a lane is state s of position (lane + 64 r) / SP
    const int e_of = g * a.S + (lane % SP < a.S ? lane % SP : 0);
    auto of_states = [&](const void *p, const SeqView &v, int r, int l0) {
        const T *base = static_cast<const T *>(p) + n * v.n + l0 * v.l;
        return base + e_of / V * v.c + e_of % V + (lane + 64 * r) / SP * v.l;
    };
    auto fetch = [&](int l0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Place p = place(i);
            nx[i] = nd[i] = ng[i] = nz[i] = seq_u32x4{};
            if (p.in && l0 + p.l < stop) {
                nx[i] = seq_load(address(a.x, a.vx, p, l0));
                nd[i] = seq_load(address(a.dt, a.vdt, p, l0));
                ng[i] = seq_load(address(a.dy, a.vdy, p, l0));
                if (GATE) nz[i] = seq_load(address(a.z, a.vz, p, l0));
            }
        }
#pragma unroll
        for (int r = 0; r < E; ++r) {
            const bool ok = lane % SP < a.S && l0 + (lane + 64 * r) / SP < stop;
            nB[r] = ok ? *of_states(a.B, a.vB, r, l0) : T(0);
            nC[r] = ok ? *of_states(a.C, a.vC, r, l0) : T(0);
        }
    };
    seq_f32x2 note[4], note_d = {};
    auto fetch_note = [&](int e) {
        const long long m = run * a.notes + e - 1;
        note_d = *reinterpret_cast<const seq_f32x2 *>(a.md + m * a.Cp + (live ? c : g * a.CG));
#pragma unroll
        for (int j = 0; j < 4; ++j) note[j] = two(a.marks + m * state, j);
    };
    const int eights = stop > begin ? (stop - begin + kT - 1) / kT : 0;
    const int stages = stop > begin ? (stop - begin + PT - 1) / PT : 0;
    if (stages > 0) fetch(begin + (stages - 1) * PT);
    if (eights > 1) fetch_note(eights - 1);

    for (int stage = stages - 1; stage >= 0; --stage) {
        const int p0 = begin + stage * PT;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Place p = place(i);
            float x[V], d[V], slope[V], dy[V], dgate[V], z[V], bias[V] = {};
            SeqElem<T>::unpack(nx[i], x);
            SeqElem<T>::unpack(nd[i], d);
            SeqElem<T>::unpack(ng[i], dy);
            SeqElem<T>::unpack(nz[i], z);
            if (a.dt_bias) seq_vector<V>(a.dt_bias, p.cb, bias);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const bool ok = p.in && p0 + p.l < stop && p.cb * V + j < a.Ch;
                float sig;
                const float raw = d[j] + bias[j], soft = seq_softplus(raw, &sig);
                d[j] = ok ? a.softplus ? soft : raw : 0.0f;
                slope[j] = ok ? a.softplus ? sig : 1.0f : 0.0f;
                x[j] = ok ? x[j] : 0.0f;
                dy[j] = ok ? dy[j] : 0.0f;
                if (GATE) {
                    const float q = seq_sigmoid(z[j]);
                    dgate[j] = ok ? dy[j] * q * (1.0f + z[j] * (1.0f - q)) : 0.0f;
                    dy[j] = ok ? dy[j] * (z[j] * q) : 0.0f;
                }
            }
            if (lane + 64 * i < VEC) {
                to_lds(my.d[p.l], p, d);
                to_lds(my.x[p.l], p, x);
                to_lds(my.dy[p.l], p, dy);
                to_lds(my.slope[p.l], p, slope);
                if (GATE) to_lds(my.dgate[GATE ? p.l : 0], p, dgate);
            }
        }
#pragma unroll
        for (int r = 0; r < E; ++r) {
            (&my.B[0][0])[lane + 64 * r] = SeqElem<T>::get(nB[r]);
            (&my.C[0][0])[lane + 64 * r] = SeqElem<T>::get(nC[r]);
        }
        seq_wave_sync();
        if (stage > 0) fetch(p0 - PT);
        auto row = [&](const float (&p)[WC], int l) { return *reinterpret_cast<const seq_f32x2 *>(&p[column(l, cl * 2)]); };
        auto states = [&](const float (&p)[SP]) { return *reinterpret_cast<const seq_f32x4 *>(&p[s]); };

#pragma unroll 1
        for (int first = PT - kT; first >= 0; first -= kT) {
            if (p0 + first >= stop) continue;
            const int e = (p0 + first - begin) / kT;
            float hs[kT + 1][4][2];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float h = e > 0 ? fmaf(seq_exp2(A[j][i] * note_d[i]), before[j][i], note[j][i]) : before[j][i];
                    hs[0][j][i] = there[i] ? h : 0.0f;
                }
            if (e > 1) fetch_note(e - 1);
#pragma unroll
            for (int q = 0; q < kT; ++q) {
                const int l = first + q;
                const seq_f32x2 d = row(my.d[l], q), x = row(my.x[l], q);
                const seq_f32x4 B = states(my.B[l]);
                float a[4][2], b[4][2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) a[j][i] = d[i] * A[j][i];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float dx = d[i] * x[i];
#pragma unroll
                    for (int j = 0; j < 4; ++j) a[j][i] = seq_exp2(a[j][i]), b[j][i] = B[j] * dx;
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) hs[q + 1][j][i] = fmaf(a[j][i], hs[q][j][i], b[j][i]);
            }
            // (else the compiler keeps the decays and the eight's numbers from the way forwards, in registers that there are not)
            seq_wave_sync();
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) asm volatile("" : "+v"(A[j][i]));
#pragma unroll
            for (int q = kT - 1; q >= 0; --q) {
                const int l = first + q;
                const seq_f32x2 d = row(my.d[l], q), x = row(my.x[l], q), dy = row(my.dy[l], q);
                const seq_f32x4 B = states(my.B[l]), C = states(my.C[l]);
                float bc[8] = {};  // dB, dC of the four states
                seq_f32x2 gB = {}, At = {}, Ch = {};
                float a[4][2], gr[4][2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        a[j][i] = d[i] * A[j][i];
                        gr[j][i] = fmaf(dy[i], C[j], carry[j][i]);
                    }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float dx = d[i] * x[i];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        a[j][i] = seq_exp2(a[j][i]);
                        bc[4 + j] = fmaf(dy[i], hs[q + 1][j][i], bc[4 + j]);
                        bc[j] = fmaf(gr[j][i], dx, bc[j]);
                        gB[i] = fmaf(gr[j][i], B[j], gB[i]);
                        if (GATE) Ch[i] = fmaf(C[j], hs[q + 1][j][i], Ch[i]);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        carry[j][i] = gr[j][i] * a[j][i];
                        const float th = carry[j][i] * hs[q][j][i];
                        dA[j][i] = fmaf(th, d[i], dA[j][i]);
                        At[i] = fmaf(th, A[j][i], At[i]);
                    }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    gB[i] = sum_states<NL>(gB[i]);
                    At[i] = sum_states<NL>(At[i]);
                    if (GATE) Ch[i] = sum_states<NL>(Ch[i]);
                }
                if (sl == 0) {
                    *reinterpret_cast<seq_f32x2 *>(&my.At[l][column(q, cl * 2)]) = At;
                    *reinterpret_cast<seq_f32x2 *>(&my.gB[l][column(q, cl * 2)]) = gB;
                    if (GATE) *reinterpret_cast<seq_f32x2 *>(&my.Ch[GATE ? l : 0][column(q, cl * 2)]) = Ch;
                }
                float u[4], v[2];
#pragma unroll
                for (int j = 0; j < 4; ++j) u[j] = swap32(bc[j], bc[j + 4]);
#pragma unroll
                for (int j = 0; j < 2; ++j) v[j] = sum_row<NL>(swap16(u[j], u[j + 2]));
                // the lower half of the wave has dB, the upper one dC; even rows states s, s + 1, odd ones s + 2, s + 3
                if (lane % 16 < NL) *reinterpret_cast<seq_f32x2 *>((lane < 32 ? my.B[l] : my.C[l]) + lane % 16 * 4 + lane / 16 % 2 * 2) = seq_f32x2{v[0], v[1]};
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        seq_wave_sync();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Place p = place(i);
            const int l = p0 + p.l;
            const bool inside = l < stop, store = p.in && l < end;
            float d[V], x[V], dy[V], slope[V], At[V], gB[V], dx[V], ddt[V], D[V] = {};
            from_lds(my.d[p.l], p, d);
            from_lds(my.x[p.l], p, x);
            from_lds(my.dy[p.l], p, dy);
            from_lds(my.slope[p.l], p, slope);
            from_lds(my.At[p.l], p, At);
            from_lds(my.gB[p.l], p, gB);
            if (a.D) seq_vector<V>(a.D, p.cb, D);
            float pD[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                // (past the end nothing has been summed; D of channels beyond the last one may be anything)
                const bool ok = inside && p.cb * V + j < a.Ch;
                dx[j] = ok ? fmaf(d[j], gB[j], D[j] * dy[j]) : 0.0f;
                ddt[j] = ok ? fmaf(kLn2, At[j], x[j] * gB[j]) * slope[j] : 0.0f;
                pD[j] = dy[j] * x[j];
            }
            if (store) {
                put(a.dx, a.vdx, p, p0, dx);
                put(a.ddt, a.vddt, p, p0, ddt);
            }
            if (GATE) {
                float dgate[V], Ch[V];
                from_lds(my.dgate[GATE ? p.l : 0], p, dgate);
                from_lds(my.Ch[GATE ? p.l : 0], p, Ch);
#pragma unroll
                for (int j = 0; j < V; ++j) dgate[j] = inside && p.cb * V + j < a.Ch ? dgate[j] * fmaf(D[j], x[j], Ch[j]) : 0.0f;
                if (store) put(a.dz, a.vdz, p, p0, dgate);
            }
            // lane ll of eight keeps the sums of the block's channel ll
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float u = sum_states<8>(pD[j]), w = sum_states<8>(ddt[j]);
                aD[i] += lane % 8 == j ? u : 0.0f;
                ab[i] += lane % 8 == j ? w : 0.0f;
            }
        }
        // dB and dC of the workgroup's channels
        __syncthreads();
        for (int i = threadIdx.x; i < PT * 2 * SP; i += 64 * kWaves) {
            const int l = i / (2 * SP), which = i / SP % 2, st = i % SP;
            if (p0 + l >= stop || st >= a.S) continue;
            float sum = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) sum += which ? all[w].C[l][st] : all[w].B[l][st];
            a.bc[((((long long)n * a.L + p0 + l) * a.G + g) * a.btiles + share) * 2 * a.S + which * a.S + st] = sum;
        }
        __syncthreads();
    }
    // zeros past the end
    const float zero[V] = {};
    for (int l0 = begin + stages * PT; l0 < end; l0 += PT)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Place p = place(i);
            if (!p.in || l0 + p.l >= end) continue;
            put(a.dx, a.vdx, p, l0, zero);
            put(a.ddt, a.vddt, p, l0, zero);
            if (GATE) put(a.dz, a.vdz, p, l0, zero);
        }
    // this run's part of the parameters' gradients; that of A where its state was
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (live && s + j < a.S) *reinterpret_cast<seq_f32x2 *>(a.hl + run * state + at[j]) = seq_f32x2{dA[j][0], dA[j][1]};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const Place p = place(i);
        float u = aD[i], w = ab[i];
        if (PT == 16) {  // (the other eight of the positions)
            u += __shfl_xor(u, 8);
            w += __shfl_xor(w, 8);
        }
        if (p.in && p.l < V) {
            float *v = a.vec + run * 2 * a.Cp + p.cb * V + p.l;
            v[0] = u;
            v[a.Cp] = w;
        }
    }
}

// What the runs and shares left in parts, summed in order: dA, dD, ddt_bias over the runs by the first `params` workgroups, dB and dC of each
// position over the shares of the channels by the others, one thread a result.  (A launch each: 4.6 and 6.4 us.)
template <typename T>
__global__ __launch_bounds__(1024) void seq_scan_parts_kernel(const SeqScanArgs a, unsigned params)
{
    if (blockIdx.x < params) {
        const long long state = (long long)a.S * a.Cp, col = (long long)blockIdx.x * kSumColumns + threadIdx.x % kSumColumns;
        const bool of_A = col < state;
        const long long e = of_A ? col : col - state, pitch = of_A ? state : 2LL * a.Cp;
        // (results of channels beyond the last one are zero)
        const float s = seq_sum_parts((of_A ? a.hl : a.vec) + e, pitch, a.N * a.chunks, e < pitch && e % a.Cp < a.Ch);
        if (threadIdx.x >= kSumColumns || e >= pitch) return;
        float *out = of_A ? a.dA + e : e < a.Cp ? (a.dD ? a.dD + e : nullptr) : a.ddt_bias ? a.ddt_bias + (e - a.Cp) : nullptr;
        if (out) *out = s;
        return;
    }
    constexpr int V = SeqElem<T>::V;
    const int Sp = (a.G * a.S + V - 1) / V * V;
    const long long total = (long long)a.N * a.L * 2 * Sp;
    for (long long t = (long long)(blockIdx.x - params) * 1024 + threadIdx.x; t < total; t += (long long)(gridDim.x - params) * 1024) {
        const int e = (int)(t % Sp), which = (int)(t / Sp % 2);
        const long long row = t / Sp / 2;
        const int n = (int)(row / a.L), l = (int)(row % a.L);
        float sum = 0;
        if (e < a.G * a.S && l < seq_length(a.lengths, n, a.L)) {
            const int g = e / a.S, s = e % a.S;
            const float *p = a.bc + ((row * a.G + g) * a.btiles * 2 + which) * a.S + s;
            int k = 0;
            for (; k + 8 <= a.btiles; k += 8) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = p[(long long)(k + i) * 2 * a.S];
#pragma unroll
                for (int i = 0; i < 8; ++i) sum += f[i];
            }
            for (; k < a.btiles; ++k) sum += p[(long long)k * 2 * a.S];
        }
        const SeqView &v = which ? a.vdC : a.vdB;
        static_cast<T *>(which ? a.dC : a.dB)[n * v.n + e / V * v.c + l * v.l + e % V] = SeqElem<T>::put(sum);
    }
}

template <typename T, int SP>
hipError_t launch(int dtype, const SeqScanArgs &a, hipStream_t s)
{
    if (a.L > kT) {
        const hipError_t e = launch_seq_scan_ends(dtype, a, s);
        if (e != hipSuccess) return e;
    }
    const unsigned grid = (unsigned)((long long)a.N * a.G * a.btiles * a.chunks);
    if (a.z)
        seq_scan_bwd_kernel<T, SP, true><<<grid, 64 * kWaves, 0, s>>>(a);
    else
        seq_scan_bwd_kernel<T, SP, false><<<grid, 64 * kWaves, 0, s>>>(a);
    const unsigned params = (unsigned)(((a.S + 2LL) * a.Cp + kSumColumns - 1) / kSumColumns);
    const long long results = ((long long)a.N * a.L * 2 * (a.G * a.S + 7) + 1023) / 1024;
    seq_scan_parts_kernel<T><<<params + (unsigned)(results < 1 << 18 ? results : 1 << 18), 1024, 0, s>>>(a, params);
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
