// C entry points of the sequence operators: checks, plans, launches (include/seq_mi355x.h).
#include <math.h>
#include <stdio.h>

#include <algorithm>
#include <iterator>
#include <new>

#include "seq_internal.h"

using namespace convmi;

namespace {
enum Kind { kConv, kScan, kRec, kNorm, kLnorm, kMv4, kAdamw };
}  // namespace

struct seq_plan {
    Kind kind;
    int dtype, W;
    seq_info_t info;
    size_t fwd_ws, bwd_ws;
    SeqConvArgs conv;  // its runs are the forward pass's
    int bwd_range, bwd_ranges;
    SeqScanArgs scan, scan_bwd;
    SeqRecArgs rec, rec_bwd;
    SeqNormArgs norm;
    SeqMv4Args mv4;
    SeqAdamwArgs adamw;        // without its tensors
    SeqAdamwTensor *tensors;   // their sizes, places and decays
    int count, bits;
    ~seq_plan() { delete[] tensors; }
};

namespace {

// (a launch has at most 2^32 work-items)
constexpr int64_t kMaxElements = 1LL << 39, kMaxItems = (1LL << 32) - 4096, kMaxStride = 1LL << 40, kMaxSpan = 1LL << 58, kMaxTileStride = 1LL << 24, kMaxNumbers = 1LL << 35, kMaxWaveStride = 1LL << 20;

bool aligned(const void *p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

size_t up(size_t bytes) { return (bytes + 255) / 256 * 256; }

bool sizes_ok(int N, int C, int L) { return N >= 1 && C >= 1 && L >= 1; }
bool sizes_supported(int64_t N, int64_t C, int64_t L, int v)
{
    return N <= 1 << 20 && C <= 1 << 20 && L <= 1 << 30 && N * L < 1LL << 31 && N * L <= kMaxElements / ((C + v - 1) / v * v);
}

// A view as the kernels take it, or false where it is not as the header says.  `out`: no two elements may share a place.
bool view_of(const seq_view_t &v, int N, int Cb, int L, int vlen, bool out, SeqView &to)
{
    if (v.n == 0 && v.c == 0 && v.l == 0) {
        to = {(long long)Cb * L * vlen, Cb > 1 ? (long long)L * vlen : 0, vlen};
        return true;
    }
    struct {
        int64_t extent, stride;
    } d[3] = {{N, v.n}, {Cb, v.c}, {L, v.l}};
    for (auto &e : d) {
        if (e.extent == 1) e.stride = 0;
        if (e.stride < 0 || e.stride > kMaxStride || e.stride % vlen || (e.extent > 1 && e.stride > kMaxSpan / (e.extent - 1))) return false;
    }
    to = {d[0].stride, d[1].stride, d[2].stride};
    if (!out) return true;
    std::sort(d, d + 3, [](auto &p, auto &q) { return p.stride < q.stride; });
    int64_t span = vlen;  // from the first to behind the last element so far
    for (auto &e : d) {
        if (e.extent == 1) continue;
        if (e.stride < span) return false;
        span += (e.extent - 1) * e.stride;
    }
    return true;
}

bool known(int dtype) { return dtype == SEQ_F32 || dtype == SEQ_BF16; }
int vlen_of(int dtype) { return dtype == SEQ_F32 ? 4 : dtype == SEQ_BF16 ? 8 : 16; }

seq_plan *new_plan(Kind kind, int dtype, int C)
{
    seq_plan *p = new (std::nothrow) seq_plan();
    if (!p) return nullptr;
    p->kind = kind;
    p->dtype = dtype;
    p->info.vlen = vlen_of(dtype);
    p->info.Cb = (C + p->info.vlen - 1) / p->info.vlen;
    p->info.Cp = p->info.Cb * p->info.vlen;
    return p;
}
conv_status_t finish(seq_plan *p, conv_status_t st, seq_handle_t *out)
{
    if (st != CONV_OK) {
        delete p;
        return st;
    }
    p->info.workspace_bytes = std::max(p->fwd_ws, p->bwd_ws);
    *out = p;
    return CONV_OK;
}

conv_status_t done(hipError_t e) { return e == hipSuccess ? CONV_OK : CONV_ELAUNCH; }

// Required pointers, 16-byte aligned; optional ones (p == NULL allowed).
template <typename... P>
bool given(P... p)
{
    return ((p != nullptr && aligned(p, 16)) && ...);
}
template <typename... P>
bool fine(P... p)
{
    return (aligned(p, 16) && ...);
}

}  // namespace

extern "C" {

conv_status_t seq_destroy(seq_handle_t h)
{
    if (!h) return CONV_EINVAL;
    delete h;
    return CONV_OK;
}

conv_status_t seq_query(seq_handle_t h, seq_info_t *info)
{
    if (!h || !info) return CONV_EINVAL;
    *info = h->info;
    return CONV_OK;
}

// ------------------------------------------------------------------ short convolution
conv_status_t seq_conv_create(const seq_conv_desc_t *d, seq_handle_t *out)
{
    if (!d || !out || !known(d->dtype) || !sizes_ok(d->N, d->C, d->L) || d->W < 1 || d->slots < 0) return CONV_EINVAL;
    const int v = vlen_of(d->dtype);
    if (!sizes_supported(d->N, d->C, d->L, v) || d->W < 2 || d->W > 8) return CONV_EUNSUPPORTED;
    seq_plan *p = new_plan(kConv, d->dtype, d->C);
    if (!p) return CONV_EUNSUPPORTED;
    SeqConvArgs &a = p->conv;
    a.N = d->N;
    a.L = d->L;
    a.Cb = p->info.Cb;
    a.Cp = p->info.Cp;
    a.silu = d->silu != 0;
    a.n_slots = d->slots;
    p->W = d->W;
    if (!view_of(d->x, a.N, a.Cb, a.L, v, false, a.vx) || !view_of(d->y, a.N, a.Cb, a.L, v, true, a.vy) ||
        !view_of(d->dy, a.N, a.Cb, a.L, v, false, a.vdy) || !view_of(d->dx, a.N, a.Cb, a.L, v, true, a.vdx))
        return finish(p, CONV_EINVAL, out);
    // Runs of positions: as long as they may be, for the weights are loaded, their gradients summed and neighbours' positions read once a run,
    // in one round of workgroups that are resident together.  That is 6 a compute unit forwards; backwards, whose registers and LDS
    // go by the number of taps, 3 or 2 in bf16 and 5 or 3 in fp32.  (8 x 2048 x 2048 bf16, 4 taps, backwards: 768 workgroups 55 us, 1024 73,
    // 1536 63, 2048 73.)
    a.past = (long long)a.N * a.Cb * a.L * 16 > kSeqPastBytes;
    a.cgroups = (a.Cb + 7) / 8;
    const int64_t columns = (int64_t)a.N * a.cgroups;
    const auto runs = [&](int64_t workgroups, int &range) {
        const int64_t want = std::max<int64_t>(1, workgroups / columns);
        range = (int)std::min<int64_t>(std::max<int64_t>(((a.L + want - 1) / want + 31) / 32 * 32, 64), 1 << 29);
        return (int)((a.L + (int64_t)range - 1) / range);
    };
    a.ranges = runs(256 * 6, a.range);
    p->bwd_ranges = runs(256 * (d->dtype == SEQ_BF16 ? d->W <= 4 ? 3 : 2 : d->W <= 4 ? 5 : 3), p->bwd_range);
    p->info.state_bytes = (size_t)a.Cb * (d->W - 1) * 16;
    p->bwd_ws = up((size_t)a.N * p->bwd_ranges * (d->W + 1) * a.Cp * 4);
    const bool fits = columns * std::max(a.ranges, p->bwd_ranges) * 256 <= kMaxItems;
    return finish(p, fits ? CONV_OK : CONV_EUNSUPPORTED, out);
}

conv_status_t seq_conv_fwd(seq_handle_t h, const void *x, const float *w, const float *bias, const void *state_in, void *y,
                           void *state_out, const int32_t *slots, const int32_t *lengths, void *stream)
{
    if (!h || h->kind != kConv || !given(x, w, y) || !fine(bias, state_in, state_out) || !aligned(slots, 4) || !aligned(lengths, 4) ||
        ((state_in || state_out) && h->conv.n_slots == 0))
        return CONV_EINVAL;
    SeqConvArgs a = h->conv;
    a.x = x;
    a.w = w;
    a.bias = bias;
    a.state_in = state_in;
    a.y = y;
    a.state_out = state_out;
    a.slots = slots;
    a.lengths = lengths;
    return done(launch_seq_conv_fwd(h->dtype, h->W, a, (hipStream_t)stream));
}

conv_status_t seq_conv_step(seq_handle_t h, const void *x, const float *w, const float *bias, void *state, void *y,
                            const int32_t *slots, void *stream)
{
    if (!h || h->kind != kConv || !given(x, w, state, y) || !fine(bias) || !aligned(slots, 4) || h->conv.n_slots == 0 || h->conv.L != 1) return CONV_EINVAL;
    SeqConvArgs a = h->conv;
    a.x = x;
    a.w = w;
    a.bias = bias;
    a.state_out = state;
    a.y = y;
    a.slots = slots;
    return done(launch_seq_conv_step(h->dtype, h->W, a, (hipStream_t)stream));
}

conv_status_t seq_conv_bwd(seq_handle_t h, const void *x, const float *w, const float *bias, const void *dy, void *dx, float *dw,
                           float *dbias, const int32_t *lengths, void *ws, size_t ws_bytes, void *stream)
{
    if (!h || h->kind != kConv || !given(x, w, dy, dx, dw) || !fine(bias, dbias, ws) || !aligned(lengths, 4)) return CONV_EINVAL;
    if (!ws || ws_bytes < h->bwd_ws) return CONV_EWORKSPACE;
    SeqConvArgs a = h->conv;
    a.x = x;
    a.w = w;
    a.bias = bias;
    a.dy = dy;
    a.dx = dx;
    a.dw = dw;
    a.dbias = dbias;
    a.lengths = lengths;
    a.range = h->bwd_range;
    a.ranges = h->bwd_ranges;
    a.part = static_cast<float *>(ws);
    return done(launch_seq_conv_bwd(h->dtype, h->W, a, (hipStream_t)stream));
}

// ------------------------------------------------------------------ selective scan
conv_status_t seq_scan_create(const seq_scan_desc_t *d, seq_handle_t *out)
{
    if (!d || !out || !known(d->dtype) || !sizes_ok(d->N, d->C, d->L) || d->S < 1 || d->G < 1 || d->slots < 0 || d->C % d->G) return CONV_EINVAL;
    const int v = vlen_of(d->dtype);
    if (!sizes_supported(d->N, d->C, d->L, v) || d->S > 64 || (int64_t)d->G * d->S > 1 << 16 || (d->G > 1 && d->C / d->G % v)) return CONV_EUNSUPPORTED;
    const int Sb = (d->G * d->S + v - 1) / v;
    if (!sizes_supported(d->N, d->G * d->S, d->L, v)) return CONV_EUNSUPPORTED;
    seq_plan *p = new_plan(kScan, d->dtype, d->C);
    if (!p) return CONV_EUNSUPPORTED;
    SeqScanArgs &a = p->scan;
    a.N = d->N;
    a.L = d->L;
    a.S = d->S;
    a.G = d->G;
    a.Ch = d->C;
    a.Cp = p->info.Cp;
    a.CG = d->C / d->G;
    a.softplus = d->softplus != 0;
    a.n_slots = d->slots;
    const int Cb = p->info.Cb;
    const struct {
        const seq_view_t &v;
        int blocks;
        bool out;
        SeqView &to;
    } views[] = {{d->x, Cb, false, a.vx},   {d->dt, Cb, false, a.vdt}, {d->B, Sb, false, a.vB},    {d->C_, Sb, false, a.vC},
                 {d->z, Cb, false, a.vz},   {d->y, Cb, true, a.vy},    {d->dy, Cb, false, a.vdy},  {d->dx, Cb, true, a.vdx},
                 {d->ddt, Cb, true, a.vddt}, {d->dB, Sb, true, a.vdB},  {d->dC, Sb, true, a.vdC},   {d->dz, Cb, true, a.vdz}};
    for (const auto &w : views) {
        if (!view_of(w.v, a.N, w.blocks, a.L, v, w.out, w.to)) return finish(p, CONV_EINVAL, out);
        // (a tile's elements are reached from its first one by 32 bits)
        if (w.to.c > kMaxTileStride || w.to.l > kMaxTileStride) return finish(p, CONV_EUNSUPPORTED, out);
    }

    // Forward: the sequence whole where the channels alone give every SIMD (1024) a wave, else in runs that make two.  Up to 64 positions whole
    // too: a wave of its own SIMD takes some 0.3 us a position, two launches more some 15.
    a.tiles = (a.CG + 63) / 64;
    const int64_t waves = (int64_t)a.N * a.G * a.tiles;
    const int64_t runs = waves >= 1024 || a.L <= 64 ? 1 : (2048 + waves - 1) / waves;
    a.chunk = (int)(std::min<int64_t>(std::max<int64_t>((a.L + runs - 1) / runs, 16) + 7, 1 << 29) / 8 * 8);
    a.chunks = (int)((a.L + (int64_t)a.chunk - 1) / a.chunk);
    const size_t state = (size_t)a.S * a.Cp * 4;
    p->info.state_bytes = state;
    const auto ends = [&](const SeqScanArgs &b) { return up((size_t)b.N * b.chunks * state) + up((size_t)b.N * b.chunks * b.Cp * 4); };
    p->fwd_ws = a.chunks > 1 ? ends(a) : 0;

    SeqScanArgs &b = p->scan_bwd;
    b = a;
    const int share = seq_scan_bwd_channels(seq_scan_states(b.S)) * kSeqBwdWaves;
    b.btiles = (b.CG + share - 1) / share;
    // Backward: runs of 64 positions, of 32 or 16 where they leave a compute unit less than two workgroups.  (8 x 48 positions of 448 channels,
    // 16 states, bf16, in runs of 64: 71 us.)
    for (b.chunk = 64; b.chunk > 16 && (int64_t)b.N * b.G * b.btiles * ((b.L + b.chunk - 1) / b.chunk) < 512;) b.chunk /= 2;
    b.chunks = (int)((b.L + (int64_t)b.chunk - 1) / b.chunk);
    b.notes = b.chunk / 8 - 1;
    p->bwd_ws = ends(b) + up((size_t)b.N * b.chunks * state) + up((size_t)b.N * b.chunks * b.notes * state) +
                up((size_t)b.N * b.chunks * b.notes * b.Cp * 4) + up((size_t)b.N * b.chunks * 2 * b.Cp * 4) +
                up((size_t)b.N * b.L * b.G * b.btiles * 2 * b.S * 4);
    const auto over_runs = [](const SeqScanArgs &q, bool sums) { return (seq_scan_waves(q, sums) + kSeqScanWaves - 1) / kSeqScanWaves * 64 * kSeqScanWaves; };
    const auto joined = [](const SeqScanArgs &q) { return q.chunks > 1 ? seq_join_groups(q) * 64 * seq_join_waves(q.chunks) : 0; };
    const int64_t items[] = {over_runs(a, true),
                             a.chunks > 1 ? over_runs(a, false) : 0,
                             joined(a),
                             b.L > 8 ? over_runs(b, false) : 0,
                             joined(b),
                             (int64_t)b.N * b.G * b.btiles * b.chunks * 64 * kSeqBwdWaves,
                             a.L == 1 ? (int64_t)a.N * ((a.Cp + 127) / 128) * 256 : 0};
    const bool fits = *std::max_element(std::begin(items), std::end(items)) <= kMaxItems && (int64_t)b.N * b.chunks < 1LL << 31;
    return finish(p, fits ? CONV_OK : CONV_EUNSUPPORTED, out);
}

static void scan_inputs(SeqScanArgs &a, const void *x, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z,
                        const float *dt_bias)
{
    a.x = x;
    a.dt = dt;
    a.A = A;
    a.B = B;
    a.C = C;
    a.D = D;
    a.z = z;
    a.dt_bias = dt_bias;
}

conv_status_t seq_scan_fwd(seq_handle_t h, const void *x, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z,
                           const float *dt_bias, const float *state_in, void *y, float *state_out, const int32_t *slots, const int32_t *lengths, void *ws,
                           size_t ws_bytes, void *stream)
{
    if (!h || h->kind != kScan || !given(x, dt, A, B, C, y) || !fine(D, z, dt_bias, state_in, state_out, ws) || !aligned(slots, 4) || !aligned(lengths, 4) ||
        ((state_in || state_out) && h->scan.n_slots == 0))
        return CONV_EINVAL;
    if (h->fwd_ws && (!ws || ws_bytes < h->fwd_ws)) return CONV_EWORKSPACE;
    SeqScanArgs a = h->scan;
    scan_inputs(a, x, dt, A, B, C, D, z, dt_bias);
    a.state_in = state_in;
    a.y = y;
    a.state_out = state_out;
    a.slots = slots;
    a.lengths = lengths;
    a.hl = static_cast<float *>(ws);
    a.sd = reinterpret_cast<float *>(static_cast<char *>(ws) + up((size_t)a.N * a.chunks * a.S * a.Cp * 4));
    return done(launch_seq_scan_fwd(h->dtype, a, (hipStream_t)stream));
}

conv_status_t seq_scan_step(seq_handle_t h, const void *x, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z,
                            const float *dt_bias, float *state, void *y, const int32_t *slots, void *stream)
{
    if (!h || h->kind != kScan || !given(x, dt, A, B, C, state, y) || !fine(D, z, dt_bias) || !aligned(slots, 4) || h->scan.n_slots == 0 || h->scan.L != 1) return CONV_EINVAL;
    SeqScanArgs a = h->scan;
    scan_inputs(a, x, dt, A, B, C, D, z, dt_bias);
    a.state_out = state;
    a.y = y;
    a.slots = slots;
    return done(launch_seq_scan_step(h->dtype, a, (hipStream_t)stream));
}

conv_status_t seq_scan_bwd(seq_handle_t h, const void *x, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z,
                           const float *dt_bias, const void *dy, void *dx, void *ddt, float *dA, void *dB, void *dC, float *dD, void *dz,
                           float *ddt_bias, const int32_t *lengths, void *ws, size_t ws_bytes, void *stream)
{
    if (!h || h->kind != kScan || !given(x, dt, A, B, C, dy, dx, ddt, dA, dB, dC) || !fine(D, z, dt_bias, dD, dz, ddt_bias, ws) || !aligned(lengths, 4) ||
        !z != !dz)
        return CONV_EINVAL;
    if (!ws || ws_bytes < h->bwd_ws) return CONV_EWORKSPACE;
    SeqScanArgs a = h->scan_bwd;
    scan_inputs(a, x, dt, A, B, C, D, z, dt_bias);
    a.dy = dy;
    a.dx = dx;
    a.ddt = ddt;
    a.dA = dA;
    a.dB = dB;
    a.dC = dC;
    a.dD = dD;
    a.dz = dz;
    a.ddt_bias = ddt_bias;
    a.lengths = lengths;
    char *at = static_cast<char *>(ws);
    const auto take = [&](size_t floats) {
        float *p = reinterpret_cast<float *>(at);
        at += up(floats * 4);
        return p;
    };
    const size_t runs = (size_t)a.N * a.chunks;
    a.hl = take(runs * a.S * a.Cp);
    a.sd = take(runs * a.Cp);
    a.gl = take(runs * a.S * a.Cp);
    a.marks = take(runs * a.notes * a.S * a.Cp);
    a.md = take(runs * a.notes * a.Cp);
    a.vec = take(runs * 2 * a.Cp);
    a.bc = reinterpret_cast<float *>(at);
    return done(launch_seq_scan_bwd(h->dtype, a, (hipStream_t)stream));
}

// ------------------------------------------------------------------ gated linear recurrence
conv_status_t seq_rec_create(const seq_rec_desc_t *d, seq_handle_t *out)
{
    if (!d || !out || !known(d->dtype) || !sizes_ok(d->N, d->C, d->L) || d->slots < 0) return CONV_EINVAL;
    const int v = vlen_of(d->dtype);
    if (!sizes_supported(d->N, d->C, d->L, v)) return CONV_EUNSUPPORTED;
    seq_plan *p = new_plan(kRec, d->dtype, d->C);
    if (!p) return CONV_EUNSUPPORTED;
    SeqRecArgs &a = p->rec;
    a.N = d->N;
    a.L = d->L;
    a.Cb = p->info.Cb;
    a.Cp = p->info.Cp;
    a.n_slots = d->slots;
    const struct {
        const seq_view_t &v;
        bool out;
        SeqView &to;
    } views[] = {{d->x, false, a.vx},   {d->f, false, a.vf},  {d->i, false, a.vi},  {d->z, false, a.vz},  {d->y, true, a.vy},
                 {d->dy, false, a.vdy}, {d->dx, true, a.vdx}, {d->df, true, a.vdf}, {d->di, true, a.vdi}, {d->dz, true, a.vdz}};
    for (const auto &w : views)
        if (!view_of(w.v, a.N, a.Cb, a.L, v, w.out, w.to)) return finish(p, CONV_EINVAL, out);
    a.rows = a.Cb > 1 && a.vx.c < a.vx.l;
    // (a wave's elements are reached from its first one by 32 bits: 128 positions, 8 blocks)
    for (const auto &w : views)
        if (w.to.l > kMaxWaveStride || (a.rows && w.to.c > kMaxTileStride)) return finish(p, CONV_EUNSUPPORTED, out);
    a.past = (long long)a.N * a.Cb * a.L * 16 > kSeqPastBytes;
    // Waves of a workgroup: as many as find positions.  Forwards up to 8 where workgroups are two or more a compute unit (8 x 2048 x 2048 bf16: 73 us, with 4 of them 77,
    // with 16 95), else up to 16 (1 x 8192 x 2048: 46 and 51); backwards 4, whose registers and LDS are three or four workgroups' a compute unit (2: 227 us, 4: 177), but 8 where
    // workgroups are about as many as compute units (1 x 8192 x 2048 bf16 138 -> 103 us, rows of 8 x 2048 x 2048 297 -> 224; at 375 of them 41 -> 45).
    const int64_t columns = a.N * seq_rec_groups(a.Cp, a.rows, v);
    a.few = columns < 512;
    // (of the same number of rounds the one with the fewest waves: 16 x 300 x 2048 bf16 35 -> 31 us, gradients 101 -> 86; but a workgroup alone on a compute unit takes powers of
    // two: 2 x 530 x 1000 11.6 us, 15.2 with the fewest)
    const auto waves = [&](int each, int most, bool fewest) {
        const int64_t all = (a.L + (int64_t)each - 1) / each, rounds = (all + most - 1) / most;
        if (fewest) return (int)((all + rounds - 1) / rounds);
        int w = 1;
        while (w < most && w < all) w *= 2;
        return w;
    };
    // Where there are less than `most` workgroups, of `each` positions at a time, they share a sequence in runs, of which another launch finds out first what they make
    // of a state, for which it reads most of the tensors: forwards below 128 workgroups (1 x 8192 x 512 bf16 33 -> 21 us, 1 x 16384 x 64 61 -> 14; 160 of them, ragged
    // fp32 rows of 5 x 777 x 1000: 21 -> 26 in four runs and 31 in two), backwards below 192 (128 of them, rows of 4 x 2048 x 2048 bf16: 172 us with eight waves each,
    // 141 in runs; 192, rows of 6 x 2048 x 2048: 197 and 207).
    const auto runs = [&](SeqRecArgs &q, int64_t each, int64_t most) {
        const int64_t want = std::min<int64_t>({(most + columns - 1) / columns, (q.L + each - 1) / each, 64});
        q.run = (int)(std::min<int64_t>(((q.L + want - 1) / want + each - 1) / each * each, 1 << 30));
        q.runs = (int)((q.L + (int64_t)q.run - 1) / q.run);
    };
    const int lanes = seq_rec_lanes(a.rows, v);
    a.waves = waves(lanes * seq_rec_positions(a.rows), a.few ? kSeqRecWaves : kSeqRecWaves / 2, !a.few);
    const int shared = lanes * seq_rec_positions(a.rows) * kSeqRecTotalsWaves;
    runs(a, a.L, 1);
    if (columns < 128 && a.L > 2 * shared) {
        a.waves = kSeqRecTotalsWaves;
        runs(a, shared, 512);
    }
    p->rec_bwd = a;
    SeqRecArgs &b = p->rec_bwd;
    const int each = lanes * kSeqRecBwdPositions;
    b.waves = waves(each, columns >= 192 && columns <= 256 ? kSeqRecBwdWaves : kSeqRecBwdWaves / 2, true);
    runs(b, b.L, 1);
    if (columns < 192 && b.L > 2 * each * b.waves) runs(b, each * b.waves, 768);
    b.rounds = (int)((std::min(b.L, b.run) + (int64_t)b.waves * each - 1) / ((int64_t)b.waves * each));
    p->info.state_bytes = (size_t)a.Cp * 4;
    p->fwd_ws = a.runs > 1 ? up((size_t)a.N * a.runs * 2 * a.Cp * 4) : 0;
    p->bwd_ws = up((size_t)a.N * b.runs * 3 * a.Cp * 4) * (b.runs > 1 ? 2 : 1) + up((size_t)a.N * b.runs * b.rounds * a.Cp * 4);
    const bool fits = columns * 64 * std::max(a.runs * a.waves, b.runs * b.waves) <= kMaxItems;
    return finish(p, fits ? CONV_OK : CONV_EUNSUPPORTED, out);
}

static void rec_inputs(SeqRecArgs &a, const void *x, const void *f, const void *i, const float *A, const void *z, const float *f_bias, const float *i_bias)
{
    a.x = x;
    a.f = f;
    a.i = i;
    a.A = A;
    a.z = z;
    a.f_bias = f_bias;
    a.i_bias = i_bias;
}

conv_status_t seq_rec_fwd(seq_handle_t h, const void *x, const void *f, const void *i, const float *A, const void *z, const float *f_bias,
                          const float *i_bias, const float *state_in, void *y, float *state_out, const int32_t *slots, const int32_t *lengths, void *ws,
                          size_t ws_bytes, void *stream)
{
    if (!h || h->kind != kRec || !given(x, f, i, A, y) || !fine(z, f_bias, i_bias, state_in, state_out, ws) || !aligned(slots, 4) || !aligned(lengths, 4) ||
        ((state_in || state_out) && h->rec.n_slots == 0))
        return CONV_EINVAL;
    if (h->fwd_ws && (!ws || ws_bytes < h->fwd_ws)) return CONV_EWORKSPACE;
    SeqRecArgs a = h->rec;
    rec_inputs(a, x, f, i, A, z, f_bias, i_bias);
    a.state_in = state_in;
    a.y = y;
    a.state_out = state_out;
    a.slots = slots;
    a.lengths = lengths;
    a.totals = static_cast<float *>(ws);
    return done(launch_seq_rec_fwd(h->dtype, a, (hipStream_t)stream));
}

conv_status_t seq_rec_step(seq_handle_t h, const void *x, const void *f, const void *i, const float *A, const void *z, const float *f_bias,
                           const float *i_bias, float *state, void *y, const int32_t *slots, void *stream)
{
    if (!h || h->kind != kRec || !given(x, f, i, A, state, y) || !fine(z, f_bias, i_bias) || !aligned(slots, 4) || h->rec.n_slots == 0 || h->rec.L != 1)
        return CONV_EINVAL;
    SeqRecArgs a = h->rec;
    rec_inputs(a, x, f, i, A, z, f_bias, i_bias);
    a.state_out = state;
    a.y = y;
    a.slots = slots;
    return done(launch_seq_rec_step(h->dtype, a, (hipStream_t)stream));
}

conv_status_t seq_rec_bwd(seq_handle_t h, const void *x, const void *f, const void *i, const float *A, const void *z, const float *f_bias,
                          const float *i_bias, const void *dy, void *dx, void *df, void *di, float *dA, void *dz, float *df_bias, float *di_bias,
                          const int32_t *lengths, void *ws, size_t ws_bytes, void *stream)
{
    if (!h || h->kind != kRec || !given(x, f, i, A, dy, dx, df, di, dA) || !fine(z, f_bias, i_bias, dz, df_bias, di_bias, ws) || !aligned(lengths, 4) || !z != !dz)
        return CONV_EINVAL;
    if (!ws || ws_bytes < h->bwd_ws) return CONV_EWORKSPACE;
    SeqRecArgs a = h->rec_bwd;
    rec_inputs(a, x, f, i, A, z, f_bias, i_bias);
    a.dy = dy;
    a.dx = dx;
    a.df = df;
    a.di = di;
    a.dA = dA;
    a.dz = dz;
    a.df_bias = df_bias;
    a.di_bias = di_bias;
    a.lengths = lengths;
    char *at = static_cast<char *>(ws);
    const size_t part = up((size_t)a.N * a.runs * 3 * a.Cp * 4);
    a.part = reinterpret_cast<float *>(at);
    if (a.runs > 1) a.totals = reinterpret_cast<float *>(at += part);
    a.marks = reinterpret_cast<float *>(at + part);
    return done(launch_seq_rec_bwd(h->dtype, a, (hipStream_t)stream));
}

// ------------------------------------------------------------------ norm
static conv_status_t norm_create(Kind kind, const seq_norm_desc_t *d, seq_handle_t *out)
{
    if (!d || !out || !known(d->dtype) || !sizes_ok(d->N, d->C, d->L) || !(d->eps >= 0) || isinf(d->eps)) return CONV_EINVAL;
    const int v = vlen_of(d->dtype);
    if (!sizes_supported(d->N, d->C, d->L, v)) return CONV_EUNSUPPORTED;
    seq_plan *p = new_plan(kind, d->dtype, d->C);
    if (!p) return CONV_EUNSUPPORTED;
    SeqNormArgs &a = p->norm;
    a.N = d->N;
    a.C = d->C;
    a.L = d->L;
    a.Cb = p->info.Cb;
    a.Cp = p->info.Cp;
    a.eps = d->eps;
    a.rows = (long long)d->N * d->L;
    a.past = a.rows * a.Cb * 16 > kSeqPastBytes;
    const struct {
        const seq_view_t &v;
        bool out;
        SeqView &to;
    } views[] = {{d->x, false, a.vx}, {d->res, false, a.vres}, {d->r, true, a.vr}, {d->y, true, a.vy}, {d->dy, false, a.vdy}, {d->dr, false, a.vdr}, {d->dx, true, a.vdx}};
    for (const auto &w : views)
        if (!view_of(w.v, a.N, a.Cb, a.L, v, w.out, w.to)) return finish(p, CONV_EINVAL, out);
    if (!view_of(d->q, a.N, (a.C + 15) / 16, a.L, 16, true, a.vq)) return finish(p, CONV_EINVAL, out);
    // backward: two workgroups a compute unit, each with a part of dw (and db); of the layer norm up to four
    a.parts = (int)std::min<int64_t>(kind == kLnorm && a.rows >= 8192 ? 1024 : 512, a.rows);
    p->bwd_ws = up((size_t)a.parts * a.Cp * 4 * (kind == kLnorm ? 2 : 1));
    return finish(p, CONV_OK, out);
}
conv_status_t seq_norm_create(const seq_norm_desc_t *d, seq_handle_t *out) { return norm_create(kNorm, d, out); }

static conv_status_t norm_fwd(seq_handle_t h, const void *x, const void *res, const float *w, void *r, void *y, int8_t *q, float *scale, void *stream)
{
    SeqNormArgs a = h->norm;
    a.x = x;
    a.res = res;
    a.w = w;
    a.r = r;
    a.y = y;
    a.q = q;
    a.scale = scale;
    return done(launch_seq_norm_fwd(h->dtype, a, (hipStream_t)stream));
}
conv_status_t seq_norm_fwd(seq_handle_t h, const void *x, const void *res, const float *w, void *r, void *y, void *stream)
{
    if (!h || h->kind != kNorm || !given(x, w, y) || !fine(res, r)) return CONV_EINVAL;
    return norm_fwd(h, x, res, w, r, y, nullptr, nullptr, stream);
}
conv_status_t seq_norm_fwd_q8(seq_handle_t h, const void *x, const void *res, const float *w, void *r, int8_t *q, float *scale, void *stream)
{
    if (!h || h->kind != kNorm || !given(x, w, q, scale) || !fine(res, r)) return CONV_EINVAL;
    return norm_fwd(h, x, res, w, r, nullptr, q, scale, stream);
}
conv_status_t seq_norm_bwd(seq_handle_t h, const void *r, const float *w, const void *dy, const void *dr, void *dx, float *dw, void *ws, size_t ws_bytes,
                           void *stream)
{
    if (!h || h->kind != kNorm || !given(r, w, dy, dx, dw) || !fine(dr, ws)) return CONV_EINVAL;
    if (!ws || ws_bytes < h->bwd_ws) return CONV_EWORKSPACE;
    SeqNormArgs a = h->norm;
    a.r = const_cast<void *>(r);
    a.w = w;
    a.dy = dy;
    a.dr = dr;
    a.dx = dx;
    a.dw = dw;
    a.part = static_cast<float *>(ws);
    return done(launch_seq_norm_bwd(h->dtype, a, (hipStream_t)stream));
}

// ------------------------------------------------------------------ layer norm
conv_status_t seq_lnorm_create(const seq_lnorm_desc_t *d, seq_handle_t *out) { return norm_create(kLnorm, d, out); }

static conv_status_t lnorm_fwd(seq_handle_t h, const void *x, const void *res, const float *w, const float *b, void *r, void *y, int8_t *q, float *scale,
                               const int32_t *lengths, void *stream)
{
    SeqNormArgs a = h->norm;
    a.x = x;
    a.res = res;
    a.w = w;
    a.b = b;
    a.r = r;
    a.y = y;
    a.q = q;
    a.scale = scale;
    a.lengths = lengths;
    return done(launch_seq_lnorm_fwd(h->dtype, a, (hipStream_t)stream));
}
conv_status_t seq_lnorm_fwd(seq_handle_t h, const void *x, const void *res, const float *w, const float *b, void *r, void *y, const int32_t *lengths,
                            void *stream)
{
    if (!h || h->kind != kLnorm || !given(x, w, y) || !fine(res, b, r) || !aligned(lengths, 4)) return CONV_EINVAL;
    return lnorm_fwd(h, x, res, w, b, r, y, nullptr, nullptr, lengths, stream);
}
conv_status_t seq_lnorm_fwd_q8(seq_handle_t h, const void *x, const void *res, const float *w, const float *b, void *r, int8_t *q, float *scale,
                               const int32_t *lengths, void *stream)
{
    if (!h || h->kind != kLnorm || !given(x, w, q, scale) || !fine(res, b, r) || !aligned(lengths, 4)) return CONV_EINVAL;
    return lnorm_fwd(h, x, res, w, b, r, nullptr, q, scale, lengths, stream);
}
conv_status_t seq_lnorm_bwd(seq_handle_t h, const void *r, const float *w, const void *dy, const void *dr, void *dx, float *dw, float *db,
                            const int32_t *lengths, void *ws, size_t ws_bytes, void *stream)
{
    if (!h || h->kind != kLnorm || !given(r, w, dy, dx, dw) || !fine(dr, db, ws) || !aligned(lengths, 4)) return CONV_EINVAL;
    if (!ws || ws_bytes < h->bwd_ws) return CONV_EWORKSPACE;
    SeqNormArgs a = h->norm;
    a.r = const_cast<void *>(r);
    a.w = w;
    a.dy = dy;
    a.dr = dr;
    a.dx = dx;
    a.dw = dw;
    a.db = db;
    a.lengths = lengths;
    a.part = static_cast<float *>(ws);
    return done(launch_seq_lnorm_bwd(h->dtype, a, (hipStream_t)stream));
}

// ------------------------------------------------------------------ products with 4-bit weights
conv_status_t seq_mv4_create(const seq_mv4_desc_t *d, seq_handle_t *out)
{
    if (!d || !out || d->M < 1 || d->C < 1 || d->K < 1 || d->dtype < SEQ_F32 || d->dtype > SEQ_I8 || (d->group != 32 && d->group != 64 && d->group != 128))
        return CONV_EINVAL;
    if (d->M > 1 << 16 || d->C > 1 << 24 || d->K > 1 << 24 || (int64_t)d->C * d->K > kMaxElements) return CONV_EUNSUPPORTED;
    seq_plan *p = new_plan(kMv4, d->dtype, d->C);
    if (!p) return CONV_EUNSUPPORTED;
    SeqMv4Args &a = p->mv4;
    a.M = d->M;
    a.C = d->C;
    a.K = d->K;
    a.group = d->group;
    a.Cx = p->info.Cp;
    a.Cs = (d->C + 127) / 128;
    a.Kp = (d->K + 15) / 16 * 16;
    const int vy = d->dtype == SEQ_F32 ? 4 : 8;
    a.Ky = (d->K + vy - 1) / vy * vy;
    if ((int64_t)(a.Kp / 16) * ((a.M + 15) / 16) * 512 > kMaxItems) return finish(p, CONV_EUNSUPPORTED, out);
    p->info.wt_bytes = (size_t)a.Cs * a.Kp * 64;
    p->info.scale_bytes = (size_t)((d->C + d->group - 1) / d->group) * a.Kp * 4;
    return finish(p, CONV_OK, out);
}
conv_status_t seq_mv4(seq_handle_t h, const void *x, const float *xscale, const void *wt, const float *scale, const float *bias, void *y, void *stream)
{
    if (!h || h->kind != kMv4 || !given(x, wt, scale, y) || !fine(xscale, bias) || (h->dtype == SEQ_I8) != (xscale != nullptr)) return CONV_EINVAL;
    SeqMv4Args a = h->mv4;
    a.x = x;
    a.xscale = xscale;
    a.wt = wt;
    a.scale = scale;
    a.bias = bias;
    a.y = y;
    return done(launch_seq_mv4(h->dtype, a, (hipStream_t)stream));
}
conv_status_t seq_mv4_quant(seq_handle_t h, const float *w, void *wt, float *scale, void *stream)
{
    if (!h || h->kind != kMv4 || !given(w, wt, scale)) return CONV_EINVAL;
    return done(launch_seq_mv4_quant(h->mv4, w, wt, scale, (hipStream_t)stream));
}
conv_status_t seq_mv4_unquant(seq_handle_t h, const void *wt, const float *scale, float *w, void *stream)
{
    if (!h || h->kind != kMv4 || !given(w, wt, scale)) return CONV_EINVAL;
    SeqMv4Args a = h->mv4;
    a.wt = wt;
    a.scale = scale;
    return done(launch_seq_mv4_unquant(a, w, (hipStream_t)stream));
}

// ------------------------------------------------------------------ AdamW
conv_status_t seq_adamw_create(const seq_adamw_desc_t *d, seq_handle_t *out)
{
    const auto share = [](double x) { return x >= 0 && x < 1; };
    const auto amount = [](double x) { return x >= 0 && !isinf(x); };
    if (!d || !out || !d->sizes || !d->decays || d->count < 1 || !known(d->dtype) || (d->bits != 8 && d->bits != 32) || !share(d->beta1) || !share(d->beta2) ||
        !amount(d->eps))
        return CONV_EINVAL;
    for (int k = 0; k < d->count; ++k)
        if (d->sizes[k] < 0 || !amount(d->decays[k])) return CONV_EINVAL;
    if (d->count > 1 << 20) return CONV_EUNSUPPORTED;
    seq_plan *p = new_plan(kAdamw, d->dtype, 1);
    if (!p) return CONV_EUNSUPPORTED;
    p->tensors = new (std::nothrow) SeqAdamwTensor[d->count]();
    if (!p->tensors) return finish(p, CONV_EUNSUPPORTED, out);
    p->count = d->count;
    p->bits = d->bits;
    int64_t blocks = 0;
    for (int k = 0; k < d->count; ++k) {
        if (d->sizes[k] > kMaxNumbers - blocks * kSeqAdamwBlock) return finish(p, CONV_EUNSUPPORTED, out);
        p->tensors[k].size = d->sizes[k];
        p->tensors[k].block = (unsigned)blocks;
        p->tensors[k].decay = (float)d->decays[k];
        blocks += (d->sizes[k] + kSeqAdamwBlock - 1) / kSeqAdamwBlock;
    }
    SeqAdamwArgs &a = p->adamw;
    a.blocks = (unsigned)blocks;
    a.log1 = log(d->beta1);  // (minus infinity for zero: nothing is kept)
    a.log2 = log(d->beta2);
    a.beta1 = (float)d->beta1;
    a.rest1 = (float)(1 - d->beta1);
    a.beta2 = (float)d->beta2;
    a.rest2 = (float)(1 - d->beta2);
    a.eps = (float)d->eps;
    p->info.state_bytes = (size_t)blocks * kSeqAdamwBlock * (d->bits / 8);
    p->info.scale_bytes = d->bits == 8 ? (size_t)blocks * 8 : 0;
    return finish(p, CONV_OK, out);
}

conv_status_t seq_adamw(seq_handle_t h, void *const *p, const void *const *g, void *const *copy, void *m, void *v, float *scales, const double *now,
                        const float *now_device, void *stream)
{
    if (!h || h->kind != kAdamw || !p || !g || !now == !now_device || !aligned(now_device, 4) || !fine(m, v, scales)) return CONV_EINVAL;
    if (h->adamw.blocks && (!m || !v || (h->bits == 8) != (scales != nullptr))) return CONV_EINVAL;
    if (now && !(now[1] >= 1)) return CONV_EINVAL;
    const auto stays = [&](int k) { return !g[k] || h->tensors[k].size == 0; };
    for (int k = 0; k < h->count; ++k)
        if (!stays(k) && (!given(p[k], g[k]) || (copy && !fine(copy[k])))) return CONV_EINVAL;
    SeqAdamwArgs a = h->adamw;
    a.m = m;
    a.v = v;
    a.scales = scales;
    a.now = now_device;
    if (now) {
        a.rate = (float)now[0];
        a.by_m = (float)(now[0] / -expm1(now[1] * h->adamw.log1));
        a.by_v = (float)(1 / sqrt(-expm1(now[1] * h->adamw.log2)));
        a.factor = (float)now[2];
    }
    unsigned workgroups = 0;
    for (int k = 0; k <= h->count; ++k) {
        if (k == h->count || a.count == kSeqAdamwTensors) {
            if (a.count == 0) break;
            const hipError_t e = launch_seq_adamw(h->dtype, h->bits, a, workgroups, (hipStream_t)stream);
            if (e != hipSuccess) return CONV_ELAUNCH;
            a.count = 0;
            workgroups = 0;
        }
        if (k == h->count || stays(k)) continue;
        SeqAdamwTensor &t = a.tensor[a.count];
        t = h->tensors[k];
        t.p = static_cast<float *>(p[k]);
        t.g = g[k];
        t.copy = copy ? static_cast<unsigned short *>(copy[k]) : nullptr;
        a.first[a.count++] = workgroups;
        workgroups += (unsigned)((t.size + kSeqAdamwShare - 1) / kSeqAdamwShare);
    }
    return CONV_OK;
}

conv_status_t seq_describe(seq_handle_t h, char *buf, size_t buflen)
{
    if (!h || !buf || buflen == 0) return CONV_EINVAL;
    switch (h->kind) {
        case kConv:
            snprintf(buf, buflen, "seq_conv dt=%d W=%d fwd: runs=%d positions/run=%d bwd: runs=%d positions/run=%d columns=%lld", h->dtype, h->W, h->conv.ranges,
                     h->conv.range, h->bwd_ranges, h->bwd_range, (long long)h->conv.N * h->conv.cgroups);
            break;
        case kScan:
            snprintf(buf, buflen, "seq_scan dt=%d states=%d of %d fwd: runs=%d positions/run=%d waves=%lld bwd: runs=%d waves=%lld", h->dtype, h->scan.S,
                     seq_scan_states(h->scan.S), h->scan.chunks, h->scan.chunk, (long long)h->scan.N * h->scan.G * h->scan.tiles * h->scan.chunks,
                     h->scan_bwd.chunks, (long long)h->scan_bwd.N * h->scan_bwd.G * h->scan_bwd.btiles * h->scan_bwd.chunks);
            break;
        case kRec:
            snprintf(buf, buflen, "seq_rec dt=%d rows=%d columns=%lld fwd: runs=%d waves=%d bwd: runs=%d waves=%d rounds=%d", h->dtype, h->rec.rows,
                     (long long)(h->rec.N * seq_rec_groups(h->rec.Cp, h->rec.rows, h->info.vlen)), h->rec.runs, h->rec.waves, h->rec_bwd.runs, h->rec_bwd.waves,
                     h->rec_bwd.rounds);
            break;
        case kNorm: snprintf(buf, buflen, "seq_norm dt=%d parts=%d", h->dtype, h->norm.parts); break;
        case kLnorm: snprintf(buf, buflen, "seq_lnorm dt=%d parts=%d", h->dtype, h->norm.parts); break;
        case kAdamw: snprintf(buf, buflen, "seq_adamw dt=%d bits=%d tensors=%d blocks=%u", h->dtype, h->bits, h->count, h->adamw.blocks); break;
        case kMv4: snprintf(buf, buflen, "seq_mv4 dt=%d group=%d rows=%d runs=%d", h->dtype, h->mv4.group, h->mv4.Kp, h->mv4.Cs); break;
    }
    return CONV_OK;
}

}  // extern "C"
