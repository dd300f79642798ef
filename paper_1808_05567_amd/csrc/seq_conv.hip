// Short causal convolution of every channel, forward, backward and over one new position.
//
//   s[l] = bias + sum_k w[W-1-k] x[l-k],  k = 0 ... W-1 positions back;   y = s sigmoid(s)
//
// 2W + 10 operations an element against 4 (bf16) or 8 bytes: bound by memory.  Measured, 4 taps, 8 sequences of 2048 positions and channels in
// bf16: forward 134 MB in 25 us (5.3 TB/s), gradients 201 MB in 55 us and 5 for their sums; one position of one sequence 2.4 us.
#include "seq_internal.h"

namespace convmi {
namespace {

// A wave takes 8 blocks x 8 positions: 128 bytes side by side whether a tensor's blocks or its positions
// follow one another.  A workgroup: 8 blocks x 32 positions at a time.
constexpr int kPos = 32;

template <typename T, int W, bool PAST>
__global__ __launch_bounds__(256) void seq_conv_fwd_kernel(const SeqConvArgs a)
{
    constexpr int V = SeqElem<T>::V;
    const int ll = threadIdx.x % 8 + threadIdx.x / 64 * 8, cbl = threadIdx.x / 8 % 8;
    int t = blockIdx.x;
    const int run = t % a.ranges;
    t /= a.ranges;
    const int cbw = t % a.cgroups * 8 + cbl, n = t / a.cgroups, cb = min(cbw, a.Cb - 1);
    const bool live = cbw < a.Cb;
    const int len = seq_length(a.lengths, n, a.L);
    const T *x = static_cast<const T *>(a.x) + n * a.vx.n + cb * a.vx.c;
    T *y = static_cast<T *>(a.y) + n * a.vy.n + cb * a.vy.c;
    const int slot = a.slots ? a.slots[n] : n;
    const bool has_slot = slot >= 0 && slot < a.n_slots;
    const long long at = ((long long)slot * a.Cb + cb) * (W - 1) * V;
    const T *state = a.state_in && has_slot ? static_cast<const T *>(a.state_in) + at : nullptr;
    float w[W][V], bias[V] = {};
#pragma unroll
    for (int k = 0; k < W; ++k) seq_vector<V>(a.w + (long long)k * a.Cp, cb, w[k]);
    if (a.bias) seq_vector<V>(a.bias, cb, bias);
    const int end = live ? min(a.L, (run + 1) * a.range) : 0;
    for (int l = run * a.range + ll; l < end; l += kPos) {
        seq_u32x4 out = {};
        if (l < len) {
            float s[V];
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] = bias[i];
#pragma unroll
            for (int k = W - 1; k >= 0; --k) {
                seq_u32x4 b = {};
                if (l >= k)
                    b = seq_load(x + (l - k) * a.vx.l);
                else if (state)
                    b = seq_load(state + (W - 1 + l - k) * V);
                float f[V];
                SeqElem<T>::unpack(b, f);
#pragma unroll
                for (int i = 0; i < V; ++i) s[i] = fmaf(w[W - 1 - k][i], f[i], s[i]);
            }
            if (a.silu)
#pragma unroll
                for (int i = 0; i < V; ++i) s[i] *= seq_sigmoid(s[i]);
            out = SeqElem<T>::pack(s);
        }
        seq_store_result<PAST>(y + l * a.vy.l, out);
    }
    if (run != 0 || !a.state_out) return;
    // The last W - 1 inputs.  By the workgroup that has read the old state, once all of it has: the new one may lie in its place.
    seq_u32x4 last = {};
    const int l = len - (W - 1) + ll;
    if (ll < W - 1) {
        if (l >= 0)
            last = seq_load(x + l * a.vx.l);
        else if (state)
            last = seq_load(state + (W - 1 + l) * V);
    }
    __syncthreads();
    if (ll < W - 1 && live && has_slot) seq_store(static_cast<T *>(a.state_out) + at + ll * V, last);
}

template <typename T, int W>
__global__ __launch_bounds__(64) void seq_conv_step_kernel(const SeqConvArgs a)
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
    T *state = static_cast<T *>(a.state_out) + ((long long)slot * a.Cb + cb) * (W - 1) * V;
    seq_u32x4 b[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) b[j] = seq_load(state + j * V);
    b[W - 1] = seq_load(static_cast<const T *>(a.x) + n * a.vx.n + cb * a.vx.c);
    float s[V] = {};
    if (a.bias) seq_vector<V>(a.bias, cb, s);
#pragma unroll
    for (int j = 0; j < W; ++j) {
        float f[V], w[V];
        SeqElem<T>::unpack(b[j], f);
        seq_vector<V>(a.w + (long long)j * a.Cp, cb, w);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = fmaf(w[i], f[i], s[i]);
    }
    if (a.silu)
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] *= seq_sigmoid(s[i]);
    seq_store(y, SeqElem<T>::pack(s));
#pragma unroll
    for (int j = 0; j < W - 1; ++j) seq_store(state + j * V, b[j + 1]);
}

//   ds = dy silu'(s),  dx[l] = sum_k w[W-1-k] ds[l+k],  dw[W-1-k] = sum_l ds[l] x[l-k],  dbias = sum_l ds[l]
//
// A workgroup walks along its run of positions, 32 at a time.  What its threads need of each other's numbers goes through rings in LDS of the last
// 128 positions, so that x and dy are loaded and ds is formed once: x of a tile is written while ds of the one before is
// formed and dx of the one before that, for positions W - 1 back, whose last ds has come by then; one barrier a tile.
// ds of the W - 1 positions behind the run is formed here too.
// Some 300 operations for the eight bf16 numbers of a block, two thirds of them for silu' and unpacking: the vector units need nearly as long as
// memory does.  (Two barriers a tile, loads of x from each thread, LDS rows in the same banks: 8 x 2048 x 2048 bf16 97 us.)
template <typename T, int W>
__global__ __launch_bounds__(256) void seq_conv_bwd_kernel(const SeqConvArgs a)
{
    constexpr int V = SeqElem<T>::V, Q = V / 4, RING = 128;
    // [block][position]: eight lanes side by side take 128 bytes in a row
    __shared__ __align__(16) seq_u32x4 rx[8][RING];
    __shared__ __align__(16) seq_f32x4 rd[Q][8][RING];
    const int wave = threadIdx.x / 64, ll = threadIdx.x % 8 + wave * 8, cbl = threadIdx.x / 8 % 8;
    int t = blockIdx.x;
    const int run = t % a.ranges;
    t /= a.ranges;
    const int group = t % a.cgroups, n = t / a.cgroups;
    const bool live = group * 8 + cbl < a.Cb;
    const int cb = live ? group * 8 + cbl : 0;
    const int len = live ? seq_length(a.lengths, n, a.L) : 0;
    const T *x = static_cast<const T *>(a.x) + n * a.vx.n + cb * a.vx.c;
    const T *dy = static_cast<const T *>(a.dy) + n * a.vdy.n + cb * a.vdy.c;
    T *dx = static_cast<T *>(a.dx) + n * a.vdx.n + cb * a.vdx.c;
    float w[W][V], bias[V] = {}, dw[W + 1][V] = {};
#pragma unroll
    for (int k = 0; k < W; ++k) seq_vector<V>(a.w + (long long)k * a.Cp, cb, w[k]);
    if (a.bias) seq_vector<V>(a.bias, cb, bias);

    const int begin = run * a.range, end = min(a.L, begin + a.range);
    const int stop = min(len, end + W - 1);  // behind the last position whose ds is formed
    const int tiles = (end - begin + kPos - 1) / kPos;
    auto load = [&](const T *p, long long stride, int l) { return l >= 0 && l < stop ? seq_load(p + l * stride) : seq_u32x4{}; };
    if (ll < W - 1) rx[cbl][(RING - 1 - ll) % RING] = load(x, a.vx.l, begin - 1 - ll);
    rx[cbl][ll] = load(x, a.vx.l, begin + ll);
    seq_u32x4 nx = load(x, a.vx.l, begin + kPos + ll), ny = load(dy, a.vdy.l, begin + ll);
    float own[V] = {};  // ds of the tile before, at this thread's place
    __syncthreads();
    for (int i = 0; i <= tiles + 1; ++i) {
        const int l = begin + i * kPos + ll, at = (i * kPos + ll) % RING;
        rx[cbl][(at + kPos) % RING] = nx;
        const seq_u32x4 cy = ny;
        nx = load(x, a.vx.l, l + 2 * kPos);
        ny = load(dy, a.vdy.l, l + kPos);
        float ds[V] = {};
        if (l < stop) {
            float g[V], s[V], f[W][V];
            SeqElem<T>::unpack(cy, g);
#pragma unroll
            for (int j = 0; j < V; ++j) s[j] = bias[j];
#pragma unroll
            for (int k = W - 1; k >= 0; --k) {
                SeqElem<T>::unpack(rx[cbl][(at + RING - k) % RING], f[k]);
#pragma unroll
                for (int j = 0; j < V; ++j) s[j] = fmaf(w[W - 1 - k][j], f[k][j], s[j]);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float p = seq_sigmoid(s[j]);
                ds[j] = a.silu ? g[j] * p * fmaf(s[j], 1.0f - p, 1.0f) : g[j];
            }
            // (what lies behind the run counts in the next one)
            if (l < end) {
#pragma unroll
                for (int j = 0; j < V; ++j) dw[W][j] += ds[j];
#pragma unroll
                for (int k = 0; k < W; ++k)
#pragma unroll
                    for (int j = 0; j < V; ++j) dw[W - 1 - k][j] = fmaf(ds[j], f[k][j], dw[W - 1 - k][j]);
            }
        }
#pragma unroll
        for (int q = 0; q < Q; ++q) rd[q][cbl][at] = seq_f32x4{ds[4 * q], ds[4 * q + 1], ds[4 * q + 2], ds[4 * q + 3]};
        const int back = l - kPos - (W - 1);  // where dx is complete
        if (live && back >= begin && back < end) {
            float d[V];
#pragma unroll
            for (int j = 0; j < V; ++j) d[j] = w[0][j] * own[j];
#pragma unroll
            for (int k = 1; k < W; ++k)
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    const seq_f32x4 e = rd[q][cbl][(at + RING - kPos - k) % RING];
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[4 * q + j] = fmaf(w[k][4 * q + j], e[j], d[4 * q + j]);
                }
            seq_store(dx + back * a.vdx.l, back < len ? SeqElem<T>::pack(d) : seq_u32x4{});
        }
#pragma unroll
        for (int j = 0; j < V; ++j) own[j] = ds[j];
        __syncthreads();
    }
    // the workgroup's sums: over the 8 positions of a wave, then over the waves in order
    float *lds = reinterpret_cast<float *>(rd);  // [wave][8][V]
#pragma unroll
    for (int k = 0; k <= W; ++k) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float s = dw[k][j];
            s += __shfl_xor(s, 1);
            s += __shfl_xor(s, 2);
            s += __shfl_xor(s, 4);
            if (threadIdx.x % 8 == 0) lds[(wave * 8 + cbl) * V + j] = s;
        }
        __syncthreads();
        if (threadIdx.x < 8 * V && group * 8 + threadIdx.x / V < a.Cb) {
            float s = 0;
#pragma unroll
            for (int v = 0; v < 4; ++v) s += lds[v * 8 * V + threadIdx.x];
            const long long part = (long long)n * a.ranges + run;
            a.part[(part * (W + 1) + k) * a.Cp + group * 8 * V + threadIdx.x] = s;
        }
        __syncthreads();
    }
}

// dw and dbias: the workgroups' sums, in order.
__global__ __launch_bounds__(1024) void seq_conv_reduce_kernel(const float *part, float *dw, float *dbias, int parts, int W, int Cp)
{
    const int col = blockIdx.x * kSumColumns + threadIdx.x % kSumColumns, total = (W + 1) * Cp;
    const float s = seq_sum_parts(part + col, total, parts, col < total);
    if (threadIdx.x >= kSumColumns || col >= total) return;
    if (col < W * Cp)
        dw[col] = s;
    else if (dbias)
        dbias[col - W * Cp] = s;
}

template <typename T, int W>
hipError_t launch(int which, const SeqConvArgs &a, hipStream_t s)
{
    const long long vectors = (long long)a.N * a.Cb;
    if (which == 1) {
        seq_conv_step_kernel<T, W><<<(unsigned)((vectors + 63) / 64), 64, 0, s>>>(a);
        return hipGetLastError();
    }
    const unsigned grid = (unsigned)((long long)a.N * a.cgroups * a.ranges);
    if (which == 0) {
        if (a.past)
            seq_conv_fwd_kernel<T, W, true><<<grid, 256, 0, s>>>(a);
        else
            seq_conv_fwd_kernel<T, W, false><<<grid, 256, 0, s>>>(a);
        return hipGetLastError();
    }
    seq_conv_bwd_kernel<T, W><<<grid, 256, 0, s>>>(a);
    seq_conv_reduce_kernel<<<((W + 1) * a.Cp + kSumColumns - 1) / kSumColumns, 1024, 0, s>>>(a.part, a.dw, a.dbias, a.N * a.ranges, W, a.Cp);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_w(int which, int W, const SeqConvArgs &a, hipStream_t s)
{
    switch (W) {
        case 2: return launch<T, 2>(which, a, s);
        case 3: return launch<T, 3>(which, a, s);
        case 4: return launch<T, 4>(which, a, s);
        case 5: return launch<T, 5>(which, a, s);
        case 6: return launch<T, 6>(which, a, s);
        case 7: return launch<T, 7>(which, a, s);
        case 8: return launch<T, 8>(which, a, s);
    }
    return hipErrorInvalidValue;
}
hipError_t launch_t(int which, int dtype, int W, const SeqConvArgs &a, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch_w<unsigned short>(which, W, a, s) : launch_w<float>(which, W, a, s);
}
}  // namespace

hipError_t launch_seq_conv_fwd(int dtype, int W, const SeqConvArgs &a, hipStream_t s) { return launch_t(0, dtype, W, a, s); }
hipError_t launch_seq_conv_step(int dtype, int W, const SeqConvArgs &a, hipStream_t s) { return launch_t(1, dtype, W, a, s); }
hipError_t launch_seq_conv_bwd(int dtype, int W, const SeqConvArgs &a, hipStream_t s) { return launch_t(2, dtype, W, a, s); }

}  // namespace convmi
