// Short causal convolution of every channel, forward, backward and over one new position.
//
//   s[l] = bias + sum_k w[W-1-k] x[l-k],  k = 0 ... W-1 positions back;   y = s sigmoid(s)
//
// 2W + 10 operations an element against 4 (bf16) or 8 bytes: bound by memory.
#include "seq_internal.h"

namespace convmi {
namespace {

// A wave takes 8 blocks x 8 positions: 128 bytes side by side whether a tensor's blocks or its positions
// follow one another.  A workgroup: 8 blocks x 32 positions at a time.
constexpr int kPos = 32;

template <typename T, int W>
__global__ __launch_bounds__(256) void seq_conv_fwd_kernel(const SeqConvArgs a)
{
    constexpr int V = SeqElem<T>::V;
    const int ll = threadIdx.x % 8 + threadIdx.x / 64 * 8, cbl = threadIdx.x / 8 % 8;
    int t = blockIdx.x;
    const int run = t % a.ranges;
    t /= a.ranges;
    const int cb = t % a.cgroups * 8 + cbl, n = t / a.cgroups;
    if (cb >= a.Cb) return;
    const int len = seq_length(a.lengths, n, a.L);
    const T *x = static_cast<const T *>(a.x) + n * a.vx.n + cb * a.vx.c;
    T *y = static_cast<T *>(a.y) + n * a.vy.n + cb * a.vy.c;
    const int slot = a.slots ? a.slots[n] : n;
    const T *state = a.state_in && slot >= 0 && slot < a.n_slots
                         ? static_cast<const T *>(a.state_in) + ((long long)slot * a.Cb + cb) * (W - 1) * V : nullptr;
    float w[W][V], bias[V] = {};
#pragma unroll
    for (int k = 0; k < W; ++k) seq_vector<V>(a.w + (long long)k * a.Cp, cb, w[k]);
    if (a.bias) seq_vector<V>(a.bias, cb, bias);
    const int end = min(a.L, (run + 1) * a.range);
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
        seq_store(y + l * a.vy.l, out);
    }
}

// The last W - 1 inputs of each sequence, those before its start taken from the old state: one thread reads all that it
// writes first, so that the state may be moved on in place.
template <typename T, int W>
__global__ __launch_bounds__(256) void seq_conv_state_kernel(const SeqConvArgs a)
{
    constexpr int V = SeqElem<T>::V;
    const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
    if (t >= (long long)a.N * a.Cb) return;
    const int n = (int)(t / a.Cb), cb = (int)(t % a.Cb);
    const int slot = a.slots ? a.slots[n] : n;
    if (slot < 0 || slot >= a.n_slots) return;
    const int len = seq_length(a.lengths, n, a.L);
    const T *x = static_cast<const T *>(a.x) + n * a.vx.n + cb * a.vx.c;
    const long long at = ((long long)slot * a.Cb + cb) * (W - 1) * V;
    seq_u32x4 b[W - 1];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int l = len - (W - 1) + j;
        b[j] = seq_u32x4{};
        if (l >= 0)
            b[j] = seq_load(x + l * a.vx.l);
        else if (a.state_in)
            b[j] = seq_load(static_cast<const T *>(a.state_in) + at + (len + j) * V);
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) seq_store(static_cast<T *>(a.state_out) + at + j * V, b[j]);
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
// A workgroup walks its run of positions from the back.  ds goes through LDS, so that each is formed once; the first
// W - 1 of a tile stay there for the tile before it, those behind the run are formed here too.
template <typename T, int W>
__global__ __launch_bounds__(256) void seq_conv_bwd_kernel(const SeqConvArgs a)
{
    constexpr int V = SeqElem<T>::V;
    __shared__ float lds[(kPos + W - 1) * 8 * V];  // [position][block][V]; at the end [wave][8][V] of one sum
    const int wave = threadIdx.x / 64, ll = threadIdx.x % 8 + wave * 8, cbl = threadIdx.x / 8 % 8;
    int t = blockIdx.x;
    const int run = t % a.ranges;
    t /= a.ranges;
    const int cb = t % a.cgroups * 8 + cbl, n = t / a.cgroups;
    const bool live = cb < a.Cb;
    const int len = live ? seq_length(a.lengths, n, a.L) : 0;
    const int cbs = live ? cb : 0;
    const T *x = static_cast<const T *>(a.x) + n * a.vx.n + cbs * a.vx.c;
    const T *dy = static_cast<const T *>(a.dy) + n * a.vdy.n + cbs * a.vdy.c;
    T *dx = static_cast<T *>(a.dx) + n * a.vdx.n + cbs * a.vdx.c;
    float w[W][V], bias[V] = {}, dw[W + 1][V] = {};
#pragma unroll
    for (int k = 0; k < W; ++k) seq_vector<V>(a.w + (long long)k * a.Cp, cbs, w[k]);
    if (a.bias) seq_vector<V>(a.bias, cbs, bias);

    // ds at position l, and the x that it came from
    auto form = [&](int l, float (&ds)[V], float (&f)[W][V]) {
#pragma unroll
        for (int i = 0; i < V; ++i) ds[i] = 0;
#pragma unroll
        for (int k = 0; k < W; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) f[k][i] = 0;
        if (l >= len) return;
        float g[V], s[V];
        SeqElem<T>::unpack(seq_load(dy + l * a.vdy.l), g);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = bias[i];
#pragma unroll
        for (int k = W - 1; k >= 0; --k) {
            if (l >= k) SeqElem<T>::unpack(seq_load(x + (l - k) * a.vx.l), f[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] = fmaf(w[W - 1 - k][i], f[k][i], s[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float p = seq_sigmoid(s[i]);
            ds[i] = a.silu ? g[i] * p * (1.0f + s[i] * (1.0f - p)) : g[i];
        }
    };
    float *mine = lds + (ll * 8 + cbl) * V;
    const int begin = run * a.range, end = min(a.L, begin + a.range);
    const int tiles = (end - begin + kPos - 1) / kPos;
    for (int i = tiles - 1; i >= 0; --i) {
        const int l = begin + i * kPos + ll;
        float ds[V], f[W][V];
        if (i == tiles - 1) {
            if (ll < W - 1) {
                form(l + kPos, ds, f);
#pragma unroll
                for (int j = 0; j < V; ++j) mine[kPos * 8 * V + j] = ds[j];
            }
        }
        form(l, ds, f);
        // (positions past the run's end belong to the next one: here they are only read)
        if (l < end) {
#pragma unroll
            for (int j = 0; j < V; ++j) dw[W][j] += ds[j];
#pragma unroll
            for (int k = 0; k < W; ++k)
#pragma unroll
                for (int j = 0; j < V; ++j) dw[W - 1 - k][j] = fmaf(ds[j], f[k][j], dw[W - 1 - k][j]);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) mine[j] = ds[j];
        __syncthreads();
        float d[V];
#pragma unroll
        for (int j = 0; j < V; ++j) d[j] = w[W - 1][j] * ds[j];
#pragma unroll
        for (int k = 1; k < W; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) d[j] = fmaf(w[W - 1 - k][j], mine[k * 8 * V + j], d[j]);
        if (live && l < end) {
            if (l >= len)
#pragma unroll
                for (int j = 0; j < V; ++j) d[j] = 0;
            seq_store(dx + l * a.vdx.l, SeqElem<T>::pack(d));
        }
        __syncthreads();
        if (ll < W - 1)
#pragma unroll
            for (int j = 0; j < V; ++j) mine[kPos * 8 * V + j] = ds[j];
    }
    // the workgroup's sums: over the 8 positions of a wave, then over the waves in order
    __syncthreads();
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
        if (threadIdx.x < 8 * V && blockIdx.x / a.ranges % a.cgroups * 8 + threadIdx.x / V < a.Cb) {
            float s = 0;
#pragma unroll
            for (int v = 0; v < 4; ++v) s += lds[v * 8 * V + threadIdx.x];
            const int c = blockIdx.x / a.ranges % a.cgroups * 8 * V + threadIdx.x;
            const long long part = (long long)n * a.ranges + run;
            a.part[(part * (W + 1) + k) * a.Cp + c] = s;
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
        seq_conv_fwd_kernel<T, W><<<grid, 256, 0, s>>>(a);
        if (a.state_out) seq_conv_state_kernel<T, W><<<(unsigned)((vectors + 255) / 256), 256, 0, s>>>(a);
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
