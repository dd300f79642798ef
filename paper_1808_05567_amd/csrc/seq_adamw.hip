// AdamW step over many tensors, the states in fp32 or as roots in 8 bits with a scale for each 256 numbers.
//
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,  p = p - rate decay p - rate (m / c1) / (sqrt(v / c2) + eps),  c = 1 - beta^t
//
// Bound by memory: every number is read and written once, in a launch for 80 tensors, whose pointers are kernel arguments (nothing is kept on the GPU for a plan, and a recorded
// step has them with it).  A workgroup has 4096 numbers of one tensor, a wave 256 at a time, so that the scales' largest are a wave's own.  Measured: 10.6 M numbers, fp32 states,
// gradients and a bf16 copy, 317 MB: 66 us (4.8 TB/s); 58.7 M with 8-bit states, bf16 gradients and copies, 940 MB: 200 us (4.7 TB/s; 135 operations a number, which keep the vector units busy for at least 0.6 of that); 64 vectors, 0.1 M: 4.
//
// Roots in 8 bits: m's is signed and v's is the fourth, for sqrt(v) is what p is divided by.  With steps of 1/127 of the largest root an m below 1.6e-5 of its block's largest becomes
// zero (without roots 4e-3 would); with steps of 1/255 a sqrt(v) below 1.5e-5 of the largest stays at one step, rather than at zero, which would divide by eps alone.
#include "seq_internal.h"

namespace convmi {
namespace {

constexpr int kEach = 4;  // numbers of a lane side by side: a wave has a block of 256

// Four numbers from element e of size on, zeros beyond.
template <typename T>
static __device__ __forceinline__ void load4(const T *p, int64_t e, int64_t size, float (&f)[kEach])
{
    if (e + kEach <= size) {
        if constexpr (sizeof(T) == 4) {
            const seq_f32x4 b = *reinterpret_cast<const seq_f32x4 *>(p + e);
#pragma unroll
            for (int i = 0; i < kEach; ++i) f[i] = b[i];
        } else {
            const seq_u32x2 b = *reinterpret_cast<const seq_u32x2 *>(p + e);
#pragma unroll
            for (int i = 0; i < kEach; ++i) f[i] = __uint_as_float(i % 2 ? b[i / 2] & 0xFFFF0000u : b[i / 2] << 16);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) f[i] = e + i < size ? SeqElem<T>::get(p[e + i]) : 0.0f;
}
template <typename T>
static __device__ __forceinline__ void store4(T *p, int64_t e, int64_t size, const float (&f)[kEach])
{
    if (e + kEach <= size) {
        if constexpr (sizeof(T) == 4)
            *reinterpret_cast<seq_f32x4 *>(p + e) = seq_f32x4{f[0], f[1], f[2], f[3]};
        else
            *reinterpret_cast<seq_u32x2 *>(p + e) = seq_u32x2{seq_pack_bf16(f[0], f[1]), seq_pack_bf16(f[2], f[3])};
        return;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (e + i < size) p[e + i] = SeqElem<T>::put(f[i]);
}

// Largest of a wave's numbers, as unsigned ones: NaN is larger than all.
static __device__ __forceinline__ float wave_max(float m)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) m = __uint_as_float(max(__float_as_uint(m), __float_as_uint(__shfl_xor(m, d))));
    return m;
}

template <typename G, int BITS>
__global__ __launch_bounds__(256) void seq_adamw_kernel(const SeqAdamwArgs a)
{
    int k = 0;  // the workgroup's tensor
    for (int step = 64; step > 0; step /= 2)
        if (k + step < a.count && a.first[k + step] <= blockIdx.x) k += step;
    const SeqAdamwTensor t = a.tensor[k];
    float lr = a.rate, by_m = a.by_m, by_v = a.by_v, factor = a.factor;
    if (a.now) {
        lr = a.now[0];
        factor = a.now[2];
        by_m = lr / -expm1f((float)(a.now[1] * a.log1));
        by_v = 1.0f / sqrtf(-expm1f((float)(a.now[1] * a.log2)));
    }
    const float keep = lr * t.decay;
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const int64_t begin = (int64_t)(blockIdx.x - a.first[k]) * kSeqAdamwShare;
#pragma unroll 1
    for (int b = wave; b < kSeqAdamwShare / kSeqAdamwBlock; b += 4) {
        const int64_t from = begin + b * kSeqAdamwBlock;
        if (from >= t.size) return;
        const int64_t e = from + lane * kEach;
        const unsigned block = t.block + (unsigned)(from / kSeqAdamwBlock);
        const int64_t at = (int64_t)block * kSeqAdamwBlock + lane * kEach;
        float p[kEach], g[kEach], m[kEach], v[kEach], root[kEach];
        load4(t.p, e, t.size, p);
        load4(static_cast<const G *>(t.g), e, t.size, g);
        if constexpr (BITS == 32) {
            load4(static_cast<const float *>(a.m), at, at + kEach, m);
            load4(static_cast<const float *>(a.v), at, at + kEach, v);
        } else {
            const unsigned bm = *reinterpret_cast<const unsigned *>(static_cast<const char *>(a.m) + at);
            const unsigned bv = *reinterpret_cast<const unsigned *>(static_cast<const char *>(a.v) + at);
            const float sm = a.scales[block], sv = a.scales[a.blocks + block];
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const float qm = (float)(int)(signed char)(bm >> 8 * i) * sm, qv = (float)(bv >> 8 * i & 255) * sv;
                m[i] = qm * fabsf(qm);
                v[i] = qv * qv * (qv * qv);
            }
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (e + i >= t.size) m[i] = v[i] = 0;
            const float s = g[i] * factor;
            {
                // (each product rounded by itself, as the formula's operations one after the other are: in 8 bits a root next to a half is rounded as theirs is)
#pragma clang fp contract(off)
                m[i] = a.rest1 * s + a.beta1 * m[i];
                v[i] = a.rest2 * (s * s) + a.beta2 * v[i];
            }
            root[i] = sqrtf(v[i]);
            p[i] = p[i] - keep * p[i] - by_m * m[i] / fmaf(root[i], by_v, a.eps);
        }
        store4(t.p, e, t.size, p);
        if (t.copy) store4(t.copy, e, t.size, p);
        if constexpr (BITS == 32) {
            store4(static_cast<float *>(a.m), at, at + kEach, m);
            store4(static_cast<float *>(a.v), at, at + kEach, v);
        } else {
            float xm = 0, xv = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                // (roots of m with its sign, and of v's root)
                m[i] = copysignf(sqrtf(fabsf(m[i])), m[i]);
                root[i] = sqrtf(root[i]);
                xm = __uint_as_float(max(__float_as_uint(xm), __float_as_uint(fabsf(m[i]))));
                xv = __uint_as_float(max(__float_as_uint(xv), __float_as_uint(root[i])));
            }
            // (not infinite: what is not zero would stand for infinity, an infinite v, which stops a parameter and does not show)
            const auto scale_of = [](float largest, float by) { return largest < INFINITY ? largest * by : NAN; };
            const float sm = scale_of(wave_max(xm), 1 / 127.0f), sv = scale_of(wave_max(xv), 1 / 255.0f);
            const float im = sm == 0 ? 0 : 1.0f / sm, iv = sv == 0 ? 0 : 1.0f / sv;
            // a root over the scale, with what its product with the rounded reciprocal is off by, so that what is next to a half goes to the side that the quotient does
            const auto over = [](float x, float scale, float inverse) {
                const float q = x * inverse;
                return fmaf(fmaf(-q, scale, x), inverse, q);
            };
            unsigned bm = 0, bv = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int qm = (int)rintf(fminf(fmaxf(over(m[i], sm, im), -127.0f), 127.0f));
                const int qv = (int)rintf(fminf(over(root[i], sv, iv), 255.0f));
                bm |= (unsigned)(qm & 255) << 8 * i;
                bv |= (unsigned)(root[i] > 0 && qv == 0 ? 1 : qv) << 8 * i;
            }
            *reinterpret_cast<unsigned *>(static_cast<char *>(a.m) + at) = bm;
            *reinterpret_cast<unsigned *>(static_cast<char *>(a.v) + at) = bv;
            if (lane == 0) {
                a.scales[block] = sm;
                a.scales[a.blocks + block] = sv;
            }
        }
    }
}

template <typename G>
hipError_t launch(int bits, const SeqAdamwArgs &a, unsigned workgroups, hipStream_t s)
{
    if (bits == 8)
        seq_adamw_kernel<G, 8><<<workgroups, 256, 0, s>>>(a);
    else
        seq_adamw_kernel<G, 32><<<workgroups, 256, 0, s>>>(a);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_seq_adamw(int dtype, int bits, const SeqAdamwArgs &a, unsigned workgroups, hipStream_t s)
{
    return dtype == SEQ_BF16 ? launch<unsigned short>(bits, a, workgroups, s) : launch<float>(bits, a, workgroups, s);
}

}  // namespace convmi
