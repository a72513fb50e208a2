// One AdamW step over many tensors (decoupled weight decay), moments in FP32 or in 8 bits.
//
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2,
//   p' = p (1 - lr wd) - lr / (1 - b1^t) * m' / (sqrt(v') / sqrt(1 - b2^t) + eps)
//
// Nothing is used twice: the floor is memory, per element 8 bytes of p, the gradient, and 16 bytes of FP32 moments or 4.125 of 8-bit
// ones.  One kernel goes once over all tensors: runs of 1024 or 2048 elements of one tensor, found in the list that travels in
// the kernel's arguments, go round the blocks that the SMs hold.  The blocks work the bias corrections out themselves from the
// step count on the device, so a captured launch can be replayed; the last block to have read the count moves it on.
// FP32 moments: 6.2 M elements in 256 tensors 36 us, 5.2 TB/s.  8-bit moments: 73.7 M elements 281 to 295 us, 4.1 TB/s (257 with a part in
// the L2), of which the issue of 97 instructions per element takes 202 at 1.87 GHz; 73 % of the issue slots are used; warps wait
// for arithmetic pipes and fixed latencies, hardly for memory.  The same 256 tensors 32 us.
//
// 8-bit moments: E4M3 codes of m and of r = sqrt(v) (which halves the range of exponents that v needs), a power-of-two
// scale (E8M0 byte) per 32 elements that brings the largest magnitude into [128, 256).  Scaling is then exact and codes
// depend on the element and its block alone.  A step changes v by a thousandth, far below half a step of a 3-bit
// mantissa: rounded to nearest it would never move, so the codes are rounded stochastically with 16 bits of a hash of
// (seed, t, element number).  The parameter's own update uses the moments before they are rounded.  A nonzero r keeps
// the code 1 at least: at 0 the next update would divide by eps.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>
#include <type_traits>
#include <string.h>

#include "fpq_kernels.h"
#include "fpq_roots.cuh"

namespace fpq {

namespace {

constexpr int ADAMW_THREADS = 256;
constexpr int ADAMW_LAUNCH = 400;          // tensors per launch: their descriptors fill most of the 32764 bytes of arguments
constexpr int ADAMW_SMALL = 16;            // tensors of the variant with short arguments

struct AdamwScalars {
    double ln_beta1, ln_beta2, lr, weight_decay;
    float beta1, rest1, beta2, rest2, eps;
    uint32_t seed;
    const float* factors;                  // {of lr, of the gradients} or NULL
    long long* step;                       // {steps made, 0}
    int last;                              // this launch moves the count on
};

template <int CAP>
struct AdamwList {
    fpq_adamw_tensor t[CAP];
    uint32_t first_run[CAP + 1];           // runs of the tensors in front
    uint64_t first_block[CAP];             // blocks of 32 elements of the tensors in front, all launches counted
    uint8_t vec[CAP];                      // every pointer aligned for four elements at a time
    int count;
};

__device__ __forceinline__ uint32_t mix(uint32_t z)
{
    z *= 0x9E3779B1u;
    z ^= z >> 15;
    z *= 0x243F6A89u;
    return z ^ (z >> 16);
}

__device__ __forceinline__ float2 values_e4m3x2(uint32_t two)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    __half2 v;
    memcpy(&v, &h, 4);
    return __half22float2(v);
}

// N values that lie side by side, as they lie, 16 (8 for four 16-bit values) bytes at a time; what they are worth is looked at where
// they are used, so that no load waits for another
template <int N, typename T>
__device__ __forceinline__ void load_words(const T* p, uint32_t* w)
{
    if constexpr (N * sizeof(T) == 4) {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else if constexpr (N * sizeof(T) == 8) {
        const uint2 q = *reinterpret_cast<const uint2*>(p);
        w[0] = q.x; w[1] = q.y;
    } else {
#pragma unroll
        for (int i = 0; i < N * (int)sizeof(T) / 16; ++i) {
            const uint4 q = reinterpret_cast<const uint4*>(p)[i];
            w[4 * i] = q.x; w[4 * i + 1] = q.y; w[4 * i + 2] = q.z; w[4 * i + 3] = q.w;
        }
    }
}

template <typename T>
__device__ __forceinline__ float value_at(const uint32_t* w, int i);
template <>
__device__ __forceinline__ float value_at<float>(const uint32_t* w, int i) { return __uint_as_float(w[i]); }
template <>
__device__ __forceinline__ float value_at<__nv_bfloat16>(const uint32_t* w, int i)
{
    return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
}
template <>
__device__ __forceinline__ float value_at<__half>(const uint32_t* w, int i)
{
    return __half2float(__ushort_as_half((unsigned short)(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu)));
}

// What a thread has of one run: P elements from e on, `left` of them the tensor's
template <typename GT, bool E4>
struct Piece {
    static constexpr int P = E4 ? 8 : 4;
    int64_t e;
    int tensor, left;
    bool fast;
    uint32_t p[P], g[P * sizeof(GT) / 4], m[E4 ? P / 4 : P], v[E4 ? P / 4 : P], m_scale, v_scale;

    template <int CAP>
    __device__ __forceinline__ void load(const AdamwList<CAP>& L, uint32_t at)
    {
        using State = typename std::conditional<E4, uint8_t, float>::type;
        int lo = 0;                        // the tensor of this run: the last one whose first run is not behind it
        for (int hi = L.count; hi - lo > 1;) {
            const int mid = (lo + hi) >> 1;
            if (L.first_run[mid] <= at)
                lo = mid;
            else
                hi = mid;
        }
        tensor = lo;
        const fpq_adamw_tensor& T = L.t[lo];
        e = (int64_t)(at - L.first_run[lo]) * (ADAMW_THREADS * P) + threadIdx.x * P;
        left = e >= T.n ? 0 : T.n - e < P ? (int)(T.n - e) : P;
        fast = left == P && L.vec[lo] != 0;
        const State *mp = (const State*)T.m + e, *vp = (const State*)T.v + e;
        const GT* gp = (const GT*)T.g + e;
        if (fast) {
            load_words<P>(T.p + e, p);
            load_words<P>(gp, g);
            load_words<P>(mp, m);
            load_words<P>(vp, v);
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                p[i] = i < left ? __float_as_uint(T.p[e + i]) : 0u;
                put(g, i, i < left ? gp + i : nullptr);
                put(m, i, i < left ? mp + i : nullptr);
                put(v, i, i < left ? vp + i : nullptr);
            }
        }
        if (E4) {
            m_scale = left ? T.m_scale[e >> 5] : 0;
            v_scale = left ? T.v_scale[e >> 5] : 0;
        }
    }

    template <typename T>
    static __device__ __forceinline__ void put(uint32_t* w, int i, const T* from)
    {
        constexpr int PER = 4 / (int)sizeof(T);
        uint32_t x = 0;
        if (from)
            x = sizeof(T) == 4 ? *reinterpret_cast<const uint32_t*>(from)
                : sizeof(T) == 2 ? *reinterpret_cast<const uint16_t*>(from) : *reinterpret_cast<const uint8_t*>(from);
        w[i / PER] = (i % PER ? w[i / PER] : 0u) | x << (32 / PER * (i % PER)) % 32;
    }
};

__device__ __forceinline__ uint32_t pack_two(float a, float b, int bf16)
{
    uint32_t w;
    if (bf16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
        memcpy(&w, &v, 4);
    } else {
        const __half2 v = __floats2half2_rn(a, b);
        memcpy(&w, &v, 4);
    }
    return w;
}

// Four E4M3 codes of q[0 .. 3] (0 <= |q| < 256), each rounded up if the remainder below its step plus 16 bits of noise carries; noise[i]
// holds them at bits 4 .. 19, the rest zero.  Below 2^-6 the steps are equal: with 2^-6 added they are the steps of that
// binade.  SIGNED: with the signs, but a zero has none; otherwise what is not zero keeps the code 1 at least.
template <bool SIGNED>
__device__ __forceinline__ uint32_t stochastic_e4m3x4(const float* q, const uint32_t* noise)
{
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = SIGNED ? fabsf(q[i]) : q[i];
        float t = a;
        uint32_t n = noise[i] - (960u << 20);
        if (a < 0.015625f) {
            t = __fadd_rn(a, 0.015625f);
            n -= 8u << 20;
        }
        c[i] = (__float_as_uint(t) + n) >> 20;
        if (!SIGNED)
            c[i] = max(c[i], min(__float_as_uint(a), 1u));
    }
    uint32_t w = (c[0] | c[1] << 8) | (c[2] << 16 | c[3] << 24);
    if (SIGNED) {
        // the top bytes of the four numbers, their signs where the code is not zero
        const uint32_t top = __byte_perm(__byte_perm(__float_as_uint(q[0]), __float_as_uint(q[1]), 0x0073),
                                         __byte_perm(__float_as_uint(q[2]), __float_as_uint(q[3]), 0x0073), 0x5410);
        w |= top & (w + 0x7f7f7f7fu) & 0x80808080u;
    }
    return w;
}

// the same where some number is not finite: that one gets the type's NaN
template <bool SIGNED>
__device__ __noinline__ uint32_t stochastic_e4m3x4_checked(float4 q, uint4 noise)
{
    float v[4] = {q.x, q.y, q.z, q.w};
    const uint32_t n[4] = {noise.x, noise.y, noise.z, noise.w};
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((__float_as_uint(v[i]) & 0x7f800000u) == 0x7f800000u) {
            bad |= 0xffu << (8 * i);
            v[i] = 0.f;
        }
    return (stochastic_e4m3x4<SIGNED>(v, n) & ~bad) | (bad & 0x7f7f7f7fu);
}

// the largest of N numbers' finite magnitudes, as bits
template <int N>
__device__ __noinline__ uint32_t largest_finite(const float (&x)[N])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
        m = max(m, a < 0x7f800000u ? a : 0u);
    }
    return m;
}

// 1 / d of a normal number (or infinity of zero), to a unit in the last place
__device__ __forceinline__ float reciprocal(float d)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
    return r;
}

template <typename GT, bool E4, int CAP>
__global__ void __launch_bounds__(ADAMW_THREADS, E4 ? 3 : 4) adamw_kernel(const __grid_constant__ AdamwList<CAP> L, const AdamwScalars s, int bf16)
{
    constexpr int P = Piece<GT, E4>::P;    // elements of a thread at a time
    constexpr bool AHEAD = E4;             // the next run is fetched in front of this one's arithmetic (73.7 M elements 272 -> 255 us; FP32 moments: no gain)
    __shared__ float shared_rate, shared_root, shared_decay, shared_factor;
    __shared__ uint32_t shared_t;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        const long long t = *reinterpret_cast<volatile long long*>(s.step) + 1;
        const double f = s.factors ? (double)s.factors[0] : 1.0;
        const double lr = s.lr * f;
        shared_rate = (float)(lr / -expm1((double)t * s.ln_beta1));
        shared_root = (float)(1.0 / sqrt(-expm1((double)t * s.ln_beta2)));
        shared_decay = (float)(1.0 - lr * s.weight_decay);
        shared_factor = s.factors ? s.factors[1] : 1.f;
        shared_t = (uint32_t)t;
        if (s.last) {
            __threadfence();
            if (atomicAdd(reinterpret_cast<unsigned long long*>(s.step) + 1, 1ull) == gridDim.x - 1) {
                s.step[0] = t;             // every block has read the count
                s.step[1] = 0;
            }
        }
    }
    __syncthreads();
    const float rate = shared_rate, root = shared_root, decay = shared_decay, factor = shared_factor;
    const bool scaled = s.factors != nullptr;
    // (neighbouring runs at the same time: a block that took a stretch of its own was 13 % slower)
    const uint32_t runs = L.first_run[L.count];
    Piece<GT, E4> next;
    if (blockIdx.x < runs)
        next.load(L, blockIdx.x);
    for (uint32_t at = blockIdx.x; at < runs; at += gridDim.x) {
        const Piece<GT, E4> now = next;
        if (AHEAD && at + gridDim.x < runs)
            next.load(L, at + gridDim.x);
        const fpq_adamw_tensor& T = L.t[now.tensor];
        const int64_t e = now.e;
        const int left = now.left;
        float m[P], v[P], r[P], p[P];
        bool odd_root = false;
#pragma unroll
        for (int i = 0; i < P; i += 2) {
            float2 m2, v2, g2 = make_float2(value_at<GT>(now.g, i), value_at<GT>(now.g, i + 1));
            if constexpr (E4) {
                // a scale byte b stands for 2^(b - 127)
                const uint32_t mb = now.m_scale, rb = now.v_scale;
                m2 = mul2(values_e4m3x2(now.m[i / 4] >> (8 * (i % 4)) & 0xffffu), both2(__uint_as_float(mb ? mb << 23 : 0x00400000u)));
                v2 = mul2(values_e4m3x2(now.v[i / 4] >> (8 * (i % 4)) & 0xffffu), both2(__uint_as_float(rb ? rb << 23 : 0x00400000u)));
                v2 = mul2(v2, v2);
            } else {
                m2 = make_float2(__uint_as_float(now.m[i]), __uint_as_float(now.m[i + 1]));
                v2 = make_float2(__uint_as_float(now.v[i]), __uint_as_float(now.v[i + 1]));
            }
            if (scaled)
                g2 = mul2(g2, both2(factor));
            // (each product and sum rounded on its own: 8-bit codes are then a function of the formula, not of a compiler's choice)
            m2 = add2(mul2(m2, both2(s.beta1)), mul2(g2, both2(s.rest1)));
            v2 = add2(mul2(v2, both2(s.beta2)), mul2(mul2(g2, g2), both2(s.rest2)));
            const float2 r2 = roots_of(v2);
            m[i] = m2.x; m[i + 1] = m2.y;
            v[i] = v2.x; v[i + 1] = v2.y;
            r[i] = r2.x; r[i + 1] = r2.y;
            odd_root |= (v2.x < 1.2621774e-29f && v2.x > 0.f) || (v2.y < 1.2621774e-29f && v2.y > 0.f) || !(v2.x + v2.y < INFINITY);
        }
        if (odd_root)                      // (2^-96, and what is not finite)
#pragma unroll
            for (int i = 0; i < P; ++i)
                r[i] = __fsqrt_rn(v[i]);
#pragma unroll
        for (int i = 0; i < P; i += 2) {
            float2 d = fma2(make_float2(r[i], r[i + 1]), both2(root), both2(s.eps));
            d = make_float2(reciprocal(d.x), reciprocal(d.y));
            d = mul2(mul2(make_float2(m[i], m[i + 1]), d), both2(-rate));
            d = fma2(make_float2(__uint_as_float(now.p[i]), __uint_as_float(now.p[i + 1])), both2(decay), d);
            p[i] = d.x;
            p[i + 1] = d.y;
        }
        uint32_t mc[P / 4], rc[P / 4];
        if constexpr (E4) {
            // the exponents of both largest magnitudes of the block, 4 threads of eight elements each
            uint32_t a = 0, b = 0;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                a = max(a, __float_as_uint(m[i]) << 1);
                b = max(b, __float_as_uint(r[i]));
            }
            const bool odd = a >= 0xff000000u || b >= 0x7f800000u;     // infinities and NaN do not count
            if (odd) {
                a = largest_finite<P>(m) << 1;
                b = largest_finite<P>(r);
            }
            uint32_t both = (a >> 24) << 16 | b >> 23;
            both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 1));
            both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, 2));
            const uint32_t mb = max((int)(both >> 16) - 7, 1), rb = max((int)(both & 0xffffu) - 7, 1);
            const float mi = __uint_as_float((254u - mb) << 23), ri = __uint_as_float((254u - rb) << 23);
            const uint64_t number = L.first_block[now.tensor] * 32u + (uint64_t)e;
            const uint32_t key = mix(shared_t * 0x9E3779B1u + s.seed + 1u + (uint32_t)(number >> 32) * 0x243F6A89u);
#pragma unroll
            for (int k = 0; k < P / 4; ++k) {
                float qm[4], qr[4];
                uint32_t nm[4], nr[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t z = mix((uint32_t)(number + 4 * k + i) ^ key);
                    nm[i] = z >> 12 & 0xffff0u;
                    nr[i] = z << 4 & 0xffff0u;
                }
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const float2 a2 = mul2(make_float2(m[4 * k + i], m[4 * k + i + 1]), both2(mi));
                    const float2 b2 = mul2(make_float2(r[4 * k + i], r[4 * k + i + 1]), both2(ri));
                    qm[i] = a2.x; qm[i + 1] = a2.y;
                    qr[i] = b2.x; qr[i + 1] = b2.y;
                }
                if (!odd) {
                    mc[k] = stochastic_e4m3x4<true>(qm, nm);
                    rc[k] = stochastic_e4m3x4<false>(qr, nr);
                } else {
                    mc[k] = stochastic_e4m3x4_checked<true>(make_float4(qm[0], qm[1], qm[2], qm[3]), make_uint4(nm[0], nm[1], nm[2], nm[3]));
                    rc[k] = stochastic_e4m3x4_checked<false>(make_float4(qr[0], qr[1], qr[2], qr[3]), make_uint4(nr[0], nr[1], nr[2], nr[3]));
                }
            }
            if (left && (e & 31) == 0) {
                T.m_scale[e >> 5] = (uint8_t)mb;
                T.v_scale[e >> 5] = (uint8_t)rb;
            }
        }
        if (now.fast) {
#pragma unroll
            for (int i = 0; i < P; i += 4)
                *reinterpret_cast<float4*>(T.p + e + i) = make_float4(p[i], p[i + 1], p[i + 2], p[i + 3]);
            if constexpr (E4) {
                *reinterpret_cast<uint2*>((uint8_t*)T.m + e) = make_uint2(mc[0], mc[1]);
                *reinterpret_cast<uint2*>((uint8_t*)T.v + e) = make_uint2(rc[0], rc[1]);
            } else {
                *reinterpret_cast<float4*>((float*)T.m + e) = make_float4(m[0], m[1], m[2], m[3]);
                *reinterpret_cast<float4*>((float*)T.v + e) = make_float4(v[0], v[1], v[2], v[3]);
            }
            if (T.copy)
#pragma unroll
                for (int i = 0; i < P; i += 4)
                    *reinterpret_cast<uint2*>((uint16_t*)T.copy + e + i) = make_uint2(pack_two(p[i], p[i + 1], bf16), pack_two(p[i + 2], p[i + 3], bf16));
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i)
                if (i < left) {
                    T.p[e + i] = p[i];
                    if (E4) {
                        ((uint8_t*)T.m)[e + i] = (uint8_t)(mc[i / 4] >> (8 * (i % 4)));
                        ((uint8_t*)T.v)[e + i] = (uint8_t)(rc[i / 4] >> (8 * (i % 4)));
                    } else {
                        ((float*)T.m)[e + i] = m[i];
                        ((float*)T.v)[e + i] = v[i];
                    }
                    if (T.copy)
                        ((uint16_t*)T.copy)[e + i] = (uint16_t)pack_two(p[i], 0.f, bf16);
                }
        }
        if (!AHEAD && at + gridDim.x < runs)
            next.load(L, at + gridDim.x);
    }
}

template <int CAP>
cudaError_t launch_list(const AdamwList<CAP>& L, const AdamwScalars& s, int g_type, int bf16, int e4, cudaStream_t st)
{
    // as many blocks as an SM holds, which go from run to run
    uint32_t most = 148 * (e4 ? 3 : 4);
    const dim3 grid(std::min(std::max(L.first_run[L.count], 1u), most));
    // (as launch_overlapped, but the list is not copied on its way)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(ADAMW_THREADS);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    void* args[] = {(void*)&L, (void*)&s, &bf16};
#define FPQ_ADAMW(GT) cudaLaunchKernelExC(&cfg, e4 ? (const void*)adamw_kernel<GT, true, CAP> : (const void*)adamw_kernel<GT, false, CAP>, args)
    return g_type == FPQ_FP32 ? FPQ_ADAMW(float) : g_type == FPQ_BF16 ? FPQ_ADAMW(__nv_bfloat16) : FPQ_ADAMW(__half);
#undef FPQ_ADAMW
}

bool vectors(const fpq_adamw_tensor& t, int g_type, int e4)
{
    const uintptr_t g = g_type == FPQ_FP32 || e4 ? 16 : 8, state = e4 ? 8 : 16;
    return (uintptr_t)t.p % 16 == 0 && (uintptr_t)t.g % g == 0 && (uintptr_t)t.m % state == 0 && (uintptr_t)t.v % state == 0 &&
           (uintptr_t)t.copy % 8 == 0;
}

template <int CAP>
fpq_status launch_all(const fpq_adamw_tensor* t, int count, AdamwScalars s, int g_type, int bf16, int e4, cudaStream_t st)
{
    const int64_t run = ADAMW_THREADS * (e4 ? 8 : 4);
    uint64_t block = 0;
    int at = 0;
    do {
        AdamwList<CAP> L;
        uint32_t runs = 0;
        int k = 0;
        for (; at < count && k < CAP; ++at) {
            if (t[at].n == 0)
                continue;
            const int64_t more = (t[at].n + run - 1) / run;
            if (runs + more > 0x7fffffff && k > 0)
                break;
            L.t[k] = t[at];
            L.first_run[k] = runs;
            L.first_block[k] = block;
            L.vec[k] = vectors(t[at], g_type, e4) ? 1 : 0;
            runs += (uint32_t)more;
            block += (uint64_t)((t[at].n + 31) / 32);
            ++k;
        }
        L.first_run[k] = runs;
        L.count = k;
        s.last = at == count;
        if (launch_list(L, s, g_type, bf16, e4, st) != cudaSuccess)
            return FPQ_ERR_CUDA;
    } while (at < count);
    return FPQ_OK;
}

}  // namespace

fpq_status launch_adamw(const fpq_adamw_tensor* t, int count, int g_type, int copy_type, int state_type, const fpq_adamw_options& o,
                        const float* factors, int64_t* step, cudaStream_t st)
{
    AdamwScalars s;
    s.ln_beta1 = log(o.beta1);
    s.ln_beta2 = log(o.beta2);
    s.lr = o.lr;
    s.weight_decay = o.weight_decay;
    s.beta1 = (float)o.beta1;
    s.rest1 = (float)(1.0 - o.beta1);
    s.beta2 = (float)o.beta2;
    s.rest2 = (float)(1.0 - o.beta2);
    s.eps = (float)o.eps;
    s.seed = o.seed;
    s.factors = factors;
    s.step = (long long*)step;
    s.last = 0;
    const int bf16 = copy_type == FPQ_BF16, e4 = state_type == FPQ_E4M3_BLOCK32;
    return count <= ADAMW_SMALL ? launch_all<ADAMW_SMALL>(t, count, s, g_type, bf16, e4, st)
                                : launch_all<ADAMW_LAUNCH>(t, count, s, g_type, bf16, e4, st);
}

}  // namespace fpq
