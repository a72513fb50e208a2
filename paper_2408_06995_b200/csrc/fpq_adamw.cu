// One AdamW step over many tensors (decoupled weight decay), moments in FP32 or in 8 bits.
//
//   m' = b1 m + (1 - b1) g,   v' = b2 v + (1 - b2) g^2,
//   p' = p (1 - lr wd) - lr / (1 - b1^t) * m' / (sqrt(v') / sqrt(1 - b2^t) + eps)
//
// Nothing is used twice, so the step is bound by memory: per element 8 bytes of p, the gradient, and 16 bytes of FP32
// moments or 4.125 of 8-bit ones.  One kernel goes once over all tensors: a block takes a run of one tensor's elements,
// found in the list of runs that travels in the kernel's arguments, and every thread has U groups of four elements in
// flight.  The blocks work the bias corrections out themselves from the step count on the device, so a captured launch
// can be replayed; the last block to have read the count moves it on.
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
#include <string.h>

#include "fpq_kernels.h"

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

template <typename T>
__device__ __forceinline__ float load_one(const T* p);
template <>
__device__ __forceinline__ float load_one<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float load_one<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }
template <>
__device__ __forceinline__ float load_one<__half>(const __half* p) { return __half2float(*p); }

__device__ __forceinline__ void load_four(const float* p, float* v)
{
    const float4 q = *reinterpret_cast<const float4*>(p);
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
}
__device__ __forceinline__ void load_four(const __nv_bfloat16* p, float* v)
{
    const uint2 q = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(q.x << 16); v[1] = __uint_as_float(q.x & 0xffff0000u);
    v[2] = __uint_as_float(q.y << 16); v[3] = __uint_as_float(q.y & 0xffff0000u);
}
__device__ __forceinline__ void load_four(const __half* p, float* v)
{
    const uint2 q = *reinterpret_cast<const uint2*>(p);
    __half2 a, b;
    memcpy(&a, &q.x, 4);
    memcpy(&b, &q.y, 4);
    const float2 x = __half22float2(a), y = __half22float2(b);
    v[0] = x.x; v[1] = x.y; v[2] = y.x; v[3] = y.y;
}

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

// magnitude bits that count towards a block's scale: infinities and NaN do not
__device__ __forceinline__ uint32_t finite_bits(float x)
{
    const uint32_t a = __float_as_uint(x) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}

// E4M3 code of q, |q| < 256, rounded up if the remainder below the code's step plus `noise` (16 bits) carries.  Below 2^-6 the
// steps are equal: with 2^-6 added they are the steps of that binade.  What is not finite gets the type's NaN.
__device__ __forceinline__ uint32_t stochastic_e4m3(float q, uint32_t noise, uint32_t least)
{
    const float a = fabsf(q);
    const bool low = a < 0.015625f;
    const uint32_t word = __float_as_uint(low ? __fadd_rn(a, 0.015625f) : a) + (noise << 4);
    uint32_t code = (word >> 20) - (low ? 968u : 960u);
    if (a > 0.f && code < least)
        code = least;
    if (code)
        code |= (__float_as_uint(q) >> 24) & 0x80u;
    return a < 512.f ? code : 0x7fu;
}

// Four elements of one tensor from `e` on; g .. hold them, those from n on as zeros.
template <typename GT, bool E4, int CAP>
__global__ void __launch_bounds__(ADAMW_THREADS) adamw_kernel(const __grid_constant__ AdamwList<CAP> L, const AdamwScalars s, int U, int bf16)
{
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
    // the tensor of this run: the last one whose first run is not behind it
    int lo = 0, hi = L.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (L.first_run[mid] <= blockIdx.x)
            lo = mid;
        else
            hi = mid;
    }
    __syncthreads();
    const float rate = shared_rate, root = shared_root, decay = shared_decay, factor = shared_factor;
    if (blockIdx.x >= L.first_run[L.count])
        return;
    const fpq_adamw_tensor& T = L.t[lo];
    const int64_t n = T.n, run = (int64_t)(blockIdx.x - L.first_run[lo]) * (U * ADAMW_THREADS * 4);
    const bool vec = L.vec[lo] != 0;
    const uint64_t number0 = L.first_block[lo] * 32u;

    for (int u = 0; u < U; ++u) {
        const int64_t e = run + (int64_t)(u * ADAMW_THREADS + threadIdx.x) * 4;
        const int left = e >= n ? 0 : n - e < 4 ? (int)(n - e) : 4;
        float p[4] = {}, g[4] = {}, m[4] = {}, v[4] = {};
        uint32_t mc = 0, rc = 0;
        const GT* gp = (const GT*)T.g + e;
        if (left == 4 && vec) {
            load_four(T.p + e, p);
            load_four(gp, g);
            if (E4) {
                mc = *reinterpret_cast<const uint32_t*>((const uint8_t*)T.m + e);
                rc = *reinterpret_cast<const uint32_t*>((const uint8_t*)T.v + e);
            } else {
                load_four((const float*)T.m + e, m);
                load_four((const float*)T.v + e, v);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < left) {
                    p[i] = T.p[e + i];
                    g[i] = load_one(gp + i);
                    if (E4) {
                        mc |= (uint32_t)((const uint8_t*)T.m)[e + i] << (8 * i);
                        rc |= (uint32_t)((const uint8_t*)T.v)[e + i] << (8 * i);
                    } else {
                        m[i] = ((const float*)T.m)[e + i];
                        v[i] = ((const float*)T.v)[e + i];
                    }
                }
        }
        if (E4 && left) {
            // a scale byte b stands for 2^(b - 127)
            const uint32_t mb = T.m_scale[e >> 5], rb = T.v_scale[e >> 5];
            const float ms = __uint_as_float(mb ? mb << 23 : 0x00400000u), rs = __uint_as_float(rb ? rb << 23 : 0x00400000u);
            const float2 m0 = values_e4m3x2(mc & 0xffffu), m1 = values_e4m3x2(mc >> 16);
            const float2 r0 = values_e4m3x2(rc & 0xffffu), r1 = values_e4m3x2(rc >> 16);
            m[0] = m0.x * ms; m[1] = m0.y * ms; m[2] = m1.x * ms; m[3] = m1.y * ms;
            v[0] = r0.x * rs; v[1] = r0.y * rs; v[2] = r1.x * rs; v[3] = r1.y * rs;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = __fmul_rn(v[i], v[i]);
        }
        // (each product and sum rounded on its own: 8-bit codes are then a function of the formula, not of a compiler's choice)
        float r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float gi = s.factors ? __fmul_rn(g[i], factor) : g[i];
            m[i] = __fadd_rn(__fmul_rn(m[i], s.beta1), __fmul_rn(gi, s.rest1));
            v[i] = __fadd_rn(__fmul_rn(v[i], s.beta2), __fmul_rn(__fmul_rn(gi, gi), s.rest2));
            r[i] = __fsqrt_rn(v[i]);
            p[i] = __fsub_rn(__fmul_rn(p[i], decay), __fmul_rn(__fdividef(m[i], __fadd_rn(__fmul_rn(r[i], root), s.eps)), rate));
        }
        if (E4) {
            // the exponents of both largest magnitudes of the block, 8 threads of four elements each
            uint32_t a = max(max(finite_bits(m[0]), finite_bits(m[1])), max(finite_bits(m[2]), finite_bits(m[3]))) >> 23;
            uint32_t b = max(max(finite_bits(r[0]), finite_bits(r[1])), max(finite_bits(r[2]), finite_bits(r[3]))) >> 23;
            uint32_t both = left ? a << 16 | b : 0u;
#pragma unroll
            for (int o = 1; o < 8; o <<= 1)
                both = __vmaxu2(both, __shfl_xor_sync(0xffffffffu, both, o));
            const uint32_t mb = max((int)(both >> 16) - 7, 1), rb = max((int)(both & 0xffffu) - 7, 1);
            const float mi = __uint_as_float((254u - mb) << 23), ri = __uint_as_float((254u - rb) << 23);
            const uint64_t number = number0 + (uint64_t)e;
            const uint32_t key = mix(shared_t * 0x9E3779B1u + s.seed + 1u + (uint32_t)(number >> 32) * 0x243F6A89u);
            mc = rc = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t z = mix((uint32_t)(number + i) ^ key);
                mc |= stochastic_e4m3(m[i] * mi, z >> 16, 0u) << (8 * i);
                rc |= stochastic_e4m3(r[i] * ri, z & 0xffffu, 1u) << (8 * i);
            }
            if (left && (e & 31) == 0) {
                T.m_scale[e >> 5] = (uint8_t)mb;
                T.v_scale[e >> 5] = (uint8_t)rb;
            }
        }
        if (left == 4 && vec) {
            *reinterpret_cast<float4*>(T.p + e) = make_float4(p[0], p[1], p[2], p[3]);
            if (E4) {
                *reinterpret_cast<uint32_t*>((uint8_t*)T.m + e) = mc;
                *reinterpret_cast<uint32_t*>((uint8_t*)T.v + e) = rc;
            } else {
                *reinterpret_cast<float4*>((float*)T.m + e) = make_float4(m[0], m[1], m[2], m[3]);
                *reinterpret_cast<float4*>((float*)T.v + e) = make_float4(v[0], v[1], v[2], v[3]);
            }
            if (T.copy)
                *reinterpret_cast<uint2*>((uint16_t*)T.copy + e) = make_uint2(pack_two(p[0], p[1], bf16), pack_two(p[2], p[3], bf16));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < left) {
                    T.p[e + i] = p[i];
                    if (E4) {
                        ((uint8_t*)T.m)[e + i] = (uint8_t)(mc >> (8 * i));
                        ((uint8_t*)T.v)[e + i] = (uint8_t)(rc >> (8 * i));
                    } else {
                        ((float*)T.m)[e + i] = m[i];
                        ((float*)T.v)[e + i] = v[i];
                    }
                    if (T.copy)
                        ((uint16_t*)T.copy)[e + i] = (uint16_t)pack_two(p[i], 0.f, bf16);
                }
        }
    }
}

template <int CAP>
cudaError_t launch_list(const AdamwList<CAP>& L, const AdamwScalars& s, int g_type, int bf16, int e4, int U, cudaStream_t st)
{
    const dim3 grid(L.first_run[L.count] ? L.first_run[L.count] : 1);
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
    void* args[] = {(void*)&L, (void*)&s, &U, &bf16};
#define FPQ_ADAMW(GT) cudaLaunchKernelExC(&cfg, e4 ? (const void*)adamw_kernel<GT, true, CAP> : (const void*)adamw_kernel<GT, false, CAP>, args)
    return g_type == FPQ_FP32 ? FPQ_ADAMW(float) : g_type == FPQ_BF16 ? FPQ_ADAMW(__nv_bfloat16) : FPQ_ADAMW(__half);
#undef FPQ_ADAMW
}

bool vectors(const fpq_adamw_tensor& t, int g_type, int e4)
{
    const uintptr_t g = g_type == FPQ_FP32 ? 16 : 8, state = e4 ? 4 : 16;
    return (uintptr_t)t.p % 16 == 0 && (uintptr_t)t.g % g == 0 && (uintptr_t)t.m % state == 0 && (uintptr_t)t.v % state == 0 &&
           (uintptr_t)t.copy % 8 == 0;
}

template <int CAP>
fpq_status launch_all(const fpq_adamw_tensor* t, int count, AdamwScalars s, int g_type, int bf16, int e4, int U, cudaStream_t st)
{
    const int64_t run = (int64_t)U * ADAMW_THREADS * 4;
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
            if (runs + more > 0x7fffffff)
                break;                     // (never the first of a launch: n < 2^40)
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
        if (launch_list(L, s, g_type, bf16, e4, U, st) != cudaSuccess)
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
    int64_t total = 0;
    for (int i = 0; i < count; ++i)
        total += t[i].n;
    // runs of 1024 elements spread small calls over the SMs, runs of 4096 spend less on finding their tensor
    const int U = total >= (int64_t)148 * 8 * 4096 ? 4 : 1;
    const int bf16 = copy_type == FPQ_BF16, e4 = state_type == FPQ_E4M3_BLOCK32;
    return count <= ADAMW_SMALL ? launch_all<ADAMW_SMALL>(t, count, s, g_type, bf16, e4, U, st)
                                : launch_all<ADAMW_LAUNCH>(t, count, s, g_type, bf16, e4, U, st);
}

}  // namespace fpq
