// Pieces that the operators on cached context (kdn_attend.cu, kdn_weigh.cu, kdn_evict.cu) share: launches, the way a call's
// records reach the device, and small PTX wrappers.
#pragma once
#include "kdn.h"
#include "kdn_context.h"

#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <atomic>
#include <cmath>
#include <cstring>

#define KDN_CUDA(call)                                                                  \
    do {                                                                                \
        cudaError_t e_ = (call);                                                        \
        if (e_ != cudaSuccess) return e_ == cudaErrorMemoryAllocation ? KDN_E_NOMEM : KDN_E_CUDA; \
    } while (0)

namespace kdn {

// ------------------------------------------------------------------------------------------ host --

// A launch that may be set up while the kernel before it in the stream drains: every kernel of these files waits for that
// kernel (dependency_wait) before it touches global memory, and reads it by plain loads: what a kernel before it writes is not
// read-only while it runs.
template <typename... Args>
kdn_status launch(const Context &c, void (*kernel)(Args...), dim3 grid, unsigned threads, size_t smem, cudaStream_t stream, Args... args)
{
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    KDN_CUDA(cudaLaunchKernelEx(&cfg, kernel, args...));
    ++*c.launches;
    return KDN_OK;
}

// The kernel's shared-memory limit on the context's device, raised the first time (the value is a constant of the kernel, so it does not matter who
// was first; two threads may both be).
template <auto kernel> kdn_status allow_smem(const Context &c, size_t bytes)
{
    static std::atomic<unsigned long long> done{ 0 };
    const unsigned long long bit = c.device < 64 ? 1ull << c.device : 0ull;
    if (done.load(std::memory_order_relaxed) & bit) return KDN_OK;
    KDN_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    done.fetch_or(bit, std::memory_order_relaxed);
    return KDN_OK;
}

constexpr double kLog2e = 1.4426950408889634;
// Whether the kernels' scores, in powers of two, can be had from a scale: fp32 holds what they are multiplied by.
inline bool usable_scale(double scale) { return (float)(scale * kLog2e) > 0.0f && std::isfinite((float)(scale * kLog2e)); }

// Tokens of one request or chunk at most: what the kernels add to a token's index stays within 31 bits.
constexpr int64_t kMostTokens = (int64_t)1 << 28;

constexpr size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool aligned(const void *p, size_t a) { return (uintptr_t)p % a == 0; }

// ---------------------------------------------------------------------------------------- device --

__device__ __forceinline__ void dependency_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void release_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

constexpr int kStatusRange = 4, kStatusTimeout = 8;          // KDN_E_RANGE, KDN_E_TIMEOUT

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// the same, but the hardware may hold the thread for a while first
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long global_timer_ns()
{
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// Bounded wait: true when the phase completed; false when the CTA is giving up or the limit passed.
static __device__ __noinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity, volatile int *abort_flag, unsigned long long limit_ns)
{
    const unsigned long long t0 = global_timer_ns();
#pragma unroll 1
    for (int i = 0; i < 2; ++i)
        if (mbar_test(bar, parity)) return true;
    for (;;) {
        if (*abort_flag) return false;
        if (global_timer_ns() - t0 > limit_ns) { *abort_flag = 1; return false; }
        if (mbar_try_wait(bar, parity)) return true;
    }
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, unsigned long long limit_ns)
{
    if (mbar_test(bar, parity)) return true;
    return mbar_wait_slow(bar, parity, abort_flag, limit_ns);
}
// The same for all lanes of a warp, which go on or give up together.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, unsigned long long limit_ns)
{
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, limit_ns));
}
template <int N> __device__ __forceinline__ void copy_async(uint32_t dst, const void *src)
{
    if (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(N) : "memory");
}
__device__ __forceinline__ void copies_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

__device__ __forceinline__ float exp2_approx(float x)       // 2 ulp, flushes results below 2^-126 to zero
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Kernels that take 2^(x * scale - m) in one multiply-add have rounded m (the largest x * scale) before: what that left is an exponent which all weights of the row
// share, 2 at most with scores up to this (in powers of two).  Beyond, it would be a weight of infinity or none at all for the row's largest score, and x * scale is rounded first.
constexpr float kHugeScore = 67108864.0f;                  // 2^26
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
// Two fp32 values in one 64-bit register for the packed instructions of sm_100.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float lo, float hi)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpack2(f32x2 v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b)
{
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ float max_or_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ float min_or_nan(float a, float b)
{
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// Half of 2^x of two numbers on the pipe of multiplications, for kernels that the special-function unit (16 results a clock and SM) holds up: 2^(n - 1) 2^f with n the
// nearest whole number and 2^f by the polynomial of degree five through its values at the Chebyshev nodes of [-1/2, 1/2], off by 2.2e-7 relative at most in
// fp32 (2^-22; worked out for these coefficients).  Halves, so that every result that fp32 holds is made without overflow; whoever adds them up doubles
// them in the same step, which gives infinity from x = 128 on.  Below x = -125.5 the result is zero; a NaN stays one.
__device__ __forceinline__ f32x2 half_exp2_pair(f32x2 x)
{
    float a, b;
    unpack2(x, a, b);
    x = pack2(min_or_nan(max_or_nan(a, -126.0f), 128.0f), min_or_nan(max_or_nan(b, -126.0f), 128.0f));
    const f32x2 whole = add2(x, pack2(12582912.0f, 12582912.0f));              // 1.5 * 2^23: n in the low bits
    const f32x2 f = fma2(add2(whole, pack2(-12582912.0f, -12582912.0f)), pack2(-1.0f, -1.0f), x);
    f32x2 y = pack2(0.0013390863314270973f, 0.0013390863314270973f);
    y = fma2(y, f, pack2(0.009676031768321991f, 0.009676031768321991f));
    y = fma2(y, f, pack2(0.055503569543361664f, 0.055503569543361664f));
    y = fma2(y, f, pack2(0.2402210682630539f, 0.2402210682630539f));
    y = fma2(y, f, pack2(0.6931471824645996f, 0.6931471824645996f));
    y = fma2(y, f, pack2(1.0000001192092896f, 1.0000001192092896f));
    float n0, n1;
    unpack2(whole, n0, n1);
    return mul2(y, pack2(__uint_as_float((__float_as_uint(n0) << 23) + 0x3f000000u), __uint_as_float((__float_as_uint(n1) << 23) + 0x3f000000u)));
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// Two values as a pair of bf16 and the pair of what that rounding left: 16 bits of each.
__device__ __forceinline__ void split_bf16x2(float a, float b, uint32_t &hi, uint32_t &lo)
{
    hi = pack_bf16x2(a, b);
    lo = pack_bf16x2(a - bf16_lo(hi), b - bf16_hi(hi));
}
// d += a b: 16 x 16 times 16 x 8, bf16 in, fp32 sums
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16x8x16_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ void split_f16x2(float a, float b, uint32_t &hi, uint32_t &lo)      // 22 bits of each
{
    hi = pack_f16x2(a, b);
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
    lo = pack_f16x2(a - f.x, b - f.y);
}
// Four 8 x 8 matrices of 16-bit elements: row i of matrix k at the address that lane 8 k + i gives.  A lane gets elements 2c, 2c + 1 of row g of
// each, or with `transposed` element g of rows 2c, 2c + 1 (g = lane / 4, c = lane % 4).
template <bool transposed> __device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at)
{
    if (transposed)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// The records of a call travel as kernel parameters, so that nothing of the host is read later and a captured launch carries
// its own.  Calls of up to Most of them hand them to the kernel that uses them; larger calls write them to the workspace
// first, kPutBytes a launch.
constexpr int kPutBytes = 28 * 1024;
struct PutLaunch {
    uint4 *dst;
    int n;                                  // 16-byte words
    uint4 data[kPutBytes / 16];
};
static __global__ void __launch_bounds__(256) kdn_put_records_kernel(const __grid_constant__ PutLaunch p)
{
    release_dependents();
    dependency_wait();
    for (int i = (int)threadIdx.x; i < p.n; i += 256) p.dst[i] = p.data[i];
}

inline kdn_status put_records(const Context &c, void *dst, const void *src, size_t bytes, cudaStream_t stream)
{
    static thread_local PutLaunch p;        // 28 KiB: too much for a caller's stack
    for (size_t at = 0; at < bytes; at += kPutBytes) {
        const size_t n = bytes - at < (size_t)kPutBytes ? bytes - at : (size_t)kPutBytes;
        p.dst = reinterpret_cast<uint4 *>(static_cast<unsigned char *>(dst) + at);
        p.n = (int)((n + 15) / 16);
        std::memcpy(p.data, static_cast<const unsigned char *>(src) + at, n);
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(1);
        cfg.blockDim = dim3(256);
        cfg.stream = stream;
        cudaLaunchAttribute attr{};
        attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr.val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        KDN_CUDA(cudaLaunchKernelEx(&cfg, kdn_put_records_kernel, p));
        ++*c.launches;
    }
    return KDN_OK;
}

}  // namespace kdn
