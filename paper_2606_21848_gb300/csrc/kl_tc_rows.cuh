// What the kernels with one query row per thread share (prefill, tree attention: thread = row of the
// block = TMEM lane): bounded waits, operand packing, packed fp32 arithmetic, shared-memory vectors.
#pragma once

#include "kl_internal.cuh"
#include "kl_tc_ptx.cuh"

namespace kl {
namespace {

constexpr uint64_t kRowsTimeoutNs = 1000000000ull;   // bound of every wait (about one second)

// Bounded wait. Warp-collective (every lane calls it in uniform control flow and gets the same
// answer), or by one lane alone (one(): the MMA issuers, whose successful waits must cost little).
// False when the CTA is aborting or the wait ran out (`limit` ns; kExact, for short limits, polls without
// suspending the thread, as in kl_decode_tc_kernel.cuh).
template <bool kExact = false>
struct Waiter {
    volatile int *abort;
    int32_t *err;
    uint64_t limit = kRowsTimeoutNs;
    __device__ bool poll(uint64_t *bar, uint32_t parity) const {
        return kExact ? ptx::mbar_test_wait(bar, parity) : ptx::mbar_try_wait(bar, parity);
    }
    __device__ bool slow(uint64_t *bar, uint32_t parity) const {
        const uint64_t t0 = ptx::globaltimer();
        while (true) {
            if (poll(bar, parity)) return true;
            if (*abort) return false;
            if (ptx::globaltimer() - t0 > limit) {
                *abort = 1;
                raise_flag(err, KL_FLAG_TIMEOUT);
                return false;
            }
        }
    }
    __device__ bool one(uint64_t *bar, uint32_t parity) const {
        return poll(bar, parity) || slow(bar, parity);
    }
    __device__ bool operator()(uint64_t *bar, uint32_t parity) const {
        return __all_sync(0xffffffffu, one(bar, parity));
    }
};

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// x = hi + lo with hi = bf16(x), lo = bf16(x - hi), for two values packed as bf16 pairs.
__device__ __forceinline__ void split2(float x0, float x1, uint32_t &hi, uint32_t &lo) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x0, x1);
    const float2 hf = __bfloat1622float2(h);
    const __nv_bfloat162 l = __floats2bfloat162_rn(x0 - hf.x, x1 - hf.y);
    hi = *reinterpret_cast<const uint32_t *>(&h);
    lo = *reinterpret_cast<const uint32_t *>(&l);
}

// The leading bf16 term of two fp32 values, packed; the values become what is left.
__device__ __forceinline__ uint32_t take_term(uint32_t &x0, uint32_t &x1) {
    const float a = __uint_as_float(x0), b = __uint_as_float(x1);
    const uint32_t t = pack2(a, b);
    x0 = __float_as_uint(a - bf16lo(t));
    x1 = __float_as_uint(b - bf16hi(t));
    return t;
}

// Whether one of two packed bf16 values is infinite or NaN.
__device__ __forceinline__ bool not_finite(uint32_t v) {
    return (v & 0x7f80u) == 0x7f80u || (v & 0x7f800000u) == 0x7f800000u;
}

// Whether one of two packed bf16 values has no finite fp16 form (a magnitude of 65536 or more).
__device__ __forceinline__ bool past_fp16(uint32_t v) {
    return (v & 0x7fffu) >= 0x4780u || (v & 0x7fff0000u) >= 0x47800000u;
}

// Instruction descriptor of kind::f16 with fp16 A and B (A and B formats 0), fp32 accumulator,
// operand majorness (0 = K-major, 1 = MN-major), N and M.
__host__ __device__ constexpr uint32_t idesc_f16(uint32_t M, uint32_t N, bool a_mn, bool b_mn) {
    return (1u << 4) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((N >> 3) << 17) |
           ((M >> 4) << 24);
}

// max(a, b, c): the three-operand PTX max.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Packed fp32 pair arithmetic (one instruction for two lanes of data).
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\t"
        "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "add.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 sub2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\t"
        "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
        "sub.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float f) {
    return make_float2(a.x * f, a.y * f);
}

// Two values as an fp16 pair (a in the low half), round to nearest even.
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(b), "f"(a));
    return d;
}

// The leading fp16 term of two fp32 values, packed; the values become what is left.
__device__ __forceinline__ uint32_t take_term_f16(uint32_t &x0, uint32_t &x1) {
    const float a = __uint_as_float(x0), b = __uint_as_float(x1);
    const uint32_t t = pack_f16(a, b);
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&t));
    x0 = __float_as_uint(a - f.x);
    x1 = __float_as_uint(b - f.y);
    return t;
}

__device__ __forceinline__ void ld_shared_v4(uint32_t addr, uint32_t *v) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(addr)
                 : "memory");
}

__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c,
                                             uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c),
                 "r"(d)
                 : "memory");
}

}  // namespace
}  // namespace kl
