// Shared by the operators around a quantised layer: element types, vector
// access at any alignment, reductions over a workgroup, argument checks.
#pragma once
#include <atomic>
#include <cmath>
#include <cstdio>
#include <type_traits>

#include "bakron.h"
#include "common.h"

namespace bk {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// N consecutive elements at an address of any alignment.  The compiler emits the
// widest global access for it: global memory takes any byte alignment here.
template <typename E, int N>
struct Pack {
    E v[N];
};
template <typename E, int N>
__device__ inline Pack<E, N> load_pack(const E* p) {
    Pack<E, N> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}
template <typename E, int N>
__device__ inline void store_pack(E* p, const Pack<E, N>& r) {
    __builtin_memcpy(p, &r, sizeof(r));
}

// N consecutive entries, `valid` of them inside the row.
template <typename E, int N>
__device__ inline void store_n(E* p, const float (&v)[N], int64_t valid) {
    if (valid >= N) {
        Pack<E, N> o;
#pragma unroll
        for (int j = 0; j < N; ++j) o.v[j] = (E)v[j];
        store_pack(p, o);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < valid) p[j] = (E)v[j];
    }
}
template <typename E, int N>
__device__ inline void load_n(const E* p, float (&v)[N], int64_t valid) {
    if (valid >= N) {
        const auto o = load_pack<E, N>(p);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = (float)o.v[j];
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = j < valid ? (float)p[j] : 0.0f;
    }
}

// A 16-byte vector of E as four registers: whole until an entry is asked for, so that
// neither a branch around a load nor a second use makes the compiler take it apart.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename E>
__device__ inline u32x4 load_words(const E* p) {
    u32x4 u;
    __builtin_memcpy(&u, p, 16);
    return u;
}
template <typename E>
__device__ inline float entry(const u32x4& u, int j) {
    if constexpr (sizeof(E) == 4) {
        return __uint_as_float(u[j]);
    } else if constexpr (std::is_same<E, bf16_t>::value) {
        return __uint_as_float(j & 1 ? u[j >> 1] & 0xffff0000u : u[j >> 1] << 16);
    } else {
        return (float)__builtin_bit_cast(f16_t, (uint16_t)(u[j >> 1] >> (16 * (j & 1))));
    }
}
// 16 bytes to an address of any even alignment, not kept in the caches.
typedef uint32_t u32x4_loose __attribute__((ext_vector_type(4), aligned(2)));
template <typename E>
__device__ inline void store_words_past(E* p, const u32x4& u) {
    __builtin_nontemporal_store(u, reinterpret_cast<u32x4_loose*>(p));
}
// -infinity in every entry.
template <typename E>
__device__ inline uint32_t minus_infinity() {
    return sizeof(E) == 4 ? 0xff800000u : std::is_same<E, bf16_t>::value ? 0xff80ff80u : 0xfc00fc00u;
}
// Makes the compiler forget what it knows of a vector, so that values derived from it
// (its entries in fp32, twice the registers) are not kept from one use to the next.
__device__ inline void forget(u32x4& u) {
    asm volatile("" : "+v"(u));
}

// max that keeps a NaN from either side (v_maximum3_f32).
__device__ inline float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

struct MaxNan {
    __device__ float operator()(float a, float b) const { return max_nan(a, b); }
};
struct MaxU32 {
    __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return a > b ? a : b; }
};
struct Add {
    __device__ float operator()(float a, float b) const { return a + b; }
};

// The value that a lane permutation inside rows of 16 lanes (a DPP control) brings.
template <int CTRL>
__device__ inline uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}
template <int CTRL>
__device__ inline float dpp(float v) {
    return __uint_as_float(dpp<CTRL>(__float_as_uint(v)));
}
constexpr int DPP_XOR1 = 0xb1, DPP_XOR2 = 0x4e, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;

// Over the 16 lanes of a row, every lane having the result: neighbours, then (all of a
// quad, of an eight being equal) mirrored.  One operation a step, no trip through LDS.
template <typename V, typename Op>
__device__ inline V row_reduce(V v, Op op) {
    v = op(v, dpp<DPP_XOR1>(v));
    v = op(v, dpp<DPP_XOR2>(v));
    v = op(v, dpp<DPP_HALF_MIRROR>(v));
    return op(v, dpp<DPP_MIRROR>(v));
}
__device__ inline float lane_value(float v, int lane) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane));
}
__device__ inline uint32_t lane_value(uint32_t v, int lane) {
    return (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
// Over the wave, in a fixed order.  All lanes have to be active.
template <typename V, typename Op>
__device__ inline V wave_reduce(V v, Op op) {
    v = row_reduce(v, op);
    return op(op(lane_value(v, 0), lane_value(v, 16)), op(lane_value(v, 32), lane_value(v, 48)));
}

// Over `waves` waves of a workgroup; `red` holds one float a wave and may be used
// again only after another barrier.
template <typename Op>
__device__ inline float group_reduce(float v, Op op, float* red, int wave, int lane, int waves) {
    v = wave_reduce(v, op);
    if (waves == 1) return v;
    if (lane == 0) red[wave] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < waves; ++w) v = op(v, red[w]);
    return v;
}

// exp(x), |x| <= 200, from the hardware's exp2 (1 ulp).  x log2 e in fp32 alone leaves a relative error of
// |x| 2^-24, which 16-bit results do not show; FINE: what the product lost and log2 e's next bits, too.
constexpr float LOG2E = 1.44269504088896340736f, LOG2E_REST = 1.925963033500e-8f, LN2 = 0.69314718055994530942f;
template <bool FINE>
__device__ inline float exp_of(float x) {
    const float t = x * LOG2E, e = __builtin_amdgcn_exp2f(t);
    if constexpr (!FINE) return e;
    return e * fmaf(fmaf(x, LOG2E_REST, fmaf(x, LOG2E, -t)), LN2, 1.0f);
}

inline bakron_status op_fail(const char* who, const char* what) {
    char buf[256];
    std::snprintf(buf, sizeof(buf), "%s: %s", who, what);
    set_last_error(buf);
    return BAKRON_EINVAL;
}

inline bakron_status op_launched(const char* who) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return BAKRON_OK;
    char buf[256];
    std::snprintf(buf, sizeof(buf), "%s: launch: %s", who, hipGetErrorString(e));
    set_last_error(buf);
    return e == hipErrorOutOfMemory ? BAKRON_ENOMEM : BAKRON_EHIP;
}

// The workspace protocol.  *query: only the size was asked for.
inline bakron_status op_workspace(const char* who, void* work, size_t* work_bytes, size_t need,
                                  bool* query) {
    *query = false;
    if (!work_bytes) return op_fail(who, "work_bytes is NULL");
    if (!work) {
        *work_bytes = need;
        *query = true;
        return BAKRON_OK;
    }
    if (need > 0 && *work_bytes < need) return op_fail(who, "workspace too small");
    if (need > 0 && ((uintptr_t)work & 255) != 0)
        return op_fail(who, "workspace not 256-byte aligned");
    return BAKRON_OK;
}

constexpr int64_t OP_T_MAX = ((int64_t)1 << 31) - 1;
// Threads of one launch (the runtime takes below 2^32).
constexpr int64_t OP_LAUNCH_MAX = (int64_t)1 << 31;

// The grid of a kernel that goes through n pieces, 256 threads a workgroup, in strides of the grid: any n,
// where one piece a thread would pass what a launch takes.
constexpr int64_t STRIDE_GROUPS = (int64_t)1 << 16;
inline dim3 stride_grid(int64_t n) {
    const int64_t groups = (n + 255) / 256;
    return dim3((unsigned)(groups < STRIDE_GROUPS ? groups : STRIDE_GROUPS));
}

// CUs of the current device (asked for once a device).
inline int op_cus() {
    static std::atomic<int> known[16];
    int dev = 0, ncu = 0;
    if (hipGetDevice(&dev) != hipSuccess) return 256;
    if (dev >= 0 && dev < 16 && (ncu = known[dev].load(std::memory_order_relaxed)) > 0) return ncu;
    if (hipDeviceGetAttribute(&ncu, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess)
        return 256;
    if (dev >= 0 && dev < 16) known[dev].store(ncu, std::memory_order_relaxed);
    return ncu;
}

}  // namespace bk
