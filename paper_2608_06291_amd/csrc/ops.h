// Shared by the operators around a quantised layer: element types, vector
// access at any alignment, reductions over a workgroup, argument checks.
#pragma once
#include <cmath>
#include <cstdio>

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

// max that keeps a NaN from either side (v_maximum3_f32).
__device__ inline float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

struct MaxNan {
    __device__ float operator()(float a, float b) const { return max_nan(a, b); }
};
struct Add {
    __device__ float operator()(float a, float b) const { return a + b; }
};

// Butterfly over the wave: every lane has the result, in an order that does
// not depend on the lane.
template <typename Op>
__device__ inline float wave_reduce(float v, Op op) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = op(v, __shfl_xor(v, off, 64));
    return v;
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

inline int op_cus() {
    int dev = 0, ncu = 0;
    if (hipGetDevice(&dev) != hipSuccess) return 256;
    if (hipDeviceGetAttribute(&ncu, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess)
        return 256;
    return ncu;
}

}  // namespace bk
