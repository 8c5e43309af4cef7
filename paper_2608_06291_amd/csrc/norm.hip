// Residual addition, RMS norm and 8-bit rows with one scale each.
//
//   h = x + r,   y = w (.) h / sqrt(mean(h^2) + eps),   s = max |y| / 127,   q = rint(y / s)
//
// Every entry is read once and stays in registers over the two reductions of its row (the
// sum of squares, then the largest |y|, which needs the first), so the kernel moves what it
// must: x and r in, h and q out.  Bound by memory: 4096 x 8192 bf16 with a residual 40 us,
// 5.9 TB/s of 235 MB (a large copy here: 5.2), 2048 x 8192 fp32 34 us; one row of 4096 3.6 us,
// all latency.  A row per workgroup of one or two vectors a thread; loads are whole vectors
// at clamped addresses, issued together (with a branch around each they went one after
// the other: 47.5 us).  fp32 rows of more than 32768 entries take 64 of them a thread, and
// about 50 registers go to memory and back: 1024 x 65536 220 us, 4.0 TB/s.
#include "ops.h"

namespace bk {

struct NormArgs {
    const void* x;
    const void* res;
    const float* w;
    void* sum;
    void* y;
    int8_t* q;
    float* scale;
    int64_t ldx, ldr, lds, ldy, ldq;
    int64_t T;
    int d;
    int dpad;        // q columns written: d rounded up, within ldq
    float eps;
    int normalise;
};

// A row belongs to blockDim.x threads (one wave, with blockDim.y rows in the
// workgroup, or the whole workgroup); thread t holds the whole vectors t, t + blockDim.x, ..
// of VEC entries, NV of them, and one entry of what is left of the row.
template <typename E, int NV>
__global__ __launch_bounds__(1024) void k_norm(NormArgs a) {
    constexpr int VEC = 16 / sizeof(E);
    __shared__ float red[3][16];
    const int tid = threadIdx.x, tpr = blockDim.x, lane = tid & 63, wave = tid >> 6;
    const int waves = tpr >> 6;
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= a.T) return;   // (a whole wave, and never one of several in a row)
    const E* const x = static_cast<const E*>(a.x) + row * a.ldx;
    const E* const res = a.res ? static_cast<const E*>(a.res) + row * a.ldr : nullptr;
    const int whole = a.d / VEC, left = whole * VEC + tid;

    // Vectors read at once: not so many that both operands wait in registers of their own.
    constexpr int STEP = NV * VEC <= 32 ? NV : 32 / VEC;
    constexpr bool EARLY = NV * VEC <= 16;   // the weights, too, before the first reduction
    float h[NV][VEC], hx = 0.0f, ssq = 0.0f;
    Pack<float, VEC> pw[NV];
#pragma unroll
    for (int i0 = 0; i0 < NV; i0 += STEP) {
        u32x4 rx[STEP], rr[STEP];
#pragma unroll
        for (int i = 0; i < STEP; ++i) rx[i] = rr[i] = u32x4(0);
        if (whole > 0) {   // (past the row its last vector, not used)
#pragma unroll
            for (int i = 0; i < STEP; ++i)
                rx[i] = load_words(x + min((i0 + i) * tpr + tid, whole - 1) * VEC);
            if (res) {
#pragma unroll
                for (int i = 0; i < STEP; ++i)
                    rr[i] = load_words(res + min((i0 + i) * tpr + tid, whole - 1) * VEC);
            }
            if (EARLY && a.w) {
#pragma unroll
                for (int i = 0; i < NV; ++i)
                    pw[i] = load_pack<float, VEC>(a.w + min(i * tpr + tid, whole - 1) * VEC);
            }
        }
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
            const bool in = (i0 + i) * tpr + tid < whole;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float v = entry<E>(rx[i], j) + entry<E>(rr[i], j);
                h[i0 + i][j] = in ? v : 0.0f;
                ssq = fmaf(h[i0 + i][j], h[i0 + i][j], ssq);
            }
        }
    }
    if (left < a.d) hx = (float)x[left] + (res ? (float)res[left] : 0.0f);
    ssq = fmaf(hx, hx, ssq);
    auto store = [&](void* base, int64_t ld) {   // h, rounded once
        E* const out = static_cast<E*>(base) + row * ld;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * tpr + tid;
            Pack<E, VEC> p;
#pragma unroll
            for (int j = 0; j < VEC; ++j) p.v[j] = (E)h[i][j];
            if (v < whole) store_pack(out + v * VEC, p);
        }
        if (left < a.d) out[left] = (E)hx;
    };
    if (a.sum) store(a.sum, a.lds);
    float r = 1.0f;
    if (a.normalise) {
        ssq = group_reduce(ssq, Add(), red[0], wave, lane, waves);
        float v = ssq / (float)a.d + a.eps;
        if (v < 0x1p-120f) {   // (eps smaller still) squares that fp32 does not hold: again, of h 2^96
            ssq = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    h[i][j] *= 0x1p96f;
                    ssq = fmaf(h[i][j], h[i][j], ssq);
                }
            }
            hx *= 0x1p96f;
            ssq = group_reduce(fmaf(hx, hx, ssq), Add(), red[2], wave, lane, waves);
            v = ssq / (float)a.d + a.eps * 0x1p96f * 0x1p96f;
        }
        r = v == 0.0f ? 0.0f : 1.0f / sqrtf(v);
        if (!(v < INFINITY)) r = NAN;   // squares beyond fp32: not silently 0
    }
    hx *= r;
    if (a.w && left < a.d) hx *= a.w[left];
    float top = fabsf(hx);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) h[i][j] *= r;
        if (a.w && whole > 0) {
            if (!EARLY) pw[i] = load_pack<float, VEC>(a.w + min(i * tpr + tid, whole - 1) * VEC);
#pragma unroll
            for (int j = 0; j < VEC; ++j) h[i][j] *= pw[i].v[j];
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) top = max_nan(top, i * tpr + tid < whole ? fabsf(h[i][j]) : 0.0f);
    }
    if (a.y) store(a.y, a.ldy);
    if (!a.q) return;
    top = group_reduce(top, MaxNan(), red[1], wave, lane, waves);
    const bool finite = top < INFINITY;
    const float s = finite ? top / 127.0f : NAN;
    if (tid == 0) a.scale[row] = s;
    // y / s as a product where 1 / s exists, so a division only for rows below 2^-119, whose scale may
    // be a few steps of the smallest number: rounded down, it takes y / s beyond 127
    const bool tiny = top < 1.5e-36f;
    const float inv = finite && !tiny ? 127.0f / top : 0.0f;
    auto code = [&](float v) {
        float c = v * inv;
        if (tiny) c = s > 0.0f ? fminf(fmaxf(v / s, -127.0f), 127.0f) : 0.0f;
        return finite ? (int8_t)(int)rintf(c) : (int8_t)0;
    };
    int8_t* const out = a.q + row * a.ldq;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = i * tpr + tid;
        Pack<int8_t, VEC> p;
#pragma unroll
        for (int j = 0; j < VEC; ++j) p.v[j] = code(h[i][j]);
        if (v < whole) store_pack(out + v * VEC, p);
    }
    if (left < a.d) out[left] = code(hx);
    for (int c = a.d + tid; c < a.dpad; c += tpr) out[c] = 0;
}

// Codes to packed rows: a thread writes 16 bytes (32 codes of 4 bits, 16 of 8) at a time.
template <int WIDTH>
__global__ __launch_bounds__(256) void k_pack(const int8_t* __restrict__ codes, int64_t m, int64_t n,
                                              int64_t np, uint32_t* __restrict__ packed) {
    constexpr int PER = 128 / WIDTH;
    const int64_t per_row = np / PER;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < m * per_row; e += (int64_t)gridDim.x * 256) {
        const int64_t i = e / per_row, c = e % per_row * PER;
        const int8_t* const src = codes + i * n;
        uint32_t out[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const uint32_t v = c + j < n ? (uint32_t)(uint8_t)src[c + j] : 0u;
            if (WIDTH == 8)
                out[j / 4] |= v << (8 * (j % 4));
            else
                out[j / 8] |= (v & 15u) << (8 * (j % 4) + (j % 8 >= 4 ? 4 : 0));
        }
        uint32_t* const dst = packed + e * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) dst[j] = out[j];
    }
}

template <typename E>
static void launch_norm(const NormArgs& a, hipStream_t st) {
    constexpr int VEC = 16 / sizeof(E);
    const int vecs = (a.d + VEC - 1) / VEC;
    constexpr int NV_MAX = 64 / VEC;
    // Threads a row: one vector a thread with few rows, where the latency of the
    // row counts; two with many.
    int nv = a.T < 1024 ? 1 : 2, tpr = 64;
    while (tpr < 1024 && tpr * nv < vecs) tpr *= 2;
    while (nv < NV_MAX && tpr * nv < vecs) nv *= 2;
    const int rows = tpr == 64 ? 4 : 1;
    if (a.T * tpr > OP_LAUNCH_MAX) {   // more threads than one launch takes
        NormArgs b = a;
        b.T = OP_LAUNCH_MAX / tpr;
        launch_norm<E>(b, st);
        b.T = a.T - OP_LAUNCH_MAX / tpr;
        const int64_t r = OP_LAUNCH_MAX / tpr;
        b.x = static_cast<const E*>(a.x) + r * a.ldx;
        if (a.res) b.res = static_cast<const E*>(a.res) + r * a.ldr;
        if (a.sum) b.sum = static_cast<E*>(a.sum) + r * a.lds;
        if (a.y) b.y = static_cast<E*>(a.y) + r * a.ldy;
        if (a.q) {
            b.q = a.q + r * a.ldq;
            b.scale = a.scale + r;
        }
        return launch_norm<E>(b, st);
    }
    const dim3 grid((unsigned)((a.T + rows - 1) / rows)), block(tpr, rows);
    switch (nv) {
        case 1: hipLaunchKernelGGL((k_norm<E, 1>), grid, block, 0, st, a); break;
        case 2: hipLaunchKernelGGL((k_norm<E, 2>), grid, block, 0, st, a); break;
        case 4: hipLaunchKernelGGL((k_norm<E, 4>), grid, block, 0, st, a); break;
        case 8: hipLaunchKernelGGL((k_norm<E, 8>), grid, block, 0, st, a); break;
        default: hipLaunchKernelGGL((k_norm<E, NV_MAX>), grid, block, 0, st, a); break;
    }
}

}  // namespace bk

extern "C" bakron_status bakron_rmsnorm_quant(const void* x, int64_t ldx, const void* residual,
                                              int64_t ldr, int32_t dtype, int64_t T, int64_t d,
                                              const float* weight, float eps, int32_t normalise,
                                              void* sum, int64_t lds, void* y, int64_t ldy,
                                              int8_t* q, int64_t ldq, float* scale,
                                              hipStream_t stream) {
    static const char who[] = "bakron_rmsnorm_quant";
    bk::set_last_error("");
    if (T < 0 || T > bk::OP_T_MAX || d < 1 || d > 65536) return bk::op_fail(who, "bad size");
    if (dtype != BAKRON_F32 && dtype != BAKRON_F16 && dtype != BAKRON_BF16)
        return bk::op_fail(who, "bad dtype");
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return bk::op_fail(who, "bad eps");
    if (!q != !scale) return bk::op_fail(who, "q and scale go together");
    if (ldx < d || (residual && ldr < d) || (sum && lds < d) || (y && ldy < d) || (q && ldq < d))
        return bk::op_fail(who, "leading dimension below d");
    if (((sum && sum == x) && lds != ldx) || ((sum && sum == residual) && lds != ldr))
        return bk::op_fail(who, "sum in place needs the same leading dimension");
    if (T == 0) return BAKRON_OK;
    if (!x) return bk::op_fail(who, "null pointer");
    const int64_t up = (d + BAKRON_PACK_COLUMNS - 1) / BAKRON_PACK_COLUMNS * BAKRON_PACK_COLUMNS;
    bk::NormArgs a{x, residual, weight, sum, y, q, scale, ldx, ldr, lds, ldy, ldq, T, (int)d,
                   (int)(ldq < up ? ldq : up), eps, normalise != 0};
    if (dtype == BAKRON_F32)
        bk::launch_norm<float>(a, stream);
    else if (dtype == BAKRON_F16)
        bk::launch_norm<bk::f16_t>(a, stream);
    else
        bk::launch_norm<bk::bf16_t>(a, stream);
    return bk::op_launched(who);
}

extern "C" bakron_status bakron_pack_codes(const int8_t* codes, int64_t m, int64_t n, int32_t width,
                                           void* packed, hipStream_t stream) {
    static const char who[] = "bakron_pack_codes";
    bk::set_last_error("");
    if (m < 1 || n < 1 || m > ((int64_t)1 << 20) || n > ((int64_t)1 << 17))
        return bk::op_fail(who, "bad size");
    if (width != 4 && width != 8) return bk::op_fail(who, "width must be 4 or 8");
    if (!codes || !packed) return bk::op_fail(who, "null pointer");
    if ((uintptr_t)packed & 15) return bk::op_fail(who, "packed must be 16-byte aligned");
    const int64_t np = (n + BAKRON_PACK_COLUMNS - 1) / BAKRON_PACK_COLUMNS * BAKRON_PACK_COLUMNS;
    const dim3 grid = bk::stride_grid(m * np * width / 128);
    if (width == 4)
        hipLaunchKernelGGL(bk::k_pack<4>, grid, dim3(256), 0, stream, codes, m, n, np,
                           static_cast<uint32_t*>(packed));
    else
        hipLaunchKernelGGL(bk::k_pack<8>, grid, dim3(256), 0, stream, codes, m, n, np,
                           static_cast<uint32_t*>(packed));
    return bk::op_launched(who);
}
