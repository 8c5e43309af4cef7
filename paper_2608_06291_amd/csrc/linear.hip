// 8-bit rows times a quantised layer's integer codes, with everything that follows in
// the epilogue:
//   z_ti = q_scale_t * sum_j s_ij q_tj c_ij + bias_i,   y = act(z) {alone | + other | * other}
// The products of 8-bit values run on the integer matrix cores and are summed exactly:
// |16 c q| <= 128 * 127 and n <= 2^17 keep the sum below 2^31.
#include "tile.h"

namespace bk {

struct LinearArgs {
    const int8_t* q;
    const char* w;           // packed codes
    const float* q_scale;
    const float* scale;
    const void* bias;
    const void* other;
    void* y;
    int64_t ldq, ldw, ldo, ldy;
    int64_t T, m;
    int chunks;              // of 128 codes
    int gsteps, ngroups;     // group_size / 64; groups of a row
    int act, combine, dtype;
    int ni, nt;              // tiles
};

// y_t,i..i+7 from the sums z (scales applied) and the bias.
template <typename E>
__device__ inline void linear_store(const LinearArgs& a, int64_t t, int64_t i, float (&z)[8]) {
    const int64_t valid = a.m - i;
    float v[8];
    if (a.bias) {
        load8(static_cast<const E*>(a.bias) + i, v, valid);
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] += v[j];
    }
    if (a.act != BAKRON_ACT_NONE) {
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = act_value(z[j], a.act);
    }
    if (a.combine != BAKRON_COMBINE_NONE) {
        load8(static_cast<const E*>(a.other) + t * a.ldo + i, v, valid);
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = a.combine == BAKRON_COMBINE_ADD ? z[j] + v[j] : z[j] * v[j];
    }
    store8(static_cast<E*>(a.y) + t * a.ldy + i, z, valid);
}

template <typename Tl, bool GROUPED>
__global__ __launch_bounds__(Tl::THREADS) void k_linear(LinearArgs a) {
    typedef typename Tl::Mma M;
    __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
    int ti, tt;
    tile_of(blockIdx.x, a.ni, a.nt, 8, &ti, &tt);
    const int64_t i0 = (int64_t)ti * Tl::ROWS, t0 = (int64_t)tt * Tl::COLS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr float UNIT = M::A_BYTES == CHUNK_BYTES ? 1.0f : 1.0f / 16.0f;

    typename Tl::Accs acc = {};
    f32x4 sum[GROUPED ? Tl::UA : 1][GROUPED ? Tl::UB : 1] = {};
    const Operand w{a.w, nullptr, a.ldw, a.m, a.ldw, 0};
    const Operand q{reinterpret_cast<const char*>(a.q), nullptr, a.ldq, a.T,
                    (int64_t)a.chunks * CHUNK_BYTES, 0};
    auto same = [](int r) { return r; };
    if constexpr (GROUPED) {
        const int64_t iw = i0 + Tl::a0(wave) + (lane >> 4) * 4;
        const int last = 2 * a.chunks - 1;
        int left = a.gsteps, g = 0;
        auto after = [&](int step, typename Tl::Accs& acc) {
            if (--left > 0 && step != last) return;
            left = a.gsteps;
            if (g < a.ngroups) {   // (past them only padding, whose sums are 0)
#pragma unroll
                for (int x = 0; x < Tl::UA; ++x) {
                    f32x4 s;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        s[j] = a.scale[min(iw + x * 16 + j, a.m - 1) * a.ngroups + g];
#pragma unroll
                    for (int y = 0; y < Tl::UB; ++y) {
                        i32x4& p = Tl::at(acc, x, y);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            sum[x][y][j] = fmaf((float)p[j], s[j], sum[x][y][j]);
                        p = i32x4{0, 0, 0, 0};
                    }
                }
            }
            ++g;
        };
        Tl::run(lds, w, i0, q, t0, a.chunks, acc, same, after);
    } else if constexpr (Tl::THREADS == 512) {
        Tl::run(lds, w, i0, q, t0, a.chunks, acc, same);
    } else {
        Tl::run(lds, w, i0, q, t0, a.chunks, acc, same, [](int, typename Tl::Accs&) {});
    }

    auto get = [&](int x, int y) {
        if constexpr (GROUPED) {
            return sum[x][y];
        } else {
            const i32x4 p = Tl::at(acc, x, y);
            return f32x4{(float)p[0], (float)p[1], (float)p[2], (float)p[3]};
        }
    };
    const auto rows = handover<Tl>(lds, wave, lane, get);
    constexpr int PER = Tl::UA * 2;   // lanes a row
    const int p = lane % PER;
    const int64_t i = i0 + Tl::a0(wave) + p * 8;
    float s[8];
    if (!GROUPED) load8(a.scale + min(i, a.m), s, a.m - i);
#pragma unroll
    for (int y = 0; y < Tl::UB; ++y) {
        rows.put(y);
#pragma unroll
        for (int tl = lane / PER; tl < 16; tl += 64 / PER) {
            const int64_t t = t0 + Tl::b0(wave) + y * 16 + tl;
            float z[8];
            rows.take(tl, p, z);
            if (t >= a.T || i >= a.m) continue;
            const float qs = (a.q_scale ? a.q_scale[t] : 1.0f) * UNIT;
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = GROUPED ? z[j] * qs : z[j] * (qs * s[j]);
            if (a.dtype == BAKRON_F32)
                linear_store<float>(a, t, i, z);
            else if (a.dtype == BAKRON_F16)
                linear_store<f16_t>(a, t, i, z);
            else
                linear_store<bf16_t>(a, t, i, z);
        }
    }
}

template <typename Tl, bool GROUPED>
static void launch_linear_tile(LinearArgs a, hipStream_t st) {
    a.ni = (int)((a.m + Tl::ROWS - 1) / Tl::ROWS);
    a.nt = (int)((a.T + Tl::COLS - 1) / Tl::COLS);
    hipLaunchKernelGGL((k_linear<Tl, GROUPED>), dim3((unsigned)(a.ni * a.nt)), dim3(Tl::THREADS), 0, st, a);
}

template <typename M, bool GROUPED>
static void launch_linear(const LinearArgs& a, hipStream_t st) {
    auto tiles = [&](int64_t b) { return ((a.m + b - 1) / b) * ((a.T + b - 1) / b); };
    const int ncu = op_cus();
    if constexpr (!GROUPED) {
        if (tiles(256) >= ncu) return launch_linear_tile<BigTile<M>, GROUPED>(a, st);
    }
    if (tiles(128) >= ncu) return launch_linear_tile<Tile<M, 128, 128, 2, 2>, GROUPED>(a, st);
    launch_linear_tile<Tile<M, 64, 64, 2, 2>, GROUPED>(a, st);
}

}  // namespace bk

extern "C" bakron_status bakron_linear(const int8_t* q, int64_t ldq, const float* q_scale,
                                       int64_t T, int64_t n, const void* packed, int32_t width,
                                       int64_t m, const float* scale, int64_t group_size,
                                       const void* bias, int32_t act, const void* other,
                                       int64_t ldo, int32_t combine, void* y, int64_t ldy,
                                       int32_t dtype, void* work, size_t* work_bytes,
                                       hipStream_t stream) {
    static const char who[] = "bakron_linear";
    bk::set_last_error("");
    if (T < 0 || T > bk::OP_T_MAX || n < 1 || m < 1 || n > ((int64_t)1 << 17) ||
        m > ((int64_t)1 << 20))
        return bk::op_fail(who, "bad size");
    if (width != 4 && width != 8) return bk::op_fail(who, "width must be 4 or 8");
    if (group_size < 0 || group_size % 64) return bk::op_fail(who, "group_size must be a multiple of 64");
    if (act < BAKRON_ACT_NONE || act > BAKRON_ACT_GELU) return bk::op_fail(who, "bad act");
    if (combine < BAKRON_COMBINE_NONE || combine > BAKRON_COMBINE_MUL)
        return bk::op_fail(who, "bad combine");
    if (dtype != BAKRON_F32 && dtype != BAKRON_F16 && dtype != BAKRON_BF16)
        return bk::op_fail(who, "bad dtype");
    bool query;
    const bakron_status st = bk::op_workspace(who, work, work_bytes, 0, &query);
    if (st != BAKRON_OK || query) return st;
    const int64_t np = (n + BAKRON_PACK_COLUMNS - 1) / BAKRON_PACK_COLUMNS * BAKRON_PACK_COLUMNS;
    if (ldq < np || ldq % 16) return bk::op_fail(who, "ldq must be a multiple of 16, at least n padded");
    if (ldq >= bk::TILE_LD_MAX) return bk::op_fail(who, "ldq too large");
    if (ldy < m || (other && ldo < m)) return bk::op_fail(who, "leading dimension below m");
    if ((combine != BAKRON_COMBINE_NONE) != (other != nullptr))
        return bk::op_fail(who, "other goes with combine");
    if (other && other == y && ldo != ldy)
        return bk::op_fail(who, "other in place needs the same leading dimension");
    if (T == 0) return BAKRON_OK;
    if (!q || !packed || !scale || !y) return bk::op_fail(who, "null pointer");
    if (((uintptr_t)q & 15) || ((uintptr_t)packed & 15))
        return bk::op_fail(who, "q and packed must be 16-byte aligned");
    if (((T + 63) / 64) * ((m + 63) / 64) > ((int64_t)1 << 24) - 1)
        return bk::op_fail(who, "too large for one call");
    bk::LinearArgs a{};
    a.q = q;
    a.w = static_cast<const char*>(packed);
    a.q_scale = q_scale;
    a.scale = scale;
    a.bias = bias;
    a.other = other;
    a.y = y;
    a.ldq = ldq;
    a.ldw = np * width / 8;
    a.ldo = ldo;
    a.ldy = ldy;
    a.T = T;
    a.m = m;
    a.chunks = (int)(np / BAKRON_PACK_COLUMNS);
    a.gsteps = (int)(group_size / 64);
    a.ngroups = group_size ? (int)((n + group_size - 1) / group_size) : 1;
    a.act = act;
    a.combine = combine;
    a.dtype = dtype;
    if (width == 4)
        group_size ? bk::launch_linear<bk::MmaI4, true>(a, stream)
                   : bk::launch_linear<bk::MmaI4, false>(a, stream);
    else
        group_size ? bk::launch_linear<bk::MmaI8, true>(a, stream)
                   : bk::launch_linear<bk::MmaI8, false>(a, stream);
    return bk::op_launched(who);
}
