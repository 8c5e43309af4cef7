// 8-bit rows times a quantised layer's integer codes, with everything that follows in
// the epilogue:
//   z_ti = q_scale_t * sum_j s_ij q_tj c_ij + bias_i,   y = act(z) {alone | + other | * other}
// The products of 8-bit values run on the integer matrix cores and are summed exactly:
// |16 c q| <= 128 * 127 and n <= 2^17 keep the sum below 2^31.
//
// Many rows: the tiles of tile.h.  2048 x 8192 x 28672 in 4 bits 389 to 428 us, 2250 to 2470 TOPS (the library's
// 8-bit product of 8192^3: 2200), in 8 bits 387, with GELU 420 to 434, with SiLU and a factor, whose 117 MB
// are read and multiplied while no tile is, 460 to 483; 4096^3 59 to 64 us, with a scale for 128 columns 93 to
// 102.  1001 x 4096 x 4096 with such scales 36 us (for 64 columns 37; 8-bit codes 29, and 22 to 24 with one
// scale a row): there each chunk's sums are scaled in fp32, two vector operations an
// accumulator against two MFMAs, and both sets of sums halve the tile that fits.
// Few rows: 1 x 4096 x 11008 in 4 bits with a scale for 128 columns 8.0 us (for 64 columns 9.9), of
// which the codes' 24 MB are 4.6 at the rate of a large copy; launch and three dependent trips to
// memory are the rest.  In 8 bits 10.8 (45 MB: 8.7), with a scale for 128 columns 12.1.
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
    int gshift;              // log2 gsteps, or -1
    int act, combine, dtype;
    int ni, nt;              // tiles
};

// Rows up to which a product is taken as one of few rows: 4096 x 11008 with 128-column groups, 32
// rows 14.5 us against 15.7 in 64 x 64 tiles, 64 rows 24.4 against 18.9.
constexpr int64_t FEW_ROWS = 32;
// And with few tiles (by 64 x 64) a CU: 7008 x 152 with 64-column groups, 2315 rows (less than half) 26.7 us
// against 35; 4096 x 160, 127 rows 8.2 against 15.2.
constexpr int64_t FEW_TILES = 2;

// y_t,i..i+N-1 from the sums z (scales applied), the bias and the entries of `other`.
template <typename E, int N>
__device__ inline void linear_store(const LinearArgs& a, int64_t t, int64_t i, float (&z)[N],
                                    const float (&bias)[N], const float (&other)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float v = act_value<sizeof(E) == 4>(z[j] + bias[j], a.act);
        if (a.combine == BAKRON_COMBINE_ADD) v += other[j];
        if (a.combine == BAKRON_COMBINE_MUL) v *= other[j];
        z[j] = v;
    }
    store_n(static_cast<E*>(a.y) + t * a.ldy + i, z, a.m - i);
}

// Everything after the sums, for a tile: z(j) gives the 8 sums of this lane's row in turn
// j.  The stores of one row may alias what the next ones read as far as the compiler
// knows, so the operands of a batch of rows are asked for before its first store.
template <typename E, int TURNS, typename Row, typename Sums>
__device__ inline void linear_rows(const LinearArgs& a, int64_t i, float unit, bool scaled, Row row,
                                   Sums sums) {
    constexpr int BATCH = TURNS < 4 ? TURNS : 32 / (4 * (int)sizeof(E));   // 32 registers of `other`
    const int64_t valid = a.m - i;
    float bias[8] = {}, s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s[j] = 1.0f;
    if (valid > 0) {
        if (a.bias) load_n(static_cast<const E*>(a.bias) + i, bias, valid);
        if (!scaled) load_n(a.scale + i, s, valid);
    }
#pragma unroll
    for (int j0 = 0; j0 < TURNS; j0 += BATCH) {
        float qs[BATCH];
        Pack<E, 8> other[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int64_t t = row(j0 + b);
            qs[b] = t < a.T && a.q_scale ? a.q_scale[t] : 1.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) other[b].v[j] = (E)0.0f;
            if (a.other && t < a.T && valid > 0) {
                const E* const p = static_cast<const E*>(a.other) + t * a.ldo + i;
                if (valid >= 8) {
                    other[b] = load_pack<E, 8>(p);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (j < valid) other[b].v[j] = p[j];
                }
            }
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            float z[8], o[8];
            sums(j0 + b, z);
            const int64_t t = row(j0 + b);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                z[j] *= qs[b] * unit * s[j];
                o[j] = (float)other[b].v[j];
            }
            if (t < a.T && valid > 0) linear_store<E>(a, t, i, z, bias, o);
        }
    }
}

template <typename Tl, int FLUSH>
__global__ __launch_bounds__(Tl::THREADS) void k_linear(LinearArgs a) {
    constexpr bool GROUPED = FLUSH > 0;
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
    if constexpr (GROUPED)
        Tl::run(lds, w, i0, q, t0, 0, a.chunks, acc, same, sum, [&](int r, int c, int k) {
            // (groups past the last one hold only padding, whose sums are 0)
            const int g = min((2 * c + k * FLUSH) / a.gsteps, a.ngroups - 1);
            return a.scale + min(i0 + r, a.m - 1) * a.ngroups + g;
        });
    else
        Tl::run(lds, w, i0, q, t0, 0, a.chunks, acc, same);

    auto get = [&](int x, int y) {
        if constexpr (GROUPED) {
            return sum[x][y];
        } else {
            const i32x4 p = Tl::at(acc, x, y);
            return f32x4{(float)p[0], (float)p[1], (float)p[2], (float)p[3]};
        }
    };
    const auto rows = handover<Tl>(lds, wave, lane, get);
    constexpr int PER = Tl::UA * 2, EACH = 64 / PER;   // lanes a row, rows at a time
    constexpr int TURNS = Tl::UB * 16 / EACH;
    const int p = lane % PER;
    const int64_t i = i0 + Tl::a0(wave) + p * 8, tw = t0 + Tl::b0(wave) + lane / PER;
    auto row = [&](int j) { return tw + j * EACH; };
    auto sums = [&](int j, float (&z)[8]) {
        if (j * EACH % 16 == 0) rows.put(j * EACH / 16);
        rows.take(j * EACH % 16 + lane / PER, p, z);
    };
    if (a.dtype == BAKRON_F32)
        linear_rows<float, TURNS>(a, i, UNIT, GROUPED, row, sums);
    else if (a.dtype == BAKRON_F16)
        linear_rows<f16_t, TURNS>(a, i, UNIT, GROUPED, row, sums);
    else
        linear_rows<bf16_t, TURNS>(a, i, UNIT, GROUPED, row, sums);
}

// Few rows (a decoding step): bound by reading the codes once, so no tile is staged.  A
// workgroup takes R units of 16 rows of codes and Y of 16 rows of q; its waves share the row's
// chunks of 128 codes in turn, every fragment straight from memory into registers, several
// chunks asked for at once.  The partial sums meet in LDS.
//
// FLUSH as in the tiles: sums are scaled once a chunk (2, or 0: at the end), or every 64 codes
// (1: groups that end inside a chunk).  In the first two cases a lane reads the 32 codes at
// 32 (lane / 16) of the chunk at once and takes them 16 and 16 (the order of the summed axis
// is free as long as q follows it): 64 or 128 bytes of a row side by side, not 32.
template <typename M, int FLUSH, int R, int Y>
__global__ __launch_bounds__(512) void k_linear_few(LinearArgs a) {
    constexpr bool GROUPED = FLUSH > 0, WIDE = FLUSH != 1;
    constexpr bool NARROW = M::A_BYTES != CHUNK_BYTES;
    constexpr float UNIT = NARROW ? 1.0f / 16.0f : 1.0f;
    extern __shared__ __attribute__((aligned(16))) char few_lds[];
    // scales as [group][row], then the partial sums as [wave][r][y][lane]
    float* const scales = reinterpret_cast<float*>(few_lds);
    const int nscales = GROUPED ? a.ngroups * R * 16 : 0;
    const int tid = threadIdx.x, lane = tid & 63, waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, kq = lane >> 4;
    const int64_t i0 = (int64_t)blockIdx.x * (R * 16);
    const int64_t t0 = (int64_t)blockIdx.y * (Y * 16);

    // byte of a chunk where this lane's first 16 entries begin, and from there to its second
    constexpr int Q_LANE = WIDE ? 32 : 16, Q_NEXT = WIDE ? 16 : 64;
    constexpr int W_LANE = NARROW ? Q_LANE / 2 : Q_LANE, W_NEXT = NARROW ? Q_NEXT / 2 : Q_NEXT;
    const char* w[R];
    const char* q[Y];
#pragma unroll
    for (int r = 0; r < R; ++r)
        w[r] = a.w + min(i0 + r * 16 + r16, a.m - 1) * a.ldw + kq * W_LANE;
#pragma unroll
    for (int y = 0; y < Y; ++y)
        q[y] = reinterpret_cast<const char*>(a.q) + min(t0 + y * 16 + r16, a.T - 1) * a.ldq + kq * Q_LANE;

    struct Block {   // a chunk
        i32x4 w[NARROW ? 1 : 2][R];
        i32x4 q[2][Y];
    };
    auto load = [&](Block& b, int c) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const char* const p = w[r] + c * M::A_BYTES;
            if constexpr (NARROW && WIDE) {
                b.w[0][r] = *reinterpret_cast<const i32x4*>(p);
            } else if constexpr (NARROW) {
                const i32x2 x = *reinterpret_cast<const i32x2*>(p), y = *reinterpret_cast<const i32x2*>(p + W_NEXT);
                b.w[0][r] = i32x4{x[0], x[1], y[0], y[1]};
            } else {
                b.w[0][r] = *reinterpret_cast<const i32x4*>(p);
                b.w[NARROW ? 0 : 1][r] = *reinterpret_cast<const i32x4*>(p + W_NEXT);
            }
        }
#pragma unroll
        for (int y = 0; y < Y; ++y)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                b.q[u][y] = *reinterpret_cast<const i32x4*>(q[y] + c * CHUNK_BYTES + u * Q_NEXT);
    };
    // A thread's first scale (32 groups of a row side by side) is asked for before the codes.
    const int sg = tid & 31, srow = tid >> 5, srows = blockDim.x >> 5;
    float sc = 0.0f;
    auto scale_at = [&](int row, int g) { return a.scale + min(i0 + row, a.m - 1) * a.ngroups + g; };
    if constexpr (GROUPED) {
        if (sg < a.ngroups) sc = *scale_at(min(srow, R * 16 - 1), sg);
    }
    // D chunks of this wave are asked for at once (4: 5% slower).
    constexpr int D = 2;
    Block b[D];
    auto load_all = [&](int c) {
#pragma unroll
        for (int k = 0; k < D; ++k)
            if (c + k * waves < a.chunks) load(b[k], c + k * waves);
    };
    load_all(wave);
    if constexpr (GROUPED) {
        for (int row = srow; row < R * 16; row += srows)
            for (int g = sg; g < a.ngroups; g += 32)
                scales[g * (R * 16) + row] = row == srow && g == sg ? sc : *scale_at(row, g);
        wait_lds();
        bare_barrier();
    }
    i32x4 acc[R][Y] = {};
    f32x4 sum[R][Y] = {};
    auto add = [&](const Block& b, int c) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            i32x4 p[Y];
            f32x4 s;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                i32x4 w = b.w[NARROW ? 0 : u][r];
                if constexpr (NARROW) w = unpack_codes(i32x2{w[2 * u], w[2 * u + 1]});
                if constexpr (GROUPED) {
                    if (FLUSH == 1 || u == 0) {
                        const int step = 2 * c + u;
                        const int g = a.gshift >= 0 ? step >> a.gshift : step / a.gsteps;
                        s = *reinterpret_cast<const f32x4*>(scales + min(g, a.ngroups - 1) * (R * 16) +
                                                            r * 16 + kq * 4);
                    }
#pragma unroll
                    for (int y = 0; y < Y; ++y) {
                        p[y] = M::mma(w, b.q[u][y], FLUSH == 1 || u == 0 ? i32x4{0, 0, 0, 0} : p[y]);
                        if (FLUSH == 1 || u == 1) {
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                sum[r][y][j] = fmaf((float)p[y][j], s[j], sum[r][y][j]);
                        }
                    }
                } else {
#pragma unroll
                    for (int y = 0; y < Y; ++y) acc[r][y] = M::mma(w, b.q[u][y], acc[r][y]);
                }
            }
        }
    };
    for (int c = wave; c < a.chunks; c += waves * D) {
        if (c != wave) load_all(c);
#pragma unroll
        for (int k = 0; k < D; ++k)
            if (c + k * waves < a.chunks) add(b[k], c + k * waves);
    }
    char* const parts = few_lds + (nscales * 4 + 15) / 16 * 16;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int y = 0; y < Y; ++y) {
            i32x4 v = acc[r][y];
            if constexpr (GROUPED) v = __builtin_bit_cast(i32x4, sum[r][y]);
            *reinterpret_cast<i32x4*>(parts + (((wave * R + r) * Y + y) * 64 + lane) * 16) = v;
        }
    __syncthreads();
    for (int u = wave; u < R * Y; u += waves) {   // a wave joins one unit
        const int r = u / Y, y = u % Y;
        i32x4 p = {0, 0, 0, 0};
        f32x4 f = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = 0; k < waves; ++k) {
            const i32x4 v = *reinterpret_cast<const i32x4*>(parts + ((k * R * Y + u) * 64 + lane) * 16);
            if constexpr (GROUPED)
                f += __builtin_bit_cast(f32x4, v);
            else
                p += v;
        }
        const int64_t t = t0 + y * 16 + r16, i = i0 + r * 16 + kq * 4;
        if (t >= a.T || i >= a.m) continue;
        const float qs = (a.q_scale ? a.q_scale[t] : 1.0f) * UNIT;
        float z[4];
        if constexpr (GROUPED) {
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] = f[j] * qs;
        } else {
            float s[4];
            load_n(a.scale + i, s, a.m - i);
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] = (float)p[j] * (qs * s[j]);
        }
        auto finish = [&](auto e) {
            typedef decltype(e) E;
            float bias[4] = {}, other[4] = {};
            if (a.bias) load_n(static_cast<const E*>(a.bias) + i, bias, a.m - i);
            if (a.other) load_n(static_cast<const E*>(a.other) + t * a.ldo + i, other, a.m - i);
            linear_store<E>(a, t, i, z, bias, other);
        };
        if (a.dtype == BAKRON_F32)
            finish(0.0f);
        else if (a.dtype == BAKRON_F16)
            finish(f16_t());
        else
            finish(bf16_t());
    }
}

template <typename Tl, int FLUSH>
static void launch_linear_tile(LinearArgs a, hipStream_t st) {
    a.ni = (int)((a.m + Tl::ROWS - 1) / Tl::ROWS);
    a.nt = (int)((a.T + Tl::COLS - 1) / Tl::COLS);
    hipLaunchKernelGGL((k_linear<Tl, FLUSH>), dim3((unsigned)(a.ni * a.nt)), dim3(Tl::THREADS), 0, st, a);
}

template <typename M, int FLUSH, int R, int Y>
static void launch_linear_few(const LinearArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)((a.m + R * 16 - 1) / (R * 16)), (unsigned)((a.T + Y * 16 - 1) / (Y * 16)));
    // as many waves as have work, 8 at most
    const int blocks = a.chunks;
    const int waves = blocks >= 8 ? 8 : blocks >= 4 ? 4 : blocks >= 2 ? 2 : 1;
    const int scales = FLUSH > 0 ? (a.ngroups * R * 16 * 4 + 15) / 16 * 16 : 0;
    hipLaunchKernelGGL((k_linear_few<M, FLUSH, R, Y>), grid, dim3(64 * waves),
                       scales + waves * R * Y * 1024, st, a);
}

// FLUSH: 0 one scale a row, 2 groups of whole chunks of 128 codes, 1 other multiples of 64.
template <typename M, int FLUSH>
static void launch_linear(const LinearArgs& a, hipStream_t st) {
    const int ncu = op_cus();
    // (a row's scales have to fit beside the partial sums)
    const bool fits = FLUSH == 0 || a.ngroups <= 256;
    if (a.T <= 16 && fits) return launch_linear_few<M, FLUSH, 1, 1>(a, st);
    if (a.T <= FEW_ROWS && fits) return launch_linear_few<M, FLUSH, 2, 2>(a, st);
    // Few tiles with a long way to sum: cut that way among the waves, too.
    if (fits && ((a.m + 63) / 64) * ((a.T + 63) / 64) * FEW_TILES <= ncu && a.chunks >= 8)
        return launch_linear_few<M, FLUSH, 2, 2>(a, st);
    const int tile = pick_tile(a.m, a.T, ncu, FLUSH == 0);
    // Three buffers of 4-bit rows leave room for two workgroups a CU, those of 8-bit rows do not.
    const bool deep = M::A_BYTES < CHUNK_BYTES || one_a_cu(128, a.m, a.T);
    if constexpr (FLUSH == 0) {
        if (tile == 256) return launch_linear_tile<BigTile<M>, 0>(a, st);
        if (tile == 128 && deep) return launch_linear_tile<Tile<M, 128, 128, 4, 2, 3>, 0>(a, st);
        if constexpr (M::A_BYTES == CHUNK_BYTES)
            if (tile == 128) return launch_linear_tile<Tile<M, 128, 128, 4, 2, 2>, 0>(a, st);
        launch_linear_tile<Tile<M, 64, 64, 2, 2, 4>, 0>(a, st);
    } else {
        if (tile == 128 && deep)
            return launch_linear_tile<Tile<M, 128, 128, 4, 2, 3, false, false, FLUSH>, FLUSH>(a, st);
        if constexpr (M::A_BYTES == CHUNK_BYTES)
            if (tile == 128)
                return launch_linear_tile<Tile<M, 128, 128, 4, 2, 2, false, false, FLUSH>, FLUSH>(a, st);
        launch_linear_tile<Tile<M, 64, 64, 2, 2, 4, false, false, FLUSH>, FLUSH>(a, st);
    }
}
template <typename M>
static void launch_linear(const LinearArgs& a, hipStream_t st) {
    if (a.gsteps == 0)
        launch_linear<M, 0>(a, st);
    else if (a.gsteps % 2 == 0)
        launch_linear<M, 2>(a, st);
    else
        launch_linear<M, 1>(a, st);
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
    a.gshift = a.gsteps > 0 && (a.gsteps & (a.gsteps - 1)) == 0 ? __builtin_ctz(a.gsteps) : -1;
    a.ngroups = group_size ? (int)((n + group_size - 1) / group_size) : 1;
    a.act = act;
    a.combine = combine;
    a.dtype = dtype;
    width == 4 ? bk::launch_linear<bk::MmaI4>(a, stream) : bk::launch_linear<bk::MmaI8>(a, stream);
    return bk::op_launched(who);
}
