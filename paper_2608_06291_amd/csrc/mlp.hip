// The hidden layer of a gated MLP and its gradients (16-bit floats, fp32 sums):
//   G = x Wg^T,  U = x Wu^T,  h = act(G) (.) U
//   dG = dh (.) U (.) act'(G),  dU = dh (.) act(G)
//   dx = dG Wg + dU Wu,  dWg = dG^T x,  dWu = dU^T x
// One tile product serves them all.  Rows of Wg and Wu are taken 16 by 16 in turn, so
// that the same lane ends with G and U of the same entries and the activation and the
// product happen on its registers.  The gradients come from the same product, with dG and
// dU (rounded to 16 bits, as operands of the products that follow) in its epilogue.
//
// G and U are computed again in the backward pass (two of its six products, and 4 T f bytes less
// to keep).  dG and dU are rounded to 16 bits, as the products that follow take them: one
// rounding more than fp32 arithmetic, so dx and the weights' gradients are off by 2.4e-3 of their
// norm in bf16 where a single rounding gives 1.7e-3 (2.9e-4 and 2.1e-4 in half precision), except where
// few entries make up a result (backward_plan).
// In half precision their range counts, too: see GradScale.
// The gradients' products read the weights, x, dG and dU as they lie (columns, see
// tile.h), with no transposed copies.
//
// Measured (bf16, 4096 -> 11008): 8192 rows 1068 to 1220 us by the box, 1210 to 1384 TFLOP/s (the
// library's product of that size: 1312 to 1363), matrix cores 68% busy, with the features, 8 bytes more an
// entry, 1240 to 1290; backward of 4096 rows 1790 to 1910 us: gated product 584, dx 518 (matrix cores 66%
// busy), dW 673 (53%), in half precision 617, 535, 679.  The first and last take 5.4 rounds of tiles in the
// time of 6; of dW both operands come by transposing reads.  One row 35 us: the weights' 180 MB at 5.2 TB/s.
#include "product.h"

namespace bk {

struct GatedArgs {
    Operand x, w;                  // w: rows of Wg at base, of Wu at base2
    int64_t T, f;
    int chunks, act;
    int ni, nt;
    // forward
    void* h;
    int64_t ldh;
    float *feat_up, *feat_gate;
    // backward
    const void* dh;
    int64_t lddh;
    void* dgu;                     // T rows: dG | dU (fp each, zeros in the padding), then their rests
    int64_t fp, ldg;               // ldg: 2 fp entries, or 4 fp with the rests
    float* top;                    // half precision: the largest |dG|, |dU| of every wave
    const float* factor;           // .. and what this second run takes them times (1: not needed)
};

// Half precision holds 6e-8 to 65504, eleven bits from 6e-5 on.  dG and dU of a loss that is a mean over
// many tokens lie below that, and large ones beyond it, where dx and dW need not.  So the gated product
// leaves the largest of them that is finite; where that is below 1 or beyond 65504 a second run of it takes
// all of them times the power of two that puts the largest at 2^14 to 2^15, and the products that
// follow undo it (in fp32).  Then no number down to 2^-29 of the largest loses a bit.  The second run is
// launched in any case and ends at once where there is nothing to do: 1111 x 1000 -> 2731 75.4 -> 79.2 us,
// and 24 more where the run is needed.
struct GradScale {
    float factor, undo;
};
__global__ __launch_bounds__(1024) void k_grad_scale(const float* __restrict__ top, int64_t n, GradScale* out) {
    __shared__ float red[16];
    float m = 0.0f;
    for (int64_t i = threadIdx.x; i < n; i += 1024) m = fmaxf(m, top[i]);
    m = group_reduce(m, MaxNan(), red, threadIdx.x >> 6, threadIdx.x & 63, 16);
    if (threadIdx.x != 0) return;
    int e = 15;
    if (m > 0.0f && (m < 1.0f || m > 65504.0f)) frexpf(m, &e);   // m < 2^e
    e = max(e, 15 - 126);                                        // (both powers are normal numbers)
    *out = GradScale{ldexpf(1.0f, 15 - e), ldexpf(1.0f, e - 15)};
}

// What few rows need beside that: x and the weights as they are, in entries.
struct FewArgs {
    const void *x, *wg, *wu;
    int64_t ldx, ldw;
    int d;
};

// Row t, features j .. j + N - 1, from G and U; `top` grows with the largest |dG|, |dU|.
template <typename E, bool BWD, int N>
__device__ inline void gated_finish(const GatedArgs& a, int64_t t, int64_t j, const float (&G)[N],
                                    const float (&U)[N], const float (&dh)[N], float factor, float& top) {
    const int64_t valid = a.f - j;
    if constexpr (!BWD) {
        if (valid <= 0) return;
        float v[N], s[N];
        if (a.feat_gate) {
#pragma unroll
            for (int r = 0; r < N; ++r) {
                act_both(G[r], a.act, &v[r], &s[r]);
                s[r] *= U[r];
            }
            store_n(a.feat_gate + t * a.f + j, s, valid);
        } else {
#pragma unroll
            for (int r = 0; r < N; ++r) v[r] = act_value(G[r], a.act);
        }
        if (a.feat_up) store_n(a.feat_up + t * a.f + j, v, valid);
        if (a.h) {
#pragma unroll
            for (int r = 0; r < N; ++r) v[r] *= U[r];
            store_n(static_cast<E*>(a.h) + t * a.ldh + j, v, valid);
        }
    } else {
        if (j >= a.fp) return;
        float dg[N], du[N];
#pragma unroll
        for (int r = 0; r < N; ++r) {
            float v, s;
            act_both(G[r], a.act, &v, &s);
            dg[r] = r < valid ? dh[r] * U[r] * s : 0.0f;   // (0 in the padding, whatever G is)
            du[r] = r < valid ? dh[r] * v : 0.0f;
            if constexpr (narrow_range<E>) {
                top = fmaxf(top, __builtin_isfinite(dg[r]) ? fabsf(dg[r]) : 0.0f);
                top = fmaxf(top, __builtin_isfinite(du[r]) ? fabsf(du[r]) : 0.0f);
                dg[r] *= factor;
                du[r] *= factor;
            }
        }
        E* const row = static_cast<E*>(a.dgu) + t * a.ldg + j;
        store_n(row, dg, N);
        store_n(row + a.fp, du, N);
        if (a.ldg > 2 * a.fp) {   // what the rounding took (nothing beside what is not finite)
#pragma unroll
            for (int r = 0; r < N; ++r) {
                const float g = (float)(E)dg[r], u = (float)(E)du[r];
                dg[r] = __builtin_isfinite(g) ? dg[r] - g : 0.0f;
                du[r] = __builtin_isfinite(u) ? du[r] - u : 0.0f;
            }
            store_n(row + 2 * a.fp, dg, N);
            store_n(row + 3 * a.fp, du, N);
        }
    }
}

template <typename Tl, bool BWD>
__global__ __launch_bounds__(Tl::THREADS) void k_gated(GatedArgs a) {
    typedef typename Tl::Mma::Elem E;
    __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
    const float factor = BWD && narrow_range<E> && a.factor ? *a.factor : 1.0f;
    if (BWD && narrow_range<E> && a.factor && factor == 1.0f) return;
    int ti, tt;
    tile_of(blockIdx.x, a.ni, a.nt, 8, &ti, &tt);
    const int64_t f0 = (int64_t)ti * (Tl::ROWS / 2), t0 = (int64_t)tt * Tl::COLS;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    static_assert(Tl::UA % 2 == 0, "gate and up rows in one wave");

    typename Tl::Accs acc = {};
    // Tile row r: gate and up in turn, 16 and 16.  The rows that a wave loads are all of
    // one matrix: 8 at a time, multiples of 32 (or 64) apart.
    const bool up = (wave >> 1) & 1;
    Operand w = a.w;
    if (up) w.base = a.w.base2;
    const int64_t first = min(f0, a.f - 1);
    auto feature = [](int r) { return (r >> 5) * 16 + (r & 15); };
    Tl::run(lds, w, first, a.x, t0, 0, a.chunks, acc, feature);

    const auto rows =
        handover<Tl>(lds, wave, lane, [&](int x, int y) { return Tl::at(acc, x, y); });
    constexpr int PER = Tl::UA;   // lanes a row: 8 features each
    const int p = lane % PER;
    const int64_t j = f0 + Tl::a0(wave) / 2 + p * 8;
    const int tl = lane / PER;
    const int64_t tw = t0 + Tl::b0(wave) + tl;
    // (all of dh before the first store, which may alias it as far as the compiler knows)
    u32x4 dh[BWD ? Tl::UB : 1];
    if constexpr (BWD) {
#pragma unroll
        for (int y = 0; y < Tl::UB; ++y) {
            dh[y] = u32x4(0);
            const E* const p = static_cast<const E*>(a.dh) + (tw + y * 16) * a.lddh + j;
            if (tl < 16 && tw + y * 16 < a.T && j + 8 <= a.f) {
                dh[y] = load_words(p);
            } else if (tl < 16 && tw + y * 16 < a.T && j < a.f) {
                float v[8];
                load_n(p, v, a.f - j);
                Pack<E, 8> e;
#pragma unroll
                for (int r = 0; r < 8; ++r) e.v[r] = (E)v[r];
                __builtin_memcpy(&dh[y], &e, 16);
            }
        }
    }
    float top = 0.0f;
#pragma unroll
    for (int y = 0; y < Tl::UB; ++y) {
        rows.put(y);
        const int64_t t = tw + y * 16;
        float G[8], U[8], d[8];
        rows.take(tl & 15, (p >> 1) * 4 + (p & 1), G);
        rows.take(tl & 15, (p >> 1) * 4 + (p & 1) + 2, U);
#pragma unroll
        for (int r = 0; r < 8; ++r) d[r] = BWD ? entry<E>(dh[BWD ? y : 0], r) : 0.0f;
        if (tl < 16 && t < a.T) gated_finish<E, BWD>(a, t, j, G, U, d, factor, top);
    }
    if constexpr (BWD && narrow_range<E>) {
        top = wave_reduce(top, MaxNan());
        if (lane == 0) a.top[(int64_t)blockIdx.x * (Tl::THREADS / 64) + wave] = top;
    }
}

constexpr int FEW_STEPS = 2;

// Few rows (a decoding step): bound by reading the weights once.  A workgroup takes 16
// features and Y units of 16 rows; its waves share the summed axis, blocks of two steps of 32 in
// turn, every fragment straight from memory (at any alignment) into registers, BLOCKS blocks asked
// for at once (which wave sums what, and in which order, does not depend on it).  The partial sums
// meet in LDS.
//
// SHIFT: rows of an odd number of entries, every other of them 2 bytes off a word.  16-byte reads
// there are several times slower (4097 -> 11008, one row 79 us, 46 with this), so a lane
// reads the words around its piece and shifts; the host makes sure that those words hold an
// entry of the matrix (launch_gated).
template <typename M, bool BWD, int Y, int BLOCKS, bool SHIFT>
__global__ __launch_bounds__(512) void k_gated_few(FewArgs f, GatedArgs a) {
    typedef typename M::Elem E;
    extern __shared__ __attribute__((aligned(16))) char few_lds[];
    const float factor = BWD && narrow_range<E> && a.factor ? *a.factor : 1.0f;
    if (BWD && narrow_range<E> && a.factor && factor == 1.0f) return;
    const int tid = threadIdx.x, lane = tid & 63, waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, kq = lane >> 4;
    const int64_t j0 = (int64_t)blockIdx.x * 16, t0 = (int64_t)blockIdx.y * (Y * 16);
    const int64_t jr = min(j0 + r16, a.f - 1);
    const E* const wg = static_cast<const E*>(f.wg) + jr * f.ldw + kq * 8;
    const E* const wu = static_cast<const E*>(f.wu) + jr * f.ldw + kq * 8;
    const E* x[Y];
#pragma unroll
    for (int y = 0; y < Y; ++y)
        x[y] = static_cast<const E*>(f.x) + min(t0 + y * 16 + r16, a.T - 1) * f.ldx + kq * 8;
    constexpr int U = FEW_STEPS;
    const int nblocks = f.d / (32 * U), nsteps = f.d / 32;   // what is left goes to the last wave

    struct Block {
        FewPiece<SHIFT> g[U], u[U], x[U][Y];
    };
    auto load = [&](Block& b, int k) {
#pragma unroll
        for (int i = 0; i < U; ++i) b.g[i].load(wg + k + i * 32);
#pragma unroll
        for (int i = 0; i < U; ++i) b.u[i].load(wu + k + i * 32);
#pragma unroll
        for (int y = 0; y < Y; ++y)
#pragma unroll
            for (int i = 0; i < U; ++i) b.x[i][y].load(x[y] + k + i * 32);
    };
    f32x4 G[Y] = {}, Up[Y] = {};
    auto add = [&](u32x4 g, u32x4 u, const u32x4 (&v)[Y]) {
#pragma unroll
        for (int y = 0; y < Y; ++y) {
            const i32x4 b = __builtin_bit_cast(i32x4, v[y]);
            G[y] = M::mma(__builtin_bit_cast(i32x4, g), b, G[y]);
            Up[y] = M::mma(__builtin_bit_cast(i32x4, u), b, Up[y]);
        }
    };
    for (int c = wave; c < nblocks; c += waves * BLOCKS) {
        Block b[BLOCKS];
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k)
            if (c + k * waves < nblocks) load(b[k], (c + k * waves) * (32 * U));
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k) {
            if (c + k * waves >= nblocks) break;
#pragma unroll
            for (int i = 0; i < U; ++i) {
                u32x4 v[Y];
#pragma unroll
                for (int y = 0; y < Y; ++y) v[y] = b[k].x[i][y].get(x[y]);
                add(b[k].g[i].get(wg), b[k].u[i].get(wu), v);
            }
        }
    }
    // What is left: whole steps one a wave, then the piece of a step.
    for (int s = nblocks * U + wave; s < nsteps; s += waves) {
        u32x4 v[Y];
#pragma unroll
        for (int y = 0; y < Y; ++y) v[y] = load_words(x[y] + s * 32);
        add(load_words(wg + s * 32), load_words(wu + s * 32), v);
    }
    if (f.d % 32 != 0 && wave == (nsteps - nblocks * U) % waves) {
        const int k = nsteps * 32, left = f.d - k - kq * 8;   // entries of this lane's pieces
        auto part = [&](const E* p) { return few_part(p + k, left, f.d); };
        u32x4 v[Y];
#pragma unroll
        for (int y = 0; y < Y; ++y) v[y] = part(x[y]);
        add(part(wg), part(wu), v);
    }
#pragma unroll
    for (int y = 0; y < Y; ++y) {
        *reinterpret_cast<f32x4*>(few_lds + ((wave * Y + y) * 128 + lane) * 16) = G[y];
        *reinterpret_cast<f32x4*>(few_lds + ((wave * Y + y) * 128 + 64 + lane) * 16) = Up[y];
    }
    __syncthreads();
    for (int y = wave; y < Y; y += waves) {   // a wave joins one unit of rows
        f32x4 g = {0.0f, 0.0f, 0.0f, 0.0f}, u = g;
        for (int k = 0; k < waves; ++k) {
            g += *reinterpret_cast<const f32x4*>(few_lds + ((k * Y + y) * 128 + lane) * 16);
            u += *reinterpret_cast<const f32x4*>(few_lds + ((k * Y + y) * 128 + 64 + lane) * 16);
        }
        const int64_t t = t0 + y * 16 + r16;
        float gv[4], uv[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) gv[r] = g[r], uv[r] = u[r];
        float dh[4] = {};
        const int64_t j = j0 + kq * 4;
        if (BWD && t < a.T && j < a.f) load_n(static_cast<const E*>(a.dh) + t * a.lddh + j, dh, a.f - j);
        float top = 0.0f;
        if (t < a.T) gated_finish<E, BWD>(a, t, j, gv, uv, dh, factor, top);
        if constexpr (BWD && narrow_range<E>) {
            top = wave_reduce(top, MaxNan());
            if (lane == 0) a.top[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * Y + y] = top;
        }
    }
}

// Rows up to which the gated product is taken as one of few rows: 4096 -> 11008, 32 rows 52 us
// (64 x 64 tiles: 50, and two copies more for rows that are no 16-byte multiples), 64 rows
// 73 against 50.  And with few tiles (by 64 x 64) a CU: 2048 -> 512, 200 rows (a quarter) 10.7 us
// against 14.3, 500 rows (half) 17.5 against 14.2.
constexpr int64_t FEW_ROWS = 32;
constexpr int64_t FEW_TILES = 4;

// Values of GatedArgs.top that a launch writes at most (the kernels for few rows: one for 16 features of
// 16 rows, in pairs; tiles: no more, a wave's part being 16 features of 32 rows or larger).  fp is a multiple
// of 64.
static int64_t gated_tops(int64_t T, int64_t fp) { return (T + 31) / 32 * 2 * (fp / 16); }

// The launches return how many values of GatedArgs.top they write.
template <typename M, bool BWD, int Y, int BLOCKS>
static int64_t launch_gated_few(const FewArgs& f, const GatedArgs& a, hipStream_t st) {
    // Words around the pieces of odd rows: the first row of each matrix begins on a word, and whole steps
    // end before the row does, so an entry before and one behind each piece are in the matrix.
    const bool shift = (f.ldx % 2 != 0 || f.ldw % 2 != 0) && f.d % 32 != 0 && (uintptr_t)f.x % 4 == 0 &&
                       (uintptr_t)f.wg % 4 == 0 && (uintptr_t)f.wu % 4 == 0;
    const dim3 grid((unsigned)(((BWD ? a.fp : a.f) + 15) / 16), (unsigned)((a.T + Y * 16 - 1) / (Y * 16)));
    const int blocks = f.d / (32 * FEW_STEPS);   // as many waves as have work, 8 at most
    const int waves = blocks >= 8 ? 8 : blocks >= 4 ? 4 : blocks >= 2 ? 2 : 1;
    if (shift)
        hipLaunchKernelGGL((k_gated_few<M, BWD, Y, 2, true>), grid, dim3(64 * waves), waves * Y * 2048, st, f, a);
    else
        hipLaunchKernelGGL((k_gated_few<M, BWD, Y, BLOCKS, false>), grid, dim3(64 * waves), waves * Y * 2048, st, f, a);
    return (int64_t)grid.x * grid.y * Y;
}

// Whether the kernel for few rows takes it: few rows, or few tiles with a long way to sum.
static bool gated_few_rows(int64_t T, int64_t f, int64_t d) {
    if (T <= FEW_ROWS) return true;
    return ((f + 31) / 32) * ((T + 63) / 64) * FEW_TILES <= op_cus() && d >= 512;
}

template <typename M, bool BWD>
static int64_t launch_gated(const FewArgs& few, GatedArgs a, hipStream_t st) {
    if (gated_few_rows(a.T, a.f, few.d))
        return a.T <= 16 ? launch_gated_few<M, BWD, 1, 4>(few, a, st)
                         : launch_gated_few<M, BWD, 2, 2>(few, a, st);
    const int64_t f = BWD ? a.fp : a.f;   // (the padding is written, too)
    auto go = [&](auto tile) {
        typedef decltype(tile) Tl;
        a.ni = (int)((f + Tl::ROWS / 2 - 1) / (Tl::ROWS / 2));
        a.nt = (int)((a.T + Tl::COLS - 1) / Tl::COLS);
        hipLaunchKernelGGL((k_gated<Tl, BWD>), dim3((unsigned)(a.ni * a.nt)), dim3(Tl::THREADS), 0, st, a);
        return (int64_t)a.ni * a.nt * (Tl::THREADS / 64);
    };
    const int tile = pick_tile(2 * f, a.T, op_cus(), true);
    if (tile == 256) return go(BigTile<M>());
    if (tile == 128 && one_a_cu(128, 2 * f, a.T)) return go(Tile<M, 128, 128, 2, 4, 3>());
    if (tile == 128) return go(Tile<M, 128, 128, 2, 4, 2>());
    return go(Tile<M, 64, 64, 2, 2, 4>());
}

// Padded copies of operands that cannot be staged as they are.
struct PadPlan {
    bool x, w;
    int64_t dp;
    size_t xbytes, wbytes;   // of one copy
};
static PadPlan pad_plan(const void* x, int64_t ldx, const void* wg, const void* wu, int64_t ldw,
                        int64_t T, int64_t d, int64_t f, bool need_x, bool need_w) {
    PadPlan p;
    p.dp = (d + 63) / 64 * 64;
    p.x = need_x && !direct_rows(x, ldx, d);
    p.w = need_w && (!direct_rows(wg, ldw, d) || !direct_rows(wu, ldw, d));
    p.xbytes = p.x ? up256((size_t)T * p.dp * 2) : 0;
    p.wbytes = p.w ? up256((size_t)f * p.dp * 2) : 0;
    return p;
}

// x and the weights as operands of the gated product, through padded copies at `*at`
// where needed.
static void gated_operands(GatedArgs& a, const PadPlan& p, const void* x, int64_t ldx,
                           const void* wg, const void* wu, int64_t ldw, int64_t d, char** at,
                           hipStream_t st) {
    // (a copy's padding is zeros; without copies what lies past d reads as zeros)
    const int64_t kbytes = p.x && p.w ? 2 * p.dp : 2 * ((d + 7) / 8 * 8);
    a.x = operand(x, 2 * ldx, a.T, kbytes);
    a.w = operand(wg, 2 * ldw, a.f, kbytes);
    a.w.base2 = static_cast<const char*>(wu);
    PadArgs c{};
    int n = 0;
    int64_t pieces = 0;
    auto copy = [&](const void* src, int64_t ld, int64_t rows, size_t bytes) {
        char* const to = *at;
        c.src[n] = static_cast<const uint16_t*>(src);
        c.dst[n] = reinterpret_cast<uint16_t*>(to);
        c.ld[n] = ld;
        pieces += rows * (p.dp / 8);
        for (int i = n; i < 3; ++i) c.end[i] = pieces;
        ++n;
        *at += bytes;
        return to;
    };
    if (p.x) a.x = operand(copy(x, ldx, a.T, p.xbytes), 2 * p.dp, a.T, kbytes);
    if (p.w) {
        a.w = operand(copy(wg, ldw, a.f, p.wbytes), 2 * p.dp, a.f, kbytes);
        a.w.base2 = copy(wu, ldw, a.f, p.wbytes);
    }
    if (n > 0) {
        c.cols = d;
        c.cols_p = p.dp;
        hipLaunchKernelGGL(k_pad_rows, stride_grid(pieces), dim3(256), 0, st, c);
    }
    a.chunks = (int)((kbytes + CHUNK_BYTES - 1) / CHUNK_BYTES);
}

// The two products of the backward pass: dx over the features (those of Wg, then those of Wu), dW over
// the tokens.
//
// Both take dG and dU in 16 bits.  Where many tokens, features and outputs count, the errors of
// that average out to as much as the result's own rounding (together 1.4 times one rounding's
// norm).  Where few do they may not (1.6 times), so there the sums go on over the rests that the
// rounding took, in 16 bits, too, and the result is as good as rounded once: for dW with one chunk
// of tokens and few features, or few weights; for dx with one chunk of tokens and few features or
// weights.  16 x 4096 x 1024: 31.5 -> 36.3 us, 1 x 1024 x 1024: 17.9 -> 20.4, 2752 x 65 x 128:
// 21.5 -> 25.7; with more features 1 x 4096 x 11008 would take 147 us instead of 133 for nothing.
struct BackwardPlan {
    int64_t fp, ldg;
    bool rests_x, rests_w;
    ProdPlan dx, dw;
    size_t dgu, partial, top;   // bytes of the workspace; top: half precision, a GradScale before the values
};
static BackwardPlan backward_plan(int64_t T, int64_t d, int64_t f, bool half, bool dx, bool dw, int ncu) {
    BackwardPlan p{};
    p.fp = (f + 63) / 64 * 64;
    p.rests_w = dw && ((T <= 64 && f <= 4096) || d * f <= (1 << 17));
    p.rests_x = dx && T <= 64 && (f <= 1024 || d * f <= (1 << 21));
    p.ldg = (p.rests_w || p.rests_x ? 4 : 2) * p.fp;
    p.dgu = up256((size_t)T * p.ldg * 2);
    if (dx) p.dx = prod_plan(d, T, (int)((p.rests_x ? 4 : 2) * p.fp / 64), ncu);
    if (dw) p.dw = prod_plan(d, 2 * p.fp, (int)((p.rests_w ? 2 : 1) * ((T + 63) / 64)), ncu);
    p.partial = std::max(p.dx.bytes, p.dw.bytes);
    p.top = half ? up256(256 + (size_t)gated_tops(T, p.fp) * sizeof(float)) : 0;
    return p;
}

template <typename M>
static void run_backward(const FewArgs& few, GatedArgs a, const BackwardPlan& p, int64_t d,
                         void* dx, int64_t lddx, void* dw_gate, void* dw_up, int64_t lddw,
                         char* top, void* partial, hipStream_t st) {
    GradScale* const scale = reinterpret_cast<GradScale*>(top);
    a.top = reinterpret_cast<float*>(top + 256);
    const int64_t tops = launch_gated<M, true>(few, a, st);
    if constexpr (narrow_range<typename M::Elem>) {
        hipLaunchKernelGGL(k_grad_scale, dim3(1), dim3(1024), 0, st, a.top, tops, scale);
        a.factor = &scale->factor;
        launch_gated<M, true>(few, a, st);
    }
    const int64_t ldg = 2 * a.ldg;   // in bytes
    const int64_t cols = (d + 7) / 8 * 8;   // (of x and the weights, as they are or padded)
    if (dx) {
        ProdArgs g{};
        g.undo = narrow_range<typename M::Elem> ? &scale->undo : nullptr;
        g.a = operand(a.w.base, a.w.ld, cols, a.f);
        g.a.base2 = a.w.base2;
        g.a.split = (int)(a.fp / 64);
        g.chunks = (p.rests_x ? 4 : 2) * g.a.split;
        g.b = operand(a.dgu, ldg, a.T, (int64_t)g.chunks * CHUNK_BYTES);
        g.d = d;
        g.out = dx;
        g.ldo = lddx;
        g.split = g.split2 = g.end = a.T;
        launch_prod<M, true, false>(g, p.dx, partial, st);
    }
    if (dw_gate) {
        ProdArgs g{};
        g.undo = narrow_range<typename M::Elem> ? &scale->undo : nullptr;
        g.a = operand(a.x.base, a.x.ld, cols, a.T);
        g.b = operand(a.dgu, ldg, 2 * a.fp, a.T);
        g.chunks = (int)((a.T + 63) / 64);
        if (p.rests_w) {   // the same x again, beside the rests
            g.a.split = g.b.split = g.chunks;
            g.a.base2 = g.a.base;
            g.b.base2 = g.b.base + 4 * a.fp;
            g.chunks *= 2;
        }
        g.d = d;
        g.out = dw_gate;
        g.out2 = dw_up;
        g.ldo = lddw;
        g.split = a.f;
        g.split2 = a.fp;
        g.end = a.fp + a.f;
        launch_prod<M, true, true>(g, p.dw, partial, st);
    }
}

}  // namespace bk

static bakron_status mlp_sizes(const char* who, int64_t ldx, int64_t T, int64_t d, int64_t ldw,
                               int64_t f, int32_t dtype, int32_t act) {
    if (T < 0 || T > bk::OP_T_MAX || d < 1 || f < 1 || d > ((int64_t)1 << 17) || f > ((int64_t)1 << 17))
        return bk::op_fail(who, "bad size");
    if (ldx < d || ldw < d) return bk::op_fail(who, "leading dimension below d");
    if (dtype != BAKRON_F16 && dtype != BAKRON_BF16) return bk::op_fail(who, "dtype must be 16-bit");
    if (act != BAKRON_ACT_SILU && act != BAKRON_ACT_GELU) return bk::op_fail(who, "bad act");
    // (the widest launch: 64-row blocks of 256 threads)
    if ((T + 63) / 64 * ((std::max(d, 2 * f) + 31) / 32 + 1) > ((int64_t)1 << 23) - 1)
        return bk::op_fail(who, "too many rows for one call");
    return BAKRON_OK;
}

extern "C" bakron_status bakron_gated_mlp(const void* x, int64_t ldx, int64_t T, int64_t d,
                                          const void* w_gate, const void* w_up, int64_t ldw,
                                          int64_t f, int32_t dtype, int32_t act, void* h,
                                          int64_t ldh, float* feat_up, float* feat_gate, void* work,
                                          size_t* work_bytes, hipStream_t stream) {
    static const char who[] = "bakron_gated_mlp";
    bk::set_last_error("");
    bakron_status st = mlp_sizes(who, ldx, T, d, ldw, f, dtype, act);
    if (st != BAKRON_OK) return st;
    if (h && ldh < f) return bk::op_fail(who, "leading dimension below f");
    const bool many = !bk::gated_few_rows(T, f, d);
    const bk::PadPlan p = bk::pad_plan(x, ldx, w_gate, w_up, ldw, T, d, f, many, many);
    bool query;
    st = bk::op_workspace(who, work, work_bytes, p.xbytes + 2 * p.wbytes, &query);
    if (st != BAKRON_OK || query) return st;
    if (T == 0) return BAKRON_OK;
    if (!x || !w_gate || !w_up || (!h && !feat_up && !feat_gate))
        return bk::op_fail(who, "null pointer");
    bk::GatedArgs a{};
    a.T = T;
    a.f = f;
    a.act = act;
    a.h = h;
    a.ldh = ldh;
    a.feat_up = feat_up;
    a.feat_gate = feat_gate;
    char* at = static_cast<char*>(work);
    bk::gated_operands(a, p, x, ldx, w_gate, w_up, ldw, d, &at, stream);
    const bk::FewArgs few{x, w_gate, w_up, ldx, ldw, (int)d};
    if (dtype == BAKRON_BF16)
        bk::launch_gated<bk::MmaBF16, false>(few, a, stream);
    else
        bk::launch_gated<bk::MmaF16, false>(few, a, stream);
    return bk::op_launched(who);
}

extern "C" bakron_status bakron_gated_mlp_backward(const void* dh, int64_t lddh, const void* x,
                                                   int64_t ldx, int64_t T, int64_t d,
                                                   const void* w_gate, const void* w_up,
                                                   int64_t ldw, int64_t f, int32_t dtype,
                                                   int32_t act, void* dx, int64_t lddx,
                                                   void* dw_gate, void* dw_up, int64_t lddw,
                                                   void* work, size_t* work_bytes,
                                                   hipStream_t stream) {
    static const char who[] = "bakron_gated_mlp_backward";
    bk::set_last_error("");
    bakron_status st = mlp_sizes(who, ldx, T, d, ldw, f, dtype, act);
    if (st != BAKRON_OK) return st;
    if (lddh < f || (dx && lddx < d) || (dw_gate && lddw < d))
        return bk::op_fail(who, "leading dimension too small");
    const bool many = !bk::gated_few_rows(T, f, d);
    const bk::PadPlan p = bk::pad_plan(x, ldx, w_gate, w_up, ldw, T, d, f, many || dw_gate, many || dx);
    const bk::BackwardPlan b =
        bk::backward_plan(std::max<int64_t>(T, 1), d, f, dtype == BAKRON_F16, dx != nullptr, dw_gate != nullptr,
                          bk::op_cus());
    bool query;
    st = bk::op_workspace(who, work, work_bytes, p.xbytes + 2 * p.wbytes + b.dgu + b.top + b.partial, &query);
    if (st != BAKRON_OK || query) return st;
    if (!dw_gate != !dw_up) return bk::op_fail(who, "dw_gate and dw_up go together");
    if (!dx && !dw_gate) return bk::op_fail(who, "null pointer");
    if (T == 0 && !dw_gate) return BAKRON_OK;
    if (T == 0) {
        for (void* w : {dw_gate, dw_up})
            hipLaunchKernelGGL(bk::k_zero_rows, dim3((unsigned)f), dim3(256), 0, stream,
                               static_cast<uint16_t*>(w), lddw, f, d);
        return bk::op_launched(who);
    }
    if (!dh || !x || !w_gate || !w_up) return bk::op_fail(who, "null pointer");
    bk::GatedArgs a{};
    a.T = T;
    a.f = f;
    a.act = act;
    a.dh = dh;
    a.lddh = lddh;
    a.fp = b.fp;
    a.ldg = b.ldg;
    char* at = static_cast<char*>(work);
    bk::gated_operands(a, p, x, ldx, w_gate, w_up, ldw, d, &at, stream);
    a.dgu = at;
    char* const top = at + b.dgu;
    char* const partial = top + b.top;
    const bk::FewArgs few{x, w_gate, w_up, ldx, ldw, (int)d};
    if (dtype == BAKRON_BF16)
        bk::run_backward<bk::MmaBF16>(few, a, b, d, dx, lddx, dw_gate, dw_up, lddw, top, partial, stream);
    else
        bk::run_backward<bk::MmaF16>(few, a, b, d, dx, lddx, dw_gate, dw_up, lddw, top, partial, stream);
    return bk::op_launched(who);
}
