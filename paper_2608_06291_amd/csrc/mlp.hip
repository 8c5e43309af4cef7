// The hidden layer of a gated MLP and its gradients (16-bit floats, fp32 sums):
//   G = x Wg^T,  U = x Wu^T,  h = act(G) (.) U
//   dG = dh (.) U (.) act'(G),  dU = dh (.) act(G)
//   dx = dG Wg + dU Wu,  dWg = dG^T x,  dWu = dU^T x
// One tile product serves them all.  Rows of Wg and Wu are taken 16 by 16 in turn, so
// that the same lane ends with G and U of the same entries and the activation and the
// product happen on its registers.  The gradients come from the same product, with dG and
// dU (rounded to 16 bits, as operands of the products that follow) in its epilogue.
#include "tile.h"

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
    void* dgu;                     // T x 2 fp: dG | dU, zeros in the padding of each
    int64_t fp;
};

template <typename Tl, bool BWD>
__global__ __launch_bounds__(Tl::THREADS) void k_gated(GatedArgs a) {
    typedef typename Tl::Mma::Elem E;
    __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
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
    Tl::run(lds, w, first, a.x, t0, a.chunks, acc, feature);

    const auto rows =
        handover<Tl>(lds, wave, lane, [&](int x, int y) { return Tl::at(acc, x, y); });
    constexpr int PER = Tl::UA;   // lanes a row: 8 features each
    const int p = lane % PER;
    const int64_t j = f0 + Tl::a0(wave) / 2 + p * 8, valid = a.f - j;
#pragma unroll
    for (int y = 0; y < Tl::UB; ++y) {
        rows.put(y);
        const int tl = lane / PER;
        const int64_t t = t0 + Tl::b0(wave) + y * 16 + tl;
        if (tl >= 16) continue;
        float G[8], U[8];
        rows.take(tl, (p >> 1) * 4 + (p & 1), G);
        rows.take(tl, (p >> 1) * 4 + (p & 1) + 2, U);
        if (t >= a.T) continue;
        if constexpr (!BWD) {
            if (valid <= 0) continue;
            float v[8], s[8];
            if (a.feat_gate) {
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    act_both(G[r], a.act, &v[r], &s[r]);
                    s[r] *= U[r];
                }
                store_n(a.feat_gate + t * a.f + j, s, valid);
            } else {
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] = act_value(G[r], a.act);
            }
            if (a.feat_up) store_n(a.feat_up + t * a.f + j, v, valid);
            if (a.h) {
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] *= U[r];
                store_n(static_cast<E*>(a.h) + t * a.ldh + j, v, valid);
            }
        } else {
            if (j >= a.fp) continue;
            float dh[8] = {}, dg[8], du[8];
            if (valid > 0) load_n(static_cast<const E*>(a.dh) + t * a.lddh + j, dh, valid);
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                float v, s;
                act_both(G[r], a.act, &v, &s);
                dg[r] = r < valid ? dh[r] * U[r] * s : 0.0f;   // (0 in the padding, whatever G is)
                du[r] = r < valid ? dh[r] * v : 0.0f;
            }
            E* const row = static_cast<E*>(a.dgu) + t * (2 * a.fp) + j;
            store_n(row, dg, 8);
            store_n(row + a.fp, du, 8);
        }
    }
}

struct ProdArgs {
    Operand a, b;                  // D[i][t] = sum_k a[i][k] b[t][k]
    int chunks, ni, nt;
    int64_t d;                     // columns of the output
    void *out, *out2;              // rows t < split of out; split2 <= t < end, of out2
    int64_t ldo, split, split2, end;
};

template <typename Tl>
__global__ __launch_bounds__(Tl::THREADS) void k_prod(ProdArgs a) {
    typedef typename Tl::Mma::Elem E;
    __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
    int ti, tt;
    tile_of(blockIdx.x, a.ni, a.nt, 8, &ti, &tt);
    const int64_t i0 = (int64_t)ti * Tl::ROWS, t0 = (int64_t)tt * Tl::COLS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

    typename Tl::Accs acc = {};
    Tl::run(lds, a.a, i0, a.b, t0, a.chunks, acc, [](int r) { return r; });

    const auto rows =
        handover<Tl>(lds, wave, lane, [&](int x, int y) { return Tl::at(acc, x, y); });
    constexpr int PER = Tl::UA * 2;   // lanes a row
    const int p = lane % PER;
    const int64_t i = i0 + Tl::a0(wave) + p * 8;
#pragma unroll
    for (int y = 0; y < Tl::UB; ++y) {
        rows.put(y);
#pragma unroll
        for (int tl = lane / PER; tl < 16; tl += 64 / PER) {
            const int64_t t = t0 + Tl::b0(wave) + y * 16 + tl;
            float v[8];
            rows.take(tl, p, v);
            if (i >= a.d || t >= a.end || (t >= a.split && t < a.split2)) continue;
            E* const row = t < a.split ? static_cast<E*>(a.out) + t * a.ldo
                                       : static_cast<E*>(a.out2) + (t - a.split2) * a.ldo;
            store_n(row + i, v, a.d - i);
        }
    }
}

// dst[r][0 .. cols_p) = src[r][0 .. cols), zeros behind; 16-bit entries.
__global__ __launch_bounds__(256) void k_pad_rows(const uint16_t* __restrict__ src, int64_t ld,
                                                  int64_t rows, int64_t cols, int64_t cols_p,
                                                  uint16_t* __restrict__ dst) {
    const int64_t per = cols_p / 8, e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= rows * per) return;
    const int64_t r = e / per, c = e % per * 8;
    Pack<uint16_t, 8> v;
    if (c + 8 <= cols) {
        v = load_pack<uint16_t, 8>(src + r * ld + c);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v.v[j] = c + j < cols ? src[r * ld + c + j] : (uint16_t)0;
    }
    store_pack(dst + e * 8, v);
}

__global__ __launch_bounds__(256) void k_zero_rows(uint16_t* p, int64_t ld, int64_t rows, int64_t cols) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < cols; c += 256) p[r * ld + c] = 0;
}

static inline size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }
static inline dim3 grid256(int64_t n) { return dim3((unsigned)((n + 255) / 256)); }

// Whether rows can be staged as they are: 16-byte pieces at 16-byte addresses.
static bool direct_rows(const void* p, int64_t ld, int64_t cols) {
    return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && cols % 8 == 0 && 2 * ld < TILE_LD_MAX;
}

template <typename M, bool BWD>
static void launch_gated(GatedArgs a, hipStream_t st) {
    const int64_t f = BWD ? a.fp : a.f;   // (the padding is written, too)
    auto tiles = [&](int64_t b) { return ((f + b / 2 - 1) / (b / 2)) * ((a.T + b - 1) / b); };
    const int ncu = op_cus();
    auto go = [&](auto tile) {
        typedef decltype(tile) Tl;
        a.ni = (int)((f + Tl::ROWS / 2 - 1) / (Tl::ROWS / 2));
        a.nt = (int)((a.T + Tl::COLS - 1) / Tl::COLS);
        hipLaunchKernelGGL((k_gated<Tl, BWD>), dim3((unsigned)(a.ni * a.nt)), dim3(Tl::THREADS), 0, st, a);
    };
    if (tiles(256) >= ncu)
        go(BigTile<M>());
    else if (tiles(128) >= ncu)
        go(Tile<M, 128, 128, 2, 2, 2>());
    else
        go(Tile<M, 64, 64, 2, 2, 4>());
}

template <typename M, bool ACOLS, bool BCOLS>
static void launch_prod(ProdArgs a, hipStream_t st) {
    auto tiles = [&](int64_t b) { return ((a.a.n + b - 1) / b) * ((a.b.n + b - 1) / b); };
    const int ncu = op_cus();
    auto go = [&](auto tile) {
        typedef decltype(tile) Tl;
        a.ni = (int)((a.a.n + Tl::ROWS - 1) / Tl::ROWS);
        a.nt = (int)((a.b.n + Tl::COLS - 1) / Tl::COLS);
        hipLaunchKernelGGL((k_prod<Tl>), dim3((unsigned)(a.ni * a.nt)), dim3(Tl::THREADS), 0, st, a);
    };
    if (tiles(256) >= ncu)
        go(BigTile<M, ACOLS, BCOLS>());
    else if (tiles(128) >= ncu)
        go(Tile<M, 128, 128, 2, 2, 2, ACOLS, BCOLS>());
    else
        go(Tile<M, 64, 64, 2, 2, 4, ACOLS, BCOLS>());
}

// Padded copies of operands that cannot be staged as they are.
struct PadPlan {
    bool x, w;
    int64_t dp;
    size_t xbytes, wbytes;   // of one copy
};
static PadPlan pad_plan(const void* x, int64_t ldx, const void* wg, const void* wu, int64_t ldw,
                        int64_t T, int64_t d, int64_t f) {
    PadPlan p;
    p.dp = (d + 63) / 64 * 64;
    p.x = !direct_rows(x, ldx, d);
    p.w = !direct_rows(wg, ldw, d) || !direct_rows(wu, ldw, d);
    p.xbytes = p.x ? up256((size_t)T * p.dp * 2) : 0;
    p.wbytes = p.w ? up256((size_t)f * p.dp * 2) : 0;
    return p;
}

static void pad_copy(const void* src, int64_t ld, int64_t rows, int64_t cols, int64_t cols_p,
                     void* dst, hipStream_t st) {
    hipLaunchKernelGGL(k_pad_rows, grid256(rows * (cols_p / 8)), dim3(256), 0, st,
                       static_cast<const uint16_t*>(src), ld, rows, cols, cols_p,
                       static_cast<uint16_t*>(dst));
}

// x and the weights as operands of the gated product, through padded copies at `*at`
// where needed.
static void gated_operands(GatedArgs& a, const PadPlan& p, const void* x, int64_t ldx,
                           const void* wg, const void* wu, int64_t ldw, int64_t d, char** at,
                           hipStream_t st) {
    // (a copy's padding is zeros; without copies what lies past d reads as zeros)
    const int64_t kbytes = p.x && p.w ? 2 * p.dp : 2 * ((d + 7) / 8 * 8);
    a.x = operand(x, 2 * ldx, a.T, kbytes);
    if (p.x) {
        pad_copy(x, ldx, a.T, d, p.dp, *at, st);
        a.x = operand(*at, 2 * p.dp, a.T, kbytes);
        *at += p.xbytes;
    }
    a.w = operand(wg, 2 * ldw, a.f, kbytes);
    a.w.base2 = static_cast<const char*>(wu);
    if (p.w) {
        pad_copy(wg, ldw, a.f, d, p.dp, *at, st);
        pad_copy(wu, ldw, a.f, d, p.dp, *at + p.wbytes, st);
        a.w = operand(*at, 2 * p.dp, a.f, kbytes);
        a.w.base2 = *at + p.wbytes;
        *at += 2 * p.wbytes;
    }
    a.chunks = (int)((kbytes + CHUNK_BYTES - 1) / CHUNK_BYTES);
}

template <typename M>
static void run_backward(const GatedArgs& a, int64_t d, void* dx, int64_t lddx, void* dw_gate,
                         void* dw_up, int64_t lddw, hipStream_t st) {
    launch_gated<M, true>(a, st);
    const int64_t ldg = 4 * a.fp;
    const int64_t cols = (d + 7) / 8 * 8;   // (of x and the weights, as they are or padded)
    if (dx) {   // over the features: those of Wg, then those of Wu
        ProdArgs g{};
        g.a = operand(a.w.base, a.w.ld, cols, a.f);
        g.a.base2 = a.w.base2;
        g.a.split = (int)(a.fp / 64);
        g.b = operand(a.dgu, ldg, a.T, ldg);
        g.chunks = 2 * g.a.split;
        g.out = dx;
        g.ldo = lddx;
        g.split = g.split2 = g.end = a.T;
        g.d = d;
        launch_prod<M, true, false>(g, st);
    }
    if (dw_gate) {   // over the tokens
        ProdArgs g{};
        g.a = operand(a.x.base, a.x.ld, cols, a.T);
        g.b = operand(a.dgu, ldg, 2 * a.fp, a.T);
        g.chunks = (int)((a.T + 63) / 64);
        g.out = dw_gate;
        g.out2 = dw_up;
        g.ldo = lddw;
        g.split = a.f;
        g.split2 = a.fp;
        g.end = a.fp + a.f;
        g.d = d;
        launch_prod<M, true, true>(g, st);
    }
}

}  // namespace bk

static bakron_status mlp_sizes(const char* who, int64_t ldx, int64_t T, int64_t d, int64_t ldw,
                               int64_t f, int32_t dtype, int32_t act) {
    if (T < 0 || d < 1 || f < 1 || d > ((int64_t)1 << 17) || f > ((int64_t)1 << 17))
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
    const bk::PadPlan p = bk::pad_plan(x, ldx, w_gate, w_up, ldw, T, d, f);
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
    if (dtype == BAKRON_BF16)
        bk::launch_gated<bk::MmaBF16, false>(a, stream);
    else
        bk::launch_gated<bk::MmaF16, false>(a, stream);
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
    const bk::PadPlan p = bk::pad_plan(x, ldx, w_gate, w_up, ldw, T, d, f);
    const int64_t fp = (f + 63) / 64 * 64;
    const size_t dgu = bk::up256((size_t)T * 2 * fp * 2);
    bool query;
    st = bk::op_workspace(who, work, work_bytes, p.xbytes + 2 * p.wbytes + dgu, &query);
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
    a.fp = fp;
    char* at = static_cast<char*>(work);
    bk::gated_operands(a, p, x, ldx, w_gate, w_up, ldw, d, &at, stream);
    a.dgu = at;
    dtype == BAKRON_BF16 ? bk::run_backward<bk::MmaBF16>(a, d, dx, lddx, dw_gate, dw_up, lddw, stream)
                         : bk::run_backward<bk::MmaF16>(a, d, dx, lddx, dw_gate, dw_up, lddw, stream);
    return bk::op_launched(who);
}
