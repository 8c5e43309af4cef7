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
    const char *x, *wg, *wu;       // rows of 16-byte multiples
    int64_t ldx, ldw;              // bytes
    int64_t kbytes;                // d in bytes
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
    void* dgu;                     // T x 2 fp: dG | dU
    void* dgut;                    // 2 fp x Tp: its transpose
    int64_t fp, Tp;
};

template <typename Tl, bool BWD>
__global__ __launch_bounds__(Tl::THREADS) void k_gated(GatedArgs a) {
    typedef typename Tl::Mma::Elem E;
    __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
    int ti, tt;
    tile_of(blockIdx.x, a.ni, a.nt, 8, &ti, &tt);
    const int64_t f0 = (int64_t)ti * (Tl::ROWS / 2), t0 = (int64_t)tt * Tl::COLS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    static_assert(Tl::UA % 2 == 0, "gate and up rows in one wave");

    typename Tl::Accs acc = {};
    auto none = [](int, typename Tl::Accs&) {};
    auto feature = [](int r) { return (int64_t)((r >> 5) * 16 + (r & 15)); };   // of tile row r
    if constexpr (Tl::THREADS == 512) {
        // (the rows that a wave loads are all of one matrix)
        const int w = __builtin_amdgcn_readfirstlane(wave);
        const bool up = (Tl::load_row_a(0, 0, w) >> 4) & 1;
        Tl::run(
            lds, (up ? a.wu : a.wg) + f0 * a.ldw, a.x + t0 * a.ldx,
            [&](int r) { return (uint32_t)(min(feature(r), a.f - 1 - f0) * a.ldw); },
            [&](int r) { return (uint32_t)(min((int64_t)r, a.T - 1 - t0) * a.ldx); }, a.kbytes, a.kbytes,
            a.chunks, acc, none);
    } else {
        Tl::run(
            lds,
            [&](int r) { return ((r >> 4) & 1 ? a.wu : a.wg) + min(f0 + feature(r), a.f - 1) * a.ldw; },
            [&](int r) { return a.x + min(t0 + r, a.T - 1) * a.ldx; }, a.kbytes, a.kbytes, a.chunks, acc,
            none);
    }

#pragma unroll
    for (int y = 0; y < Tl::UB; ++y) {
        const int64_t t = t0 + Tl::b0(wave) + y * 16 + (lane & 15);
#pragma unroll
        for (int x = 0; x < Tl::UA; x += 2) {
            const f32x4 G = Tl::at(acc, x, y), U = Tl::at(acc, x + 1, y);
            const int64_t j = f0 + (Tl::a0(wave) + x * 16) / 2 + (lane >> 4) * 4;
            const int64_t valid = a.f - j;
            if constexpr (!BWD) {
                if (t >= a.T || valid <= 0) continue;
                float h[4], v[4], s[4];
                if (a.feat_gate) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        act_both(G[r], a.act, &v[r], &s[r]);
                        s[r] *= U[r];
                    }
                    store4(a.feat_gate + t * a.f + j, s, valid);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = act_value(G[r], a.act);
                }
                if (a.feat_up) store4(a.feat_up + t * a.f + j, v, valid);
                if (a.h) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) h[r] = v[r] * U[r];
                    store4(static_cast<E*>(a.h) + t * a.ldh + j, h, valid);
                }
            } else {
                // zeros in the padding of both layouts, which the products read
                if (j >= a.fp) continue;
                float dg[4] = {0.0f, 0.0f, 0.0f, 0.0f}, du[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (t < a.T && valid > 0) {
                    float dh[4];
                    load4(static_cast<const E*>(a.dh) + t * a.lddh + j, dh, valid);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v, s;
                        act_both(G[r], a.act, &v, &s);
                        if (r < valid) {
                            dg[r] = dh[r] * U[r] * s;
                            du[r] = dh[r] * v;
                        }
                    }
                }
                if (t < a.T && a.dgu) {
                    E* const row = static_cast<E*>(a.dgu) + t * (2 * a.fp) + j;
                    store4(row, dg, 4);
                    store4(row + a.fp, du, 4);
                }
                if (t < a.Tp && a.dgut) {
                    E* const col = static_cast<E*>(a.dgut) + j * a.Tp + t;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        col[r * a.Tp] = (E)dg[r];
                        col[(a.fp + r) * a.Tp] = (E)du[r];
                    }
                }
            }
        }
    }
}

struct ProdArgs {
    const char *a, *b;             // D[i][t] = sum_k a[i][k] b[t][k]
    int64_t lda, ldb, kbytes;      // bytes
    int64_t ni_rows, nt_rows;
    int chunks, ni, nt;
    void *out, *out2;              // rows t < split of out; from split2 on, of out2
    int64_t ldo, split, split2;
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
    auto none = [](int, typename Tl::Accs&) {};
    if constexpr (Tl::THREADS == 512)
        Tl::run(
            lds, a.a + i0 * a.lda, a.b + t0 * a.ldb,
            [&](int r) { return (uint32_t)(min((int64_t)r, a.ni_rows - 1 - i0) * a.lda); },
            [&](int r) { return (uint32_t)(min((int64_t)r, a.nt_rows - 1 - t0) * a.ldb); }, a.kbytes,
            a.kbytes, a.chunks, acc, none);
    else
        Tl::run(
            lds, [&](int r) { return a.a + min(i0 + r, a.ni_rows - 1) * a.lda; },
            [&](int r) { return a.b + min(t0 + r, a.nt_rows - 1) * a.ldb; }, a.kbytes, a.kbytes,
            a.chunks, acc, none);
#pragma unroll
    for (int y = 0; y < Tl::UB; ++y) {
        const int64_t t = t0 + Tl::b0(wave) + y * 16 + (lane & 15);
        if (t >= a.nt_rows || (t >= a.split && t < a.split2)) continue;
        E* const row = t < a.split ? static_cast<E*>(a.out) + t * a.ldo
                                   : static_cast<E*>(a.out2) + (t - a.split2) * a.ldo;
#pragma unroll
        for (int x = 0; x < Tl::UA; ++x) {
            const int64_t i = i0 + Tl::a0(wave) + x * 16 + (lane >> 4) * 4;
            float v[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = Tl::at(acc, x, y)[r];
            if (i < a.ni_rows) store4(row + i, v, a.ni_rows - i);
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

// dst[c][r] = src[r][c] for r < rows, 0 for rows <= r < rows_p; 16-bit entries, one
// 64 x 64 block a workgroup.
__global__ __launch_bounds__(256) void k_transpose(const uint16_t* __restrict__ src, int64_t ld,
                                                   int64_t rows, int64_t cols, int64_t rows_p,
                                                   uint16_t* __restrict__ dst, int64_t ldd) {
    __shared__ uint16_t s[64][66];
    const int64_t nb = (cols + 63) / 64;
    const int64_t r0 = (int64_t)blockIdx.x / nb * 64, c0 = (int64_t)blockIdx.x % nb * 64;
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int64_t r = r0 + k * 4 + y, c = c0 + x;
        s[k * 4 + y][x] = r < rows && c < cols ? src[r * ld + c] : (uint16_t)0;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int64_t c = c0 + k * 4 + y, r = r0 + x;
        if (c < cols && r < rows_p) dst[c * ldd + r] = s[x][k * 4 + y];
    }
}

__global__ __launch_bounds__(256) void k_zero_rows(uint16_t* p, int64_t ld, int64_t rows, int64_t cols) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < cols; c += 256) p[r * ld + c] = 0;
}

static inline int64_t up64(int64_t v) { return (v + 63) / 64 * 64; }
static inline size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }
static inline dim3 grid256(int64_t n) { return dim3((unsigned)((n + 255) / 256)); }

// Whether rows can be staged as they are: 16-byte pieces at 16-byte addresses.
static bool direct_rows(const void* p, int64_t ld, int64_t cols) {
    return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && cols % 8 == 0;
}

template <typename M, bool BWD>
static void launch_gated(GatedArgs a, hipStream_t st) {
    auto tiles = [&](int64_t b) { return ((a.f + b / 2 - 1) / (b / 2)) * ((a.T + b - 1) / b); };
    const int ncu = op_cus();
    auto go = [&](auto tile) {
        typedef decltype(tile) Tl;
        a.ni = (int)((a.f + Tl::ROWS / 2 - 1) / (Tl::ROWS / 2));
        a.nt = (int)((a.T + Tl::COLS - 1) / Tl::COLS);
        hipLaunchKernelGGL((k_gated<Tl, BWD>), dim3((unsigned)(a.ni * a.nt)), dim3(Tl::THREADS), 0, st, a);
    };
    if (tiles(256) >= ncu && std::max(a.ldx, a.ldw) < TILE_LD_MAX)
        go(BigTile<M>());
    else if (tiles(128) >= ncu)
        go(Tile<M, 128, 128, 2, 2>());
    else
        go(Tile<M, 64, 64, 2, 2>());
}

template <typename M>
static void launch_prod(ProdArgs a, hipStream_t st) {
    auto tiles = [&](int64_t b) { return ((a.ni_rows + b - 1) / b) * ((a.nt_rows + b - 1) / b); };
    const int ncu = op_cus();
    auto go = [&](auto tile) {
        typedef decltype(tile) Tl;
        a.ni = (int)((a.ni_rows + Tl::ROWS - 1) / Tl::ROWS);
        a.nt = (int)((a.nt_rows + Tl::COLS - 1) / Tl::COLS);
        hipLaunchKernelGGL((k_prod<Tl>), dim3((unsigned)(a.ni * a.nt)), dim3(Tl::THREADS), 0, st, a);
    };
    if (tiles(256) >= ncu && std::max(a.lda, a.ldb) < TILE_LD_MAX)
        go(BigTile<M>());
    else if (tiles(128) >= ncu)
        go(Tile<M, 128, 128, 2, 2>());
    else
        go(Tile<M, 64, 64, 2, 2>());
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
    p.dp = up64(d);
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
static void transpose(const void* src, int64_t ld, int64_t rows, int64_t cols, int64_t rows_p,
                      void* dst, int64_t ldd, hipStream_t st) {
    hipLaunchKernelGGL(k_transpose, dim3((unsigned)((rows_p + 63) / 64 * ((cols + 63) / 64))),
                       dim3(256), 0, st, static_cast<const uint16_t*>(src), ld, rows, cols, rows_p,
                       static_cast<uint16_t*>(dst), ldd);
}

// Puts x and the weights into `a`, through padded copies at `*at` where needed.
static void gated_operands(GatedArgs& a, const PadPlan& p, const void* x, int64_t ldx,
                           const void* wg, const void* wu, int64_t ldw, int64_t d, char** at,
                           hipStream_t st) {
    a.x = static_cast<const char*>(x);
    a.ldx = 2 * ldx;
    if (p.x) {
        pad_copy(x, ldx, a.T, d, p.dp, *at, st);
        a.x = *at;
        a.ldx = 2 * p.dp;
        *at += p.xbytes;
    }
    a.wg = static_cast<const char*>(wg);
    a.wu = static_cast<const char*>(wu);
    a.ldw = 2 * ldw;
    if (p.w) {
        pad_copy(wg, ldw, a.f, d, p.dp, *at, st);
        pad_copy(wu, ldw, a.f, d, p.dp, *at + p.wbytes, st);
        a.wg = *at;
        a.wu = *at + p.wbytes;
        a.ldw = 2 * p.dp;
        *at += 2 * p.wbytes;
    }
    // (a copy's padding is zeros; without copies the pieces past d are)
    a.kbytes = p.x && p.w ? 2 * p.dp : 2 * ((d + 7) / 8 * 8);
    a.chunks = (int)((a.kbytes + CHUNK_BYTES - 1) / CHUNK_BYTES);
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
    // (every tile of the gated product covers the padding it has to clear)
    const int64_t fp = (f + 31) / 32 * 32, Tp = bk::up64(T);
    const size_t dgu = bk::up256((size_t)T * 2 * fp * 2), dgut = bk::up256((size_t)Tp * 2 * fp * 2);
    const size_t wt = bk::up256((size_t)d * 2 * fp * 2), xt = bk::up256((size_t)d * Tp * 2);
    bool query;
    st = bk::op_workspace(who, work, work_bytes, p.xbytes + 2 * p.wbytes + dgu + dgut + wt + xt, &query);
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
    a.Tp = Tp;
    char* at = static_cast<char*>(work);
    bk::gated_operands(a, p, x, ldx, w_gate, w_up, ldw, d, &at, stream);
    char* const dgu_at = at;
    char* const dgut_at = dgu_at + dgu;
    char* const wt_at = dgut_at + dgut;
    char* const xt_at = wt_at + wt;
    a.dgu = dx ? dgu_at : nullptr;
    a.dgut = dw_gate ? dgut_at : nullptr;
    const bool bf16 = dtype == BAKRON_BF16;
    bf16 ? bk::launch_gated<bk::MmaBF16, true>(a, stream) : bk::launch_gated<bk::MmaF16, true>(a, stream);
    if (dx) {
        bk::transpose(w_gate, ldw, f, d, fp, wt_at, 2 * fp, stream);
        bk::transpose(w_up, ldw, f, d, fp, wt_at + 2 * fp, 2 * fp, stream);
        bk::ProdArgs g{};
        g.a = wt_at;
        g.b = dgu_at;
        g.lda = g.ldb = 4 * fp;
        g.kbytes = 4 * fp;
        g.ni_rows = d;
        g.nt_rows = T;
        g.chunks = (int)(g.kbytes / bk::CHUNK_BYTES);
        g.out = dx;
        g.ldo = lddx;
        g.split = T;
        g.split2 = T;
        bf16 ? bk::launch_prod<bk::MmaBF16>(g, stream) : bk::launch_prod<bk::MmaF16>(g, stream);
    }
    if (dw_gate) {
        bk::transpose(x, ldx, T, d, Tp, xt_at, Tp, stream);
        bk::ProdArgs g{};
        g.a = xt_at;
        g.b = dgut_at;
        g.lda = g.ldb = 2 * Tp;
        g.kbytes = 2 * Tp;
        g.ni_rows = d;
        g.nt_rows = fp + f;   // (the rest of dU^T is padding)
        g.chunks = (int)(g.kbytes / bk::CHUNK_BYTES);
        g.out = dw_gate;
        g.out2 = dw_up;
        g.ldo = lddw;
        g.split = f;
        g.split2 = fp;
        bf16 ? bk::launch_prod<bk::MmaBF16>(g, stream) : bk::launch_prod<bk::MmaF16>(g, stream);
    }
    return bk::op_launched(who);
}
