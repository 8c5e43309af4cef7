// What the operators that multiply rows with 16-bit weights share: products of two operands as they
// lie in memory, cut along the summed axis where tiles are few, padded copies of rows that cannot
// be staged, and pieces of rows at any alignment.
#pragma once
#include "tile.h"

namespace bk {

template <typename E>
constexpr bool narrow_range = std::is_same<E, f16_t>::value;

// 8 entries of a row on their way.  SHIFT: rows of an odd number of entries, every other of them 2 bytes
// off a word.  16-byte reads there are several times slower, so a lane reads the words around
// its piece and shifts; the caller makes sure that those words hold an entry of the matrix.
template <bool SHIFT>
struct FewPiece {
    u32x4 w;
    uint32_t next;
    template <typename E>
    __device__ inline void load(const E* p) {
        if constexpr (SHIFT) {
            const uintptr_t at = (uintptr_t)p & ~(uintptr_t)3;
            __builtin_memcpy(&w, (const void*)at, 16);
            __builtin_memcpy(&next, (const void*)(at + ((uintptr_t)p & 2 ? 16 : 12)), 4);
        } else {
            w = load_words(p);
        }
    }
    // `row`: any address of the same row's parity
    template <typename E>
    __device__ inline u32x4 get(const E* row) const {
        if constexpr (SHIFT) {
            if ((uintptr_t)row & 2)
                return u32x4{__builtin_amdgcn_alignbit(w[1], w[0], 16), __builtin_amdgcn_alignbit(w[2], w[1], 16),
                             __builtin_amdgcn_alignbit(w[3], w[2], 16), __builtin_amdgcn_alignbit(next, w[3], 16)};
        }
        return w;
    }
};

// The last `left` < 32 entries (of a lane's eight) of a row of d: 8 entries from p on, zeros past the row; the
// row's last 8 entries moved down where it has as many.
template <typename E>
__device__ inline u32x4 few_part(const E* p, int left, int d) {
    u32x4 r = u32x4(0);
    if (left >= 8) {
        r = load_words(p);
    } else if (left > 0 && d >= 8) {
        unsigned __int128 v;
        const u32x4 last = load_words(p + left - 8);
        __builtin_memcpy(&v, &last, 16);
        v >>= 16 * (8 - left);
        __builtin_memcpy(&r, &v, 16);
    } else if (left > 0) {
        uint16_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < left ? __builtin_bit_cast(uint16_t, p[e]) : (uint16_t)0;
        __builtin_memcpy(&r, v, 16);
    }
    return r;
}

struct ProdArgs {
    Operand a, b;                  // D[i][t] = sum_k a[i][k] b[t][k]
    int chunks, ni, nt;
    int64_t d;                     // columns of the output
    void *out, *out2;              // rows t < split of out; split2 <= t < end, of out2
    int64_t ldo, split, split2, end;
    int parts, part_chunks;        // the summed axis in parts of so many chunks
    float* partial;                // parts x end x dp, where there are several
    int64_t dp;
    const float* undo;             // the outputs are taken times this, or NULL
    // ACC: a product of several calls.  The sums stay in fp32 (end x dp) between them; the last call stores.
    float* sums;
    bool first, last;
};

// PAST: whole vectors are stored past the caches.
template <typename E, bool ACC, bool PAST = false>
__device__ inline void prod_store(const ProdArgs& a, int64_t t, int64_t i, float undo, float (&v)[8]) {
    if (t >= a.end || (t >= a.split && t < a.split2)) return;
    if constexpr (ACC) {
        float* const sum = a.sums + t * a.dp + i;
        if (!a.first) {
            const auto x = load_pack<float, 8>(sum);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += x.v[j];
        }
        if (!a.last) return store_n(sum, v, 8);
    }
    if constexpr (narrow_range<E>) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= undo;
    }
    E* const row = t < a.split ? static_cast<E*>(a.out) + t * a.ldo
                               : static_cast<E*>(a.out2) + (t - a.split2) * a.ldo;
    if (PAST && a.d - i >= 8) {
        Pack<E, 8> o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o.v[j] = (E)v[j];
        u32x4 u;
        __builtin_memcpy(&u, &o, 16);
        store_words_past(row + i, u);
    } else {
        store_n(row + i, v, a.d - i);
    }
}

// Workgroup `block` of a product.
template <typename Tl, bool ACC, bool PAST>
__device__ inline void prod_tile(const ProdArgs& a, int block, char* lds) {
    typedef typename Tl::Mma::Elem E;
    int ti, tt, part = 0, chunks = a.chunks;
    if (a.parts > 1) {
        part = block % (uint32_t)a.parts;
        tile_of(block / (uint32_t)a.parts, a.ni, a.nt, 8, &ti, &tt);
        chunks = min(a.part_chunks, a.chunks - part * a.part_chunks);
    } else {
        tile_of(block, a.ni, a.nt, 8, &ti, &tt);
    }
    const int64_t i0 = (int64_t)ti * Tl::ROWS, t0 = (int64_t)tt * Tl::COLS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

    typename Tl::Accs acc = {};
    Tl::run(lds, a.a, i0, a.b, t0, part * a.part_chunks, chunks, acc, [](int r) { return r; });

    const auto rows =
        handover<Tl>(lds, wave, lane, [&](int x, int y) { return Tl::at(acc, x, y); });
    constexpr int PER = Tl::UA * 2;   // lanes a row
    const float undo = narrow_range<E> && a.undo ? *a.undo : 1.0f;
    const int p = lane % PER;
    const int64_t i = i0 + Tl::a0(wave) + p * 8;
#pragma unroll
    for (int y = 0; y < Tl::UB; ++y) {
        rows.put(y);
#pragma unroll
        for (int k = 0; k < 16 * PER / 64; ++k) {
            const int tl = k * (64 / PER) + lane / PER;
            const int64_t t = t0 + Tl::b0(wave) + y * 16 + tl;
            float v[8];
            rows.take(tl, p, v);
            if (i < a.d && t < a.end) {
                if (a.parts > 1)
                    store_n(a.partial + (part * a.end + t) * a.dp + i, v, 8);
                else
                    prod_store<E, ACC, PAST>(a, t, i, undo, v);
            }
        }
    }
}

template <typename Tl, bool ACC, bool PAST>
__global__ __launch_bounds__(Tl::THREADS) void k_prod(ProdArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
    prod_tile<Tl, ACC, PAST>(a, (int)blockIdx.x, lds);
}
// Two products in one launch: the first `first` workgroups are the one's.
template <typename Ta, typename Tb>
__global__ __launch_bounds__(Ta::THREADS) void k_prod_two(ProdArgs a, ProdArgs b, int first) {
    static_assert(Ta::THREADS == Tb::THREADS && Ta::LDS == Tb::LDS, "tiles of one size");
    __shared__ __attribute__((aligned(1024))) char lds[Ta::LDS];
    if ((int)blockIdx.x < first)
        prod_tile<Ta, false, false>(a, (int)blockIdx.x, lds);
    else
        prod_tile<Tb, false, false>(b, (int)blockIdx.x - first, lds);
}

// Sums the parts, in their order.
template <typename E, bool ACC>
__global__ __launch_bounds__(256) void k_prod_join(ProdArgs a) {
    const int64_t per = a.dp / 8, e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e >= a.end * per) return;
    const int64_t t = e / per, i = e % per * 8;
    if (i >= a.d) return;
    float v[8] = {};
    for (int p = 0; p < a.parts; ++p) {
        const auto x = load_pack<float, 8>(a.partial + (p * a.end + t) * a.dp + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += x.v[j];
    }
    prod_store<E, ACC>(a, t, i, narrow_range<E> && a.undo ? *a.undo : 1.0f, v);
}

// Up to three matrices of the same width copied into rows of cols_p, zeros behind;
// 16-bit entries.
struct PadArgs {
    const uint16_t* src[3];
    uint16_t* dst[3];
    int64_t ld[3], end[3];   // end: 8-entry pieces up to and with this one
    int64_t cols, cols_p;
};
static __global__ __launch_bounds__(256) void k_pad_rows(PadArgs a) {
    const int64_t per = a.cols_p / 8;
    for (int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x; n < a.end[2]; n += (int64_t)gridDim.x * 256) {
        const int i = n < a.end[0] ? 0 : n < a.end[1] ? 1 : 2;
        const int64_t e = n - (i == 0 ? 0 : i == 1 ? a.end[0] : a.end[1]), r = e / per, c = e % per * 8;
        const uint16_t* const src = i == 0 ? a.src[0] : i == 1 ? a.src[1] : a.src[2];
        uint16_t* const dst = i == 0 ? a.dst[0] : i == 1 ? a.dst[1] : a.dst[2];
        const uint16_t* const row = src + r * (i == 0 ? a.ld[0] : i == 1 ? a.ld[1] : a.ld[2]);
        Pack<uint16_t, 8> v;
        if (c + 8 <= a.cols) {
            v = load_pack<uint16_t, 8>(row + c);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v.v[j] = c + j < a.cols ? row[c + j] : (uint16_t)0;
        }
        store_pack(dst + e * 8, v);
    }
}

static __global__ __launch_bounds__(256) void k_zero_rows(uint16_t* p, int64_t ld, int64_t rows, int64_t cols) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < cols; c += 256) p[r * ld + c] = 0;
}

static inline size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }
static inline dim3 grid256(int64_t n) { return dim3((unsigned)((n + 255) / 256)); }

// Whether rows can be staged as they are: 16-byte pieces at 16-byte addresses.
static bool direct_rows(const void* p, int64_t ld, int64_t cols) {
    return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && cols % 8 == 0 && 2 * ld < TILE_LD_MAX;
}

// How a product is cut: tile edge, and parts of the summed axis (of 4 chunks at least),
// by the least time: 1.55 us for a chunk's round of 256 x 256, the partial sums written and read
// at 4 TB/s, 4 us for the launch that joins them.
struct ProdPlan {
    int tile, parts, part_chunks;
    size_t bytes;   // of the partial sums
    double us;
};
static ProdPlan prod_plan(int64_t i, int64_t t, int chunks, int ncu) {
    ProdPlan best{64, 1, chunks, 0, 0.0};
    double least = 1e30;
    for (int tile : {256, 128, 64}) {
        const int64_t tiles = ((i + tile - 1) / tile) * ((t + tile - 1) / tile);
        for (int parts = 1; parts <= 32 && (parts == 1 || chunks / parts >= 4); ++parts) {
            const int each = (chunks + parts - 1) / parts, n = (chunks + each - 1) / each;
            if (n != parts) continue;
            const double us = tile_rounds(tile, tiles * n, ncu) * (each * 1.55 + 6.0) +
                              (n > 1 ? 8.0 * n * i * t / 4e6 + 4.0 : 0.0);
            if (us < least) {
                least = us;
                best = ProdPlan{tile, n, each, 0, us};
            }
        }
    }
    if (best.parts > 1)
        best.bytes = up256((size_t)best.parts * t * ((i + 7) / 8 * 8) * sizeof(float));
    return best;
}

// Both of two products that need not wait for each other in one launch, by the same model: one launch (4 us) less,
// and CUs that the one leaves idle go to the other.  Tiles of 128 or 64, the same for both.
struct TwoPlans {
    ProdPlan a, b;
    double us;
};
static TwoPlans two_plans(int64_t ia, int64_t ta, int chunks_a, int64_t ib, int64_t tb, int chunks_b, int ncu) {
    TwoPlans best{};
    best.us = 1e30;
    auto tiles = [](int64_t i, int64_t t, int tile) { return ((i + tile - 1) / tile) * ((t + tile - 1) / tile); };
    auto join = [](int n, int64_t i, int64_t t) { return n > 1 ? 8.0 * n * i * t / 4e6 + 4.0 : 0.0; };
    auto cut = [](int chunks, int parts, int* each) {   // whether the parts come out as so many
        *each = (chunks + parts - 1) / parts;
        return (parts == 1 || chunks / parts >= 4) && (chunks + *each - 1) / *each == parts;
    };
    for (int tile : {128, 64}) {
        const int64_t na = tiles(ia, ta, tile), nb = tiles(ib, tb, tile);
        for (int pa = 1, ea; pa <= 32; ++pa) {
            if (!cut(chunks_a, pa, &ea)) continue;
            for (int pb = 1, eb; pb <= 32; ++pb) {
                if (!cut(chunks_b, pb, &eb)) continue;
                const int64_t n = na * pa + nb * pb;
                // as long as all of them take, and as the longest does (those of a come first)
                const double mean = (double)(na * chunks_a + nb * chunks_b) / n;
                const double all = tile_rounds(tile, n, ncu) * (mean * 1.55 + 6.0);
                const double longest = tile_rounds(tile, std::min<int64_t>(n, 2 * ncu), ncu) * (std::max(ea, eb) * 1.55 + 6.0);
                const double us = std::max(all, longest) + join(pa, ia, ta) + join(pb, ib, tb);
                if (us < best.us) best = TwoPlans{{tile, pa, ea, 0, 0.0}, {tile, pb, eb, 0, 0.0}, us};
            }
        }
    }
    auto bytes = [](const ProdPlan& p, int64_t i, int64_t t) {
        return p.parts > 1 ? up256((size_t)p.parts * t * ((i + 7) / 8 * 8) * sizeof(float)) : 0;
    };
    best.a.bytes = bytes(best.a, ia, ta);
    best.b.bytes = bytes(best.b, ib, tb);
    return best;
}
// a by columns of its first operand, b by columns of both.
template <typename M>
static void launch_two(ProdArgs a, ProdArgs b, const ProdPlan& pa, const ProdPlan& pb, char* partial, hipStream_t st) {
    auto set = [](ProdArgs& g, const ProdPlan& q, char* partial) {
        g.parts = q.parts;
        g.part_chunks = q.part_chunks;
        g.partial = reinterpret_cast<float*>(partial);
        g.dp = (g.d + 7) / 8 * 8;
        g.ni = (int)((g.a.n + q.tile - 1) / q.tile);
        g.nt = (int)((g.b.n + q.tile - 1) / q.tile);
    };
    set(a, pa, partial);
    set(b, pb, partial + pa.bytes);
    const int first = a.ni * a.nt * a.parts, n = first + b.ni * b.nt * b.parts;
    auto go = [&](auto ta, auto tb) {
        typedef decltype(ta) Ta;
        typedef decltype(tb) Tb;
        hipLaunchKernelGGL((k_prod_two<Ta, Tb>), dim3((unsigned)n), dim3(Ta::THREADS), 0, st, a, b, first);
    };
    if (pa.tile == 128 && n <= op_cus())
        go(Tile<M, 128, 128, 2, 4, 3, true, false>(), Tile<M, 128, 128, 2, 4, 3, true, true>());
    else if (pa.tile == 128)
        go(Tile<M, 128, 128, 2, 4, 2, true, false>(), Tile<M, 128, 128, 2, 4, 2, true, true>());
    else
        go(Tile<M, 64, 64, 2, 2, 4, true, false>(), Tile<M, 64, 64, 2, 2, 4, true, true>());
    for (const ProdArgs* g : {&a, &b})
        if (g->parts > 1)
            hipLaunchKernelGGL((k_prod_join<typename M::Elem, false>), grid256(g->end * (g->dp / 8)), dim3(256), 0, st, *g);
}

template <typename M, bool ACOLS, bool BCOLS, bool ACC = false, bool PAST = false>
static void launch_prod(ProdArgs a, const ProdPlan& p, void* partial, hipStream_t st) {
    a.parts = p.parts;
    a.part_chunks = p.part_chunks;
    a.partial = static_cast<float*>(partial);
    a.dp = (a.d + 7) / 8 * 8;
    auto go = [&](auto tile) {
        typedef decltype(tile) Tl;
        a.ni = (int)((a.a.n + Tl::ROWS - 1) / Tl::ROWS);
        a.nt = (int)((a.b.n + Tl::COLS - 1) / Tl::COLS);
        hipLaunchKernelGGL((k_prod<Tl, ACC, PAST>), dim3((unsigned)(a.ni * a.nt * a.parts)), dim3(Tl::THREADS), 0, st,
                           a);
    };
    if (p.tile == 256)
        go(BigTile<M, ACOLS, BCOLS>());
    else if (p.tile == 128 && one_a_cu(128, a.a.n, a.b.n, p.parts))
        go(Tile<M, 128, 128, 2, 4, 3, ACOLS, BCOLS>());
    else if (p.tile == 128)
        go(Tile<M, 128, 128, 2, 4, 2, ACOLS, BCOLS>());
    else
        go(Tile<M, 64, 64, 2, 2, 4, ACOLS, BCOLS>());
    if (a.parts > 1)
        hipLaunchKernelGGL((k_prod_join<typename M::Elem, ACC>), grid256(a.end * (a.dp / 8)), dim3(256), 0, st, a);
}

}  // namespace bk
