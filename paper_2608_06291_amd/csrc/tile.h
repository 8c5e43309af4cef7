// Products of two matrices whose rows are contiguous along the summed axis, on the
// matrix cores:  D[i][t] = sum_k A[i][k] B[t][k]  for 16-bit floats and 8-bit integers.
//
// A workgroup computes BM x BN of D from chunks of 128 bytes of k (64 16-bit or 128
// 8-bit entries) of BM rows of A and BN rows of B, double-buffered in LDS and written
// there by direct global loads.  A lane's 16-byte piece of a row is what one MFMA of 16 x 16
// takes, for either type.  The pieces of a row are permuted by the row (by address, on
// the way in), so that the 16 rows of a fragment read meet different banks.
#pragma once
#include "ops.h"

namespace bk {

typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8_t __attribute__((ext_vector_type(8)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x2 __attribute__((ext_vector_type(2)));

constexpr int CHUNK_BYTES = 128;
// BigTile's 32-bit offsets reach 256 rows of fewer bytes than this.
constexpr int64_t TILE_LD_MAX = (int64_t)1 << 23;

// Operand types: what a 16-byte piece holds, the accumulator, bytes of A a chunk.
struct MmaF16 {
    typedef f16_t Elem;
    typedef f32x4 Acc;
    static constexpr int A_BYTES = CHUNK_BYTES;
    static __device__ inline Acc mma(i32x4 a, i32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                      __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};
struct MmaBF16 {
    typedef bf16_t Elem;
    typedef f32x4 Acc;
    static constexpr int A_BYTES = CHUNK_BYTES;
    static __device__ inline Acc mma(i32x4 a, i32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                       __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
    }
};
struct MmaI8 {   // A in 8 bits
    typedef int8_t Elem;
    typedef i32x4 Acc;
    static constexpr int A_BYTES = CHUNK_BYTES;
    static __device__ inline Acc mma(i32x4 a, i32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
    }
};
struct MmaI4 {   // A packed in 4 bits; the sums come out 16 times as large
    typedef int8_t Elem;
    typedef i32x4 Acc;
    static constexpr int A_BYTES = CHUNK_BYTES / 2;
    static __device__ inline Acc mma(i32x4 a, i32x4 b, Acc c) {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
    }
};

// 16 codes of 4 bits to 16 bytes, each 16 times the code: the code in the upper half
// of its byte needs no sign extension.
__device__ inline i32x4 unpack_codes(i32x2 p) {
    const uint32_t u = (uint32_t)p[0], v = (uint32_t)p[1];
    return i32x4{(int32_t)((u << 4) & 0xf0f0f0f0u), (int32_t)(u & 0xf0f0f0f0u),
                 (int32_t)((v << 4) & 0xf0f0f0f0u), (int32_t)(v & 0xf0f0f0f0u)};
}

// 16 bytes of zeros: where a lane whose piece lies past the end of k reads.
static __device__ const uint4 tile_zeros = {0, 0, 0, 0};

// One operand: `row(r)` gives the address of row r of the tile.
// Stages chunk bytes [off, off + BYTES) of ROWS rows; pieces at or past `end` are zeros.
template <int ROWS, int BYTES, int WAVES>
struct Stager {
    static constexpr int PER_ROW = BYTES / 16;            // 16-byte pieces of a row
    static constexpr int ROWS_PER = 64 / PER_ROW;         // rows a wave writes at once
    static constexpr int N = ROWS / ROWS_PER / WAVES;     // loads a wave issues
    static_assert(N >= 1 && N * ROWS_PER * WAVES == ROWS, "tile rows");

    const char* src[N];   // this lane's piece of chunk 0
    int piece;            // its byte offset in the chunk

    // Piece held in slot `slot` of LDS row r.
    static __device__ inline int permuted(int r, int slot) {
        return BYTES == 128 ? slot ^ (r & 7) : slot ^ ((r >> 2) & 3);
    }
    template <typename RowFn>
    __device__ inline void init(RowFn row, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int r = (i * WAVES + wave) * ROWS_PER + lane / PER_ROW;
            piece = permuted(r, lane % PER_ROW) * 16;
            src[i] = row(r) + piece;
        }
    }
    // (the permutation has period 8 or 16 in r, and r steps by multiples of WAVES *
    // ROWS_PER, so `piece` is the same for every i)
    static_assert((WAVES * ROWS_PER) % (BYTES == 128 ? 8 : 16) == 0, "one piece a lane");

    __device__ inline void load(char* lds, int64_t off, int64_t end, int wave) const {
        const bool out = off + piece >= end;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const char* p = out ? reinterpret_cast<const char*>(&tile_zeros) : src[i] + off;
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void*)p,
                (__attribute__((address_space(3))) void*)(lds + (i * WAVES + wave) * 1024), 16, 0, 0);
        }
    }
};

// The tile's main loop.  acc[x][y] gets rows x, columns y of 16 of the wave's part;
// lane l of it holds D[4 (l / 16) + 0..3][l % 16].
template <typename M, int BM, int BN, int WM, int WN>
struct Tile {
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int TM = BM / WM, TN = BN / WN;      // a wave's part
    static constexpr int X = TM / 16, Y = TN / 16;
    static constexpr int A_LDS = BM * M::A_BYTES, B_LDS = BN * CHUNK_BYTES;
    static constexpr int LDS = 2 * (A_LDS + B_LDS);
    static constexpr int ROWS = BM, COLS = BN;
    typedef M Mma;
    typedef typename M::Acc Acc;
    typedef Acc Accs[X][Y];
    // Units of 16 rows of A and of 16 rows of B in a wave's part, and where they begin.
    static constexpr int UA = X, UB = Y;
    static __device__ inline int a0(int wave) { return wave / WN * TM; }
    static __device__ inline int b0(int wave) { return wave % WN * TN; }
    static __device__ inline Acc& at(Accs& acc, int a, int b) { return acc[a][b]; }

    // `after(c, acc)` runs when chunk c has been added.
    template <typename RowA, typename RowB, typename After>
    static __device__ inline void run(char* lds, RowA row_a, RowB row_b, int64_t a_end, int64_t b_end,
                                      int chunks, Acc (&acc)[X][Y], After after) {
        const int tid = threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wm = wave / WN, wn = wave % WN;
        Stager<BM, M::A_BYTES, WAVES> sa;
        Stager<BN, CHUNK_BYTES, WAVES> sb;
        sa.init(row_a, wave, lane);
        sb.init(row_b, wave, lane);
        const int r16 = lane & 15, kq = lane >> 4;
        if (chunks > 0) {
            sa.load(lds, 0, a_end, wave);
            sb.load(lds + A_LDS, 0, b_end, wave);
        }
        for (int c = 0; c < chunks; ++c) {
            char* const cur = lds + (c & 1) * (A_LDS + B_LDS);
            char* const nxt = lds + ((c + 1) & 1) * (A_LDS + B_LDS);
            __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this wave's direct loads landed
            __syncthreads();                      // everybody's, and the other buffer is free
            if (c + 1 < chunks) {
                sa.load(nxt, (int64_t)(c + 1) * M::A_BYTES, a_end, wave);
                sb.load(nxt + A_LDS, (int64_t)(c + 1) * CHUNK_BYTES, b_end, wave);
            }
            const char* const A = cur + wm * TM * M::A_BYTES;
            const char* const B = cur + A_LDS + wn * TN * CHUNK_BYTES;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                i32x4 b[Y];
#pragma unroll
                for (int y = 0; y < Y; ++y) {
                    const int r = y * 16 + r16;
                    b[y] = *reinterpret_cast<const i32x4*>(B + r * CHUNK_BYTES +
                                                           (((s * 4 + kq) ^ (r & 7)) << 4));
                }
#pragma unroll
                for (int x = 0; x < X; ++x) {
                    const int r = x * 16 + r16;
                    i32x4 a;
                    if constexpr (M::A_BYTES == CHUNK_BYTES) {
                        a = *reinterpret_cast<const i32x4*>(A + r * CHUNK_BYTES +
                                                            (((s * 4 + kq) ^ (r & 7)) << 4));
                    } else {
                        const int k8 = s * 4 + kq;   // 8-byte piece
                        a = unpack_codes(*reinterpret_cast<const i32x2*>(
                            A + r * M::A_BYTES + ((((k8 >> 1) ^ ((r >> 2) & 3)) << 4) | ((k8 & 1) << 3))));
                    }
#pragma unroll
                    for (int y = 0; y < Y; ++y) acc[x][y] = M::mma(a, b[y], acc[x][y]);
                }
                after(2 * c + s, acc);
            }
        }
    }
};

template <int N>
__device__ inline void wait_loads() {   // all but the last N of this wave's
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ inline void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// A barrier that waits for no memory operation and that none is moved across.
__device__ inline void bare_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
}

// The same product for many tiles: 256 x 256, eight waves in two groups of four, one of
// each group on every SIMD, half a phase apart.  While the waves of one group feed the matrix cores
// (16 MFMAs a phase, at raised priority), those of the other read the fragments of
// their next phase from LDS and issue global loads; barriers keep the two in step.
//
// A wave's part is 128 rows of B times 64 rows of A.  Its four phases a chunk are the
// products of the halves  B0 A0, B0 A1, B1 A1, B1 A0,  so that a phase reads 8, 4, 8, 4
// fragments (A0 of the next chunk in the last one).  A half is dead once both groups have
// read it, and the same half of the chunk after next is loaded over it: B0 in phase 1, A0 and A1 in
// phase 2, B1 in phase 3, five phases or more before they are read.  Loads past the last
// chunk read it again, so that the waits can count.
template <typename M>
struct BigTile {
    static constexpr int THREADS = 512, ROWS = 256, COLS = 256;
    static constexpr int A_LDS = ROWS * M::A_BYTES, B_LDS = COLS * CHUNK_BYTES;
    static constexpr int LDS = 2 * (A_LDS + B_LDS);
    static constexpr int NA = M::A_BYTES / 64;   // loads of a half of A by a wave (of B: 2)
    typedef M Mma;
    typedef typename M::Acc Acc;
    typedef Acc Accs[8][4];
    static constexpr int UA = 4, UB = 8;
    static __device__ inline int a0(int wave) { return (wave & 3) * 64; }
    static __device__ inline int b0(int wave) { return (wave >> 2) * 128; }
    static __device__ inline Acc& at(Accs& acc, int a, int b) { return acc[b][a]; }

    // One operand's loads: 32-bit offsets of this lane's pieces from a base that moves
    // on with the chunks.
    template <int BYTES, int N>
    struct Source {
        const char* base;
        uint32_t off[2][N];   // [half][load]
        int piece;
    };
    static __device__ inline int load_row_b(int half, int i, int wave) {   // first of 8 rows
        return i * 128 + half * 64 + wave * 8;
    }
    static __device__ inline int load_row_a(int half, int i, int wave) {   // of 8, or of 16 of 64 bytes
        return M::A_BYTES == CHUNK_BYTES ? i * 128 + wave / 4 * 64 + half * 32 + wave % 4 * 8
                                         : wave / 2 * 64 + half * 32 + wave % 2 * 16;
    }
    template <int BYTES, int N>
    static __device__ inline void load(const Source<BYTES, N>& s, int half, char* lds, int row_of_load,
                                       int i, int chunk, int last, int64_t end) {
        char* const to = lds + row_of_load * BYTES;
        const int c = min(chunk, last);
        const char* base = s.base + (int64_t)c * BYTES;
        const char* p = base + s.off[half][i];
        if ((int64_t)(c + 1) * BYTES > end && (int64_t)c * BYTES + s.piece >= end)
            p = reinterpret_cast<const char*>(&tile_zeros);
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                         (__attribute__((address_space(3))) void*)to, 16, 0, 0);
    }

    // base_a, base_b: where the tile's rows begin; off_a(r), off_b(r): bytes from there to
    // row r (rows of one load share base_a).  All rows are read up to a_end, b_end bytes.
    template <typename OffA, typename OffB, typename After>
    static __device__ inline void run(char* lds, const char* base_a, const char* base_b, OffA off_a,
                                      OffB off_b, int64_t a_end, int64_t b_end, int chunks, Accs& acc,
                                      After after) {
        const int tid = threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int group = wave >> 2;
        constexpr int BUF = A_LDS + B_LDS;
        Source<M::A_BYTES, NA> sa;
        Source<CHUNK_BYTES, 2> sb;
        sa.base = base_a;
        sb.base = base_b;
        {
            constexpr int PR = M::A_BYTES / 16;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < NA; ++i) {
                    const int r = load_row_a(h, i, wave) + lane / PR;
                    sa.piece = Stager<256, M::A_BYTES, 8>::permuted(r, lane % PR) * 16;
                    sa.off[h][i] = off_a(r) + sa.piece;
                }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = load_row_b(h, i, wave) + lane / 8;
                    sb.piece = Stager<256, CHUNK_BYTES, 8>::permuted(r, lane % 8) * 16;
                    sb.off[h][i] = off_b(r) + sb.piece;
                }
        }
        const int last = chunks - 1;
        auto load_a = [&](int half, int c) {
            char* const to = lds + (c & 1) * BUF;
#pragma unroll
            for (int i = 0; i < NA; ++i)
                load(sa, half, to, load_row_a(half, i, wave), i, c, last, a_end);
        };
        auto load_b = [&](int half, int c) {
            char* const to = lds + (c & 1) * BUF + A_LDS;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                load(sb, half, to, load_row_b(half, i, wave), i, c, last, b_end);
        };
        const int r16 = lane & 15, kq = lane >> 4;
        // byte offsets of the fragments of the two steps of a chunk in a row
        int fa[2], fb[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int k = s * 4 + kq;
            fb[s] = A_LDS + (b0(wave) + r16) * CHUNK_BYTES + ((k ^ (r16 & 7)) << 4);
            fa[s] = (a0(wave) + r16) * M::A_BYTES +
                    (M::A_BYTES == CHUNK_BYTES
                         ? (k ^ (r16 & 7)) << 4
                         : (((k >> 1) ^ ((r16 >> 2) & 3)) << 4) | ((k & 1) << 3));
        }
        auto read_a = [&](int half, const char* buf, i32x4 (&a)[2][2]) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const char* const p = buf + fa[s] + (half * 2 + y) * 16 * M::A_BYTES;
                    if constexpr (M::A_BYTES == CHUNK_BYTES)
                        a[y][s] = *reinterpret_cast<const i32x4*>(p);
                    else
                        a[y][s] = unpack_codes(*reinterpret_cast<const i32x2*>(p));
                }
        };
        auto read_b = [&](int half, const char* buf, i32x4 (&b)[4][2]) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    b[x][s] = *reinterpret_cast<const i32x4*>(buf + fb[s] + (half * 4 + x) * 16 * CHUNK_BYTES);
        };
        i32x4 a_0[2][2], a_1[2][2], b_[4][2];
        auto products = [&](const i32x4 (&a)[2][2], int ha, int hb) {
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int y = 0; y < 2; ++y)
                        acc[hb * 4 + x][ha * 2 + y] = M::mma(a[y][s], b_[x][s], acc[hb * 4 + x][ha * 2 + y]);
            __builtin_amdgcn_s_setprio(0);
        };

        load_b(0, 0), load_a(0, 0), load_a(1, 0), load_b(1, 0);
        load_b(0, 1), load_a(0, 1), load_a(1, 1), load_b(1, 1);
        wait_loads<4 + 2 * NA>();   // chunk 0
        bare_barrier();
        read_a(0, lds, a_0);
        wait_lds();
        if (group == 1) bare_barrier();
#pragma nounroll
        for (int c = 0; c < chunks; ++c) {
            const char* const cur = lds + (c & 1) * BUF;
            const char* const nxt = lds + ((c + 1) & 1) * BUF;
            // phase 0: B0 A0
            read_b(0, cur, b_);
            wait_loads<6 + 2 * NA>();   // A1 of this chunk, read in phase 1
            wait_lds();
            bare_barrier();
            products(a_0, 0, 0);
            bare_barrier();
            // phase 1: B0 A1
            read_a(1, cur, a_1);
            wait_loads<4 + 2 * NA>();   // B1 of this chunk, read in phase 2
            load_b(0, c + 2);
            wait_lds();
            bare_barrier();
            products(a_1, 1, 0);
            bare_barrier();
            // phase 2: B1 A1
            read_b(1, cur, b_);
            wait_loads<4 + NA>();       // A0 and B0 of the next chunk, read in phases 3 and 0
            load_a(0, c + 2);
            load_a(1, c + 2);
            wait_lds();
            bare_barrier();
            products(a_1, 1, 1);
            bare_barrier();
            // phase 3: B1 A0
            i32x4 a_n[2][2];
            read_a(0, nxt, a_n);
            load_b(1, c + 2);
            wait_lds();
            bare_barrier();
            products(a_0, 0, 1);
            after(c, acc);
            bare_barrier();
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int s = 0; s < 2; ++s) a_0[y][s] = a_n[y][s];
        }
        if (group == 0) bare_barrier();
        wait_loads<0>();   // none may land after the workgroup has gone
    }
};

// Workgroup v runs on XCD v mod 8, each with an L2 of its own: every XCD takes a
// contiguous range of the tiles, which go down strips `strip` tiles wide.
__device__ inline void tile_of(int v, int ni, int nt, int strip, int* i, int* t) {
    const int n = ni * nt;
    const int per = n / 8, rest = n % 8, x = v & 7, k = v >> 3;
    const int id = x * per + min(x, rest) + k;   // (XCDs below `rest` hold one more)
    const int first = id / (strip * nt) * strip, w = min(strip, ni - first);
    const int in = id - first * nt;
    *i = first + in % w;
    *t = in / w;
}

// Four consecutive outputs, `valid` of them inside the row.
template <typename E>
__device__ inline void store4(E* p, const float (&v)[4], int64_t valid) {
    if (valid >= 4) {
        Pack<E, 4> o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o.v[j] = (E)v[j];
        store_pack(p, o);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < valid) p[j] = (E)v[j];
    }
}
template <typename E>
__device__ inline void load4(const E* p, float (&v)[4], int64_t valid) {
    if (valid >= 4) {
        const auto o = load_pack<E, 4>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)o.v[j];
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = j < valid ? (float)p[j] : 0.0f;
    }
}

// Activations and their slopes in fp32, with the library's exp and erf.
__device__ inline float act_value(float z, int act) {
    if (act == BAKRON_ACT_SILU) return z / (1.0f + expf(-z));
    if (act == BAKRON_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    return z;
}
__device__ inline void act_both(float z, int act, float* value, float* slope) {
    if (act == BAKRON_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-z));
        *value = z * s;
        *slope = s * (1.0f + z * (1.0f - s));
    } else {
        const float c = 0.5f * (1.0f + erff(z * 0.70710678118654752f));
        *value = z * c;
        *slope = c + z * 0.39894228040143268f * expf(-0.5f * z * z);
    }
}

}  // namespace bk
