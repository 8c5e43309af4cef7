// Products on the matrix cores:  D[i][t] = sum_k A[i][k] B[t][k]  for 16-bit floats and
// 8-bit integers.
//
// A workgroup computes a tile of D from chunks of 128 bytes of k (64 16-bit or 128 8-bit
// entries), double-buffered in LDS and written there by direct global loads.  Either
// operand is held in memory with k contiguous (rows), or, in 16 bits, with i or t
// contiguous (columns; the fragments are then read with the transposing LDS read).  The
// pieces of a staged row are permuted by the row, by address on the way in, so that the
// rows of a fragment read meet different banks.
#pragma once
#include "ops.h"

namespace bk {

typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8_t __attribute__((ext_vector_type(8)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x2 __attribute__((ext_vector_type(2)));

constexpr int CHUNK_BYTES = 128;
// 32-bit offsets reach 256 rows of fewer bytes than this.
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

// How an operand lies in LDS, for UNITS units of 16 of its rows (or columns) a chunk.
//
// Rows (k contiguous): a row of BYTES bytes is cut into 16-byte pieces; slot s of row r
// holds piece s ^ (r & 7), or s ^ ((r >> 2) & 3) in rows of 64 bytes.  A lane's 16 (or 8,
// packed) bytes of a fragment are one read.  Packed rows are read 16 bytes (32 codes) a lane, for
// both steps of a chunk: lane q = lane / 16 has codes 32 q .. 32 q + 31, 16 for each step, and
// the other operand's pieces follow (the order of the summed axis is free).  Only where sums end every
// 64 codes (FLUSH = 1) the steps are the chunk's halves.
//
// Columns (k outside): row k holds UNITS units of 16 entries (32 bytes); unit u of row k lies at
// u ^ f(k), f(k) from the bits of k that differ between the 16 rows that a transposing read
// touches (k = 8 q + 4 e + r: q and r, for 16 lanes of rows r and 4 x 4 entries each).
template <int BYTES>
__device__ inline int row_piece(int r, int slot) {
    return BYTES == 128 ? slot ^ (r & 7) : slot ^ ((r >> 2) & 3);
}
template <int UNITS>
__device__ inline int col_twist(int k) {
    return UNITS >= 8 ? (k & 3) | ((k >> 3) & 1) << 2 : ((k >> 1) & 1) | ((k >> 3) & 1) << 1;
}
typedef int16_t i16x4 __attribute__((ext_vector_type(4)));
__device__ inline i32x2 read_transposed(const char* p) {
    return __builtin_bit_cast(i32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) i16x4*)p));
}

// An operand in memory.  Rows: row(r) is r rows of `ld` bytes on, r < n; k runs over
// [0, k_end) bytes of it.  Columns: k rows of `ld` bytes, k < k_end, of n entries (n a
// multiple of 8).  With `split` > 0 the chunks from `split` on start over at base2, those from
// 2 * split on at base again (and may be as many as before).  Past its end an operand reads as
// zeros; past n (never used) as some entry before it.
struct Operand {
    const char* base;
    const char* base2;
    int64_t ld, n, k_end;
    int split;
};
inline Operand operand(const void* base, int64_t ld, int64_t n, int64_t k_end) {
    return Operand{static_cast<const char*>(base), nullptr, ld, n, k_end, 0};
}

__device__ inline uint32_t lds_address(char* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)p;
}
// 16 bytes a lane from p to LDS address `to` (the same in all lanes) + 16 * lane.  In
// assembly because the compiler waits for every load of its own before a transposing LDS
// read, which it cannot tell from the place being loaded; all waits are wait_loads().  It
// writes no register but m0, which cannot be declared (the compiler keeps it for itself and need not
// honour that): a kernel that loads this way must use m0 for nothing else, no builtin load to LDS
// among it.  A test holds the built kernels to that.
__device__ inline void load_lds(const char* p, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(
                     __builtin_amdgcn_readfirstlane(to)),
                 "v"(p)
                 : "memory");
}
// The same from base (the same in all lanes) + off.
__device__ inline void load_lds(const char* base, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(
                     __builtin_amdgcn_readfirstlane(to)),
                 "v"(off), "s"(base)
                 : "memory");
}
// 4 bytes a lane.
__device__ inline void load_lds_word(const float* p, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(
                     __builtin_amdgcn_readfirstlane(to)),
                 "v"(p)
                 : "memory");
}
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

// N loads of a wave from one operand: each lane's pieces as 32-bit offsets from a base
// that moves on with the chunks (a scalar: a load takes no vector arithmetic).
template <bool COLS, int BYTES, int N>
struct Source {
    static constexpr int UNIT = COLS ? 64 : BYTES;   // of k in a chunk
    const char *base, *base2;
    int64_t step;        // bytes from chunk to chunk
    int split, last;
    int whole;           // chunks before the one in which the operand ends
    uint32_t off[N];
    int at[N];           // Columns: row in the chunk; rows: at[0] the piece's byte
    int64_t end;         // k_end

    __device__ inline void init(const Operand& o, int64_t first, int end_chunk) {
        base = o.base + (COLS ? 2 * first : first * o.ld);
        base2 = o.base2 + (COLS ? 2 * first : first * o.ld);
        step = COLS ? 64 * o.ld : BYTES;
        split = o.split;
        last = end_chunk - 1;
        end = o.k_end;
        whole = (int)(end / UNIT);
    }
    // Load i: the lane's piece of tile row `tile_row`, or the 8 columns at `tile_col` of row k.
    __device__ inline void set_row(int i, const Operand& o, int64_t first, int tile_row, int piece) {
        at[0] = piece;
        off[i] = (uint32_t)(min((int64_t)tile_row, o.n - 1 - first) * o.ld) + piece;
    }
    __device__ inline void set_col(int i, const Operand& o, int64_t first, int k, int tile_col) {
        at[i] = k;
        off[i] = (uint32_t)(k * o.ld) + (first + tile_col < o.n ? 2 * tile_col : 0);
    }
    // Where a chunk lies: worked out before the barrier that its loads come after, because nothing
    // runs beside scalar arithmetic that all waves do at once behind one.
    struct Chunk {
        const char* b;
        int number;   // in its part
    };
    __device__ inline Chunk chunk(int number) const {
        int c = min(number, last);   // (past the last chunk: that one again, not used)
        const char* b = base;
        if (split > 0) {
            if (c >= 2 * split) c -= 2 * split;
            if (c >= split) {
                b = base2;
                c -= split;
            }
        }
        return Chunk{b + c * step, c};
    }
    // All loads of a chunk, number i to to + i * stride.
    __device__ inline void load(const Chunk& c, uint32_t to, int stride) const {
        if (c.number < whole) {
#pragma unroll
            for (int i = 0; i < N; ++i) load_lds(c.b, off[i], to + i * stride);
        } else {   // the operand ends in this chunk: zeros from there on
            const int64_t left = end - (int64_t)c.number * UNIT;
#pragma unroll
            for (int i = 0; i < N; ++i)
                load_lds(at[COLS ? i : 0] < left ? c.b + off[i] : reinterpret_cast<const char*>(&tile_zeros),
                         to + i * stride);
        }
    }
    __device__ inline void load(int number, uint32_t to, int stride) const { load(chunk(number), to, stride); }
};

// The small tile: WM x WN waves, BUFS buffers, so that BUFS - 1 chunks are on their way
// while one is multiplied, and one barrier a chunk.  FLUSH > 0: the sums of every FLUSH steps
// (half chunks) are handed to `flush` and begin at zero again.
template <typename M, int BM, int BN, int WM, int WN, int BUFS, bool ACOLS = false, bool BCOLS = false,
          int FLUSH = 0>
struct Tile {
    static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
    static constexpr int ROWS = BM, COLS = BN;
    static constexpr int TM = BM / WM, TN = BN / WN;      // a wave's part
    static constexpr int UA = TM / 16, UB = TN / 16;      // in units of 16
    static constexpr int A_LDS = BM * M::A_BYTES, B_LDS = BN * CHUNK_BYTES;
    // the scales of the chunk's 2 / FLUSH groups for every row of A
    static constexpr int S_LDS = FLUSH ? 2 / FLUSH * BM * 4 : 0;
    static constexpr int BUF = A_LDS + B_LDS + S_LDS;
    static constexpr int LDS = BUFS * BUF;
    typedef M Mma;
    typedef typename M::Acc Acc;
    typedef Acc Accs[UA][UB];
    static __device__ inline int a0(int wave) { return wave / WN * TM; }
    static __device__ inline int b0(int wave) { return wave % WN * TN; }
    static __device__ inline Acc& at(Accs& acc, int a, int b) { return acc[a][b]; }

    // All loads of one operand of R rows (columns).
    template <bool C, int R, int BYTES>
    struct Loads {
        static constexpr int PIECES = C ? R / 8 : BYTES / 16;   // of an LDS row
        static constexpr int PER = 64 / PIECES;                 // LDS rows a load writes
        static constexpr int N = (C ? 64 : R) / PER / WAVES;
        static_assert(N >= 1, "every wave loads");
        Source<C, BYTES, N> s;
        template <typename RowFn>
        __device__ inline void init(const Operand& o, int64_t first, int end_chunk, int wave, int lane,
                                    RowFn row) {
            s.init(o, first, end_chunk);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int r = (i * WAVES + wave) * PER + lane / PIECES, slot = lane % PIECES;
                if constexpr (C) {
                    const int unit = (slot >> 1) ^ col_twist<R / 16>(r);
                    s.set_col(i, o, first, r, unit * 16 + (slot & 1) * 8);
                } else {
                    // (row_piece has a period that divides the rows between two loads)
                    s.set_row(i, o, first, row(r), row_piece<BYTES>(r, slot) * 16);
                }
            }
        }
        typedef typename Source<C, BYTES, N>::Chunk Chunk;
        __device__ inline void load(const Chunk& chunk, uint32_t lds, int wave) const {
            s.load(chunk, lds + wave * 1024, WAVES * 1024);
        }
    };
    static constexpr bool PAIRED = M::A_BYTES != CHUNK_BYTES && FLUSH != 1;
    // A fragment: unit u of R / 16, step s.
    template <bool C, int R, int BYTES>
    static __device__ inline i32x4 fragment(const char* lds, int u, int s, int lane) {
        const int r16 = lane & 15, kq = lane >> 4;
        if constexpr (C) {
            const int k = s * 32 + kq * 8 + (r16 >> 2);
            const char* const p = lds + k * (2 * R) + ((u ^ col_twist<R / 16>(k)) << 5) + (r16 & 3) * 8;
            const i32x2 x = read_transposed(p), y = read_transposed(p + 4 * 2 * R);
            return i32x4{x[0], x[1], y[0], y[1]};
        } else {
            const int r = u * 16 + r16, k = PAIRED ? 2 * kq + s : s * 4 + kq;
            if constexpr (BYTES == CHUNK_BYTES) {
                return *reinterpret_cast<const i32x4*>(lds + r * BYTES + (row_piece<BYTES>(r, k) << 4));
            } else if constexpr (PAIRED) {
                const i32x4 w =
                    *reinterpret_cast<const i32x4*>(lds + r * BYTES + (row_piece<BYTES>(r, kq) << 4));
                return unpack_codes(i32x2{w[2 * s], w[2 * s + 1]});
            } else
                return unpack_codes(*reinterpret_cast<const i32x2*>(
                    lds + r * BYTES + (row_piece<BYTES>(r, k >> 1) << 4) + ((k & 1) << 3)));
        }
    }

    // Chunks c0 .. c0 + chunks - 1 of the tile that begins at row `ia` of A and row `ib` of
    // B; row_a maps rows of the tile to
    // rows of the operand, counted from ia.  With FLUSH, scale(row, c, k) is the address of
    // the scale of tile row `row` for the k-th FLUSH steps of chunk c, and what is flushed is
    // sum[x][y] += acc * scale.  LDS is free to use again on return.
    template <typename RowA, typename Scale>
    static __device__ inline void run(char* lds, const Operand& oa, int64_t ia, const Operand& ob,
                                      int64_t ib, int c0, int chunks, Accs& acc, RowA row_a,
                                      f32x4 (&sum)[FLUSH ? UA : 1][FLUSH ? UB : 1], Scale scale) {
        const int tid = threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        Loads<ACOLS, BM, M::A_BYTES> la;
        Loads<BCOLS, BN, CHUNK_BYTES> lb;
        la.init(oa, ia, c0 + chunks, wave, lane, row_a);
        lb.init(ob, ib, c0 + chunks, wave, lane, [](int r) { return r; });
        const uint32_t base = lds_address(lds);
        constexpr int S_LOADS = FLUSH ? (2 / FLUSH * BM + THREADS - 1) / THREADS : 0;
        constexpr int LOADS = la.N + lb.N + S_LOADS;   // of a chunk
        // What the loads of a chunk start from.
        struct Ahead {
            typename decltype(la)::Chunk a;
            typename decltype(lb)::Chunk b;
            const float* scale[FLUSH ? S_LOADS : 1];
        };
        auto ahead = [&](int c) {
            Ahead h{la.s.chunk(c0 + c), lb.s.chunk(c0 + c), {}};
            if constexpr (FLUSH > 0) {
                // (with fewer scales than threads the waves past them load the same again)
#pragma unroll
                for (int i = 0; i < S_LOADS; ++i) {
                    const int e = (i * WAVES + wave) * 64 % (2 / FLUSH * BM);
                    h.scale[i] = scale((e + lane) % BM, c0 + min(c, chunks - 1), e / BM);
                }
            }
            return h;
        };
        auto load = [&](const Ahead& h, int buf) {
            const uint32_t to = base + buf * BUF;
            la.load(h.a, to, wave);
            lb.load(h.b, to + A_LDS, wave);
            if constexpr (FLUSH > 0) {
#pragma unroll
                for (int i = 0; i < S_LOADS; ++i)
                    load_lds_word(h.scale[i],
                                  to + A_LDS + B_LDS + (i * WAVES + wave) * 64 % (2 / FLUSH * BM) * 4);
            }
        };
#pragma unroll
        for (int c = 0; c < BUFS - 1; ++c) load(ahead(c), c);   // (chunks past the last read it again)
        Ahead next = ahead(BUFS - 1);
        int buf = 0;
        for (int c = 0; c < chunks; ++c) {
            const char* const cur = lds + buf * BUF;
            wait_loads<(BUFS - 2) * LOADS>();
            bare_barrier();   // everybody's loads of this chunk landed, and the buffer before is free
            load(next, buf == 0 ? BUFS - 1 : buf - 1);
            next = ahead(c + BUFS);
            buf = buf == BUFS - 1 ? 0 : buf + 1;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                i32x4 b[UB];
#pragma unroll
                for (int y = 0; y < UB; ++y)
                    b[y] = fragment<BCOLS, BN, CHUNK_BYTES>(cur + A_LDS, b0(wave) / 16 + y, s, lane);
#pragma unroll
                for (int x = 0; x < UA; ++x) {
                    const i32x4 a = fragment<ACOLS, BM, M::A_BYTES>(cur, a0(wave) / 16 + x, s, lane);
                    if constexpr (FLUSH > 0) {
                        constexpr bool FIRST_ONLY = FLUSH == 1;
#pragma unroll
                        for (int y = 0; y < UB; ++y)
                            acc[x][y] = M::mma(a, b[y], FIRST_ONLY || s == 0 ? Acc{} : acc[x][y]);
                        if (FLUSH == 1 || s == 1) {
                            const f32x4 sc = *reinterpret_cast<const f32x4*>(
                                cur + A_LDS + B_LDS +
                                ((FLUSH == 1 ? s * BM : 0) + a0(wave) + x * 16 + (lane >> 4) * 4) * 4);
#pragma unroll
                            for (int y = 0; y < UB; ++y)
#pragma unroll
                                for (int j = 0; j < 4; ++j)
                                    sum[x][y][j] = fmaf((float)acc[x][y][j], sc[j], sum[x][y][j]);
                        }
                    } else {
#pragma unroll
                        for (int y = 0; y < UB; ++y) acc[x][y] = M::mma(a, b[y], acc[x][y]);
                    }
                }
            }
        }
        wait_loads<0>();   // the loads past the last chunk
        __syncthreads();
    }
    template <typename RowA>
    static __device__ inline void run(char* lds, const Operand& oa, int64_t ia, const Operand& ob,
                                      int64_t ib, int c0, int chunks, Accs& acc, RowA row_a) {
        static_assert(FLUSH == 0, "scales missing");
        f32x4 none[1][1];
        run(lds, oa, ia, ob, ib, c0, chunks, acc, row_a, none, [](int, int, int) { return (const float*)nullptr; });
    }
};

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
//
// 4096 x 4096 x 22016 bf16: 522 us, 1415 TFLOP/s (the library's product: 1326), 630 with the same
// tile, two buffers and one barrier a chunk.  Bound by power and issue: matrix cores 67%
// busy at that rate, LDS 26% of the cycles and no bank conflicts.  Two steps that mattered: loads from a
// scalar base (vector addresses: 572 us) and loads in assembly (the compiler's own waits before
// transposing reads: 674).  One workgroup a CU, so a tile's prologue and epilogue overlap nothing: 15
// to 25 us a round.
template <typename M, bool ACOLS = false, bool BCOLS = false>
struct BigTile {
    static constexpr int THREADS = 512, ROWS = 256, COLS = 256;
    static constexpr int A_LDS = ROWS * M::A_BYTES, B_LDS = COLS * CHUNK_BYTES;
    static constexpr int A_HALF = A_LDS / 2, B_HALF = B_LDS / 2;
    static constexpr int LDS = 2 * (A_LDS + B_LDS);
    static constexpr bool PAIRED = M::A_BYTES != CHUNK_BYTES;
    static constexpr int NA = M::A_BYTES / 64;   // loads of a half of A by a wave (of B: 2)
    typedef M Mma;
    typedef typename M::Acc Acc;
    typedef Acc Accs[8][4];
    static constexpr int UA = 4, UB = 8;
    static __device__ inline int a0(int wave) { return (wave & 3) * 64; }
    static __device__ inline int b0(int wave) { return (wave >> 2) * 128; }
    static __device__ inline Acc& at(Accs& acc, int a, int b) { return acc[b][a]; }

    // A half of an operand, in LDS 128 rows (or 64 rows of 128 columns): G groups of
    // 128 / G of them, those of half h being at 256 / G * g + 128 / G * h in the tile.
    template <bool C, int BYTES, int G, int N>
    struct Half {
        Source<C, BYTES, N> s[2];
        static __device__ inline int tile_index(int h, int j) {   // j of the half's 128
            return j / (128 / G) * (256 / G) + h * (128 / G) + j % (128 / G);
        }
        template <typename RowFn>
        __device__ inline void init(const Operand& o, int64_t first, int end_chunk, int wave, int lane,
                                    RowFn row) {
            constexpr int PIECES = C ? 16 : BYTES / 16, PER = 64 / PIECES;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[h].init(o, first, end_chunk);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int r = (i * 8 + wave) * PER + lane / PIECES, slot = lane % PIECES;
                    if constexpr (C) {
                        const int unit = (slot >> 1) ^ col_twist<8>(r);
                        s[h].set_col(i, o, first, r, tile_index(h, unit * 16) + (slot & 1) * 8);
                    } else {
                        s[h].set_row(i, o, first, row(tile_index(h, r)), row_piece<BYTES>(r, slot) * 16);
                    }
                }
            }
        }
        __device__ inline void load(int h, int chunk, uint32_t lds, int wave) const {
            s[h].load(chunk, lds + wave * 1024, 8 * 1024);
        }
    };
    // Byte offsets in a half of this lane's reads: rows, per step; columns, per unit.
    template <bool C, int BYTES, int U>
    struct Reads {
        int at[C ? U : 2];
        __device__ inline void init(int unit0, int lane) {   // the wave's first unit of the half
            const int r16 = lane & 15, kq = lane >> 4;
            if constexpr (C) {
                const int k = kq * 8 + (r16 >> 2);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    at[u] = k * 256 + (((unit0 + u) ^ col_twist<8>(k)) << 5) + (r16 & 3) * 8;
            } else {
#pragma unroll
                for (int st = 0; st < 2; ++st)
                    at[st] = (unit0 * 16 + r16) * BYTES +
                             (row_piece<BYTES>(r16, BYTES != CHUNK_BYTES ? kq
                                                    : PAIRED             ? 2 * kq + st
                                                                         : st * 4 + kq)
                              << 4);
            }
        }
        __device__ inline i32x4 get(const char* half, int u, int st) const {
            if constexpr (C) {
                const char* const p = half + at[u] + st * (32 * 256);
                const i32x2 x = read_transposed(p), y = read_transposed(p + 4 * 256);
                return i32x4{x[0], x[1], y[0], y[1]};
            } else {
                const char* const p = half + at[st] + u * 16 * BYTES;
                const i32x4 w = *reinterpret_cast<const i32x4*>(p);
                if constexpr (BYTES == CHUNK_BYTES)
                    return w;
                else
                    return unpack_codes(i32x2{w[2 * st], w[2 * st + 1]});
            }
        }
    };

    // Arguments as of Tile::run.  The 8 or 16 rows of A that one load
    // stages have to lie in one matrix: row_a may choose oa.base by the wave.
    template <typename RowA>
    static __device__ inline void run(char* lds, const Operand& oa, int64_t ia, const Operand& ob,
                                      int64_t ib, int c0, int chunks, Accs& acc, RowA row_a) {
        const int tid = threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int group = wave >> 2;
        constexpr int BUF = A_LDS + B_LDS;
        Half<ACOLS, M::A_BYTES, 4, NA> ha;
        Half<BCOLS, CHUNK_BYTES, 2, 2> hb;
        ha.init(oa, ia, c0 + chunks, wave, lane, row_a);
        hb.init(ob, ib, c0 + chunks, wave, lane, [](int r) { return r; });
        Reads<ACOLS, M::A_BYTES, 2> ra;
        Reads<BCOLS, CHUNK_BYTES, 4> rb;
        ra.init((wave & 3) * 2, lane);
        rb.init(group * 4, lane);
        const uint32_t base = lds_address(lds);
        auto load_a = [&](int half, int c) {
            ha.load(half, c0 + c, base + (c & 1) * BUF + half * A_HALF, wave);
        };
        auto load_b = [&](int half, int c) {
            hb.load(half, c0 + c, base + (c & 1) * BUF + A_LDS + half * B_HALF, wave);
        };
        auto read_a = [&](int half, const char* buf, i32x4 (&a)[2][2]) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int s = 0; s < 2; ++s) a[y][s] = ra.get(buf + half * A_HALF, y, s);
        };
        auto read_b = [&](int half, const char* buf, i32x4 (&b)[4][2]) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int s = 0; s < 2; ++s) b[x][s] = rb.get(buf + A_LDS + half * B_HALF, x, s);
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
            bare_barrier();
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int s = 0; s < 2; ++s) a_0[y][s] = a_n[y][s];
        }
        if (group == 0) bare_barrier();
        wait_loads<0>();   // the loads past the last chunk
        __syncthreads();
    }
};

// Hands a wave's part of D on in rows: the four consecutive i of one t that a lane holds
// go through LDS (4 KiB a wave, permuted like the operands), and come back eight at a
// time, neighbouring lanes holding neighbouring ones, so that global memory is read and
// written in whole lines.  get(a, b): the accumulator of units a, b as fp32.
//
// One lane reads what others wrote, with no workgroup barrier between: every lane of the wave
// has to come through put() and take() together.  The wave barriers keep the compiler from
// letting lanes with nothing to store run ahead to the next put(); callers put their conditions
// around the stores alone.
template <typename Tl, typename Get>
struct Handover {
    static constexpr int SLOTS = Tl::UA * 4;   // 16-byte slots of a t
    char* lds;
    int lane;
    Get get;
    __device__ inline void put(int b) const {
        const int t = lane & 15;
        __builtin_amdgcn_wave_barrier();   // the last take() is over
#pragma unroll
        for (int a = 0; a < Tl::UA; ++a)
            *reinterpret_cast<f32x4*>(lds + t * (SLOTS * 16) + (((a * 4 + (lane >> 4)) ^ (t & (SLOTS - 1))) << 4)) =
                get(a, b);
        __builtin_amdgcn_wave_barrier();
    }
    // i = 8 p .. 8 p + 7 of row t of the unit put last
    __device__ inline void take(int t, int p, float (&v)[8]) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(
                lds + t * (SLOTS * 16) + (((2 * p + h) ^ (t & (SLOTS - 1))) << 4));
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * h + j] = x[j];
        }
    }
};
template <typename Tl, typename Get>
__device__ inline Handover<Tl, Get> handover(char* lds, int wave, int lane, Get get) {
    return Handover<Tl, Get>{lds + wave * (Tl::UA * 1024), lane, get};
}

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

// Which tile, by the rounds of workgroups that n of them take: a round of 256 x 256 (one a
// CU) is the unit; 128 x 128 takes 0.63 of it with two a CU and 0.42 with one, 64 x 64 0.30
// and 0.20; a round that leaves half of the CUs idle 0.8 (16-bit product 1024 to 8192 x 4096 x 4096
// to 11008 with each tile forced: 256 x 256 ahead by 20% on full rounds, 12% behind at half a
// round).
inline double tile_rounds(int tile, int64_t n, int ncu) {
    if (tile == 256) {
        const int64_t rest = n % ncu;
        return (double)(n / ncu) + (rest == 0 ? 0.0 : 2 * rest <= ncu ? 0.8 : 1.0);
    }
    const double two = tile == 128 ? 0.63 : 0.30, one = tile == 128 ? 0.42 : 0.20;
    const int64_t rest = n % (2 * ncu);
    return (double)(n / (2 * ncu)) * two + (rest == 0 ? 0.0 : rest <= ncu ? one : two);
}
// The tile of least rounds for i x t outputs; `big`: 256 x 256 can be had.
inline int pick_tile(int64_t i, int64_t t, int ncu, bool big) {
    auto rounds = [&](int b) { return tile_rounds(b, ((i + b - 1) / b) * ((t + b - 1) / b), ncu); };
    int best = 64;
    if (rounds(128) <= rounds(64)) best = 128;
    if (big && rounds(256) <= rounds(best)) best = 256;
    return best;
}
// Tiles that leave every CU with one workgroup at most have its LDS to themselves: a third buffer
// puts two chunks on their way (16-bit product 512 x 4096 x 4096: 50.6 -> 48.6 us, 441 x 2944 x 3304:
// 49.7 -> 39.0; 8-bit rows 1001 x 4096 x 4096: 27.6 -> 23.7; a fourth adds nothing).  More tiles are
// better off as two workgroups of two buffers a CU (1111 x 1000 x 2731: 24.4 us, 28.1 with three).
inline bool one_a_cu(int tile, int64_t i, int64_t t, int parts = 1) {
    return ((i + tile - 1) / tile) * ((t + tile - 1) / tile) * parts <= op_cus();
}

// Activations and their slopes in fp32, from the hardware's exp2 and reciprocal (1 ulp each).  FINE is for a
// product that stays in 32 bits, whose sums are exact: the exponent in two parts (exp_of), so that the tails of
// negative z are good to a few units (2048 x 8192 x 28672 with SiLU 425 -> 439 us).  Elsewhere what z itself is off by,
// or 16 bits of the result, exceed |z| 2^-24.
//
// The normal distribution function of GELU: erfc(x) = exp(-x^2) t P(t), t = 1 / (1 + 3 x / 8), P the polynomial
// of degree 8 that fits erfc(x) exp(x^2) / t for 0 <= x <= 10.3 with the least largest relative error (1.4e-8,
// found by reweighted least squares; in fp32 4e-7).  The slope needs its exponential, too; with the
// library's erf a tile's epilogue takes four times as long (2048 x 8192 x 28672 in 16 bits: 489 us with it, 433
// with this, 403 without activation).
template <bool FINE>
__device__ inline float sigmoid(float z) {
    const float x = FINE ? fminf(fmaxf(z, -200.0f), 200.0f) : z;
    return __builtin_amdgcn_rcpf(1.0f + exp_of<FINE>(-x));
}
template <bool FINE>
__device__ inline float normal_cdf(float z, float* gauss) {
    const float a = FINE ? fminf(fabsf(z), 20.0f) : fabsf(z);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.375f * 0.70710678118654752f, a, 1.0f));
    const float s = -0.5f * a * a;
    float g = exp_of<FINE>(s);
    if constexpr (FINE) g = fmaf(g, fmaf(-0.5f * a, a, -s), g);   // what a^2 lost
    float p = fmaf(0.06120906425710221f, t, -0.28577612992898005f);
    p = fmaf(p, t, 0.42928293498449f);
    p = fmaf(p, t, -0.22595198671736783f);
    p = fmaf(p, t, 0.27139938997970775f);
    p = fmaf(p, t, 0.12247014955191404f);
    p = fmaf(p, t, 0.2050722040962771f);
    p = fmaf(p, t, 0.21068280898732053f);
    p = fmaf(p, t, 0.21161156018602867f);
    const float tail = 0.5f * p * t * g;
    *gauss = g;
    return z > 0.0f ? 1.0f - tail : tail;
}
template <bool FINE = false>
__device__ inline float act_value(float z, int act) {
    if (act == BAKRON_ACT_SILU) return z * sigmoid<FINE>(z);
    float g;
    if (act == BAKRON_ACT_GELU) return z * normal_cdf<FINE>(z, &g);
    return z;
}
__device__ inline void act_both(float z, int act, float* value, float* slope) {
    if (act == BAKRON_ACT_SILU) {
        const float s = sigmoid<false>(z);
        *value = z * s;
        *slope = s * (1.0f + z * (1.0f - s));
    } else {
        float g;
        const float c = normal_cdf<false>(z, &g);
        *value = z * c;
        *slope = fmaf(z * 0.39894228040143268f, g, c);
    }
}

}  // namespace bk
