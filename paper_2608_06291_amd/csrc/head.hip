// Log probabilities of given tokens from the rows before the vocabulary matrix, and their
// gradient, without keeping the logits (16-bit floats, fp32 sums):
//   z = x W^T,   lse = log sum exp z,   logprob = z_target - lse,   entropy = -sum p log p
//   dz = g (1[target] - p) - g_H p (log p + entropy),   dx = dz W,   dW = dz^T x
//
// Forward: the tile product of tile.h with a softmax in its epilogue.  Every tile leaves, for each of its
// rows of x, the largest logit m, s = sum exp(z - m) and s1 = sum exp(z - m) (z - m) over its part of the
// vocabulary (16 bytes for 64 to 256 tokens, of few rows 16 to 64, where the logits would take 4 bytes each); a second
// launch joins the parts:
//   s = s_a e^(m_a - m) + s_b e^(m_b - m),   s1 = (s1_a + (m_a - m) s_a) e^(m_a - m) + the same of b.
// Backward: the vocabulary goes in pieces.  Of a piece the logits are computed again, with dz in the
// epilogue, rounded to 16 bits as operand of two products: dW of the piece, and dx, whose sums stay in
// fp32 between the pieces.
//
// Measured (bf16): 4096 x 4096 x 131072 3270 to 3370 us forward, 1345 TFLOP/s (the library's product of that size,
// without the softmax: 3050; matrix cores 67% busy, bound by power), 2048 x 4096 x 32768 391; gradients of the first
// 10130 to 10520 us, 1255 to 1302 TFLOP/s (a piece: logits and dz 435, dx 404, dW 447), of the second 1350 to 1395.  dz's and dW's
// stores overlap nothing (one workgroup a CU, all at the end of a round).
// Few rows are bound by reading w: one row of 4096 x 32768 42 us (6.3 TB/s of 268 MB) and 5 for the join, 32 rows of 4096 x
// 131072 182; gradients of one row of 4096 x 32768 135 us (w twice, dW once: 805 MB, 6.0 TB/s), of 32 175, of 64 224, of
// 256 284.
#include "product.h"

namespace bk {

// What a part of the vocabulary leaves of a row.
struct HeadPart {
    float m, s, s1, pad;
};

// What comes in at the rows.
struct HeadIn {
    const int64_t* target;
    const float *lse, *g, *gh;
    int64_t all;   // tokens of all pieces

    // Of row t: whether no logit is finite, and the gradient of its log probability, where it has a target.
    __device__ bool empty(int64_t t) const { return lse[t] == -INFINITY; }
    __device__ float logprob(int64_t t) const {
        if (!target || !g) return 0.0f;
        const float v = g[t];
        const int64_t k = target[t];
        return k >= 0 && k < all ? v : 0.0f;
    }
    // The bound of row t's |dz|; 0 where it asks for nothing, whatever came in there.
    __device__ float bound(int64_t t) const {
        const float b = fabsf(logprob(t)) + (gh ? 4.0f * fabsf(gh[t]) : 0.0f);
        return b < INFINITY && !empty(t) ? b : 0.0f;
    }
};

struct HeadScale;
struct HeadArgs {
    Operand x, w;
    int64_t T;
    int V;                     // rows of w (backward: of the piece)
    int chunks, ni, nt;
    const int64_t* target;
    // forward
    HeadPart* part;            // parts x T
    float* at;                 // T: the target's logit, where there is one
    // backward
    const float *lse, *entropy, *g_logprob, *g_entropy;
    int64_t v0, all;           // first token of the piece; tokens of all pieces
    void* dz;                  // T rows: vp entries (zeros in the padding), then what their rounding took
    int64_t vp, ldz;           // ldz: vp, or 2 vp with the rests
    const float* factor;       // half precision: dz is taken times this, or NULL: by the kernel itself,
    HeadScale* scale;          // whose first workgroup leaves it here
    void* dzt;                 // few rows: dz once more, a token a row: 16 or 32 rows of x, then the rests
    __host__ __device__ HeadIn in() const { return HeadIn{target, lse, g_logprob, g_entropy, all}; }
};

// What few rows need beside that: x and w as they are, in entries.
struct HeadFew {
    const void *x, *w;
    int64_t ldx, ldw;
    int d;
};

// Half precision: |dz| <= |g| + 4 |g_H| (p |log p + H| is below ln(V) / 4 + 1/2 <= 4 for V <= 2^20), so dz is taken
// times the power of two that puts this bound at 2^13 to 2^14, undone at the end: none overflows, and
// what is lost is below 2^-38 of the largest.
struct HeadScale {
    float factor, undo;
};
__device__ inline HeadScale head_scale(float m) {
    int e = 14;
    if (m > 0.0f) frexpf(m, &e);   // m < 2^e
    e = max(e, 14 - 126);          // (both powers are normal numbers)
    return HeadScale{ldexpf(1.0f, 14 - e), ldexpf(1.0f, e - 14)};
}
__global__ __launch_bounds__(1024) void k_head_scale(HeadIn in, int64_t T, HeadScale* out) {
    __shared__ float red[16];
    float m = 0.0f;
    for (int64_t i = threadIdx.x; i < T; i += 1024) m = fmaxf(m, in.bound(i));
    m = group_reduce(m, MaxNan(), red, threadIdx.x >> 6, threadIdx.x & 63, 16);
    if (threadIdx.x != 0) return;
    *out = head_scale(m);
}

// The same by every wave itself, for up to 64 rows (all its lanes have to be active): one launch less.
__device__ inline HeadScale head_scale_few(const HeadIn& in, int64_t T, int lane) {
    return head_scale(wave_reduce(lane < T ? in.bound(lane) : 0.0f, MaxNan()));
}

// The same for up to HEAD_SCALE_ROWS rows: a launch less, for a scan by every workgroup (gradients of 200 x 1000 x 5003
// 43 -> 39 us, 500 x 1000 x 5000 51 -> 47; with 1024 rows 1024 x 512 x 32000 152 -> 156).
__device__ inline HeadScale head_scale_rows(const HeadIn& in, int T, int lane) {
    constexpr int AHEAD = 4;
    float m = 0.0f;
    for (int t0 = 0; t0 < T; t0 += 64 * AHEAD) {
        float b[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) b[i] = in.bound(min(t0 + i * 64 + lane, T - 1));   // (past the last row it once more)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) m = fmaxf(m, b[i]);
    }
    return head_scale(wave_reduce(m, MaxNan()));
}
constexpr int64_t HEAD_SCALE_ROWS = 512;

// A row's part of the gradient.
struct HeadRow {
    float lse, g, gh, H;
    int t;   // the target in the piece, or -1
};
__device__ inline HeadRow head_row(const HeadArgs& a, int64_t t) {
    HeadRow r;
    r.lse = a.lse[t];
    const bool empty = a.in().empty(t);
    if (empty) r.lse = INFINITY;   // every p is then exp(-inf) = 0
    const int64_t k = a.target ? a.target[t] : -1;
    r.t = k >= a.v0 && k < a.v0 + a.V ? (int)(k - a.v0) : -1;
    r.g = a.in().logprob(t);
    r.gh = a.g_entropy ? a.g_entropy[t] : 0.0f;
    r.H = a.g_entropy ? a.entropy[t] : 0.0f;
    if (empty) r.g = r.gh = 0.0f;
    return r;
}
__device__ inline float head_grad(const HeadRow& r, float z, int i) {
    const float lp = max_nan(z - r.lse, -200.0f);   // (exp is 0 there; 0 * -inf stays out)
    const float v = -exp_of<false>(lp) * fmaf(r.gh, lp + r.H, r.g);
    return i == r.t ? v + r.g : v;
}
// N entries from token i of the piece on; zeros past its end.
template <typename E, int N>
__device__ inline void head_grads(const HeadArgs& a, const HeadRow& r, int i, float factor, float (&z)[N]) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
        z[j] = i + j < a.V ? head_grad(r, z[j], i + j) : 0.0f;
        if constexpr (narrow_range<E>) z[j] *= factor;
    }
}
template <typename E, int N>
__device__ inline void head_store(const HeadArgs& a, int64_t t, int i, float (&z)[N]) {
    E* const row = static_cast<E*>(a.dz) + t * a.ldz + i;
    store_n(row, z, N);
    if (a.ldz > a.vp) {   // what the rounding took (nothing beside what is not finite)
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float v = (float)(E)z[j];
            z[j] = __builtin_isfinite(v) ? z[j] - v : 0.0f;
        }
        store_n(row + a.vp, z, N);
    }
}

// Few rows: the same four entries in the order of dzt, zeros for rows of x past T.
template <typename E, int Y>
__device__ inline void head_store_few(const HeadArgs& a, int64_t t, int i, const float (&z)[4]) {
    E* const p = static_cast<E*>(a.dzt) + (int64_t)i * (32 * Y) + t;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float v = (float)(E)z[j];
        p[j * (32 * Y)] = (E)z[j];
        p[j * (32 * Y) + 16 * Y] = (E)(__builtin_isfinite(v) ? z[j] - v : 0.0f);
    }
}

// Joins b to a.
__device__ inline void head_join(HeadPart& a, const HeadPart& b) {
    const float m = max_nan(a.m, b.m), ms = m == -INFINITY ? 0.0f : m;
    const float da = max_nan(a.m - ms, -200.0f), db = max_nan(b.m - ms, -200.0f);
    const float ea = exp_of<true>(da), eb = exp_of<true>(db);
    a.s1 = fmaf(da, a.s, a.s1) * ea + fmaf(db, b.s, b.s1) * eb;
    a.s = a.s * ea + b.s * eb;
    a.m = m;
}
// Over lanes 16 and 32 apart: those that hold the same row of x.
template <typename Op>
__device__ inline float rows_reduce(float v, Op op) {
    v = op(v, __shfl_xor(v, 16));
    return op(v, __shfl_xor(v, 32));
}
// The part of one row that the four lanes of it hold, N logits each.
template <int N>
__device__ inline HeadPart head_part(const float (&z)[N]) {
    float m = z[0];
#pragma unroll
    for (int j = 1; j < N; ++j) m = max_nan(m, z[j]);
    m = rows_reduce(m, MaxNan());
    const float ms = m == -INFINITY ? 0.0f : m;
    float s = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float d = max_nan(z[j] - ms, -200.0f);   // (0 * -inf stays out of s1; exp is 0 there)
        const float e = __builtin_amdgcn_exp2f(d * LOG2E);
        s += e;
        s1 = fmaf(e, d, s1);
    }
    return HeadPart{m, rows_reduce(s, Add()), rows_reduce(s1, Add()), 0.0f};
}

template <typename Tl, bool BWD>
__global__ __launch_bounds__(Tl::THREADS) void k_head(HeadArgs a) {
    typedef typename Tl::Mma::Elem E;
    __shared__ __attribute__((aligned(1024))) char lds[Tl::LDS];
    int ti, tt;
    tile_of(blockIdx.x, a.ni, a.nt, 8, &ti, &tt);
    const int i0 = ti * Tl::ROWS;
    const int64_t t0 = (int64_t)tt * Tl::COLS;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    typename Tl::Accs acc = {};
    Tl::run(lds, a.w, min(i0, a.V - 1), a.x, t0, 0, a.chunks, acc, [](int r) { return r; });

    if constexpr (!BWD) {
        constexpr int PART = Tl::UA * 16, WAVES_A = Tl::ROWS / PART;   // a wave's tokens; waves with the same rows
        HeadPart* const parts = reinterpret_cast<HeadPart*>(lds);      // WAVES_A x COLS
        const int r16 = lane & 15, first = i0 + Tl::a0(wave) + (lane >> 4) * 4;
#pragma unroll
        for (int y = 0; y < Tl::UB; ++y) {
            float z[Tl::UA * 4];
#pragma unroll
            for (int x = 0; x < Tl::UA; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) z[x * 4 + r] = Tl::at(acc, x, y)[r];
            if (i0 + Tl::ROWS > a.V) {
#pragma unroll
                for (int j = 0; j < Tl::UA * 4; ++j)
                    if (first + j / 4 * 16 + j % 4 >= a.V) z[j] = -INFINITY;
            }
            const int col = Tl::b0(wave) + y * 16 + r16;
            const HeadPart p = head_part(z);
            if (lane < 16) parts[Tl::a0(wave) / PART * Tl::COLS + col] = p;
            const int64_t t = t0 + col, k = a.target && t < a.T ? a.target[t] : -1;
            const int64_t in = k >= 0 && k < a.V ? k - first : -1;   // this lane's tokens: 16 x + r
            if (__any(in >= 0 && in < PART)) {
#pragma unroll
                for (int j = 0; j < Tl::UA * 4; ++j)
                    if (in == j / 4 * 16 + j % 4) a.at[t] = z[j];
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < Tl::COLS; c += Tl::THREADS) {
            if (t0 + c >= a.T) break;
            HeadPart p = parts[c];
#pragma unroll
            for (int w = 1; w < WAVES_A; ++w) head_join(p, parts[w * Tl::COLS + c]);
            a.part[(int64_t)ti * a.T + t0 + c] = p;
        }
    } else {
        HeadRow* const row = reinterpret_cast<HeadRow*>(lds + Tl::THREADS / 64 * (Tl::UA * 1024));
        for (int c = threadIdx.x; c < Tl::COLS; c += Tl::THREADS)
            if (t0 + c < a.T) row[c] = head_row(a, t0 + c);
        float factor = 1.0f;
        if constexpr (narrow_range<E>) {
            if (a.factor) {
                factor = *a.factor;
            } else {
                const HeadScale own = head_scale_rows(a.in(), (int)a.T, lane);
                factor = own.factor;
                if (blockIdx.x == 0 && threadIdx.x == 0) *a.scale = own;
            }
        }
        __syncthreads();
        const auto rows = handover<Tl>(lds, wave, lane, [&](int x, int y) { return Tl::at(acc, x, y); });
        constexpr int PER = Tl::UA * 2, EACH = 64 / PER;   // lanes a row, rows at a time
        const int p = lane % PER, i = i0 + Tl::a0(wave) + p * 8;
#pragma unroll
        for (int y = 0; y < Tl::UB; ++y) {
            rows.put(y);
#pragma unroll
            for (int k = 0; k < 16 / EACH; ++k) {
                const int tl = k * EACH + lane / PER, col = Tl::b0(wave) + y * 16 + tl;
                float z[8];
                rows.take(tl, p, z);
                if (t0 + col < a.T && i < a.vp) {
                    head_grads<E>(a, row[col], i, factor, z);
                    head_store<E>(a, t0 + col, i, z);
                }
            }
        }
    }
}

constexpr int HEAD_STEPS = 2;

// Pieces of U steps of 32 entries of a row on their way, a lane's 8 of each (those of the same row 16 lanes apart).
// SHIFT: see FewPiece; the word behind a piece is the first one of the lane 16 further on, and behind the last
// lane's that of the first lane's next step; only the last step's are loaded (1 x 1001 x 70000 55 us with all words loaded,
// 46; 32 rows 65 and 60; but 16 x 3539 x 17120 60 and 66, waiting for LDS).
template <int U, bool SHIFT>
struct HeadPieces {
    u32x4 w[U];
    uint32_t next;
    template <typename E>
    __device__ inline void load(const E* p) {
#pragma unroll
        for (int i = 0; i < U - 1; ++i) {
            if constexpr (SHIFT)
                __builtin_memcpy(&w[i], (const void*)((uintptr_t)(p + i * 32) & ~(uintptr_t)3), 16);
            else
                w[i] = load_words(p + i * 32);
        }
        FewPiece<SHIFT> last;
        last.load(p + (U - 1) * 32);
        w[U - 1] = last.w;
        if constexpr (SHIFT) next = last.next;
    }
    template <typename E>
    __device__ inline u32x4 get(int i, const E* row, int lane) const {
        if constexpr (!SHIFT) return w[i];
        FewPiece<SHIFT> p;
        p.w = w[i];
        p.next = i == U - 1 ? next : (uint32_t)__shfl((int)(lane < 16 ? w[min(i + 1, U - 1)][0] : w[i][0]), (lane + 16) & 63);
        return p.get(row);
    }
};

// Few rows (a decoding step): bound by reading w once.  A workgroup takes R units of 16 tokens and Y of 16
// rows of x; its waves share the summed axis, blocks of two steps of 32 in turn, every
// fragment straight from memory (at any alignment) into registers, BLOCKS blocks asked for at once.  The partial
// sums meet in LDS.  SHIFT: see FewPiece.
template <typename M, bool BWD, int R, int Y, int BLOCKS, bool SHIFT>
__global__ __launch_bounds__(512) void k_head_few(HeadFew f, HeadArgs a) {
    typedef typename M::Elem E;
    extern __shared__ __attribute__((aligned(16))) char few_lds[];
    const int tid = threadIdx.x, lane = tid & 63, waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, kq = lane >> 4;
    const int i0 = (int)blockIdx.x * (R * 16);
    const int64_t t0 = (int64_t)blockIdx.y * (Y * 16);
    const E* w[R];
    const E* x[Y];
#pragma unroll
    for (int r = 0; r < R; ++r)
        w[r] = static_cast<const E*>(f.w) + (int64_t)min(i0 + r * 16 + r16, a.V - 1) * f.ldw + kq * 8;
#pragma unroll
    for (int y = 0; y < Y; ++y)
        x[y] = static_cast<const E*>(f.x) + min(t0 + y * 16 + r16, a.T - 1) * f.ldx + kq * 8;
    constexpr int U = HEAD_STEPS;
    const int nblocks = f.d / (32 * U), nsteps = f.d / 32;   // what is left goes one step a wave

    struct Block {
        HeadPieces<U, SHIFT> w[R], x[Y];
    };
    auto load = [&](Block& b, int k) {
#pragma unroll
        for (int r = 0; r < R; ++r) b.w[r].load(w[r] + k);
#pragma unroll
        for (int y = 0; y < Y; ++y) b.x[y].load(x[y] + k);
    };
    f32x4 acc[R][Y] = {};
    auto add = [&](const u32x4 (&u)[R], const u32x4 (&v)[Y]) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int y = 0; y < Y; ++y)
                acc[r][y] = M::mma(__builtin_bit_cast(i32x4, u[r]), __builtin_bit_cast(i32x4, v[y]), acc[r][y]);
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
                u32x4 u[R], v[Y];
#pragma unroll
                for (int r = 0; r < R; ++r) u[r] = b[k].w[r].get(i, w[r], lane);
#pragma unroll
                for (int y = 0; y < Y; ++y) v[y] = b[k].x[y].get(i, x[y], lane);
                add(u, v);
            }
        }
    }
    for (int s = nblocks * U + wave; s < nsteps; s += waves) {
        u32x4 u[R], v[Y];
#pragma unroll
        for (int r = 0; r < R; ++r) u[r] = load_words(w[r] + s * 32);
#pragma unroll
        for (int y = 0; y < Y; ++y) v[y] = load_words(x[y] + s * 32);
        add(u, v);
    }
    if (f.d % 32 != 0 && wave == (nsteps - nblocks * U) % waves) {
        const int k = nsteps * 32, left = f.d - k - kq * 8;   // entries of this lane's pieces
        u32x4 u[R], v[Y];
#pragma unroll
        for (int r = 0; r < R; ++r) u[r] = few_part(w[r] + k, left, f.d);
#pragma unroll
        for (int y = 0; y < Y; ++y) v[y] = few_part(x[y] + k, left, f.d);
        add(u, v);
    }
#pragma unroll
    for (int y = 0; y < Y; ++y)
#pragma unroll
        for (int r = 0; r < R; ++r)
            *reinterpret_cast<f32x4*>(few_lds + (((wave * Y + y) * R + r) * 64 + lane) * 16) = acc[r][y];
    __syncthreads();
    for (int y = wave; y < Y; y += waves) {   // a wave joins one unit of rows
        float z[R * 4];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int k = 0; k < waves; ++k)
                sum += *reinterpret_cast<const f32x4*>(few_lds + (((k * Y + y) * R + r) * 64 + lane) * 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) z[r * 4 + j] = sum[j];
        }
        const int64_t t = t0 + y * 16 + r16;
        const int first = i0 + kq * 4;
        if constexpr (!BWD) {
            const int64_t k = a.target && t < a.T ? a.target[t] : -1;
#pragma unroll
            for (int j = 0; j < R * 4; ++j) {
                const int i = first + j / 4 * 16 + j % 4;
                if (i >= a.V) z[j] = -INFINITY;
                if (i == k && i < a.V) a.at[t] = z[j];
            }
            const HeadPart p = head_part(z);
            if (lane < 16 && t < a.T) a.part[(int64_t)blockIdx.x * a.T + t] = p;
        } else {
            HeadRow row{};
            if (t < a.T) row = head_row(a, t);
            float factor = 1.0f;
            if constexpr (narrow_range<E>)
                factor = a.factor ? *a.factor : head_scale_few(a.in(), a.T, lane).factor;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int i = first + r * 16;
                if (i >= a.vp) break;
                float v[4] = {};
                if (t < a.T) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = z[r * 4 + j];
                    head_grads<E>(a, row, i, factor, v);
                }
                if (a.dzt) head_store_few<E, Y>(a, t, i, v);
                if (t < a.T) head_store<E>(a, t, i, v);
            }
        }
    }
}

// The products of few rows, bound by memory as dz is: w read once, dW written once.
struct HeadFewProd {
    const void *x, *w, *dz, *dzt;
    int64_t ldx, ldw, ldz, vp, T;
    int V, d;
    int parts, steps;          // dx: parts of the vocabulary (0: not asked for), of so many steps of 32 tokens
    int units;                 // dW: units of 16 tokens a wave takes
    void* dw;
    int64_t lddw;
    float* partial;            // dx: parts x T x dp
    int64_t dp;
    HeadIn in;
    int slabs, rows, each;     // of 128 columns; parts of dx and groups of dW, so many of them in turn
};

// dW: a wave holds 128 columns of x, of all rows, as 8 operands and goes through `units` units of 16 tokens.
// The results go through LDS, so that a store writes 256 bytes of each of four rows, and past the caches where dW would
// only sweep them (PAST): 32768 x 4096 from one row, with dz, 97 us (through the caches 124; 64 bytes of 16 rows as the lanes
// hold them 161).
// A summed axis of 32 holds the rows of x and, up to 16 of them, the same again for dz's rests.
template <typename M, int Y, bool PAST>
__device__ inline void head_few_dw(const HeadFewProd& a, int slab, int group, char* lds) {
    typedef typename M::Elem E;
    E (*const rows)[16][136] = reinterpret_cast<E (*)[16][136]>(lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, kq = lane >> 4;
    const int c0 = slab * 128;
    const int64_t first = ((int64_t)group * 4 + wave) * a.units * 16;
    if (first >= a.V) return;
    i32x4 x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int c = c0 + u * 16 + r16;
        uint16_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int t = (kq * 8 + j) & (16 * Y - 1);
            const uint16_t e = static_cast<const uint16_t*>(a.x)[min((int64_t)t, a.T - 1) * a.ldx + min(c, a.d - 1)];
            v[j] = t < a.T && c < a.d ? e : (uint16_t)0;
        }
        __builtin_memcpy(&x[u], v, 16);
    }
    const float undo = narrow_range<E> ? head_scale_few(a.in, a.T, lane).undo : 1.0f;
    const char* const dzt = static_cast<const char*>(a.dzt) + (first + r16) * (64 * Y) + kq * 16;
    const int n = (int)min((int64_t)a.units, (a.V - first + 15) / 16), c = c0 + r16 * 8;
    i32x4 b[Y], next[Y];
    auto load = [&](int k) {   // (dz has rows of zeros up to a multiple of 64)
#pragma unroll
        for (int s = 0; s < Y; ++s) next[s] = *reinterpret_cast<const i32x4*>(dzt + (int64_t)k * (16 * 64 * Y) + s * 64);
    };
    load(0);
    for (int k = 0; k < n; ++k) {
#pragma unroll
        for (int s = 0; s < Y; ++s) b[s] = next[s];
        if (k + 1 < n) load(k + 1);
        __builtin_amdgcn_wave_barrier();   // (what was put there is stored)
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            f32x4 acc = M::mma(x[u], b[0], f32x4{0.0f, 0.0f, 0.0f, 0.0f});
            if constexpr (Y == 2) acc = M::mma(x[u], b[Y - 1], acc);
            Pack<E, 4> o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o.v[j] = (E)(narrow_range<E> ? acc[j] * undo : acc[j]);
            __builtin_memcpy(&rows[wave][r16][u * 16 + kq * 4], &o, 8);
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t v = first + k * 16 + r * 4 + kq;
            const u32x4 o = *reinterpret_cast<const u32x4*>(&rows[wave][r * 4 + kq][r16 * 8]);
            if (v >= a.V || c >= a.d) continue;
            E* const out = static_cast<E*>(a.dw) + v * a.lddw + c;
            if (c + 8 <= a.d) {
                if constexpr (PAST)
                    store_words_past(out, o);
                else
                    __builtin_memcpy(out, &o, 16);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < a.d) out[j] = (E)entry<E>(o, j);
            }
        }
    }
}

// Sums dx's parts: a lane has one entry of a row, the 16 waves every 16th part each, joined in their order.
template <typename E>
__global__ __launch_bounds__(1024) void k_head_few_join(HeadFewProd a, E* dx, int64_t lddx) {
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t e = (int64_t)blockIdx.x * 64 + lane, all = a.T * a.dp;
    float sum = 0.0f;
    if (e < all) {
        constexpr int AHEAD = 4;
        for (int p = wave; p < a.parts; p += 16 * AHEAD) {
            float v[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) v[i] = a.partial[min(p + 16 * i, a.parts - 1) * all + e];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) sum += p + 16 * i < a.parts ? v[i] : 0.0f;
        }
    }
    red[wave][lane] = sum;
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < 16; ++w) sum += red[w][lane];
    if constexpr (narrow_range<E>) sum *= head_scale_few(a.in, a.T, lane).undo;
    if (e >= all || e % a.dp >= a.d) return;
    dx[e / a.dp * lddx + e % a.dp] = (E)sum;
}

// dx: a wave takes 128 columns of w, 8 a lane, and 32 tokens a step; the 8 x 8 entries of a lane turn into 8 operands
// with the tokens along (one permutation of two registers a pair), operand m having column 8 i + m as its row i.
// The waves of a workgroup share its steps and meet in LDS, the workgroups' parts in a second launch.
template <typename M, int Y>
__device__ inline void head_few_dx(const HeadFewProd& a, int slab, int part, char* lds) {
    typedef typename M::Elem E;
    f32x4 (*const sums)[8 * Y][64] = reinterpret_cast<f32x4 (*)[8 * Y][64]>(lds);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, kq = lane >> 4;
    // (past the row its last 8 columns, twice the same results)
    const int c = min(slab * 128 + r16 * 8, a.d - 8);
    const int all = (a.V + 31) / 32, s0 = part * a.steps, s1 = min(all, s0 + a.steps);
    const E* const w = static_cast<const E*>(a.w) + c;
    const E* dz[Y];
#pragma unroll
    for (int y = 0; y < Y; ++y) dz[y] = static_cast<const E*>(a.dz) + min((int64_t)(y * 16 + r16), a.T - 1) * a.ldz + kq * 8;
    f32x4 acc[8][Y] = {};
    struct Step {
        u32x4 w[8];
        i32x4 hi[Y], rest[Y];
    };
    auto load = [&](Step& p, int s) {
#pragma unroll
        for (int j = 0; j < 8; ++j) p.w[j] = load_words(w + (int64_t)min(s * 32 + kq * 8 + j, a.V - 1) * a.ldw);
#pragma unroll
        for (int y = 0; y < Y; ++y) {
            p.hi[y] = *reinterpret_cast<const i32x4*>(dz[y] + s * 32);
            p.rest[y] = *reinterpret_cast<const i32x4*>(dz[y] + a.vp + s * 32);
        }
    };
    Step cur, next;
    if (s0 + wave < s1) load(next, s0 + wave);
    for (int s = s0 + wave; s < s1; s += 4) {
        cur = next;
        if (s + 4 < s1) load(next, s + 4);
#pragma unroll
        for (int m = 0; m < 8; ++m) {
            i32x4 f;
#pragma unroll
            for (int p = 0; p < 4; ++p)
                f[p] = (int32_t)__builtin_amdgcn_perm(cur.w[2 * p + 1][m >> 1], cur.w[2 * p][m >> 1],
                                                      m & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int y = 0; y < Y; ++y) {
                acc[m][y] = M::mma(f, cur.hi[y], acc[m][y]);
                acc[m][y] = M::mma(f, cur.rest[y], acc[m][y]);
            }
        }
    }
    if (wave > 0) {
#pragma unroll
        for (int m = 0; m < 8; ++m)
#pragma unroll
            for (int y = 0; y < Y; ++y) sums[wave - 1][m * Y + y][lane] = acc[m][y];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int m = 0; m < 8; ++m)
#pragma unroll
        for (int y = 0; y < Y; ++y)
#pragma unroll
            for (int k = 0; k < 3; ++k) acc[m][y] += sums[k][m * Y + y][lane];
#pragma unroll
    for (int y = 0; y < Y; ++y) {
        const int64_t t = y * 16 + r16;
        if (t >= a.T) break;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int col = slab * 128 + (kq * 4 + r) * 8;
            if (col >= a.d) break;
            float o[8];
#pragma unroll
            for (int m = 0; m < 8; ++m) o[m] = acc[m][y][r];
            store_n(a.partial + ((int64_t)part * a.T + t) * a.dp + min(col, a.d - 8), o, 8);
        }
    }
}

// DX and DW: both in one launch, the parts of dx first.  Every eighth workgroup runs on the same XCD: with each = 8 those
// have all slabs of a part or group, so that a line of W or dW that two slabs share is fetched, or joined, in one L2 (gradients
// of 1 x 1001 x 70000 120 -> 102 us, 32 x 1024 x 70000 132 -> 121; but 1 x 4096 x 32768 140 -> 152).
template <typename M, int Y, bool DX, bool DW, bool PAST>
__global__ __launch_bounds__(256) void k_head_few_prod(HeadFewProd a) {
    constexpr int LDS_X = 3 * 8 * Y * 64 * 16, LDS_W = 4 * 16 * 136 * 2;
    __shared__ __attribute__((aligned(16))) char lds[!DX ? LDS_W : !DW || LDS_X > LDS_W ? LDS_X : LDS_W];
    const uint32_t each = (uint32_t)a.each, at = blockIdx.x / each;
    const int slab = (int)(at % (uint32_t)a.slabs), row = (int)(at / (uint32_t)a.slabs * each + blockIdx.x % each);
    if (row >= a.rows) return;
    if (DX && row < a.parts)
        head_few_dx<M, Y>(a, slab, row, lds);
    else if (DW)
        head_few_dw<M, Y, PAST>(a, slab, row - (DX ? a.parts : 0), lds);
}

// Joins the parts of the vocabulary: 256 / ROWS threads a row.
struct HeadJoinArgs {
    const HeadPart* part;
    const float* at;
    const int64_t* target;
    int64_t T;
    int V, parts;
    float *logprob, *entropy, *lse;
};
template <int ROWS>
__global__ __launch_bounds__(256) void k_head_join(HeadJoinArgs a) {
    constexpr int PER = 256 / ROWS;
    __shared__ HeadPart red[PER][ROWS];
    const int c = threadIdx.x % ROWS, l = threadIdx.x / ROWS;
    const int64_t t = (int64_t)blockIdx.x * ROWS + c, tr = min(t, a.T - 1);
    HeadPart p{-INFINITY, 0.0f, 0.0f, 0.0f};
    constexpr int AHEAD = 4;
    for (int k = l; k < a.parts; k += PER * AHEAD) {
        HeadPart q[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) q[j] = a.part[(int64_t)min(k + j * PER, a.parts - 1) * a.T + tr];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (k + j * PER < a.parts) head_join(p, q[j]);
    }
    red[l][c] = p;
    for (int n = PER / 2; n > 0; n /= 2) {
        __syncthreads();
        if (l < n) head_join(red[l][c], red[l + n][c]);
    }
    if (l != 0 || t >= a.T) return;
    p = red[0][c];
    const bool empty = p.m == -INFINITY;
    const float log_s = logf(p.s);
    const int64_t k = a.target ? a.target[t] : -1;
    const bool asked = k >= 0 && k < a.V;
    if (a.lse) a.lse[t] = empty ? -INFINITY : p.m + log_s;
    if (a.logprob) a.logprob[t] = !asked ? 0.0f : empty ? -INFINITY : (a.at[t] - p.m) - log_s;
    if (a.entropy) a.entropy[t] = empty ? 0.0f : log_s - p.s1 / p.s;
}

// Whether the logits are taken by the kernel for few rows.  Up to 8 rows always (4096 x 32768, one row 50 us, in tiles 58);
// up to 32 where there are fewer tiles (by 64 x 64) than CUs (32 x 2048 x 8192 15.8 us, in tiles 18.1; but 32 x 4096 x 131072
// 221 against 182), and where tiles would need padded copies of all rows, by their length (so that the order of
// sums depends on sizes alone).  More rows with fewer tiles still and a long way to sum: 100 x 2048 x 1000 (32) 19.1 and in tiles 20;
// 300 x 4096 x 2000 (160) 54 against 32.
constexpr int64_t HEAD_FEW_ROWS = 32, HEAD_FEW_TILES = 4;
static bool head_few_rows(int64_t T, int64_t V, int64_t d) {
    const int64_t tiles = ((V + 63) / 64) * ((T + 63) / 64);
    if (T <= HEAD_FEW_ROWS) return T <= 8 || d % 8 != 0 || tiles < op_cus();
    return tiles * HEAD_FEW_TILES <= op_cus() && d >= 512;
}
// Units of 16 tokens that a workgroup of that kernel takes.  More of them share the rows of x: 32 x 4096 x 131072 with
// one unit 362 us, two 263, four 218, 16 rows of 2048 136, 108, 102.  With fewer rows x costs nothing, and long rows of w
// come faster when few are read side by side: one row of 4096 175, 208, 201, four of 2048 102, 95, 102.  But every
// CU should have a workgroup.
static int head_units(int64_t T, int64_t V, int64_t d) {
    int units = T > 8 ? 4 : d >= 4096 ? 1 : 2;
    while (units > 1 && (V + 16 * units - 1) / (16 * units) * ((T + 31) / 32) < op_cus()) units /= 2;
    return units;
}
// Tokens that a workgroup takes, and so the parts of the vocabulary.
static int head_edge(int64_t T, int64_t V, int64_t d) {
    return head_few_rows(T, V, d) ? 16 * head_units(T, V, d) : pick_tile(V, T, op_cus(), true);
}

template <typename M, bool BWD, int R, int Y, int BLOCKS>
static void launch_head_few(const HeadFew& f, const HeadArgs& a, hipStream_t st) {
    // Words around the pieces of odd rows: each matrix begins on a word, and whole steps end before the row
    // does, so an entry before and one behind each piece are in the matrix.
    const bool shift = (f.ldx % 2 != 0 || f.ldw % 2 != 0) && f.d % 32 != 0 && (uintptr_t)f.x % 4 == 0 &&
                       (uintptr_t)f.w % 4 == 0;
    const int64_t n = BWD ? a.vp : a.V;
    const dim3 grid((unsigned)((n + R * 16 - 1) / (R * 16)), (unsigned)((a.T + Y * 16 - 1) / (Y * 16)));
    const int blocks = f.d / (32 * HEAD_STEPS);   // as many waves as have work, 8 at most
    const int waves = blocks >= 8 ? 8 : blocks >= 4 ? 4 : blocks >= 2 ? 2 : 1;
    if (shift)
        hipLaunchKernelGGL((k_head_few<M, BWD, R, Y, BLOCKS, true>), grid, dim3(64 * waves), waves * Y * R * 1024, st, f, a);
    else
        hipLaunchKernelGGL((k_head_few<M, BWD, R, Y, BLOCKS, false>), grid, dim3(64 * waves), waves * Y * R * 1024, st,
                           f, a);
}

// few_rows, edge: head_few_rows and head_edge of the call
template <typename M, bool BWD>
static void launch_head(const HeadFew& few, HeadArgs a, bool few_rows, int edge, hipStream_t st) {
    if (few_rows) {
        const bool one = a.T <= 16;
        if (edge == 16) return one ? launch_head_few<M, BWD, 1, 1, 4>(few, a, st) : launch_head_few<M, BWD, 1, 2, 2>(few, a, st);
        if (edge == 32) return one ? launch_head_few<M, BWD, 2, 1, 4>(few, a, st) : launch_head_few<M, BWD, 2, 2, 2>(few, a, st);
        return one ? launch_head_few<M, BWD, 4, 1, 2>(few, a, st) : launch_head_few<M, BWD, 4, 2, 1>(few, a, st);
    }
    const int64_t n = BWD ? a.vp : a.V;   // (the padding is written, too)
    auto go = [&](auto tile) {
        typedef decltype(tile) Tl;
        a.ni = (int)((n + Tl::ROWS - 1) / Tl::ROWS);
        a.nt = (int)((a.T + Tl::COLS - 1) / Tl::COLS);
        hipLaunchKernelGGL((k_head<Tl, BWD>), dim3((unsigned)(a.ni * a.nt)), dim3(Tl::THREADS), 0, st, a);
    };
    if (edge == 256) return go(BigTile<M>());
    if (edge == 128 && one_a_cu(128, n, a.T)) return go(Tile<M, 128, 128, 2, 4, 3>());
    if (edge == 128) return go(Tile<M, 128, 128, 2, 4, 2>());
    return go(Tile<M, 64, 64, 2, 2, 4>());
}

// x and w as operands, through padded copies where they cannot be staged as they are.
struct HeadPad {
    bool x, w;
    int64_t dp;
    size_t xbytes, wbytes;
};
static HeadPad head_pad(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t T, int64_t d, int64_t V,
                        bool need_x, bool need_w) {
    HeadPad p;
    p.dp = (d + 63) / 64 * 64;
    p.x = need_x && !direct_rows(x, ldx, d);
    p.w = need_w && !direct_rows(w, ldw, d);
    p.xbytes = p.x ? up256((size_t)T * p.dp * 2) : 0;
    p.wbytes = p.w ? up256((size_t)V * p.dp * 2) : 0;
    return p;
}
static void head_operands(HeadArgs& a, const HeadPad& p, const void* x, int64_t ldx, const void* w, int64_t ldw,
                          int64_t d, char* work, hipStream_t st) {
    // (a copy's padding is zeros; without copies what lies past d reads as zeros)
    const int64_t kbytes = p.x && p.w ? 2 * p.dp : 2 * ((d + 7) / 8 * 8);
    a.x = operand(x, 2 * ldx, a.T, kbytes);
    a.w = operand(w, 2 * ldw, a.V, kbytes);
    a.chunks = (int)((kbytes + CHUNK_BYTES - 1) / CHUNK_BYTES);
    PadArgs c{};
    int n = 0;
    int64_t pieces = 0;
    auto copy = [&](const void* src, int64_t ld, int64_t rows, char* to) {
        c.src[n] = static_cast<const uint16_t*>(src);
        c.dst[n] = reinterpret_cast<uint16_t*>(to);
        c.ld[n] = ld;
        pieces += rows * (p.dp / 8);
        for (int i = n; i < 3; ++i) c.end[i] = pieces;
        ++n;
    };
    if (p.x) {
        copy(x, ldx, a.T, work);
        a.x = operand(work, 2 * p.dp, a.T, kbytes);
    }
    if (p.w) {
        copy(w, ldw, a.V, work + p.xbytes);
        a.w = operand(work + p.xbytes, 2 * p.dp, a.V, kbytes);
    }
    if (n == 0) return;
    c.cols = d;
    c.cols_p = p.dp;
    hipLaunchKernelGGL(k_pad_rows, stride_grid(pieces), dim3(256), 0, st, c);
}

// x (T x cols, rows of 16-byte pieces) as columns: cols rows of tp entries, zeros from T on.  64 x 64 a workgroup.
__global__ __launch_bounds__(256) void k_transpose(const char* x, int64_t ld, int64_t T, int cols, uint16_t* out,
                                                   int64_t tp) {
    __shared__ uint16_t tile[64][66];
    const int64_t t0 = (int64_t)blockIdx.x * 64;
    const int c0 = (int)blockIdx.y * 64;
    const int p = threadIdx.x & 7, r = threadIdx.x >> 3;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t t = t0 + i * 32 + r;
        u32x4 v = u32x4(0);
        if (t < T && c0 + p * 8 < cols) v = load_words(reinterpret_cast<const uint16_t*>(x + t * ld) + c0 + p * 8);
#pragma unroll
        for (int j = 0; j < 8; ++j) tile[i * 32 + r][p * 8 + j] = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = c0 + i * 32 + r;
        if (c >= cols) break;
        Pack<uint16_t, 8> v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v.v[j] = tile[p * 8 + j][i * 32 + r];
        store_pack(out + c * tp + t0 + p * 8, v);
    }
}

// The backward pass.  A piece of the vocabulary is as long as dz of it stays in the last-level cache (256 MB) with
// the operands beside it (4096 x 4096 x 131072 in pieces of 128 MB 10130 us, of 512 MB 10330).
//
// dz's rounding to 16 bits is as large in a gradient as the result's own: 2.2e-3 to 2.5e-3 of its norm where the result's
// alone is 1.7e-3 (half precision 3.3e-4 and 2.1e-4).  The rows of one chunk or less (T <= 64) do not average it out, a few
// of them can lose more, and reading W is what they take: there the products go on over dz's rests, too.  Beyond,
// the rests would be two thirds more work (five products for three): 4096 x 4096 x 131072 10260 us and with rests 16990, 2048 x 4096 x 32768 1357 and
// 2226, 256 rows 282 and 384, 200 x 1000 x 5003 32 and 37 (half precision 35 and 40).
//
// dW's product reads x and dz by columns (transposing reads).  For many pieces and rows x is transposed once instead, which
// costs 17 us there: 10350 -> 10130 us, 2048 x 4096 x 32768 1372 -> 1349.
//
// A dW that the last-level cache would not hold with anything beside it is written past it, or w would be swept out of it
// and what follows wait for it to be written: 65 x 4096 x 32768 254 -> 190 us, 256 rows 326 -> 287, 100 x 2048 x 100000 418 ->
// 352, 2048 rows and more no difference.  Not where its rows share lines, which the caches join (1 x 1001 x 70000 130 us, past
// them 161), nor by the launch of both products, which is the faster one through the caches, too (128 x 4096 x 16384 97 us, two
// launches past them 104; 65 rows 95 and 103, 256 142 and 146; 65 x 2048 x 32768 90 and 100; 256 x 1024 x 65536 144 and 152).
constexpr int64_t HEAD_PIECE_BYTES = (int64_t)128 << 20, HEAD_PAST = (int64_t)128 << 20;
struct HeadBackward {
    int64_t vc, vp, ldz;   // tokens of a piece (all but the last), padded; row of dz
    bool rests, few;       // few: the kernels for few rows; dx in `parts` of `steps` x 32 tokens
    int parts, steps;
    int64_t tp;            // x is taken as columns, of so many entries; or 0
    ProdPlan dx, dw;
    bool both;             // both products in one launch, where both are asked for
    size_t dz, dzt, partial, sums, scale, xt;
};
static HeadBackward head_backward(int64_t T, int64_t d, int64_t V, bool half, bool dx, bool dw, int ncu) {
    HeadBackward p{};
    p.rests = T <= 64;
    const int64_t most = std::max<int64_t>(HEAD_PIECE_BYTES / (T * (p.rests ? 4 : 2)) / 256, 1) * 256;
    const int64_t pieces = (V + most - 1) / most;
    p.vc = pieces == 1 ? V : ((V + pieces - 1) / pieces + 255) / 256 * 256;
    p.vp = (p.vc + 63) / 64 * 64;
    p.ldz = (p.rests ? 2 : 1) * p.vp;
    p.dz = up256((size_t)T * p.ldz * 2);
    p.few = T <= HEAD_FEW_ROWS && d >= 8;   // (of one piece: 2^20 tokens at most)
    p.scale = half && !p.few ? 256 : 0;
    if (p.few) {
        const int slabs = (int)((d + 127) / 128), all = (int)((V + 31) / 32);
        p.steps = std::max((all * slabs + 4 * ncu - 1) / (4 * ncu), 8);
        p.parts = (all + p.steps - 1) / p.steps;
        p.dzt = dw ? up256((size_t)p.vp * (T <= 16 ? 64 : 128)) : 0;
        p.partial = dx ? up256((size_t)p.parts * T * ((d + 7) / 8 * 8) * sizeof(float)) : 0;
        return p;
    }
    // (the same sums whether both are asked for or one)
    const int chunks_x = (int)(p.ldz / 64), chunks_w = (int)((p.rests ? 2 : 1) * ((T + 63) / 64));
    p.dx = prod_plan(d, T, chunks_x, ncu);
    p.dw = prod_plan(d, p.vp, chunks_w, ncu);
    if (p.vc == V) {
        const TwoPlans two = two_plans(d, T, chunks_x, d, p.vp, chunks_w, ncu);
        p.both = two.us < p.dx.us + p.dw.us + 4.0;
        if (p.both) {
            p.dx = two.a;
            p.dw = two.b;
        }
    }
    if (!dx) p.dx.bytes = 0;
    if (!dw) p.dw.bytes = 0;
    p.partial = p.both ? p.dx.bytes + p.dw.bytes : std::max(p.dx.bytes, p.dw.bytes);
    p.sums = dx && p.vc < V ? up256((size_t)T * ((d + 7) / 8 * 8) * sizeof(float)) : 0;
    p.tp = dw && !p.both && T >= 512 && V >= 8192 && 2 * (T + 63) < TILE_LD_MAX ? (T + 63) / 64 * 64 : 0;
    p.xt = up256((size_t)((d + 7) / 8 * 8) * p.tp * 2);
    return p;
}

template <typename M, int Y>
static void run_head_few(const HeadFew& few, HeadArgs a, const HeadBackward& p, int64_t d, int edge, void* dx, int64_t lddx,
                         void* dw, int64_t lddw, float* partial, hipStream_t st) {
    typedef typename M::Elem E;
    a.vp = p.vp;
    a.ldz = p.ldz;
    launch_head<M, true>(few, a, true, edge, st);
    const int64_t slabs = (d + 127) / 128, units = (a.V + 15) / 16;
    HeadFewProd g{few.x, few.w, a.dz, a.dzt, few.ldx, few.ldw, p.ldz, p.vp, a.T, a.V, (int)d, dx ? p.parts : 0, p.steps,
                  (int)std::max<int64_t>(1, std::min<int64_t>(16, units * slabs / (16 * op_cus()))), dw, lddw, partial,
                  (d + 7) / 8 * 8, a.in(), (int)slabs, 0, 8};
    const int64_t groups = dw ? (units + 4 * g.units - 1) / (4 * g.units) : 0;
    // (of 32 rows dx's LDS would keep half of dW's workgroups out: 32 x 4096 x 32768 174 us, in one launch 204; 16 x 1024 x
    // 4096 24.0, in one launch 19.6)
    const bool past = 2 * a.V * d >= HEAD_PAST && ((uintptr_t)dw & 15) == 0 && lddw % 8 == 0;
    // long rows whose slabs share no line: slab by slab (of 2048 entries and more the same or better, of 1024 5 to 9% slower)
    const bool apart = (((dx ? (uintptr_t)few.w | few.ldw * 2 : 0) | (dw ? (uintptr_t)dw | lddw * 2 : 0)) & 127) == 0;
    if (apart && slabs > 16) g.each = 1;
    auto go = [&](auto kernel, int64_t rows) {
        g.rows = (int)rows;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((rows + g.each - 1) / g.each * g.each * slabs)), dim3(256), 0, st, g);
    };
    if (Y == 1 && dx && dw) {
        go(past ? k_head_few_prod<M, 1, true, true, true> : k_head_few_prod<M, 1, true, true, false>, p.parts + groups);
    } else {
        if (dx) go(k_head_few_prod<M, Y, true, false, false>, p.parts);
        if (dw) go(past ? k_head_few_prod<M, Y, false, true, true> : k_head_few_prod<M, Y, false, true, false>, groups);
    }
    if (dx)
        hipLaunchKernelGGL(k_head_few_join<E>, dim3((unsigned)((a.T * g.dp + 63) / 64)), dim3(1024), 0, st, g,
                           static_cast<E*>(dx), lddx);
}

template <typename M>
static void run_head_backward(HeadFew few, HeadArgs a, const HeadBackward& p, int64_t d, int64_t V,
                              bool few_rows, int edge, void* dx, int64_t lddx, void* dw, int64_t lddw, HeadScale* scale, void* partial,
                              float* sums, uint16_t* xt, hipStream_t st) {
    typedef typename M::Elem E;
    constexpr bool HALF = narrow_range<E>;
    a.scale = scale;
    a.all = V;
    if (HALF && !p.few && (few_rows || a.T > HEAD_SCALE_ROWS)) {
        hipLaunchKernelGGL(k_head_scale, dim3(1), dim3(1024), 0, st, a.in(), a.T, scale);
        a.factor = &scale->factor;
    }
    if (p.few) {
        if (a.T <= 16)
            run_head_few<M, 1>(few, a, p, d, edge, dx, lddx, dw, lddw, static_cast<float*>(partial), st);
        else
            run_head_few<M, 2>(few, a, p, d, edge, dx, lddx, dw, lddw, static_cast<float*>(partial), st);
        return;
    }
    const Operand w = a.w;
    const char* const few_w = static_cast<const char*>(few.w);
    const int64_t cols = (d + 7) / 8 * 8;   // (of x and w, as they are or padded)
    if (p.tp)
        hipLaunchKernelGGL(k_transpose, dim3((unsigned)(p.tp / 64), (unsigned)((cols + 63) / 64)), dim3(256), 0, st,
                           a.x.base, a.x.ld, a.T, (int)cols, xt, p.tp);
    for (a.v0 = 0; a.v0 < V; a.v0 += p.vc) {
        a.V = (int)std::min(p.vc, V - a.v0);
        a.vp = ((int64_t)a.V + 63) / 64 * 64;   // (p.vp but for the last piece)
        a.ldz = (p.rests ? 2 : 1) * a.vp;
        a.w.base = w.base + a.v0 * w.ld;
        a.w.n = a.V;
        few.w = few_w + 2 * a.v0 * few.ldw;
        launch_head<M, true>(few, a, few_rows, edge, st);
        ProdArgs gx{}, gw{};
        gx.undo = gw.undo = HALF ? &scale->undo : nullptr;
        gx.d = gw.d = d;
        if (dx) {
            gx.a = operand(a.w.base, w.ld, cols, a.V);
            gx.chunks = (int)(a.ldz / 64);
            if (p.rests) {   // the same w again, beside the rests
                gx.a.base2 = gx.a.base;
                gx.a.split = gx.chunks / 2;
            }
            gx.b = operand(a.dz, 2 * a.ldz, a.T, (int64_t)gx.chunks * CHUNK_BYTES);
            gx.out = dx;
            gx.ldo = lddx;
            gx.split = gx.split2 = gx.end = a.T;
            gx.sums = sums;
            gx.first = a.v0 == 0;
            gx.last = a.v0 + a.V == V;
        }
        if (dw) {
            gw.a = operand(a.x.base, a.x.ld, cols, a.T);
            gw.b = operand(a.dz, 2 * a.ldz, a.vp, a.T);
            gw.chunks = (int)((a.T + 63) / 64);
            if (p.rests) {
                gw.a.split = gw.b.split = gw.chunks;
                gw.a.base2 = gw.a.base;
                gw.b.base2 = gw.b.base + 2 * a.vp;
                gw.chunks *= 2;
            }
            gw.out = static_cast<E*>(dw) + a.v0 * lddw;
            gw.ldo = lddw;
            gw.split = gw.split2 = gw.end = a.V;
        }
        if (p.both && dx && dw) {
            launch_two<M>(gx, gw, p.dx, p.dw, static_cast<char*>(partial), st);
            return;
        }
        if (dx) {
            ProdPlan plan = p.dx;
            if (a.vp != p.vp) {   // the last piece is shorter: no more parts than it has, none empty
                plan.parts = std::min(plan.parts, (gx.chunks + plan.part_chunks - 1) / plan.part_chunks);
                if (plan.parts == 1) plan.part_chunks = gx.chunks;
            }
            if (p.vc < V)
                launch_prod<M, true, false, true>(gx, plan, partial, st);
            else
                launch_prod<M, true, false>(gx, plan, partial, st);
        }
        if (!dw) continue;
        const bool past = 2 * V * d >= HEAD_PAST && ((uintptr_t)dw & 15) == 0 && lddw % 8 == 0;
        if (p.tp) gw.a = operand(xt, 2 * p.tp, cols, 2 * p.tp);
        if (p.tp)
            past ? launch_prod<M, false, true, false, true>(gw, p.dw, partial, st)
                 : launch_prod<M, false, true>(gw, p.dw, partial, st);
        else
            past ? launch_prod<M, true, true, false, true>(gw, p.dw, partial, st)
                 : launch_prod<M, true, true>(gw, p.dw, partial, st);
    }
}

}  // namespace bk

static bakron_status head_sizes(const char* who, int64_t ldx, int64_t T, int64_t d, int64_t ldw, int64_t V,
                                int32_t dtype) {
    if (T < 0 || T > bk::OP_T_MAX || d < 1 || V < 1 || d > ((int64_t)1 << 17) || V > ((int64_t)1 << 20))
        return bk::op_fail(who, "bad size");
    if (ldx < d || ldw < d) return bk::op_fail(who, "leading dimension below d");
    if (dtype != BAKRON_F16 && dtype != BAKRON_BF16) return bk::op_fail(who, "dtype must be 16-bit");
    // (the widest launches: 64 x 64 blocks of 256 threads, and 16 threads a row)
    if (T > bk::OP_LAUNCH_MAX / 16 || (T + 63) / 64 * ((std::max(d, V) + 63) / 64) > ((int64_t)1 << 23) - 1)
        return bk::op_fail(who, "too many rows for one call");
    return BAKRON_OK;
}

extern "C" bakron_status bakron_head_logprobs(const void* x, int64_t ldx, int64_t T, int64_t d, const void* w,
                                              int64_t ldw, int64_t V, int32_t dtype, const int64_t* target,
                                              float* logprob, float* entropy, float* lse, void* work,
                                              size_t* work_bytes, hipStream_t stream) {
    static const char who[] = "bakron_head_logprobs";
    bk::set_last_error("");
    bakron_status st = head_sizes(who, ldx, T, d, ldw, V, dtype);
    if (st != BAKRON_OK) return st;
    const int edge = bk::head_edge(T, V, d), parts = (int)((V + edge - 1) / edge);
    const bool many = !bk::head_few_rows(T, V, d);
    const bk::HeadPad p = bk::head_pad(x, ldx, w, ldw, T, d, V, many, many);
    const size_t part = bk::up256((size_t)parts * T * sizeof(bk::HeadPart)), at = bk::up256((size_t)T * sizeof(float));
    bool query;
    st = bk::op_workspace(who, work, work_bytes, p.xbytes + p.wbytes + part + at, &query);
    if (st != BAKRON_OK || query) return st;
    if (logprob && !target) return bk::op_fail(who, "logprob needs targets");
    if (T == 0) return BAKRON_OK;
    if (!x || !w || (!logprob && !entropy && !lse)) return bk::op_fail(who, "null pointer");
    char* const to = static_cast<char*>(work) + p.xbytes + p.wbytes;
    bk::HeadArgs a{};
    a.T = T;
    a.V = (int)V;
    a.target = logprob ? target : nullptr;
    a.part = reinterpret_cast<bk::HeadPart*>(to);
    a.at = reinterpret_cast<float*>(to + part);
    bk::head_operands(a, p, x, ldx, w, ldw, d, static_cast<char*>(work), stream);
    const bk::HeadFew few{x, w, ldx, ldw, (int)d};
    if (dtype == BAKRON_BF16)
        bk::launch_head<bk::MmaBF16, false>(few, a, !many, edge, stream);
    else
        bk::launch_head<bk::MmaF16, false>(few, a, !many, edge, stream);
    const bk::HeadJoinArgs j{a.part, a.at, target, T, (int)V, parts, logprob, entropy, lse};
    if (T <= 64)
        hipLaunchKernelGGL(bk::k_head_join<1>, dim3((unsigned)T), dim3(256), 0, stream, j);
    else
        hipLaunchKernelGGL(bk::k_head_join<16>, dim3((unsigned)((T + 15) / 16)), dim3(256), 0, stream, j);
    return bk::op_launched(who);
}

extern "C" bakron_status bakron_head_logprobs_backward(const void* x, int64_t ldx, int64_t T, int64_t d,
                                                       const void* w, int64_t ldw, int64_t V, int32_t dtype,
                                                       const int64_t* target, const float* lse,
                                                       const float* entropy, const float* g_logprob,
                                                       const float* g_entropy, void* dx, int64_t lddx, void* dw,
                                                       int64_t lddw, void* work, size_t* work_bytes,
                                                       hipStream_t stream) {
    static const char who[] = "bakron_head_logprobs_backward";
    bk::set_last_error("");
    bakron_status st = head_sizes(who, ldx, T, d, ldw, V, dtype);
    if (st != BAKRON_OK) return st;
    if ((dx && lddx < d) || (dw && lddw < d)) return bk::op_fail(who, "leading dimension below d");
    const bk::HeadBackward b = bk::head_backward(std::max<int64_t>(T, 1), d, V, dtype == BAKRON_F16, dx != nullptr,
                                                 dw != nullptr, bk::op_cus());
    const bool many = !b.few && !bk::head_few_rows(T, b.vc, d);
    const bk::HeadPad p = bk::head_pad(x, ldx, w, ldw, T, d, V, many || (dw && !b.few), many || (dx && !b.few));
    bool query;
    st = bk::op_workspace(who, work, work_bytes, p.xbytes + p.wbytes + b.dz + b.dzt + b.partial + b.sums + b.scale + b.xt,
                          &query);
    if (st != BAKRON_OK || query) return st;
    if (!dx && !dw) return bk::op_fail(who, "null pointer");
    if (g_logprob && !target) return bk::op_fail(who, "g_logprob needs targets");
    if (g_entropy && !entropy) return bk::op_fail(who, "g_entropy needs the entropies");
    if (T == 0 && !dw) return BAKRON_OK;
    if (T == 0) {
        hipLaunchKernelGGL(bk::k_zero_rows, dim3((unsigned)std::min<int64_t>(V, 65535)), dim3(256), 0, stream,
                           static_cast<uint16_t*>(dw), lddw, V, d);
        return bk::op_launched(who);
    }
    if (!x || !w || !lse) return bk::op_fail(who, "null pointer");
    char* const to = static_cast<char*>(work) + p.xbytes + p.wbytes;
    char* const partial = to + b.dz + b.dzt;
    char* const sums = partial + b.partial;
    bk::HeadScale* const scale = reinterpret_cast<bk::HeadScale*>(sums + b.sums);
    uint16_t* const xt = reinterpret_cast<uint16_t*>(sums + b.sums + b.scale);
    bk::HeadArgs a{};
    a.T = T;
    a.V = (int)V;
    a.target = g_logprob ? target : nullptr;
    a.lse = lse;
    a.entropy = entropy;
    a.g_logprob = g_logprob;
    a.g_entropy = g_entropy;
    a.dz = to;
    a.dzt = b.dzt ? to + b.dz : nullptr;
    bk::head_operands(a, p, x, ldx, w, ldw, d, static_cast<char*>(work), stream);
    const bk::HeadFew few{x, w, ldx, ldw, (int)d};
    const int edge = b.few ? 16 * bk::head_units(T, V, d) : bk::head_edge(T, b.vc, d);
    if (dtype == BAKRON_BF16)
        bk::run_head_backward<bk::MmaBF16>(few, a, b, d, V, !many, edge, dx, lddx, dw, lddw, scale, partial,
                                           reinterpret_cast<float*>(sums), xt, stream);
    else
        bk::run_head_backward<bk::MmaF16>(few, a, b, d, V, !many, edge, dx, lddx, dw, lddw, scale, partial,
                                          reinterpret_cast<float*>(sums), xt, stream);
    return bk::op_launched(who);
}
