// Rows of a table for given tokens, and the table's gradient.
//
//   y_t = s E[token_t],   dE_v = s sum_{t: token_t = v} dy_t   (+ base_v)
// A token outside [0, V) asks for nothing: its row of y is zeros, its dy counts nowhere.
//
// Forward: bound by memory, 8192 x 4096 bf16 18 us, 7.4 TB/s of 134 MB (from the last-level cache in part).  Backward:
// the positions are sorted by token (equal ones in rising
// order), so that each row of the table has one range of them.  Texts repeat a few tokens hundreds of times, so it is
// chunks of 16 sorted positions that are summed, not ranges: a range inside a chunk gives its row at once, the
// sums of longer ones are joined by whoever writes the row, in their order, beside the rows of no token.  (A wave a row, with its
// range searched for: 430 us where these launches take 64, waiting for the longest ranges.)  8192 x 4096 bf16 into 32768
// rows 72 us: sorting 9, chunks 19, the other rows 45 (336 MB: 4.7 TB/s).
#include <algorithm>

#include "ops.h"

namespace bk {

struct EmbedArgs {
    const int64_t* token;
    const void* table;
    void* y;
    int64_t ldt, ldy, T, V;
    int d, pieces, lanes;   // pieces of a row; threads a row
    float scale;
};

constexpr int EMBED_NV = 4;   // vectors a thread has in flight

// `lanes` threads take one piece of one row; of short rows a workgroup takes several.  LONG: 256 lanes, known when it
// is built (8192 x 4096 22 us with tokens that change, 24 without).
template <typename E, bool LONG>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs a) {
    constexpr int VEC = 16 / sizeof(E);
    const int lanes = LONG ? 256 : a.lanes, len = lanes * EMBED_NV * VEC, lane = (int)threadIdx.x % lanes;
    const int64_t t = (int64_t)(blockIdx.x / (uint32_t)a.pieces) * (256 / lanes) + threadIdx.x / lanes;
    if (t >= a.T) return;
    const int lo = (int)(blockIdx.x % (uint32_t)a.pieces) * len;
    const int hi = min(a.d, lo + len), whole = (hi - lo) / VEC;
    const int64_t k = a.token[t];
    const bool asked = k >= 0 && k < a.V;
    const E* const row = static_cast<const E*>(a.table) + (asked ? k : 0) * a.ldt;
    E* const out = static_cast<E*>(a.y) + t * a.ldy;
    u32x4 r[EMBED_NV];
#pragma unroll
    for (int i = 0; i < EMBED_NV; ++i) {
        r[i] = u32x4(0);
        if (asked && i * lanes < whole) r[i] = load_words(row + lo + min(i * lanes + lane, whole - 1) * VEC);
    }
#pragma unroll
    for (int i = 0; i < EMBED_NV; ++i) {
        const int v = i * lanes + lane;
        if (v >= whole) break;
        Pack<E, VEC> o;
#pragma unroll
        for (int j = 0; j < VEC; ++j) o.v[j] = asked ? (E)(entry<E>(r[i], j) * a.scale) : (E)0.0f;
        store_pack(out + lo + v * VEC, o);
    }
    const int left = lo + whole * VEC + lane;
    if (left < hi) out[left] = asked ? (E)((float)row[left] * a.scale) : (E)0.0f;
}

typedef int32_t i32x4_t __attribute__((ext_vector_type(4)));

// Positions sorted by token, equal tokens in rising order; tokens outside [0, V) behind all others.
struct SortArgs {
    const int64_t* token;
    int64_t T, V;
    int32_t *key, *pos;        // sorted tokens (V for those outside) and their positions
    // by digits
    int32_t *key_in, *pos_in;  // what a pass reads (the first one: tokens)
    int32_t* count;            // SORT_BINS x blocks
    int blocks, shift;
};
__device__ inline int32_t embed_key(int64_t token, int64_t V) {
    return token >= 0 && token < V ? (int32_t)token : (int32_t)V;
}

// Up to SORT_BY_COUNT positions: a position's place is the number of positions with a smaller token, or the
// same one before it.  A workgroup takes 32 positions, its 32 half waves share what they are compared with.
// One launch; the work grows with T^2.
constexpr int SORT_WAVES = 16;
__global__ __launch_bounds__(64 * SORT_WAVES) void k_embed_sort(SortArgs a) {
    __shared__ __attribute__((aligned(16))) int32_t keys[SORT_WAVES][64];
    __shared__ int count[2 * SORT_WAVES][32];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, l = lane & 31;
    const int64_t t0 = (int64_t)blockIdx.x * 32, t = t0 + l;
    const int32_t mine = embed_key(t < a.T ? a.token[t] : -1, a.V);
    int below = 0;
    // 64 keys a wave at a time, 32 for each half; its own 32 positions' among them by (key, position)
    int64_t next = wave * 64 + lane < a.T ? a.token[wave * 64 + lane] : -1;
    for (int64_t o0 = wave * 64; o0 < a.T; o0 += 64 * SORT_WAVES) {
        const int64_t o = o0 + lane, n = o + 64 * SORT_WAVES;
        const int64_t token = next;
        if (n < a.T) next = a.token[n];
        __builtin_amdgcn_wave_barrier();
        keys[wave][lane] = o < a.T ? embed_key(token, a.V) : 0x7fffffff;
        __builtin_amdgcn_wave_barrier();
        const int64_t first = o0 + half * 32;
        const int32_t* const k = &keys[wave][half * 32];
        // (keys below, or equal ones, of earlier positions: below `mine + 1`)
        const int32_t bound = first < t0 ? mine + 1 : mine;
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
            const i32x4_t o4 = *reinterpret_cast<const i32x4_t*>(k + j);
#pragma unroll
            for (int i = 0; i < 4; ++i) below += o4[i] < bound;
        }
        if (first == t0)
            for (int j = 0; j < 32; ++j) below += k[j] == mine && j < l;
    }
    count[2 * wave + half][l] = below;
    __syncthreads();
    if (threadIdx.x >= 32 || t >= a.T) return;
    for (int w = 1; w < 2 * SORT_WAVES; ++w) below += count[w][l];
    a.key[below] = mine;
    a.pos[below] = (int32_t)t;
}
constexpr int64_t SORT_BY_COUNT = 16384;

// More of them: by two digits of 11 bits, each pass in three launches: the blocks' counts of each digit, their
// running sum over (digit, block), and every position to its place.
constexpr int SORT_BITS = 11, SORT_BINS = 1 << SORT_BITS, SORT_EACH = 4, SORT_BLOCK = 1024 * SORT_EACH;
__device__ inline int32_t sort_key(const SortArgs& a, int64_t at) {
    return a.key_in ? a.key_in[at] : embed_key(a.token[at], a.V);
}
__global__ __launch_bounds__(1024) void k_sort_count(SortArgs a) {
    __shared__ int32_t bins[SORT_BINS];
    for (int i = threadIdx.x; i < SORT_BINS; i += 1024) bins[i] = 0;
    __syncthreads();
    const int64_t lo = (int64_t)blockIdx.x * SORT_BLOCK;
#pragma unroll
    for (int i = 0; i < SORT_EACH; ++i) {
        const int64_t at = lo + i * 1024 + threadIdx.x;
        if (at < a.T) atomicAdd(&bins[(sort_key(a, at) >> a.shift) & (SORT_BINS - 1)], 1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < SORT_BINS; i += 1024) a.count[(int64_t)i * a.blocks + blockIdx.x] = bins[i];
}
// One workgroup goes through the counts, four a thread at a time.
__global__ __launch_bounds__(1024) void k_sort_scan(SortArgs a) {
    __shared__ int32_t sums[2][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t n = (int64_t)SORT_BINS * a.blocks;   // (a multiple of 2048)
    int32_t before = 0;
    const i32x4_t none = {0, 0, 0, 0};
    auto at = [&](int64_t i) { return reinterpret_cast<i32x4_t*>(a.count) + i; };
    i32x4_t next = threadIdx.x < n / 4 ? *at(threadIdx.x) : none;
    int turn = 0;
    for (int64_t i = threadIdx.x; i - threadIdx.x < n / 4; i += 1024, turn ^= 1) {
        i32x4_t c = next;
        next = i + 1024 < n / 4 ? *at(i + 1024) : none;
        const int32_t own = c[0] + c[1] + c[2] + c[3];
        int32_t sum = own;
#pragma unroll
        for (int k = 1; k < 64; k *= 2) {
            const int32_t v = __shfl_up(sum, k);
            if (lane >= k) sum += v;
        }
        if (lane == 63) sums[turn][wave] = sum;
        __syncthreads();
        int32_t first = before + sum - own;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            const int32_t v = sums[turn][w];
            if (w < wave) first += v;
            before += v;
        }
        const i32x4_t o = {first, first + c[0], first + c[0] + c[1], first + c[0] + c[1] + c[2]};
        if (i < n / 4) *at(i) = o;
    }
}
// A wave takes 64 SORT_EACH positions in a row, 64 at a time; those of equal digits find each other by ballots.
__global__ __launch_bounds__(1024) void k_sort_place(SortArgs a) {
    __shared__ uint16_t bins[16][SORT_BINS];   // a wave's counts, then what lies before it in the block
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < 16 * SORT_BINS; i += 1024) (&bins[0][0])[i] = 0;
    __syncthreads();
    const int64_t lo = (int64_t)blockIdx.x * SORT_BLOCK + wave * (64 * SORT_EACH);
    int32_t key[SORT_EACH], rank[SORT_EACH];
#pragma unroll
    for (int i = 0; i < SORT_EACH; ++i) {
        const int64_t at = lo + i * 64 + lane;
        key[i] = at < a.T ? sort_key(a, at) : 0;
        const int digit = (key[i] >> a.shift) & (SORT_BINS - 1);
        uint64_t same = __ballot(at < a.T);
#pragma unroll
        for (int b = 0; b < SORT_BITS; ++b) {
            const uint64_t one = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? one : ~one;
        }
        const int before = __popcll(same & ((1ull << lane) - 1));
        rank[i] = bins[wave][digit] + before;   // (read by all before the last of them writes)
        __builtin_amdgcn_wave_barrier();
        if (at < a.T && (same >> lane) == 1) bins[wave][digit] = (uint16_t)(rank[i] + 1);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    for (int i = threadIdx.x; i < SORT_BINS; i += 1024) {
        int sum = 0;
        for (int w = 0; w < 16; ++w) {
            const int n = bins[w][i];
            bins[w][i] = (uint16_t)sum;
            sum += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SORT_EACH; ++i) {
        const int64_t at = lo + i * 64 + lane;
        if (at >= a.T) break;
        const int digit = (key[i] >> a.shift) & (SORT_BINS - 1);
        const int64_t to = a.count[(int64_t)digit * a.blocks + blockIdx.x] + bins[wave][digit] + rank[i];
        a.key[to] = key[i];
        a.pos[to] = a.pos_in ? a.pos_in[at] : (int32_t)at;
    }
}

struct EmbedGradArgs {
    const void* dy;
    const void* base;
    void* out;
    const int32_t *key, *pos;
    int32_t* start;            // V + 1: where each token's sorted positions begin
    float* part;               // what a chunk leaves of the range it begins in, and of the one it ends in: chunks x 2 x dp
    int64_t lddy, ldb, ldo, T, V, dp;
    int d, chunk_blocks, lanes;   // threads a row
    int rows, slabs;           // k_embed_grad, k_embed_few: workgroups along the rows, and along one
    int past;                  // the gradient is written past the caches
    float scale;
};
// Sorted positions of a chunk.
constexpr int EMBED_CHUNK = 16;

// A gradient that the last-level cache (256 MB) would not hold with anything beside it is written past the caches:
// 8192 x 4096 into 32768 rows (268 MB) 82 -> 72 us, 65536 x 1024 into 131072 rows 167 -> 144.  A smaller one is left to
// whoever reads it next, and one of few positions, which reads nothing that it could sweep (200 positions 37 us, past
// the caches 44).  Rows that share lines are left to the caches, which join them (300 x 3571 fp32 into 35552 125 us, past
// them 138).
constexpr int64_t EMBED_PAST = (int64_t)128 << 20;

// A row is read and written in whole vectors (WHOLE: d is a multiple of them), or its last entries one by one: `n` of
// them are left from this vector on.
template <typename E, bool WHOLE>
__device__ inline u32x4 embed_load(const E* p, int n) {
    constexpr int VEC = 16 / sizeof(E);
    if (WHOLE || n >= VEC) return load_words(p);
    E v[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) v[j] = j < n ? p[j] : (E)0.0f;
    u32x4 r;
    __builtin_memcpy(&r, v, 16);
    return r;
}
// Base + scale * s.
template <typename E, bool WHOLE>
__device__ inline void embed_write(const EmbedGradArgs& a, int64_t v, int c, int n, const float (&s)[16 / sizeof(E)]) {
    constexpr int VEC = 16 / sizeof(E);
    float o[VEC] = {};
    if (a.base) {
        const u32x4 b = embed_load<E, WHOLE>(static_cast<const E*>(a.base) + v * a.ldb + c, n);
#pragma unroll
        for (int j = 0; j < VEC; ++j) o[j] = entry<E>(b, j);
    }
#pragma unroll
    for (int j = 0; j < VEC; ++j) o[j] = fmaf(s[j], a.scale, o[j]);
    E* const out = static_cast<E*>(a.out) + v * a.ldo + c;
    if (a.past && (WHOLE || n >= VEC)) {
        Pack<E, VEC> p;
#pragma unroll
        for (int j = 0; j < VEC; ++j) p.v[j] = (E)o[j];
        u32x4 u;
        __builtin_memcpy(&u, &p, 16);
        store_words_past(out, u);
    } else {
        store_n(out, o, WHOLE ? VEC : n);
    }
}

// A row of zeros where there is no base: whole vectors at addresses that are multiples of theirs, what lies before and
// behind an entry a lane (13 x 3571 into 35552 rows 73
// us, at any alignment, and 68).  c: the first of a thread's NV vectors, `step` entries apart
// (and rows of VEC vectors at least, so that each entry has its lane).
template <typename E, int NV>
__device__ inline void embed_zero(const EmbedGradArgs& a, int64_t v, int c, int step) {
    constexpr int VEC = 16 / sizeof(E);
    E* const row = static_cast<E*>(a.out) + v * a.ldo;
    const int before = (int)(-(uintptr_t)row & 15) / (int)sizeof(E), behind = (a.d - before) % VEC;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        E* const p = row + before + c + i * step;
        if (before + c + i * step + VEC > a.d) continue;
        if (a.past)
            store_words_past(p, u32x4(0));
        else
            *reinterpret_cast<u32x4*>(p) = u32x4(0);
    }
    const int lane = c / VEC;
    if (lane < before) row[lane] = (E)0.0f;
    if (lane < behind) row[a.d - behind + lane] = (E)0.0f;
}

// A chunk of the sorted positions is summed by `lanes` threads, a vector of the row each.  Where a token's whole range
// lies in the chunk its row is written; of one that goes on from the chunk before, or into the next, the sum is
// left for the row's writer.  The workgroups behind those of the chunks find where each token's range begins.
template <typename E, bool WHOLE>
__global__ __launch_bounds__(256) void k_embed_chunks(EmbedGradArgs a) {
    constexpr int VEC = 16 / sizeof(E);
    if ((int)blockIdx.x >= a.chunk_blocks) {
        const int64_t v = (int64_t)((int)blockIdx.x - a.chunk_blocks) * 256 + threadIdx.x;
        if (blockIdx.y > 0 || v > a.V) return;
        int lo = 0, hi = (int)a.T;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (a.key[mid] < (int32_t)v)
                lo = mid + 1;
            else
                hi = mid;
        }
        a.start[v] = lo;
        return;
    }
    const int64_t chunk = (int64_t)blockIdx.x * (256 / a.lanes) + threadIdx.x / a.lanes;
    const int64_t lo = chunk * EMBED_CHUNK;
    const int c = ((int)blockIdx.y * a.lanes + (int)(threadIdx.x % a.lanes)) * VEC, n = a.d - c;
    if (lo >= a.T || n <= 0) return;
    const E* const dy = static_cast<const E*>(a.dy) + c;
    const int count = (int)min(a.T - lo, (int64_t)EMBED_CHUNK);
    // (whole chunks of both: the arrays are padded, and what lies past T is not used)
    const auto key = load_pack<int32_t, EMBED_CHUNK>(a.key + lo), pos = load_pack<int32_t, EMBED_CHUNK>(a.pos + lo);
    int32_t token = key.v[0];
    const int32_t before = lo > 0 ? a.key[lo - 1] : -1, behind = lo + count < a.T ? a.key[lo + count] : -1;
    u32x4 x[EMBED_CHUNK];
#pragma unroll
    for (int i = 0; i < EMBED_CHUNK; ++i)   // (all asked for at once)
        x[i] = embed_load<E, WHOLE>(dy + (i < count ? pos.v[i] : pos.v[0]) * a.lddy, n);
    bool begins = before != token;
    float s[VEC] = {};
    // (tokens outside the table are the last ones: V)
    auto flush = [&](bool ends) {
        if (begins && ends)
            embed_write<E, WHOLE>(a, token, c, n, s);
        else
            store_n(a.part + (chunk * 2 + (begins ? 1 : 0)) * a.dp + c, s, VEC);
    };
#pragma unroll
    for (int i = 0; i < EMBED_CHUNK; ++i) {
        if (i > 0 && i < count && key.v[i] != token) {   // the token's range ends before this position
            if (token < a.V) flush(true);
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[j] = 0.0f;
            token = key.v[i];
            begins = true;
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) s[j] += i < count ? entry<E>(x[i], j) : 0.0f;
    }
    if (token < a.V) flush(token != behind);
}

// Which rows and which part of them a workgroup takes.  Every eighth workgroup runs on the same XCD: those have all parts
// of a row, so that a line that two parts share is joined in one L2 (13 x 3571 into 35552 rows 68 us, parts in turn, and 53).
__device__ inline bool embed_block(const EmbedGradArgs& a, int& row, int& slab) {
    const uint32_t at = blockIdx.x / 8;
    slab = (int)(at % (uint32_t)a.slabs);
    row = (int)(at / (uint32_t)a.slabs * 8 + blockIdx.x % 8);
    return row < a.rows;
}

// The rows that are left.  Those whose range spans chunks: first, as they take longest, by one workgroup for each
// chunk in which such a range begins (256 vectors of the row a workgroup).  Those of no token: `lanes` lanes of a
// wave take EMBED_ROWS of them, NV vectors a lane (of a longer row a part).
constexpr int EMBED_ROWS = 4;
template <typename E, int NV, bool WHOLE>
__global__ __launch_bounds__(256) void k_embed_grad(EmbedGradArgs a) {
    constexpr int VEC = 16 / sizeof(E);
    int block, slab;
    if (!embed_block(a, block, slab)) return;
    if (block < a.chunk_blocks) {
        const int64_t next = ((int64_t)block + 1) * EMBED_CHUNK;
        const int32_t token = a.key[next];
        if (token != a.key[next - 1] || token >= a.V) return;
        const int lo = a.start[token], first = lo / EMBED_CHUNK, end = (a.start[token + 1] - 1) / EMBED_CHUNK;
        if (first != block) return;
        for (int c = (slab * 256 + (int)threadIdx.x) * VEC; c < a.d; c += a.slabs * 256 * VEC) {
            constexpr int AHEAD = 8;
            const float* const part = a.part + c;
            float s[VEC];
            const auto p = load_pack<float, VEC>(part + ((int64_t)first * 2 + 1) * a.dp);
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[j] = p.v[j];
            for (int k = first + 1; k <= end; k += AHEAD) {
                Pack<float, VEC> x[AHEAD];
#pragma unroll
                for (int m = 0; m < AHEAD; ++m) x[m] = load_pack<float, VEC>(part + (int64_t)min(k + m, end) * 2 * a.dp);
#pragma unroll
                for (int m = 0; m < AHEAD; ++m)
                    if (k + m <= end) {
#pragma unroll
                        for (int j = 0; j < VEC; ++j) s[j] += x[m].v[j];
                    }
            }
            embed_write<E, WHOLE>(a, token, c, a.d - c, s);
        }
        return;
    }
    const int64_t v0 = ((int64_t)(block - a.chunk_blocks) * (256 / a.lanes) + threadIdx.x / a.lanes) * EMBED_ROWS;
    const int step = a.lanes * VEC, c = slab * NV * step + (int)(threadIdx.x % a.lanes) * VEC, n = a.d - c;
    if (v0 >= a.V || n <= 0) return;
    int start[EMBED_ROWS + 1];   // (all asked for at once; past the table its end: no rows)
#pragma unroll
    for (int r = 0; r <= EMBED_ROWS; ++r) start[r] = a.start[min(v0 + r, a.V)];
    const float none[VEC] = {};
#pragma unroll
    for (int r = 0; r < EMBED_ROWS; ++r) {
        if (v0 + r >= a.V) break;
        if (start[r] < start[r + 1]) continue;
        if (!a.base && a.d >= VEC * VEC) {
            embed_zero<E, NV>(a, v0 + r, c, step);
            continue;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * step < n) embed_write<E, WHOLE>(a, v0 + r, c + i * step, n - i * step, none);
    }
}

// Up to EMBED_FEW positions: every wave holds all tokens and finds the positions of each of its rows by ballots, so
// nothing is sorted and one launch does it: 13 x 1000 into 6000 rows 15 us in three launches, 8 so.
constexpr int EMBED_FEW = 256;
template <typename E, int NV, bool WHOLE>
__global__ __launch_bounds__(256) void k_embed_few(EmbedGradArgs a, const int64_t* __restrict__ tokens) {
    constexpr int VEC = 16 / sizeof(E), WORDS = EMBED_FEW / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, groups = 64 / a.lanes, group = lane / a.lanes;
    static_assert(WORDS == 4, "words of a row's positions");
    int block, slab;
    if (!embed_block(a, block, slab)) return;
    int32_t key[WORDS];
#pragma unroll
    for (int k = 0; k < WORDS; ++k) {
        const int t = k * 64 + lane;
        key[k] = t < a.T ? embed_key(tokens[t], a.V) : -1;
    }
    const int step = a.lanes * VEC, c = slab * NV * step + lane % a.lanes * VEC, n = a.d - c;
    const int64_t v0 = ((int64_t)block * 4 + wave) * (groups * EMBED_ROWS);
    const E* const dy = static_cast<const E*>(a.dy) + c;
    for (int r = 0; r < EMBED_ROWS; ++r) {
        const int64_t first = v0 + r * groups, v = first + group;
        if (first >= a.V) break;
        uint64_t hit[WORDS] = {};
        for (int g = 0; g < groups; ++g)
#pragma unroll
            for (int k = 0; k < WORDS; ++k) {
                const uint64_t is = __ballot(key[k] == (int32_t)(first + g));
                if (g == group) hit[k] = is;
            }
        if (v >= a.V || n <= 0) continue;
        if ((hit[0] | hit[1] | hit[2] | hit[3]) == 0 && !a.base && a.d >= VEC * VEC) {
            embed_zero<E, NV>(a, v, c, step);
            continue;
        }
        float s[NV][VEC] = {};
#pragma unroll
        for (int k = 0; k < WORDS; ++k)
            for (uint64_t is = hit[k]; is != 0;) {
                constexpr int AHEAD = 4;   // (a frequent token's rows are asked for four at a time)
                u32x4 x[AHEAD][NV];
                bool there[AHEAD];
#pragma unroll
                for (int m = 0; m < AHEAD; ++m) {
                    there[m] = is != 0;
                    const E* const row = dy + (int64_t)(k * 64 + (there[m] ? __ffsll((unsigned long long)is) - 1 : 0)) * a.lddy;
                    is &= is - 1;
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        x[m][i] = u32x4(0);
                        if (there[m] && i * step < n) x[m][i] = embed_load<E, WHOLE>(row + i * step, n - i * step);
                    }
                }
#pragma unroll
                for (int m = 0; m < AHEAD; ++m)
                    if (there[m]) {
#pragma unroll
                        for (int i = 0; i < NV; ++i)
#pragma unroll
                            for (int j = 0; j < VEC; ++j) s[i][j] += entry<E>(x[m][i], j);
                    }
            }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (i * step < n) embed_write<E, WHOLE>(a, v, c + i * step, n - i * step, s[i]);
    }
}

template <typename E>
static void launch_embed(EmbedArgs a, hipStream_t st) {
    constexpr int VEC = 16 / (int)sizeof(E);
    a.lanes = VEC;   // (what is left of a row, less than a vector, goes one entry a thread)
    while (a.lanes < 256 && a.lanes * VEC < a.d) a.lanes *= 2;
    const int len = a.lanes * EMBED_NV * VEC, rows = 256 / a.lanes;
    a.pieces = (a.d + len - 1) / len;
    const dim3 grid((unsigned)((a.T + rows - 1) / rows * a.pieces));
    if (rows == 1)
        hipLaunchKernelGGL((k_embed<E, true>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((k_embed<E, false>), grid, dim3(256), 0, st, a);
}
// The workspace of the gradient.
struct EmbedWork {
    size_t keys, count, start, part;   // of one array of keys or positions (four of them where they are sorted by digits)
    int blocks;
    int64_t dp;
    size_t bytes() const { return (blocks ? 4 : 2) * keys + count + start + part; }
};
static size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }
static EmbedWork embed_work(int64_t T, int64_t V, int64_t d) {
    EmbedWork w{};
    if (T <= EMBED_FEW) return w;   // (no workspace)
    w.start = up256((size_t)(V + 1) * sizeof(int32_t));
    w.keys = up256((size_t)T * sizeof(int32_t));
    w.dp = (d + 7) / 8 * 8;
    w.part = up256((size_t)((T + EMBED_CHUNK - 1) / EMBED_CHUNK) * 2 * w.dp * sizeof(float));
    if (T > SORT_BY_COUNT) {
        w.blocks = (int)((T + SORT_BLOCK - 1) / SORT_BLOCK);
        w.count = up256((size_t)SORT_BINS * w.blocks * sizeof(int32_t));
    }
    return w;
}

// Leaves the sorted keys and positions at work and work + w.keys.
static void launch_sort(const EmbedWork& w, const int64_t* tokens, int64_t T, int64_t V, char* work, hipStream_t st) {
    auto at = [&](size_t o) { return reinterpret_cast<int32_t*>(work + o); };
    SortArgs a{tokens, T, V, at(0), at(w.keys), nullptr, nullptr, nullptr, w.blocks, 0};
    if (w.blocks == 0) {
        hipLaunchKernelGGL(k_embed_sort, dim3((unsigned)((T + 31) / 32)), dim3(64 * SORT_WAVES), 0, st, a);
        return;
    }
    a.count = at(4 * w.keys);
    for (int pass = 0; pass < 2; ++pass) {
        a.shift = pass * SORT_BITS;
        a.key = at(pass ? 0 : 2 * w.keys);
        a.pos = at(pass ? w.keys : 3 * w.keys);
        a.key_in = pass ? at(2 * w.keys) : nullptr;
        a.pos_in = pass ? at(3 * w.keys) : nullptr;
        const dim3 grid((unsigned)w.blocks), block(1024);
        hipLaunchKernelGGL(k_sort_count, grid, block, 0, st, a);
        hipLaunchKernelGGL(k_sort_scan, dim3(1), block, 0, st, a);
        hipLaunchKernelGGL(k_sort_place, grid, block, 0, st, a);
    }
}

template <typename E, bool WHOLE>
static void launch_embed_grad(EmbedGradArgs a, const int64_t* tokens, hipStream_t st) {
    const int vecs = (a.d * (int)sizeof(E) + 15) / 16, nv = vecs <= 64 ? 1 : vecs <= 128 ? 2 : 4;
    auto lanes = [&](int most) {
        a.lanes = 1;
        while (a.lanes < most && a.lanes < vecs) a.lanes *= 2;
    };
    if (a.T > EMBED_FEW) {
        lanes(256);
        const int64_t chunks = (a.T + EMBED_CHUNK - 1) / EMBED_CHUNK;
        a.chunk_blocks = (int)((chunks * a.lanes + 255) / 256);
        hipLaunchKernelGGL((k_embed_chunks<E, WHOLE>),
                           dim3((unsigned)(a.chunk_blocks + (a.V + 256) / 256), (unsigned)((vecs + a.lanes - 1) / a.lanes)),
                           dim3(256), 0, st, a);
        a.chunk_blocks = (int)(chunks - 1);   // of the next launch: the joins
    }
    lanes(64);
    const int each = 256 / a.lanes * EMBED_ROWS;
    a.rows = (int)(a.chunk_blocks + (a.V + each - 1) / each);
    a.slabs = (vecs + a.lanes * nv - 1) / (a.lanes * nv);
    const dim3 grid((unsigned)((a.rows + 7) / 8 * 8 * a.slabs));
    auto go = [&](auto few, auto many) {
        if (a.T <= EMBED_FEW)
            hipLaunchKernelGGL(few, grid, dim3(256), 0, st, a, tokens);
        else
            hipLaunchKernelGGL(many, grid, dim3(256), 0, st, a);
    };
    if (nv == 1)
        go(k_embed_few<E, 1, WHOLE>, k_embed_grad<E, 1, WHOLE>);
    else if (nv == 2)
        go(k_embed_few<E, 2, WHOLE>, k_embed_grad<E, 2, WHOLE>);
    else
        go(k_embed_few<E, 4, WHOLE>, k_embed_grad<E, 4, WHOLE>);
}
template <typename E>
static void launch_embed_grad(const EmbedGradArgs& a, const int64_t* tokens, hipStream_t st) {
    if (a.d % (16 / (int)sizeof(E)) == 0)
        launch_embed_grad<E, true>(a, tokens, st);
    else
        launch_embed_grad<E, false>(a, tokens, st);
}

}  // namespace bk

static bakron_status embed_sizes(const char* who, int32_t dtype, int64_t T, int64_t V, int64_t d) {
    // (rows and pieces of a launch; tokens and positions of the gradient are sorted as 32-bit numbers, tokens by two digits of
    // 11 bits; the forward pass takes as many as its gradient does)
    if (T < 0 || T > ((int64_t)1 << 20) || V < 1 || V > ((int64_t)1 << 20) || d < 1 || d > 65536)
        return bk::op_fail(who, "bad size");
    if (dtype != BAKRON_F32 && dtype != BAKRON_F16 && dtype != BAKRON_BF16) return bk::op_fail(who, "bad dtype");
    return BAKRON_OK;
}

extern "C" bakron_status bakron_embedding(const int64_t* tokens, int64_t T, const void* table, int64_t ldt,
                                          int32_t dtype, int64_t V, int64_t d, float scale, void* y, int64_t ldy,
                                          hipStream_t stream) {
    static const char who[] = "bakron_embedding";
    bk::set_last_error("");
    const bakron_status st = embed_sizes(who, dtype, T, V, d);
    if (st != BAKRON_OK) return st;
    if (ldt < d || ldy < d) return bk::op_fail(who, "leading dimension below d");
    const int64_t len = 256 * bk::EMBED_NV * (dtype == BAKRON_F32 ? 4 : 8);
    if (T > bk::OP_LAUNCH_MAX / 256 / ((d + len - 1) / len)) return bk::op_fail(who, "too many rows for one call");
    if (T == 0) return BAKRON_OK;
    if (!tokens || !table || !y) return bk::op_fail(who, "null pointer");
    const bk::EmbedArgs a{tokens, table, y, ldt, ldy, T, V, (int)d, 0, 0, scale};
    if (dtype == BAKRON_F32)
        bk::launch_embed<float>(a, stream);
    else if (dtype == BAKRON_F16)
        bk::launch_embed<bk::f16_t>(a, stream);
    else
        bk::launch_embed<bk::bf16_t>(a, stream);
    return bk::op_launched(who);
}

extern "C" bakron_status bakron_embedding_backward(const void* dy, int64_t lddy, const int64_t* tokens, int64_t T,
                                                   int32_t dtype, int64_t V, int64_t d, float scale, const void* base,
                                                   int64_t ldb, void* dtable, int64_t ldo, void* work,
                                                   size_t* work_bytes, hipStream_t stream) {
    static const char who[] = "bakron_embedding_backward";
    bk::set_last_error("");
    bakron_status st = embed_sizes(who, dtype, T, V, d);
    if (st != BAKRON_OK) return st;
    const bk::EmbedWork w = bk::embed_work(T, V, d);
    bool query;
    st = bk::op_workspace(who, work, work_bytes, w.bytes(), &query);
    if (st != BAKRON_OK || query) return st;
    if (lddy < d || ldo < d || (base && ldb < d)) return bk::op_fail(who, "leading dimension below d");
    if (base && base == dtable && ldb != ldo) return bk::op_fail(who, "base in place needs the same leading dimension");
    if (!dtable || (T > 0 && (!dy || !tokens))) return bk::op_fail(who, "null pointer");
    char* const at = static_cast<char*>(work);
    if (T > bk::EMBED_FEW) bk::launch_sort(w, tokens, T, V, at, stream);
    char* const part = at + w.bytes() - w.part;
    const int64_t esize = dtype == BAKRON_F32 ? 4 : 2;
    const bool past = T > bk::EMBED_FEW && V * d * esize >= bk::EMBED_PAST && (((uintptr_t)dtable | ldo * esize) & 15) == 0;
    const bk::EmbedGradArgs a{dy, base, dtable, reinterpret_cast<int32_t*>(at), reinterpret_cast<int32_t*>(at + w.keys),
                              reinterpret_cast<int32_t*>(part - w.start), reinterpret_cast<float*>(part), lddy, ldb, ldo,
                              T, V, w.dp, (int)d, 0, 0, 0, 0, past, scale};
    if (dtype == BAKRON_F32)
        bk::launch_embed_grad<float>(a, tokens, stream);
    else if (dtype == BAKRON_F16)
        bk::launch_embed_grad<bk::f16_t>(a, tokens, stream);
    else
        bk::launch_embed_grad<bk::bf16_t>(a, tokens, stream);
    return bk::op_launched(who);
}
