// Rows of a table for given tokens, and the table's gradient.
//
//   y_t = s E[token_t],   dE_v = s sum_{t: token_t = v} dy_t   (+ base_v)
// A token outside [0, V) asks for nothing: its row of y is zeros, its dy counts nowhere.
//
// Forward: bound by memory.  Backward: the positions are sorted by token (equal ones in rising
// order), so that each row of the table has one range of them, summed in that order by whoever writes the row.
#include "ops.h"

namespace bk {

struct EmbedArgs {
    const int64_t* token;
    const void* table;
    void* y;
    int64_t ldt, ldy, T, V;
    int d, pieces;   // of a row
    float scale;
};

constexpr int EMBED_NV = 4;   // vectors a thread has in flight

// A workgroup of 256 threads takes one piece of one row.
template <typename E>
__global__ __launch_bounds__(256) void k_embed(EmbedArgs a) {
    constexpr int VEC = 16 / sizeof(E), LEN = 256 * EMBED_NV * VEC;
    const int64_t t = blockIdx.x / (uint32_t)a.pieces;
    const int lo = (int)(blockIdx.x % (uint32_t)a.pieces) * LEN;
    const int hi = min(a.d, lo + LEN), whole = (hi - lo) / VEC;
    const int64_t k = a.token[t];
    const bool asked = k >= 0 && k < a.V;
    const E* const row = static_cast<const E*>(a.table) + (asked ? k : 0) * a.ldt;
    E* const out = static_cast<E*>(a.y) + t * a.ldy;
    u32x4 r[EMBED_NV];
#pragma unroll
    for (int i = 0; i < EMBED_NV; ++i) r[i] = u32x4(0);
    if (asked && whole > 0) {
#pragma unroll
        for (int i = 0; i < EMBED_NV; ++i)
            r[i] = load_words(row + lo + min(i * 256 + (int)threadIdx.x, whole - 1) * VEC);
    }
#pragma unroll
    for (int i = 0; i < EMBED_NV; ++i) {
        const int v = i * 256 + (int)threadIdx.x;
        if (v >= whole) break;
        Pack<E, VEC> o;
#pragma unroll
        for (int j = 0; j < VEC; ++j) o.v[j] = asked ? (E)(entry<E>(r[i], j) * a.scale) : (E)0.0f;
        store_pack(out + lo + v * VEC, o);
    }
    const int left = lo + whole * VEC + (int)threadIdx.x;
    if (left < hi) out[left] = asked ? (E)((float)row[left] * a.scale) : (E)0.0f;
}

// Sorting by counting: a position's place is the number of positions with a smaller token, or the same one
// before it.  64 positions a workgroup, whose 16 waves share the comparisons.  Tokens outside [0, V)
// sort behind all others.
constexpr int SORT_WAVES = 16;
struct SortArgs {
    const int64_t* token;
    int64_t T, V;
    int32_t *key, *pos;   // sorted tokens (V for those outside) and their positions
};
__device__ inline uint32_t embed_key(int64_t token, int64_t V) {
    return token >= 0 && token < V ? (uint32_t)token : (uint32_t)V;
}
__global__ __launch_bounds__(64 * SORT_WAVES) void k_embed_sort(SortArgs a) {
    __shared__ uint32_t keys[SORT_WAVES][64];
    __shared__ int count[SORT_WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t t = (int64_t)blockIdx.x * 64 + lane;
    const uint32_t mine = embed_key(t < a.T ? a.token[t] : -1, a.V);
    int below = 0;
    // 64 keys of the others a wave at a time, read back one by one by all lanes
    for (int64_t o0 = wave * 64; o0 < a.T; o0 += 64 * SORT_WAVES) {
        keys[wave][lane] = o0 + lane < a.T ? embed_key(a.token[o0 + lane], a.V) : 0xffffffffu;
        __builtin_amdgcn_wave_barrier();
#pragma unroll 16
        for (int k = 0; k < 64; ++k) {
            const uint32_t o = keys[wave][k];
            below += o < mine || (o == mine && o0 + k < t);
        }
        __builtin_amdgcn_wave_barrier();
    }
    count[wave][lane] = below;
    __syncthreads();
    if (wave > 0 || t >= a.T) return;
    for (int w = 1; w < SORT_WAVES; ++w) below += count[w][lane];
    a.key[below] = (int32_t)mine;
    a.pos[below] = (int32_t)t;
}

struct EmbedGradArgs {
    const void* dy;
    const void* base;
    void* out;
    const int32_t *key, *pos;
    int64_t lddy, ldb, ldo, T, V;
    int d, pieces;
    float scale;
};

// The first of n sorted keys that is not below v, found by a wave: 64 probes a step.
__device__ inline int64_t lower_bound(const int32_t* key, int64_t n, int32_t v, int lane) {
    int64_t lo = 0, hi = n;   // the answer is in [lo, hi]
    while (lo < hi) {
        const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
        const uint64_t below = __ballot(at < hi && key[at] < v);
        const int c = __popcll(below);   // probes 0 .. c - 1 are below v
        if (c == 0) return lo;
        hi = min(hi, lo + c * step);
        lo = lo + (c - 1) * step + 1;
    }
    return lo;
}

// A wave takes one vector a lane of one row of the table.
template <typename E>
__global__ __launch_bounds__(256) void k_embed_grad(EmbedGradArgs a) {
    constexpr int VEC = 16 / sizeof(E);
    const int lane = threadIdx.x & 63;
    const int64_t v = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (v >= a.V) return;
    const int c = ((int)blockIdx.y * 64 + lane) * VEC;
    const int64_t lo = lower_bound(a.key, a.T, (int32_t)v, lane), hi = lower_bound(a.key, a.T, (int32_t)v + 1, lane);
    if (c >= a.d) return;
    const int n = min(VEC, a.d - c);
    float s[VEC] = {};
    for (int64_t k = lo; k < hi; ++k) {
        const E* const p = static_cast<const E*>(a.dy) + a.pos[k] * a.lddy + c;
        if (n == VEC) {
            const u32x4 x = load_words(p);
#pragma unroll
            for (int j = 0; j < VEC; ++j) s[j] += entry<E>(x, j);
        } else {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (j < n) s[j] += (float)p[j];
        }
    }
    E* const out = static_cast<E*>(a.out) + v * a.ldo + c;
    const E* const base = a.base ? static_cast<const E*>(a.base) + v * a.ldb + c : nullptr;
    Pack<E, VEC> o;
#pragma unroll
    for (int j = 0; j < VEC; ++j) o.v[j] = (E)fmaf(s[j], a.scale, base && j < n ? (float)base[j] : 0.0f);
    if (n == VEC) {
        store_pack(out, o);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (j < n) out[j] = o.v[j];
    }
}

template <typename E>
static void launch_embed(EmbedArgs a, hipStream_t st) {
    const int len = 256 * EMBED_NV * 16 / (int)sizeof(E);
    a.pieces = (a.d + len - 1) / len;
    hipLaunchKernelGGL(k_embed<E>, dim3((unsigned)(a.T * a.pieces)), dim3(256), 0, st, a);
}
template <typename E>
static void launch_embed_grad(EmbedGradArgs a, hipStream_t st) {
    const int len = 64 * 16 / (int)sizeof(E);
    a.pieces = (a.d + len - 1) / len;
    hipLaunchKernelGGL(k_embed_grad<E>, dim3((unsigned)((a.V + 3) / 4), (unsigned)a.pieces), dim3(256), 0, st, a);
}

}  // namespace bk

static bakron_status embed_sizes(const char* who, int32_t dtype, int64_t T, int64_t V, int64_t d) {
    // (rows and pieces of a launch; positions are sorted as 32-bit numbers, all against all)
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
    const bk::EmbedArgs a{tokens, table, y, ldt, ldy, T, V, (int)d, 0, scale};
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
    const size_t keys = ((size_t)T * sizeof(int32_t) + 255) / 256 * 256;
    bool query;
    st = bk::op_workspace(who, work, work_bytes, 2 * keys, &query);
    if (st != BAKRON_OK || query) return st;
    if (lddy < d || ldo < d || (base && ldb < d)) return bk::op_fail(who, "leading dimension below d");
    if (base && base == dtable && ldb != ldo) return bk::op_fail(who, "base in place needs the same leading dimension");
    if (!dtable || (T > 0 && (!dy || !tokens))) return bk::op_fail(who, "null pointer");
    int32_t* const key = static_cast<int32_t*>(work);
    int32_t* const pos = reinterpret_cast<int32_t*>(static_cast<char*>(work) + keys);
    if (T > 0)
        hipLaunchKernelGGL(bk::k_embed_sort, dim3((unsigned)((T + 63) / 64)), dim3(64 * bk::SORT_WAVES), 0, stream,
                           bk::SortArgs{tokens, T, V, key, pos});
    const bk::EmbedGradArgs a{dy, base, dtable, key, pos, lddy, ldb, ldo, T, V, (int)d, 0, scale};
    if (dtype == BAKRON_F32)
        bk::launch_embed_grad<float>(a, stream);
    else if (dtype == BAKRON_F16)
        bk::launch_embed_grad<bk::f16_t>(a, stream);
    else
        bk::launch_embed_grad<bk::bf16_t>(a, stream);
    return bk::op_launched(who);
}
