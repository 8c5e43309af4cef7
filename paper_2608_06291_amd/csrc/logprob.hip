// Log probabilities of given tokens with entropy and top alternatives, and their
// gradient.
//
// For a row z:  m = max z,  s = sum exp(z - m),  s1 = sum exp(z - m) (z - m),
//   lse = m + log s,   logprob = (z_target - m) - log s,   entropy = log s - s1 / s
// (from lse itself a log probability would take lse's rounding, 5e-4 at logits around 1e4).
// Parts of a row join by rescaling to the larger m:
//   s = s_a e^(m_a - m) + s_b e^(m_b - m),
//   s1 = (s1_a + (m_a - m) s_a) e^(m_a - m) + (s1_b + (m_b - m) s_b) e^(m_b - m).
//
// Top k without sorting: a workgroup holds its part of the row in registers, cuts
// its threads into 32 groups and takes the k-th largest group maximum as a bound.
// At least k entries are not below it, and of a row in random order only about
// 32 (H_32 - H_(32-k)) (31 for k = 20) are, so the candidates are ranked by counting.  Where fewer than k
// groups hold an entry there is no bound, and more than 1024 candidates are then gone through k times: 16-bit
// rows (or parts of one) of 1025 to 128 (k - 1) tokens, fp32 ones to 64 (k - 1) (8192 x 2000 bf16: 230 us for
// k = 20, 35 for 5).
//
// Bound by memory: 2048 x 131072 bf16 (537 MB) with 5 alternatives and masked rows 107 to 114 us, 4.7 to 5.0
// TB/s, without alternatives 96 to 103, in fp32 187; the gradient of 4096 x 32768 (537 MB) 91 us, 5.9 TB/s, in
// fp32 178 (a large copy here: 5.2).  What kept the first kernel at 328 us: loads behind branches, one after
// another, entries held in fp32 (twice the registers, half the workgroups), and the
// masked rows' thousands of equal logits going through one counter.  One row of 131072 with 20
// alternatives takes 12 us in two launches, latency.
#include "ops.h"

namespace bk {

constexpr int LP_THREADS = 512;
constexpr int LP_WAVES = LP_THREADS / 64;
constexpr int LP_REGS = 32;           // 32-bit registers of logits a thread holds at most
constexpr int LP_TOP = 32;            // alternatives at most
constexpr int LP_CAND = 1024;         // candidates that are ranked by counting
constexpr int LP_PARTS = 64;          // parts of a row at most
constexpr int LP_JOIN = 256;          // candidates that the join ranks by counting

// What a part of a row leaves for the join.
struct LpPart {
    float m, s, s1, pad;
};

struct LpArgs {
    const void* z;
    int64_t ld;
    const int64_t* target;
    int64_t T;
    int V, part_len, parts, top;
    float *logprob, *entropy, *lse, *top_logprob;
    int64_t* top_index;
    LpPart* part;              // T x parts
    uint64_t* cand;            // T x parts x top, sorted
};

// Order of the alternatives: larger logit first (NaN before all, -0 = +0), then
// smaller index.  Never 0, which stands for none.
__device__ inline uint32_t lp_key(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return v != v ? 0xffffffffu : (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ inline float lp_unkey(uint32_t k) {
    return k == 0xffffffffu ? NAN : __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}
__device__ inline uint64_t lp_rank(float v, int index) {
    return ((uint64_t)lp_key(v) << 32) | (uint32_t)(0x7fffffff - index);
}
__device__ inline int lp_index(uint64_t r) { return 0x7fffffff - (int)(uint32_t)r; }

// The largest of the wave: by the upper halves, then by the lower ones among equals.
__device__ inline uint64_t wave_max_u64(uint64_t v) {
    const uint32_t hi = (uint32_t)(v >> 32);
    const uint32_t top = wave_reduce(hi, MaxU32());
    const uint32_t lo = wave_reduce(hi == top ? (uint32_t)v : 0u, MaxU32());
    return ((uint64_t)top << 32) | lo;
}

// Writes what a row's statistics give.
__device__ inline void lp_store(const LpArgs& a, int64_t row, float m, float s, float s1, float zt,
                                bool asked) {
    const bool empty = m == -INFINITY;
    const float lse = empty ? -INFINITY : m + logf(s);
    if (a.lse) a.lse[row] = lse;
    if (a.logprob) a.logprob[row] = !asked ? 0.0f : empty ? -INFINITY : (zt - m) - logf(s);
    if (a.entropy) a.entropy[row] = empty ? 0.0f : logf(s) - s1 / s;
}

// One workgroup takes one part of one row.  NV: 16-byte vectors a thread holds.
template <typename E, int NV, bool TOP>
__global__ __launch_bounds__(LP_THREADS, 6) void k_logprob(LpArgs a) {
    constexpr int VEC = 16 / sizeof(E);
    __shared__ float red[3][LP_WAVES];
    __shared__ float group_max[32];
    __shared__ float bound;
    __shared__ int count;
    __shared__ uint64_t cand[LP_CAND];
    __shared__ uint64_t best[LP_WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x / (uint32_t)a.parts;
    const int p = (int)(blockIdx.x % (uint32_t)a.parts);
    const E* const z = static_cast<const E*>(a.z) + row * a.ld;
    const int lo = p * a.part_len, hi = min(a.V, lo + a.part_len);

    // The part's whole vectors; what is left of it, less than one, goes one entry a thread.
    const int whole = (hi - lo) / VEC;
    u32x4 r[NV];
    if (whole > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            r[i] = load_words(z + lo + min(i * LP_THREADS + tid, whole - 1) * VEC);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i * LP_THREADS + tid >= whole) r[i] = u32x4(minus_infinity<E>());
    const int left = lo + whole * VEC + tid;
    const float extra = left < hi ? (float)z[left] : -INFINITY;
    float m = extra;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) m = max_nan(m, entry<E>(r[i], j));
    if constexpr (TOP) {   // maxima of 32 groups of 16 threads
        const float g = row_reduce(m, MaxNan());
        if ((lane & 15) == 0) group_max[wave * 4 + (lane >> 4)] = g;
        if (tid == 0) count = 0;
    }
    m = group_reduce(m, MaxNan(), red[0], wave, lane, LP_WAVES);
    if constexpr (TOP) {
        // the k-th largest of the group maxima: a wave ranks four of them, 16 lanes each
        const int g = wave * 4 + (lane >> 4), l = lane & 15;
        const uint64_t own = lp_rank(group_max[g], g);
        const uint64_t b0 = __ballot(lp_rank(group_max[l], l) > own);
        const uint64_t b1 = __ballot(lp_rank(group_max[l + 16], l + 16) > own);
        const int sh = lane & 48;
        const int above = __popc((uint32_t)(b0 >> sh) & 0xffffu) + __popc((uint32_t)(b1 >> sh) & 0xffffu);
        if (l == 0 && above == a.top - 1) bound = group_max[g];
    }
    const float ms = m == -INFINITY ? 0.0f : m;
    float s = 0.0f, s1 = 0.0f;
    auto add = [&](float x) {
        // (the bound keeps 0 * -inf out of s1; exp is 0 there)
        const float d = max_nan(x - ms, -200.0f);
        const float e = __builtin_amdgcn_exp2f(d * LOG2E);
        s += e;
        s1 = fmaf(e, d, s1);
    };
    add(extra);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        forget(r[i]);
#pragma unroll
        for (int j = 0; j < VEC; ++j) add(entry<E>(r[i], j));
    }
    s = wave_reduce(s, Add());
    s1 = wave_reduce(s1, Add());
    if (lane == 0) {
        red[1][wave] = s;
        red[2][wave] = s1;
    }
    __syncthreads();
    s = red[1][0];
    s1 = red[2][0];
#pragma unroll
    for (int w = 1; w < LP_WAVES; ++w) {
        s += red[1][w];
        s1 += red[2][w];
    }
    if (tid == 0) {
        if (a.parts == 1) {
            const int64_t t = a.target ? a.target[row] : -1;
            const bool asked = t >= 0 && t < a.V;
            lp_store(a, row, m, s, s1, asked ? (float)z[t] : 0.0f, asked);
        } else {
            a.part[row * a.parts + p] = LpPart{m, s, s1, 0.0f};
        }
    }
    if constexpr (TOP) {
        const float log_s = m == -INFINITY ? 0.0f : logf(s);
        const int64_t part = row * a.parts + p;
        auto put = [&](int k, uint64_t v) {
            if (a.parts == 1) {
                a.top_index[row * a.top + k] = lp_index(v);
                a.top_logprob[row * a.top + k] = (lp_unkey((uint32_t)(v >> 32)) - ms) - log_s;
            } else {
                a.cand[part * a.top + k] = v;
            }
        };
        // Every entry of the list has its own rank, whatever order it was filled in.
        auto rank = [&](int n) {
            for (int i = tid; i < n; i += LP_THREADS) {
                const uint64_t v = cand[i];
                int above = 0;
                for (int k = 0; k < n; ++k) above += cand[k] > v;
                if (above < a.top) put(above, v);
            }
        };
        const float b = bound;
        // Lists the entries not below b (NaN among them); or, where those are too many,
        // the ones above b alone: masked rows have thousands of -inf.
        int ties = b == -INFINITY, n;
        for (;;) {
            auto below = [&](float v) { return v < b || (ties && v == b); };
            auto offer = [&](float v, int c) {
                if (below(v)) return;
                const int at = atomicAdd(&count, 1);
                if (at < LP_CAND) cand[at] = lp_rank(v, c);
            };
            if (left < hi) offer(extra, left);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                forget(r[i]);
                float top = entry<E>(r[i], 0);
#pragma unroll
                for (int j = 1; j < VEC; ++j) top = max_nan(top, entry<E>(r[i], j));
                const int v = i * LP_THREADS + tid;
                if (below(top) || v >= whole) continue;
                int c = lo + v * VEC;
                asm volatile("" : "+v"(c));   // (computed here, not kept for every vector)
#pragma unroll
                for (int j = 0; j < VEC; ++j) offer(entry<E>(r[i], j), c + j);
            }
            __syncthreads();
            n = count;
            if (ties || n <= LP_CAND) break;
            __syncthreads();
            if (tid == 0) count = 0;
            __syncthreads();
            ties = 1;
        }
        if (n <= LP_CAND) {
            rank(n);
            // then the first entries equal to b, in the order of their indices
            for (int c0 = lo; ties && n < a.top && c0 < hi; c0 += LP_THREADS) {
                const bool is = c0 + tid < hi && (float)z[c0 + tid] == b;
                const uint64_t mask = __ballot(is);
                __syncthreads();
                if (lane == 0) best[wave] = __popcll(mask);
                __syncthreads();
                int at = n + __popcll(mask & ((1ull << lane) - 1));
                for (int w = 0; w < LP_WAVES; ++w) {
                    if (w < wave) at += (int)best[w];
                    n += (int)best[w];
                }
                if (is && at < a.top) put(at, lp_rank(b, c0 + tid));
            }
            for (int k = n + tid; k < a.top; k += LP_THREADS) put(k, 0);   // (part shorter than top)
        } else {
            // no bound, or a row in an order that defeats it (one group of threads far below the
            // others): the largest entry below the last one, top times
            uint64_t mine = 0, v = ~0ull;
            for (int k = 0; k < a.top; ++k) {
                if (k == 0 || mine == v) {
                    mine = 0;
                    for (int c = lo + tid; c < hi; c += LP_THREADS) {
                        const uint64_t o = lp_rank((float)z[c], c);
                        if (o < v && o > mine) mine = o;
                    }
                }
                v = wave_max_u64(mine);
                if (lane == 0) best[wave] = v;
                __syncthreads();
                v = best[0];
                for (int w = 1; w < LP_WAVES; ++w) v = best[w] > v ? best[w] : v;
                __syncthreads();
                if (tid == 0) put(k, v);
            }
        }
    }
}

// One wave joins the parts of a row, lane l holding part l.  The parts' sorted candidates
// wait in LDS.  With c the least number of candidates a part that makes `top` in all, the
// q-th largest (q = ceil(top / c)) of the parts' c-th candidates has q c >= top candidates at
// or above it: those, few more than `top` as a rule, are ranked by counting.  Where they are
// many (masked rows) the largest head of all lists is taken `top` times instead, 0.25 us each.
template <typename E>
__global__ __launch_bounds__(64) void k_logprob_join(LpArgs a) {
    __shared__ uint64_t lists[LP_PARTS * LP_TOP];
    __shared__ uint64_t chosen[LP_JOIN];
    __shared__ int count;
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    const uint64_t* const cand = a.cand + row * a.parts * a.top;
    for (int i = lane; i < a.parts * a.top; i += 64) lists[i] = cand[i];
    LpPart q{-INFINITY, 0.0f, 0.0f, 0.0f};
    if (lane < a.parts) q = a.part[row * a.parts + lane];
    const int64_t t = a.target ? a.target[row] : -1;
    const bool asked = t >= 0 && t < a.V;
    const float zt = asked ? (float)(static_cast<const E*>(a.z) + row * a.ld)[t] : 0.0f;
    const float m = wave_reduce(q.m, MaxNan());
    const float ms = m == -INFINITY ? 0.0f : m;
    const float d = max_nan(q.m - ms, -200.0f);
    const float e = __builtin_amdgcn_exp2f(d * LOG2E);
    const float s = wave_reduce(q.s * e, Add());
    const float s1 = wave_reduce(fmaf(d, q.s, q.s1) * e, Add());
    if (lane == 0) lp_store(a, row, m, s, s1, zt, asked);
    if (a.top == 0) return;
    const float log_s = m == -INFINITY ? 0.0f : logf(s);
    if (lane == 0) count = 0;
    __syncthreads();
    const int c = (a.top + a.parts - 1) / a.parts, q_th = (a.top + c - 1) / c;
    const uint64_t mark = lane < a.parts ? lists[lane * a.top + c - 1] : 0;
    int higher = 0;
    for (int i = 0; i < a.parts; ++i) higher += lists[i * a.top + c - 1] > mark;
    const uint64_t who = __ballot(mark != 0 && higher == q_th - 1);   // marks are distinct, but for 0
    const int from = who ? __ffsll((unsigned long long)who) - 1 : 0;
    const uint64_t bound =
        who ? ((uint64_t)lane_value((uint32_t)(mark >> 32), from) << 32) | lane_value((uint32_t)mark, from) : 1;
    for (int i = lane; i < a.parts * a.top; i += 64) {
        const uint64_t v = lists[i];
        if (v >= bound) {
            const int k = atomicAdd(&count, 1);
            if (k < LP_JOIN) chosen[k] = v;
        }
    }
    __syncthreads();
    const int n = count;
    auto put = [&](int k, uint64_t v) {
        a.top_index[row * a.top + k] = lp_index(v);
        a.top_logprob[row * a.top + k] = (lp_unkey((uint32_t)(v >> 32)) - ms) - log_s;
    };
    if (n <= LP_JOIN) {
        for (int i = lane; i < n; i += 64) {
            const uint64_t v = chosen[i];
            int above = 0;
            for (int k = 0; k < n; ++k) above += chosen[k] > v;
            if (above < a.top) put(above, v);
        }
        return;
    }
    int at = lane * a.top;
    const int end = lane < a.parts ? at + a.top : at;
    uint64_t head = at < end ? lists[at] : 0, mine = 0;
    for (int k = 0; k < a.top; ++k) {
        const uint64_t v = wave_max_u64(head);
        if (lane == k) mine = v;
        if (v == head) {   // keys are distinct: one lane
            ++at;
            head = at < end ? lists[at] : 0;
        }
    }
    if (lane < a.top) put(lane, mine);
}

struct LpGradArgs {
    const void* z;
    int64_t ld;
    const int64_t* target;
    const float *lse, *entropy, *g_logprob, *g_entropy;
    void* d;
    int64_t ldd;
    int V, pieces;
};

constexpr int LPG_NV = 4;   // vectors a thread has in flight

template <typename E, bool ENT>
__global__ __launch_bounds__(256) void k_logprob_grad(LpGradArgs a) {
    constexpr int VEC = 16 / sizeof(E);
    const int64_t row = blockIdx.x / (uint32_t)a.pieces;
    const int lo = (int)(blockIdx.x % (uint32_t)a.pieces) * (256 * LPG_NV * VEC);
    const E* const z = static_cast<const E*>(a.z) + row * a.ld;
    E* const out = static_cast<E*>(a.d) + row * a.ldd;
    // The piece's whole vectors; what is left of the row, less than one, goes one entry a
    // thread of the last piece.
    const int hi = min(a.V, lo + 256 * LPG_NV * VEC), whole = (hi - lo) / VEC;
    u32x4 r[LPG_NV];
    if (whole > 0) {
#pragma unroll
        for (int i = 0; i < LPG_NV; ++i)
            r[i] = load_words(z + lo + min(i * 256 + (int)threadIdx.x, whole - 1) * VEC);
    }
    float lse = a.lse[row];
    const bool empty = lse == -INFINITY;
    if (empty) lse = INFINITY;   // every p is then exp(-inf) = 0
    const int64_t t64 = a.target ? a.target[row] : -1;
    const bool asked = t64 >= 0 && t64 < a.V && !empty;
    const int t = asked ? (int)t64 : -1;
    const float gl = asked && a.g_logprob ? a.g_logprob[row] : 0.0f;
    const float gh = ENT ? a.g_entropy[row] : 0.0f, H = ENT ? a.entropy[row] : 0.0f;
    auto grad = [&](float x, int c) {
        const float lp = max_nan(x - lse, -200.0f);   // (exp is 0 there; 0 * -inf stays out)
        const float p = exp_of<sizeof(E) == 4>(lp);
        float g = gl;
        if (ENT) g = fmaf(gh, lp + H, gl);
        const float v = -p * g;
        return c == t ? v + gl : v;
    };
#pragma unroll
    for (int i = 0; i < LPG_NV; ++i) {
        const int v = i * 256 + (int)threadIdx.x;
        if (v >= whole) break;
        Pack<E, VEC> o;
#pragma unroll
        for (int j = 0; j < VEC; ++j) o.v[j] = (E)grad(entry<E>(r[i], j), lo + v * VEC + j);
        store_pack(out + lo + v * VEC, o);
    }
    const int left = lo + whole * VEC + (int)threadIdx.x;
    if (left < hi) out[left] = (E)grad((float)z[left], left);
}

// Parts of a row: as long as the registers allow with many rows; with few, so many
// that every CU has a workgroup, down to one vector a thread.
struct LpGeom {
    int parts, len, nv;
};
static LpGeom lp_geom(int64_t T, int64_t V, int esize) {
    const int64_t vec = 16 / esize, least = LP_THREADS * vec, most = LP_THREADS * LP_REGS * 4 / esize;
    int64_t parts = (V + most - 1) / most;
    const int64_t fill = (2 * 256 + T - 1) / T;   // two workgroups a CU
    if (parts < fill) parts = std::min<int64_t>(fill, (V + least - 1) / least);
    parts = std::min<int64_t>(parts, LP_PARTS);
    // (parts <= LP_PARTS always holds `most` entries a part at V <= 2^20)
    int64_t len = (V + parts - 1) / parts;
    len = (len + vec - 1) / vec * vec;
    LpGeom g;
    g.parts = (int)((V + len - 1) / len);
    g.len = (int)len;
    g.nv = (int)((len + least - 1) / least);
    return g;
}

template <typename E, int NV>
static void launch_logprob_nv(const LpArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)(a.T * a.parts));
    if (a.top)
        hipLaunchKernelGGL((k_logprob<E, NV, true>), grid, dim3(LP_THREADS), 0, st, a);
    else
        hipLaunchKernelGGL((k_logprob<E, NV, false>), grid, dim3(LP_THREADS), 0, st, a);
}

template <typename E>
static void launch_logprob(const LpArgs& a, int nv, hipStream_t st) {
    if (nv <= 1)
        launch_logprob_nv<E, 1>(a, st);
    else if (nv <= 2)
        launch_logprob_nv<E, 2>(a, st);
    else if (nv <= 4)
        launch_logprob_nv<E, 4>(a, st);
    else
        launch_logprob_nv<E, 8>(a, st);
    if (a.parts > 1)
        hipLaunchKernelGGL(k_logprob_join<E>, dim3((unsigned)a.T), dim3(64), 0, st, a);
}

template <typename E>
static void launch_logprob_grad(LpGradArgs a, int64_t T, hipStream_t st) {
    const int per = 256 * LPG_NV * 16 / (int)sizeof(E);
    a.pieces = (a.V + per - 1) / per;
    const dim3 grid((unsigned)(T * a.pieces));
    if (a.g_entropy)
        hipLaunchKernelGGL((k_logprob_grad<E, true>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((k_logprob_grad<E, false>), grid, dim3(256), 0, st, a);
}

}  // namespace bk

static bakron_status logprob_sizes(const char* who, int32_t dtype, int64_t T, int64_t V, int64_t ld) {
    if (dtype != BAKRON_F32 && dtype != BAKRON_F16 && dtype != BAKRON_BF16)
        return bk::op_fail(who, "bad dtype");
    if (T < 0 || T > bk::OP_T_MAX || V < 1 || V > ((int64_t)1 << 20) || ld < V) return bk::op_fail(who, "bad size");
    return BAKRON_OK;
}

extern "C" bakron_status bakron_token_logprobs(const void* logits, int64_t ld, int32_t dtype,
                                               int64_t T, int64_t V, const int64_t* target,
                                               int32_t top, float* logprob, float* entropy,
                                               float* lse, float* top_logprob, int64_t* top_index,
                                               void* work, size_t* work_bytes, hipStream_t stream) {
    static const char who[] = "bakron_token_logprobs";
    bk::set_last_error("");
    bakron_status st = logprob_sizes(who, dtype, T, V, ld);
    if (st != BAKRON_OK) return st;
    if (top < 0 || top > bk::LP_TOP || top > V) return bk::op_fail(who, "bad number of alternatives");
    const int esize = dtype == BAKRON_F32 ? 4 : 2;
    const bk::LpGeom g = bk::lp_geom(T ? T : 1, V, esize);
    if (T > bk::OP_LAUNCH_MAX / bk::LP_THREADS / g.parts)
        return bk::op_fail(who, "too many rows for one call");
    const size_t stats = (size_t)T * g.parts * sizeof(bk::LpPart);
    const size_t need = g.parts > 1 ? stats + (size_t)T * g.parts * top * sizeof(uint64_t) : 0;
    bool query;
    st = bk::op_workspace(who, work, work_bytes, need, &query);
    if (st != BAKRON_OK || query) return st;
    if (logprob && !target) return bk::op_fail(who, "logprob needs targets");
    if ((top > 0) != (top_logprob != nullptr) || (top > 0) != (top_index != nullptr))
        return bk::op_fail(who, "top outputs go with top");
    if (T == 0) return BAKRON_OK;
    if (!logits) return bk::op_fail(who, "null pointer");
    bk::LpArgs a{logits, ld, target, T, (int)V, g.len, g.parts, top, logprob, entropy, lse,
                 top_logprob, top_index, static_cast<bk::LpPart*>(work),
                 reinterpret_cast<uint64_t*>(static_cast<char*>(work) + stats)};
    if (dtype == BAKRON_F32)
        bk::launch_logprob<float>(a, g.nv, stream);
    else if (dtype == BAKRON_F16)
        bk::launch_logprob<bk::f16_t>(a, g.nv, stream);
    else
        bk::launch_logprob<bk::bf16_t>(a, g.nv, stream);
    return bk::op_launched(who);
}

extern "C" bakron_status bakron_token_logprobs_backward(
    const void* logits, int64_t ld, int32_t dtype, int64_t T, int64_t V, const int64_t* target,
    const float* lse, const float* entropy, const float* g_logprob, const float* g_entropy, void* d,
    int64_t ldd, hipStream_t stream) {
    static const char who[] = "bakron_token_logprobs_backward";
    bk::set_last_error("");
    bakron_status st = logprob_sizes(who, dtype, T, V, ld);
    if (st != BAKRON_OK) return st;
    if (ldd < V) return bk::op_fail(who, "bad size");
    const int64_t per = 256 * bk::LPG_NV * 16 / (dtype == BAKRON_F32 ? 4 : 2);
    if (T > bk::OP_LAUNCH_MAX / 256 / ((V + per - 1) / per))
        return bk::op_fail(who, "too many rows for one call");
    if (d == logits && ldd != ld) return bk::op_fail(who, "in place needs ldd = ld");
    if (g_logprob && !target) return bk::op_fail(who, "g_logprob needs targets");
    if (g_entropy && !entropy) return bk::op_fail(who, "g_entropy needs the entropies");
    if (T == 0) return BAKRON_OK;
    if (!logits || !lse || !d) return bk::op_fail(who, "null pointer");
    bk::LpGradArgs a{logits, ld, target, lse, entropy, g_logprob, g_entropy, d, ldd, (int)V, 0};
    if (dtype == BAKRON_F32)
        bk::launch_logprob_grad<float>(a, T, stream);
    else if (dtype == BAKRON_F16)
        bk::launch_logprob_grad<bk::f16_t>(a, T, stream);
    else
        bk::launch_logprob_grad<bk::bf16_t>(a, T, stream);
    return bk::op_launched(who);
}
