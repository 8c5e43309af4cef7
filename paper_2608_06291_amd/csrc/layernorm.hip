// Layer norm and RMS norm of a residual stream with the rows' statistics, and their gradients.
//
//   h = x + r (rounded once, as the stream holds it),   n = (h - mean) / sqrt(var + eps),   y = w (.) n + b
//   g = w (.) dy,   dx = (g - mean(g) - n mean(g n)) / sqrt(var + eps) + d_sum
//   dw = sum_t dy_t (.) n_t,   db = sum_t dy_t
// with mean 0, var = mean(h^2) and no mean(g) for the RMS norm.
//
// Bound by memory: a row is read once and stays in registers over its reductions.  4096 x 8192 bf16 with a residual
// 44 to 53 us, 5.1 to 6.1 TB/s of 269 MB (a large copy here: 5.1), 2048 x 8192 fp32 44; its gradients 53 and 5 for the join
// of the columns' sums, 268 MB at 5.0 TB/s and 34 more of partial sums (dx and the columns apart, which reads x and dy twice:
// 89).  Rows of more than 16384 16-bit or 8192 fp32 entries do not leave registers for the columns' sums and go that way:
// 1024 x 32768 bf16 69 us.
#include <algorithm>

#include "ops.h"

namespace bk {

struct LnArgs {
    const void* x;
    const void* res;
    const float *w, *b;
    void *sum, *y;
    float *mean, *rstd;
    int64_t ldx, ldr, lds, ldy, T;
    int d, centre;
    float eps;
};

// Two sums over `waves` waves of a workgroup at once; `red` as of group_reduce, twice as long.
__device__ inline void group_sum2(float& a, float& b, float* red, int wave, int lane, int waves) {
    a = wave_reduce(a, Add());
    b = wave_reduce(b, Add());
    if (waves == 1) return;
    if (lane == 0) {
        red[2 * wave] = a;
        red[2 * wave + 1] = b;
    }
    __syncthreads();
    a = red[0];
    b = red[1];
    for (int w = 1; w < waves; ++w) {
        a += red[2 * w];
        b += red[2 * w + 1];
    }
}

// A row belongs to blockDim.x threads (one wave, with blockDim.y rows in the workgroup, or the
// whole workgroup); thread t holds the whole vectors t, t + blockDim.x, .. of VEC entries, NV of them,
// and one entry of what is left of the row.  Loads are whole vectors at clamped addresses, issued together.
//
// The mean's own rounding would be an error of every n where |mean| is far beyond the deviation, so the
// entries less the rounded mean are summed as well, and what that leaves is taken off.
template <typename E, int NV>
__global__ __launch_bounds__(1024) void k_layernorm(LnArgs a) {
    constexpr int VEC = 16 / sizeof(E);
    __shared__ float red[3][32];
    const int tid = threadIdx.x, tpr = blockDim.x, lane = tid & 63, wave = tid >> 6;
    const int waves = tpr >> 6;
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= a.T) return;   // (a whole wave, and never one of several in a row)
    const E* const x = static_cast<const E*>(a.x) + row * a.ldx;
    const E* const res = a.res ? static_cast<const E*>(a.res) + row * a.ldr : nullptr;
    const int whole = a.d / VEC, left = whole * VEC + tid;

    constexpr int STEP = NV * VEC <= 32 ? NV : 32 / VEC;   // vectors read at once
    float h[NV][VEC], hx = 0.0f, s = 0.0f;
#pragma unroll
    for (int i0 = 0; i0 < NV; i0 += STEP) {
        u32x4 rx[STEP], rr[STEP];
#pragma unroll
        for (int i = 0; i < STEP; ++i) rx[i] = rr[i] = u32x4(0);
        if (whole > 0) {   // (past the row its last vector, not used)
#pragma unroll
            for (int i = 0; i < STEP; ++i) rx[i] = load_words(x + min((i0 + i) * tpr + tid, whole - 1) * VEC);
            if (res) {
#pragma unroll
                for (int i = 0; i < STEP; ++i) rr[i] = load_words(res + min((i0 + i) * tpr + tid, whole - 1) * VEC);
            }
        }
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
            const bool in = (i0 + i) * tpr + tid < whole;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                float v = entry<E>(rx[i], j);
                if (res) v = (float)(E)(v + entry<E>(rr[i], j));
                h[i0 + i][j] = in ? v : 0.0f;
                s += h[i0 + i][j];
            }
        }
    }
    if (left < a.d) {
        hx = (float)x[left];
        if (res) hx = (float)(E)(hx + (float)res[left]);
    }
    s += hx;
    auto store = [&](void* base, int64_t ld) {
        E* const out = static_cast<E*>(base) + row * ld;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * tpr + tid;
            Pack<E, VEC> p;
#pragma unroll
            for (int j = 0; j < VEC; ++j) p.v[j] = (E)h[i][j];
            if (v < whole) store_pack(out + v * VEC, p);
        }
        if (left < a.d) out[left] = (E)hx;
    };
    if (a.sum) store(a.sum, a.lds);
    const float inv_d = 1.0f / (float)a.d;
    float mean = 0.0f, rest = 0.0f, sq = 0.0f;
    if (a.centre) {
        mean = group_reduce(s, Add(), red[0], wave, lane, waves) * inv_d;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const bool in = i * tpr + tid < whole;
#pragma unroll
            for (int j = 0; j < VEC; ++j) h[i][j] = in ? h[i][j] - mean : 0.0f;
        }
        hx = left < a.d ? hx - mean : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            rest += h[i][j];
            sq = fmaf(h[i][j], h[i][j], sq);
        }
    rest += hx;
    sq = fmaf(hx, hx, sq);
    group_sum2(rest, sq, red[1], wave, lane, waves);
    rest = a.centre ? rest * inv_d : 0.0f;
    const float v = fmaxf(sq * inv_d - rest * rest, 0.0f) + a.eps;
    const float r = v < INFINITY && sq < INFINITY ? 1.0f / sqrtf(v) : NAN;   // squares beyond fp32: not silently 0
    if (tid == 0) {
        if (a.mean) a.mean[row] = mean + rest;
        if (a.rstd) a.rstd[row] = r;
    }
    if (!a.y) return;
    const float off = -rest * r;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        Pack<float, VEC> w, b;
        const int at = min(i * tpr + tid, whole - 1) * VEC;
        if (a.w && whole > 0) w = load_pack<float, VEC>(a.w + at);
        if (a.b && whole > 0) b = load_pack<float, VEC>(a.b + at);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            float n = fmaf(h[i][j], r, off);
            if (a.w) n *= w.v[j];
            if (a.b) n += b.v[j];
            h[i][j] = n;
        }
    }
    if (left < a.d) {
        hx = fmaf(hx, r, off);
        if (a.w) hx *= a.w[left];
        if (a.b) hx += a.b[left];
    }
    store(a.y, a.ldy);
}

struct LnGradArgs {
    const void *dy, *x, *ds;
    const float *w, *mean, *rstd;
    void* dx;
    float *dw, *db;
    float* part;   // slices x 2 x dp, dp: d rounded up to a multiple of 8
    int64_t lddy, ldx, ldds, lddx, T;
    int d, slices, dx_blocks;
};

// dx, a row a group of threads as above.
template <typename E, int NV>
__device__ inline void layernorm_dx(const LnGradArgs& a) {
    constexpr int VEC = 16 / sizeof(E);
    __shared__ float red[32];
    const int tid = threadIdx.x, tpr = blockDim.x, lane = tid & 63, wave = tid >> 6;
    const int waves = tpr >> 6;
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= a.T) return;
    const E* const x = static_cast<const E*>(a.x) + row * a.ldx;
    const E* const dy = static_cast<const E*>(a.dy) + row * a.lddy;
    const int whole = a.d / VEC, left = whole * VEC + tid;
    const float mean = a.mean ? a.mean[row] : 0.0f, r = a.rstd[row];
    u32x4 rx[NV], rg[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) rx[i] = rg[i] = u32x4(0);
    if (whole > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            rx[i] = load_words(x + min(i * tpr + tid, whole - 1) * VEC);
            rg[i] = load_words(dy + min(i * tpr + tid, whole - 1) * VEC);
        }
    }
    float sg = 0.0f, sn = 0.0f;
    auto weight = [&](int i) {
        Pack<float, VEC> w;
        if (a.w && whole > 0) return load_pack<float, VEC>(a.w + min(i * tpr + tid, whole - 1) * VEC);
#pragma unroll
        for (int j = 0; j < VEC; ++j) w.v[j] = 1.0f;
        return w;
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i * tpr + tid >= whole) rg[i] = u32x4(0);
        const auto w = weight(i);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float g = entry<E>(rg[i], j) * w.v[j], n = (entry<E>(rx[i], j) - mean) * r;
            sg += g;
            sn += i * tpr + tid < whole ? g * n : 0.0f;
        }
    }
    float gx = 0.0f, nx = 0.0f;
    if (left < a.d) {
        gx = (float)dy[left] * (a.w ? a.w[left] : 1.0f);
        nx = ((float)x[left] - mean) * r;
    }
    sg += gx;
    sn = fmaf(gx, nx, sn);
    group_sum2(sg, sn, red, wave, lane, waves);
    sg = a.mean ? sg / (float)a.d : 0.0f;
    sn /= (float)a.d;
    E* const out = static_cast<E*>(a.dx) + row * a.lddx;
    const E* const ds = a.ds ? static_cast<const E*>(a.ds) + row * a.ldds : nullptr;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = i * tpr + tid;
        if (v >= whole) break;
        const auto w = weight(i);
        u32x4 rs = u32x4(0);
        if (ds) rs = load_words(ds + v * VEC);
        Pack<E, VEC> o;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float g = entry<E>(rg[i], j) * w.v[j], n = (entry<E>(rx[i], j) - mean) * r;
            o.v[j] = (E)fmaf(g - sg - n * sn, r, entry<E>(rs, j));
        }
        store_pack(out + v * VEC, o);
    }
    if (left < a.d) out[left] = (E)fmaf(gx - sg - nx * sn, r, ds ? (float)ds[left] : 0.0f);
}

template <typename E, int NV>
__global__ __launch_bounds__(1024) void k_layernorm_dx(LnGradArgs a) {
    layernorm_dx<E, NV>(a);
}
// Few rows: dx by the first dx_blocks workgroups, dw and db by the others, a vector of columns a thread and all rows.
// Neither needs the other, nor a join: 1 x 4096 f16 13.8 us a call in two launches with a workspace, 9.6 so.
template <typename E, int NV>
__global__ __launch_bounds__(1024) void k_layernorm_few(LnGradArgs a) {
    constexpr int VEC = 16 / sizeof(E), AHEAD = 4;
    if ((int)blockIdx.x < a.dx_blocks) return layernorm_dx<E, NV>(a);
    const int threads = blockDim.x * blockDim.y, tid = threadIdx.y * blockDim.x + threadIdx.x;
    const int c = (((int)blockIdx.x - a.dx_blocks) * threads + tid) * VEC;
    if (c >= a.d) return;
    float dw[VEC] = {}, db[VEC] = {};
    const int T = (int)a.T;
    if (c + VEC <= a.d) {
        for (int t0 = 0; t0 < T; t0 += AHEAD) {
            u32x4 x[AHEAD], g[AHEAD];
            float mean[AHEAD], r[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int64_t t = min(t0 + i, T - 1);
                x[i] = load_words(static_cast<const E*>(a.x) + t * a.ldx + c);
                g[i] = load_words(static_cast<const E*>(a.dy) + t * a.lddy + c);
                mean[i] = a.mean ? a.mean[t] : 0.0f;
                r[i] = a.rstd[t];
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (t0 + i < T) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const float dy = entry<E>(g[i], j);
                        dw[j] = fmaf(dy, (entry<E>(x[i], j) - mean[i]) * r[i], dw[j]);
                        db[j] += dy;
                    }
                }
        }
    } else {
        for (int64_t t = 0; t < T; ++t)
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (c + j < a.d) {
                    const float dy = (float)static_cast<const E*>(a.dy)[t * a.lddy + c + j];
                    const float x = (float)static_cast<const E*>(a.x)[t * a.ldx + c + j];
                    dw[j] = fmaf(dy, (x - (a.mean ? a.mean[t] : 0.0f)) * a.rstd[t], dw[j]);
                    db[j] += dy;
                }
    }
    if (a.dw) store_n(a.dw + c, dw, a.d - c);
    if (a.db) store_n(a.db + c, db, a.d - c);
}
constexpr int64_t LN_FEW_ROWS = 32;

// Partial sums of dw and db over a slice of the rows: a thread has VEC columns, the four waves of a
// workgroup the same columns and every fourth row, joined in LDS.
template <typename E>
__global__ __launch_bounds__(256) void k_layernorm_dw(LnGradArgs a) {
    constexpr int VEC = 16 / sizeof(E);
    __shared__ float red[3][2 * VEC][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = ((int)blockIdx.x * 64 + lane) * VEC;
    const int64_t per = (a.T + a.slices - 1) / a.slices;
    const int64_t lo = blockIdx.y * per, hi = min(a.T, lo + per);
    float dw[VEC] = {}, db[VEC] = {};
    if (c < a.d) {
        for (int64_t t = lo + wave; t < hi; t += 4) {
            const float mean = a.mean ? a.mean[t] : 0.0f, r = a.rstd[t];
            const E* const x = static_cast<const E*>(a.x) + t * a.ldx + c;
            const E* const dy = static_cast<const E*>(a.dy) + t * a.lddy + c;
            float vx[VEC], vg[VEC];
            if (c + VEC <= a.d) {
                const u32x4 px = load_words(x), pg = load_words(dy);
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    vx[j] = entry<E>(px, j);
                    vg[j] = entry<E>(pg, j);
                }
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    vx[j] = c + j < a.d ? (float)x[j] : 0.0f;
                    vg[j] = c + j < a.d ? (float)dy[j] : 0.0f;
                }
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                dw[j] = fmaf(vg[j], (vx[j] - mean) * r, dw[j]);
                db[j] += vg[j];
            }
        }
    }
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            red[wave - 1][j][lane] = dw[j];
            red[wave - 1][VEC + j][lane] = db[j];
        }
    }
    __syncthreads();
    if (wave > 0) return;
    const int64_t dp = (a.d + 7) / 8 * 8;
    float* const part = a.part + blockIdx.y * 2 * dp + c;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        if (c + j >= a.d) break;
        part[j] = dw[j] + red[0][j][lane] + red[1][j][lane] + red[2][j][lane];
        part[dp + j] = db[j] + red[0][VEC + j][lane] + red[1][VEC + j][lane] + red[2][VEC + j][lane];
    }
}

// Sums the slices: a lane has one column of dw or db, the 16 waves every 16th slice each, joined in their order.
__global__ __launch_bounds__(1024) void k_layernorm_join(LnGradArgs a) {
    __shared__ float red[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int dp = (a.d + 7) / 8 * 8, c = (int)blockIdx.x * 64 + lane;
    float sum = 0.0f;
    if (c < 2 * dp) {
        constexpr int AHEAD = 8;
        for (int s = wave; s < a.slices; s += 16 * AHEAD) {
            float v[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) v[i] = a.part[(int64_t)min(s + 16 * i, a.slices - 1) * 2 * dp + c];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) sum += s + 16 * i < a.slices ? v[i] : 0.0f;
        }
    }
    red[wave][lane] = sum;
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < 16; ++w) sum += red[w][lane];
    if (c < a.d && a.dw) a.dw[c] = sum;
    if (c >= dp && c < dp + a.d && a.db) a.db[c - dp] = sum;
}

// Both at once, for rows that a workgroup's registers hold with the columns' sums beside them: a workgroup takes
// every G-th block of rows (a row a group of tpr threads), the next rows on their way while one is summed, and
// keeps sum dy n and sum dy of its columns.  x and dy are read once.  What is left of a row (less than a
// vector) goes one entry a thread.
template <typename E, int NV>
__global__ __launch_bounds__(1024) void k_layernorm_grad(LnGradArgs a) {
    constexpr int VEC = 16 / sizeof(E);
    extern __shared__ __attribute__((aligned(16))) float sums[];   // rows of the workgroup beyond one: their columns' sums
    __shared__ __attribute__((aligned(16))) float red[2][32];
    const int tid = threadIdx.x, tpr = blockDim.x, lane = tid & 63, wave = tid >> 6;
    const int waves = tpr >> 6, ys = blockDim.y;
    const int whole = a.d / VEC, left = whole * VEC + tid;
    const bool more = left < a.d;
    float dw[NV][VEC] = {}, db[NV][VEC] = {}, dwx = 0.0f, dbx = 0.0f;
    const float inv_d = 1.0f / (float)a.d;

    struct Row {
        u32x4 x[NV], g[NV];
        float xl, gl, mean, r;
    };
    auto load = [&](Row& row, int64_t t) {
        const E* const x = static_cast<const E*>(a.x) + t * a.ldx;
        const E* const dy = static_cast<const E*>(a.dy) + t * a.lddy;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            row.x[i] = row.g[i] = u32x4(0);
            if (whole > 0) {
                row.x[i] = load_words(x + min(i * tpr + tid, whole - 1) * VEC);
                row.g[i] = load_words(dy + min(i * tpr + tid, whole - 1) * VEC);
            }
        }
        row.xl = more ? (float)x[left] : 0.0f;
        row.gl = more ? (float)dy[left] : 0.0f;
        row.mean = a.mean ? a.mean[t] : 0.0f;
        row.r = a.rstd[t];
    };
    Pack<float, VEC> w[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) w[i].v[j] = 1.0f;
        if (a.w && whole > 0) w[i] = load_pack<float, VEC>(a.w + min(i * tpr + tid, whole - 1) * VEC);
    }
    const float wl = a.w && more ? a.w[left] : 1.0f;

    const int64_t step = (int64_t)gridDim.x * ys;
    int64_t t = (int64_t)blockIdx.x * ys + threadIdx.y;
    Row cur, next;
    if (t < a.T) load(next, t);
    int turn = 0;
    // (with several rows a workgroup each is one wave: no barrier in here)
    for (; t < a.T; t += step, turn ^= 1) {
        cur = next;
        u32x4 rs[NV];
        float rsl = 0.0f;
        if (a.dx && a.ds) {
            const E* const ds = static_cast<const E*>(a.ds) + t * a.ldds;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                rs[i] = u32x4(0);
                if (whole > 0) rs[i] = load_words(ds + min(i * tpr + tid, whole - 1) * VEC);
            }
            if (more) rsl = (float)ds[left];
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) rs[i] = u32x4(0);
        }
        if (t + step < a.T) load(next, t + step);
        float sg = 0.0f, sn = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (i * tpr + tid < whole) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float dy = entry<E>(cur.g[i], j), g = dy * w[i].v[j];
                    const float n = (entry<E>(cur.x[i], j) - cur.mean) * cur.r;
                    sg += g;
                    sn = fmaf(g, n, sn);
                    dw[i][j] = fmaf(dy, n, dw[i][j]);
                    db[i][j] += dy;
                }
            }
        }
        const float gl = cur.gl * wl, nl = more ? (cur.xl - cur.mean) * cur.r : 0.0f;
        sg += gl;
        sn = fmaf(gl, nl, sn);
        dwx = fmaf(cur.gl, nl, dwx);
        dbx += cur.gl;
        if (!a.dx) continue;
        group_sum2(sg, sn, red[turn], wave, lane, waves);
        sg = a.mean ? sg * inv_d : 0.0f;
        sn *= inv_d;
        E* const out = static_cast<E*>(a.dx) + t * a.lddx;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = i * tpr + tid;
            Pack<E, VEC> o;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float g = entry<E>(cur.g[i], j) * w[i].v[j], n = (entry<E>(cur.x[i], j) - cur.mean) * cur.r;
                o.v[j] = (E)fmaf(g - sg - n * sn, cur.r, entry<E>(rs[i], j));
            }
            if (v < whole) store_pack(out + v * VEC, o);
        }
        if (more) out[left] = (E)fmaf(gl - sg - nl * sn, cur.r, rsl);
    }
    // the rows of a workgroup, in their order
    const int64_t dp = (a.d + 7) / 8 * 8;
    float* const part = a.part + (int64_t)blockIdx.x * 2 * dp;
    for (int y = 1; y < ys; ++y) {
        if ((int)threadIdx.y == y) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    sums[(i * VEC + j) * 64 + lane] = dw[i][j];
                    sums[(NV * VEC + i * VEC + j) * 64 + lane] = db[i][j];
                }
            sums[2 * NV * VEC * 64 + lane] = dwx;
            sums[2 * NV * VEC * 64 + 64 + lane] = dbx;
        }
        __syncthreads();
        if (threadIdx.y == 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    dw[i][j] += sums[(i * VEC + j) * 64 + lane];
                    db[i][j] += sums[(NV * VEC + i * VEC + j) * 64 + lane];
                }
            dwx += sums[2 * NV * VEC * 64 + lane];
            dbx += sums[2 * NV * VEC * 64 + 64 + lane];
        }
        __syncthreads();
    }
    if (threadIdx.y != 0) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = i * tpr + tid;
        if (v >= whole) break;
        store_n(part + v * VEC, dw[i], VEC);
        store_n(part + dp + v * VEC, db[i], VEC);
    }
    if (more) {
        part[left] = dwx;
        part[dp + left] = dbx;
    }
}

// Threads a row, vectors a thread and rows a workgroup.
struct LnGeom {
    int tpr, nv, rows;
};
static LnGeom ln_geom(int64_t T, int64_t d, int vec, int nv_max) {
    const int vecs = (int)((d + vec - 1) / vec);
    LnGeom g{64, T < 1024 ? 1 : 2, 1};
    while (g.tpr < 1024 && g.tpr * g.nv < vecs) g.tpr *= 2;
    while (g.nv < nv_max && g.tpr * g.nv < vecs) g.nv *= 2;
    if (g.tpr == 64) g.rows = 4;
    return g;
}

template <typename E>
static void launch_layernorm(const LnArgs& a, hipStream_t st) {
    constexpr int VEC = 16 / sizeof(E), NV_MAX = 64 / VEC;
    const LnGeom g = ln_geom(a.T, a.d, VEC, NV_MAX);
    const dim3 grid((unsigned)((a.T + g.rows - 1) / g.rows)), block(g.tpr, g.rows);
    switch (g.nv) {
        case 1: hipLaunchKernelGGL((k_layernorm<E, 1>), grid, block, 0, st, a); break;
        case 2: hipLaunchKernelGGL((k_layernorm<E, 2>), grid, block, 0, st, a); break;
        case 4: hipLaunchKernelGGL((k_layernorm<E, 4>), grid, block, 0, st, a); break;
        case 8: hipLaunchKernelGGL((k_layernorm<E, 8>), grid, block, 0, st, a); break;
        default: hipLaunchKernelGGL((k_layernorm<E, NV_MAX>), grid, block, 0, st, a); break;
    }
}

// The gradients together, where a row is at most two vectors a thread of 1024; else dx, then dw and db from x and
// dy read once more.  Slices of the rows: together, one a CU, more where each still has 16 blocks of rows, because a
// slice's sums are as much to write and read as two rows; else so many that every CU has two workgroups.
constexpr int LN_GRAD_NV = 2;   // vectors a thread
static bool ln_together(int64_t d, int esize) { return d * esize <= LN_GRAD_NV * 16 * 1024; }
static int ln_slices(int64_t T, int64_t d, int esize) {
    if (ln_together(d, esize)) {
        const LnGeom g = ln_geom(1 << 20, d, 16 / esize, LN_GRAD_NV);
        const int64_t blocks = (T + g.rows - 1) / g.rows, cus = op_cus();
        const int64_t most = cus * std::max(1, 512 / (g.tpr * g.rows));   // so many have room
        return (int)std::max<int64_t>(1, std::min({blocks, most, std::max(cus, blocks / 16)}));
    }
    const int64_t blocks = (d * esize + 1023) / 1024;   // of columns
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(512 / blocks + 1, (T + 15) / 16), 256));
}

template <typename E>
static void launch_layernorm_grad(LnGradArgs a, hipStream_t st) {
    constexpr int VEC = 16 / sizeof(E), NV_MAX = 64 / VEC;
    const bool columns = a.dw || a.db;
    // dx in the place of dy or x: where others than the row's own threads read them, the columns' sums come first
    if (columns && a.dx && (a.dx == a.dy || a.dx == a.x) && (a.T <= LN_FEW_ROWS || !ln_together(a.d, sizeof(E)))) {
        LnGradArgs c = a;
        c.dx = nullptr;
        a.dw = a.db = nullptr;
        launch_layernorm_grad<E>(c, st);
        return launch_layernorm_grad<E>(a, st);
    }
    if (columns) a.slices = ln_slices(a.T, a.d, sizeof(E));
    if (columns && a.T <= LN_FEW_ROWS) {
        const LnGeom g = ln_geom(a.T, a.d, VEC, NV_MAX);
        const int each = g.tpr * g.rows * VEC;   // columns a workgroup
        a.dx_blocks = a.dx ? (int)((a.T + g.rows - 1) / g.rows) : 0;
        const dim3 grid((unsigned)(a.dx_blocks + (a.d + each - 1) / each)), block(g.tpr, g.rows);
        switch (g.nv) {
            case 1: hipLaunchKernelGGL((k_layernorm_few<E, 1>), grid, block, 0, st, a); break;
            case 2: hipLaunchKernelGGL((k_layernorm_few<E, 2>), grid, block, 0, st, a); break;
            case 4: hipLaunchKernelGGL((k_layernorm_few<E, 4>), grid, block, 0, st, a); break;
            case 8: hipLaunchKernelGGL((k_layernorm_few<E, 8>), grid, block, 0, st, a); break;
            default: hipLaunchKernelGGL((k_layernorm_few<E, NV_MAX>), grid, block, 0, st, a); break;
        }
        return;
    }
    if (columns && ln_together(a.d, sizeof(E))) {
        const LnGeom g = ln_geom(1 << 20, a.d, VEC, LN_GRAD_NV);
        const dim3 grid((unsigned)a.slices), block(g.tpr, g.rows);
        const int lds = g.rows > 1 ? (2 * g.nv * VEC + 2) * 64 * (int)sizeof(float) : 0;
        hipLaunchKernelGGL((k_layernorm_grad<E, LN_GRAD_NV>), grid, block, lds, st, a);
    } else if (a.dx) {
        const LnGeom g = ln_geom(a.T, a.d, VEC, NV_MAX);
        const dim3 grid((unsigned)((a.T + g.rows - 1) / g.rows)), block(g.tpr, g.rows);
        switch (g.nv) {
            case 1: hipLaunchKernelGGL((k_layernorm_dx<E, 1>), grid, block, 0, st, a); break;
            case 2: hipLaunchKernelGGL((k_layernorm_dx<E, 2>), grid, block, 0, st, a); break;
            case 4: hipLaunchKernelGGL((k_layernorm_dx<E, 4>), grid, block, 0, st, a); break;
            case 8: hipLaunchKernelGGL((k_layernorm_dx<E, 8>), grid, block, 0, st, a); break;
            default: hipLaunchKernelGGL((k_layernorm_dx<E, NV_MAX>), grid, block, 0, st, a); break;
        }
    }
    if (!columns) return;
    if (!ln_together(a.d, sizeof(E))) {
        const dim3 grid((unsigned)((a.d + 64 * VEC - 1) / (64 * VEC)), (unsigned)a.slices);
        hipLaunchKernelGGL(k_layernorm_dw<E>, grid, dim3(256), 0, st, a);
    }
    hipLaunchKernelGGL(k_layernorm_join, dim3((unsigned)((2 * ((a.d + 7) / 8 * 8) + 63) / 64)), dim3(1024), 0, st, a);
}

}  // namespace bk

static bakron_status layernorm_sizes(const char* who, int32_t dtype, int64_t T, int64_t d) {
    if (T < 0 || T > bk::OP_T_MAX || d < 1 || d > 65536) return bk::op_fail(who, "bad size");
    if (dtype != BAKRON_F32 && dtype != BAKRON_F16 && dtype != BAKRON_BF16) return bk::op_fail(who, "bad dtype");
    const int vec = dtype == BAKRON_F32 ? 4 : 8;
    if (T > bk::OP_LAUNCH_MAX / bk::ln_geom(T, d, vec, 64 / vec).tpr)
        return bk::op_fail(who, "too many rows for one call");
    return BAKRON_OK;
}

extern "C" bakron_status bakron_layernorm(const void* x, int64_t ldx, const void* residual, int64_t ldr, int32_t dtype,
                                          int64_t T, int64_t d, const float* weight, const float* bias, float eps,
                                          int32_t centre, void* sum, int64_t lds, void* y, int64_t ldy, float* mean,
                                          float* rstd, hipStream_t stream) {
    static const char who[] = "bakron_layernorm";
    bk::set_last_error("");
    const bakron_status st = layernorm_sizes(who, dtype, T, d);
    if (st != BAKRON_OK) return st;
    if (!(eps >= 1e-30f) || !std::isfinite(eps)) return bk::op_fail(who, "bad eps");
    if (ldx < d || (residual && ldr < d) || (sum && lds < d) || (y && ldy < d))
        return bk::op_fail(who, "leading dimension below d");
    if ((sum && sum == x && lds != ldx) || (sum && sum == residual && lds != ldr))
        return bk::op_fail(who, "sum in place needs the same leading dimension");
    if (mean && !centre) return bk::op_fail(who, "mean goes with centre");
    if (T == 0) return BAKRON_OK;
    if (!x || (!sum && !y && !mean && !rstd)) return bk::op_fail(who, "null pointer");
    const bk::LnArgs a{x, residual, weight, bias, sum, y, mean, rstd, ldx, ldr, lds, ldy, T, (int)d, centre != 0, eps};
    if (dtype == BAKRON_F32)
        bk::launch_layernorm<float>(a, stream);
    else if (dtype == BAKRON_F16)
        bk::launch_layernorm<bk::f16_t>(a, stream);
    else
        bk::launch_layernorm<bk::bf16_t>(a, stream);
    return bk::op_launched(who);
}

extern "C" bakron_status bakron_layernorm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx,
                                                   int32_t dtype, int64_t T, int64_t d, const float* weight,
                                                   const float* mean, const float* rstd, const void* d_sum,
                                                   int64_t ldds, void* dx, int64_t lddx, float* dweight, float* dbias,
                                                   void* work, size_t* work_bytes, hipStream_t stream) {
    static const char who[] = "bakron_layernorm_backward";
    bk::set_last_error("");
    bakron_status st = layernorm_sizes(who, dtype, T, d);
    if (st != BAKRON_OK) return st;
    const int esize = dtype == BAKRON_F32 ? 4 : 2;
    const size_t need = (dweight || dbias) && T > bk::LN_FEW_ROWS ? (size_t)bk::ln_slices(T, d, esize) * 2 * ((d + 7) / 8 * 8) * sizeof(float) : 0;
    bool query;
    st = bk::op_workspace(who, work, work_bytes, need, &query);
    if (st != BAKRON_OK || query) return st;
    if (lddy < d || ldx < d || (d_sum && ldds < d) || (dx && lddx < d))
        return bk::op_fail(who, "leading dimension below d");
    if (dx && ((dx == d_sum && lddx != ldds) || (dx == dy && lddx != lddy) || (dx == x && lddx != ldx)))
        return bk::op_fail(who, "dx in place needs the same leading dimension");
    if (!dx && !dweight && !dbias) return bk::op_fail(who, "null pointer");
    if (T > 0 && (!dy || !x || !rstd)) return bk::op_fail(who, "null pointer");
    if (T == 0 && !dweight && !dbias) return BAKRON_OK;
    bk::LnGradArgs a{dy, x, d_sum, weight, mean, rstd, T > 0 ? dx : nullptr, dweight, dbias, static_cast<float*>(work),
                     lddy, ldx, ldds, lddx, T, (int)d, 0, 0};
    if (dtype == BAKRON_F32)
        bk::launch_layernorm_grad<float>(a, stream);
    else if (dtype == BAKRON_F16)
        bk::launch_layernorm_grad<bk::f16_t>(a, stream);
    else
        bk::launch_layernorm_grad<bk::bf16_t>(a, stream);
    return bk::op_launched(who);
}
