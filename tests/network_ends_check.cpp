// CPU check of the host code of the operators at the ends of a network: the launches that calls
// make, recorded instead of made.  The kernels are not run.  Prints one line a check; exit
// status = number of failing ones.
//
//   network_ends_check                the checks
//   network_ends_check head T D V     kernel of the loss (few rows: units of 16 tokens, negative; else the tile's edge),
//                                     pieces of the gradients, edge and parts for dx, edge and parts for dW, columns of x
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <hip/hip_runtime.h>

namespace {
int launches = 0, fails = 0;
template <typename... A>
void record(dim3 grid, dim3 block, A&&...) {
    ++launches;
    // what one launch takes
    const double threads = (double)grid.x * block.x * ((double)grid.y * block.y) * grid.z * block.z;
    if (threads >= 4294967296.0 || grid.x == 0 || grid.y == 0 || grid.y > 65535 || block.x * block.y > 1024) {
        std::printf("a launch of %u x %u workgroups of %u x %u threads\n", grid.x, grid.y, block.x, block.y);
        ++fails;
    }
}
}  // namespace
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, shared, stream, ...) record(grid, block)

#include "layernorm.hip"
#define up256 up256_embedding
#include "embedding.hip"
#undef up256
#include "head.hip"

void bk::set_last_error(const char*) {}

static void* const P = reinterpret_cast<void*>(4096);
static float* const F = reinterpret_cast<float*>(4096);
static int64_t* const I = reinterpret_cast<int64_t*>(4096);

static void check(bakron_status st, bool taken, const char* what, int64_t a, int64_t b, int64_t c) {
    const bool ok = (st != BAKRON_EINVAL) == taken;   // (without a device launches fail after that)
    std::printf("%s %s %lld %lld %lld\n", ok ? "ok" : "FAIL", what, (long long)a, (long long)b, (long long)c);
    if (!ok) ++fails;
}

int main(int argc, char** argv) {
    if (argc == 5 && std::strcmp(argv[1], "head") == 0) {
        const int64_t T = std::atoll(argv[2]), d = std::atoll(argv[3]), V = std::atoll(argv[4]);
        const bk::HeadBackward b = bk::head_backward(T, d, V, true, true, true, 256);
        std::printf("%d %d %d %d %d %d %lld\n", bk::head_few_rows(T, V, d) ? -bk::head_units(T, V, d) : bk::head_edge(T, V, d),
                    (int)((V + b.vc - 1) / b.vc), b.dx.tile, b.dx.parts, b.dw.tile, b.dw.parts, (long long)b.tp);
        return 0;
    }
    const int64_t wide = 1 << 17, all = 1 << 20;
    size_t size = ~(size_t)0;
    for (int64_t T : {(int64_t)1, (int64_t)16, (int64_t)32, (int64_t)33, (int64_t)64, (int64_t)65, (int64_t)511, (int64_t)8191,
                      (int64_t)32000})
        for (int64_t d : {(int64_t)1, (int64_t)7, (int64_t)8, (int64_t)131, wide - 1, wide})
            for (int64_t V : {(int64_t)1, (int64_t)65, (int64_t)8192, all - 1, all}) {
                check(bakron_head_logprobs(P, d, T, d, P, d, V, BAKRON_BF16, I, F, F, F, P, &size, nullptr), true, "head", T, d, V);
                check(bakron_head_logprobs_backward(P, d, T, d, P, d, V, BAKRON_F16, I, F, F, F, F, P, d, P, d, P, &size, nullptr),
                      true, "head backward", T, d, V);
            }
    check(bakron_head_logprobs(P, 64, 1 << 25, 64, P, 64, all, BAKRON_BF16, I, F, F, F, P, &size, nullptr), false, "head", 1 << 25, 64, all);
    check(bakron_head_logprobs(P, 64, bk::OP_T_MAX, 64, P, 64, 1, BAKRON_BF16, I, F, F, F, P, &size, nullptr), false, "head", -1, 64, 1);
    check(bakron_head_logprobs(P, 8, ((int64_t)1 << 27) + 1, 8, P, 8, 64, BAKRON_BF16, I, F, F, F, P, &size, nullptr), false, "head", 500000000, 8, 64);
    for (int64_t T : {(int64_t)1 << 27, ((int64_t)1 << 26) + 5}) {
        check(bakron_head_logprobs(P, 8, T, 8, P, 8, 64, BAKRON_BF16, I, F, F, F, P, &size, nullptr), true, "head", T, 8, 64);
        check(bakron_head_logprobs_backward(P, 8, T, 8, P, 8, 64, BAKRON_BF16, I, F, F, F, F, P, 8, P, 8, P, &size, nullptr), true,
              "head backward", T, 8, 64);
    }
    for (int dtype : {BAKRON_F32, BAKRON_F16, BAKRON_BF16}) {
        for (int64_t d : {(int64_t)1, (int64_t)64, (int64_t)1000, (int64_t)16384, (int64_t)16385, (int64_t)65536})
            for (int64_t T : {(int64_t)1, (int64_t)1023, (int64_t)100000, (int64_t)2000000}) {
                check(bakron_layernorm(P, d, P, d, dtype, T, d, F, F, 1e-5f, 1, P, d, P, d, F, F, nullptr), true, "norm", dtype, T, d);
                check(bakron_layernorm_backward(P, d, P, d, dtype, T, d, F, F, F, P, d, P, d, F, F, P, &size, nullptr), true,
                      "norm backward", dtype, T, d);
            }
        check(bakron_layernorm(P, 65536, P, 65536, dtype, bk::OP_T_MAX, 65536, F, F, 1e-5f, 1, P, 65536, P, 65536, F, F, nullptr), false,
              "norm", dtype, -1, 65536);
        for (int64_t d : {(int64_t)1, (int64_t)8, (int64_t)1000, (int64_t)65536})
            for (int64_t T : {(int64_t)1, (int64_t)16385, (int64_t)500000, all})
                for (int64_t V : {(int64_t)1, all}) {
                    const int64_t len = 256 * bk::EMBED_NV * (dtype == BAKRON_F32 ? 4 : 8);
                    check(bakron_embedding(I, T, P, d, dtype, V, d, 1.0f, P, d, nullptr), T * ((d + len - 1) / len) <= 1 << 23, "embedding",
                          T, d, V);
                    check(bakron_embedding_backward(P, d, I, T, dtype, V, d, 1.0f, P, d, P, d, P, &size, nullptr), true,
                          "embedding backward", T, d, V);
                }
    }
    std::printf("launches %d fails %d\n", launches, fails);
    return fails;
}
