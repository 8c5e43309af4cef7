// CPU check of the host code of the operators around a quantised layer: the launches that
// calls at the limits of their sizes make, recorded instead of made.  The kernels are
// not run.  Prints one line a check; exit status = number of failing ones.
#include <cstdio>
#include <hip/hip_runtime.h>

namespace {
struct Launch {
    dim3 grid, block;
};
Launch last;
int launches = 0, fails = 0;
template <typename... A>
void record(dim3 grid, dim3 block, A&&...) {
    last = Launch{grid, block};
    ++launches;
    // what one launch takes
    const double threads = (double)grid.x * block.x * ((double)grid.y * block.y) * grid.z * block.z;
    if (threads >= 4294967296.0 || grid.x == 0 || grid.y > 65535 || (double)grid.x * block.x >= 4294967296.0) {
        std::printf("a launch of %u x %u workgroups of %u x %u threads\n", grid.x, grid.y, block.x, block.y);
        ++fails;
    }
}
void check(bool ok, const char* what) {
    std::printf("%s %s\n", ok ? "ok" : "FAIL", what);
    if (!ok) ++fails;
}
}  // namespace
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, shared, stream, ...) record(grid, block)

#define FEW_ROWS FEW_ROWS_LINEAR   // (each source has limits of its own under these names)
#define FEW_TILES FEW_TILES_LINEAR
#include "norm.hip"
#include "linear.hip"
#undef FEW_ROWS
#undef FEW_TILES
#include "logprob.hip"
#include "mlp.hip"

void bk::set_last_error(const char*) {}

static void* const P = reinterpret_cast<void*>(4096);

int main() {
    const int before = fails;
    for (int width : {4, 8}) bakron_pack_codes(static_cast<int8_t*>(P), 1 << 20, 1 << 17, width, P, nullptr);
    size_t size = ~(size_t)0;
    // odd rows: both weights and x are copied
    for (int64_t T : {(int64_t)1000, (int64_t)50000})
        bakron_gated_mlp(P, 131071, T, 131071, P, P, 131071, 1 << 17, BAKRON_BF16, BAKRON_ACT_SILU, P, 1 << 17, nullptr,
                         nullptr, P, &size, nullptr);
    check(fails == before && launches >= 6, "launches at the largest sizes");
    std::printf("fails %d\n", fails);
    return fails;
}
