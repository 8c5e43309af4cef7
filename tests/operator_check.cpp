// CPU check of the host code of the operators around a quantised layer: the launches that
// calls at the limits of their sizes make, recorded instead of made.  The kernels are
// not run.  Prints one line a check; exit status = number of failing ones.
//
//   operator_check                    the checks
//   operator_check tile I T           edge of the tiles of a product of I x T outputs on 256 CUs
//   operator_check backward T D F     of the gradients: edge and parts for dx, edge and parts for dW
#include <cstdio>
#include <cstdlib>
#include <cstring>
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

int main(int argc, char** argv) {
    if (argc == 4 && std::strcmp(argv[1], "tile") == 0) {
        std::printf("%d\n", bk::pick_tile(std::atoll(argv[2]), std::atoll(argv[3]), 256, true));
        return 0;
    }
    if (argc == 5 && std::strcmp(argv[1], "backward") == 0) {
        const bk::BackwardPlan p =
            bk::backward_plan(std::atoll(argv[2]), std::atoll(argv[3]), std::atoll(argv[4]), true, true, true, 256);
        std::printf("%d %d %d %d\n", p.dx.tile, p.dx.parts, p.dw.tile, p.dw.parts);
        return 0;
    }
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
