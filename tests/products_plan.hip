// The products' plan, as the library makes it, for tests on the host.
#include "dense.hpp"

extern "C" void products_plan(int64_t M, int64_t N, int64_t K, int32_t P, int64_t matrices, int32_t half, uint64_t parts_most, double elsewhere, int32_t* out) {
    const no::DensePlan p = no::dense_plan(M, N, K, P, matrices, half != 0, parts_most, elsewhere);
    out[0] = p.kind;
    out[1] = p.splits;
}
