// C ABI of dropout from a counter.  See include/lsr_dropout.h for its contract.
#include "lsr_dropout.h"

#include <hip/hip_runtime.h>
#include <math.h>

#include "dropout.hpp"
#include "host_checks.hpp"

extern "C" int lsr_dropout(int64_t n, int32_t dtype, const void* X, void* Y, double p, uint64_t seed, uint64_t offset, const uint64_t* state,
                           lsr_stream_t stream) {
    using namespace lsr;
    if (dtype != LSR_F32 && dtype != LSR_BF16) return LSR_ERR_DTYPE;
    if (n < 1 || n >= (int64_t(1) << 40) || !(p >= 0.0 && p <= 1.0)) return LSR_ERR_SHAPE;
    if (!X || !Y) return LSR_ERR_NULL;
    const uintptr_t off = dtype == LSR_F32 ? 3 : 1;
    if ((reinterpret_cast<uintptr_t>(X) & off) || (reinterpret_cast<uintptr_t>(Y) & off) || (reinterpret_cast<uintptr_t>(state) & 7)) return LSR_ERR_ALIGN;
    int n_cus = 0;
    const int rc = check_device(&n_cus);
    if (rc != LSR_OK) return rc;
    DropoutParams q = {};
    q.X = X; q.Y = Y; q.n = n; q.seed = seed; q.offset = offset; q.state = state;
    q.least = (uint32_t)nearbyint(p * 65536.0);
    q.scale = q.least < 65536 ? (float)(65536.0 / (65536 - q.least)) : 0.f;
    const int64_t blocks = (n + 8 * DROP_THREADS - 1) / (8 * DROP_THREADS), most = int64_t(1) << 23;
    const unsigned grid = (unsigned)(blocks < most ? blocks : most);
    if (dtype == LSR_F32) dropout_kernel<float><<<grid, DROP_THREADS, 0, stream>>>(q);
    else dropout_kernel<uint16_t><<<grid, DROP_THREADS, 0, stream>>>(q);
    return launch_status();
}
