// The attention kernels' instances for one storage type, query type and head dimension (SKA_S, SKA_T, SKA_D; the function's name: SKA_NAME).
#include <algorithm>

#include "sinkhorn_attn_cache.h"
#include "ska_cache_launch.h"
#include "ska_cache_plan.h"

namespace {
static_assert(CaJoin::THREADS == NTHREADS, "the join's workgroups");
template <typename S, typename T, int D> int launch(int nq, bool both, const CaArgs &a, hipStream_t st)
{
    constexpr int MOST = ca_most(sizeof(S) == 4, D);
    const dim3 grid((unsigned)(a.side[0].wgs + a.side[1].wgs));
    if (both) hipLaunchKernelGGL((ca_attn_kernel<S, T, D, 1, true>), grid, dim3(64 * CA_WAVES), 0, st, a);
    else if (nq == 2) hipLaunchKernelGGL((ca_attn_kernel<S, T, D, 2, false>), grid, dim3(64 * CA_WAVES), 0, st, a);
    else hipLaunchKernelGGL((ca_attn_kernel<S, T, D, MOST, false>), grid, dim3(64 * CA_WAVES), 0, st, a);
    if (hipGetLastError() != hipSuccess) return SKA_EHIP;
    if (a.parts > 1) {
        const CaJoin join(a.parts, D);
        const long rows = (long)a.B * a.Hk * a.Lq * a.G;
        for (long first = 0; first < rows; first += join.most()) {
            const long n = std::min(rows - first, join.most());
            hipLaunchKernelGGL((ca_join_kernel<T, D>), dim3((unsigned)((n + join.per - 1) / join.per)), dim3(NTHREADS), 0, st, a, first, join.slices);
            if (hipGetLastError() != hipSuccess) return SKA_EHIP;
        }
    }
    return SKA_OK;
}
}  // namespace

SKA_DECLARE_CACHE(SKA_NAME) { return launch<SKA_S, SKA_T, SKA_D>(nq, both, *static_cast<const CaArgs *>(args), st); }
