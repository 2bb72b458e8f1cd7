// The softmax attention kernels' instances for one storage type and head dimension (SKA_T, SKA_D; the function's name: SKA_NAME).
#include "sinkhorn_attn_layer.h"
#include "ska_softmax_launch.h"

namespace {
template <typename T, int D> int launch(int what, int nw, const SmArgs &a, hipStream_t st)
{
    const dim3 grid((unsigned)((a.total + 7) / 8 * 8));
    switch (what) {
    case SM_FWD:
        if (nw == 1) hipLaunchKernelGGL((sm_rows_kernel<T, D, 1, false>), grid, dim3(64), 0, st, a);
        else hipLaunchKernelGGL((sm_rows_kernel<T, D, 4, false>), grid, dim3(256), 0, st, a);
        break;
    case SM_DQ:
        if (nw == 1) hipLaunchKernelGGL((sm_rows_kernel<T, D, 1, true>), grid, dim3(64), 0, st, a);
        else hipLaunchKernelGGL((sm_rows_kernel<T, D, 4, true>), grid, dim3(256), 0, st, a);
        break;
    default:
        if (nw == 1) hipLaunchKernelGGL((sm_keys_kernel<T, D, 1>), grid, dim3(64), 0, st, a);
        else hipLaunchKernelGGL((sm_keys_kernel<T, D, 4>), grid, dim3(256), 0, st, a);
    }
    if (hipGetLastError() != hipSuccess) return SKA_EHIP;
    if (a.parts > 1) {
        const int threads = (what == SM_DKV ? 2 * D : D) / 4;
        int slices = 1;   // as many as there are parts, or threads
        while (slices * 2 <= a.parts && slices * 2 * threads <= NTHREADS) slices *= 2;
        const long per = NTHREADS / threads / slices, rows = (long)a.B * a.Hk * (what == SM_DKV ? (long)a.Lk : (long)a.Lq * a.G);
        const dim3 jg((unsigned)((rows + per - 1) / per));
        if (what == SM_FWD) hipLaunchKernelGGL((sm_join_kernel<T, D, SM_JOIN_O>), jg, dim3(NTHREADS), 0, st, a, slices);
        else if (what == SM_DQ) hipLaunchKernelGGL((sm_join_kernel<T, D, SM_JOIN_DQ>), jg, dim3(NTHREADS), 0, st, a, slices);
        else hipLaunchKernelGGL((sm_join_kernel<T, D, SM_JOIN_DKV>), jg, dim3(NTHREADS), 0, st, a, slices);
        if (hipGetLastError() != hipSuccess) return SKA_EHIP;
    }
    return SKA_OK;
}
}  // namespace

SKA_DECLARE_SOFTMAX(SKA_NAME) { return launch<SKA_T, SKA_D>(what, nw, *static_cast<const SmArgs *>(args), st); }
