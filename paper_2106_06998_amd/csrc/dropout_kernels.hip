// Dropout without a stored mask: y = kept x / (1 - p), dx = kept dy / (1 - p), the mask drawn from the seed in both (drop.h).
// One 16-byte vector a lane; bound by HBM (each value read and written once).
#include "drop.h"
#include "launch.h"
#include "norm_core.h"

namespace xc {

namespace {

template <int DT>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const void *x, void *y, long long n, DropArgs d)   // y may be x
{
    typedef typename NormElem<DT>::t elem_t;
    constexpr int V = NormElem<DT>::V;
    const uint64_t key = drop_key(d);
    for (long long e = ((long long)blockIdx.x * kThreads + threadIdx.x) * V; e < n; e += (long long)gridDim.x * kThreads * V) {
        const Part p{0, 0, (int)min((long long)V, n - e)};
        float t[V];
        unpack<DT>(load_part<DT>(static_cast<const elem_t *>(x) + e, p), t);
        drop_values<V>(d, key, (uint64_t)e, true, t);
        store_part<DT>(static_cast<elem_t *>(y) + e, pack<DT>(t), p);
    }
}

}  // namespace

void host_dropout_mask(const xconv_drop *d, long long first, long long n, uint8_t *mask)
{
    const uint64_t key = drop_key(d->seed, 0);
    for (long long i = 0; i < n; ++i) {
        const uint64_t e = (uint64_t)(first + i);
        mask[i] = (uint8_t)(((stream_word(key, e >> 2) >> (16 * (e & 3))) & 0xffffu) >= (uint64_t)d->drop_q16);
    }
}

hipError_t launch_dropout(int dtype, const void *X, void *Y, long long n, const xconv_drop *drop, hipStream_t st)
{
    const int V = dtype == XCONV_F32 ? 4 : 8;
    const dim3 grid((unsigned)std::min<long long>(((n + V - 1) / V + kThreads - 1) / kThreads, 1 << 23));
    const DropArgs d = drop_args(drop);
    if (dtype == XCONV_F32) hipLaunchKernelGGL(dropout_kernel<XCONV_F32>, grid, dim3(kThreads), 0, st, X, Y, n, d);
    else if (dtype == XCONV_BF16) hipLaunchKernelGGL(dropout_kernel<XCONV_BF16>, grid, dim3(kThreads), 0, st, X, Y, n, d);
    else hipLaunchKernelGGL(dropout_kernel<XCONV_F16>, grid, dim3(kThreads), 0, st, X, Y, n, d);
    return hipGetLastError();
}

}  // namespace xc
