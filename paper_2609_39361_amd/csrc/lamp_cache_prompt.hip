// lamp_cache_prompt.hip -- the kernels of the attention over the 8-bit paged cache
// that hold the form for many rows (lamp_cache_many.h).
#include <hip/hip_runtime.h>

#include "lamp_cache_many.h"

namespace lamp {
namespace {

template <int D, int KT, bool WIDE>
__global__ __launch_bounds__(THREADS, 2) void cache_prompt_kernel(CacheAttnParams p)
{
    __shared__ PromptShared<D, KT> sh;
    cache_prompt<D, KT, WIDE>(p, (int)blockIdx.x, sh);
}

// Both forms side by side: a batch of chunks and single tokens.
template <int D, int KT, int KF, bool WIDE>
__global__ __launch_bounds__(THREADS, 2) void cache_mixed_kernel(CacheAttnParams p)
{
    constexpr size_t A = sizeof(PromptShared<D, KT>), B = sizeof(FewShared<D, WAVES>);
    __shared__ __attribute__((aligned(16))) char sh[A > B ? A : B];
    const int x = (int)blockIdx.x;
    if (x < p.units[1]) cache_prompt<D, KT, WIDE>(p, x, *reinterpret_cast<PromptShared<D, KT> *>(sh));
    else cache_few<D, KF, WAVES>(p, x - p.units[1], *reinterpret_cast<FewShared<D, WAVES> *>(sh));
}

template <int D, int KT, int KF, bool WIDE>
hipError_t launch_prompt(const CacheAttnParams &p, hipStream_t s)
{
    if (p.units[0] && !p.apart) cache_mixed_kernel<D, KT, KF, WIDE><<<dim3((unsigned)(p.units[0] + p.units[1])), THREADS, 0, s>>>(p);
    else cache_prompt_kernel<D, KT, WIDE><<<dim3((unsigned)p.units[1]), THREADS, 0, s>>>(p);
    return hipGetLastError();
}

template <int D, int KT, int KF>
hipError_t launch_prompt_of(const CacheAttnParams &p, hipStream_t s)
{
    return 1 << p.b.page_shift >= KT ? launch_prompt<D, KT, KF, true>(p, s) : launch_prompt<D, KT, KF, false>(p, s);
}

} // namespace

hipError_t launch_cache_prompt(int D, const CacheAttnParams &p, hipStream_t s)
{
    switch (D) {
    case 64: return launch_prompt_of<64, 64, 64>(p, s);
    case 128: return launch_prompt_of<128, 64, 64>(p, s);
    default: return launch_prompt_of<256, 32, 32>(p, s);
    }
}

} // namespace lamp
