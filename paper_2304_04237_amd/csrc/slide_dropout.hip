// Dropout whose mask is never stored: y = residual + keep(i) / (1 - p) * x, the mask drawn again from the element's number
// wherever it is needed (the backward is the same kernel on dout without a residual).
#include "slide_region.h"

namespace slide {
namespace region {

template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, const T* residual, T* y, long long n, Random r)
{
    const uint32_t call = r.call();
    for (long long g = (long long)blockIdx.x * 256 + threadIdx.x; 8 * g < n; g += (long long)gridDim.x * 256) {
        const Words w = philox((uint32_t)g, (uint32_t)(g >> 32) | 0x80000000u, 0xffffffffu, call, r.key0, r.key1);
        for (int e = 0; e < 8 && 8 * g + e < n; ++e) {
            const long long i = 8 * g + e;
            const float kept = half_word(w, e) >= r.threshold ? Elem<T>::load(x + i) * r.scale : 0.0f;
            Elem<T>::store(y + i, residual ? kept + Elem<T>::load(residual + i) : kept);
        }
    }
}

hipError_t launch_dropout(const void* x, const void* residual, void* y, long long n, int dtype, const Random& r, hipStream_t st)
{
    const int blocks = (int)std::min<long long>((n + 2047) / 2048, 16384);
    if (dtype == 0) dropout_kernel<float><<<blocks, 256, 0, st>>>((const float*)x, (const float*)residual, (float*)y, n, r);
    else dropout_kernel<bf16_bits><<<blocks, 256, 0, st>>>((const bf16_bits*)x, (const bf16_bits*)residual, (bf16_bits*)y, n, r);
    return hipGetLastError();
}

}  // namespace region
}  // namespace slide
