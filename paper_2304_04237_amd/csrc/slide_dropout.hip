// Dropout whose mask is never stored: y = residual + keep(i) / (1 - p) * x, the mask drawn again from the element's number
// wherever it is needed (the backward is the same kernel on dout without a residual).
//
// One evaluation of the generator (7 rounds of two products of 32 x 32 bits, a quarter of the rate of other instructions) serves eight
// elements, 16 bytes of bf16; the kernel is bound by memory (5.9 TB/s on a training batch of stage 1, a large copy 4.9).
#include "slide_region.h"

namespace slide {
namespace region {

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));

// Eight elements in registers: loaded and stored whole, or one by one
template <typename T> struct Eight;
template <> struct Eight<bf16_bits> {
    u4 v;
    __device__ __forceinline__ void load(const bf16_bits* p) { v = *(const u4*)p; }
    __device__ __forceinline__ void store(bf16_bits* p) const { *(u4*)p = v; }
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(e & 1 ? v[e >> 1] & 0xffff0000u : v[e >> 1] << 16); }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{x[2 * i], x[2 * i + 1]}, bf2));
    }
};
template <> struct Eight<float> {
    f4 v[2];
    __device__ __forceinline__ void load(const float* p) { v[0] = *(const f4*)p; v[1] = ((const f4*)p)[1]; }
    __device__ __forceinline__ void store(float* p) const { *(f4*)p = v[0]; ((f4*)p)[1] = v[1]; }
    __device__ __forceinline__ float get(int e) const { return v[e >> 2][e & 3]; }
    __device__ __forceinline__ void set(const float (&x)[8])
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = x[e];
    }
};

__device__ __forceinline__ float kept(float x, float residual, const Words& w, int e, const Random& r)
{
    return half_word(w, e) >= r.threshold ? __builtin_fmaf(x, r.scale, residual) : residual;
}

// VEC: x, residual and y are 16-byte aligned; the last n % 8 elements go one by one
template <typename T, bool RESIDUAL, bool VEC>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, const T* residual, T* y, long long n, Random r)
{
    const long long g = (long long)blockIdx.x * 256 + threadIdx.x, i = 8 * g;
    if (i >= n) return;
    const bool whole = VEC && i + 8 <= n;
    Eight<T> a, b;
    if (whole) {
        a.load(x + i);
        if (RESIDUAL) b.load(residual + i);
    }
    const Words w = philox((uint32_t)g, (uint32_t)(g >> 32) | 0x80000000u, 0xffffffffu, r.call(), r.key0, r.key1);
    if (whole) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = kept(a.get(e), RESIDUAL ? b.get(e) : 0.0f, w, e, r);
        a.set(z);
        a.store(y + i);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < n) Elem<T>::store(y + i + e, kept(Elem<T>::load(x + i + e), RESIDUAL ? Elem<T>::load(residual + i + e) : 0.0f, w, e, r));
    }
}

template <typename T, bool RESIDUAL>
static hipError_t run(const T* x, const T* residual, T* y, long long n, const Random& r, hipStream_t st)
{
    const bool vec = (((uintptr_t)x | (uintptr_t)residual | (uintptr_t)y) & 15) == 0;
    // (eight elements a thread: 25.9 million bf16 elements with a residual in 25.5 us, without in 18.3; four times as many, loaded at once,
    // take 28.2 and 20.4)
    const unsigned blocks = (unsigned)((n + 2047) / 2048);
    if (vec) dropout_kernel<T, RESIDUAL, true><<<blocks, 256, 0, st>>>(x, residual, y, n, r);
    else dropout_kernel<T, RESIDUAL, false><<<blocks, 256, 0, st>>>(x, residual, y, n, r);
    return hipGetLastError();
}

hipError_t launch_dropout(const void* x, const void* residual, void* y, long long n, int dtype, const Random& r, hipStream_t st)
{
    if (dtype == 0) return residual ? run<float, true>((const float*)x, (const float*)residual, (float*)y, n, r, st)
                                    : run<float, false>((const float*)x, nullptr, (float*)y, n, r, st);
    return residual ? run<bf16_bits, true>((const bf16_bits*)x, (const bf16_bits*)residual, (bf16_bits*)y, n, r, st)
                    : run<bf16_bits, false>((const bf16_bits*)x, nullptr, (bf16_bits*)y, n, r, st);
}

}  // namespace region
}  // namespace slide
