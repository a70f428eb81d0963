// Region attention, forward and backward: one wave per row (or per key), float32 vector arithmetic.
//
//   S = scale q.k;  lse = log sum exp S;  P = exp(S - lse);  out = sum keep / (1 - p) P v
//   D = dout.out;  dS = P (keep / (1 - p) dout.v - D);  dq = scale sum dS k;  dk = scale sum dS q;  dv = sum keep / (1 - p) P dout
//
// A lane holds channels lane and lane + 64; the running maximum and sum of the softmax are those of one pass over the keys.
#include "slide_region.h"

namespace slide {
namespace region {

__device__ __forceinline__ float wave_sum(float x)
{
    for (int w = 32; w > 0; w >>= 1) x += __shfl_xor(x, w);
    return x;
}

// the factor of one attention weight
__device__ __forceinline__ float keep_factor(const Args& a, uint32_t call, int bh, int i, int r, int j, int n)
{
    if (a.rnd.threshold == 0) return 1.0f;
    const Words w = philox((uint32_t)j * a.quads + (n >> 2), (uint32_t)i * a.pairs + (r >> 1), (uint32_t)bh, call, a.rnd.key0, a.rnd.key1);
    return half_word(w, 4 * (r & 1) + (n & 3)) >= a.rnd.threshold ? a.rnd.scale : 0.0f;
}

template <typename T>
__device__ __forceinline__ void load_row(const void* x, long long at, int d, int lane, float (&v)[2])
{
    for (int u = 0; u < 2; ++u) v[u] = lane + 64 * u < d ? Elem<T>::load((const T*)x + at + lane + 64 * u) : 0.0f;
}

template <typename T>
__device__ __forceinline__ void store_row(void* x, long long at, int d, int lane, const float (&v)[2])
{
    for (int u = 0; u < 2; ++u)
        if (lane + 64 * u < d) Elem<T>::store((T*)x + at + lane + 64 * u, v[u]);
}

// block: one wave; grid (rows of a group, groups, B * kv).  BWD: dq and D instead of out and lse
template <typename T, bool BWD>
__global__ __launch_bounds__(64) void row_kernel(Args a, const void* dout, void* out, float* lse, void* dq, float* D)
{
    const int r = blockIdx.x, i = blockIdx.y, bh = blockIdx.z, b = bh / a.kv, m = bh - b * a.kv, lane = threadIdx.x;
    const int place = r / a.g, head = m * a.g + r - place * a.g;
    int vh, vw;
    const int px = a.qm.pixel(i, place, a.qm.H, a.qm.W);
    if (px < 0) return;
    a.qm.limits(b, vh, vw);
    const bool valid = a.qm.pixel(i, place, vh, vw) >= 0;
    const long long n_pix = (long long)a.qm.H * a.qm.W;
    const long long o_at = ((long long)b * n_pix + px) * a.heads * a.d + head * a.d;
    const long long l_at = ((long long)b * a.heads + head) * n_pix + px;
    const uint32_t call = a.rnd.threshold ? a.rnd.call() : 0;
    float q[2] = {}, acc[2] = {}, g[2] = {}, top = -INFINITY, sum = 0.0f, delta = 0.0f, l = 0.0f;
    if (valid) {
        load_row<T>(a.q, b * a.qs.image + px * a.qs.pixel + head * a.d, a.d, lane, q);
        if (BWD) {
            float o[2];
            load_row<T>(dout, o_at, a.d, lane, g);
            load_row<T>(out, o_at, a.d, lane, o);
            delta = wave_sum(g[0] * o[0] + g[1] * o[1]);
            l = lse[l_at];
        }
        int kh, kw;
        a.km.limits(b, kh, kw);
        for (int t = 0; t < a.T; ++t) {
            const int j = a.index[((long long)bh * a.qm.regions + i) * a.T + t];
            if (j < 0 || j >= a.km.regions) continue;
            for (int n = 0; n < a.km.places; ++n) {
                const int kx = a.km.pixel(j, n, kh, kw);
                if (kx < 0) continue;
                float k[2], v[2];
                load_row<T>(a.k, b * a.ks.image + kx * a.ks.pixel + m * a.d, a.d, lane, k);
                load_row<T>(a.v, b * a.vs.image + kx * a.vs.pixel + m * a.d, a.d, lane, v);
                const float s = wave_sum(q[0] * k[0] + q[1] * k[1]) * a.scale;
                const float keep = keep_factor(a, call, bh, i, r, j, n);
                if (BWD) {
                    const float ds = expf(s - l) * (keep * wave_sum(g[0] * v[0] + g[1] * v[1]) - delta) * a.scale;
                    for (int u = 0; u < 2; ++u) acc[u] += ds * k[u];
                } else {
                    const float next = fmaxf(top, s), back = top == -INFINITY ? 0.0f : expf(top - next);
                    const float p = s == -INFINITY ? 0.0f : expf(s - next);
                    top = next;
                    sum = sum * back + p;
                    for (int u = 0; u < 2; ++u) acc[u] = acc[u] * back + keep * p * v[u];
                }
            }
        }
    }
    if (BWD) {
        store_row<T>(dq, o_at, a.d, lane, acc);
        if (lane == 0) D[l_at] = delta;
    } else {
        const float inv = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);
        for (int u = 0; u < 2; ++u) acc[u] *= inv;
        store_row<T>(out, o_at, a.d, lane, acc);
        if (lane == 0 && lse) lse[l_at] = sum == 0.0f ? -INFINITY : top + logf(sum);
    }
}

// block: one wave per key; grid (places of a key region, regions, B * kv)
template <typename T>
__global__ __launch_bounds__(64) void key_kernel(Args a, const void* dout, const float* lse, const float* D, void* dk, void* dv)
{
    const int n = blockIdx.x, j = blockIdx.y, bh = blockIdx.z, b = bh / a.kv, m = bh - b * a.kv, lane = threadIdx.x;
    const int kx = a.km.pixel(j, n, a.km.H, a.km.W);
    if (kx < 0) return;
    int kh, kw, vh, vw;
    a.km.limits(b, kh, kw);
    a.qm.limits(b, vh, vw);
    const long long n_pix = (long long)a.qm.H * a.qm.W;
    const long long k_at = ((long long)b * a.km.H * a.km.W + kx) * a.kv * a.d + m * a.d;
    const uint32_t call = a.rnd.threshold ? a.rnd.call() : 0;
    float k[2], v[2], gk[2] = {}, gv[2] = {};
    if (a.km.pixel(j, n, kh, kw) >= 0) {
        load_row<T>(a.k, b * a.ks.image + kx * a.ks.pixel + m * a.d, a.d, lane, k);
        load_row<T>(a.v, b * a.vs.image + kx * a.vs.pixel + m * a.d, a.d, lane, v);
        for (long long e = 0; e < (long long)a.qm.regions * a.T; ++e) {
            if (a.index[(long long)bh * a.qm.regions * a.T + e] != j) continue;
            const int i = (int)(e / a.T);
            for (int r = 0; r < a.R; ++r) {
                const int place = r / a.g, head = m * a.g + r - place * a.g;
                const int px = a.qm.pixel(i, place, vh, vw);
                if (px < 0) continue;
                float q[2], g[2];
                load_row<T>(a.q, b * a.qs.image + px * a.qs.pixel + head * a.d, a.d, lane, q);
                load_row<T>(dout, ((long long)b * n_pix + px) * a.heads * a.d + head * a.d, a.d, lane, g);
                const long long l_at = ((long long)b * a.heads + head) * n_pix + px;
                const float p = expf(wave_sum(q[0] * k[0] + q[1] * k[1]) * a.scale - lse[l_at]);
                const float keep = keep_factor(a, call, bh, i, r, j, n);
                const float ds = p * (keep * wave_sum(g[0] * v[0] + g[1] * v[1]) - D[l_at]) * a.scale;
                for (int u = 0; u < 2; ++u) { gk[u] += ds * q[u]; gv[u] += keep * p * g[u]; }
            }
        }
    }
    store_row<T>(dk, k_at, a.d, lane, gk);
    store_row<T>(dv, k_at, a.d, lane, gv);
}

size_t bwd_workspace_bytes(const Args& a) { return (size_t)a.B * a.heads * a.qm.H * a.qm.W * sizeof(float); }

hipError_t launch_bwd(const Args& a, const void* dout, const void* out, const float* lse, void* dq, void* dk, void* dv,
                      void* workspace, hipStream_t st)
{
    const dim3 rows(a.R, a.qm.regions, a.B * a.kv), keys(a.km.places, a.km.regions, a.B * a.kv);
    float* D = (float*)workspace;
    if (a.dtype == 0) {
        row_kernel<float, true><<<rows, 64, 0, st>>>(a, dout, const_cast<void*>(out), const_cast<float*>(lse), dq, D);
        key_kernel<float><<<keys, 64, 0, st>>>(a, dout, lse, D, dk, dv);
    } else {
        row_kernel<bf16_bits, true><<<rows, 64, 0, st>>>(a, dout, const_cast<void*>(out), const_cast<float*>(lse), dq, D);
        key_kernel<bf16_bits><<<keys, 64, 0, st>>>(a, dout, lse, D, dk, dv);
    }
    return hipGetLastError();
}

}  // namespace region
}  // namespace slide
