// Region selection: which regions of keys the rows of a group attend.
//
//   score(i, j) = (sum of q over the group's valid rows) . (sum of k over region j's valid places) / (number of those places)
//
// The T highest, ties to the lowest index.  Sums and products are held in 64 bits: a selection is a decision, and in 32 bits the
// order of two near scores would hang on the order of a sum.
#include "slide_region.h"

namespace slide {
namespace region {

// one block per (region, kv head, image): the sum over the region's places (and, for queries, the g heads) of each channel
template <typename T>
__global__ __launch_bounds__(256) void pool_kernel(const T* x, Strides s, Map m, int kv, int g, int d, int mean, double* out, int* count)
{
    const int r = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    int vh, vw;
    m.limits(b, vh, vw);
    const long long at = ((long long)b * kv + h) * m.regions + r;
    int n = 0;
    for (int p = 0; p < m.places; ++p) n += m.pixel(r, p, vh, vw) >= 0;
    for (int c = threadIdx.x; c < d; c += blockDim.x) {
        double sum = 0.0;
        for (int p = 0; p < m.places; ++p) {
            const int px = m.pixel(r, p, vh, vw);
            if (px < 0) continue;
            for (int e = 0; e < g; ++e) sum += (double)Elem<T>::load(x + b * s.image + px * s.pixel + (h * g + e) * d + c);
        }
        out[at * d + c] = mean && n ? sum / n : sum;
    }
    if (threadIdx.x == 0) count[at] = n;
}

// one block per (group, kv head, image)
__global__ __launch_bounds__(256) void select_kernel(const double* qp, const int* qn, const double* kp, const int* kn, int kv, int G,
                                                     int J, int d, int T, int* index)
{
    extern __shared__ double score[];           // [J], then the four waves' best
    __shared__ double best_s[4];
    __shared__ int best_j[4], chosen;
    const int i = blockIdx.x;
    const long long bh = (long long)blockIdx.z * kv + blockIdx.y;
    const long long group = bh * G + i;
    int* list = index + group * T;
    const bool any = qn[group] > 0;
    const double none = -INFINITY;
    for (int j = threadIdx.x; j < J; j += 256) {
        double s = none;
        if (any && kn[bh * J + j] > 0) {
            s = 0.0;
            for (int c = 0; c < d; ++c) s += qp[group * d + c] * kp[(bh * J + j) * d + c];
            if (!(s > -1.7976931348623157e308)) s = -1.7976931348623157e308;       // -inf and NaN: the lowest that can be chosen
        }
        score[j] = s;
    }
    __syncthreads();
    for (int t = 0; t < T; ++t) {
        double s = none;
        int at = J;
        for (int j = threadIdx.x; j < J; j += 256)
            if (score[j] > s) { s = score[j]; at = j; }
        for (int w = 32; w > 0; w >>= 1) {
            const double os = __shfl_xor(s, w);
            const int oj = __shfl_xor(at, w);
            if (os > s || (os == s && oj < at)) { s = os; at = oj; }
        }
        if ((threadIdx.x & 63) == 0) { best_s[threadIdx.x >> 6] = s; best_j[threadIdx.x >> 6] = at; }
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < 4; ++w)
                if (best_s[w] > best_s[0] || (best_s[w] == best_s[0] && best_j[w] < best_j[0])) { best_s[0] = best_s[w]; best_j[0] = best_j[w]; }
            chosen = best_s[0] > none ? best_j[0] : -1;
            if (chosen >= 0) score[chosen] = none;
            list[t] = chosen;
        }
        __syncthreads();
        if (chosen < 0) {
            for (int u = t + threadIdx.x; u < T; u += 256) list[u] = -1;
            break;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {                     // ascending
        int n = 0;
        while (n < T && list[n] >= 0) ++n;
        for (int u = 1; u < n; ++u) {
            const int x = list[u];
            int v = u - 1;
            for (; v >= 0 && list[v] > x; --v) list[v + 1] = list[v];
            list[v + 1] = x;
        }
    }
}

size_t select_workspace_bytes(const Args& a)
{
    const size_t n = (size_t)a.B * a.kv * (a.qm.regions + a.km.regions);
    return n * a.d * sizeof(double) + n * sizeof(int);
}

template <typename T>
static hipError_t select_t(const Args& a, int* index, void* workspace, hipStream_t st)
{
    const size_t nq = (size_t)a.B * a.kv * a.qm.regions, nk = (size_t)a.B * a.kv * a.km.regions;
    double* qp = (double*)workspace;
    double* kp = qp + nq * a.d;
    int* qn = (int*)(kp + nk * a.d);
    int* kn = qn + nq;
    pool_kernel<T><<<dim3(a.qm.regions, a.kv, a.B), 256, 0, st>>>((const T*)a.q, a.qs, a.qm, a.kv, a.g, a.d, 0, qp, qn);
    pool_kernel<T><<<dim3(a.km.regions, a.kv, a.B), 256, 0, st>>>((const T*)a.k, a.ks, a.km, a.kv, 1, a.d, 1, kp, kn);
    static LdsOptIn lds;
    hipError_t e = lds.ensure({(const void*)select_kernel}, 16384 * 8);
    if (e != hipSuccess) return e;
    select_kernel<<<dim3(a.qm.regions, a.kv, a.B), 256, (size_t)a.km.regions * 8, st>>>(qp, qn, kp, kn, a.kv, a.qm.regions, a.km.regions,
                                                                                  a.d, a.T, index);
    return hipGetLastError();
}

hipError_t launch_select(const Args& a, int* index, void* workspace, hipStream_t st)
{
    return a.dtype == 0 ? select_t<float>(a, index, workspace, st) : select_t<bf16_bits>(a, index, workspace, st);
}

}  // namespace region
}  // namespace slide
