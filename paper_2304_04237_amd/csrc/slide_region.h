// Shared by the kernels of region attention (slide_region_*.hip) and of dropout (slide_dropout.hip).
//
// A map is cut into regions; group i is a region of queries together with the g = heads / kv_heads query heads that share one
// key head, R = (places of the region) * g rows, row r = place * g + head.  Every row of a group attends the keys of the same T
// regions, so a group is a dense [R] x [T * places] problem, with rows and keys that may lie outside the map or outside the
// image's own size.
#pragma once
#include "slide_internal.h"
#include "slide_device.h"

namespace slide {
namespace region {

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;

// Division of numbers below 2^31 by a number that the host knows: one product.  (n m) >> (31 + s) with m = floor(2^(31 + s) / x) + 1,
// s = ceil(log2 x), is exact for n < 2^31: m x exceeds 2^(31 + s) by at most x <= 2^s.
struct Div {
    uint32_t x, m, s;
    __host__ static Div by(uint32_t x)
    {
        uint32_t s = 0;
        while ((1ull << s) < x) ++s;
        return Div{x, (uint32_t)((1ull << (31 + s)) / x + 1), s};
    }
    __device__ __forceinline__ int of(int n) const { return (int)(__umulhi((uint32_t)n << 1, m) >> s); }
};

// A map of pixels cut into regions: what the kernels need to find a pixel.
struct Map {
    int H, W;               // pixels
    int h, w;               // a region, no larger than the map
    int across, regions;    // regions side by side, and in all
    int places;             // h * w
    const int* size;        // [B][2] valid height and width of each image, or null
    Div by_across, by_w;
    // valid height and width of image b, within the map
    __device__ __forceinline__ void limits(int b, int& vh, int& vw) const
    {
        vh = size ? min(max(size[2 * b], 0), H) : H;
        vw = size ? min(max(size[2 * b + 1], 0), W) : W;
    }
    // pixel at `place` of region `r`, or -1 outside (vh, vw)
    __device__ __forceinline__ int pixel(int r, int place, int vh, int vw) const
    {
        const int ry = by_across.of(r), rx = r - ry * across;
        const int py = by_w.of(place), px = place - py * w;
        const int y = ry * h + py, x = rx * w + px;
        return y < vh && x < vw ? y * W + x : -1;
    }
};

struct Strides { long long pixel, image; };     // in elements

// The generator: Philox-4x32 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) with 7 rounds, the
// fewest that the paper reports to pass its whole battery of tests; a round is two 32 x 32 -> 64 bit products.  The seed is the
// key; the counter says which element and which call.  Elements take 16 bits each: eight per evaluation.
struct Random {
    uint32_t key0, key1;
    uint32_t offset;                    // the number of the call ...
    const long long* offset_device;     // ... plus what this holds when the kernel runs, if it is not null
    uint32_t threshold;                 // an element is dropped where its 16 bits are below this; 0: nothing is
    float scale;                        // 65536 / (65536 - threshold)
    __device__ __forceinline__ uint32_t call() const { return offset + (offset_device ? (uint32_t)*offset_device : 0u); }
};

struct Words { uint32_t w[4]; };

__device__ __forceinline__ Words philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1)
{
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        const uint32_t n0 = (uint32_t)(b >> 32) ^ c1 ^ k0, n2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)b; c3 = (uint32_t)a; c0 = n0; c2 = n2;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    return Words{{c0, c1, c2, c3}};
}

// half word e (0..7) of the four words
__device__ __forceinline__ uint32_t half_word(const Words& w, int e) { return (w.w[e >> 1] >> (16 * (e & 1))) & 0xffffu; }

struct Args {
    int B, heads, kv, g, d, T, dtype;
    int R;                              // rows of a group
    int quads, pairs;                   // ceil(key places / 4), ceil(R / 2): the dropout counter counts patches of 4 keys and 2 rows
    Div by_g, by_slots;                 // slots: 4 * quads, what a listed region takes in a group's row of keys
    Map qm, km;
    Strides qs, ks, vs;
    Strides os;                         // of dout and out (backward)
    int hd, dl;                         // q, k, v, dout and out as they are loaded: elements between heads, channels (zeros behind d)
    float scale;
    Random rnd;
    const void* q; const void* k; const void* v;
    const int* index;                   // [B][kv][qm.regions][T]
};

// A launch has fewer than 2^32 threads (the runtime refuses more): launch(blocks, first), for as many blocks at a time as that allows.
template <typename F> inline hipError_t in_launches(long long blocks, int threads, F launch)
{
    const long long most = ((1ll << 32) - 1) / threads;
    for (long long first = 0; first < blocks; first += most) {
        launch((unsigned)std::min(blocks - first, most), (int)first);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// ---- region selection (slide_region_select.hip)
size_t select_workspace_bytes(const Args& a);
hipError_t launch_select(const Args& a, int* index, void* workspace, hipStream_t st);

// ---- region attention (slide_region_fwd.hip, slide_region_bwd.hip)
size_t fwd_workspace_bytes(const Args& a);
hipError_t launch_fwd(const Args& a, void* out, float* lse, void* workspace, hipStream_t st);
size_t bwd_workspace_bytes(const Args& a);
hipError_t launch_bwd(const Args& a, const void* dout, const void* out, const float* lse, void* dq, void* dk, void* dv,
                      void* workspace, hipStream_t st);

// ---- dropout (slide_dropout.hip): y = residual + keep * scale * x over n contiguous elements; residual may be null
hipError_t launch_dropout(const void* x, const void* residual, void* y, long long n, int dtype, const Random& r, hipStream_t st);

}  // namespace region
}  // namespace slide
