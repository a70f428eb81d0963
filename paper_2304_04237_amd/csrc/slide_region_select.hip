// Region selection: which regions of keys the rows of a group attend.
//
//   score(i, j) = (sum of q over the group's valid rows) . (sum of k over region j's valid places) / (number of those places)
//
// The T highest, ties to the lowest index.  Sums and products are held in 64 bits: a selection is a decision, and in 32 bits the
// order of two near scores would hang on the order of a sum.  Two launches: sums of the regions of q and k (bound by reading them
// once), then scores by 64-bit matrix products into LDS and a search for the T-th highest, bit by bit.
#include "slide_region.h"

namespace slide {
namespace region {

typedef double d4 __attribute__((ext_vector_type(4)));
typedef double d2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int POOL = 256, PICK = 512;       // threads of a pooling and of a picking block

// One side of the problem (queries, or keys with g = 1) as the pooling kernel sees it.  A thread owns one piece (E channels) of one
// key head and every lanes-th place of its region; a block takes `packed` regions if they are small, and `together` key heads.
struct Side {
    const void* x;
    Strides s;
    Map m;
    int g;
    int pieces, together, units;        // pieces of a head, key heads of a block, threads that one place takes (pieces * together)
    int lanes, packed;                  // places in flight per region, regions per block
    int head_blocks, blocks;
    double* sum;                        // [B * kv][regions][dp], zeros behind d
    int* count;                         // [B][regions]
    int mean;                           // divide by the count
};

struct SelectArgs {
    Side q, k;
    int B, kv, d, dp, T, groups;
    int* index;
};

template <typename T, int E> struct Piece {
    __device__ static __forceinline__ void add(double (&s)[E], const T* p)
    {
        static_assert(E == 1, "one channel at a time");
        s[0] += (double)Elem<T>::load(p);
    }
};
template <> struct Piece<bf16_bits, 8> {
    __device__ static __forceinline__ void add(double (&s)[8], const bf16_bits* p)
    {
        const u4 x = *(const u4*)p;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s[2 * e] += (double)__uint_as_float(x[e] << 16);
            s[2 * e + 1] += (double)__uint_as_float(x[e] & 0xffff0000u);
        }
    }
};
template <> struct Piece<float, 4> {
    __device__ static __forceinline__ void add(double (&s)[4], const float* p)
    {
        const u4 x = *(const u4*)p;
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += (double)__uint_as_float(x[e]);
    }
};

template <typename T, int E>
__device__ __forceinline__ void pool(const Side& a, int block, int B, int kv, int d, int dp, double* red)
{
    const int hb = block % a.head_blocks;
    block /= a.head_blocks;
    const int per_image = (a.m.regions + a.packed - 1) / a.packed;
    const int b = block / per_image, r0 = (block - b * per_image) * a.packed;
    const int t = threadIdx.x, unit = t % a.units, l = t / a.units;
    const int pl = l % a.lanes, rl = l / a.lanes;
    const int piece = unit % a.pieces, head = hb * a.together + unit / a.pieces, r = r0 + rl;
    const bool live = rl < a.packed && r < a.m.regions && head < kv;
    int vh, vw;
    a.m.limits(b, vh, vw);
    double s[E] = {};
    int n = 0;
    if (live) {
        const T* x = (const T*)a.x + b * a.s.image + (long long)head * a.g * d + piece * E;
#pragma unroll 4
        for (int p = pl; p < a.m.places; p += a.lanes) {
            const int px = a.m.pixel(r, p, vh, vw);
            if (px < 0) continue;
            ++n;
            const T* at = x + px * a.s.pixel;
            for (int e = 0; e < a.g; ++e) Piece<T, E>::add(s, at + e * d);
        }
    }
    // lanes of a wave first, where a wave holds whole places of one region; then through LDS, in the lanes' order
    const bool waves = a.units <= 32 && (a.units & (a.units - 1)) == 0 && a.lanes * a.units >= 64;
    if (waves) {
        for (int w = a.units; w < 64; w <<= 1) {
#pragma unroll
            for (int e = 0; e < E; ++e) s[e] += __shfl_xor(s[e], w);
            n += __shfl_xor(n, w);
        }
    }
    int* counts = (int*)(red + E * POOL);
#pragma unroll
    for (int e = 0; e < E; ++e) red[e * POOL + t] = s[e];
    counts[t] = n;
    __syncthreads();
    const int step = waves ? 64 / a.units : 1;
    for (int o = t; o < a.packed * a.units * E; o += POOL) {
        const int e = o % E, u = o / E % a.units, q = o / E / a.units;
        const int region = r0 + q, m = hb * a.together + u / a.pieces, c = (u % a.pieces) * E + e;
        if (region >= a.m.regions || m >= kv) continue;
        double sum = 0.0;
        int valid = 0;
        for (int i = 0; i < a.lanes; i += step) {
            const int from = (q * a.lanes + i) * a.units + u;
            sum += red[e * POOL + from];
            valid += counts[from];
        }
        double* out = a.sum + (((long long)b * kv + m) * a.m.regions + region) * dp;
        out[c] = a.mean && valid ? sum / valid : sum;
        if (c == 0) {
            if (m == 0) a.count[(long long)b * a.m.regions + region] = valid;
            for (int z = d; z < dp; ++z) out[z] = 0.0;
        }
    }
}

template <typename T, int E>
__global__ __launch_bounds__(POOL) void region_pool_kernel(SelectArgs f, int first)
{
    __shared__ double red[E * POOL + POOL / 2];
    const int block = blockIdx.x + first;
    if (block < f.q.blocks) pool<T, E>(f.q, block, f.B, f.kv, f.d, f.dp, red);
    else pool<T, E>(f.k, block - f.q.blocks, f.B, f.kv, f.d, f.dp, red);
}

// A score as a number whose order is the score's: 0 for a region that cannot be picked, above it -infinity and NaN.
__device__ __forceinline__ uint64_t rank_of(double s)
{
    if (!(s > -1.7976931348623157e308)) s = -1.7976931348623157e308;
    s += 0.0;                                                       // (-0 is 0)
    const uint64_t u = __builtin_bit_cast(uint64_t, s);
    return u ^ ((uint64_t)((int64_t)u >> 63) | 0x8000000000000000ull);
}

// The T highest of a group's J ranks, written in ascending order of the regions.  One wave; get(u): rank of region 64 u + lane, 0 behind J.
template <typename Get>
__device__ __forceinline__ void pick(Get get, int chunks, int T, int* list)
{
    const int lane = threadIdx.x & 63;
    auto at_least = [&](uint64_t x) {
        int n = 0;
        for (int u = 0; u < chunks; ++u) n += __popcll(__ballot(get(u) >= x));
        return n;
    };
    const int usable = at_least(1), want = min(T, usable);
    uint64_t least = 1;                     // the highest rank that `want` regions reach
    if (usable > T) {
        // bit by bit from the top; mostly the wanted ones are of the highest one's sign and, within four times, size, and the search
        // starts below those bits (10 of some 22 steps)
        uint64_t highest = 0;
        for (int u = 0; u < chunks; ++u) highest = max(highest, get(u));
#pragma unroll
        for (int w = 32; w > 0; w >>= 1) highest = max(highest, (uint64_t)__shfl_xor((unsigned long long)highest, w));
        const uint64_t prefix = highest >> 53 << 53;
        const bool near = at_least(prefix) >= want;
        least = near ? prefix : 0;
        for (int bit = near ? 52 : 63; bit >= 0; --bit) {
            const uint64_t x = least | 1ull << bit;
            const int n = at_least(x);
            if (n >= want) least = x;
            if (n == want) break;
        }
    }
    int above = 0;
    for (int u = 0; u < chunks; ++u) above += __popcll(__ballot(get(u) > least));
    int equal_left = want - above, written = 0;
    for (int u = 0; u < chunks && written < want; ++u) {
        const uint64_t x = get(u);
        const uint64_t equal = __ballot(x == least), below = (1ull << lane) - 1;
        const bool taken = x > least || (x == least && __popcll(equal & below) < equal_left);
        const uint64_t mask = __ballot(taken);
        if (taken) list[written + __popcll(mask & below)] = 64 * u + lane;
        written += __popcll(mask);
        equal_left -= min(equal_left, (int)__popcll(equal));
    }
    for (int u = want + lane; u < T; u += 64) list[u] = -1;
}

// NG groups of one key head per block: scores of 16 x 16 groups and regions by v_mfma_f64_16x16x4_f64 (left lane: group lane % 16, channels
// 8 s + 2 (lane / 16) and the next; right likewise the region; register r of the result: group 4 r + lane / 16, region lane % 16), then one
// wave per group.  CHUNKS: regions in a lane's registers; 0: read again from LDS.
template <int CHUNKS>
__global__ __launch_bounds__(PICK) void region_pick_kernel(SelectArgs f, int NG, int stride, int first)
{
    extern __shared__ uint64_t rank[];              // [NG][stride]
    const int G = f.q.m.regions, J = f.k.m.regions, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per_head = (G + NG - 1) / NG;
    const int block = blockIdx.x + first, bm = block / per_head, i0 = (block - bm * per_head) * NG, b = bm / f.kv;
    const int col = lane & 15, part = lane >> 4;
    const int gi = min(i0 + min(col, NG - 1), G - 1);
    const double* qp = f.q.sum + ((long long)bm * G + gi) * f.dp + 2 * part;
    // With many regions two tiles at a time: their loads and their chains of products overlap (512 regions: 46 against 39 us)
    constexpr int W = CHUNKS == 1 || CHUNKS == 2 ? 1 : 2;
    for (int j0 = 16 * W * wave; j0 < J; j0 += W * PICK / 4) {
        const double* kp[W];
        d4 acc[W] = {};
#pragma unroll
        for (int u = 0; u < W; ++u) kp[u] = f.k.sum + ((long long)bm * J + min(j0 + 16 * u + col, J - 1)) * f.dp + 2 * part;
#pragma unroll 4
        for (int c = 0; c < f.dp; c += 8) {
            const d2 x = *(const d2*)(qp + c);
            d2 y[W];
#pragma unroll
            for (int u = 0; u < W; ++u) y[u] = *(const d2*)(kp[u] + c);
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int u = 0; u < W; ++u) acc[u] = __builtin_amdgcn_mfma_f64_16x16x4f64(x[e], y[u][e], acc[u], 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < W; ++u) {
            const int j = j0 + 16 * u + col;
            const bool usable = j < J && f.k.count[(long long)b * J + min(j, J - 1)] > 0;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (4 * r + part < NG && j < stride) rank[(4 * r + part) * stride + j] = usable ? rank_of(acc[u][r]) : 0;
        }
    }
    __syncthreads();
    for (int n = wave; n < NG && i0 + n < G; n += PICK / 64) {
        int* list = f.index + ((long long)bm * G + i0 + n) * f.T;
        const bool any = f.q.count[(long long)b * G + i0 + n] > 0;
        const uint64_t* row = rank + n * stride;
        if constexpr (CHUNKS > 0) {
            uint64_t mine[CHUNKS];
#pragma unroll
            for (int u = 0; u < CHUNKS; ++u) mine[u] = any && 64 * u + lane < J ? row[64 * u + lane] : 0;
            // (a constant number of chunks: the loops unroll and the ranks stay in registers)
            pick([&](int u) { return mine[u]; }, CHUNKS, f.T, list);
        } else {
            pick([&](int u) { return any && 64 * u + lane < J ? row[64 * u + lane] : 0ull; }, (J + 63) / 64, f.T, list);
        }
    }
}

static int padded(int d) { return (d + 7) & ~7; }           // (whole steps of two matrix instructions)

struct SelectRoom { size_t q, k, nq, nk, end; };

static SelectRoom room(const Args& a)
{
    const size_t bm = (size_t)a.B * a.kv, dp = padded(a.d);
    SelectRoom r;
    r.q = 0;
    r.k = r.q + bm * a.qm.regions * dp * sizeof(double);
    r.nq = r.k + bm * a.km.regions * dp * sizeof(double);
    r.nk = r.nq + ((size_t)a.B * a.qm.regions + 3) / 4 * 16;
    r.end = r.nk + (size_t)a.B * a.km.regions * sizeof(int);
    return r;
}

size_t select_workspace_bytes(const Args& a) { return room(a).end; }

static Side side_of(const Args& a, const void* x, const Strides& s, const Map& m, int g, int E)
{
    Side o{};
    o.x = x; o.s = s; o.m = m; o.g = g;
    o.pieces = a.d / E;
    o.together = std::min(a.kv, std::max(1, POOL / o.pieces));
    o.units = o.pieces * o.together;
    const int lanes = POOL / o.units;
    o.lanes = 1;
    while (o.lanes * 2 <= lanes && o.lanes * 8 < m.places * g) o.lanes *= 2;      // (eight loads or so for each thread)
    o.packed = lanes / o.lanes;
    o.head_blocks = (a.kv + o.together - 1) / o.together;
    o.blocks = a.B * ((m.regions + o.packed - 1) / o.packed) * o.head_blocks;
    return o;
}

template <typename T, int E>
static hipError_t run(const Args& a, int* index, unsigned char* ws, hipStream_t st)
{
    const SelectRoom r = room(a);
    SelectArgs f{};
    f.q = side_of(a, a.q, a.qs, a.qm, a.g, E);
    f.k = side_of(a, a.k, a.ks, a.km, 1, E);
    f.q.sum = (double*)(ws + r.q); f.k.sum = (double*)(ws + r.k);
    f.q.count = (int*)(ws + r.nq); f.k.count = (int*)(ws + r.nk);
    f.k.mean = 1;
    f.B = a.B; f.kv = a.kv; f.d = a.d; f.dp = padded(a.d); f.T = a.T;
    f.index = index;
    hipError_t e = in_launches(f.q.blocks + f.k.blocks, POOL, [&](unsigned blocks, int first) {
        region_pool_kernel<T, E><<<blocks, POOL, 0, st>>>(f, first);
    });
    if (e != hipSuccess) return e;

    // groups per block: 16 fill a matrix instruction; fewer where their ranks would not let two blocks into a compute unit
    const int J = a.km.regions, stride = (J + 15) / 16 * 16 + 2;
    int NG = 16;
    while (NG > 4 && NG * stride * 8 > 80 * 1024) NG /= 2;
    while (NG > 1 && NG * stride * 8 > 144 * 1024) NG /= 2;
    const int blocks = a.B * a.kv * ((a.qm.regions + NG - 1) / NG), lds = NG * stride * 8;
    static LdsOptIn opt;
    e = opt.ensure({(const void*)region_pick_kernel<0>, (const void*)region_pick_kernel<1>, (const void*)region_pick_kernel<2>,
                    (const void*)region_pick_kernel<4>, (const void*)region_pick_kernel<8>, (const void*)region_pick_kernel<16>}, 144 * 1024);
    if (e != hipSuccess) return e;
    const auto kernel = J <= 64 ? region_pick_kernel<1> : J <= 128 ? region_pick_kernel<2> : J <= 256 ? region_pick_kernel<4>
                      : J <= 512 ? region_pick_kernel<8> : J <= 1024 ? region_pick_kernel<16> : region_pick_kernel<0>;
    return in_launches(blocks, PICK, [&](unsigned n, int first) { kernel<<<n, PICK, lds, st>>>(f, NG, stride, first); });
}

hipError_t launch_select(const Args& a, int* index, void* workspace, hipStream_t st)
{
    unsigned char* ws = (unsigned char*)workspace;
    const bool f32 = a.dtype == 0;
    const int n = f32 ? 4 : 8;
    const auto whole = [&](const void* p, const Strides& s) { return ((uintptr_t)p & 15) == 0 && s.pixel % n == 0 && s.image % n == 0; };
    const bool vec = a.d % n == 0 && whole(a.q, a.qs) && whole(a.k, a.ks);
    if (f32) return vec ? run<float, 4>(a, index, ws, st) : run<float, 1>(a, index, ws, st);
    return vec ? run<bf16_bits, 8>(a, index, ws, st) : run<bf16_bits, 1>(a, index, ws, st);
}

}  // namespace region
}  // namespace slide
