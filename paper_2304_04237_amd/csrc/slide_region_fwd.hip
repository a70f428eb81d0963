// Region attention, forward, on the matrix cores.
//
// One wave takes 32 NR rows of a group and walks over the group's keys, the slots of the listed regions one after the other, 32 at
// a time: S^T = K Q^T (keys are rows of the result, so a lane holds 16 keys of one query row and the softmax needs one exchange
// between the lane halves), P = exp2(S c - m) with a running maximum m and sum, O^T += V^T P^T.  P stays in the registers in which the
// first product leaves it.  K and V come by way of 32 rows of LDS each that only this wave uses, loaded one tile ahead.  Waves share
// nothing, so no barrier is passed and the waves of a compute unit cover each other's latencies.
//
// What bounds it: heads of 32 in bf16 the vector work (64 x 56x56, 4 regions of 8x8: 48 us, vector instructions issue 72 % of the time, matrix
// instructions 15 %).  It is 8.4 vector instructions per weight, of which the softmax itself is four (an exponential, a multiply-add, an
// addition, half a maximum, half a conversion); the others make values canonical before the maximum, look up the keys and stage them.
// float32: the matrix instructions (28x28, 4 regions of 7x7: 51 us, busy 59 % of the time).
//
// Few rows over many keys (one new token) leave most of the chip idle that way.  Then the keys of a group are split: the four waves
// of a block take a quarter each of a share of the keys and join their sums in LDS, and where one block per 32 rows is still too
// little, shares go to several blocks, whose float32 sums a second kernel joins.  What is divided is the list's full length: a list that ends
// early leaves the later shares idle (one token, 64 entries of 64 tokens: 23 us, with 32 of them 18.6, with 4 17.7).
#include "slide_region_mma.h"

namespace slide {
namespace region {

struct FwdArgs {
    Args a;
    void* out;
    float* lse;
    int tiles;              // of 32 NR rows in a group
    int slots;              // keys of a group, with every listed region's slots a multiple of 4
    int vec, vec_o;         // q, k, v in whole 16-byte pieces; out in whole quads
    int items;              // waves (SPLIT: blocks) with work
    int shares;             // SPLIT: blocks that share the keys of 32 rows
    float* part;            // SPLIT, shares > 1: [rows' item][share][32][D] sums, then [2][32] maxima and sums
};

// out and lse of a row from its sums: o[0..3] channels c ..
template <typename T>
__device__ __forceinline__ void finish(const FwdArgs& f, long long out_at, int c, const float (&o)[4], float up)
{
    const float x[4] = {up != 0.0f ? o[0] * up : 0.0f, up != 0.0f ? o[1] * up : 0.0f, up != 0.0f ? o[2] * up : 0.0f, up != 0.0f ? o[3] * up : 0.0f};
    store4((T*)f.out + out_at + c, x, f.a.d - c, f.vec_o);
}

template <typename T, int D, int NR, bool DROP, bool SPLIT, bool VEC>
__global__ __launch_bounds__(256) void region_fwd_kernel(FwdArgs f)
{
    const Args& a = f.a;
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int work = SPLIT ? (int)xcd_order(blockIdx.x, gridDim.x) : (int)xcd_order(blockIdx.x, gridDim.x) * 4 + wave;
    if (work >= f.items) return;
    const int item = SPLIT ? work / f.shares : work, share = SPLIT ? work - item * f.shares : 0;
    unsigned char* tile_k = lds + wave * 2 * Tile<T, D>::BYTES;
    unsigned char* tile_v = tile_k + Tile<T, D>::BYTES;
    int first = 0, end = f.slots;
    if (SPLIT) {
        const int key_tiles = (f.slots + 31) / 32, parts = 4 * f.shares, w = 4 * share + wave;
        first = (int)((long long)key_tiles * w / parts) * 32;
        end = min(f.slots, (int)((long long)key_tiles * (w + 1) / parts) * 32);
    }
    const int group = item / f.tiles, row0 = (item - group * f.tiles) * 32 * NR;
    const int bm = group / a.qm.regions, i = group - bm * a.qm.regions;
    const int b = bm / a.kv, m = bm - b * a.kv;
    const int col = lane & 31, h = lane >> 5;

    // this lane's rows
    Operand<T, D> q[NR];
    long long out_at[NR];           // element of the row in out, -1: none
    long long lse_at[NR];
    {
        int vh, vw;
        a.qm.limits(b, vh, vw);
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const int r = row0 + 32 * n + col;
            const int place = a.by_g.of(r), head = m * a.g + r - place * a.g;
            const int px = r < a.R ? a.qm.pixel(i, place, a.qm.H, a.qm.W) : -1;
            const bool ok = r < a.R && a.qm.pixel(i, place, vh, vw) >= 0;
            const long long n_px = (long long)a.qm.H * a.qm.W;
            out_at[n] = px < 0 ? -1 : ((long long)b * n_px + px) * a.heads * a.d + head * a.d;
            lse_at[n] = px < 0 ? -1 : (((long long)b * a.heads + head) * n_px + px) * 2 + ok;      // (lowest bit: the row is valid)
            load_operand<T, D, VEC>(q[n], (const T*)a.q + b * a.qs.image + (ok ? px : 0) * a.qs.pixel + head * a.hd, ok, a.dl, h);
        }
    }
    const uint32_t call = DROP ? a.rnd.call() : 0;
    const float c2 = a.scale * LOG2E;
    f16v o[NR][D / 32];
    float top[NR], sub[NR], sum[NR];        // running maximum (of S c2), what is subtracted (0 while there is none), this lane's sum
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        top[n] = -INFINITY; sub[n] = 0.0f; sum[n] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) o[n][dt] = f16v{};
    }

    const T* kp = (const T*)a.k + b * a.ks.image + m * a.hd;
    const T* vp = (const T*)a.v + b * a.vs.image + m * a.hd;
    Walk walk;
    walk.list = a.index + (long long)group * a.T;
    a.km.limits(b, walk.vh, walk.vw);
    end = min(end, walk.length(a));
    Rows<T, D> k, v;
    int region = walk.look(a, first + col, end);
    uint32_t word, next_word = 0;
    uint32_t ok, next_ok;
    auto fetch = [&]() {
        const int px = Walk::pixel(a, region, walk.place, walk.vh, walk.vw);
        next_ok = (uint32_t)__ballot(px >= 0);
        if (DROP) next_word = (uint32_t)region * a.quads + (walk.place >> 2);
        k.template load<VEC>(kp, row_offset<VEC, T>(px, a.ks.pixel, 0), a.dl, lane);
        v.template load<VEC>(vp, row_offset<VEC, T>(px, a.vs.pixel, 0), a.dl, lane);
    };
    fetch();
    region = walk.look(a, first + 32 + col, end);
    for (int x = first; x < end; x += 32) {
        ok = next_ok; word = next_word;
        wave_order();
        k.stage(tile_k, ok, a.dl, lane);
        v.stage(tile_v, ok, a.dl, lane);
        wave_order();
        fetch();
        region = walk.look(a, x + 64 + col, end);
        if (ok == 0) continue;
        Operand<T, D> kk;
        read_operand<D>(kk, tile_k, lane);
        Weights<T> w[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            f16v s = dot<D>(kk, q[n], f16v{});
            if (ok != 0xffffffffu) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!((ok >> acc_row(r, 0)) >> (4 * h) & 1)) s[r] = -INFINITY;
            }
            float most = s[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) most = fmaxf(most, s[r]);
            most = halves_max(most) * c2;
            // the maximum moves only where a weight would pass 2^8: below that the sums lose nothing, and most tiles need no rescaling
            if (__ballot(most > (top[n] == -INFINITY ? -INFINITY : top[n] + 8.0f))) {
                const float next = fmaxf(top[n], most);
                const float back = next == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top[n] - next);
                top[n] = next;
                sub[n] = next == -INFINITY ? 0.0f : next;
                sum[n] *= back;
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) o[n][dt] *= back;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c2, -sub[n]));
                sum[n] += s[r];
            }
            if (DROP) {
                uint32_t words[4][2];
                row_keep(a.rnd, call, word, (uint32_t)i * a.pairs + ((row0 + 32 * n + col) >> 1), bm, words);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if ((words[r >> 2][(r & 3) >> 1] >> (16 * (r & 1)) & 0xffffu) < a.rnd.threshold) s[r] = 0.0f;
            }
            w[n].set(s);
        }
        accumulate<D, NR>(o, tile_v, w, lane);
    }

    if constexpr (SPLIT) {
        // [wave][D][32] sums and [wave][2][32] maxima and sums; thread: row col, every eighth quad of channels
        static_assert(NR == 1, "the split form takes 32 rows");
        float* sums = (float*)lds;
        float* stat = sums + 4 * D * 32;
        const float total = halves_sum(sum[0]);
        __syncthreads();                                    // (the tiles are in the same place)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) sums[(wave * D + 32 * dt + acc_row(r, h)) * 32 + col] = o[0][dt][r];
        if (h == 0) { stat[wave * 64 + col] = top[0]; stat[wave * 64 + 32 + col] = total; }
        __syncthreads();
        float most = -INFINITY, all = 0.0f, back[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) most = fmaxf(most, stat[w * 64 + col]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float t = stat[w * 64 + col];
            back[w] = t == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(t - most);
            all += back[w] * stat[w * 64 + 32 + col];
        }
        if (out_at[0] < 0) return;
        const bool valid = lse_at[0] & 1;
        float* part = f.part + ((long long)item * f.shares + share) * (D * 32 + 64);
        const float up = !valid || all == 0.0f ? 0.0f : (DROP ? a.rnd.scale : 1.0f) / all;
        for (int c = 4 * (threadIdx.x >> 5); c < D; c += 32) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = 0.0f;
#pragma unroll
                for (int w = 0; w < 4; ++w) x[e] = __builtin_fmaf(back[w], sums[(w * D + c + e) * 32 + col], x[e]);
            }
            if (f.shares == 1) {
                finish<T>(f, out_at[0], c, x, up);
            } else {
                *(f4*)(part + col * D + c) = f4{x[0], x[1], x[2], x[3]};
            }
        }
        if (threadIdx.x < 32) {
            if (f.shares > 1) { part[D * 32 + col] = most; part[D * 32 + 32 + col] = all; }
            else if (f.lse) f.lse[lse_at[0] >> 1] = up == 0.0f ? -INFINITY : ((most == -INFINITY ? 0.0f : most) + log2f(all)) * LN2;
        }
    } else {
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const float total = halves_sum(sum[n]);
            if (out_at[n] < 0) continue;
            const float up = !(lse_at[n] & 1) || total == 0.0f ? 0.0f : (DROP ? a.rnd.scale : 1.0f) / total;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const float x[4] = {o[n][dt][r], o[n][dt][r + 1], o[n][dt][r + 2], o[n][dt][r + 3]};
                    finish<T>(f, out_at[n], 32 * dt + acc_row(r, h), x, up);
                }
            if (h == 0 && f.lse) f.lse[lse_at[n] >> 1] = up == 0.0f ? -INFINITY : (sub[n] + log2f(total)) * LN2;
        }
    }
}

// Joins the sums of the blocks that shared a row's keys.  One wave per row of 32; a lane takes D / 64 channels.
template <typename T, int D>
__global__ __launch_bounds__(256) void region_fwd_join_kernel(FwdArgs f)
{
    const Args& a = f.a;
    const int lane = threadIdx.x & 63, item = blockIdx.x, group = item / f.tiles;
    const int col = 4 * blockIdx.y + (threadIdx.x >> 6), r = (item - group * f.tiles) * 32 + col;
    if (r >= a.R) return;
    const int bm = group / a.qm.regions, i = group - bm * a.qm.regions, b = bm / a.kv, m = bm - b * a.kv;
    const int place = a.by_g.of(r), head = m * a.g + r - place * a.g, px = a.qm.pixel(i, place, a.qm.H, a.qm.W);
    if (px < 0) return;
    int vh, vw;
    a.qm.limits(b, vh, vw);
    const bool valid = a.qm.pixel(i, place, vh, vw) >= 0;
    constexpr int SIZE = D * 32 + 64;
    const float* part = f.part + (long long)item * f.shares * SIZE;
    float most = -INFINITY, all = 0.0f, x[(D + 63) / 64] = {};
    for (int s = lane; s < f.shares; s += 64) most = fmaxf(most, part[(long long)s * SIZE + D * 32 + col]);
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) most = fmaxf(most, __shfl_xor(most, w));
    for (int s0 = 0; s0 < f.shares; s0 += 64) {
        const int s = s0 + lane;
        const float* p = part + (long long)s * SIZE + D * 32 + col;
        const float t = s < f.shares ? p[0] : -INFINITY;
        const float mine = t == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(t - most);
        float sum = s < f.shares ? mine * p[32] : 0.0f;
#pragma unroll
        for (int w = 32; w > 0; w >>= 1) sum += __shfl_xor(sum, w);
        all += sum;
        const int n = min(64, f.shares - s0);
#pragma unroll 8
        for (int k = 0; k < n; ++k) {
            const float back = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), k));
            const float* from = part + (long long)(s0 + k) * SIZE + col * D;
#pragma unroll
            for (int u = 0; u < (D + 63) / 64; ++u)
                if (lane + 64 * u < D) x[u] = __builtin_fmaf(back, from[lane + 64 * u], x[u]);
        }
    }
    const float up = !valid || all == 0.0f ? 0.0f : a.rnd.scale / all;
    const long long n_px = (long long)a.qm.H * a.qm.W, at = ((long long)b * n_px + px) * a.heads * a.d + head * a.d;
#pragma unroll
    for (int u = 0; u < (D + 63) / 64; ++u)
        if (lane + 64 * u < a.d) Elem<T>::store((T*)f.out + at + lane + 64 * u, up != 0.0f ? x[u] * up : 0.0f);
    if (lane == 0 && f.lse)
        f.lse[((long long)b * a.heads + head) * n_px + px] = up == 0.0f ? -INFINITY : ((most == -INFINITY ? 0.0f : most) + log2f(all)) * LN2;
}

// How a problem is cut.  A block per 32 rows and share of the keys (SPLIT) where a wave per 32 rows would not give every SIMD one (8 new
// tokens, 32 heads of 128 over 4096 keys: 236 us by 32 waves, 28 split), and for heads of 128 half of them (704 waves of float32: 53 us, split
// 87); then as many shares as give every SIMD one wave, of at least eight key tiles each.
struct Cut { bool split; int tiles, shares; };

static Cut cut(const Args& a)
{
    const int cus = device_cu_count();
    const long long groups = (long long)a.B * a.kv * a.qm.regions;
    Cut c{false, (a.R + 31) / 32, 1};
    const long long items = groups * c.tiles;
    const int key_tiles = (4 * a.quads * a.T + 31) / 32;
    c.split = items < (a.d > 64 ? 2ll : 4ll) * cus && key_tiles > 1;
    if (c.split) c.shares = (int)std::max(1ll, std::min((cus + items - 1) / items, (long long)key_tiles / 8));
    return c;
}

static int padded(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }

size_t fwd_workspace_bytes(const Args& a)
{
    const Cut c = cut(a);
    return packing(a, false).end + (c.shares > 1 ? (size_t)a.B * a.kv * a.qm.regions * c.tiles * c.shares * (padded(a.d) * 32 + 64) * sizeof(float) : 0);
}

template <typename T, int D>
static hipError_t run_split(FwdArgs& f, const Cut& c, hipStream_t st)
{
    f.tiles = c.tiles;
    f.shares = c.shares;
    const int items = f.a.B * f.a.kv * f.a.qm.regions * f.tiles;
    f.items = items * f.shares;
    const int lds = std::max(8 * Tile<T, D>::BYTES, 4 * (D * 32 + 64) * (int)sizeof(float));
    // (what is not in whole pieces takes the kernel with dropout, which drops nothing below a threshold of 0)
    static LdsOptIn opt;
    hipError_t e = opt.ensure({(const void*)region_fwd_kernel<T, D, 1, true, true, true>, (const void*)region_fwd_kernel<T, D, 1, false, true, true>,
                               (const void*)region_fwd_kernel<T, D, 1, true, true, false>}, lds);
    if (e != hipSuccess) return e;
    const auto kernel = !f.vec ? region_fwd_kernel<T, D, 1, true, true, false>
                      : f.a.rnd.threshold ? region_fwd_kernel<T, D, 1, true, true, true> : region_fwd_kernel<T, D, 1, false, true, true>;
    kernel<<<f.items, 256, lds, st>>>(f);
    if ((e = hipGetLastError()) != hipSuccess || f.shares == 1) return e;
    region_fwd_join_kernel<T, D><<<dim3(items, (std::min(f.a.R, 32) + 3) / 4), 256, 0, st>>>(f);
    return hipGetLastError();
}

template <typename T, int D, int NR>
static hipError_t run(FwdArgs& f, hipStream_t st)
{
    f.tiles = (f.a.R + 32 * NR - 1) / (32 * NR);
    const long long items = (long long)f.a.B * f.a.kv * f.a.qm.regions * f.tiles;
    f.items = (int)items;
    const int blocks = (int)((items + 3) / 4), lds = 8 * Tile<T, D>::BYTES;
    static LdsOptIn opt;
    const hipError_t e = opt.ensure({(const void*)region_fwd_kernel<T, D, NR, true, false, true>, (const void*)region_fwd_kernel<T, D, NR, false, false, true>,
                                     (const void*)region_fwd_kernel<T, D, 1, true, false, false>}, lds);
    if (e != hipSuccess) return e;
    const auto kernel = !f.vec ? region_fwd_kernel<T, D, 1, true, false, false>
                      : f.a.rnd.threshold ? region_fwd_kernel<T, D, NR, true, false, true> : region_fwd_kernel<T, D, NR, false, false, true>;
    kernel<<<blocks, 256, lds, st>>>(f);
    return hipGetLastError();
}

template <typename T>
static hipError_t run_t(FwdArgs& f, unsigned char* ws, hipStream_t st)
{
    const Args& a = f.a;
    const Packing copies = packing(a, false);
    if (copies.on) {
        const hipError_t e = pack<T>(f.a, copies, nullptr, nullptr, ws, st);
        if (e != hipSuccess) return e;
    }
    f.part = (float*)(ws + copies.end);
    const long long nq = (long long)a.qm.H * a.qm.W, nk = (long long)a.km.H * a.km.W;
    f.vec = pieces(a.q, a.qs, a.dl, sizeof(T), nq) && pieces(a.k, a.ks, a.dl, sizeof(T), nk) && pieces(a.v, a.vs, a.dl, sizeof(T), nk);
    f.vec_o = a.d % 4 == 0 && ((uintptr_t)f.out & (4 * sizeof(T) - 1)) == 0;
    const Cut c = cut(a);
    if (c.split) return a.d <= 32 ? run_split<T, 32>(f, c, st) : a.d <= 64 ? run_split<T, 64>(f, c, st) : run_split<T, 128>(f, c, st);
    // Two row tiles per wave load and stage every key half as often, where the registers hold them (bf16; one tile: 2 x 200 x 333
    // pixels, heads of 32: 130 against 115 us; 16384 tokens, heads of 64: 95 against 72).  With heads of 32 an odd tile left over costs more than
    // that where there are few (50 x 40 x 48 pixels, 80 rows: 102 us by two, 80 by one).
    const int tiles = (a.R + 31) / 32;
    const bool two = a.R > 32 && f.vec && !(a.d <= 32 && tiles < 8 && tiles % 2);
    if (a.d <= 32) return two ? run<T, 32, 2>(f, st) : run<T, 32, 1>(f, st);
    if (a.d <= 64) return two && sizeof(T) == 2 ? run<T, 64, 2>(f, st) : run<T, 64, 1>(f, st);
    return run<T, 128, 1>(f, st);
}

hipError_t launch_fwd(const Args& a, void* out, float* lse, void* workspace, hipStream_t st)
{
    FwdArgs f{};
    f.a = a; f.out = out; f.lse = lse;
    f.slots = 4 * a.quads * a.T;
    return a.dtype == 0 ? run_t<float>(f, (unsigned char*)workspace, st) : run_t<bf16_bits>(f, (unsigned char*)workspace, st);
}

}  // namespace region
}  // namespace slide
