// Region attention, forward, on the matrix cores.
//
// One wave takes 32 NR rows of a group and walks over the group's keys, the slots of the listed regions one after the other, 32 at
// a time: S^T = K Q^T (keys are rows of the result, so a lane holds 16 keys of one query row and the softmax needs one exchange
// between the lane halves), P = exp2(S c - m) with a running maximum m and sum, O^T += V^T P^T.  P stays in the registers in which the
// first product leaves it.  K goes from memory into operands, V through 32 rows of LDS that only this wave uses; both are loaded
// one tile ahead.  Waves share nothing, so no barrier is passed and the waves of a compute unit cover each other's latencies.
#include "slide_region_mma.h"

namespace slide {
namespace region {

struct FwdArgs {
    Args a;
    void* out;
    float* lse;
    int tiles;              // of 32 NR rows in a group
    int slots;              // keys of a group, with every listed region's slots a multiple of 4
    int vec_q, vec_k, vec_v, vec_o;
    int items;              // waves with work
};

template <typename T, int D, int NR, bool DROP>
__global__ __launch_bounds__(256) void region_fwd_kernel(FwdArgs f)
{
    const Args& a = f.a;
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int item = (int)xcd_order(blockIdx.x, gridDim.x) * 4 + wave;
    if (item >= f.items) return;
    unsigned char* tile = lds + wave * Tile<T, D>::BYTES;
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
            load_operand<T, D>(q[n], (const T*)a.q + b * a.qs.image + (ok ? px : 0) * a.qs.pixel + head * a.d, ok, a.d, h, f.vec_q);
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

    const T* kp = (const T*)a.k + b * a.ks.image + m * a.d;
    const T* vp = (const T*)a.v + b * a.vs.image + m * a.d;
    Walk walk;
    walk.list = a.index + (long long)group * a.T;
    a.km.limits(b, walk.vh, walk.vw);
    Operand<T, D> k[2], v;
    int region = walk.look(a, col, f.slots);
    uint32_t word, next_word = 0;
    uint32_t ok, next_ok;
    auto fetch = [&](Operand<T, D>& kk) {
        const int px = Walk::pixel(a, region, walk.place, walk.vh, walk.vw);
        next_ok = (uint32_t)__ballot(px >= 0);
        if (DROP) next_word = (uint32_t)region * a.quads + (walk.place >> 2);
        load_operand<T, D>(kk, kp + (px < 0 ? 0 : px) * a.ks.pixel, px >= 0, a.d, h, f.vec_k);
        load_operand<T, D>(v, vp + (px < 0 ? 0 : px) * a.vs.pixel, px >= 0, a.d, h, f.vec_v);
    };
    fetch(k[0]);
    region = walk.look(a, 32 + col, f.slots);

    auto step = [&](const Operand<T, D>& kk, Operand<T, D>& kn, int x) {
        ok = next_ok; word = next_word;
        wave_order();
        stage<D>(tile, v, lane);
        wave_order();
        if (x + 32 < f.slots) {
            fetch(kn);
            region = walk.look(a, x + 64 + col, f.slots);
        }
        if (ok == 0) return;
        uint32_t quad[4];
        if (DROP) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t lo = __builtin_amdgcn_readlane(word, 8 * u), hi = __builtin_amdgcn_readlane(word, 8 * u + 4);
                quad[u] = h ? hi : lo;
            }
        }
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
                row_keep(a.rnd, call, quad, (uint32_t)i * a.pairs + ((row0 + 32 * n + col) >> 1), bm, words);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if ((words[r >> 2][(r & 3) >> 1] >> (16 * (r & 1)) & 0xffffu) < a.rnd.threshold) s[r] = 0.0f;
            }
            w[n].set(s);
        }
        accumulate<D, NR>(o, tile, w, lane);
    };
    for (int x = 0; x < f.slots; x += 64) {
        step(k[0], k[1], x);
        if (x + 32 < f.slots) step(k[1], k[0], x + 32);
    }

#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const float total = halves_sum(sum[n]);
        if (out_at[n] < 0) continue;
        const bool valid = lse_at[n] & 1;
        const float up = !valid || total == 0.0f ? 0.0f : (DROP ? a.rnd.scale : 1.0f) / total;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int c = 32 * dt + acc_row(r, h);
                const float x[4] = {valid ? o[n][dt][r] * up : 0.0f, valid ? o[n][dt][r + 1] * up : 0.0f,
                                    valid ? o[n][dt][r + 2] * up : 0.0f, valid ? o[n][dt][r + 3] * up : 0.0f};
                store4((T*)f.out + out_at[n] + c, x, a.d - c, f.vec_o);
            }
        if (h == 0 && f.lse) f.lse[lse_at[n] >> 1] = !valid || total == 0.0f ? -INFINITY : (sub[n] + log2f(total)) * LN2;
    }
}

template <typename T, int D, int NR>
static hipError_t run(FwdArgs& f, hipStream_t st)
{
    f.tiles = (f.a.R + 32 * NR - 1) / (32 * NR);
    const long long items = (long long)f.a.B * f.a.kv * f.a.qm.regions * f.tiles;
    f.items = (int)items;
    const int blocks = (int)((items + 3) / 4), lds = 4 * Tile<T, D>::BYTES;
    if (f.a.rnd.threshold) region_fwd_kernel<T, D, NR, true><<<blocks, 256, lds, st>>>(f);
    else region_fwd_kernel<T, D, NR, false><<<blocks, 256, lds, st>>>(f);
    return hipGetLastError();
}

template <typename T>
static hipError_t run_t(FwdArgs& f, hipStream_t st)
{
    const Args& a = f.a;
    f.vec_q = pieces(a.q, a.qs, a.d, sizeof(T));
    f.vec_k = pieces(a.k, a.ks, a.d, sizeof(T));
    f.vec_v = pieces(a.v, a.vs, a.d, sizeof(T));
    f.vec_o = a.d % 4 == 0 && ((uintptr_t)f.out & (4 * sizeof(T) - 1)) == 0;
    // two row tiles per wave read every key operand half as often, where the registers hold them
    const bool two = a.R > 32;
    if (a.d <= 32) return two ? run<T, 32, 2>(f, st) : run<T, 32, 1>(f, st);
    if (a.d <= 64) return two && sizeof(T) == 2 ? run<T, 64, 2>(f, st) : run<T, 64, 1>(f, st);
    return run<T, 128, 1>(f, st);
}

size_t fwd_workspace_bytes(const Args&) { return 0; }

hipError_t launch_fwd(const Args& a, void* out, float* lse, void*, hipStream_t st)
{
    FwdArgs f{};
    f.a = a; f.out = out; f.lse = lse;
    f.slots = 4 * a.quads * a.T;
    return a.dtype == 0 ? run_t<float>(f, st) : run_t<bf16_bits>(f, st);
}

}  // namespace region
}  // namespace slide
