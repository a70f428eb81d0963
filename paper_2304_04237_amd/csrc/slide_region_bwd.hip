// Region attention, backward, on the matrix cores.
//
//   P = exp(S - lse);  D = dout.out;  dS = P (F dP - D),  dP = dout.v,  F the weights' dropout factors
//   dq = scale sum dS k   (row kernel: a wave per 32 rows of a group, over the group's keys, like the forward)
//   dk = scale sum dS q,  dv = sum F P dout   (key kernel: a wave per 32 keys of a region, over the rows of the groups that list it)
//
// Between the two a kernel turns the lists around (which groups list region j, in ascending order, so that sums have one order).
// A block takes at most `share` of a region's groups; what is beyond goes to further blocks, whose float32 sums a last kernel adds up.
#include "slide_region_mma.h"

namespace slide {
namespace region {

struct BwdArgs {
    Args a;
    const void* dout;
    const void* out;
    const float* lse;
    void* dq;
    void* dk;
    void* dv;
    float* row_lse;         // [groups][row_tiles * 32]: lse in units of log 2, +infinity for a row that takes no part
    float* row_D;
    int2* sorted;           // [B * kv][regions of q * T]: (group, region) of every entry that counts, by region, then by group
    int* start;             // [B * kv][J + 1]
    float* partial;         // [B * kv][key tiles][2 windows][2][32][D]
    int slots, row_tiles, key_tiles, items;
    int entries;            // regions of q * T
    int share, windows;     // entries per block of the key kernel, ceil(entries / share)
    int team;               // waves that share a tile of keys, 1 or 4
    int invert_waves;       // waves per region in the inversion, 1 or 16
    Div by_rows;            // 2 pairs: slots of a group in the key kernel
    int vec, vec_dq, vec_dk;        // inputs in whole 16-byte pieces; dq, dk and dv in whole quads
};

template <typename T> __device__ __forceinline__ float piece_dot(const u4& a, const u4& b);
template <> __device__ __forceinline__ float piece_dot<bf16_bits>(const u4& a, const u4& b)
{
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        s = __builtin_fmaf(__uint_as_float(a[e] << 16), __uint_as_float(b[e] << 16), s);
        s = __builtin_fmaf(__uint_as_float(a[e] & 0xffff0000u), __uint_as_float(b[e] & 0xffff0000u), s);
    }
    return s;
}
template <> __device__ __forceinline__ float piece_dot<float>(const u4& a, const u4& b)
{
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_fmaf(__uint_as_float(a[e]), __uint_as_float(b[e]), s);
    return s;
}

// dq and, for the key kernel, every row's lse and D.
// bf16: out was rounded, so dout.out is off by up to 2^-8 of its terms.  The sum of P F dP, which is D without that, is only known at
// the end; until then the rounded D0 is used, and dq is corrected by (D - D0) sum P k, for one more product.
// SPLIT: the four waves of a block take a quarter each of the keys of the same rows and add their sums in LDS.
template <typename T, int D, bool DROP, bool SPLIT, bool VEC>
__global__ __launch_bounds__(256, 1) void region_dq_kernel(BwdArgs f)
{
    constexpr bool FIX = sizeof(T) == 2;
    const Args& a = f.a;
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int item = SPLIT ? (int)xcd_order(blockIdx.x, gridDim.x) : (int)xcd_order(blockIdx.x, gridDim.x) * 4 + wave;
    if (item >= f.items) return;
    unsigned char* tile_k = lds + wave * 2 * Tile<T, D>::BYTES;
    unsigned char* tile_v = tile_k + Tile<T, D>::BYTES;
    const int group = item / f.row_tiles, row0 = (item - group * f.row_tiles) * 32;
    const int bm = group / a.qm.regions, i = group - bm * a.qm.regions;
    const int b = bm / a.kv, m = bm - b * a.kv;
    const int col = lane & 31, h = lane >> 5, r = row0 + col;

    // this lane's row.  With dropout dP is used without the factor 1 / keep of the weights that are kept, and D divided by it:
    // keep (dP - D / keep); what is summed of it is multiplied at the end
    const float keep = DROP ? a.rnd.scale : 1.0f;
    Operand<T, D> q, g;
    long long out_at;
    float row_lse, D0, D1 = 0.0f;
    {
        int vh, vw;
        a.qm.limits(b, vh, vw);
        const int place = a.by_g.of(r), head = m * a.g + r - place * a.g;
        const int px = r < a.R ? a.qm.pixel(i, place, a.qm.H, a.qm.W) : -1;
        const bool ok = r < a.R && a.qm.pixel(i, place, vh, vw) >= 0;
        const long long n_px = (long long)a.qm.H * a.qm.W;
        out_at = px < 0 ? -1 : ((long long)b * n_px + px) * a.heads * a.d + head * a.d;
        const long long at = ok ? b * a.os.image + px * a.os.pixel + head * a.hd : 0;
        load_operand<T, D, VEC>(q, (const T*)a.q + b * a.qs.image + (ok ? px * a.qs.pixel + head * a.hd : 0), ok, a.dl, h);
        load_operand<T, D, VEC>(g, (const T*)f.dout + at, ok, a.dl, h);
        Operand<T, D> o;
        load_operand<T, D, VEC>(o, (const T*)f.out + at, ok, a.dl, h);
        float s = 0.0f;
#pragma unroll
        for (int u = 0; u < (int)(sizeof(o) / 16); ++u)
            s += piece_dot<T>(__builtin_bit_cast(u4, o.v[u]), __builtin_bit_cast(u4, g.v[u]));
        D0 = halves_sum(s) / keep;
        const float l = ok ? f.lse[((long long)b * a.heads + head) * n_px + px] : -INFINITY;
        row_lse = l == -INFINITY ? INFINITY : l * LOG2E;
    }
    const uint32_t call = DROP ? a.rnd.call() : 0;
    const float c2 = a.scale * LOG2E;
    constexpr int NA = FIX ? 2 : 1;
    f16v acc[NA][D / 32];           // sums of dS k, then of P k
#pragma unroll
    for (int n = 0; n < NA; ++n)
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt) acc[n][dt] = f16v{};

    const T* kp = (const T*)a.k + b * a.ks.image + m * a.hd;
    const T* vp = (const T*)a.v + b * a.vs.image + m * a.hd;
    Walk walk;
    walk.list = a.index + (long long)group * a.T;
    a.km.limits(b, walk.vh, walk.vw);
    int first = 0, slots = walk.length(a);
    if (SPLIT) {
        const int tiles = (slots + 31) / 32;
        first = tiles * wave / 4 * 32;
        slots = min(slots, tiles * (wave + 1) / 4 * 32);
    }
    Rows<T, D> kn, vn;
    int region = walk.look(a, first + col, slots);
    uint32_t next_word = 0, next_ok;
    auto fetch = [&]() {
        const int px = Walk::pixel(a, region, walk.place, walk.vh, walk.vw);
        next_ok = (uint32_t)__ballot(px >= 0);
        if (DROP) next_word = (uint32_t)region * a.quads + (walk.place >> 2);
        kn.template load<VEC>(kp, row_offset<VEC, T>(px, a.ks.pixel, 0), a.dl, lane);
        vn.template load<VEC>(vp, row_offset<VEC, T>(px, a.vs.pixel, 0), a.dl, lane);
    };
    fetch();
    region = walk.look(a, first + 32 + col, slots);
    for (int x = first; x < slots; x += 32) {
        const uint32_t ok = next_ok, word = next_word;
        wave_order();
        kn.stage(tile_k, ok, a.dl, lane);
        vn.stage(tile_v, ok, a.dl, lane);
        wave_order();
        fetch();
        region = walk.look(a, x + 64 + col, slots);
        if (ok == 0) continue;
        Operand<T, D> k, v;
        read_operand<D>(k, tile_k, lane);
        read_operand<D>(v, tile_v, lane);
        f16v s = dot<D>(k, q, f16v{});
        f16v p = dot<D>(v, g, f16v{});              // dP
        if (ok != 0xffffffffu) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (!((ok >> acc_row(r, 0)) >> (4 * h) & 1)) s[r] = -INFINITY;
        }
        if (DROP) {
            uint32_t words[4][2];
            row_keep(a.rnd, call, word, (uint32_t)i * a.pairs + (r >> 1), bm, words);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                p[r] = (words[r >> 2][(r & 3) >> 1] >> (16 * (r & 1)) & 0xffffu) < a.rnd.threshold ? 0.0f : p[r];
        }
        f16v ds;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c2, -row_lse));
            if (FIX) D1 = __builtin_fmaf(s[r], p[r], D1);
            ds[r] = s[r] * (p[r] - D0);
        }
        Weights<T> w[NA];
        w[0].set(ds);
        if (FIX) w[NA - 1].set(s);
        accumulate<D, NA>(acc, tile_k, w, lane);
    }

    float exact = FIX ? halves_sum(D1) : D0;
    float* sums = (float*)lds;                      // SPLIT: [wave][D][32], then the waves' parts of D
    if constexpr (SPLIT) {
        __syncthreads();                            // (the tiles are in the same place)
        if (FIX) {
            float* D_of = sums + 4 * D * 32;
            if (h == 0) D_of[wave * 32 + col] = exact;
            __syncthreads();
            exact = (D_of[col] + D_of[32 + col]) + (D_of[64 + col] + D_of[96 + col]);
        }
    }
    const float fix = exact - D0;
    if (h == 0 && (!SPLIT || wave == 0)) {
        const long long at = (long long)group * f.row_tiles * 32 + r;
        f.row_lse[at] = row_lse;
        f.row_D[at] = row_lse != INFINITY ? exact : 0.0f;        // (keys may hold anything)
    }
    const bool valid = row_lse != INFINITY;
    const float up = a.scale * keep;
    if (FIX) {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int u = 0; u < 16; ++u) acc[0][dt][u] = __builtin_fmaf(-fix, acc[NA - 1][dt][u], acc[0][dt][u]);
    }
    if constexpr (SPLIT) {
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int u = 0; u < 16; ++u) sums[(wave * D + 32 * dt + acc_row(u, h)) * 32 + col] = acc[0][dt][u];
        __syncthreads();
        if (out_at < 0) return;
        for (int c = 4 * (threadIdx.x >> 5); c < D; c += 32) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float* s = sums + (c + e) * 32 + col;
                x[e] = (s[0] + s[D * 32]) + (s[2 * D * 32] + s[3 * D * 32]);
                x[e] = valid ? x[e] * up : 0.0f;
            }
            store4((T*)f.dq + out_at + c, x, a.d - c, f.vec_dq);
        }
    } else {
        if (out_at < 0) return;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int u = 0; u < 16; u += 4) {
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = valid ? acc[0][dt][u + e] * up : 0.0f;
                const int c = 32 * dt + acc_row(u, h);
                store4((T*)f.dq + out_at + c, x, a.d - c, f.vec_dq);
            }
    }
}

// The lists turned around: a wave per region of keys, or sixteen, each over its part, per N regions where the lists are long, go over
// all entries of their image and head, first counting, then writing in order.  So the time grows with entries times regions.
template <int N>
__global__ __launch_bounds__(1024) void region_invert_kernel(BwdArgs f, int first_block)
{
    const Args& a = f.a;
    __shared__ int less_of[16], mine_of[16][N];
    const int lane = threadIdx.x & 63, J = a.km.regions, units = (J + N - 1) / N;
    const int waves = f.invert_waves, wave = (threadIdx.x >> 6) & (waves - 1), base = (threadIdx.x >> 6) - wave;
    const long long block = (long long)blockIdx.x + first_block, id = waves == 1 ? block * 4 + base : block;
    const bool live = id < (long long)a.B * a.kv * units;
    const int bm = live ? (int)(id / units) : 0, j = live ? (int)(id - (long long)bm * units) * N : 0;
    const int* list = a.index + (long long)bm * f.entries;
    const int run = (f.entries + 64 * waves - 1) / (64 * waves) * 64;
    const int first = min(wave * run, f.entries), end = live ? min(first + run, f.entries) : 0;
    int less = 0, mine[N] = {};
#pragma unroll 8
    for (int e = first + lane; e < end; e += 64) {
        const int x = list[e];
        less += (uint32_t)x < (uint32_t)j;
#pragma unroll
        for (int n = 0; n < N; ++n) mine[n] += x == j + n;
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
        less += __shfl_xor(less, s);
#pragma unroll
        for (int n = 0; n < N; ++n) mine[n] += __shfl_xor(mine[n], s);
    }
    if (lane == 0) {
        less_of[base + wave] = less;
#pragma unroll
        for (int n = 0; n < N; ++n) mine_of[base + wave][n] = mine[n];
    }
    __syncthreads();
    if (!live) return;
    int at = 0, hits = 0;
    int2* to[N];
    for (int w = 0; w < waves; ++w) at += less_of[base + w];
    int* start = f.start + (long long)bm * (J + 1);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (wave == 0 && lane == 0 && j + n < J) start[j + n] = at;
        int before = 0, all = 0;
        for (int w = 0; w < waves; ++w) {
            before += w < wave ? mine_of[base + w][n] : 0;
            all += mine_of[base + w][n];
        }
        to[n] = f.sorted + (long long)bm * f.entries + at + before;
        if (j + n < J) { at += all; hits += mine[n]; }
    }
    if (wave == 0 && lane == 0 && j + N >= J) start[J] = at;
    if (hits == 0) return;
    const int last = min(j + N, J);
#pragma unroll 4
    for (int e0 = first; e0 < end; e0 += 64) {
        const int e = e0 + lane, x = e < end ? list[e] : -1;
        if (!__ballot(x >= j && x < last)) continue;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const bool hit = x == j + n && j + n < last;
            const uint64_t mask = __ballot(hit);
            if (hit) to[n][__popcll(mask & ((1ull << lane) - 1))] = int2{e / a.T, x};
            to[n] += __popcll(mask);
        }
    }
}

// Random bits seen from a key (lane) and 16 rows (registers): a patch of 4 keys and 2 rows is four lanes wide, so each of four lanes makes two
// of their eight evaluations.  pair: the counter word of the pair that row lane % 32 is one of.
// Returns for row pair p (registers 2 p, 2 p + 1) the two words that hold this lane's keys.
__device__ __forceinline__ void key_keep(const Random& rnd, uint32_t call, uint32_t quad, uint32_t pair, int h, uint32_t bm, uint32_t (&words)[8][2])
{
    const int k = threadIdx.x & 3;
    Words x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int p = 4 * u + k, row = 8 * (p >> 1) + 4 * h + 2 * (p & 1);      // rows acc_row(2 p, h) and the next
        x[u] = philox(quad, (uint32_t)__builtin_amdgcn_ds_bpermute(4 * row, (int)pair), bm, call, rnd.key0, rnd.key1);
    }
    auto from = [&](auto lane4, uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp(v, decltype(lane4)::value * 0x55, 0xf, 0xf, true); };
    auto pairs = [&](auto lane4) {
        constexpr int p = decltype(lane4)::value;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t lo = from(lane4, x[u].w[2 * e]), hi = from(lane4, x[u].w[2 * e + 1]);
                words[4 * u + p][e] = k & 2 ? hi : lo;
            }
    };
    pairs(std::integral_constant<int, 0>{}); pairs(std::integral_constant<int, 1>{});
    pairs(std::integral_constant<int, 2>{}); pairs(std::integral_constant<int, 3>{});
}

// dk and dv of 32 keys of a region, by one wave or a team of four that divide the entries among them and add their sums in LDS.
template <typename T, int D, bool DROP, int TEAM, bool VEC>
__global__ __launch_bounds__(64 * TEAM, sizeof(T) == 2 && D <= 64 ? (D == 32 ? 3 : 2) : 1) void region_dkdv_kernel(BwdArgs f)
{
    const Args& a = f.a;
    extern __shared__ __align__(16) unsigned char lds[];
    const int lane = threadIdx.x & 63, wave = TEAM == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    unsigned char* tile_q = lds + wave * (2 * Tile<T, D>::BYTES + 256);
    unsigned char* tile_g = tile_q + Tile<T, D>::BYTES;
    float* stat = (float*)(tile_g + Tile<T, D>::BYTES);        // lse, then D, of 32 rows
    const int J = a.km.regions, col = lane & 31, h = lane >> 5;

    // this block's work: the first `share` entries of a region, or, behind all of those, the entries of a window that lie beyond.
    // (Each part is spread over the XCDs: there is little to do in the second.)
    const int firsts = a.B * a.kv * J * f.key_tiles;
    const bool beyond = (int)blockIdx.x >= firsts;
    int unit = beyond ? (int)xcd_order(blockIdx.x - firsts, gridDim.x - firsts) : (int)xcd_order(blockIdx.x, firsts);
    const int kt = unit % f.key_tiles;
    unit /= f.key_tiles;
    const int units = beyond ? f.windows : J, bm = unit / units;
    unit -= bm * units;
    const int b = bm / a.kv, m = bm - b * a.kv;
    const int* start = f.start + (long long)bm * (J + 1);
    const int2* sorted = f.sorted + (long long)bm * f.entries;
    int j = unit, from, to, slot = -1;
    if (!beyond) {
        from = start[j];
        const int end = start[j + 1];
        to = min(end, from + f.share);
        if (end > to) slot = 2 * (from / f.share);
    } else {
        const int window = unit;
        if ((long long)window * f.share >= start[J]) return;
        j = sorted[window * f.share].y;
        from = max(window * f.share, start[j] + f.share);
        to = min(start[j + 1], (window + 1) * f.share);
        if (from >= to) return;
        slot = 2 * window + 1;
    }
    j = __builtin_amdgcn_readfirstlane(j); from = __builtin_amdgcn_readfirstlane(from); to = __builtin_amdgcn_readfirstlane(to);
    slot = __builtin_amdgcn_readfirstlane(slot);
    if (TEAM > 1) {
        const int n = to - from, mine = (int)((long long)n * wave / TEAM);
        to = from + (int)((long long)n * (wave + 1) / TEAM);
        from += mine;
    }

    Operand<T, D> k, v;
    long long out_at;
    bool valid;
    uint32_t quad;
    {
        int vh, vw;
        a.km.limits(b, vh, vw);
        const int place = kt * 32 + col;
        const int px = place < a.km.places ? a.km.pixel(j, place, a.km.H, a.km.W) : -1;
        valid = place < a.km.places && a.km.pixel(j, place, vh, vw) >= 0;
        out_at = px < 0 ? -1 : ((long long)b * a.km.H * a.km.W + px) * a.kv * a.d + m * a.d;
        quad = (uint32_t)j * a.quads + (place >> 2);
        const long long at = valid ? px : 0;
        load_operand<T, D, VEC>(k, (const T*)a.k + b * a.ks.image + at * a.ks.pixel + m * a.hd, valid, a.dl, h);
        load_operand<T, D, VEC>(v, (const T*)a.v + b * a.vs.image + at * a.vs.pixel + m * a.hd, valid, a.dl, h);
    }
    const uint32_t call = DROP ? a.rnd.call() : 0;
    const float c2 = a.scale * LOG2E, keep = DROP ? a.rnd.scale : 1.0f;         // (as in the row kernel, row_D is divided by it)
    f16v dk[1][D / 32], dv[1][D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) { dk[0][dt] = f16v{}; dv[0][dt] = f16v{}; }

    int qh, qw;
    a.qm.limits(b, qh, qw);
    const long long n_px = (long long)a.qm.H * a.qm.W;
    Rows<T, D> q, g;
    float st;
    uint32_t next_ok = 0;
    const T* qp = (const T*)a.q + b * a.qs.image;
    const T* gp = (const T*)f.dout + b * a.os.image;
    // The rows of the groups one after the other, each group's padded to whole pairs (a patch of the dropout counter): slot y is row
    // y % (2 pairs) of the group of entry from + y / (2 pairs), and a tile holds rows of several groups.
    int entries = to - from;
    if (a.qm.size) {
        // Nothing to do where every group lies outside its image.  (A row that does not count is zeros with a weight of zero, which is nothing
        // unless a key is not finite; such a key's gradients are not finite either where rows that count attend it.)
        bool any = false;
        for (int e = lane; e - lane < entries && !any; e += 64)
            any = __ballot(a.qm.pixel(sorted[from + min(e, entries - 1)].x, 0, qh, qw) >= 0);
        entries = any ? entries : 0;
    }
    const int steps = (entries * (2 * a.pairs) + 31) / 32;
    int row = 0;                                // this lane's row of the tile that is loaded next, its entry in bounds or not
    bool there = false;
    uint32_t next_pair = 0, pair;
    auto look = [&](int s) {
        const int y = 32 * s + col, e = f.by_rows.of(y);
        row = y - e * (2 * a.pairs);
        there = e < entries && row < a.R;
        return sorted[from + min(e, entries - 1)].x;
    };
    const float* rows_of_image = (h ? f.row_D : f.row_lse) + (long long)bm * a.qm.regions * f.row_tiles * 32;
    auto fetch = [&](int i) {
        const int r = there ? row : 0;
        const int place = a.by_g.of(r), head = m * a.g + r - place * a.g;
        const int at = a.qm.pixel(i, place, qh, qw), px = there ? at : -1;
        next_ok = (uint32_t)__ballot(px >= 0);
        q.template load<VEC>(qp, row_offset<VEC, T>(px, a.qs.pixel, head * a.hd), a.dl, lane);
        g.template load<VEC>(gp, row_offset<VEC, T>(px, a.os.pixel, head * a.hd), a.dl, lane);
        const float x = rows_of_image[i * (f.row_tiles * 32) + r];
        st = there ? x : h ? 0.0f : INFINITY;
        if (DROP) next_pair = (uint32_t)i * a.pairs + (r >> 1);
    };
    int next = 0;
    if (steps > 0) {
        next = look(0);
        fetch(next);
        next = look(1);
    }
    for (int s = 0; s < steps; ++s) {
        wave_order();
        q.stage(tile_q, next_ok, a.dl, lane);
        g.stage(tile_g, next_ok, a.dl, lane);
        stat[lane] = st;
        wave_order();
        pair = next_pair;
        fetch(next);                            // (zeros' worth of rows behind the end)
        next = look(s + 2);
        Operand<T, D> qc, gc;
        read_operand<D>(qc, tile_q, lane);
        read_operand<D>(gc, tile_g, lane);
        float lse[16], Dr[16];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const f4 x = *(const f4*)(stat + acc_row(4 * u, h)), y = *(const f4*)(stat + 32 + acc_row(4 * u, h));
#pragma unroll
            for (int e = 0; e < 4; ++e) { lse[4 * u + e] = x[e]; Dr[4 * u + e] = y[e]; }
        }
        f16v p = dot<D>(qc, k, f16v{});
        f16v ds = dot<D>(gc, v, f16v{});            // dP
        uint32_t words[8][2];
        if (DROP) {
            key_keep(a.rnd, call, quad, pair, h, bm, words);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                ds[r] = (words[r >> 1][r & 1] >> (16 * (lane & 1)) & 0xffffu) < a.rnd.threshold ? 0.0f : ds[r];
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], c2, -lse[r]));
            ds[r] = p[r] * (ds[r] - Dr[r]);
            if (DROP) p[r] = (words[r >> 1][r & 1] >> (16 * (lane & 1)) & 0xffffu) < a.rnd.threshold ? 0.0f : p[r];
        }
        Weights<T> wk[1], wv[1];
        wv[0].set(p);
        wk[0].set(ds);
        accumulate<D, 1>(dv, tile_g, wv, lane);
        accumulate<D, 1>(dk, tile_q, wk, lane);
    }

    if constexpr (TEAM > 1) {
        // waves 2 and 3 hand their sums to 0 and 1, then 1 to 0; a lane's registers stay its own
        static_assert(TEAM == 4, "two rounds");
        float* room = (float*)lds + lane;
        constexpr int N = 2 * (D / 32) * 16;
#pragma unroll
        for (int half = 2; half > 0; half >>= 1) {
            __syncthreads();
            float* to_lds = room + (wave & (half - 1)) * N * 64;
            if (wave >= half && wave < 2 * half) {
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        to_lds[(dt * 32 + r) * 64] = dk[0][dt][r];
                        to_lds[(dt * 32 + 16 + r) * 64] = dv[0][dt][r];
                    }
            }
            __syncthreads();
            if (wave < half) {
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        dk[0][dt][r] += to_lds[(dt * 32 + r) * 64];
                        dv[0][dt][r] += to_lds[(dt * 32 + 16 + r) * 64];
                    }
            }
        }
        if (wave > 0) return;
    }
    float* part = f.partial + (((long long)bm * f.key_tiles + kt) * 2 * f.windows + max(slot, 0)) * (2 * 32 * D);
    const float up = a.scale * keep;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int u = 0; u < 16; u += 4) {
            const int c = 32 * dt + acc_row(u, h);
            float x[4], y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = valid ? dk[0][dt][u + e] * up : 0.0f;
                y[e] = valid ? dv[0][dt][u + e] * keep : 0.0f;
            }
            if (slot >= 0) {
                float* p = part + col * D + c;
                *(f4*)p = f4{x[0], x[1], x[2], x[3]};
                *(f4*)(p + 32 * D) = f4{y[0], y[1], y[2], y[3]};
            } else if (out_at >= 0) {
                store4((T*)f.dk + out_at + c, x, a.d - c, f.vec_dk);
                store4((T*)f.dv + out_at + c, y, a.d - c, f.vec_dk);
            }
        }
}

// The regions that more than `share` groups list: adds up the float32 sums of their waves, in order; twice four channels of a key a thread.
template <typename T, int D>
__global__ __launch_bounds__(256) void region_dkdv_join_kernel(BwdArgs f)
{
    const Args& a = f.a;
    const int J = a.km.regions;
    const int window = blockIdx.x % f.windows, kt = blockIdx.x / f.windows % f.key_tiles, bm = blockIdx.x / f.windows / f.key_tiles;
    const int b = bm / a.kv, m = bm - b * a.kv;
    const int* start = f.start + (long long)bm * (J + 1);
    // a region whose first wave wrote to this window reaches into the next one
    if ((long long)(window + 1) * f.share >= start[J]) return;
    const int j = f.sorted[(long long)bm * f.entries + (window + 1) * f.share].y;
    const int s = start[j], e = start[j + 1];
    if (s / f.share != window || e - s <= f.share) return;
    const float* part = f.partial + ((long long)bm * f.key_tiles + kt) * 2 * f.windows * (2 * 32 * D);
    const int last = (e - 1) / f.share;
#pragma unroll
    for (int u = blockIdx.y * 512 + threadIdx.x, n = 0; n < 2; ++n, u += 256) {
        const int c = 4 * u % D, place = kt * 32 + 4 * u / D % 32, side = 4 * u / D / 32;
        const int px = place < a.km.places ? a.km.pixel(j, place, a.km.H, a.km.W) : -1;
        if (px < 0) continue;
        f4 sum = *(const f4*)(part + (long long)(2 * window) * (2 * 32 * D) + 4 * u);
#pragma unroll 4
        for (int w = (s + f.share) / f.share; w <= last; ++w) sum += *(const f4*)(part + (long long)(2 * w + 1) * (2 * 32 * D) + 4 * u);
        const float x[4] = {sum[0], sum[1], sum[2], sum[3]};
        store4((T*)(side ? f.dv : f.dk) + ((long long)b * a.km.H * a.km.W + px) * a.kv * a.d + m * a.d + c, x, a.d - c, f.vec_dk);
    }
}

static int padded(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }

// sizes that the workspace and the launches share
static void plan(BwdArgs& f)
{
    const Args& a = f.a;
    f.slots = 4 * a.quads * a.T;
    f.row_tiles = (a.R + 31) / 32;
    const long long slots = 2ll * a.pairs;
    f.by_rows = Div::by((uint32_t)slots);
    f.key_tiles = (a.km.places + 31) / 32;
    f.entries = a.qm.regions * a.T;
    // Four waves per tile of keys where a region has 24 row tiles or more on average (16384 tokens, 128 row tiles per region: 155
    // against 218 us); with few, as at stage 1 (8), the joining costs more than the finer division gives.
    const long long average = ((long long)f.entries + a.km.regions - 1) / a.km.regions;
    // (With 2^22 tiles the chip is full anyway, and the grid's threads stay below 2^32.)
    f.team = average * slots >= 24 * 32 && (long long)a.B * a.kv * a.km.regions * f.key_tiles < 1 << 22 ? 4 : 1;
    // A block's share: twice what a region has on average, at least 8 row tiles; less where there would be too few waves for the chip, but
    // four row tiles, for less costs more in sums that are written and joined than it gains (28 x 46, regions of 13 x 5, heads of 128:
    // 74 us with one entry a block, 45 so; float32, 38 x 53: 289 and 181), and heads of 128, of which a SIMD holds one wave, fill the chip with fewer.
    const long long all = (long long)a.B * a.kv * f.key_tiles * f.entries * f.team;
    const long long fill = std::max({(long long)f.team, all / ((a.d > 64 ? 4ll : 16ll) * device_cu_count()), (4 * 32 * f.team + slots - 1) / slots});
    f.share = (int)std::min({std::max(2 * average, (8 * 32 + slots - 1) / slots), fill, (1ll << 30) / slots});
    f.windows = (f.entries + f.share - 1) / f.share;
}

struct Room { size_t lse, D, sorted, start, partial, end; };

static Room room(const BwdArgs& f)
{
    const Args& a = f.a;
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t bm = (size_t)a.B * a.kv, rows = bm * a.qm.regions * f.row_tiles * 32 * sizeof(float);
    Room r;
    r.lse = 0;
    r.D = up(rows);
    r.sorted = r.D + up(rows);
    r.start = r.sorted + up(bm * f.entries * sizeof(int2));
    r.partial = r.start + up(bm * (a.km.regions + 1) * sizeof(int));
    r.end = r.partial + bm * f.key_tiles * 2 * f.windows * (2 * 32 * padded(a.d)) * sizeof(float);
    return r;
}

size_t bwd_workspace_bytes(const Args& a)
{
    BwdArgs f{};
    f.a = a;
    plan(f);
    return packing(a, true).end + room(f).end;
}

template <typename T, int D>
static hipError_t run_rows(BwdArgs& f, hipStream_t st)
{
    f.items = f.a.B * f.a.kv * f.a.qm.regions * f.row_tiles;
    // SPLIT where a wave per 32 rows would not give every SIMD one (50 x 47, 448 waves over 2500 keys: 70 us, split 29), and with
    // heads of 128, of which a SIMD holds one wave, or half of them (704 waves of float32: 67 us, split 111).
    const bool split = f.items < (D == 128 ? 2 : 4) * device_cu_count() && f.slots > 4 * 32;
    const int blocks = split ? f.items : (f.items + 3) / 4, lds = split ? std::max(8 * Tile<T, D>::BYTES, 4 * D * 32 * 4 + 512) : 8 * Tile<T, D>::BYTES;
    static LdsOptIn opt;
    const hipError_t e = opt.ensure({(const void*)region_dq_kernel<T, D, true, false, false>, (const void*)region_dq_kernel<T, D, true, false, true>,
                                     (const void*)region_dq_kernel<T, D, false, false, true>, (const void*)region_dq_kernel<T, D, true, true, false>,
                                     (const void*)region_dq_kernel<T, D, true, true, true>, (const void*)region_dq_kernel<T, D, false, true, true>},
                                    std::max(8 * Tile<T, D>::BYTES, 4 * D * 32 * 4 + 512));
    if (e != hipSuccess) return e;
    // (what is not in whole pieces takes the kernels with dropout, which drop nothing below a threshold of 0)
    const auto kernel = !f.vec ? (split ? region_dq_kernel<T, D, true, true, false> : region_dq_kernel<T, D, true, false, false>)
                      : f.a.rnd.threshold ? (split ? region_dq_kernel<T, D, true, true, true> : region_dq_kernel<T, D, true, false, true>)
                                          : (split ? region_dq_kernel<T, D, false, true, true> : region_dq_kernel<T, D, false, false, true>);
    kernel<<<blocks, 256, lds, st>>>(f);
    return hipGetLastError();
}

template <typename T, int D>
static hipError_t run_keys(BwdArgs& f, hipStream_t st)
{
    const long long items = (long long)f.a.B * f.a.kv * f.key_tiles * (f.a.km.regions + f.windows);
    const int one = 2 * Tile<T, D>::BYTES + 256, lds = f.team == 1 ? one : std::max(4 * one, 2 * 2 * D * 32 * 4);
    static LdsOptIn opt;
    hipError_t e = opt.ensure({(const void*)region_dkdv_kernel<T, D, true, 4, true>, (const void*)region_dkdv_kernel<T, D, false, 4, true>,
                               (const void*)region_dkdv_kernel<T, D, true, 4, false>}, 4 * one);
    if (e != hipSuccess) return e;
    const bool team = f.team > 1;
    const auto kernel = !f.vec ? (team ? region_dkdv_kernel<T, D, true, 4, false> : region_dkdv_kernel<T, D, true, 1, false>)
                      : f.a.rnd.threshold ? (team ? region_dkdv_kernel<T, D, true, 4, true> : region_dkdv_kernel<T, D, true, 1, true>)
                                          : (team ? region_dkdv_kernel<T, D, false, 4, true> : region_dkdv_kernel<T, D, false, 1, true>);
    kernel<<<(int)items, 64 * f.team, lds, st>>>(f);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (f.entries > f.share) {
        region_dkdv_join_kernel<T, D><<<dim3(f.a.B * f.a.kv * f.key_tiles * f.windows, D / 32), 256, 0, st>>>(f);
        e = hipGetLastError();
    }
    return e;
}

template <typename T>
static hipError_t run_t(BwdArgs& f, unsigned char* ws, hipStream_t st)
{
    const Args& a = f.a;
    const Packing copies = packing(a, true);
    hipError_t e;
    if (copies.on && (e = pack<T>(f.a, copies, &f.dout, &f.out, ws, st)) != hipSuccess) return e;
    ws += copies.end;
    const long long nq = (long long)a.qm.H * a.qm.W, nk = (long long)a.km.H * a.km.W;
    f.vec = pieces(a.q, a.qs, a.dl, sizeof(T), nq) && pieces(a.k, a.ks, a.dl, sizeof(T), nk) && pieces(a.v, a.vs, a.dl, sizeof(T), nk) &&
            pieces(f.dout, a.os, a.dl, sizeof(T), nq) && pieces(f.out, a.os, a.dl, sizeof(T), nq);
    plan(f);
    const Room r = room(f);
    f.row_lse = (float*)(ws + r.lse); f.row_D = (float*)(ws + r.D); f.sorted = (int2*)(ws + r.sorted);
    f.start = (int*)(ws + r.start); f.partial = (float*)(ws + r.partial);
    const uintptr_t quad = 4 * sizeof(T) - 1;
    f.vec_dq = a.d % 4 == 0 && ((uintptr_t)f.dq & quad) == 0;
    f.vec_dk = a.d % 4 == 0 && ((uintptr_t)f.dk & quad) == 0 && ((uintptr_t)f.dv & quad) == 0;
    e = a.d <= 32 ? run_rows<T, 32>(f, st) : a.d <= 64 ? run_rows<T, 64>(f, st) : run_rows<T, 128>(f, st);
    if (e != hipSuccess) return e;
    // (196 entries: 5.5 us by one wave, 8.3 by four; 16384: 109 by one, 19 by four, 12 by sixteen)
    f.invert_waves = f.entries >= 2048 ? 16 : 1;
    const int lists = a.B * a.kv, regions = lists * a.km.regions;
    // Four regions a block where that still fills the chip (8262 regions: 77 us by one, 46 by four; 312: 9.5 and 14).
    if (f.invert_waves == 1) region_invert_kernel<1><<<(regions + 3) / 4, 256, 0, st>>>(f, 0);
    else if (regions < 4 * device_cu_count()) region_invert_kernel<1><<<regions, 1024, 0, st>>>(f, 0);
    else e = in_launches((long long)lists * ((a.km.regions + 3) / 4), 1024, [&](unsigned blocks, int first) {
        region_invert_kernel<4><<<blocks, 1024, 0, st>>>(f, first);
    });
    if (e != hipSuccess || (e = hipGetLastError()) != hipSuccess) return e;
    return a.d <= 32 ? run_keys<T, 32>(f, st) : a.d <= 64 ? run_keys<T, 64>(f, st) : run_keys<T, 128>(f, st);
}

hipError_t launch_bwd(const Args& a, const void* dout, const void* out, const float* lse, void* dq, void* dk, void* dv,
                      void* workspace, hipStream_t st)
{
    BwdArgs f{};
    f.a = a; f.dout = dout; f.out = out; f.lse = lse; f.dq = dq; f.dk = dk; f.dv = dv;
    return a.dtype == 0 ? run_t<float>(f, (unsigned char*)workspace, st) : run_t<bf16_bits>(f, (unsigned char*)workspace, st);
}

}  // namespace region
}  // namespace slide
