// Pieces of the matrix-core kernels of region attention (slide_region_fwd.hip, slide_region_bwd.hip).
//
// Tiles are 32 x 32.  bf16: v_mfma_f32_32x32x16_bf16, a lane holding 8 consecutive elements of the contracted axis; float32:
// v_mfma_f32_32x32x2_f32, a lane holding one.  A product's result has column lane % 32 and, in register r, row
// 8 (r / 4) + 4 (lane / 32) + r % 4.  A result that becomes the right operand of the next product (weights, logit gradients) stays in
// its registers: the contracted axis may be numbered as one likes as long as the left operand follows, so slot e of a lane in
// step t is the row that register 8 t + e holds.  The left operand of that product is the transpose of a staged tile
// (keys x channels): bf16 by the transposing LDS read, float32 by reading a column.
#pragma once
#include "slide_region.h"

namespace slide {
namespace region {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef short short4_t __attribute__((ext_vector_type(4)));

typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));

// two floats rounded to bf16 (to nearest, ties to even) in one dword: one instruction
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, bf2)); }

// row that register r of a product's result is in lane half h
__device__ __forceinline__ constexpr int acc_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// The registers of an operand with D contracted channels (or 32 contracted rows), per lane
template <typename T, int D> struct Operand;
template <int D> struct Operand<bf16_bits, D> { u4 v[D / 16]; };
template <int D> struct Operand<float, D> { f4 v[D / 8]; };

// Memory piece i (16 bytes) of an operand's lane half h starts at this channel
template <typename T, int D> __device__ __forceinline__ constexpr int piece_channel(int i, int h)
{
    return sizeof(T) == 2 ? 16 * i + 8 * h : h * (D / 2) + 4 * i;
}

// One 16-byte piece of a pixel's channels, element by element, zeros beyond `left` channels
__device__ __forceinline__ u4 gather_piece(const bf16_bits* p, int left)
{
    u4 x = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < left) x[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
    return x;
}
__device__ __forceinline__ f4 gather_piece(const float* p, int left)
{
    f4 x = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) x[e] = p[e];
    return x;
}

// The operand whose lane is one pixel's channels at p; zeros where the pixel does not count, and beyond its d channels.
// VEC: the pieces are whole and 16-byte aligned; where, as mostly, nothing is to be left out, the loads follow each other without a test.
template <typename T, int D, bool VEC>
__device__ __forceinline__ void load_operand(Operand<T, D>& o, const T* p, bool ok, int d, int h)
{
    typedef decltype(gather_piece(p, 0)) Piece;
    constexpr int N = sizeof(T) == 2 ? D / 16 : D / 8;
    if constexpr (VEC) {
        if (d == D && __ballot(ok) == ~0ull) {
#pragma unroll
            for (int i = 0; i < N; ++i) o.v[i] = *(const Piece*)(p + piece_channel<T, D>(i, h));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) o.v[i] = Piece{0, 0, 0, 0};
            if (ok) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (piece_channel<T, D>(i, h) < d) o.v[i] = *(const Piece*)(p + piece_channel<T, D>(i, h));
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = piece_channel<T, D>(i, h);
            o.v[i] = gather_piece(p + c, ok ? d - c : 0);
        }
    }
}

// acc += A^T B over the D channels of two operands (rows: A's lanes, columns: B's lanes)
template <int D>
__device__ __forceinline__ f16v dot(const Operand<bf16_bits, D>& a, const Operand<bf16_bits, D>& b, f16v acc)
{
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a.v[i]), __builtin_bit_cast(bf8, b.v[i]), acc, 0, 0, 0);
    return acc;
}
template <int D>
__device__ __forceinline__ f16v dot(const Operand<float, D>& a, const Operand<float, D>& b, f16v acc)
{
#pragma unroll
    for (int i = 0; i < D / 2; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[i >> 2][i & 3], b.v[i >> 2][i & 3], acc, 0, 0, 0);
    return acc;
}

// A tile of 32 pixels x D channels in LDS that this wave alone uses.  The 16-byte pieces of a row are exchanged by a number that the
// row gives, so that neither eight rows' reads of one piece nor a transposing read of four rows meet in a bank.
template <typename T, int D> struct Tile {
    static constexpr int BYTES = 32 * D * (int)sizeof(T);
    static __device__ __forceinline__ int exchange(int row)
    {
        if constexpr (sizeof(T) == 4) return row & 7;
        else if constexpr (D == 32) return (row & 2) | ((row >> 2) & 1);        // (two rows in 128 bytes)
        else return 2 * (row & 3) | ((row >> 2) & 1);
    }
    // byte of piece c of a row
    static __device__ __forceinline__ int at(int row, int c) { return row * D * (int)sizeof(T) + ((c ^ exchange(row)) << 4); }
};

// Where a row of a tile begins: in 16-byte pieces if the tensor is made of whole pieces (VEC), else in elements
template <bool VEC> struct Offset { typedef uint32_t type; };
template <> struct Offset<false> { typedef long long type; };

// ... of pixel px; of pixel 0 for a row that does not count (which is read all the same, and left out on its way to the tile)
template <bool VEC, typename T>
__device__ __forceinline__ typename Offset<VEC>::type row_offset(int px, long long pixel_stride, int channel)
{
    if constexpr (VEC) return (uint32_t)max(px, 0) * (uint32_t)(pixel_stride * (int)sizeof(T) >> 4) + (uint32_t)(channel * (int)sizeof(T) >> 4);
    else return max(px, 0) * pixel_stride + channel;
}

// 32 rows of D channels on their way from memory to a tile.  Consecutive lanes take consecutive pieces of a row: a load in which every lane
// has a row of its own takes the vector cache four times as long (59 against 16 accesses; 16384 tokens: dq 146 against 118 us).
// Loading makes no decision, so that it can be scheduled into the products; what does not count is set to zero by stage().
template <typename T, int D> struct Rows {
    static constexpr int PER_ROW = D * (int)sizeof(T) / 16, N = 32 * PER_ROW / 64, E = 16 / (int)sizeof(T);
    typedef typename std::conditional<sizeof(T) == 2, u4, f4>::type Piece;
    Piece v[N];

    // at: the offset of row lane % 32
    template <bool VEC>
    __device__ __forceinline__ void load(const T* base, typename Offset<VEC>::type at, int d, int lane)
    {
        const int c = lane % PER_ROW;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (VEC) {
                const uint32_t off = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * ((64 * i + lane) / PER_ROW), (int)at);
                v[i] = ((const Piece*)base)[(uint64_t)off + (c * E < d ? c : 0)];
            } else {
                const long long off = __shfl(at, (64 * i + lane) / PER_ROW);
                v[i] = gather_piece(base + off + c * E, d - c * E);
            }
        }
    }
    // ok: the rows that count, one bit each
    __device__ __forceinline__ void stage(unsigned char* tile, uint32_t ok, int d, int lane)
    {
        if (ok != 0xffffffffu || d != D) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (!(ok >> ((64 * i + lane) / PER_ROW) & 1) || lane % PER_ROW * E >= d) v[i] = Piece{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < N; ++i) *(Piece*)(tile + Tile<T, D>::at((64 * i + lane) / PER_ROW, lane % PER_ROW)) = v[i];
    }
};

// The tile as an operand: a lane's row is lane % 32
template <int D>
__device__ __forceinline__ void read_operand(Operand<bf16_bits, D>& o, const unsigned char* tile, int lane)
{
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o.v[i] = *(const u4*)(tile + Tile<bf16_bits, D>::at(lane & 31, 2 * i + (lane >> 5)));
}
template <int D>
__device__ __forceinline__ void read_operand(Operand<float, D>& o, const unsigned char* tile, int lane)
{
#pragma unroll
    for (int i = 0; i < D / 8; ++i) o.v[i] = *(const f4*)(tile + Tile<float, D>::at(lane & 31, (lane >> 5) * (D / 8) + i));
}

// Weights of 32 rows (registers of a product's result) as a right operand
template <typename T> struct Weights;
template <> struct Weights<bf16_bits> {
    u4 v[2];
    // rounded to bf16 (to nearest): the products take no more
    __device__ __forceinline__ void set(const f16v& p)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = pack_bf16(p[2 * i], p[2 * i + 1]);
    }
};
template <> struct Weights<float> {
    f16v v;
    __device__ __forceinline__ void set(const f16v& p) { v = p; }
};

// The transpose of channels 32 dt .. 32 dt + 31 of a tile as a left operand, rows numbered as Weights' slots
template <int D>
__device__ __forceinline__ void read_transposed(u4 (&a)[2], const unsigned char* tile, int dt, int lane)
{
    const int s = lane & 15, h = lane >> 5, dh = (lane >> 4) & 1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned char* p = tile + Tile<bf16_bits, D>::at(8 * i + 4 * h + (s >> 2), 4 * dt + 2 * dh + ((s >> 1) & 1)) + 8 * (s & 1);
        const u2 x = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)p));
        a[i >> 1][2 * (i & 1)] = x[0];
        a[i >> 1][2 * (i & 1) + 1] = x[1];
    }
}

// acc[dt] += (channels x rows of the tile) (rows x columns of w), for NC sets of columns
template <int D, int NC>
__device__ __forceinline__ void accumulate(f16v (&acc)[NC][D / 32], const unsigned char* tile, const Weights<bf16_bits> (&w)[NC], int lane)
{
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
        u4 a[2];
        read_transposed<D>(a, tile, dt, lane);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c)
                acc[c][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a[t]), __builtin_bit_cast(bf8, w[c].v[t]), acc[c][dt], 0, 0, 0);
    }
}
template <int D, int NC>
__device__ __forceinline__ void accumulate(f16v (&acc)[NC][D / 32], const unsigned char* tile, const Weights<float> (&w)[NC], int lane)
{
    const int h = lane >> 5;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float a = *(const float*)(tile + Tile<float, D>::at(acc_row(r, h), 8 * dt + ((lane & 31) >> 2)) + 4 * (lane & 3));
#pragma unroll
            for (int c = 0; c < NC; ++c) acc[c][dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w[c].v[r], acc[c][dt], 0, 0, 0);
        }
}

// LDS operations of a wave run in order; this keeps the compiler from moving them past each other
__device__ __forceinline__ void wave_order() { asm volatile("" ::: "memory"); }

// the larger, the sum, of the two lane halves' values
__device__ __forceinline__ float halves_max(float x)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float halves_sum(float x)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// four consecutive channels c .. c + 3 of a pixel
__device__ __forceinline__ void store4(bf16_bits* p, const float (&x)[4], int left, bool vec)
{
    if (vec) {
        if (left > 0)
            *(u2*)p = u2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = f32_to_bf16(x[e]);
    }
}
__device__ __forceinline__ void store4(float* p, const float (&x)[4], int left, bool vec)
{
    if (vec) {
        if (left > 0) *(f4*)p = f4{x[0], x[1], x[2], x[3]};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = x[e];
    }
}

// The keys of a group: slot x of the concatenated regions -> pixel.
struct Walk {
    const int* list;
    int vh, vw;             // valid height and width of the image
    int entry, place;       // of this lane's slot in the tile that is looked up next
    __device__ __forceinline__ int look(const Args& a, int x, int end)
    {
        entry = a.by_slots.of(x);
        place = x - entry * 4 * a.quads;
        const int j = list[min(entry, a.T - 1)];
        return x < end ? j : -1;
    }
    // slots up to the last entry that is a region: a region of queries outside its image, or in sight of few regions, has a list that ends early
    __device__ __forceinline__ int length(const Args& a) const
    {
        int last = 0;
        for (int t0 = 0; t0 < a.T; t0 += 64) {
            const int t = t0 + (threadIdx.x & 63), j = list[min(t, a.T - 1)];
            const uint64_t regions = __ballot(t < a.T && (uint32_t)j < (uint32_t)a.km.regions);
            if (regions) last = t0 + 64 - __builtin_clzll(regions);
        }
        return last * 4 * a.quads;
    }
    // pixel of (region j, place), -1 if there is none
    static __device__ __forceinline__ int pixel(const Args& a, int j, int place, int vh, int vw)
    {
        const bool listed = (uint32_t)j < (uint32_t)a.km.regions && place < a.km.places;
        const int px = a.km.pixel(listed ? j : 0, listed ? place : 0, vh, vw);
        return listed ? px : -1;
    }
};

// Random bits of the attention weights of one row tile: this lane's row (its pair and parity) and its 16 keys.  word: the counter word of
// the four keys that this lane's key (lane % 32) is one of.  Two rows share an evaluation, so each lane of a pair makes half of them and
// passes on what the other needs.  words[u][e]: elements 4 u + 2 e and the next, in halves.
__device__ __forceinline__ void row_keep(const Random& rnd, uint32_t call, uint32_t word, uint32_t pair, uint32_t bm, uint32_t (&words)[4][2])
{
    const bool odd = threadIdx.x & 1, upper = threadIdx.x & 32;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        // this lane's evaluation: keys 4 lane half + 8 u .. for an even lane, 16 further for an odd one
        const uint32_t e0 = __builtin_amdgcn_readlane(word, 8 * u), e1 = __builtin_amdgcn_readlane(word, 8 * u + 4);
        const uint32_t o0 = __builtin_amdgcn_readlane(word, 8 * u + 16), o1 = __builtin_amdgcn_readlane(word, 8 * u + 20);
        const uint32_t even_quad = upper ? e1 : e0, odd_quad = upper ? o1 : o0;
        const Words x = philox(odd ? odd_quad : even_quad, pair, bm, call, rnd.key0, rnd.key1);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t first = x.w[e], second = x.w[2 + e];             // the even row's words, the odd row's
            const uint32_t mine = odd ? second : first, pass = odd ? first : second;
            const uint32_t got = __builtin_amdgcn_mov_dpp(pass, 0xB1, 0xf, 0xf, true);         // from lane ^ 1
            words[u][e] = odd ? got : mine;
            words[2 + u][e] = odd ? mine : got;
        }
    }
}

// whether the pieces of a tensor's pixels are whole, 16-byte aligned, and counted within an image by 32 bits
inline bool pieces(const void* p, const Strides& s, int d, size_t esz, long long pixels)
{
    const long long n = 16 / esz;
    return ((uintptr_t)p & 15) == 0 && s.pixel % n == 0 && s.image % n == 0 && d % n == 0 && pixels * (s.pixel / n) < (1ll << 32) - 65536;
}

// Copies of q, k, v (dout, out) whose heads are whole pieces, zeros behind d, for head sizes and strides that are not.  One launch; the products'
// kernels then load whole pieces (9 lists of 16 from 204 x 267 pixels, heads of 17: 2190 us without).
struct Copies {
    const void* from[5];
    void* to[5];
    Strides strides[5];
    int heads[5];
    long long pixels[5], first[6];          // of an image; first piece of each tensor in the launch
    int n, d, dp;
};

template <typename T>
static __global__ __launch_bounds__(256) void region_copy_kernel(Copies f)
{
    constexpr int E = 16 / (int)sizeof(T);
    typedef decltype(gather_piece((const T*)nullptr, 0)) Piece;
    const int pieces = f.dp / E;
    for (long long at = (long long)blockIdx.x * 256 + threadIdx.x; at < f.first[f.n]; at += (long long)gridDim.x * 256) {
        int t = 0;
        while (at >= f.first[t + 1]) ++t;
        const long long x = at - f.first[t], head = x / pieces, pixel = head / f.heads[t], b = pixel / f.pixels[t];
        const int c = (int)(x - head * pieces) * E, h = (int)(head - pixel * f.heads[t]);
        const T* from = (const T*)f.from[t] + b * f.strides[t].image + (pixel - b * f.pixels[t]) * f.strides[t].pixel + h * f.d + c;
        ((Piece*)f.to[t])[x] = gather_piece(from, f.d - c);
    }
}

// Whether a call works on copies, and the workspace's bytes for them.  Not where fewer keys are attended than there are (one token over a
// long sequence): then the kernels gather the elements themselves, as they do for tensors that are merely not aligned.
struct Packing { bool on; int dp; size_t bytes[5], end; };

inline Packing packing(const Args& a, bool backward)
{
    const int esz = a.dtype == 0 ? 4 : 2, E = 16 / esz;
    Packing p{};
    p.dp = (a.d + E - 1) / E * E;
    const long long nq = (long long)a.qm.H * a.qm.W, nk = (long long)a.km.H * a.km.W;
    bool whole = a.d % E == 0;
    for (const Strides& s : {a.qs, a.ks, a.vs}) whole = whole && s.pixel % E == 0 && s.image % E == 0;
    const bool often = backward || (long long)a.qm.regions * a.T * a.km.places >= nk;
    const bool small = std::max(nq * a.heads, nk * a.kv) * (p.dp / E) < (1ll << 32) - 65536;
    p.on = !whole && often && small;
    for (int t = 0; t < 5 && p.on; ++t) {
        p.bytes[t] = t >= 3 && !backward ? 0 : ((size_t)a.B * (t == 1 || t == 2 ? nk * a.kv : nq * a.heads) * p.dp * esz + 255) / 256 * 256;
        p.end += p.bytes[t];
    }
    return p;
}

// Makes the copies at ws and has a (dout, out) refer to them
template <typename T>
static hipError_t pack(Args& a, const Packing& p, const void** dout, const void** out, unsigned char* ws, hipStream_t st)
{
    constexpr int E = 16 / (int)sizeof(T);
    Copies f{};
    f.n = dout ? 5 : 3; f.d = a.d; f.dp = p.dp;
    const void* from[5] = {a.q, a.k, a.v, dout ? *dout : nullptr, out ? *out : nullptr};
    Strides* strides[5] = {&a.qs, &a.ks, &a.vs, &a.os, &a.os};
    for (int t = 0; t < f.n; ++t) {
        const bool keys = t == 1 || t == 2;
        f.from[t] = from[t]; f.to[t] = ws; f.strides[t] = *strides[t];
        f.heads[t] = keys ? a.kv : a.heads;
        f.pixels[t] = keys ? (long long)a.km.H * a.km.W : (long long)a.qm.H * a.qm.W;
        f.first[t + 1] = f.first[t] + a.B * f.pixels[t] * f.heads[t] * (p.dp / E);
        ws += p.bytes[t];
    }
    for (int t = 0; t < f.n; ++t) *strides[t] = Strides{(long long)f.heads[t] * p.dp, f.pixels[t] * f.heads[t] * p.dp};
    a.q = f.to[0]; a.k = f.to[1]; a.v = f.to[2];
    if (dout) { *dout = f.to[3]; *out = f.to[4]; }
    a.hd = a.dl = p.dp;
    const long long blocks = (f.first[f.n] + 255) / 256;
    region_copy_kernel<T><<<(int)std::min<long long>(blocks, 1 << 20), 256, 0, st>>>(f);
    return hipGetLastError();
}

// Workgroups go to the eight XCDs in turn, each with an L2 of its own: work items that share keys are given to one XCD in a row.
__device__ __forceinline__ uint32_t xcd_order(uint32_t block, uint32_t blocks)
{
    const uint32_t whole = blocks & ~7u;
    return block < whole ? (block & 7) * (whole >> 3) + (block >> 3) : block;
}

}  // namespace region
}  // namespace slide
