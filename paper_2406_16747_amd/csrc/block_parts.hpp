// Attention over blocks of 64 tokens: what the selection, the forward, the backward and the cache in 8 bits share.
#pragma once
#include "attn_tiles.hpp"

namespace spk {

constexpr int BT = SPARSEK_BLOCK_TOKENS;   // tokens per block
static_assert(BT == KT, "a block is one key tile");

// A block whose largest magnitude is below this is held as zeros with scale 0: 127 / max (or 448 / max) stays finite.
constexpr float TINY_MAX = 0x1p-100f;

inline int block_count(int n) { return (n + BT - 1) / BT; }

// Selected (query, block) pairs of one key/value head at most: query i has i / 64 blocks behind it.
inline long long block_pairs(int n, int top)
{
    const long long nb = n / BT, rest = n % BT, full = std::min<long long>(nb, top);   // blocks 0 .. full-1 have fewer than top behind them
    return BT * (full * (full - 1) / 2 + (nb - full) * top) + rest * std::min<long long>(nb, top);
}

// The lists that the attention kernels walk: for every key block the queries that selected it, ascending.  Everything per
// (batch, key/value head); rows are (list entry, query head of the group), entry-major.
//   masks[chunk][block]  which of the chunk's 64 queries selected the block
//   off[chunk][block]    list entries of the block that come from earlier chunks
//   total, base[block]   length and start of the block's list
//   list[entry]          the query;  pos[query][slot]: the entry of the query's slot, -1 where the slot is empty
//   units[]              (block, first row) of every piece of at most `unit` rows, block by block; nunits; first_unit[block]
// A counting sort whose result depends on nothing but idx.
struct BlockLists {
    unsigned long long* masks;
    int32_t *off, *total, *base, *first_unit, *list, *pos, *nunits;
    int2* units;
    int B, H, Hkv, G, n, nb, top;
    int unit, maxu;          // rows per unit, units at most
    long long pairs;
};

struct BlockLayout {
    BlockLists l;
    size_t bytes;
};
// Carves the lists out of ws (null: sizes only).
inline BlockLayout block_lists_layout(const sparsek_block_cfg& c, int unit, void* ws)
{
    BlockLayout y;
    BlockLists& l = y.l;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* p = (char*)ws + at;
        at = align_up(at + bytes, 256);
        return (void*)p;
    };
    l.B = c.B; l.H = c.H; l.Hkv = c.Hkv; l.G = c.H / c.Hkv; l.n = c.n; l.nb = block_count(c.n); l.top = c.top;
    l.unit = unit;
    l.pairs = block_pairs(c.n, c.top);
    l.maxu = (int)(l.pairs * l.G / unit + (l.pairs ? l.nb : 0));
    const size_t BG = (size_t)c.B * c.Hkv, nb = l.nb;
    l.masks = (unsigned long long*)take(BG * nb * nb * 8);
    l.off = (int32_t*)take(BG * nb * nb * 4);
    l.total = (int32_t*)take(BG * nb * 4);
    l.base = (int32_t*)take(BG * nb * 4);
    l.first_unit = (int32_t*)take(BG * nb * 4);
    l.list = (int32_t*)take(BG * l.pairs * 4);
    l.pos = (int32_t*)take(BG * c.n * c.top * 4);
    l.nunits = (int32_t*)take(BG * 4);
    l.units = (int2*)take(BG * l.maxu * 8);
    y.bytes = at;
    return y;
}
// Fills the lists from idx [B,Hkv,n,top]; entries that are no block behind their query, and repeated ones, are left out.
int launch_block_lists(const BlockLists& l, const int32_t* idx, hipStream_t st);

// One launch-argument bundle for the kernels of the forward and the backward.
struct BlockArgs {
    BlockLists l;
    const uint16_t *q, *k, *v, *o, *dO;
    const float* lse;
    float c2, scale;
};

#ifdef __HIPCC__
// 64 rows of D bf16 (contiguous rows at src, row r clamped to r_max) into a RowTile; 256 threads.
template <int D>
__device__ __forceinline__ void load_rows(unsigned char* tile, const uint16_t* src, int r_max, int tid)
{
    constexpr int CPR = D / 8;   // 16-byte pieces per row
#pragma unroll
    for (int t = 0; t < BT * CPR / 256; t++) {
        const int id = tid + 256 * t, r = id / CPR, c = id % CPR;
        const u32x4 x = *(const u32x4*)(src + (size_t)min(r, r_max) * D + 8 * c);
        *(u32x4*)(tile + RowTile<D>::offset(r) + 16 * c) = x;
    }
}

// Rounds to whole numbers of at most 127: the mean key of a block, the pooled query, a block held in 8 bits.  The factor is the
// reciprocal of the largest magnitude, rounded, times 127 (or 448), rounded; the product with it is rounded once and then to the
// nearest whole number (even on ties): the same in every kernel.  What a code of 1 stands for: the magnitude times 1/127 (1/448).
__device__ __forceinline__ float code_factor(float top, float most) { return top >= TINY_MAX ? (1.0f / top) * most : 0.0f; }
__device__ __forceinline__ float code_scale(float top, float most) { return top >= TINY_MAX ? top * (1.0f / most) : 0.0f; }
__device__ __forceinline__ int code_i8(float x, float f)
{
    const float y = rintf(x * f);
    return (int)fminf(fmaxf(y, -127.0f), 127.0f);   // (a NaN becomes -127)
}
__device__ __forceinline__ unsigned pack4(int a, int b, int c, int d)
{
    return (a & 255) | (b & 255) << 8 | (c & 255) << 16 | (unsigned)d << 24;
}

// fp16 holds a partial result relative to the largest value of its block: h = x * 2^(127 - E) with E the biased exponent
// of that value, so |h| < 4, and 2^-12 relative is lost where bf16 would lose 2^-9.
__device__ __forceinline__ int scale_exp(unsigned top_bits) { return min(max((int)(top_bits >> 23) & 255, 1), 253); }
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2v __attribute__((ext_vector_type(2)));

// The largest of a workgroup's 256 values (>= 0, as bits); red: 4 words of LDS.  Two barriers.
__device__ __forceinline__ unsigned block_max_bits(unsigned x, unsigned* red, int tid)
{
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) x = max(x, (unsigned)__shfl_xor((int)x, s, 64));
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = x;
    __syncthreads();
    return max(max(red[0], red[1]), max(red[2], red[3]));
}
#endif

}  // namespace spk
