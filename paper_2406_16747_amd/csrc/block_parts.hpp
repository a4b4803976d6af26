// Attention over blocks of 64 tokens: what the selection, the forward, the backward and the cache in 8 bits share.
#pragma once
#include "attn_tiles.hpp"

namespace spk {

constexpr int BT = SPARSEK_BLOCK_TOKENS;   // tokens per block
static_assert(BT == KT, "a block is one key tile");

// A block whose largest magnitude is below this is held as zeros with scale 0: 127 / max (or 448 / max) stays finite.
constexpr float TINY_MAX = 0x1p-100f;

inline int block_count(int n) { return (n + BT - 1) / BT; }

// The lists that the attention kernels walk: for every key block the queries that attend it -- its own ones first, then those that
// selected it, ascending.  They are made for stretches of `cq` queries (a multiple of 64): what a stretch's queries leave behind per
// block is joined before the next one's, in the same memory.  Everything per (batch, key/value head); rows are (list entry, query head
// of the group), entry-major.  Stretch c, block j:
//   counts[chunk][block]   how many of the chunk's 64 queries selected the block
//   off[chunk][block]      list entries of the block that come from earlier chunks of the stretch
//   total, base[c][block]  length and start of the block's list
//   list[c][entry]         the query;  pos[query][slot]: the entry of the query's own block (slot 0) and of its selected ones, -1: none
//   units[c][]             (block, first row) of every piece of at most `unit` rows, block by block; nunits[c]; first_unit[c][block]
// A counting sort whose result depends on nothing but idx.
struct BlockLists {
    uint8_t* counts;
    int32_t *off, *total, *base, *first_unit, *list, *pos, *nunits;
    int2 *units, *order;     // (block, first row), block by block, and as they are worked through
    int B, H, Hkv, G, n, nb, top;
    int cq, nc, unit, maxu;  // queries per stretch, stretches, rows per unit, units of a stretch at most
    int slots;               // top + 1
    size_t entries;          // of a stretch at most

    __host__ __device__ size_t cbg(int c, int bg) const { return (size_t)c * B * Hkv + bg; }
};

struct BlockLayout {
    BlockLists l;
    size_t bytes;
};
// Carves the lists out of ws (null: sizes only).
inline BlockLayout block_lists_layout(const sparsek_block_cfg& c, int cq, int unit, void* ws)
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
    l.cq = cq;
    l.nc = (c.n + cq - 1) / cq;
    l.unit = unit;
    l.slots = c.top + 1;
    l.entries = (size_t)std::min(cq, c.n) * l.slots;
    l.maxu = (int)(l.entries * l.G / unit + std::min<size_t>(l.nb, l.entries));
    const size_t BG = (size_t)c.B * c.Hkv, nb = l.nb, S = BG * l.nc;
    l.counts = (uint8_t*)take(BG * nb * nb);
    l.off = (int32_t*)take(BG * nb * nb * 4);
    l.total = (int32_t*)take(S * nb * 4);
    l.base = (int32_t*)take(S * nb * 4);
    l.first_unit = (int32_t*)take(S * nb * 4);
    l.list = (int32_t*)take(S * l.entries * 4);
    l.pos = (int32_t*)take(BG * c.n * l.slots * 4);
    l.nunits = (int32_t*)take(S * 4);
    l.units = (int2*)take(S * l.maxu * 8);
    l.order = (int2*)take(S * l.maxu * 8);
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
// Notes the rows of the pieces that load_rows (or a loop like it) found to be not finite in rows[2], as bits.
template <int D>
__device__ __forceinline__ void note_rows(unsigned* rows, unsigned bad, int tid)
{
    for (; bad; bad &= bad - 1) {
        const int r = (tid + 256 * (__ffs(bad) - 1)) / (D / 8);
        atomicOr(&rows[r >> 5], 1u << (r & 31));
    }
}
// The largest magnitude of 8 bf16 values, as bits of a float.
__device__ __forceinline__ unsigned top_of_8(u32x4 x)
{
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 4; e++) top = max(top, max(x[e] << 16 & 0x7FFFFFFFu, x[e] & 0x7FFF0000u));
    return top;
}
constexpr unsigned INF_BITS = 0x7F800000u;
// Whether the smallest of a block's pieces of 8 values (`low`, inverted; 0: none but zeros) lies more than 2^13 below its largest value:
// relative to that, fp16 still has all its bits down to 2^-27.
__device__ __forceinline__ bool is_wide(unsigned top, unsigned low) { return low && (top >> 23) > (~low >> 23) + 13; }

// 64 rows of D bf16 (contiguous rows at src, row r clamped to r_max) into a RowTile; 256 threads.  Returns the largest finite magnitude
// that the thread has seen, as bits.  Pieces with an infinity or a NaN become zeros (a weight of zero times one of those would reach
// rows that do not attend the key), and are noted in `bad`, a bit each.
template <int D>
__device__ __forceinline__ unsigned load_rows(unsigned char* tile, const uint16_t* src, int r_max, int tid, unsigned& bad)
{
    constexpr int CPR = D / 8;   // 16-byte pieces per row
    unsigned top = 0;
#pragma unroll
    for (int t = 0; t < BT * CPR / 256; t++) {
        const int id = tid + 256 * t, r = id / CPR, c = id % CPR;
        u32x4 x = *(const u32x4*)(src + (size_t)min(r, r_max) * D + 8 * c);
        const unsigned y = top_of_8(x);
        if (y >= INF_BITS) {
            x = u32x4{0, 0, 0, 0};
            bad |= 1u << t;
        }
        top = max(top, y >= INF_BITS ? 0u : y);
        *(u32x4*)(tile + RowTile<D>::offset(r) + 16 * c) = x;
    }
    return top;
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

// fp16 holds values relative to the largest of their block, with biased exponent E: x * 2^(140 - E), so that the largest lies in
// [2^13, 2^14) and only what is below 2^-27 of it loses bits that fp16's normal numbers have: 2^-11 relative, where bf16 has 2^-8.
__device__ __forceinline__ int scale_exp(unsigned top_bits) { return min(max((int)(top_bits >> 23) & 255, 14), 253); }
__device__ __forceinline__ float scale_down(int E) { return __uint_as_float((unsigned)(267 - E) << 23); }   // 2^(140 - E)
__device__ __forceinline__ float scale_up(int E) { return __uint_as_float((unsigned)(E - 13) << 23); }      // 2^(E - 140)
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2v __attribute__((ext_vector_type(2)));

// Orders a wave's own LDS accesses across its lanes (the hardware keeps a wave's LDS operations in order).
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Stores through a buffer of `bytes` bytes at p (both the same for the whole wave): what lies outside is dropped.  A condition on the
// store itself is a branch around it, behind which the compiler waits for everything that the wave has under way.
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef __amdgpu_buffer_rsrc_t buffer_t;
__device__ __forceinline__ buffer_t buffer_of(const void* p, int bytes)
{
    const uint64_t at = (uint64_t)p;
    void* base = (void*)((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(at >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)at));
    return __builtin_amdgcn_make_buffer_rsrc(base, 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
__device__ __forceinline__ void store_words(buffer_t b, int offset, u32x4 v) { __builtin_amdgcn_raw_buffer_store_b128(v, b, offset, 0, 0); }
// Whole lines that nobody reads soon: they leave the caches to what is read again.
__device__ __forceinline__ void stream_words(buffer_t b, int offset, u32x4 v) { __builtin_amdgcn_raw_buffer_store_b128(v, b, offset, 0, 2); }
__device__ __forceinline__ void store_words(buffer_t b, int offset, u32x2 v) { __builtin_amdgcn_raw_buffer_store_b64(v, b, offset, 0, 0); }

// Workgroup id -> (batch and head, item): workgroups go to the chip's 8 partitions in turn; of every 8 heads each partition gets
// one, so that what a head's workgroups share stays in one L2.  Those of up to 7 heads that are left over go to all of them.
__device__ __forceinline__ void deal_head(unsigned id, int items, int BG, int& bg, int& item)
{
    const unsigned whole = BG & ~7;
    if (id < whole * items) {
        const unsigned slot = id >> 3;
        bg = (int)(slot / items * 8 + (id & 7));
        item = (int)(slot % items);
    } else {
        const unsigned rest = id - whole * items;
        bg = (int)(whole + rest / items);
        item = (int)(rest % items);
    }
}

// The largest of a workgroup's 256 values (>= 0, as bits); red: 4 words of LDS.  Two barriers.
__device__ __forceinline__ unsigned wave_max_bits(unsigned x)
{
    int y = (int)x;
#pragma unroll
    for (int s = 0; s < 4; s++) y = max(y, dpp_i32(y, s));
    return (unsigned)max(max(__builtin_amdgcn_readlane(y, 15), __builtin_amdgcn_readlane(y, 31)), max(__builtin_amdgcn_readlane(y, 47), __builtin_amdgcn_readlane(y, 63)));
}
__device__ __forceinline__ unsigned block_max_bits(unsigned x, unsigned* red, int tid)
{
    x = wave_max_bits(x);
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = x;
    __syncthreads();
    return max(max(red[0], red[1]), max(red[2], red[3]));
}
// The largest of a workgroup's 256 values (>= 0, as bits) twice; red: 8 words of LDS.  Two barriers.
__device__ __forceinline__ void block_max_bits2(unsigned& x, unsigned& y, unsigned* red, int tid)
{
    x = wave_max_bits(x);
    y = wave_max_bits(y);
    __syncthreads();
    if ((tid & 63) == 0) {
        red[tid >> 6] = x;
        red[4 + (tid >> 6)] = y;
    }
    __syncthreads();
    x = max(max(red[0], red[1]), max(red[2], red[3]));
    y = max(max(red[4], red[5]), max(red[6], red[7]));
}
#endif

}  // namespace spk
