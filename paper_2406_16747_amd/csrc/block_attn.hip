// Attention over the blocks of 64 tokens that every query selected, and over the query's own block (forward).
//
// Queries that lie side by side select different blocks, so a tile of queries against the union of their blocks would do
// several times the work.  The kernels go by key block instead: block_tiles_kernel takes a block's K and V into LDS once and
// walks the queries that attend it, 32 rows (query, head of the group) to a wave: S^T = K.Q^T, the softmax of these 64 keys alone,
// O^T = V^T.P^T, and leaves the normalised partial result, with the log of its denominator, in list order.  block_join_kernel adds up
// the partial results of every row with their weights.
// A (row, block) pair moves a row of q in and D halves out and in again, for 4*64*D flops.  32 heads of 128 (8 of keys), 32768 tokens,
// 16 blocks: 2550 to 2600 us, of which the tiles take 1350, the join 925 (4.9 TB/s: memory), the selection 285.  The tiles are bound by issue: matrix
// pipes, vector ALU and LDS are busy 22, 40 and 33 % of the time and take turns rather than overlap (waves wait to issue half of their
// cycles, for memory a quarter); with the 4.6 GB of partial results written to one place they took 1150 where 1350 is usual.
#include "block_parts.hpp"

#include <cmath>
#include <type_traits>

namespace spk {

// ---- the lists ----

// A chunk's selection [64][top] and its 64 queries as bits, for the key blocks j0 .. j0 + MASK_BLOCKS - 1.  LDS: masks, then the selection.
constexpr int MASK_BLOCKS = 4096;
inline size_t chunk_lds(const BlockLists& l) { return (size_t)std::min(MASK_BLOCKS, l.nb) * 8 + (size_t)BT * l.top * 4; }
struct ChunkLds {
    unsigned long long* masks;
    int* sel;
};
__device__ __forceinline__ ChunkLds chunk_lds_at(unsigned char* lds, const BlockLists& l)
{
    return ChunkLds{(unsigned long long*)lds, (int*)(lds + (size_t)min(MASK_BLOCKS, l.nb) * 8)};
}
__device__ __forceinline__ void chunk_masks(ChunkLds m, const BlockLists& l, const int32_t* idx, int bg, int c, int j0, int tid)
{
    const int jn = min(MASK_BLOCKS, c - j0), count = min(BT, l.n - c * BT) * l.top;
    for (int x = tid; x < jn; x += 256) m.masks[x] = 0;
    if (j0 == 0) {
        const int32_t* row = idx + ((size_t)bg * l.n + (size_t)c * BT) * l.top;
#pragma unroll 4
        for (int x = tid; x < count; x += 256) m.sel[x] = row[x];
    }
    __syncthreads();
    for (int x = tid; x < count; x += 256) {
        const int j = m.sel[x];
        if (j >= j0 && j - j0 < jn) atomicOr(&m.masks[j - j0], 1ull << (x / l.top));
    }
    __syncthreads();
}

// counts: a workgroup per (chunk, batch and head).
__global__ __launch_bounds__(256) void block_counts_kernel(BlockLists l, const int32_t* __restrict__ idx)
{
    extern __shared__ unsigned char lds[];
    const ChunkLds m = chunk_lds_at(lds, l);
    const int c = blockIdx.x, bg = blockIdx.y, tid = threadIdx.x;
    for (int j0 = 0; j0 < c; j0 += MASK_BLOCKS) {
        chunk_masks(m, l, idx, bg, c, j0, tid);
        for (int x = tid; x < min(MASK_BLOCKS, c - j0); x += 256) l.counts[((size_t)bg * l.nb + c) * l.nb + j0 + x] = (uint8_t)__popcll(m.masks[x]);
        __syncthreads();
    }
}

// off and total: a workgroup of 1024 per (64 blocks, stretch, batch and head), its 16 waves share the stretch's chunks.
__global__ __launch_bounds__(1024) void block_offsets_kernel(BlockLists l)
{
    __shared__ int part[16][64];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, j = blockIdx.x * 64 + lane, bg = blockIdx.z;
    const int first = (int)blockIdx.y * (l.cq / BT), count = min(l.cq / BT, l.nb - first);
    if ((int)blockIdx.x * 64 >= first + count) return;   // nobody sees these blocks yet
    const int per = (count + 15) / 16, c1 = l.top ? first + min(count, wv * per + per) : 0;
    const int c0 = max(first + wv * per, j + 1);         // (a chunk selects blocks behind its own only)
    const uint8_t* m = l.counts + (size_t)bg * l.nb * l.nb + j;
    int sum = 0;
#pragma unroll 8
    for (int c = c0; c < c1; c++) sum += m[(size_t)c * l.nb];
    part[wv][lane] = sum;
    __syncthreads();
    const int own = j >= first && j < first + count ? min(BT, l.n - j * BT) : 0;
    int run = own, all = own;
#pragma unroll
    for (int w = 0; w < 16; w++) {
        run += w < wv ? part[w][lane] : 0;
        all += part[w][lane];
    }
    if (j >= first + count) return;
    int32_t* off = l.off + (size_t)bg * l.nb * l.nb + j;
#pragma unroll 8
    for (int c = c0; c < c1; c++) {
        off[(size_t)c * l.nb] = run;
        run += m[(size_t)c * l.nb];
    }
    if (wv == 0) l.total[l.cbg(blockIdx.y, bg) * l.nb + j] = all;
}

// base and units: a workgroup of 1024 per (stretch, batch and head).
__global__ __launch_bounds__(1024) void block_units_kernel(BlockLists l)
{
    __shared__ int2 wsum[16];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const size_t cbg = l.cbg(blockIdx.x, blockIdx.y);
    const int seen = min(l.nb, ((int)blockIdx.x + 1) * (l.cq / BT));   // blocks that the stretch's queries can see
    int2 done = make_int2(0, 0);   // list entries and units ahead of this round of 1024 blocks
    for (int j0 = 0; j0 < seen; j0 += 1024) {
        const int j = j0 + tid;
        const int mine = j < seen ? l.total[cbg * l.nb + j] : 0;
        const int units = (int)(((long long)mine * l.G + l.unit - 1) / l.unit);
        int2 s = make_int2(mine, units);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int x = __shfl_up(s.x, d, 64), y = __shfl_up(s.y, d, 64);
            if (lane >= d) { s.x += x; s.y += y; }
        }
        if (lane == 63) wsum[wv] = s;
        __syncthreads();
        int2 before = done, all = make_int2(0, 0);
#pragma unroll
        for (int w = 0; w < 16; w++) {
            if (w < wv) { before.x += wsum[w].x; before.y += wsum[w].y; }
            all.x += wsum[w].x;
            all.y += wsum[w].y;
        }
        if (j < seen) {
            l.base[cbg * l.nb + j] = before.x + s.x - mine;
            const int u0 = before.y + s.y - units;
            l.first_unit[cbg * l.nb + j] = u0;
            for (int u = 0; u < units; u++)
                if (u0 + u < l.maxu) l.units[cbg * l.maxu + u0 + u] = make_int2(j, u * l.unit);
        }
        done.x += all.x;
        done.y += all.y;
        __syncthreads();
    }
    if (tid == 0) l.nunits[cbg] = min(done.y, l.maxu);
}

// order: the units by the chunk of their first query, a workgroup of 1024 per (stretch, batch and head).  Units that are worked on
// side by side find query rows that their neighbours have read in the caches then, which is worth more than a block's own K and V
// (32 heads of 32768: 2712 us, 2778 block by block; 17 us of it are this kernel's).
constexpr int ORDER_BUCKETS = 1024;
__global__ __launch_bounds__(1024) void block_order_kernel(BlockLists l)
{
    __shared__ int at[ORDER_BUCKETS], wsum[16];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const size_t cbg = l.cbg(blockIdx.x, blockIdx.y);
    const int q0 = (int)blockIdx.x * l.cq, units = l.nunits[cbg], per = ((l.cq / BT + ORDER_BUCKETS - 1) / ORDER_BUCKETS) * BT;
    const int2* in = l.units + cbg * l.maxu;
    const int32_t *list = l.list + cbg * l.entries, *base = l.base + cbg * l.nb;
    auto bucket = [&](int2 u) { return (list[base[u.x] + u.y / l.G] - q0) / per; };
    at[tid] = 0;
    __syncthreads();
#pragma unroll 4
    for (int x = tid; x < units; x += 1024) atomicAdd(&at[bucket(in[x])], 1);
    __syncthreads();
    const int mine = at[tid];
    int s = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(s, d, 64);
        if (lane >= d) s += x;
    }
    if (lane == 63) wsum[wv] = s;
    __syncthreads();
    s -= mine;
#pragma unroll
    for (int w = 0; w < 16; w++) s += w < wv ? wsum[w] : 0;
    at[tid] = s;
    __syncthreads();
#pragma unroll 4
    for (int x = tid; x < units; x += 1024) {
        const int2 u = in[x];
        l.order[cbg * l.maxu + atomicAdd(&at[bucket(u)], 1)] = u;   // (which of a bucket's comes first changes no result)
    }
}

// list and pos: a workgroup per (chunk, batch and head).
__global__ __launch_bounds__(256) void block_place_kernel(BlockLists l, const int32_t* __restrict__ idx)
{
    extern __shared__ unsigned char lds[];
    const ChunkLds m = chunk_lds_at(lds, l);
    const int c = blockIdx.x, bg = blockIdx.y, tid = threadIdx.x, rows = min(BT, l.n - c * BT);
    const size_t cbg = l.cbg(c * BT / l.cq, bg);
    int32_t *list = l.list + cbg * l.entries, *pos = l.pos + ((size_t)bg * l.n + (size_t)c * BT) * l.slots;
    const int32_t *base = l.base + cbg * l.nb, *off = l.off + ((size_t)bg * l.nb + c) * l.nb;
    if (tid < rows) {
        list[base[c] + tid] = c * BT + tid;
        pos[(size_t)tid * l.slots] = base[c] + tid;
    }
    for (int j0 = 0; j0 == 0 || j0 < c; j0 += MASK_BLOCKS) {
        chunk_masks(m, l, idx, bg, c, j0, tid);
        for (int x = tid; x < rows * l.top; x += 256) {
            const int r = x / l.top, s = x - r * l.top, j = m.sel[x];
            if (j < 0 || j >= c) {
                if (j0 == 0) pos[(size_t)r * l.slots + 1 + s] = -1;
                continue;
            }
            if (j < j0 || j >= j0 + MASK_BLOCKS) continue;
            int p = base[j] + off[j] + __popcll(m.masks[j - j0] & ((1ull << r) - 1));
            for (int y = 0; y < s; y++) p = m.sel[x - s + y] == j ? -1 : p;   // (a repeated block counts once)
            if (p >= 0) list[p] = c * BT + r;
            pos[(size_t)r * l.slots + 1 + s] = p;
        }
        __syncthreads();
    }
}

// All of it in one launch where a (batch, head) has few blocks and pairs: a workgroup of 1024 each, counts and offsets in LDS.  Four
// launches of 3 us each are most of a short sequence's lists.
constexpr int FEW_BLOCKS = 64, FEW_PAIRS = 16384;
__global__ __launch_bounds__(1024) void block_short_lists_kernel(BlockLists l, const int32_t* __restrict__ idx)
{
    __shared__ unsigned long long masks[FEW_BLOCKS][FEW_BLOCKS];   // [chunk][block]
    __shared__ uint16_t off[FEW_BLOCKS][FEW_BLOCKS];
    __shared__ int base[FEW_BLOCKS], repeated;
    __shared__ uint8_t sel[FEW_PAIRS];   // the pairs' blocks; 255: not one of them
    const int bg = blockIdx.x, tid = threadIdx.x, nb = l.nb, pairs = l.n * l.top;
    const int32_t* row = idx + (size_t)bg * pairs;
    int first[4];   // (on their way while the masks are cleared)
#pragma unroll
    for (int y = 0; y < 4; y++) first[y] = tid + 1024 * y < pairs ? row[tid + 1024 * y] : -1;
    if (tid == 0) repeated = 0;
    for (int x = tid; x < nb * FEW_BLOCKS; x += 1024) masks[x / FEW_BLOCKS][x % FEW_BLOCKS] = 0;
    __syncthreads();
    auto take = [&](int x, int j) {
        const int i = x / l.top, c = i / BT;
        const bool ok = j >= 0 && j < c;
        const unsigned long long bit = 1ull << (i % BT);
        sel[x] = ok ? (uint8_t)j : 255;
        if (ok && (atomicOr(&masks[c][j], bit) & bit)) repeated = 1;
    };
#pragma unroll
    for (int y = 0; y < 4; y++)
        if (tid + 1024 * y < pairs) take(tid + 1024 * y, first[y]);
#pragma unroll 4
    for (int x = tid + 4096; x < pairs; x += 1024) take(x, row[x]);
    __syncthreads();
    if (tid < 64) {   // a lane per block
        const int j = tid, own = j < nb ? min(BT, l.n - j * BT) : 0;
        int run = own;
#pragma unroll 8
        for (int c = 0; c < nb; c++) {
            const int count = __popcll(masks[c][j]);   // (0 where c <= j)
            off[c][j] = (uint16_t)run;
            run += count;
        }
        const int units = (int)(((long long)run * l.G + l.unit - 1) / l.unit);
        int2 s = make_int2(run, units);
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int x = __shfl_up(s.x, d, 64), y = __shfl_up(s.y, d, 64);
            if (j >= d) { s.x += x; s.y += y; }
        }
        base[j] = s.x - run;
        if (j < nb) {
            l.total[(size_t)bg * nb + j] = run;
            l.base[(size_t)bg * nb + j] = s.x - run;
            const int u0 = s.y - units;
            l.first_unit[(size_t)bg * nb + j] = u0;
            for (int u = 0; u < units; u++)
                if (u0 + u < l.maxu) l.order[(size_t)bg * l.maxu + u0 + u] = make_int2(j, u * l.unit);
        }
        if (j == 63) l.nunits[bg] = min(s.y, l.maxu);
    }
    __syncthreads();
    int32_t *list = l.list + (size_t)bg * l.entries, *pos = l.pos + (size_t)bg * l.n * l.slots;
    for (int i = tid; i < l.n; i += 1024) {
        const int p = base[i / BT] + i % BT;
        list[p] = i;
        pos[(size_t)i * l.slots] = p;
    }
#pragma unroll 4
    for (int x = tid; x < pairs; x += 1024) {
        const int j = sel[x], i = x / l.top, s = x - i * l.top, c = i / BT;
        int p = -1;
        if (j < 255) {
            p = base[j] + off[c][j] + __popcll(masks[c][j] & ((1ull << (i % BT)) - 1));
            if (repeated)
                for (int y = 0; y < s; y++) p = sel[x - s + y] == j ? -1 : p;   // (a repeated block counts once)
            if (p >= 0) list[p] = i;
        }
        pos[(size_t)i * l.slots + 1 + s] = p;
    }
}

int launch_block_lists(const BlockLists& l, const int32_t* idx, hipStream_t st)
{
    const int BG = l.B * l.Hkv;
    if (l.nb <= FEW_BLOCKS && l.nc == 1 && (long long)l.n * l.top <= FEW_PAIRS) {
        hipLaunchKernelGGL(block_short_lists_kernel, dim3(BG), dim3(1024), 0, st, l, idx);
        return launch_status();
    }
    const size_t lds = chunk_lds(l);
    if (l.top) hipLaunchKernelGGL(block_counts_kernel, dim3(l.nb, BG), dim3(256), lds, st, l, idx);
    hipLaunchKernelGGL(block_offsets_kernel, dim3((l.nb + 63) / 64, l.nc, BG), dim3(1024), 0, st, l);
    hipLaunchKernelGGL(block_units_kernel, dim3(l.nc, BG), dim3(1024), 0, st, l);
    hipLaunchKernelGGL(block_place_kernel, dim3(l.nb, BG), dim3(256), lds, st, l, idx);
    hipLaunchKernelGGL(block_order_kernel, dim3(l.nc, BG), dim3(1024), 0, st, l);
    return launch_status();
}

// ---- the forward ----

constexpr double FWD_STRETCH_BYTES = 8e9;

struct BlockFwd {
    BlockArgs a;
    uint16_t* o;
    float* lse;
    _Float16* part;    // [nbg][entry rows of a stretch][D]
    float2* meta;      // log2 of the row's denominator, and the factor that the halves stand for
    float* mass;       // [B,Hkv,nb] or null
    int c, bg0, nbg;   // the stretch, the first of the heads (of all batches) and their number
    bool stream;       // the partial results are more than the chip's last cache holds
};

template <int D>
__device__ __forceinline__ f16x8 transposed_half(uint32_t at) { return __builtin_bit_cast(f16x8, transposed_operand<D>(at)); }

// The softmax of one tile of 32 rows against the block's 64 keys: S^T = K.Q^T; put(x, p) takes the weights (times 2^UP), x in the order of
// P^T as the operand of O^T = V^T.P^T.  A lane has one column (row of q); with `own` it sees keys 0 .. limit of the block.
template <int D, int UP, class Put>
__device__ __forceinline__ void block_weights(uint32_t rk, const bf16x8 (&qf)[D / 16], float c2, bool own, int limit, int half, float& m, float& den,
                                              Put put)
{
    using S = RowTile<D>;
    constexpr int DS = D / 16;
    f32x16 s[2];
#pragma unroll
    for (int kh = 0; kh < 2; kh++) {
        bf16x8 ka[DS];   // (all of them on their way before the first product waits for one)
#pragma unroll
        for (int x = 0; x < DS; x++) ka[x] = row_operand(rk + 2 * kh * S::R16 + 32 * x);
        __builtin_amdgcn_sched_barrier(0);
        s[kh] = f32x16{0};
#pragma unroll
        for (int x = 0; x < DS; x++) s[kh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[x], qf[x], s[kh], 0, 0, 0);
    }
    if (own)
#pragma unroll
        for (int kh = 0; kh < 2; kh++)
#pragma unroll
            for (int r = 0; r < 16; r++) s[kh][r] = 32 * kh + 8 * (r / 4) + 4 * half + r % 4 > limit ? -INFINITY : s[kh][r];
    m = -INFINITY;
#pragma unroll
    for (int kh = 0; kh < 2; kh++)
#pragma unroll
        for (int r = 0; r < 16; r++) m = fmaxf(m, s[kh][r]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    const float most = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
    m = most * c2;
    const float at = m == -INFINITY ? 0.0f : m;
    float ref = at - UP, by = c2;
    const bool large = fabsf(at) >= 0x1p22f;
    if (__any(large)) {   // the roundings of m and m - UP count: such a row's logits become distances from the largest first
        const float off = fmaf(most, c2, -at);
#pragma unroll
        for (int kh = 0; kh < 2; kh++)
#pragma unroll
            for (int r = 0; r < 16; r++) s[kh][r] = large ? fmaf(s[kh][r], c2, -at) - off : s[kh][r];
        by = large ? 1.0f : c2;
        ref = large ? (float)-UP : ref;
    }
    den = 0.0f;
#pragma unroll
    for (int kh = 0; kh < 2; kh++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[kh][r], by, -ref));
            den += p;
            put(16 * kh + r, p);
        }
    const auto sl = __builtin_amdgcn_permlane32_swap(__float_as_uint(den), __float_as_uint(den), false, false);
    den = __uint_as_float(sl[0]) + __uint_as_float(sl[1]);
}

template <int D>
struct FwdBlockSmem {
    static constexpr int RS = 128 + 16;     // bytes between rows: half a row of 128 columns
    unsigned char k[RowTile<D>::BYTES], v[RowTile<D>::BYTES];
    unsigned char rows[4][32 * RS];         // a wave's rows on their way in and its results on their way out
    unsigned red[8], bad[2][2];             // bad: keys that are not finite, or have values that are not, as bits
};
static_assert(sizeof(FwdBlockSmem<128>) <= 160 * 1024 / 3, "three workgroups per CU");

template <int D>
__global__ __launch_bounds__(256, 3) void block_tiles_kernel(BlockFwd f)
{
    __shared__ __attribute__((aligned(16))) FwdBlockSmem<D> sm;
    constexpr int CPR = D / 8;
    const BlockLists& l = f.a.l;
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
    int bg, un;
    deal_head(blockIdx.x, l.maxu, f.nbg, bg, un);
    bg += f.bg0;
    const size_t cbg = l.cbg(f.c, bg);
    if (un >= l.nunits[cbg]) return;
    const int2 u = l.order[cbg * l.maxu + un];
    const int j = u.x, first = u.y, G = l.G;
    const int base = l.base[cbg * l.nb + j];
    const int end = min(l.total[cbg * l.nb + j] * G, first + l.unit);
    const size_t kv = ((size_t)bg * l.n + (size_t)j * BT) * D;
    const int last = l.n - 1 - j * BT;
    // V goes to fp16 relative to its largest magnitude, and so do the weights (times 2^15): a weight is rounded to 2^-11 where bf16
    // would keep 2^-8, at the same rate.  What is not finite in a key or in its values is left out of that and of the products, and makes
    // the rows that attend the key NaN.  A block is wide when some 8 values side by side (not all 0) lie more than 2^13 below the largest:
    // its own rows see some of its tokens only, and one that they do not see must not push what they see out of fp16's range.
    u32x4 vr[BT * CPR / 256];
    unsigned top = 0, low = 0, bad_k = 0, bad_v = 0;   // low: of the smallest pieces, inverted
#pragma unroll
    for (int t = 0; t < BT * CPR / 256; t++) {
        const int id = tid + 256 * t;
        vr[t] = *(const u32x4*)(f.a.v + kv + (size_t)min(id / CPR, last) * D + 8 * (id % CPR));
    }
    load_rows<D>(sm.k, f.a.k + kv, last, tid, bad_k);
#pragma unroll
    for (int t = 0; t < BT * CPR / 256; t++) {
        const unsigned y = top_of_8(vr[t]);
        if (y >= INF_BITS) {
            vr[t] = u32x4{0, 0, 0, 0};
            bad_v |= 1u << t;
        }
        top = max(top, y >= INF_BITS ? 0u : y);
        low = max(low, y >= INF_BITS || y == 0 ? 0u : ~y);
    }
    if (tid < 4) (&sm.bad[0][0])[tid] = 0;
    block_max_bits2(top, low, sm.red, tid);   // (with a barrier inside)
    const int E = scale_exp(top);
    const bool wide = __builtin_amdgcn_readfirstlane((int)is_wide(top, low));
    note_rows<D>(sm.bad[0], bad_k, tid);
    note_rows<D>(sm.bad[1], bad_v, tid);
    const float down = scale_down(E), up = scale_up(E);
#pragma unroll
    for (int t = 0; t < BT * CPR / 256; t++) {
        const int id = tid + 256 * t;
        f16x8 y;
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] = (_Float16)(__uint_as_float(e & 1 ? vr[t][e / 2] & 0xFFFF0000u : vr[t][e / 2] << 16) * down);
        if (wide) y = __builtin_bit_cast(f16x8, vr[t]);   // (as they are, in bf16)
        *(f16x8*)(sm.v + RowTile<D>::offset(id / CPR) + 16 * (id % CPR)) = y;
    }
    __syncthreads();
    const unsigned long long badk = (unsigned long long)sm.bad[0][1] << 32 | sm.bad[0][0], badv = (unsigned long long)sm.bad[1][1] << 32 | sm.bad[1][0];
    const uint32_t rk = lds_address(sm.k) + row_lane<D>(lane), tv = lds_address(sm.v) + transposed_lane<D>(lane);
    const int b = bg / l.Hkv, g = bg % l.Hkv;
    const int32_t* list = l.list + cbg * l.entries + base;
    const size_t row0 = ((size_t)(bg - f.bg0) * l.entries + base) * G;
    constexpr int RS = FwdBlockSmem<D>::RS, NH = D / 64;
    unsigned char* rows = sm.rows[wv];
    const int own_end = j >= f.c * (l.cq / BT) && j < (f.c + 1) * (l.cq / BT) ? min(BT, last + 1) * G : 0;
    // Rows come and go in whole lines, 8 lanes to 64 columns of a row, and change places with the operands' layout in LDS, 64 columns
    // at a time.  The rows of the next tile and the queries of the one behind it are on their way while a tile is computed.
    const int lrow = lane >> 3, lcol = 8 * (lane & 7);
    const uint16_t* q0 = f.a.q + ((size_t)b * l.H + g * G) * l.n * D + lcol;
    auto entry = [&](int r) { return list[min(r, end - 1) / G]; };
    auto load_q = [&](int r, int i, u32x4 (&to)[4 * NH]) {   // r, i: of the lane's column
        const int at = min(r, end - 1) % G * l.n + i;
#pragma unroll
        for (int t = 0; t < 4; t++) {
            const uint16_t* row = q0 + (size_t)__shfl(at, 8 * t + lrow, 64) * D;
#pragma unroll
            for (int h = 0; h < NH; h++) to[4 * h + t] = *(const u32x4*)(row + 64 * h);
        }
    };
    bf16x8 qf[D / 16];
    auto take_q = [&](const u32x4 (&from)[4 * NH]) {
#pragma unroll
        for (int h = 0; h < NH; h++) {
#pragma unroll
            for (int t = 0; t < 4; t++) *(u32x4*)(rows + (8 * t + lrow) * RS + 2 * lcol) = from[4 * h + t];
            wave_lds_order();
#pragma unroll
            for (int x = 0; x < 4; x++) qf[4 * h + x] = *(const bf16x8*)(rows + col * RS + 32 * x + 16 * half);
            wave_lds_order();
        }
    };
    // The factor of a row's result, NaN where it attends what is not finite, and its denominator likewise.
    auto factor = [&](int i, float& den) {
        float inv = den > 0.0f ? 1.0f / den : den;   // (nothing but -inf: weight 0 in the sum)
        if (badk | badv) {
            const unsigned long long attended = (2ull << min(BT - 1, i - j * BT)) - 1;
            inv = (badk | badv) & attended ? __uint_as_float(0x7FC00000u) : inv;
            den = badk & attended ? __uint_as_float(0x7FC00000u) : den;
        }
        return inv;
    };
    // 64 columns of 32 rows' results, times `by`, go out.  (Rows behind the last one lie outside the buffer and are dropped.)
    auto leave = [&](buffer_t dst, int h, const f32x16 (&acc)[2], float by) {
#pragma unroll
        for (int x = 0; x < 2; x++)
#pragma unroll
            for (int y = 0; y < 4; y += 2) {
                // columns 8 y .. 8 y + 7 from both halves of the wave to its lower lanes, the next 8 to its upper lanes
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const f16x2v a = {(_Float16)(acc[x][4 * y + 2 * e] * by), (_Float16)(acc[x][4 * y + 2 * e + 1] * by)};
                    const f16x2v c = {(_Float16)(acc[x][4 * y + 4 + 2 * e] * by), (_Float16)(acc[x][4 * y + 5 + 2 * e] * by)};
                    const auto sw = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, c), false, false);
                    w[e] = sw[0];
                    w[2 + e] = sw[1];
                }
                *(u32x4*)(rows + col * RS + 64 * x + 16 * (y + half)) = w;
            }
        wave_lds_order();
#pragma unroll
        for (int t = 0; t < 4; t++) {
            const u32x4 w = *(const u32x4*)(rows + (8 * t + lrow) * RS + 2 * lcol);
            if (f.stream) stream_words(dst, 2 * D * (8 * t + lrow) + 128 * h + 2 * lcol, w);
            else store_words(dst, 2 * D * (8 * t + lrow) + 128 * h + 2 * lcol, w);
        }
        wave_lds_order();
    };
    // (the upper lanes' copy of the logarithms lies outside the buffer)
    auto leave_meta = [&](int r0, int count, float logden, float up) {
        store_words(buffer_of(f.meta + row0 + r0, 8 * count), half ? 0x7FFFFFF0 : 8 * col, u32x2{__float_as_uint(logden), __float_as_uint(up)});
    };
    int r0 = first + 32 * wv;
    if (r0 >= end) return;
    u32x4 next[4 * NH];
    if (!wide) {
        int i = entry(r0 + col), i_next = entry(r0 + 128 + col);
        load_q(r0 + col, i, next);
        take_q(next);
        for (; r0 < end; r0 += 128) {
            const int r = r0 + col;
            const int i_then = entry(r + 256);
            load_q(r + 128, i_next, next);
            f16x8 pb[4];
            float m, den;
            block_weights<D, 15>(rk, qf, f.a.c2, r0 < own_end, i - j * BT, half, m, den, [&](int x, float p) { pb[x / 8][x % 8] = (_Float16)p; });
            const float inv = factor(i, den);
            const int count = min(32, end - r0);
            const auto dst = buffer_of(f.part + (row0 + r0) * D, 2 * D * count);
            leave_meta(r0, count, m + log2f(den * 0x1p-15f), up);
#pragma unroll
            for (int h = 0; h < NH; h++) {
                f32x16 acc[2];
#pragma unroll
                for (int x = 0; x < 2; x++) acc[x] = f32x16{0};
#pragma unroll
                for (int y = 0; y < 4; y++)
#pragma unroll
                    for (int x = 0; x < 2; x++)
                        acc[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(transposed_half<D>(tv + y * RowTile<D>::R16 + 64 * (2 * h + x)), pb[y], acc[x], 0, 0, 0);
                leave(dst, h, acc, inv);
            }
            take_q(next);   // (here and not ahead of the loop's next round: the wait for these loads leaves the stores under way)
            i = i_next;
            i_next = i_then;
        }
    } else {
        // Rare, and so without loads ahead: V in bf16, which holds any size, weights as the sum of two bf16 numbers (2^-16; at most 2^-7, so that
        // no sum of products passes what fp32 holds), results relative to the row's own largest, for which the products are made twice (32 heads of 32768, 16
        // blocks, every block wide: the attention 2608 us, 2336 as it is).
        for (; r0 < end; r0 += 128) {
            const int i = entry(r0 + col);
            load_q(r0 + col, i, next);
            take_q(next);
            bf16x8 ph[4], pl[4];
            float m, den;
            block_weights<D, -7>(rk, qf, f.a.c2, r0 < own_end, i - j * BT, half, m, den, [&](int x, float p) {
                const __bf16 hi = (__bf16)p;
                ph[x / 8][x % 8] = hi;
                pl[x / 8][x % 8] = (__bf16)(p - (float)hi);
            });
            const float inv = factor(i, den);
            auto product = [&](int h, f32x16 (&acc)[2]) {
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    acc[x] = f32x16{0};
#pragma unroll
                    for (int y = 0; y < 4; y++) {
                        const bf16x8 vt = transposed_operand<D>(tv + y * RowTile<D>::R16 + 64 * (2 * h + x));
                        acc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt, ph[y], acc[x], 0, 0, 0);
                        acc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vt, pl[y], acc[x], 0, 0, 0);
                    }
#pragma unroll
                    for (int e = 0; e < 16; e++) acc[x][e] *= inv;
                }
            };
            f32x16 acc[2];
            float most = 0.0f;
#pragma unroll 1
            for (int h = 0; h < NH; h++) {
                product(h, acc);
#pragma unroll
                for (int x = 0; x < 2; x++)
#pragma unroll
                    for (int e = 0; e < 16; e++) most = fmaxf(most, fabsf(acc[x][e]));
            }
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(most), __float_as_uint(most), false, false);
            const int F = scale_exp(max((unsigned)sw[0], (unsigned)sw[1]));
            const int count = min(32, end - r0);
            const auto dst = buffer_of(f.part + (row0 + r0) * D, 2 * D * count);
            leave_meta(r0, count, m + log2f(den * 0x1p7f), scale_up(F));
#pragma unroll 1
            for (int h = 0; h < NH; h++) {
                product(h, acc);
                leave(dst, h, acc, scale_down(F));
            }
        }
    }
}

// D / 8 lanes per row (query, head of the group): the weights of its slots, then the sum of the partial results.
template <int D>
__global__ __launch_bounds__(256) void block_join_kernel(BlockFwd f, int rows_per_head)
{
    constexpr int LPR = D / 8;
    const BlockLists& l = f.a.l;
    const int G = l.G, tid = threadIdx.x, t = tid % LPR, lane0 = (tid & 63) - t;
    int bg, item;
    deal_head(blockIdx.x, rows_per_head, f.nbg, bg, item);
    bg += f.bg0;
    const int q0 = f.c * l.cq, nq = min(l.cq, l.n - q0);
    const int rr = item * (256 / LPR) + tid / LPR;
    const int row = min(rr, nq * G - 1);          // (lanes without a row follow the last one, and store nothing)
    const int i = q0 + row / G, gh = row % G, b = bg / l.Hkv, g = bg % l.Hkv;
    const int32_t* pos = l.pos + ((size_t)bg * l.n + i) * l.slots;
    const size_t rows0 = (size_t)(bg - f.bg0) * l.entries * G + gh;
    float M = -INFINITY;
    for (int s = t; s < l.slots; s += LPR) {
        const int p = pos[s];
        if (p >= 0) M = fmaxf(M, f.meta[rows0 + (size_t)p * G].x);
    }
#pragma unroll
    for (int d = 1; d < LPR; d <<= 1) M = fmaxf(M, __shfl_xor(M, d, 64));
    const float ref = M == -INFINITY ? 0.0f : M;
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0}, L = 0.0f;
    auto add = [&](auto stream, int s0) {
        const int p = s0 + t < l.slots ? pos[s0 + t] : -1;
        float w = 0.0f, ws = 0.0f;
        if (p >= 0) {
            const float2 mt = f.meta[rows0 + (size_t)p * G];
            w = __builtin_amdgcn_exp2f(mt.x - ref);
            ws = w * (mt.y * 0x1p-7f);   // (up to 65 results: their sum before the division stays in fp32's range whatever the values)
        }
        L += w;
        const int count = min(LPR, l.slots - s0);
#pragma unroll 4
        for (int s = 0; s < count; s++) {
            const int ps = __shfl(p, lane0 + s, 64);
            const float wss = __shfl(ws, lane0 + s, 64);
            if (ps < 0) continue;
            const f16x8* at = (const f16x8*)(f.part + (rows0 + (size_t)ps * G) * D + 8 * t);
            f16x8 v;
            if constexpr (stream) v = __builtin_nontemporal_load(at);
            else v = *at;
#pragma unroll
            for (int e = 0; e < 8; e++) acc[e] = fmaf(wss, (float)v[e], acc[e]);
        }
    };
    if (f.stream)
        for (int s0 = 0; s0 < l.slots; s0 += LPR) add(std::true_type{}, s0);
    else
        for (int s0 = 0; s0 < l.slots; s0 += LPR) add(std::false_type{}, s0);
#pragma unroll
    for (int d = 1; d < LPR; d <<= 1) L += __shfl_xor(L, d, 64);
    if (rr >= nq * G) return;
    const float inv = 0x1p7f / L;
    const size_t at = ((size_t)b * l.H + g * G + gh) * l.n + i;
    u32x4 out;
#pragma unroll
    for (int e = 0; e < 4; e++) out[e] = pack_bf16x2(acc[2 * e] * inv, acc[2 * e + 1] * inv);
    __builtin_nontemporal_store(out, (u32x4*)(f.o + at * D + 8 * t));
    // (L = 0: logits of -inf alone, of a query that is not finite; any other row has a weight of 1 among its blocks)
    if (t == 0) f.lse[at] = L == 0.0f ? __uint_as_float(0x7FC00000u) : (ref + log2f(L)) * 0.6931471805599453f;
}

// mass_j: the weights that the block's keys got from the stretch's queries and the heads of the group join what earlier stretches gave.
// A workgroup per block; the order of the sum is fixed.
__global__ __launch_bounds__(256) void block_mass_kernel(BlockFwd f)
{
    __shared__ float red[4];
    const BlockLists& l = f.a.l;
    const int j = blockIdx.x, bg = f.bg0 + blockIdx.y, tid = threadIdx.x, G = l.G, b = bg / l.Hkv, g = bg % l.Hkv;
    const size_t cbg = l.cbg(f.c, bg), h0 = (size_t)b * l.H + g * G;
    const int rows = l.total[cbg * l.nb + j] * G, base = l.base[cbg * l.nb + j];
    const int32_t* list = l.list + cbg * l.entries + base;
    const float2* meta = f.meta + ((size_t)blockIdx.y * l.entries + base) * G;
    float sum = 0.0f;
#pragma unroll 4
    for (int r = tid; r < rows; r += 256) sum += __builtin_amdgcn_exp2f(meta[r].x - f.lse[(h0 + r % G) * l.n + list[r / G]] * 1.4426950408889634f);
    sum = wave_sum_f32(sum);
    if ((tid & 63) == 0) red[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) {
        sum = (red[0] + red[1]) + (red[2] + red[3]);
        float* m = f.mass + (size_t)bg * l.nb + j;
        *m = j < f.c * (l.cq / BT) ? *m + sum : sum;   // (a block's first stretch is the one it lies in)
    }
}

// Queries per stretch and heads per launch: what they leave behind is at most FWD_STRETCH_BYTES of workspace.  As many queries as fit
// come first, because all the rows that a stretch has for a block share one load of K and V.  (Stretches whose results would stay in
// the chip's last cache, of 256 MB, do not pay: 32 heads of 32768, 16 blocks: 3.28 ms with 256 MB and 2.94 with 1 GB against 2.70 in one.)
static int fwd_stretch(const sparsek_block_cfg& c)
{
    const double per_query = (double)(c.H / c.Hkv) * (c.top + 1) * c.d * 2, blocks = block_count(c.n);
    const double stretches = std::ceil(blocks / std::max(1.0, std::floor(FWD_STRETCH_BYTES / per_query / BT)));
    return (int)std::ceil(blocks / stretches) * BT;
}
static int fwd_heads(const sparsek_block_cfg& c, int cq)
{
    const double per_head = (double)std::min(cq, c.n) * (c.H / c.Hkv) * (c.top + 1) * c.d * 2;
    return (int)std::max(1.0, std::min((double)c.B * c.Hkv, std::floor(FWD_STRETCH_BYTES / per_head)));
}

// Rows that share a block's K and V in LDS: more of them where that leaves three workgroups for every compute unit, and beyond 512 four
// rounds of those (32 heads of 32768, 16 blocks: 2695 us with 512, 2631 with 1024, 2597 with 2048, 2591 with 4096; two prompts of 16
// heads of 5003: 299.5 with 512, 301 with 1024).
static int fwd_unit(const sparsek_block_cfg& c)
{
    const double rows = (double)c.B * c.H * c.n * (c.top + 1);
    return rows >= 768 * 8192.0 ? 2048 : rows >= 768 * 4096.0 ? 1024 : rows >= 768 * 512.0 ? 512 : rows >= 768 * 256.0 ? 256 : 128;
}

struct FwdLayout {
    BlockLayout y;
    int heads;
    size_t part, meta, bytes;
};
static FwdLayout fwd_layout(const sparsek_block_cfg& c, void* ws)
{
    FwdLayout f;
    const int cq = fwd_stretch(c);
    f.y = block_lists_layout(c, cq, fwd_unit(c), ws);
    f.heads = fwd_heads(c, cq);
    const size_t rows = (size_t)f.heads * f.y.l.entries * f.y.l.G;
    f.part = f.y.bytes;
    f.meta = align_up(f.part + rows * c.d * 2, 256);
    f.bytes = align_up(f.meta + rows * 8, 256);
    return f;
}

size_t block_fwd_ws_bytes(const sparsek_block_cfg& c) { return fwd_layout(c, nullptr).bytes; }

int launch_block_fwd(const sparsek_block_cfg& c, const void* q, const void* k, const void* v, const int32_t* idx, void* o, float* lse,
                     float* mass, void* ws, hipStream_t st)
{
    const FwdLayout y = fwd_layout(c, ws);
    BlockFwd f;
    f.a.l = y.y.l;
    f.a.q = (const uint16_t*)q; f.a.k = (const uint16_t*)k; f.a.v = (const uint16_t*)v;
    f.a.scale = c.softmax_scale;
    f.a.c2 = c.softmax_scale * 1.4426950408889634f;
    f.o = (uint16_t*)o; f.lse = lse; f.mass = mass;
    f.part = (_Float16*)((char*)ws + y.part); f.meta = (float2*)((char*)ws + y.meta);
    const BlockLists& l = f.a.l;
    const int BG = c.B * c.Hkv;
    if (int rc = launch_block_lists(l, idx, st)) return rc;
    for (f.bg0 = 0; f.bg0 < BG; f.bg0 += y.heads)
        for (f.c = 0; f.c < l.nc; f.c++) {
            f.nbg = std::min(y.heads, BG - f.bg0);
            // (two prompts of 16 heads of 5003, 533 MB: 370 us as they are, 296 streamed; 48 heads of 2000, 61 MB: the join alone 14.5 and 18.4)
            f.stream = (double)f.nbg * l.entries * l.G * c.d * 2 > 256e6;
            const int nq = std::min(l.cq, c.n - f.c * l.cq), seen = std::min(l.nb, (f.c + 1) * (l.cq / BT));
            const int items = (int)(((long long)nq * l.G * (c.d / 8) + 255) / 256);
#define FWD(D)                                                                                                   \
    hipLaunchKernelGGL((block_tiles_kernel<D>), dim3((unsigned)l.maxu * f.nbg), dim3(256), 0, st, f);            \
    hipLaunchKernelGGL((block_join_kernel<D>), dim3((unsigned)items * f.nbg), dim3(256), 0, st, f, items)
            if (c.d == 128) {
                FWD(128);
            } else {
                FWD(64);
            }
#undef FWD
            if (mass) hipLaunchKernelGGL(block_mass_kernel, dim3(seen, f.nbg), dim3(256), 0, st, f);
        }
    return launch_status();
}

}  // namespace spk
