// Attention over the blocks of 64 tokens that every query selected, and over the query's own block (forward).
//
// Queries that lie side by side select different blocks, so a tile of queries against the union of their blocks would do
// several times the work.  The kernels go by key block instead: block_tiles_kernel takes a block's K and V into LDS once and
// walks the queries that selected it, 32 rows (query, head of the group) to a wave: S^T = K.Q^T, the softmax of these 64 keys alone,
// O^T = V^T.P^T, and leaves the normalised partial result, with the log of its denominator, in list order.  block_join_kernel takes
// 64 queries at a time, does their own block (causal) in the same way and adds the partial results with their weights.
// What bounds it is memory: a selected (row, block) pair moves D halves out and in again and a row of q in, for 4*64*D flops.
#include "block_parts.hpp"

namespace spk {

// ---- the lists ----

__global__ __launch_bounds__(256) void block_masks_zero_kernel(u32x4* p, size_t n16)
{
    for (size_t x = blockIdx.x * (size_t)256 + threadIdx.x; x < n16; x += (size_t)gridDim.x * 256) p[x] = u32x4{0, 0, 0, 0};
}

__global__ __launch_bounds__(256) void block_masks_kernel(BlockLists l, const int32_t* __restrict__ idx)
{
    const int bg = blockIdx.y;
    const size_t x = blockIdx.x * (size_t)256 + threadIdx.x;
    if (x >= (size_t)l.n * l.top) return;
    const int i = (int)(x / l.top), c = i / BT, j = idx[(size_t)bg * l.n * l.top + x];
    if (j >= 0 && j < c) atomicOr(&l.masks[((size_t)bg * l.nb + c) * l.nb + j], 1ull << (i % BT));
}

// off and total: a workgroup of 1024 per 64 blocks, its 16 waves share the chunks.
__global__ __launch_bounds__(1024) void block_offsets_kernel(BlockLists l)
{
    __shared__ int part[16][64];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, j = blockIdx.x * 64 + lane, bg = blockIdx.y;
    const int jc = min(j, l.nb - 1);
    const int per = (l.nb + 15) / 16, c0 = wv * per, c1 = min(l.nb, c0 + per);
    const unsigned long long* m = l.masks + (size_t)bg * l.nb * l.nb + jc;
    int sum = 0;
#pragma unroll 8
    for (int c = c0; c < c1; c++) sum += __popcll(m[(size_t)c * l.nb]);
    part[wv][lane] = sum;
    __syncthreads();
    int run = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 16; w++) {
        run += w < wv ? part[w][lane] : 0;
        all += part[w][lane];
    }
    if (j >= l.nb) return;
    int32_t* off = l.off + (size_t)bg * l.nb * l.nb + j;
#pragma unroll 8
    for (int c = c0; c < c1; c++) {
        off[(size_t)c * l.nb] = run;
        run += __popcll(m[(size_t)c * l.nb]);
    }
    if (wv == 0) l.total[(size_t)bg * l.nb + j] = all;
}

// base and units: a workgroup of 1024 per (batch, head).
__global__ __launch_bounds__(1024) void block_units_kernel(BlockLists l)
{
    __shared__ int2 wsum[16];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, bg = blockIdx.x;
    int2 done = make_int2(0, 0);   // list entries and units ahead of this round of 1024 blocks
    for (int j0 = 0; j0 < l.nb; j0 += 1024) {
        const int j = j0 + tid;
        const int mine = j < l.nb ? l.total[(size_t)bg * l.nb + j] : 0;
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
        if (j < l.nb) {
            l.base[(size_t)bg * l.nb + j] = before.x + s.x - mine;
            const int u0 = before.y + s.y - units;
            l.first_unit[(size_t)bg * l.nb + j] = u0;
            for (int u = 0; u < units; u++)
                if (u0 + u < l.maxu) l.units[(size_t)bg * l.maxu + u0 + u] = make_int2(j, u * l.unit);
        }
        done.x += all.x;
        done.y += all.y;
        __syncthreads();
    }
    if (tid == 0) l.nunits[bg] = min(done.y, l.maxu);
}

__global__ __launch_bounds__(256) void block_place_kernel(BlockLists l, const int32_t* __restrict__ idx)
{
    const int bg = blockIdx.y;
    const size_t x = blockIdx.x * (size_t)256 + threadIdx.x;
    if (x >= (size_t)l.n * l.top) return;
    const int i = (int)(x / l.top), s = (int)(x % l.top), c = i / BT;
    const int32_t* row = idx + ((size_t)bg * l.n + i) * l.top;
    const int j = row[s];
    bool ok = j >= 0 && j < c;
    for (int y = 0; y < s; y++) ok &= row[y] != j;   // (a repeated block counts once)
    int p = -1;
    if (ok) {
        const size_t cj = ((size_t)bg * l.nb + c) * l.nb + j;
        p = l.base[(size_t)bg * l.nb + j] + l.off[cj] + __popcll(l.masks[cj] & ((1ull << (i % BT)) - 1));
        l.list[(size_t)bg * l.pairs + p] = i;
    }
    l.pos[(size_t)bg * l.n * l.top + x] = p;
}

int launch_block_lists(const BlockLists& l, const int32_t* idx, hipStream_t st)
{
    if (!l.pairs) {   // nobody has a block behind it to select, but the slots are read
        if (l.top) hipLaunchKernelGGL(block_place_kernel, dim3((unsigned)(((size_t)l.n * l.top + 255) / 256), l.B * l.Hkv), dim3(256), 0, st, l, idx);
        return launch_status();
    }
    const int BG = l.B * l.Hkv;
    const size_t n16 = align_up((size_t)BG * l.nb * l.nb * 8, 256) / 16;
    hipLaunchKernelGGL(block_masks_zero_kernel, dim3((unsigned)std::min<size_t>(2048, (n16 + 255) / 256)), dim3(256), 0, st, (u32x4*)l.masks, n16);
    const dim3 pairs((unsigned)(((size_t)l.n * l.top + 255) / 256), BG);
    hipLaunchKernelGGL(block_masks_kernel, pairs, dim3(256), 0, st, l, idx);
    hipLaunchKernelGGL(block_offsets_kernel, dim3((l.nb + 63) / 64, BG), dim3(1024), 0, st, l);
    hipLaunchKernelGGL(block_units_kernel, dim3(BG), dim3(1024), 0, st, l);
    hipLaunchKernelGGL(block_place_kernel, pairs, dim3(256), 0, st, l, idx);
    return launch_status();
}

// ---- the forward ----

struct BlockFwd {
    BlockArgs a;
    uint16_t* o;
    float* lse;
    _Float16* part;    // [entry rows][D], a row as the two lanes of its column hold it: [lane / 32][D / 2]
    float2* meta;      // log2 of the denominator, and the factor that the halves stand for
    float* own;        // the same log2 for every query's own block [B,H,n]
    float* mass;       // [B,Hkv,nb] or null
};

// One tile of 32 rows against the block's keys: S^T = K.Q^T for NKH halves of 32 keys, softmax, O^T = V^T.P^T.  A lane has one
// column (row of q).  causal >= 0: the column sees keys 0 .. causal of the block.
template <int D, int NKH, bool CAUSAL>
__device__ __forceinline__ void block_column(uint32_t rk, uint32_t tv, const bf16x8 (&qf)[D / 16], float c2, int causal, int half,
                                             f32x16 (&acc)[D / 32], float& m, float& l)
{
    using S = RowTile<D>;
    constexpr int DS = D / 16, DB = D / 32;
    f32x16 s[NKH];
#pragma unroll
    for (int kh = 0; kh < NKH; kh++) {
        s[kh] = f32x16{0};
#pragma unroll
        for (int x = 0; x < DS; x++) s[kh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_operand(rk + 2 * kh * S::R16 + 32 * x), qf[x], s[kh], 0, 0, 0);
    }
    m = -INFINITY;
#pragma unroll
    for (int kh = 0; kh < NKH; kh++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
            if (CAUSAL && 32 * kh + 8 * (r / 4) + 4 * half + r % 4 > causal) s[kh][r] = -INFINITY;
            m = fmaxf(m, s[kh][r]);
        }
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    m = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * c2;
    const float ref = m == -INFINITY ? 0.0f : m;
    l = 0.0f;
    bf16x8 pb[NKH][2];
#pragma unroll
    for (int kh = 0; kh < NKH; kh++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[kh][r], c2, -ref));
            l += p;
            pb[kh][r >> 3][r & 7] = (__bf16)p;   // the operand of the second product: 2^-9 of every weight, as in the other attention kernels
        }
    const auto sl = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(sl[0]) + __uint_as_float(sl[1]);
#pragma unroll
    for (int x = 0; x < DB; x++) acc[x] = f32x16{0};
#pragma unroll
    for (int g = 0; g < 2 * NKH; g++)
#pragma unroll
        for (int x = 0; x < DB; x++)
            acc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_operand<D>(tv + g * S::R16 + 64 * x), pb[g >> 1][g & 1], acc[x], 0, 0, 0);
}

template <int D>
struct FwdBlockSmem {
    unsigned char k[RowTile<D>::BYTES], v[RowTile<D>::BYTES];
    unsigned red[4];
};

template <int D>
__global__ __launch_bounds__(256, 2) void block_tiles_kernel(BlockFwd f)
{
    __shared__ __attribute__((aligned(16))) FwdBlockSmem<D> sm;
    const BlockLists& l = f.a.l;
    const int bg = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, col = lane & 31, half = lane >> 5;
    if ((int)blockIdx.x >= l.nunits[bg]) return;
    const int2 u = l.units[(size_t)bg * l.maxu + blockIdx.x];
    const int j = u.x, first = u.y, G = l.G;
    const int base = l.base[(size_t)bg * l.nb + j];
    const int end = min(l.total[(size_t)bg * l.nb + j] * G, first + l.unit);
    const size_t kv = ((size_t)bg * l.n + (size_t)j * BT) * D;
    load_rows<D>(sm.k, f.a.k + kv, BT - 1, tid);
    load_rows<D>(sm.v, f.a.v + kv, BT - 1, tid);
    // the largest |v| of the block scales its partial results
    unsigned top = 0;
    for (int x = tid; x < BT * D / 8; x += 256) {
        const u32x4 y = *(const u32x4*)(f.a.v + kv + 8 * x);
#pragma unroll
        for (int e = 0; e < 4; e++) top = max(top, max(y[e] << 16 & 0x7FFFFFFFu, y[e] & 0x7FFF0000u));
    }
    const int E = scale_exp(block_max_bits(top, sm.red, tid));
    const float down = __uint_as_float((unsigned)(254 - E) << 23), up = __uint_as_float((unsigned)E << 23);
    const uint32_t rk = lds_address(sm.k) + row_lane<D>(lane), tv = lds_address(sm.v) + transposed_lane<D>(lane);
    const int b = bg / l.Hkv, g = bg % l.Hkv;
    const int32_t* list = l.list + (size_t)bg * l.pairs + base;
    const size_t row0 = ((size_t)bg * l.pairs + base) * G;
    for (int r0 = first + 32 * wv; r0 < end; r0 += 128) {
        const int r = r0 + col, rc = min(r, end - 1);
        const int i = list[rc / G], h = g * G + rc % G;
        const uint16_t* qr = f.a.q + (((size_t)b * l.H + h) * l.n + i) * D + 8 * half;
        bf16x8 qf[D / 16];
#pragma unroll
        for (int x = 0; x < D / 16; x++) qf[x] = *(const bf16x8*)(qr + 16 * x);
        f32x16 acc[D / 32];
        float m, den;
        block_column<D, 2, false>(rk, tv, qf, f.a.c2, 0, half, acc, m, den);
        if (r < end) {
            const float inv = den > 0.0f ? down / den : den;   // (nothing but -inf: weight 0 in the sum)
            _Float16* pr = f.part + (row0 + r) * D + half * (D / 2);
#pragma unroll
            for (int x = 0; x < D / 32; x++)
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    f16x8 v;
#pragma unroll
                    for (int e = 0; e < 8; e++) v[e] = (_Float16)(acc[x][8 * y + e] * inv);
                    *(f16x8*)(pr + 16 * x + 8 * y) = v;
                }
            if (half == 0) f.meta[row0 + r] = make_float2(m + log2f(den), up);
        }
    }
}

// 64 queries of a key/value head's group per workgroup: wave wv takes 32 of them (wv & 1) and every second head.
template <int D>
__global__ __launch_bounds__(256, 2) void block_join_kernel(BlockFwd f)
{
    __shared__ __attribute__((aligned(16))) FwdBlockSmem<D> sm;
    const BlockLists& l = f.a.l;
    const int bg = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, col = lane & 31, half = lane >> 5;
    const int qb = gridDim.x - 1 - blockIdx.x, G = l.G, b = bg / l.Hkv, g = bg % l.Hkv, qh = wv & 1;
    const size_t kv = ((size_t)bg * l.n + (size_t)qb * BT) * D;
    const int last = l.n - 1 - qb * BT;
    load_rows<D>(sm.k, f.a.k + kv, last, tid);
    load_rows<D>(sm.v, f.a.v + kv, last, tid);
    __syncthreads();
    const int i = qb * BT + 32 * qh + col, ic = min(i, l.n - 1);
    const uint32_t rk = lds_address(sm.k) + row_lane<D>(lane), tv = lds_address(sm.v) + transposed_lane<D>(lane);
    const int32_t* pos = l.pos + ((size_t)bg * l.n + ic) * l.top;
    for (int gh = wv >> 1; gh < G; gh += 2) {
        const size_t row = ((size_t)b * l.H + g * G + gh) * l.n + ic;
        const uint16_t* qr = f.a.q + row * D + 8 * half;
        bf16x8 qf[D / 16];
#pragma unroll
        for (int x = 0; x < D / 16; x++) qf[x] = *(const bf16x8*)(qr + 16 * x);
        f32x16 acc[D / 32];
        float m, den;
        if (qh == 0) block_column<D, 1, true>(rk, tv, qf, f.a.c2, col, half, acc, m, den);
        else block_column<D, 2, true>(rk, tv, qf, f.a.c2, 32 + col, half, acc, m, den);
        const size_t rows0 = (size_t)bg * l.pairs * G + gh;
        float M = m;
        if (i < l.n && half == 0) f.own[row] = m + log2f(den);
        for (int s = 0; s < l.top; s++) {
            const int p = pos[s];
            if (p >= 0) M = fmaxf(M, f.meta[rows0 + (size_t)p * G].x);
        }
        const float w0 = __builtin_amdgcn_exp2f(m - M);
        float L = den * w0;
#pragma unroll
        for (int x = 0; x < D / 32; x++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[x][r] *= w0;
        for (int s = 0; s < l.top; s++) {
            const int p = pos[s];
            if (p < 0) continue;
            const size_t pr = rows0 + (size_t)p * G;
            const float2 mt = f.meta[pr];
            const float w = __builtin_amdgcn_exp2f(mt.x - M), ws = w * mt.y;
            L += w;
            const _Float16* src = f.part + pr * D + half * (D / 2);
#pragma unroll
            for (int x = 0; x < D / 32; x++)
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    const f16x8 v = *(const f16x8*)(src + 16 * x + 8 * y);
#pragma unroll
                    for (int e = 0; e < 8; e++) acc[x][8 * y + e] = fmaf(ws, (float)v[e], acc[x][8 * y + e]);
                }
        }
        if (i < l.n) {
            const float inv = 1.0f / L;
            uint16_t* orow = f.o + row * D + 4 * half;
#pragma unroll
            for (int x = 0; x < D / 32; x++)
#pragma unroll
                for (int y = 0; y < 4; y++) {
                    const uint2 v = make_uint2(pack_bf16x2(acc[x][4 * y] * inv, acc[x][4 * y + 1] * inv), pack_bf16x2(acc[x][4 * y + 2] * inv, acc[x][4 * y + 3] * inv));
                    *(uint2*)(orow + 32 * x + 8 * y) = v;
                }
            if (half == 0) f.lse[row] = (M + log2f(L)) * 0.6931471805599453f;
        }
    }
}

// mass_j = the weights that the block's keys got from all queries and heads of the group.  A workgroup per block; the order of
// the sum is fixed.
__global__ __launch_bounds__(256) void block_mass_kernel(BlockFwd f)
{
    __shared__ float red[4];
    const BlockLists& l = f.a.l;
    const int j = blockIdx.x, bg = blockIdx.y, tid = threadIdx.x, G = l.G, b = bg / l.Hkv, g = bg % l.Hkv;
    const float LOG2E = 1.4426950408889634f;
    const size_t h0 = (size_t)b * l.H + g * G;
    float sum = 0.0f;
    const int own = min(BT, l.n - j * BT) * G;
    for (int r = tid; r < own; r += 256) {
        const size_t row = (h0 + r % G) * l.n + j * BT + r / G;
        sum += __builtin_amdgcn_exp2f(f.own[row] - f.lse[row] * LOG2E);
    }
    const int rows = l.pairs ? l.total[(size_t)bg * l.nb + j] * G : 0;
    if (rows) {
        const int base = l.base[(size_t)bg * l.nb + j];
        const int32_t* list = l.list + (size_t)bg * l.pairs + base;
        const float2* meta = f.meta + ((size_t)bg * l.pairs + base) * G;
        for (int r = tid; r < rows; r += 256) sum += __builtin_amdgcn_exp2f(meta[r].x - f.lse[(h0 + r % G) * l.n + list[r / G]] * LOG2E);
    }
    sum = wave_sum_f32(sum);
    if ((tid & 63) == 0) red[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) f.mass[(size_t)bg * l.nb + j] = (red[0] + red[1]) + (red[2] + red[3]);
}

constexpr int FWD_UNIT = 256;   // rows that share a block's K and V in LDS

struct FwdLayout {
    BlockLayout y;
    size_t part, meta, own, bytes;
};
static FwdLayout fwd_layout(const sparsek_block_cfg& c, void* ws)
{
    FwdLayout f;
    f.y = block_lists_layout(c, FWD_UNIT, ws);
    const size_t rows = (size_t)c.B * c.Hkv * f.y.l.pairs * f.y.l.G;
    f.part = f.y.bytes;
    f.meta = align_up(f.part + rows * c.d * 2, 256);
    f.own = align_up(f.meta + rows * 8, 256);
    f.bytes = align_up(f.own + (size_t)c.B * c.H * c.n * 4, 256);
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
    f.part = (_Float16*)((char*)ws + y.part); f.meta = (float2*)((char*)ws + y.meta); f.own = (float*)((char*)ws + y.own);
    const BlockLists& l = f.a.l;
    const int BG = c.B * c.Hkv;
    if (int rc = launch_block_lists(l, idx, st)) return rc;
#define FWD(D)                                                                                                \
    if (l.maxu) hipLaunchKernelGGL((block_tiles_kernel<D>), dim3(l.maxu, BG), dim3(256), 0, st, f);           \
    hipLaunchKernelGGL((block_join_kernel<D>), dim3(l.nb, BG), dim3(256), 0, st, f)
    if (c.d == 128) {
        FWD(128);
    } else {
        FWD(64);
    }
#undef FWD
    if (mass) hipLaunchKernelGGL(block_mass_kernel, dim3(l.nb, BG), dim3(256), 0, st, f);
    return launch_status();
}

}  // namespace spk
