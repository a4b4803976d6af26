// Attention over selected blocks of 64 tokens, backward: with p_ij = exp(s_ij - lse_i), delta_i = dO_i.o_i and
// ds_ij = p_ij (dO_i.v_j - delta_i) scale:  dq_i = sum_j ds_ij k_j,  dk_j = sum_i ds_ij q_i,  dv_j = sum_i p_ij dO_i.
//
// By key block, like the forward (see block_attn.hip).  block_bwd_tiles_kernel holds a block's K and V in LDS and walks the
// rows that attend it, 64 at a time: S = Q.K^T and dP = dO.V^T with a lane per key, so that P and dS are the operands of
// dV^T += dO^T.P and dK^T += Q^T.dS as they stand (sums stay in registers for a whole unit of rows); dS passes through LDS for
// dQ^T = K^T.dS^T, whose partial results go out in list order.  A block whose rows are one unit is finished there; the sums of
// the others go out and block_kv_join_kernel adds them up.  block_dq_join_kernel adds up the partial dq of every row.
//
// The tiles are bound by issue and by waiting: two waves per SIMD (256 registers for d = 128) and five products a pair, three of them in two
// parts.  4 x 16 heads of 128, 8192 tokens, 8 blocks: 930 to 1000 us (matrix pipes 34 %, vector ALU 37 %, LDS 31 % of the time); dO.o 53 us
// (5.1 TB/s), the join of dq 277 (4.7 TB/s).
#include "block_parts.hpp"

namespace spk {

struct BlockBwd {
    BlockArgs a;
    uint16_t *dq, *dk, *dv;
    float2* rows;       // [B,H,n]: lse * log2(e), dO.o
    _Float16* part;     // partial dq: [B,Hkv][entry rows][D]
    float2* meta;       // what the halves of each half of D stand for
    float* kvpart;      // [B,Hkv][units][2 halves of the keys][dV, dK][D / 32][4][64 lanes][4]
};

// dO.o and the logarithm of the denominator, a wave per 64 / (D / 8) rows.
template <int D>
__global__ __launch_bounds__(256) void block_delta_kernel(BlockBwd f, size_t nrows)
{
    constexpr int LPR = D / 8;
    const size_t row = (blockIdx.x * (size_t)256 + threadIdx.x) / LPR;
    const int c = threadIdx.x % LPR;
    float s = 0.0f;
    if (row < nrows) {
        const u32x4 x = *(const u32x4*)(f.a.o + row * D + 8 * c), y = *(const u32x4*)(f.a.dO + row * D + 8 * c);
#pragma unroll
        for (int e = 0; e < 4; e++) {
            s = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), s);
            s = fmaf(__uint_as_float(x[e] & 0xFFFF0000u), __uint_as_float(y[e] & 0xFFFF0000u), s);
        }
    }
#pragma unroll
    for (int d = 1; d < LPR; d <<= 1) s += __shfl_xor(s, d, 64);
    if (row < nrows && c == 0) f.rows[row] = make_float2(f.a.lse[row] * 1.4426950408889634f, s);
}

template <int D>
struct BwdBlockSmem {
    unsigned char k[RowTile<D>::BYTES], v[RowTile<D>::BYTES], q[RowTile<D>::BYTES], g[RowTile<D>::BYTES];   // g: dO
    unsigned char ds[RowTile<64>::BYTES];   // [key][row]
    struct Rows {                           // of one tile
        float lse2[BT], delta[BT];
        int limit[BT];                      // keys 0 .. limit are attended; BT more: one of the block's own rows that is not finite
        int at[BT];                         // the row's place in [G,n]
        unsigned bad[2];                    // rows whose lse or dO.o is not finite, as bits
    } rows[2];                              // the tile in use and the next one
};
static_assert(sizeof(BwdBlockSmem<128>) <= 80 * 1024, "two workgroups per CU");

// The rows of a tile on their way to the q and g tiles: untracked direct-to-LDS loads, a wave-load per group of rows.
template <int D>
__device__ __forceinline__ void issue_query_rows(BwdBlockSmem<D>& sm, const typename BwdBlockSmem<D>::Rows& rows, const uint16_t* q, const uint16_t* dO,
                                                 int wv, int lane)
{
    using S = RowTile<D>;
    constexpr int LPR = D / 8;
#pragma unroll
    for (int x = 0; x < S::NL / 4; x++) {
        const int L = wv + 4 * x;
        const size_t off = (size_t)rows.at[S::row(L, lane / LPR)] * D + 8 * (lane % LPR);
        async_load_lds16_from(q + off, sm.q + L * S::GS);
        async_load_lds16_from(dO + off, sm.g + L * S::GS);
    }
}

// 64 rows against 64 keys.  Wave (kb = wv & 1, rb = wv >> 1): keys 32 kb .. and rows 32 rb .. of S and dP; its share of dV^T and
// dK^T (those keys, those rows) joins acc_v, acc_k.  Weights are the sum of two bf16 numbers (2^-16): as one, 2^-8, they leave dV 1.4 times
// the error of its own rounding (for 3 % of a training step).  Score gradients cancel in their sums (a row's add up to 0), so dS is two
// bf16 numbers too, and of any size, as the keys and values of a block may be: fp16 relative to a bound of the row's goes by values that
// the row may not attend, and takes as long (4 x 16 heads of 8192 1953 us against 1942).  The first is in LDS then, the second in dl.
template <int D>
__device__ __forceinline__ void bwd_block_tile(BwdBlockSmem<D>& sm, const typename BwdBlockSmem<D>::Rows& rows, int lane, int wv, bool own, float c2,
                                               f32x16 (&acc_v)[D / 32], f32x16 (&acc_k)[D / 32], bf16x8 (&dl)[2])
{
    using S = RowTile<D>;
    constexpr int DS = D / 16, DB = D / 32;
    const int kb = wv & 1, rb = wv >> 1, col = lane & 31, half = lane >> 5;
    const uint32_t rk = lds_address(sm.k) + row_lane<D>(lane) + 2 * kb * S::R16, rv = lds_address(sm.v) + row_lane<D>(lane) + 2 * kb * S::R16;
    const uint32_t rq = lds_address(sm.q) + row_lane<D>(lane) + 2 * rb * S::R16, rg = lds_address(sm.g) + row_lane<D>(lane) + 2 * rb * S::R16;
    f32x16 s = {0}, dp = {0};
#pragma unroll
    for (int x = 0; x < DS; x++) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_operand(rq + 32 * x), row_operand(rk + 32 * x), s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row_operand(rg + 32 * x), row_operand(rv + 32 * x), dp, 0, 0, 0);
    }
    if (own)   // (some of the rows are the block's own queries)
#pragma unroll
        for (int g4 = 0; g4 < 4; g4++) {
            const int4 L4 = *(const int4*)&rows.limit[32 * rb + 8 * g4 + 4 * half];
            const int ll[4] = {L4.x, L4.y, L4.z, L4.w};
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float x = ll[e] < BT ? s[4 * g4 + e] : __uint_as_float(0x7FC00000u);
                const bool behind = 32 * kb + col > (ll[e] & BT - 1);
                s[4 * g4 + e] = behind ? -INFINITY : x;
                dp[4 * g4 + e] = behind ? 0.0f : dp[4 * g4 + e];   // (infinite, perhaps: values that the row does not attend)
            }
        }
    bf16x8 pb[2], pl[2], db[2];
#pragma unroll
    for (int g4 = 0; g4 < 4; g4++) {
        const int r0 = 32 * rb + 8 * g4 + 4 * half;
        const float4 L4 = *(const float4*)&rows.lse2[r0], D4 = *(const float4*)&rows.delta[r0];
        const float ll[4] = {L4.x, L4.y, L4.z, L4.w}, dd[4] = {D4.x, D4.y, D4.z, D4.w};
        bf16x4 first;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int r = 4 * g4 + e;
            const float p = __builtin_amdgcn_exp2f(fmaf(s[r], c2, -ll[e]));
            const float ds = p * (dp[r] - dd[e]);
            pb[r >> 3][r & 7] = (__bf16)p;
            pl[r >> 3][r & 7] = (__bf16)(p - (float)pb[r >> 3][r & 7]);
            db[r >> 3][r & 7] = first[e] = (__bf16)ds;
            dl[r >> 3][r & 7] = (__bf16)(ds - (float)first[e]);
        }
        *(bf16x4*)(sm.ds + RowTile<64>::offset(32 * kb + col) + 2 * r0) = first;
    }
    const uint32_t tq = lds_address(sm.q) + transposed_lane<D>(lane) + 2 * rb * S::R16, tg = lds_address(sm.g) + transposed_lane<D>(lane) + 2 * rb * S::R16;
#pragma unroll
    for (int g = 0; g < 2; g++)
#pragma unroll
        for (int x = 0; x < DB; x++) {
            const bf16x8 gt = transposed_operand<D>(tg + g * S::R16 + 64 * x);
            acc_v[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(gt, pb[g], acc_v[x], 0, 0, 0);
            acc_v[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(gt, pl[g], acc_v[x], 0, 0, 0);
            const bf16x8 qt = transposed_operand<D>(tq + g * S::R16 + 64 * x);
            acc_k[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qt, db[g], acc_k[x], 0, 0, 0);
            acc_k[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qt, dl[g], acc_k[x], 0, 0, 0);
        }
}

// dQ^T of rows 32 rb .. and the D/2 columns of half kb: the two numbers of dS pass through LDS one after the other (two barriers).
template <int D>
__device__ __forceinline__ void bwd_block_dq(BwdBlockSmem<D>& sm, int lane, int wv, float scale, const bf16x8 (&dl)[2], f32x16 (&acc_q)[D / 64])
{
    constexpr int DB = D / 32;
    const int kb = wv & 1, rb = wv >> 1, col = lane & 31, half = lane >> 5;
    const uint32_t tk = lds_address(sm.k) + transposed_lane<D>(lane) + 64 * (DB / 2) * kb, td = lds_address(sm.ds) + transposed_lane<64>(lane) + 64 * rb;
#pragma unroll
    for (int x = 0; x < DB / 2; x++) acc_q[x] = f32x16{0};
#pragma unroll 1
    for (int part = 0; part < 2; part++) {
        if (part) {
            __syncthreads();   // the first numbers have been read
#pragma unroll
            for (int g4 = 0; g4 < 4; g4++) {
                bf16x4 w;
#pragma unroll
                for (int e = 0; e < 4; e++) w[e] = dl[g4 >> 1][4 * (g4 & 1) + e];
                *(bf16x4*)(sm.ds + RowTile<64>::offset(32 * kb + col) + 2 * (32 * rb + 8 * g4 + 4 * half)) = w;
            }
            __syncthreads();
        }
#pragma unroll
        for (int g = 0; g < 4; g++) {
            const bf16x8 d8 = transposed_operand<64>(td + g * RowTile<64>::R16);
#pragma unroll
            for (int x = 0; x < DB / 2; x++)
                acc_q[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed_operand<D>(tk + g * RowTile<D>::R16 + 64 * x), d8, acc_q[x], 0, 0, 0);
        }
    }
#pragma unroll
    for (int x = 0; x < DB / 2; x++)
#pragma unroll
        for (int r = 0; r < 16; r++) acc_q[x][r] *= scale;
}

// The two row halves' shares of dV^T and dK^T are added up in LDS (over the q, g tiles and what follows); waves 0 and 1 have the sums.
template <int D>
__device__ __forceinline__ void add_row_halves(BwdBlockSmem<D>& sm, int lane, int wv, f32x16 (&acc_v)[D / 32], f32x16 (&acc_k)[D / 32])
{
    float4* buf = (float4*)&sm + (wv & 1) * (2 * (D / 32) * 4 * 64);
    __syncthreads();
    if (wv >= 2) {
#pragma unroll
        for (int x = 0; x < D / 32; x++)
#pragma unroll
            for (int y = 0; y < 4; y++) {
                buf[(x * 4 + y) * 64 + lane] = make_float4(acc_v[x][4 * y], acc_v[x][4 * y + 1], acc_v[x][4 * y + 2], acc_v[x][4 * y + 3]);
                buf[((D / 32 + x) * 4 + y) * 64 + lane] = make_float4(acc_k[x][4 * y], acc_k[x][4 * y + 1], acc_k[x][4 * y + 2], acc_k[x][4 * y + 3]);
            }
    }
    __syncthreads();
    if (wv < 2) {
#pragma unroll
        for (int x = 0; x < D / 32; x++)
#pragma unroll
            for (int y = 0; y < 4; y++) {
                const float4 a = buf[(x * 4 + y) * 64 + lane], b = buf[((D / 32 + x) * 4 + y) * 64 + lane];
                acc_v[x][4 * y] += a.x; acc_v[x][4 * y + 1] += a.y; acc_v[x][4 * y + 2] += a.z; acc_v[x][4 * y + 3] += a.w;
                acc_k[x][4 * y] += b.x; acc_k[x][4 * y + 1] += b.y; acc_k[x][4 * y + 2] += b.z; acc_k[x][4 * y + 3] += b.w;
            }
    }
}
static_assert(2 * 2 * 4 * 4 * 64 * 16 <= sizeof(BwdBlockSmem<128>) && 2 * 2 * 2 * 4 * 64 * 16 <= sizeof(BwdBlockSmem<64>), "room for the sums");

// dV and dK of 32 keys, as the lanes of waves 0 and 1 hold them, to their rows.
template <int D>
__device__ __forceinline__ void store_kv(const BlockBwd& f, size_t kv, int key, int last, int half, const f32x16 (&acc_v)[D / 32], const f32x16 (&acc_k)[D / 32])
{
    if (key > last) return;
    uint16_t *ok = f.dk + kv + (size_t)key * D + 4 * half, *ov = f.dv + kv + (size_t)key * D + 4 * half;
    const float c = f.a.scale;
#pragma unroll
    for (int x = 0; x < D / 32; x++)
#pragma unroll
        for (int y = 0; y < 4; y++) {
            *(uint2*)(ov + 32 * x + 8 * y) = make_uint2(pack_bf16x2(acc_v[x][4 * y], acc_v[x][4 * y + 1]), pack_bf16x2(acc_v[x][4 * y + 2], acc_v[x][4 * y + 3]));
            *(uint2*)(ok + 32 * x + 8 * y) = make_uint2(pack_bf16x2(acc_k[x][4 * y] * c, acc_k[x][4 * y + 1] * c), pack_bf16x2(acc_k[x][4 * y + 2] * c, acc_k[x][4 * y + 3] * c));
        }
}

template <int D>
__global__ __launch_bounds__(256, D == 128 ? 2 : 3) void block_bwd_tiles_kernel(BlockBwd f)
{
    __shared__ __attribute__((aligned(16))) BwdBlockSmem<D> sm;
    constexpr int DB = D / 32;
    const BlockLists& l = f.a.l;
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
    int bg, un;
    deal_head(blockIdx.x, l.maxu, l.B * l.Hkv, bg, un);
    if (un >= l.nunits[bg]) return;
    const int2 u = l.order[(size_t)bg * l.maxu + un];
    const int j = u.x, first = u.y, G = l.G, b = bg / l.Hkv, g = bg % l.Hkv;
    const int base = l.base[(size_t)bg * l.nb + j], rows = l.total[(size_t)bg * l.nb + j] * G, end = min(rows, first + l.unit);
    const size_t kv = ((size_t)bg * l.n + (size_t)j * BT) * D;
    const int last = l.n - 1 - j * BT;
    // (rows that attend a key which is not finite have an lse or an o that is not, and the others must not see it)
    unsigned unused = 0;
    load_rows<D>(sm.k, f.a.k + kv, last, tid, unused);
    load_rows<D>(sm.v, f.a.v + kv, last, tid, unused);
    const int32_t* list = l.list + (size_t)bg * l.entries + base;
    const size_t row0 = ((size_t)bg * l.entries + base) * G, head0 = (size_t)b * l.H + g * G;
    const uint16_t *q0 = f.a.q + head0 * l.n * D, *g0 = f.a.dO + head0 * l.n * D;
    const float2* meta_in = f.rows + head0 * l.n;
    const int own_end = min(BT, last + 1) * G, kb = wv & 1, rt = 32 * (wv >> 1) + col;
    // A tile's rows are on their way while the dQ of the tile before is formed; what is known of them (by the first wave, a row to a
    // lane) two tiles ahead (the query) and one (its logarithm and dO.o).
    auto entry = [&](int r) { return list[min(r, end - 1) / G]; };
    auto place = [&](int r, int i) { return min(r, end - 1) % G * l.n + i; };
    auto put = [&](typename BwdBlockSmem<D>::Rows& rows, int r, int i, float2 m) {
        const bool bad = r < end && !(fabsf(m.x) < INFINITY && fabsf(m.y) < INFINITY);   // (a dO that is not finite leaves no dO.o finite)
        const unsigned long long all = __ballot(bad);
        if (lane < 2) rows.bad[lane] = (unsigned)(all >> (32 * lane));
        // such a row: weights of NaN for the keys that it attends (all of a selected block, in the own block by `limit`), q and dO of 0
        if (bad) m = make_float2(r < own_end ? 0.0f : __uint_as_float(0x7FC00000u), 0.0f);
        rows.lse2[lane] = r < end ? m.x : INFINITY;   // (a row that does not exist: p = 0)
        rows.delta[lane] = r < end ? m.y : 0.0f;
        rows.limit[lane] = min(BT - 1, i - j * BT) + (bad && r < own_end ? BT : 0);
        rows.at[lane] = place(r, i);
    };
    int i_next = 0;
    if (wv == 0) {
        const int i = entry(first + lane);
        i_next = entry(first + BT + lane);
        put(sm.rows[0], first + lane, i, meta_in[place(first + lane, i)]);
    }
    f32x16 acc_v[DB], acc_k[DB];
#pragma unroll
    for (int x = 0; x < DB; x++) acc_v[x] = acc_k[x] = f32x16{0};
    __syncthreads();
    issue_query_rows<D>(sm, sm.rows[0], q0, g0, wv, lane);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    int buf = 0;
    unsigned bad0 = sm.rows[0].bad[0], bad1 = sm.rows[0].bad[1];
    for (int r0 = first; r0 < end; r0 += BT, buf ^= 1) {
        __syncthreads();   // the tile's rows have landed
        bad0 = __builtin_amdgcn_readfirstlane(bad0);
        bad1 = __builtin_amdgcn_readfirstlane(bad1);
        if (bad0 | bad1) {
            for (int x = tid; x < BT * (D / 8); x += 256) {
                const int r = x / (D / 8), c = x % (D / 8);
                if ((r >> 5 ? bad1 : bad0) >> (r & 31) & 1) {
                    *(u32x4*)(sm.q + RowTile<D>::offset(r) + 16 * c) = u32x4{0, 0, 0, 0};
                    *(u32x4*)(sm.g + RowTile<D>::offset(r) + 16 * c) = u32x4{0, 0, 0, 0};
                }
            }
            __syncthreads();
        }
        float2 m = make_float2(0.0f, 0.0f);
        int i_then = 0;
        if (wv == 0) {
            m = meta_in[place(r0 + BT + lane, i_next)];
            i_then = entry(r0 + 2 * BT + lane);
        }
        bf16x8 dl[2];
        bwd_block_tile<D>(sm, sm.rows[buf], lane, wv, r0 < own_end, f.a.c2, acc_v, acc_k, dl);
        if (wv == 0) {
            put(sm.rows[buf ^ 1], r0 + BT + lane, i_next, m);
            i_next = i_then;
        }
        __syncthreads();   // dS is there, and nobody reads the rows any more
        if (r0 + BT < end) issue_query_rows<D>(sm, sm.rows[buf ^ 1], q0, g0, wv, lane);
        bad0 = sm.rows[buf ^ 1].bad[0];
        bad1 = sm.rows[buf ^ 1].bad[1];
        f32x16 acc_q[DB / 2];
        bwd_block_dq<D>(sm, lane, wv, f.a.scale, dl, acc_q);
        // the partial dq of rows 32 rb + col, columns of half kb, relative to the largest of them
        float top = 0.0f;
#pragma unroll
        for (int x = 0; x < DB / 2; x++)
#pragma unroll
            for (int e = 0; e < 16; e++) top = fmaxf(top, fabsf(acc_q[x][e]));
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
        const int E = scale_exp(max((unsigned)sw[0], (unsigned)sw[1]));
        const float down = scale_down(E);
        const int count = min(BT, end - r0);
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(scale_up(E)), buffer_of(f.meta + row0 + r0, 8 * count), half ? 0x7FFFFFF0 : 8 * rt + 4 * kb, 0, 0);
        const auto dst = buffer_of(f.part + (row0 + r0) * D, 2 * D * count);
#pragma unroll
        for (int x = 0; x < DB / 2; x++)
#pragma unroll
            for (int y = 0; y < 4; y += 2) {
                // columns 8 y .. 8 y + 7 from both halves of the wave to its lower lanes, the next 8 to its upper lanes
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const f16x2v a = {(_Float16)(acc_q[x][4 * y + 2 * e] * down), (_Float16)(acc_q[x][4 * y + 2 * e + 1] * down)};
                    const f16x2v c = {(_Float16)(acc_q[x][4 * y + 4 + 2 * e] * down), (_Float16)(acc_q[x][4 * y + 5 + 2 * e] * down)};
                    const auto sx = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, c), false, false);
                    w[e] = sx[0];
                    w[2 + e] = sx[1];
                }
                store_words(dst, rt * 2 * D + D * kb + 64 * x + 16 * (y + half), w);
            }
        // the next rows are there when no more than this tile's stores are under way (memory operations end in order)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(DB + 1) : "memory");
    }
    add_row_halves<D>(sm, lane, wv, acc_v, acc_k);
    if (wv >= 2) return;
    if (rows <= l.unit) {
        store_kv<D>(f, kv, 32 * wv + col, last, half, acc_v, acc_k);
        return;
    }
    float4* out = (float4*)f.kvpart + (((size_t)bg * l.maxu + l.first_unit[(size_t)bg * l.nb + j] + first / l.unit) * 2 + wv) * (2 * DB * 4 * 64);
#pragma unroll
    for (int x = 0; x < DB; x++)
#pragma unroll
        for (int y = 0; y < 4; y++) {
            out[(x * 4 + y) * 64 + lane] = make_float4(acc_v[x][4 * y], acc_v[x][4 * y + 1], acc_v[x][4 * y + 2], acc_v[x][4 * y + 3]);
            out[((DB + x) * 4 + y) * 64 + lane] = make_float4(acc_k[x][4 * y], acc_k[x][4 * y + 1], acc_k[x][4 * y + 2], acc_k[x][4 * y + 3]);
        }
}

// dK and dV of the blocks with several units: a workgroup per (every KV_JOIN-th block and 32 of its columns, batch and head), its first two
// waves dV and its last two dK, of 32 keys each.  (Most blocks have one unit: a workgroup for each of them takes 76 us for 64 heads of
// 128 blocks, most of it to start workgroups that find nothing.)
constexpr int KV_JOIN = 16;
template <int D>
__global__ __launch_bounds__(256) void block_kv_join_kernel(BlockBwd f)
{
    constexpr int DB = D / 32;
    const BlockLists& l = f.a.l;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, x = blockIdx.x % DB, bg = blockIdx.y;
    for (int j = blockIdx.x / DB; j < l.nb; j += KV_JOIN) {
        const int rows = l.total[(size_t)bg * l.nb + j] * l.G;
        if (rows <= l.unit) continue;
        const int units = (int)(((long long)rows + l.unit - 1) / l.unit), u0 = l.first_unit[(size_t)bg * l.nb + j];
        const float4* in = (const float4*)f.kvpart + (((size_t)bg * l.maxu + u0) * 2 + (wv & 1)) * (2 * DB * 4 * 64) + (((wv >> 1) * DB + x) * 4) * 64 + lane;
        float4 s[4];
#pragma unroll
        for (int y = 0; y < 4; y++) s[y] = make_float4(0, 0, 0, 0);
#pragma unroll 4
        for (int u = 0; u < units; u++)
#pragma unroll
            for (int y = 0; y < 4; y++) {
                const float4 v = in[(size_t)u * (4 * DB * 4 * 64) + y * 64];
                s[y].x += v.x; s[y].y += v.y; s[y].z += v.z; s[y].w += v.w;
            }
        const int key = 32 * (wv & 1) + (lane & 31);
        if (j * BT + key >= l.n) continue;
        const float c = wv >> 1 ? f.a.scale : 1.0f;
        uint16_t* out = (wv >> 1 ? f.dk : f.dv) + ((size_t)bg * l.n + (size_t)j * BT + key) * D + 32 * x + 4 * (lane >> 5);
#pragma unroll
        for (int y = 0; y < 4; y++) *(uint2*)(out + 8 * y) = make_uint2(pack_bf16x2(s[y].x * c, s[y].y * c), pack_bf16x2(s[y].z * c, s[y].w * c));
    }
}

// D / 8 lanes per row (query, head of the group).
template <int D>
__global__ __launch_bounds__(256) void block_dq_join_kernel(BlockBwd f, int items)
{
    constexpr int LPR = D / 8;
    const BlockLists& l = f.a.l;
    const int G = l.G, tid = threadIdx.x, t = tid % LPR, lane0 = (tid & 63) - t;
    int bg, item;
    deal_head(blockIdx.x, items, l.B * l.Hkv, bg, item);
    const int rr = item * (256 / LPR) + tid / LPR, row = min(rr, l.n * G - 1);
    const int i = row / G, gh = row % G, b = bg / l.Hkv, g = bg % l.Hkv;
    const int32_t* pos = l.pos + ((size_t)bg * l.n + i) * l.slots;
    const size_t rows0 = (size_t)bg * l.entries * G + gh;
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (int s0 = 0; s0 < l.slots; s0 += LPR) {
        const int p = s0 + t < l.slots ? pos[s0 + t] : -1, count = min(LPR, l.slots - s0);
#pragma unroll 4
        for (int s = 0; s < count; s++) {
            const int ps = __shfl(p, lane0 + s, 64);
            if (ps < 0) continue;
            const size_t pr = rows0 + (size_t)ps * G;
            const float up = ((const float*)(f.meta + pr))[2 * t / LPR];
            const f16x8 v = *(const f16x8*)(f.part + pr * D + 8 * t);
#pragma unroll
            for (int e = 0; e < 8; e++) acc[e] = fmaf(up, (float)v[e], acc[e]);
        }
    }
    if (rr >= l.n * G) return;
    u32x4 out;
#pragma unroll
    for (int e = 0; e < 4; e++) out[e] = pack_bf16x2(acc[2 * e], acc[2 * e + 1]);
    *(u32x4*)(f.dq + (((size_t)b * l.H + g * G + gh) * l.n + i) * D + 8 * t) = out;
}

// Rows whose dK and dV are summed in registers: most blocks have fewer and are finished by one workgroup (4 x 16 heads of 8192:
// 2224, 2069, 1992 and 1994 us with 512, 1024, 2048 and 4096); where there are few rows altogether, a popular block's are
// shared out to more of the chip.
static int bwd_unit(const sparsek_block_cfg& c)
{
    const double rows = (double)c.B * c.H * c.n * (c.top + 1);
    return rows >= 512 * 1024.0 ? 2048 : rows >= 256 * 1024.0 ? 1024 : 512;
}

struct BwdLayout {
    BlockLayout y;
    size_t rows, part, meta, kvpart, bytes;
};
static BwdLayout bwd_layout(const sparsek_block_cfg& c, void* ws)
{
    BwdLayout f;
    f.y = block_lists_layout(c, block_count(c.n) * BT, bwd_unit(c), ws);
    const size_t BG = (size_t)c.B * c.Hkv, rows = BG * f.y.l.entries * f.y.l.G;
    f.rows = f.y.bytes;
    f.part = align_up(f.rows + (size_t)c.B * c.H * c.n * 8, 256);
    f.meta = align_up(f.part + rows * c.d * 2, 256);
    f.kvpart = align_up(f.meta + rows * 8, 256);
    f.bytes = align_up(f.kvpart + BG * f.y.l.maxu * (size_t)BT * c.d * 8, 256);
    return f;
}

size_t block_bwd_ws_bytes(const sparsek_block_cfg& c) { return bwd_layout(c, nullptr).bytes; }

int launch_block_bwd(const sparsek_block_cfg& c, const void* q, const void* k, const void* v, const int32_t* idx, const void* o,
                     const float* lse, const void* dO, void* dq, void* dk, void* dv, void* ws, hipStream_t st)
{
    const BwdLayout y = bwd_layout(c, ws);
    BlockBwd f;
    f.a.l = y.y.l;
    f.a.q = (const uint16_t*)q; f.a.k = (const uint16_t*)k; f.a.v = (const uint16_t*)v;
    f.a.o = (const uint16_t*)o; f.a.dO = (const uint16_t*)dO; f.a.lse = lse;
    f.a.scale = c.softmax_scale;
    f.a.c2 = c.softmax_scale * 1.4426950408889634f;
    f.dq = (uint16_t*)dq; f.dk = (uint16_t*)dk; f.dv = (uint16_t*)dv;
    f.rows = (float2*)((char*)ws + y.rows);
    f.part = (_Float16*)((char*)ws + y.part); f.meta = (float2*)((char*)ws + y.meta); f.kvpart = (float*)((char*)ws + y.kvpart);
    const BlockLists& l = f.a.l;
    const int BG = c.B * c.Hkv;
    if (int rc = launch_block_lists(l, idx, st)) return rc;
    const size_t nrows = (size_t)c.B * c.H * c.n;
#define BWD(D)                                                                                                                                   \
    hipLaunchKernelGGL((block_delta_kernel<D>), dim3((unsigned)((nrows * (D / 8) + 255) / 256)), dim3(256), 0, st, f, nrows);                     \
    hipLaunchKernelGGL((block_bwd_tiles_kernel<D>), dim3((unsigned)l.maxu * BG), dim3(256), 0, st, f);                                           \
    hipLaunchKernelGGL((block_kv_join_kernel<D>), dim3(std::min(l.nb, KV_JOIN) * (D / 32), BG), dim3(256), 0, st, f);                                               \
    const int items = (int)(((long long)c.n * l.G * (D / 8) + 255) / 256);                                                                       \
    hipLaunchKernelGGL((block_dq_join_kernel<D>), dim3((unsigned)items * BG), dim3(256), 0, st, f, items)
    if (c.d == 128) {
        BWD(128);
    } else {
        BWD(64);
    }
#undef BWD
    return launch_status();
}

}  // namespace spk
