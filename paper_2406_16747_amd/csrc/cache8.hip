// A key/value cache in blocks of 64 tokens, held in 8 bits with a scale for each block and head.
//
// A page holds one block of one key/value head: keys [64][D] and values transposed [D][64], so that both products of the
// attention read their 8-bit operands as they lie (16 bytes a lane).  The table names a head's pages by age; the unfinished
// block at the end of a sequence is kept in bf16, values transposed as well.  Page numbers outside the pool are never
// followed: such a page is neither written nor attended.
//
// What bounds the kernels is memory where there is much to move (four prompts of 8192 go in at 5.2 TB/s, 64 sequences of up to 8192 are
// attended at 5.4 TB/s of the kernel's time) and the length of a chain of dependent steps where there is little: a token's append takes
// 3 us, 6 to 8 where it ends a block; the choice among 1024 blocks 12; the attention of 200 tokens 8; an eviction from 129 blocks 6.
#include "block_parts.hpp"

namespace spk {

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct CacheArgs {
    sparsek_cache8 t;
    int B, H, Hkv, G, cap, pages;
    const int32_t* lens;
};

__device__ __forceinline__ int clamp_len(int len, int cap) { return min(max(len, 0), cap * BT + BT - 1); }

// ---- append ----

// 64 tokens x D in the registers of 256 threads: piece t of thread tid is 16 bytes (8 columns) of token tid / (D/8) + (2048/D) t.
template <int D>
struct BlockRegs {
    static constexpr int CPR = D / 8, RG = 256 / CPR, NT = BT / RG;
};

__device__ __forceinline__ float half_of(u32x4 x, int e) { return __uint_as_float(e & 1 ? x[e / 2] & 0xFFFF0000u : x[e / 2] << 16); }

template <int FORMAT>
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d, float f)
{
    if constexpr (FORMAT == SPARSEK_I8) {
        return pack4(code_i8(a, f), code_i8(b, f), code_i8(c, f), code_i8(d, f));
    } else {
        const float m = 448.0f;   // (the product may be a rounding above it)
        a = fminf(fmaxf(a * f, -m), m); b = fminf(fmaxf(b * f, -m), m); c = fminf(fmaxf(c * f, -m), m); d = fminf(fmaxf(d * f, -m), m);
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    }
}

template <int D>
struct AppendSmem {
    static constexpr int VS = BT + 8;                                       // bf16 values between the columns of vt
    double sums[4][D];                                                      // of a wave's tokens
    __attribute__((aligned(16))) uint16_t vt[D * VS];                       // the block's values, transposed
    unsigned red[12];
    // Token x of a column.  Its groups of 8 tokens change places from 16 columns to the next: a token's columns, 8 to a lane, go to banks
    // of their own (as they lie, to two; four prompts of 8192 into the cache 42 us then).
    static __device__ __forceinline__ int at(int col, int x) { return col * VS + ((x >> 3 ^ (col >> 4 & 7)) << 3) + (x & 7); }
};

template <class F>
__device__ __forceinline__ double both_words(double x, F f)
{
    const unsigned long long b = __builtin_bit_cast(unsigned long long, x);
    const auto lo = f((unsigned)b), hi = f((unsigned)(b >> 32));
    return __builtin_bit_cast(double, (unsigned long long)hi[0] << 32 | lo[0]) + __builtin_bit_cast(double, (unsigned long long)hi[1] << 32 | lo[1]);
}
// The sum over a wave's lanes that have the same place among CPR = 8 or 16 neighbours.
template <int CPR>
__device__ __forceinline__ double sum_columns(double x)
{
    if constexpr (CPR == 8)
        x = both_words(x, [](unsigned y) { return u32x2{y, (unsigned)__builtin_amdgcn_mov_dpp((int)y, 0x128, 0xF, 0xF, true)}; });   // (8 lanes on, of 16)
    x = both_words(x, [](unsigned y) { const auto s = __builtin_amdgcn_permlane16_swap(y, y, false, false); return u32x2{(unsigned)s[0], (unsigned)s[1]}; });
    return both_words(x, [](unsigned y) { const auto s = __builtin_amdgcn_permlane32_swap(y, y, false, false); return u32x2{(unsigned)s[0], (unsigned)s[1]}; });
}

// A whole block goes to its page: codes, scales and the mean key.  The keys are in registers, the values (transposed) in sm.vt; every
// thread has seen the end of what was written there.
template <int D, int FORMAT>
__device__ __forceinline__ void store_block(AppendSmem<D>& sm, const CacheArgs& a, int page, const u32x4 (&kr)[BlockRegs<D>::NT], unsigned tv, int tid)
{
    using R = BlockRegs<D>;
    const float most = FORMAT == SPARSEK_I8 ? 127.0f : 448.0f;
    const int tok = tid / R::CPR, c = tid % R::CPR;
    unsigned tk = 0;
    double s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < R::NT; t++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float k = half_of(kr[t], e);
            s[e] += (double)k;
            tk = max(tk, __float_as_uint(fabsf(k)));
        }
#pragma unroll
    for (int e = 0; e < 8; e++) s[e] = sum_columns<R::CPR>(s[e]);
    if ((tid & 63) < R::CPR)
#pragma unroll
        for (int e = 0; e < 8; e++) sm.sums[tid >> 6][8 * c + e] = s[e];
    tk = wave_max_bits(tk);
    tv = wave_max_bits(tv);
    __syncthreads();   // the sums and values are there
    float mean = 0.0f;
    if (tid < D) {
        double y = 0;
#pragma unroll
        for (int g = 0; g < 4; g++) y += sm.sums[g][tid];
        mean = (float)(y / BT);
    }
    const unsigned tm = wave_max_bits(__float_as_uint(fabsf(mean)));
    if ((tid & 63) == 0) {
        sm.red[tid >> 6] = tk;
        sm.red[4 + (tid >> 6)] = tv;
        sm.red[8 + (tid >> 6)] = tm;
    }
    __syncthreads();
    auto top_of = [&](int x) { return __uint_as_float(max(max(sm.red[x], sm.red[x + 1]), max(sm.red[x + 2], sm.red[x + 3]))); };
    const float topk = top_of(0), topv = top_of(4), topm = top_of(8);
    const float fk = code_factor(topk, most), fv = code_factor(topv, most);
    unsigned char* kp = (unsigned char*)a.t.k8 + (size_t)page * BT * D;
#pragma unroll
    for (int t = 0; t < R::NT; t++) {
        u32x2 w;
        w[0] = codes4<FORMAT>(half_of(kr[t], 0), half_of(kr[t], 1), half_of(kr[t], 2), half_of(kr[t], 3), fk);
        w[1] = codes4<FORMAT>(half_of(kr[t], 4), half_of(kr[t], 5), half_of(kr[t], 6), half_of(kr[t], 7), fk);
        __builtin_nontemporal_store(w, (u32x2*)(kp + (tok + R::RG * t) * D + 8 * c));
    }
    unsigned char* vp = (unsigned char*)a.t.v8 + (size_t)page * BT * D;
#pragma unroll
    for (int t = 0; t < BT * D / 16 / 256; t++) {
        const int x = tid + 256 * t;
        const u32x4 lo = *(const u32x4*)&sm.vt[AppendSmem<D>::at(x / 4, 16 * (x % 4))], hi = *(const u32x4*)&sm.vt[AppendSmem<D>::at(x / 4, 16 * (x % 4) + 8)];
        u32x4 w;
        w[0] = codes4<FORMAT>(half_of(lo, 0), half_of(lo, 1), half_of(lo, 2), half_of(lo, 3), fv);
        w[1] = codes4<FORMAT>(half_of(lo, 4), half_of(lo, 5), half_of(lo, 6), half_of(lo, 7), fv);
        w[2] = codes4<FORMAT>(half_of(hi, 0), half_of(hi, 1), half_of(hi, 2), half_of(hi, 3), fv);
        w[3] = codes4<FORMAT>(half_of(hi, 4), half_of(hi, 5), half_of(hi, 6), half_of(hi, 7), fv);
        __builtin_nontemporal_store(w, (u32x4*)(vp + 16 * x));
    }
    if (tid < D) a.t.km[(size_t)page * D + tid] = (int8_t)code_i8(mean, code_factor(topm, 127.0f));
    if (tid == 0) {
        // (what is not finite must not get lost: NaN for whoever attends the block)
        a.t.ks[page] = topk < INFINITY ? code_scale(topk, most) : __uint_as_float(0x7FC00000u);
        a.t.vs[page] = topv < INFINITY ? code_scale(topv, most) : __uint_as_float(0x7FC00000u);
        a.t.kms[page] = code_scale(topm, 127.0f);
    }
}

// One workgroup of 256 per (block that new tokens touch, batch and head).  The first one also has the last block when that stays
// unfinished: both use the bf16 block, the one reads what the other overwrites.
template <int D, int FORMAT>
__global__ __launch_bounds__(256) void cache8_append_kernel(CacheArgs a, const int32_t* __restrict__ counts, int c, const uint16_t* __restrict__ k,
                                                            const uint16_t* __restrict__ v)
{
    using R = BlockRegs<D>;
    __shared__ AppendSmem<D> sm;
    const int tid = threadIdx.x, bg = blockIdx.y, b = bg / a.Hkv;
    const int len = clamp_len(a.lens[b], a.cap);
    const int count = min(counts ? min(max(counts[b], 0), c) : c, a.cap * BT + BT - 1 - len);   // (what does not fit is dropped)
    if (count <= 0) return;
    const int after = len + count, first = len / BT, j = first + blockIdx.x;
    if (j * BT >= after) return;
    const uint16_t *kn = k + (size_t)bg * c * D, *vn = v + (size_t)bg * c * D;
    uint16_t *kt = (uint16_t*)a.t.kt + (size_t)bg * BT * D, *vt = (uint16_t*)a.t.vt + (size_t)bg * BT * D;
    const int page = (j + 1) * BT <= after ? a.t.table[(size_t)bg * a.cap + j] : -1;
    if (page >= 0 && page < a.pages) {
        u32x4 kr[R::NT];
        unsigned tv = 0;
        const int old = max(0, len - j * BT);   // tokens of the block that are there already (in the first one only)
        const int tok0 = tid / R::CPR, col = 8 * (tid % R::CPR);
#pragma unroll
        for (int t = 0; t < R::NT; t++) {
            const int x = tok0 + R::RG * t;
            const size_t at = (size_t)(j * BT + x - len) * D + col;
            if (x < old) {
                kr[t] = *(const u32x4*)(kt + x * D + col);
                continue;
            }
            kr[t] = __builtin_nontemporal_load((const u32x4*)(kn + at));
            const u32x4 vr = __builtin_nontemporal_load((const u32x4*)(vn + at));
            tv = max(tv, top_of_8(vr));
#pragma unroll
            for (int e = 0; e < 8; e++) sm.vt[AppendSmem<D>::at(col + e, x)] = (uint16_t)(e & 1 ? vr[e / 2] >> 16 : vr[e / 2] & 0xFFFFu);
        }
        if (old) {   // (8 tokens of a column at a time, the last of them perhaps in part)
            u32x4 vo[D * 8 / 256];
#pragma unroll
            for (int y = 0; y < D * 8 / 256; y++) vo[y] = *(const u32x4*)(vt + 8 * (tid + 256 * y));
            const int t0 = 8 * (tid & 7);
#pragma unroll
            for (int y = 0; y < D * 8 / 256; y++) {
                uint16_t* to = &sm.vt[AppendSmem<D>::at(tid / 8 + 32 * y, t0)];
                if (t0 + 8 <= old) {
                    *(u32x4*)to = vo[y];
                    tv = max(tv, top_of_8(vo[y]));
                } else {
#pragma unroll
                    for (int e = 0; e < 7; e++)
                        if (t0 + e < old) {
                            const unsigned w = e & 1 ? vo[y][e / 2] >> 16 : vo[y][e / 2] & 0xFFFFu;
                            tv = max(tv, (w & 0x7FFFu) << 16);
                            to[e] = (uint16_t)w;
                        }
                }
            }
        }
        store_block<D, FORMAT>(sm, a, page, kr, tv, tid);
    }
    if (blockIdx.x != 0) return;
    __syncthreads();                // everybody has read what is overwritten now
    const int whole = after / BT;   // the block that stays unfinished, if it has tokens
    const int t0 = max(len, whole * BT);
    for (int x = tid; x < (after - t0) * D; x += 256) {
        const int tok = t0 + x / D, col = x % D;
        kt[(tok % BT) * D + col] = kn[(size_t)(tok - len) * D + col];
        vt[col * BT + tok % BT] = vn[(size_t)(tok - len) * D + col];
    }
}

// ---- the `need` largest of n keys in LDS, by a workgroup of NT ----
// Radix: four passes of 8 bits over the keys, counters in LDS that every wave adds up for itself: one barrier a pass.  (A wave that
// bisects takes 35 us for 512 rows of 2048, 16 waves with a bound each 46, passes with a barrier ahead of and behind the sum 17.)
struct TopBounds {
    unsigned thr, left;   // keys above thr, and `left` of those equal to it
};
template <int NT>
struct TopSmem {
    unsigned hist[3][256];
    int wsum[NT / 64][2];
};
template <int NT>
__device__ __forceinline__ TopBounds wg_top(TopSmem<NT>& sm, const unsigned* keys, int n, unsigned need)
{
    const int tid = threadIdx.x, lane = tid & 63;
    unsigned prefix = 0;
    if (tid < 256) sm.hist[0][tid] = 0;
    __syncthreads();
#pragma unroll
    for (int pass = 0; pass < 4; pass++) {
        const int shift = 24 - 8 * pass;
        unsigned* hist = sm.hist[pass % 3];
        for (int x = tid; x < n; x += NT)
            if (pass == 0 || keys[x] >> (shift + 8) == prefix) atomicAdd(&hist[keys[x] >> shift & 255], 1u);
        if (tid < 256) sm.hist[(pass + 1) % 3][tid] = 0;   // (read in the pass before the last one: everybody is past that)
        __syncthreads();
        // lane: digits 255 - 4 lane .. 252 - 4 lane; the threshold's digit is where the sum from the top reaches `need`
        const u32x4 c = *(const u32x4*)&hist[252 - 4 * lane];
        const unsigned mine = c[0] + c[1] + c[2] + c[3];
        unsigned sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const unsigned y = (unsigned)__shfl_up((int)sum, d, 64);
            if (lane >= d) sum += y;
        }
        unsigned above = sum - mine, digit = 0, left = 0;
#pragma unroll
        for (int e = 3; e >= 0; e--) {
            if (above < need && above + c[e] >= need) {
                digit = 252 - 4 * lane + e;
                left = need - above;
            }
            above += c[e];
        }
        const unsigned long long found = __ballot(left > 0);
        const int at = __ffsll(found) - 1;
        prefix = prefix << 8 | (unsigned)__builtin_amdgcn_readlane((int)digit, at);
        need = (unsigned)__builtin_amdgcn_readlane((int)left, at);
    }
    return TopBounds{prefix, need};
}

// order[place] = x for every x < n: those that belong to the largest (of equal ones the first) ahead of the others, both in order.
// Thread t has the keys t R .. t R + R - 1.  Ends with a barrier.
template <int NT>
__device__ __forceinline__ void wg_order(TopSmem<NT>& sm, const unsigned* keys, int n, TopBounds t, int budget, int* order)
{
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, R = (n + NT - 1) / NT, x0 = min(n, tid * R), x1 = min(n, x0 + R);
    int g = 0, e = 0;
    for (int x = x0; x < x1; x++) {
        g += keys[x] > t.thr;
        e += keys[x] == t.thr;
    }
    int gs = g, es = e;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(gs, d, 64), z = __shfl_up(es, d, 64);
        if (lane >= d) { gs += y; es += z; }
    }
    if (lane == 63) {
        sm.wsum[wv][0] = gs;
        sm.wsum[wv][1] = es;
    }
    __syncthreads();
    gs -= g;
    es -= e;
    for (int w = 0; w < wv; w++) {
        gs += sm.wsum[w][0];
        es += sm.wsum[w][1];
    }
    int kept = gs + min(es, (int)t.left);
    for (int x = x0; x < x1; x++) {
        const unsigned k = keys[x];
        const bool in = k > t.thr || (k == t.thr && es < (int)t.left);
        order[in ? kept : budget + x - kept] = x;
        es += k == t.thr;
        kept += in;
    }
    __syncthreads();
}

// ---- selection of blocks for a single query ----

template <int D>
__global__ __launch_bounds__(1024) void cache8_select_kernel(CacheArgs a, const uint16_t* __restrict__ q, int top, int32_t* __restrict__ idx)
{
    extern __shared__ unsigned keys[];   // [cap], and the pages, then the order [cap]
    int* at = (int*)(keys + a.cap);
    __shared__ __attribute__((aligned(16))) TopSmem<1024> sm;
    __shared__ unsigned q8[D / 4];
    constexpr int LPB = D / 16, BPR = 1024 / LPB;   // lanes per block (16 bytes each), blocks per round
    const int tid = threadIdx.x, bg = blockIdx.x, b = bg / a.Hkv, g = bg % a.Hkv;
    const int len = clamp_len(a.lens[b], a.cap);
    const int nb = len > 0 ? (len - 1) / BT : 0;   // blocks behind the query's own
    int32_t* out = idx + (size_t)bg * top;
    if (nb <= top) {
        for (int x = tid; x < top; x += 1024) out[x] = x < nb ? x : -1;
        return;
    }
    for (int x = tid; x < nb; x += 1024) at[x] = a.t.table[(size_t)bg * a.cap + x];
    if (tid < 64) {   // the group's queries, added up and rounded
        constexpr int PL = D / 64;
        float x[PL];
        float most = 0.0f;
        double s[PL];
#pragma unroll
        for (int e = 0; e < PL; e++) s[e] = 0;
#pragma unroll 4
        for (int h = 0; h < a.G; h++)
#pragma unroll
            for (int e = 0; e < PL; e++) s[e] += (double)bf16_to_f32(q[((size_t)b * a.H + g * a.G + h) * D + PL * tid + e]);
#pragma unroll
        for (int e = 0; e < PL; e++) {
            x[e] = (float)s[e];
            most = fmaxf(most, fabsf(x[e]));
        }
        const float f = code_factor(wave_max_f32(most), 127.0f);
#pragma unroll
        for (int e = 0; e < PL; e++) ((int8_t*)q8)[PL * tid + e] = (int8_t)code_i8(x[e], f);
    }
    __syncthreads();
    const int c = tid % LPB;
    i32x4 qv;
#pragma unroll
    for (int e = 0; e < 4; e++) qv[e] = (int)q8[4 * c + e];
    constexpr int UNR = 4;   // rounds whose loads are under way together
    for (int x0 = tid / LPB; x0 < nb; x0 += UNR * BPR) {
        i32x4 m[UNR];
        float ms[UNR];
#pragma unroll
        for (int u = 0; u < UNR; u++) {
            const int page = at[min(x0 + u * BPR, nb - 1)], p = page >= 0 && page < a.pages ? page : 0;
            m[u] = *(const i32x4*)(a.t.km + (size_t)p * D + 16 * c);
            ms[u] = a.t.kms[p];
        }
#pragma unroll
        for (int u = 0; u < UNR; u++) {
            const int x = x0 + u * BPR, page = at[min(x, nb - 1)];
            int s = 0;
#pragma unroll
            for (int e = 0; e < 4; e++) s = __builtin_amdgcn_sdot4(m[u][e], qv[e], s, false);
#pragma unroll
            for (int d = 1; d < LPB; d <<= 1) s += __shfl_xor(s, d, 64);
            if (c == 0 && x < nb) keys[x] = page >= 0 && page < a.pages ? min(max(score_key((float)s * ms[u]), 2u), 0xFFFFFFFEu) : 1u;
        }
    }
    __syncthreads();
    wg_order(sm, keys, nb, wg_top(sm, keys, nb, (unsigned)top), top, at);
    for (int x = tid; x < top; x += 1024) out[x] = at[x];
}

// ---- attention of a single query per sequence ----

// A workgroup has 4 waves, and a wave takes whole blocks: S = K.Q^T (64 tokens by 16 heads), the running softmax, O^T += V^T.P^T.
// A block goes through LDS, in loads of whole lines: loaded as the operands have it, 16 bytes of a row to a lane, every lane is a line
// of its own to the cache, which takes four times as many cycles (a sequence of 32768 tokens 29.8 us so, 26.7 through LDS; 64 of up to
// 8192 155 and 150).  Between S and O nothing is exchanged: row m of S's tile t is token 16 (m / 4) + 4 t + m % 4, so a lane's 16 weights are those of the 16 tokens whose values it reads for every column.  Codes of 8
// bits are exact in fp16; so is q relative to its largest value (what fp16 drops lies 2^-27 below it), and weights lose 2^-11
// where bf16 would lose 2^-8.  What bounds it is memory: a wave has the keys of one block or the values of another on
// their way while it computes.
constexpr int MAX_UPW = 5, MAX_CAP = 8192;   // units of a wave, blocks of a row at most
struct AttnArgs {
    CacheArgs c;
    const uint16_t* q;
    const int32_t* idx;    // [B,Hkv,top] or null: all blocks
    int top, splits, upw;  // parts of a row, units per wave
    float c2;
    float* part_o;         // [B,H,splits][D]
    float2* part_ml;       // [B,H,splits]: the largest logit (times log2 e), the sum
    float* weight;         // [B,H,units]: log2 of a unit's share before the division
    int units;             // units per row at most
    bool accumulate;
    uint16_t* o;
    float* lse;
};

// 8 codes as fp16
template <int FORMAT>
__device__ __forceinline__ f16x8 widen(unsigned lo, unsigned hi)
{
    const unsigned w[2] = {lo, hi};
    u32x4 r;
#pragma unroll
    for (int x = 0; x < 2; x++) {
        if constexpr (FORMAT == SPARSEK_I8) {
            // 0x6400 | b is 1024 + b for a byte b = code + 128
            const unsigned y = w[x] ^ 0x80808080u;
            const f16x2v off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
            r[2 * x] = __builtin_bit_cast(unsigned, __builtin_bit_cast(f16x2v, __builtin_amdgcn_perm(0x64646464u, y, 0x04010400u)) + off);
            r[2 * x + 1] = __builtin_bit_cast(unsigned, __builtin_bit_cast(f16x2v, __builtin_amdgcn_perm(0x64646464u, y, 0x04030402u)) + off);
        } else {
            r[2 * x] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[x], 1.0f, false));
            r[2 * x + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[x], 1.0f, true));
        }
    }
    return __builtin_bit_cast(f16x8, r);
}

typedef float f32x4m __attribute__((ext_vector_type(4)));

// 8 bf16 values, 0 where one is not finite.
__device__ __forceinline__ u32x4 finite_halves(u32x4 w)
{
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const unsigned bad = ((w[e] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;   // (an exponent of ones carries into the sign's place)
        w[e] &= ~(bad | (bad - (bad >> 15)));
    }
    return w;
}

// The units of a row: the whole blocks, or those that idx names and the one the query ends, if it does; and the unfinished block
// behind them.
struct RowUnits {
    int whole, tail, nsel;   // whole blocks, tokens of the unfinished one, units ahead of it
    int own;                 // with idx: the whole block that the query ends, -1: none
};
__device__ __forceinline__ RowUnits row_units(const AttnArgs& a, int b)
{
    const int len = clamp_len(a.c.lens[b], a.c.cap);
    RowUnits r;
    r.whole = len / BT;
    r.tail = len % BT;
    r.own = a.idx && r.whole && !r.tail ? r.whole - 1 : -1;
    r.nsel = a.idx ? a.top + (r.own >= 0 ? 1 : 0) : r.whole;
    return r;
}
// The place in the table of unit u < nsel, -1: none (no whole block behind the query's own, or one named before).
// seen: the blocks that units ahead of `first` name, as bits (first == 0: not read).
__device__ __forceinline__ int unit_block(const AttnArgs& a, const RowUnits& r, size_t bg, int u, int first, const unsigned* seen)
{
    if (!a.idx) return u;
    if (u == a.top) return r.own;
    const int32_t* row = a.idx + bg * a.top;
    const int x = row[u];
    bool ok = x >= 0 && x < (r.own >= 0 ? r.own : r.whole);
    if (ok && first) ok = !(seen[x >> 5] >> (x & 31) & 1);
    for (int s = first; s < u; s++) ok &= row[s] != x;
    return ok ? x : -1;
}

// Unit u's weights join the mass of its place in the table.  (One that was left out has none and may name any place.)
__device__ __forceinline__ void add_mass(const AttnArgs& a, const RowUnits& ru, size_t bg, int u, float sum)
{
    const int j = u == ru.nsel ? ru.whole : !a.idx ? u : u == a.top ? ru.own : a.idx[bg * a.top + u];
    if (j >= 0 && j < a.c.cap && sum != 0.0f) a.c.t.mass[bg * a.c.cap + j] += sum;
}

// The running softmax over a unit's logits (in s, times log2 e); put(t, r, p) takes the weight of s[t][r], times 2^15.
struct SoftRow {
    float m, l;
};
template <class Put>
__device__ __forceinline__ float soft_unit(const f32x4m (&s)[4], SoftRow& row, float& corr, Put put)
{
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; t++)
#pragma unroll
        for (int r = 0; r < 4; r++) top = fmaxf(top, s[t][r]);
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto c = __builtin_amdgcn_permlane16_swap(__float_as_uint(top), __float_as_uint(top), false, false);
    top = fmaxf(__uint_as_float(c[0]), __uint_as_float(c[1]));
    const float mx = fmaxf(row.m, top), ref = mx == -INFINITY ? 0.0f : mx;
    corr = __builtin_amdgcn_exp2f(row.m - ref);
    row.m = mx;
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < 4; t++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const float p = __builtin_amdgcn_exp2f(s[t][r] - ref + 15.0f);   // (ref - 15 would be rounded where it is large, past fp16's range)
            sum += p;
            put(t, r, p);
        }
    const auto d = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    sum = __uint_as_float(d[0]) + __uint_as_float(d[1]);
    const auto e = __builtin_amdgcn_permlane16_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    sum = __uint_as_float(e[0]) + __uint_as_float(e[1]);
    row.l = fmaf(row.l, corr, sum);
    return ref + log2f(sum * 0x1p-15f);   // log2 of the unit's share
}

// The largest logit of keys that were attended but have none above -inf: they are infinite themselves, or their query is, or their scale
// is NaN.  No finite logit is below it, and still it is not the -inf of no keys at all: what remains of such a row alone is 0 / 0.
constexpr float NO_LOGIT = -__FLT_MAX__;
__device__ __forceinline__ float log_of(float top, float sum)   // a row's lse; sum: times 2^15
{
    if (top == -INFINITY) return -INFINITY;
    return sum == 0.0f ? __uint_as_float(0x7FC00000u) : (top + log2f(sum * 0x1p-15f)) * 0.6931471805599453f;
}

// A wave's block in LDS: 64 rows of D bytes of keys, D rows of 64 bytes of values.  The pieces (16 bytes) of a row change places so that the
// 8 lanes that read at a time find them in different banks; a row's stay among each other, so the loads see whole lines.
template <int D>
struct CacheTile {
    static constexpr int BYTES = BT * D, LOADS = BYTES / 1024;   // of the keys, and of the values; wave-loads of each
    __device__ static int key_swap(int row) { return D == 128 ? (row & 3) | (row >> 4 & 1) << 2 : row >> 4 & 3; }
    __device__ static int value_swap(int row) { return row >> 2 & 3; }
    // where in the page the piece lies that wave-load x brings to the lane's place
    __device__ static uint32_t key_at(int x, int lane)
    {
        const int row = x * (1024 / D) + lane / (D / 16);
        return (uint32_t)(row * D + 16 * ((lane % (D / 16)) ^ key_swap(row)));
    }
    __device__ static uint32_t value_at(int x, int lane)
    {
        const int row = 16 * x + lane / 4;
        return (uint32_t)(row * BT + 16 * ((lane & 3) ^ value_swap(row)));
    }
};

template <int D, int FORMAT>
__global__ __launch_bounds__(256, D == 128 ? 2 : 4) void cache8_attn_kernel(AttnArgs a)
{
    using T = CacheTile<D>;
    constexpr int KH = D / 64, NX = D / 16, RO = D + 4;
    __shared__ __attribute__((aligned(16))) unsigned char tiles[4][2 * T::BYTES];   // a wave's keys and values; its result at the end
    __shared__ float sm_[4][16], sl[4][16], shares[4 * MAX_UPW + 1][16];
    __shared__ unsigned seen[MAX_CAP / 32];
    static_assert(16 * RO * 4 <= 2 * T::BYTES, "room for a wave's result");
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, grp = lane >> 4;
    const int groups = (a.c.G + 15) / 16;
    const int split = blockIdx.x, g = blockIdx.y / groups, rg = blockIdx.y % groups, b = blockIdx.z;
    const size_t bg = (size_t)b * a.c.Hkv + g;
    const int u0 = split * 4 * a.upw + wv * a.upw;
    // (the pages are asked for ahead of the length, of which they depend in number only)
    const int early = a.c.t.table[bg * a.c.cap + min(u0 + min(lane, a.upw - 1), a.c.cap - 1)];
    const RowUnits ru = row_units(a, b);
    const int nu = ru.nsel + (ru.tail ? 1 : 0);
    const bool alone = a.splits == 1 && groups == 1;   // the workgroup has all units of all heads of the group
    if (split * 4 * a.upw >= nu && !alone) return;   // (the join leaves such parts out)
    const int live = min(16, a.c.G - rg * 16);
    const size_t head0 = (size_t)b * a.c.H + g * a.c.G + rg * 16;
    // the wave's units, one to a lane: page (of any unit that has one where there is none), scales
    const int count = max(0, min(a.upw, ru.nsel - u0)), first = split * 4 * a.upw;
    int page = -1;
    if (a.idx && first) {   // (a selection longer than a workgroup's share: what the others name, for repeated blocks)
        for (int x = tid; x < MAX_CAP / 32; x += 256) seen[x] = 0;
        __syncthreads();
        for (int x = tid; x < min(first, a.top); x += 256) {
            const int j = a.idx[bg * a.top + x];
            if (j >= 0 && j < MAX_CAP) atomicOr(&seen[j >> 5], 1u << (j & 31));
        }
        __syncthreads();
    }
    if (lane < count) {
        if (a.idx) {
            const int j = unit_block(a, ru, bg, u0 + lane, first, seen);
            if (j >= 0) page = a.c.t.table[bg * a.c.cap + j];
        } else {
            page = early;
        }
        if (page >= a.c.pages) page = -1;
    }
    const unsigned long long have = __ballot(page >= 0);
    const int some = have ? __builtin_amdgcn_readlane(page, __ffsll(have) - 1) : 0;
    if (page < 0) page = some;
    float ks = 0.0f, vs = 0.0f;
    if (lane < count && have) {
        ks = a.c.t.ks[page];
        vs = a.c.t.vs[page];
    }
    // Q^T: head col, columns 64 half + 16 grp + 8 sub .., relative to the head's largest value
    const uint16_t* qr = a.q + (head0 + min(col, live - 1)) * D + 16 * grp;
    u32x4 qw[KH][2];
    unsigned top = 0;
#pragma unroll
    for (int h = 0; h < KH; h++)
#pragma unroll
        for (int s = 0; s < 2; s++) {
            qw[h][s] = *(const u32x4*)(qr + 64 * h + 8 * s);
#pragma unroll
            for (int e = 0; e < 4; e++) top = max(top, max(qw[h][s][e] << 16 & 0x7FFFFFFFu, qw[h][s][e] & 0x7FFF0000u));
        }
    top = max(top, (unsigned)__shfl_xor((int)top, 16, 64));
    top = max(top, (unsigned)__shfl_xor((int)top, 32, 64));
    const int E = scale_exp(top);
    const float down = scale_down(E), c2q = a.c2 * scale_up(E);
    f16x8 qf[KH][2];
#pragma unroll
    for (int h = 0; h < KH; h++)
#pragma unroll
        for (int s = 0; s < 2; s++)
#pragma unroll
            for (int e = 0; e < 8; e++) qf[h][s][e] = (_Float16)(half_of(qw[h][s], e) * down);
    f32x4m acc[NX];
#pragma unroll
    for (int x = 0; x < NX; x++) acc[x] = f32x4m{0, 0, 0, 0};
    SoftRow row = {-INFINITY, 0.0f};
    // the weights of the live heads' units; the other lanes' lie outside the buffer
    const bool weighs = a.accumulate && !alone;
    const buffer_t wbuf = buffer_of(weighs ? a.weight + head0 * a.units : nullptr, weighs ? live * a.units * 4 : 0);
    const int wat = grp == 0 && col < live ? col * a.units * 4 : 0x7FFFFF00;
    if (have) {
        unsigned char *kt = tiles[wv], *vt = kt + T::BYTES;
        // A whole cache is streamed past the chip's caches (64 sequences of up to 8192: 148 us -> 130).  Blocks that were chosen are likely
        // to be chosen by the next token again (16 sequences, 16 of 1024 blocks, this kernel alone: 14.4 us where the last cache has them,
        // 14.7 streamed; 15.6 and 14.7 where every selection is a new one), and more than 16 heads of a group read a block several times.
        const bool stream = !a.idx && a.c.G <= 16;
        auto load_k = [&](int i) {
            const unsigned char* kp = (const unsigned char*)a.c.t.k8 + (size_t)__builtin_amdgcn_readlane(page, i) * T::BYTES;
            if (stream) {
#pragma unroll
                for (int x = 0; x < T::LOADS; x++) async_stream_lds16(kp, T::key_at(x, lane), kt + 1024 * x);
            } else {
#pragma unroll
                for (int x = 0; x < T::LOADS; x++) async_load_lds16(kp, T::key_at(x, lane), kt + 1024 * x);
            }
        };
        auto load_v = [&](int i) {
            const unsigned char* vp = (const unsigned char*)a.c.t.v8 + (size_t)__builtin_amdgcn_readlane(page, i) * T::BYTES;
            if (stream) {
#pragma unroll
                for (int x = 0; x < T::LOADS; x++) async_stream_lds16(vp, T::value_at(x, lane), vt + 1024 * x);
            } else {
#pragma unroll
                for (int x = 0; x < T::LOADS; x++) async_load_lds16(vp, T::value_at(x, lane), vt + 1024 * x);
            }
        };
        load_k(0);
        load_v(0);
        for (int i = 0; i < count; i++) {
            const float f = readlane_f32(ks, i) * c2q, vscale = readlane_f32(vs, i);
            const bool there = have >> i & 1;
            // the keys are there when no more than the values' loads are under way (memory operations end in order)
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(T::LOADS) : "memory");
            f32x4m s[4];
#pragma unroll
            for (int t = 0; t < 4; t++) {
                s[t] = f32x4m{0, 0, 0, 0};
                const int row = 16 * (col >> 2) + 4 * t + (col & 3);
#pragma unroll
                for (int h = 0; h < KH; h++) {
                    const u32x4 w = *(const u32x4*)(kt + row * D + 16 * ((4 * h + grp) ^ T::key_swap(row)));
                    s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen<FORMAT>(w[0], w[1]), qf[h][0], s[t], 0, 0, 0);
                    s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen<FORMAT>(w[2], w[3]), qf[h][1], s[t], 0, 0, 0);
                }
            }
#pragma unroll
            for (int t = 0; t < 4; t++)
#pragma unroll
                for (int r = 0; r < 4; r++) s[t][r] = there ? s[t][r] * f : -INFINITY;
            // the next keys; the values are there when no more than those are under way
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (i + 1 < count) {
                load_k(i + 1);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(T::LOADS) : "memory");
            } else {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
            f16x8 pb[2];
            float corr;
            const float share = soft_unit(s, row, corr, [&](int t, int r, float p) { pb[t >> 1][4 * (t & 1) + r] = (_Float16)p; });
#pragma unroll
            for (int x = 0; x < NX; x++) {
                const int vr = 16 * x + col;
                const u32x4 w = *(const u32x4*)(vt + vr * BT + 16 * (grp ^ T::value_swap(vr)));
                f32x4m y = {0, 0, 0, 0};
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen<FORMAT>(w[0], w[1]), pb[0], y, 0, 0, 0);
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen<FORMAT>(w[2], w[3]), pb[1], y, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; r++) acc[x][r] = fmaf(acc[x][r], corr, vscale * y[r]);
            }
            if (alone) shares[u0 + i][col] = share;
            else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(share), wbuf, wat + 4 * (u0 + i), 0, 0);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (i + 1 < count) load_v(i + 1);
        }
    } else {   // nothing to attend: the units have no share
        for (int i = 0; i < count; i++) {
            if (alone) shares[u0 + i][col] = -INFINITY;
            else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(-INFINITY), wbuf, wat + 4 * (u0 + i), 0, 0);
        }
    }
    if (ru.tail && ru.nsel >= u0 && ru.nsel < u0 + a.upw) {   // the unfinished block, in bf16
        const uint16_t *kp = (const uint16_t*)a.c.t.kt + bg * BT * D, *vp = (const uint16_t*)a.c.t.vt + (bg * D + col) * BT + 16 * grp;
        f32x4m s[4];
#pragma unroll
        for (int t = 0; t < 4; t++) {
            s[t] = f32x4m{0, 0, 0, 0};
            const int tok = min(16 * (col >> 2) + 4 * t + (col & 3), ru.tail - 1);
#pragma unroll
            for (int h = 0; h < KH; h++)
#pragma unroll
                for (int x = 0; x < 2; x++)
                    s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8*)(kp + tok * D + 64 * h + 16 * grp + 8 * x), *(const bf16x8*)(qr + 64 * h + 8 * x), s[t], 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; r++) s[t][r] = 16 * grp + 4 * t + r < ru.tail ? s[t][r] * a.c2 : -INFINITY;
        }
        // Values as they lie, in bf16, and weights as the sum of two bf16 numbers (2^-16): a column knows nothing of the others' sizes, and
        // an infinity or a NaN in one stays there (the second products leave it out: 0 times infinity).  What lies behind the last token may be
        // anything and becomes 0.
        auto values = [&](int x, int y) {
            u32x4 w = *(const u32x4*)(vp + 16 * x * BT + 8 * y);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int tok = 16 * grp + 8 * y + 2 * e;
                w[e] = tok + 1 < ru.tail ? w[e] : tok < ru.tail ? w[e] & 0xFFFFu : 0u;
            }
            return w;
        };
        bf16x8 ph[2], pl[2];
        float corr;
        const float share = soft_unit(s, row, corr, [&](int t, int r, float p) {
            const __bf16 hi = (__bf16)p;
            ph[t >> 1][4 * (t & 1) + r] = hi;
            pl[t >> 1][4 * (t & 1) + r] = (__bf16)(p - (float)hi);
        });
        if (alone) shares[ru.nsel][col] = share;
        else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(share), wbuf, wat + 4 * ru.nsel, 0, 0);
#pragma unroll
        for (int x = 0; x < NX; x++) {
            f32x4m y = {0, 0, 0, 0};
#pragma unroll
            for (int z = 0; z < 2; z++) {
                const u32x4 w = values(x, z);
                y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), ph[z], y, 0, 0, 0);
                y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, finite_halves(w)), pl[z], y, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; r++) acc[x][r] = fmaf(acc[x][r], corr, y[r]);
        }
    }
    // the four waves' results are joined; rows 4 grp + r of tile x are columns of the head
    if (grp == 0) {
        const bool some = have || (ru.tail && ru.nsel >= u0 && ru.nsel < u0 + a.upw);
        sm_[wv][col] = row.m == -INFINITY && some ? NO_LOGIT : row.m;
        sl[wv][col] = row.l;
    }
#pragma unroll
    for (int x = 0; x < NX; x++) *(f32x4m*)((float*)tiles[wv] + col * RO + 16 * x + 4 * grp) = acc[x];   // (the wave's own blocks are read)
    __syncthreads();
    for (int x = tid; x < live * D; x += 256) {
        const int h = x / D, d = x % D;
        const float M = fmaxf(fmaxf(sm_[0][h], sm_[1][h]), fmaxf(sm_[2][h], sm_[3][h]));
        float sum = 0.0f, den = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; w++) {
            const float f = sm_[w][h] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm_[w][h] - M);
            sum += f * ((const float*)tiles[w])[h * RO + d];
            den += f * sl[w][h];
        }
        if (alone) {
            const bool some_key = M > -INFINITY;
            a.o[(head0 + h) * D + d] = f32_to_bf16(some_key ? sum / den : 0.0f);
            if (d == 0) a.lse[head0 + h] = log_of(M, den);
            continue;
        }
        const size_t at = (head0 + h) * a.splits + split;
        a.part_o[at * D + d] = sum;
        if (d == 0) a.part_ml[at] = make_float2(M, den);
    }
    if (alone && a.accumulate && tid < nu) {   // (one group of heads: nobody else adds to these masses)
        float sum = 0.0f;
        for (int h = 0; h < live; h++) {
            const float M = fmaxf(fmaxf(sm_[0][h], sm_[1][h]), fmaxf(sm_[2][h], sm_[3][h]));
            if (M == -INFINITY) continue;
            float den = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; w++) den += sm_[w][h] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm_[w][h] - M) * sl[w][h];
            if (shares[tid][h] != -INFINITY) sum += __builtin_amdgcn_exp2f(shares[tid][h] - (M + log2f(den * 0x1p-15f)));
        }
        add_mass(a, ru, bg, tid, sum);
    }
}

// The parts of a head are joined (workgroups 0 .. H-1 of a sequence), and the shares of its blocks join the masses (the others).
template <int D>
__global__ __launch_bounds__(256) void cache8_join_kernel(AttnArgs a, int mass_wgs)
{
    constexpr int EPL = D / 64, UNR = 8;   // columns per lane
    __shared__ float red[4][D], ms[4], ls[4], logs[4];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, b = blockIdx.y, G = a.c.G;
    const RowUnits ru = row_units(a, b);
    const int nu = ru.nsel + (ru.tail ? 1 : 0), splits = (nu + 4 * a.upw - 1) / (4 * a.upw);
    if ((int)blockIdx.x < a.c.H) {   // a wave takes every fourth part, 8 of them under way together
        const size_t row = (size_t)b * a.c.H + blockIdx.x;
        const float2* ml = a.part_ml + row * a.splits;
        const float* po = a.part_o + row * a.splits * D + EPL * lane;
        float M = -INFINITY, L = 0.0f, sum[EPL];
#pragma unroll
        for (int e = 0; e < EPL; e++) sum[e] = 0.0f;
        for (int s0 = wv; s0 < splits; s0 += 4 * UNR) {
            float2 p[UNR];
            float x[UNR][EPL];
#pragma unroll
            for (int u = 0; u < UNR; u++) {
                const int s = min(s0 + 4 * u, splits - 1);
                p[u] = ml[s];
#pragma unroll
                for (int e = 0; e < EPL; e++) x[u][e] = po[(size_t)s * D + e];
            }
            float top = M;
#pragma unroll
            for (int u = 0; u < UNR; u++) {
                if (s0 + 4 * u >= splits) p[u].x = -INFINITY;
                top = fmaxf(top, p[u].x);
            }
            if (top == -INFINITY) continue;
            const float corr = __builtin_amdgcn_exp2f(M - top);
            M = top;
            L *= corr;
#pragma unroll
            for (int e = 0; e < EPL; e++) sum[e] *= corr;
#pragma unroll
            for (int u = 0; u < UNR; u++) {
                if (p[u].x == -INFINITY) continue;   // (a part without keys)
                const float w = __builtin_amdgcn_exp2f(p[u].x - top);
                L = fmaf(w, p[u].y, L);
#pragma unroll
                for (int e = 0; e < EPL; e++) sum[e] = fmaf(w, x[u][e], sum[e]);
            }
        }
        if (lane == 0) { ms[wv] = M; ls[wv] = L; }
#pragma unroll
        for (int e = 0; e < EPL; e++) red[wv][EPL * lane + e] = sum[e];
        __syncthreads();
        const float top = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
        float all = 0.0f, y = 0.0f;
        if (top > -INFINITY)
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float f = __builtin_amdgcn_exp2f(ms[w] - top);
                all = fmaf(f, ls[w], all);
                if (tid < D) y = fmaf(f, red[w][tid], y);
            }
        if (tid < D) a.o[row * D + tid] = f32_to_bf16(top > -INFINITY ? y / all : 0.0f);
        if (tid == 0) a.lse[row] = log_of(top, all);
        return;
    }
    auto total = [&](int h) {   // log2 of head h's sum, by a wave
        const float2* p = a.part_ml + ((size_t)b * a.c.H + h) * a.splits;
        float M = -INFINITY, L = 0.0f;
        for (int s = lane; s < splits; s += 64) {
            const float2 x = p[s];
            const float top = fmaxf(M, x.x);
            if (x.x > -INFINITY) L = L * __builtin_amdgcn_exp2f(M - top) + x.y * __builtin_amdgcn_exp2f(x.x - top);
            M = top;
        }
        const float top = wave_max_f32(M);
        L = wave_sum_f32(M > -INFINITY ? L * __builtin_amdgcn_exp2f(M - top) : 0.0f);
        return top + log2f(L * 0x1p-15f);
    };
    const int g = (blockIdx.x - a.c.H) / mass_wgs, part = (blockIdx.x - a.c.H) % mass_wgs;
    if (part * 256 >= nu) return;
    const size_t bg = (size_t)b * a.c.Hkv + g;
    const int u = part * 256 + tid;
    float sum = 0.0f;
    for (int r0 = 0; r0 < G; r0 += 4) {   // a wave per head
        float w[4];
#pragma unroll
        for (int x = 0; x < 4; x++) w[x] = u < nu && r0 + x < G ? a.weight[((size_t)b * a.c.H + g * G + r0 + x) * a.units + u] : -INFINITY;
        if (r0 + wv < G) {
            const float all = total(g * G + r0 + wv);
            if (lane == 0) logs[wv] = all;
        }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < 4; x++)
            if (w[x] != -INFINITY) sum += __builtin_amdgcn_exp2f(w[x] - logs[x]);
        __syncthreads();
    }
    if (u < nu) add_mass(a, ru, bg, u, sum);
}

// ---- eviction ----

__global__ __launch_bounds__(256) void cache8_evict_kernel(CacheArgs a, int budget, int sink, int recent, int32_t* __restrict__ table,
                                                           float* __restrict__ mass, int32_t* __restrict__ lens)
{
    extern __shared__ unsigned keys[];   // [cap], and the order [cap]
    int* order = (int*)(keys + a.cap);
    __shared__ __attribute__((aligned(16))) TopSmem<256> sm;
    const int tid = threadIdx.x, bg = blockIdx.x, b = bg / a.Hkv, cap = a.cap;
    const int len = clamp_len(a.lens[b], cap), nb = len / BT;
    const size_t row = (size_t)bg * cap;
    const int32_t* table_in = a.t.table + row;
    const float* mass_in = a.t.mass + row;
    if (bg % a.Hkv == 0 && tid == 0) lens[b] = min(nb, budget) * BT + len % BT;
    if (nb <= budget) {
        for (int x = tid; x < cap; x += 256) {
            table[row + x] = table_in[x];
            mass[row + x] = mass_in[x];
        }
        return;
    }
#pragma unroll 8
    for (int x = tid; x < nb; x += 256) {
        const float m = fabsf(mass_in[x]) <= INFINITY ? mass_in[x] : __uint_as_float(0x7FC00000u);   // (a NaN of either sign: the largest)
        keys[x] = x < sink || x >= nb - recent ? 0xFFFFFFFFu : min(max(score_key(m), 1u), 0xFFFFFFFEu);
    }
    __syncthreads();
    const TopBounds t = budget > 0 ? wg_top(sm, keys, nb, (unsigned)budget) : TopBounds{0xFFFFFFFFu, 0u};
    wg_order(sm, keys, nb, t, budget, order);
#pragma unroll 4
    for (int x = tid; x < cap; x += 256) {
        const int y = x < nb ? order[x] : x;
        table[row + x] = table_in[y];
        mass[row + x] = x < budget ? mass_in[y] : x == budget && nb < cap ? mass_in[nb] : 0.0f;   // (the unfinished block's goes along)
    }
}

// ---- launches ----

static CacheArgs cache_args(const sparsek_cache8_cfg& c, const sparsek_cache8& t, const int32_t* lens)
{
    return CacheArgs{t, c.B, c.H, c.Hkv, c.H / c.Hkv, c.cap, c.pages, lens};
}

#define BY_FORMAT(c, LAUNCH)                                                          \
    if (c.d == 128 && c.format == SPARSEK_I8) { LAUNCH(128, SPARSEK_I8); }            \
    else if (c.d == 128) { LAUNCH(128, SPARSEK_E4M3); }                               \
    else if (c.format == SPARSEK_I8) { LAUNCH(64, SPARSEK_I8); }                      \
    else { LAUNCH(64, SPARSEK_E4M3); }

int launch_cache8_append(const sparsek_cache8_cfg& c, const sparsek_cache8& t, const int32_t* lens, const int32_t* counts, int count,
                         const void* k, const void* v, hipStream_t st)
{
    const CacheArgs a = cache_args(c, t, lens);
    const dim3 grid((unsigned)((count + 2 * BT - 2) / BT), c.B * c.Hkv);   // blocks that `count` tokens from any place touch
#define APPEND(D, F) hipLaunchKernelGGL((cache8_append_kernel<D, F>), grid, dim3(256), 0, st, a, counts, count, (const uint16_t*)k, (const uint16_t*)v)
    BY_FORMAT(c, APPEND)
#undef APPEND
    return launch_status();
}

int launch_cache8_select(const sparsek_cache8_cfg& c, const sparsek_cache8& t, const int32_t* lens, const void* q, int top, int32_t* idx, hipStream_t st)
{
    const CacheArgs a = cache_args(c, t, lens);
    const size_t lds = (size_t)c.cap * 8;
    if (c.d == 128) hipLaunchKernelGGL((cache8_select_kernel<128>), dim3(c.B * c.Hkv), dim3(1024), lds, st, a, (const uint16_t*)q, top, idx);
    else hipLaunchKernelGGL((cache8_select_kernel<64>), dim3(c.B * c.Hkv), dim3(1024), lds, st, a, (const uint16_t*)q, top, idx);
    return launch_status();
}

struct Cache8Layout {
    int units, splits, upw, groups;
    size_t part_o, part_ml, weight, bytes;
};
static Cache8Layout cache8_layout(const sparsek_cache8_cfg& c, int top)
{
    Cache8Layout y;
    y.units = (top ? top : c.cap) + 1;   // and the query's own block
    y.groups = (c.H / c.Hkv + 15) / 16;
    // Units per wave.  Up to 20 units and 16 heads of a group are one workgroup's, which needs no second launch.  Beyond that
    // as many as leave 8 waves for each of 256 compute units, 5 at most (sequences are shorter than the longest, and the waves that
    // they leave idle weigh less the fewer units each has: 64 sequences of up to 8192 127.5 us with 5, 128.3 with 4, 130 with 3, 136 with 2).
    const long long all = (long long)c.B * c.Hkv * y.groups * y.units;
    if (y.units <= 4 * MAX_UPW && y.groups == 1) y.upw = (y.units + 3) / 4;
    else y.upw = (int)std::max<long long>(1, std::min<long long>(MAX_UPW, all / 2048));
    y.splits = (y.units + 4 * y.upw - 1) / (4 * y.upw);
    const size_t parts = (size_t)c.B * c.H * y.splits;
    y.part_o = 0;
    y.part_ml = align_up(parts * c.d * 4, 256);
    y.weight = y.part_ml + align_up(parts * 8, 256);
    y.bytes = y.weight + align_up((size_t)c.B * c.H * y.units * 4, 256);
    return y;
}
size_t cache8_attn_ws_bytes(const sparsek_cache8_cfg& c, int top) { return cache8_layout(c, top).bytes; }

int launch_cache8_attn(const sparsek_cache8_cfg& c, const sparsek_cache8& t, const int32_t* lens, const void* q, const int32_t* idx, int top,
                       int accumulate, void* o, float* lse, void* ws, hipStream_t st)
{
    const Cache8Layout y = cache8_layout(c, idx ? top : 0);
    AttnArgs a;
    a.c = cache_args(c, t, lens);
    a.q = (const uint16_t*)q;
    a.idx = idx;
    a.top = idx ? top : 0;
    a.splits = y.splits;
    a.upw = y.upw;
    a.c2 = c.softmax_scale * 1.4426950408889634f;
    char* w = (char*)ws;
    a.part_o = (float*)(w + y.part_o); a.part_ml = (float2*)(w + y.part_ml);
    a.weight = (float*)(w + y.weight);
    a.accumulate = accumulate;
    a.units = y.units;
    a.o = (uint16_t*)o;
    a.lse = lse;
    const int mass_wgs = accumulate ? (y.units + 255) / 256 : 0;
#define ATTN(D, F) hipLaunchKernelGGL((cache8_attn_kernel<D, F>), dim3(y.splits, c.Hkv * y.groups, c.B), dim3(256), 0, st, a)
    BY_FORMAT(c, ATTN)
#undef ATTN
    if (y.splits == 1 && y.groups == 1) return launch_status();
    const dim3 join(c.H + c.Hkv * mass_wgs, c.B);
    if (c.d == 128) hipLaunchKernelGGL((cache8_join_kernel<128>), join, dim3(256), 0, st, a, std::max(mass_wgs, 1));
    else hipLaunchKernelGGL((cache8_join_kernel<64>), join, dim3(256), 0, st, a, std::max(mass_wgs, 1));
    return launch_status();
}

int launch_cache8_evict(const sparsek_cache8_cfg& c, const sparsek_cache8& t, const int32_t* lens, int budget, int sink, int recent,
                        int32_t* table, float* mass, int32_t* lens_out, hipStream_t st)
{
    const CacheArgs a = cache_args(c, t, lens);
hipLaunchKernelGGL(cache8_evict_kernel, dim3(c.B * c.Hkv), dim3(256), (size_t)c.cap * 8, st, a, budget, sink, recent, table, mass, lens_out);
    return launch_status();
}

}  // namespace spk
