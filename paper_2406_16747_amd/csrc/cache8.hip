// A key/value cache in blocks of 64 tokens, held in 8 bits with a scale for each block and head.
//
// A page holds one block of one key/value head: keys [64][D] and values transposed [D][64], so that both products of the
// attention read their 8-bit operands as they lie (16 bytes a lane).  The table names a head's pages by age; the unfinished
// block at the end of a sequence is kept in bf16, values transposed as well.  Page numbers outside the pool are never
// followed: such a page is neither written nor attended.
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
    u32x4 k[NT], v[NT];
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
    double sums[256 / (D / 8)][D];
    unsigned char vt[D][BT + 16];
    unsigned red[4];
};

// A whole block goes to its page: codes, scales and the mean key.
template <int D, int FORMAT>
__device__ __forceinline__ void store_block(AppendSmem<D>& sm, const CacheArgs& a, int page, const BlockRegs<D>& r, int tid)
{
    using R = BlockRegs<D>;
    const float most = FORMAT == SPARSEK_I8 ? 127.0f : 448.0f;
    const int tok = tid / R::CPR, c = tid % R::CPR;
    unsigned tk = 0, tv = 0;
    double s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < R::NT; t++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float k = half_of(r.k[t], e);
            s[e] += (double)k;
            tk = max(tk, __float_as_uint(fabsf(k)));
            tv = max(tv, __float_as_uint(fabsf(half_of(r.v[t], e))));
        }
    const float topk = __uint_as_float(block_max_bits(tk, sm.red, tid)), topv = __uint_as_float(block_max_bits(tv, sm.red, tid));
    const float fk = code_factor(topk, most), fv = code_factor(topv, most);
#pragma unroll
    for (int e = 0; e < 8; e++) sm.sums[tok][8 * c + e] = s[e];
    unsigned char* kp = (unsigned char*)a.t.k8 + (size_t)page * BT * D;
#pragma unroll
    for (int t = 0; t < R::NT; t++) {
        u32x2 w;
        w[0] = codes4<FORMAT>(half_of(r.k[t], 0), half_of(r.k[t], 1), half_of(r.k[t], 2), half_of(r.k[t], 3), fk);
        w[1] = codes4<FORMAT>(half_of(r.k[t], 4), half_of(r.k[t], 5), half_of(r.k[t], 6), half_of(r.k[t], 7), fk);
        *(u32x2*)(kp + (tok + R::RG * t) * D + 8 * c) = w;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const unsigned x = codes4<FORMAT>(half_of(r.v[t], 4 * h), half_of(r.v[t], 4 * h + 1), half_of(r.v[t], 4 * h + 2), half_of(r.v[t], 4 * h + 3), fv);
#pragma unroll
            for (int e = 0; e < 4; e++) sm.vt[8 * c + 4 * h + e][tok + R::RG * t] = (unsigned char)(x >> (8 * e));
        }
    }
    __syncthreads();
    unsigned char* vp = (unsigned char*)a.t.v8 + (size_t)page * BT * D;
    for (int x = tid; x < D * (BT / 16); x += 256) *(u32x4*)(vp + 16 * x) = *(const u32x4*)&sm.vt[x / 4][16 * (x % 4)];
    float mean = 0.0f;
    if (tid < D) {
        double y = 0;
#pragma unroll
        for (int g = 0; g < R::RG; g++) y += sm.sums[g][tid];
        mean = (float)(y / BT);
    }
    const float topm = __uint_as_float(block_max_bits(__float_as_uint(fabsf(mean)), sm.red, tid));
    if (tid < D) a.t.km[(size_t)page * D + tid] = (int8_t)code_i8(mean, code_factor(topm, 127.0f));
    if (tid == 0) {
        a.t.ks[page] = code_scale(topk, most);
        a.t.vs[page] = code_scale(topv, most);
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
    __shared__ __attribute__((aligned(16))) AppendSmem<D> sm;
    const int tid = threadIdx.x, bg = blockIdx.y, b = bg / a.Hkv;
    const int len = clamp_len(a.lens[b], a.cap);
    const int count = min(counts ? min(max(counts[b], 0), c) : c, a.cap * BT + BT - 1 - len);   // (what does not fit is dropped)
    if (count <= 0) return;
    const int after = len + count, first = len / BT, j = first + blockIdx.x;
    if (j * BT >= after) return;
    const uint16_t *kn = k + (size_t)bg * c * D, *vn = v + (size_t)bg * c * D;
    uint16_t *kt = (uint16_t*)a.t.kt + (size_t)bg * BT * D, *vt = (uint16_t*)a.t.vt + (size_t)bg * BT * D;
    if ((j + 1) * BT <= after) {
        R r;
        const int page = a.t.table[(size_t)bg * a.cap + j];
#pragma unroll
        for (int t = 0; t < R::NT; t++) {
            const int tok = j * BT + tid / R::CPR + R::RG * t, col = 8 * (tid % R::CPR);
            if (tok >= len) {
                r.k[t] = *(const u32x4*)(kn + (size_t)(tok - len) * D + col);
                r.v[t] = *(const u32x4*)(vn + (size_t)(tok - len) * D + col);
            } else {
                r.k[t] = *(const u32x4*)(kt + (tok % BT) * D + col);
#pragma unroll
                for (int e = 0; e < 4; e++) r.v[t][e] = (unsigned)vt[(col + 2 * e) * BT + tok % BT] | (unsigned)vt[(col + 2 * e + 1) * BT + tok % BT] << 16;
            }
        }
        if (page >= 0 && page < a.pages) store_block<D, FORMAT>(sm, a, page, r, tid);
    }
    const int whole = after / BT;   // the block that stays unfinished, if it has tokens
    if (blockIdx.x != 0) return;
    __syncthreads();                // everybody has read what is overwritten now
    const int t0 = max(len, whole * BT);
    for (int x = tid; x < (after - t0) * D; x += 256) {
        const int tok = t0 + x / D, col = x % D;
        kt[(tok % BT) * D + col] = kn[(size_t)(tok - len) * D + col];
        vt[col * BT + tok % BT] = vn[(size_t)(tok - len) * D + col];
    }
}

// ---- the `top` largest of n keys in LDS, by radix: four passes of 8 bits ----

// What a workgroup of 1024 keeps in LDS beside the keys.
struct TopSmem {
    unsigned hist[256], digit, left;
    int wsum[16][2];
};

// The threshold of the `need` largest (need <= n, need >= 1) and how many of those equal to it belong to them.
__device__ __forceinline__ void top_threshold(TopSmem& sm, const unsigned* keys, int n, unsigned need, unsigned& thr, unsigned& equal)
{
    const int tid = threadIdx.x, lane = tid & 63;
    unsigned prefix = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) sm.hist[tid] = 0;
        __syncthreads();
        for (int x = tid; x < n; x += 1024)
            if (shift == 24 || keys[x] >> (shift + 8) == prefix) atomicAdd(&sm.hist[keys[x] >> shift & 255], 1u);
        __syncthreads();
        if (tid < 64) {   // lane: digits 255 - 4 lane .. 252 - 4 lane
            unsigned c[4], mine = 0;
#pragma unroll
            for (int e = 0; e < 4; e++) mine += c[e] = sm.hist[255 - 4 * lane - e];
            unsigned sum = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const unsigned y = (unsigned)__shfl_up((int)sum, d, 64);
                if (lane >= d) sum += y;
            }
            unsigned above = sum - mine;
            if (above < need && sum >= need) {
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    if (above < need && above + c[e] >= need) {
                        sm.digit = 255 - 4 * lane - e;
                        sm.left = need - above;
                    }
                    above += c[e];
                }
            }
        }
        __syncthreads();
        prefix = prefix << 8 | sm.digit;
        need = sm.left;
    }
    thr = prefix;
    equal = need;
    __syncthreads();
}

// emit(x, kept, place): every x < n in order, whether it belongs to the `need` largest (of equal ones the first), and its place
// among the kept ones or among the others.
template <typename F>
__device__ __forceinline__ void top_emit(TopSmem& sm, const unsigned* keys, int n, unsigned thr, unsigned equal, F&& emit)
{
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const unsigned long long below = (1ull << lane) - 1;
    int kept = 0, eqs = 0;
    for (int x0 = 0; x0 < n; x0 += 1024) {
        const int x = x0 + tid;
        const unsigned key = x < n ? keys[x] : 0;
        const bool gt = x < n && key > thr, eq = x < n && key == thr;
        const unsigned long long mg = __ballot(gt), me = __ballot(eq);
        if (lane == 0) {
            sm.wsum[wv][0] = __popcll(mg);
            sm.wsum[wv][1] = __popcll(me);
        }
        __syncthreads();
        int g = kept, e = eqs, ga = 0, ea = 0;
#pragma unroll
        for (int w = 0; w < 16; w++) {
            const int a = sm.wsum[w][0], c = sm.wsum[w][1];
            if (w < wv) { g += a; e += c; }
            ga += a;
            ea += c;
        }
        // kept so far = those above the threshold + the first `equal` of those at it
        g += __popcll(mg & below);
        e += __popcll(me & below);
        const int before = g + min(e, (int)equal);
        if (x < n) {
            const bool in = gt || (eq && e < (int)equal);
            emit(x, in, in ? before : x - before);
        }
        kept += ga;
        eqs += ea;
        __syncthreads();
    }
}

// ---- selection of blocks for a single query ----

template <int D>
__global__ __launch_bounds__(1024) void cache8_select_kernel(CacheArgs a, const uint16_t* __restrict__ q, int top, int32_t* __restrict__ idx)
{
    extern __shared__ unsigned keys[];
    __shared__ TopSmem sm;
    __shared__ unsigned q8[D / 4];
    constexpr int LPB = D / 16;   // lanes per block: 16 bytes each
    const int tid = threadIdx.x, bg = blockIdx.x, b = bg / a.Hkv, g = bg % a.Hkv;
    const int len = clamp_len(a.lens[b], a.cap);
    const int nb = len > 0 ? (len - 1) / BT : 0;   // blocks behind the query's own
    int32_t* out = idx + (size_t)bg * top;
    if (nb <= top) {
        for (int x = tid; x < top; x += 1024) out[x] = x < nb ? x : -1;
        return;
    }
    if (tid < 64) {   // the group's queries, added up and rounded
        constexpr int PL = D / 64;
        float x[PL];
        float most = 0.0f;
#pragma unroll
        for (int e = 0; e < PL; e++) {
            double s = 0;
            for (int h = 0; h < a.G; h++) s += (double)bf16_to_f32(q[((size_t)b * a.H + g * a.G + h) * D + PL * tid + e]);
            x[e] = (float)s;
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
    for (int x0 = 0; x0 < nb; x0 += 1024 / LPB) {
        const int x = x0 + tid / LPB;
        const int page = a.t.table[(size_t)bg * a.cap + min(x, nb - 1)];
        const bool ok = page >= 0 && page < a.pages;
        const i32x4 m = *(const i32x4*)(a.t.km + (size_t)(ok ? page : 0) * D + 16 * c);
        int s = 0;
#pragma unroll
        for (int e = 0; e < 4; e++) s = __builtin_amdgcn_sdot4(m[e], qv[e], s, false);
#pragma unroll
        for (int d = 1; d < LPB; d <<= 1) s += __shfl_xor(s, d, 64);
        if (c == 0 && x < nb) keys[x] = ok ? max(score_key((float)s * a.t.kms[page]), 1u) : 0u;
    }
    __syncthreads();
    unsigned thr, equal;
    top_threshold(sm, keys, nb, top, thr, equal);
    top_emit(sm, keys, nb, thr, equal, [&](int x, bool in, int place) {
        if (in) out[place] = x;
    });
}

// ---- attention of a single query per sequence ----

// A workgroup has 4 waves, and a wave takes whole blocks: S = K.Q^T (64 tokens by 16 heads), the running softmax, O^T += V^T.P^T.
// The pieces of a block go from memory to the matrix instructions without LDS or lane exchange: row m of S's tile t is token
// 16 (m / 4) + 4 t + m % 4, so a lane's 16 weights are those of the 16 tokens whose values it loads for every column.
struct AttnArgs {
    CacheArgs c;
    const uint16_t* q;
    const int32_t* idx;    // [B,Hkv,top] or null: all blocks
    int top, splits;
    float c2;
    float *part_o, *part_m, *part_l;   // [B,Hkv,row groups,splits][16][D], [..][16]
    float* weight;                     // [B,H,units]: log2 of a unit's share before the division; null: no masses
    int units;                         // units per row at most
    uint16_t* o;
    float* lse;
};

template <int FORMAT>
__device__ __forceinline__ bf16x8 widen(unsigned lo, unsigned hi)
{
    bf16x8 r;
    const unsigned w[2] = {lo, hi};
#pragma unroll
    for (int x = 0; x < 2; x++) {
        if constexpr (FORMAT == SPARSEK_I8) {
#pragma unroll
            for (int e = 0; e < 4; e++) r[4 * x + e] = (__bf16)(float)((int)(w[x] << (24 - 8 * e)) >> 24);
        } else {
            const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[x], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[x], true);
            r[4 * x] = (__bf16)a[0]; r[4 * x + 1] = (__bf16)a[1]; r[4 * x + 2] = (__bf16)b[0]; r[4 * x + 3] = (__bf16)b[1];
        }
    }
    return r;
}

typedef float f32x4m __attribute__((ext_vector_type(4)));

// What unit u of a row is: the place in the table, or -1 (no such block, one named before, a page outside the pool); the
// unfinished block is the unit behind the others.
struct RowUnits {
    int whole, tail, nsel;   // whole blocks, tokens of the unfinished one, units that idx names (or whole)
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
// (wave-uniform u; all lanes)
__device__ __forceinline__ int unit_block(const AttnArgs& a, const RowUnits& r, size_t bg, int u, int lane)
{
    if (!a.idx) return u;
    if (u == a.top) return r.own;
    const int32_t* row = a.idx + bg * a.top;
    const int x = row[u];
    if (x < 0 || x >= (r.own >= 0 ? r.own : r.whole)) return -1;
    bool seen = false;
    for (int s = lane; s < u; s += 64) seen |= row[s] == x;
    return __any(seen) ? -1 : x;
}

template <int D, int FORMAT>
__global__ __launch_bounds__(256, 2) void cache8_attn_kernel(AttnArgs a)
{
    constexpr int KH = D / 64, NX = D / 16;
    __shared__ float so[4][16][D + 4], sm_[4][16], sl[4][16];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, grp = lane >> 4;
    const int groups = (a.c.G + 15) / 16;
    const int split = blockIdx.x, g = blockIdx.y / groups, rg = blockIdx.y % groups, b = blockIdx.z;
    const size_t bg = (size_t)b * a.c.Hkv + g;
    const RowUnits ru = row_units(a, b);
    const int nu = ru.nsel + (ru.tail ? 1 : 0);
    const int head = g * a.c.G + rg * 16 + col;
    const bool live = rg * 16 + col < a.c.G;
    const size_t prow = (bg * groups + rg) * a.splits + split;
    // Q^T: head col, columns 64 half + 16 grp + 8 sub ..
    bf16x8 qf[KH][2];
    const uint16_t* qr = a.q + ((size_t)b * a.c.H + (live ? head : g * a.c.G)) * D;
#pragma unroll
    for (int h = 0; h < KH; h++)
#pragma unroll
        for (int s = 0; s < 2; s++) qf[h][s] = *(const bf16x8*)(qr + 64 * h + 16 * grp + 8 * s);
    f32x4m acc[NX];
#pragma unroll
    for (int x = 0; x < NX; x++) acc[x] = f32x4m{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;
    for (int u = split * 4 + wv; u < nu; u += a.splits * 4) {
        f32x4m s[4];
        float vscale = 1.0f;
        const bool tail = u == ru.nsel;
        const unsigned char* vp = nullptr;
        bool skip = false;
        if (!tail) {
            const int j = unit_block(a, ru, bg, u, lane);
            const int page = j >= 0 ? a.c.t.table[bg * a.c.cap + j] : -1;
            skip = page < 0 || page >= a.c.pages;
            if (!skip) {
                const unsigned char* kp = (const unsigned char*)a.c.t.k8 + (size_t)page * BT * D + (16 * (col >> 2) + (col & 3)) * D + 16 * grp;
                const float ks = a.c.t.ks[page] * a.c2;
                vscale = a.c.t.vs[page];
                vp = (const unsigned char*)a.c.t.v8 + (size_t)page * BT * D + col * BT + 16 * grp;
#pragma unroll
                for (int t = 0; t < 4; t++) {
                    s[t] = f32x4m{0, 0, 0, 0};
#pragma unroll
                    for (int h = 0; h < KH; h++) {
                        const u32x4 w = *(const u32x4*)(kp + 4 * t * D + 64 * h);
                        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FORMAT>(w[0], w[1]), qf[h][0], s[t], 0, 0, 0);
                        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FORMAT>(w[2], w[3]), qf[h][1], s[t], 0, 0, 0);
                    }
                    s[t] *= ks;
                }
            }
        } else {
            const uint16_t* kp = (const uint16_t*)a.c.t.kt + bg * BT * D;
#pragma unroll
            for (int t = 0; t < 4; t++) {
                s[t] = f32x4m{0, 0, 0, 0};
                const int tok = min(16 * (col >> 2) + 4 * t + (col & 3), ru.tail - 1);
#pragma unroll
                for (int h = 0; h < KH; h++)
#pragma unroll
                    for (int x = 0; x < 2; x++)
                        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8*)(kp + tok * D + 64 * h + 16 * grp + 8 * x), qf[h][x], s[t], 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; r++) s[t][r] = 16 * grp + 4 * t + r < ru.tail ? s[t][r] * a.c2 : -INFINITY;
            }
        }
        if (skip) {
            if (a.weight && live && grp == 0) a.weight[((size_t)b * a.c.H + head) * a.units + u] = -INFINITY;
            continue;
        }
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; t++)
#pragma unroll
            for (int r = 0; r < 4; r++) top = fmaxf(top, s[t][r]);
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mx = fmaxf(m, top), mn = mx == -INFINITY ? 0.0f : mx, corr = __builtin_amdgcn_exp2f(m - mn);
        m = mx;
        float sum = 0.0f;
        bf16x8 pb[2];
#pragma unroll
        for (int t = 0; t < 4; t++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const float p = __builtin_amdgcn_exp2f(s[t][r] - mn);
                sum += p;
                pb[t >> 1][4 * (t & 1) + r] = (__bf16)(p * vscale);   // the operand of the second product: 2^-9 of every weight
            }
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        if (a.weight && live && grp == 0) a.weight[((size_t)b * a.c.H + head) * a.units + u] = mn + log2f(sum);
        l = l * corr + sum;
#pragma unroll
        for (int x = 0; x < NX; x++) {
            acc[x] *= corr;
            if (!tail) {
                const u32x4 w = *(const u32x4*)(vp + 16 * x * BT);
                acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FORMAT>(w[0], w[1]), pb[0], acc[x], 0, 0, 0);
                acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FORMAT>(w[2], w[3]), pb[1], acc[x], 0, 0, 0);
            } else {
                const uint16_t* vr = (const uint16_t*)a.c.t.vt + (bg * D + 16 * x + col) * BT + 16 * grp;
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    u32x4 w = *(const u32x4*)(vr + 8 * y);
#pragma unroll
                    for (int e = 0; e < 4; e++) {   // what lies behind the last token may be anything
                        const int tok = 16 * grp + 8 * y + 2 * e;
                        w[e] = tok + 1 < ru.tail ? w[e] : tok < ru.tail ? w[e] & 0xFFFFu : 0u;
                    }
                    acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), pb[y], acc[x], 0, 0, 0);
                }
            }
        }
    }
    // the four waves' results are joined; rows 4 grp + r of tile x are columns of the head
    if (grp == 0) { sm_[wv][col] = m; sl[wv][col] = l; }
#pragma unroll
    for (int x = 0; x < NX; x++) *(f32x4m*)&so[wv][col][16 * x + 4 * grp] = acc[x];
    __syncthreads();
    for (int x = tid; x < 16 * D; x += 256) {
        const int h = x / D, d = x % D;
        const float M = fmaxf(fmaxf(sm_[0][h], sm_[1][h]), fmaxf(sm_[2][h], sm_[3][h]));
        float sum = 0.0f, den = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; w++) {
            const float f = sm_[w][h] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(sm_[w][h] - M);
            sum += f * so[w][h][d];
            den += f * sl[w][h];
        }
        a.part_o[prow * 16 * D + x] = sum;
        if (d == 0) {
            a.part_m[prow * 16 + h] = M;
            a.part_l[prow * 16 + h] = den;
        }
    }
}

// The splits of a head are joined (workgroups 0 .. H-1 of a sequence), and the shares of its blocks join the masses (the others).
template <int D>
__global__ __launch_bounds__(256) void cache8_join_kernel(AttnArgs a, int mass_wgs)
{
    const int tid = threadIdx.x, b = blockIdx.y, G = a.c.G, groups = (G + 15) / 16;
    auto total = [&](int h, float& M, float& L) {   // of head h
        const int g = h / G, r = h % G;
        const size_t p0 = (((size_t)b * a.c.Hkv + g) * groups + r / 16) * a.splits;
        M = -INFINITY;
        for (int s = 0; s < a.splits; s++) M = fmaxf(M, a.part_m[(p0 + s) * 16 + r % 16]);
        L = 0.0f;
        if (M > -INFINITY)
            for (int s = 0; s < a.splits; s++) L += a.part_l[(p0 + s) * 16 + r % 16] * __builtin_amdgcn_exp2f(a.part_m[(p0 + s) * 16 + r % 16] - M);
    };
    if ((int)blockIdx.x < a.c.H) {
        const int h = blockIdx.x, g = h / G, r = h % G;
        const size_t p0 = (((size_t)b * a.c.Hkv + g) * groups + r / 16) * a.splits;
        float M, L;
        total(h, M, L);
        if (tid < D) {
            float sum = 0.0f;
            if (M > -INFINITY)
                for (int s = 0; s < a.splits; s++) {
                    const float m = a.part_m[(p0 + s) * 16 + r % 16];
                    if (m > -INFINITY) sum += a.part_o[((p0 + s) * 16 + r % 16) * D + tid] * __builtin_amdgcn_exp2f(m - M);
                }
            a.o[((size_t)b * a.c.H + h) * D + tid] = f32_to_bf16(L > 0.0f ? sum / L : M > -INFINITY ? sum : 0.0f);
        }
        if (tid == 0) a.lse[(size_t)b * a.c.H + h] = M > -INFINITY ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
        return;
    }
    const int g = (blockIdx.x - a.c.H) / mass_wgs, part = (blockIdx.x - a.c.H) % mass_wgs;
    const size_t bg = (size_t)b * a.c.Hkv + g;
    const RowUnits ru = row_units(a, b);
    const int nu = ru.nsel + (ru.tail ? 1 : 0);
    if (part * 256 >= nu) return;
    const int u = part * 256 + tid;
    float sum = 0.0f;
    for (int r = 0; r < G; r++) {
        float M, L;
        total(g * G + r, M, L);
        const float w = u < nu ? a.weight[((size_t)b * a.c.H + g * G + r) * a.units + u] : -INFINITY;
        if (w > -INFINITY) sum += __builtin_amdgcn_exp2f(w - (M + log2f(L)));
    }
    if (u < nu) {
        const int j = u == ru.nsel ? ru.whole : !a.idx ? u : u == a.top ? ru.own : a.idx[bg * a.top + u];
        // (a unit that was left out has weight 0 and may name any place)
        if (j >= 0 && j < a.c.cap && sum != 0.0f) a.c.t.mass[bg * a.c.cap + j] += sum;
    }
}

// ---- eviction ----

__global__ __launch_bounds__(1024) void cache8_evict_kernel(CacheArgs a, int budget, int sink, int recent, int32_t* table, float* mass, int32_t* lens)
{
    extern __shared__ unsigned keys[];
    __shared__ TopSmem sm;
    const int tid = threadIdx.x, bg = blockIdx.x, b = bg / a.Hkv, cap = a.cap;
    const int len = clamp_len(a.lens[b], cap), nb = len / BT;
    const size_t row = (size_t)bg * cap;
    if (nb <= budget) {
        for (int x = tid; x < cap; x += 1024) {
            table[row + x] = a.t.table[row + x];
            mass[row + x] = a.t.mass[row + x];
        }
        if (bg % a.Hkv == 0 && tid == 0) lens[b] = len;
        return;
    }
    const float tail = nb < cap ? a.t.mass[row + nb] : 0.0f;
    for (int x = tid; x < nb; x += 1024)
        keys[x] = x < sink || x >= nb - recent ? 0xFFFFFFFFu : min(score_key(a.t.mass[row + x]), 0xFFFFFFFEu);
    __syncthreads();
    unsigned thr, equal;
    if (budget > 0) top_threshold(sm, keys, nb, budget, thr, equal);
    else { thr = 0xFFFFFFFFu; equal = 0; }
    top_emit(sm, keys, nb, thr, equal, [&](int x, bool in, int place) {
        table[row + (in ? place : budget + place)] = a.t.table[row + x];
        if (in) mass[row + place] = a.t.mass[row + x];
    });
    for (int x = budget + tid; x < cap; x += 1024) {
        mass[row + x] = x == budget ? tail : 0.0f;
        if (x >= nb) table[row + x] = a.t.table[row + x];
    }
    if (bg % a.Hkv == 0 && tid == 0) lens[b] = budget * BT + len % BT;
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
    const size_t lds = (size_t)c.cap * 4;
    if (c.d == 128) hipLaunchKernelGGL((cache8_select_kernel<128>), dim3(c.B * c.Hkv), dim3(1024), lds, st, a, (const uint16_t*)q, top, idx);
    else hipLaunchKernelGGL((cache8_select_kernel<64>), dim3(c.B * c.Hkv), dim3(1024), lds, st, a, (const uint16_t*)q, top, idx);
    return launch_status();
}

struct Cache8Layout {
    int units, splits, groups;
    size_t part_o, part_m, part_l, weight, bytes;
};
static Cache8Layout cache8_layout(const sparsek_cache8_cfg& c, int top)
{
    Cache8Layout y;
    y.units = (top ? top : c.cap) + 1;   // and the query's own block
    y.groups = (c.H / c.Hkv + 15) / 16;
    // enough workgroups for two on each of 256 compute units, and at least one unit for every wave
    const long long rows = (long long)c.B * c.Hkv * y.groups;
    y.splits = (int)std::max<long long>(1, std::min<long long>((512 + rows - 1) / rows, (y.units + 3) / 4));
    const size_t parts = (size_t)rows * y.splits * 16;
    y.part_o = 0;
    y.part_m = align_up(parts * c.d * 4, 256);
    y.part_l = y.part_m + align_up(parts * 4, 256);
    y.weight = y.part_l + align_up(parts * 4, 256);
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
    a.c2 = c.softmax_scale * 1.4426950408889634f;
    char* w = (char*)ws;
    a.part_o = (float*)(w + y.part_o); a.part_m = (float*)(w + y.part_m); a.part_l = (float*)(w + y.part_l);
    a.weight = accumulate ? (float*)(w + y.weight) : nullptr;
    a.units = y.units;
    a.o = (uint16_t*)o;
    a.lse = lse;
    const int mass_wgs = accumulate ? (y.units + 255) / 256 : 0;
#define ATTN(D, F) hipLaunchKernelGGL((cache8_attn_kernel<D, F>), dim3(y.splits, c.Hkv * y.groups, c.B), dim3(256), 0, st, a)
    BY_FORMAT(c, ATTN)
#undef ATTN
    const dim3 join(c.H + c.Hkv * mass_wgs, c.B);
    if (c.d == 128) hipLaunchKernelGGL((cache8_join_kernel<128>), join, dim3(256), 0, st, a, std::max(mass_wgs, 1));
    else hipLaunchKernelGGL((cache8_join_kernel<64>), join, dim3(256), 0, st, a, std::max(mass_wgs, 1));
    return launch_status();
}

int launch_cache8_evict(const sparsek_cache8_cfg& c, const sparsek_cache8& t, const int32_t* lens, int budget, int sink, int recent,
                        int32_t* table, float* mass, int32_t* lens_out, hipStream_t st)
{
    const CacheArgs a = cache_args(c, t, lens);
    hipLaunchKernelGGL(cache8_evict_kernel, dim3(c.B * c.Hkv), dim3(1024), (size_t)c.cap * 4, st, a, budget, sink, recent, table, mass, lens_out);
    return launch_status();
}

}  // namespace spk
