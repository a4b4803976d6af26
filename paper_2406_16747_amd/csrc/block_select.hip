// Selection of key blocks by a cheap score, for every query (prefill and training).
//
// mean_j = the mean key of block j (summed in fp64, which is exact for bf16 keys within 2^39 of each other), held as whole
// numbers m8_j of at most 127 with a scale ms_j; the queries of a group are added up and rounded the same way.  The score of
// block j for query i is float(p8_i . m8_j) * ms_j: the product is exact in 32 bits whatever the order of its sums, so the
// choice has one answer.  v_mfma_i32_16x16x64_i8 does it, 16 blocks by 16 queries at a time.
#include "block_parts.hpp"

namespace spk {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// One workgroup of 256 per (whole block, batch and head): m8 and ms.
template <int D>
__global__ __launch_bounds__(256) void block_means_kernel(const uint16_t* __restrict__ k, int n, int nbw, int8_t* __restrict__ km,
                                                          float* __restrict__ kms)
{
    constexpr int CPR = D / 8, RG = 256 / CPR;   // 16-byte pieces per row, groups of rows
    __shared__ double sums[RG][D];
    __shared__ unsigned red[4];
    const int tid = threadIdx.x, j = blockIdx.x;
    const size_t bg = blockIdx.y;
    const uint16_t* src = k + (bg * n + (size_t)j * BT) * D;
    double s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int t = 0; t < BT / RG; t++) {
        const u32x4 x = *(const u32x4*)(src + (size_t)(tid / CPR + RG * t) * D + 8 * (tid % CPR));
#pragma unroll
        for (int e = 0; e < 8; e++) s[e] += (double)__uint_as_float(e & 1 ? x[e / 2] & 0xFFFF0000u : x[e / 2] << 16);
    }
#pragma unroll
    for (int e = 0; e < 8; e++) sums[tid / CPR][8 * (tid % CPR) + e] = s[e];
    __syncthreads();
    float mean = 0.0f;
    if (tid < D) {
        double y = 0;
#pragma unroll
        for (int r = 0; r < RG; r++) y += sums[r][tid];
        mean = (float)(y / BT);
    }
    const float top = __uint_as_float(block_max_bits(__float_as_uint(fabsf(mean)), red, tid));
    if (tid < D) km[(bg * nbw + j) * D + tid] = (int8_t)code_i8(mean, code_factor(top, 127.0f));
    if (tid == 0) kms[bg * nbw + j] = code_scale(top, 127.0f);
}

// One workgroup of 4 waves per (64 queries, batch and head), a wave per 16 queries.  The `top` largest of up to thousands of
// scores by radix: four passes over the scores, 8 bits of their order-preserving image a pass, in counters per query; a
// pass forms the scores again (the matrix instructions cost less than keeping them).  A last pass writes what is above the
// threshold and, of those equal to it, the first ones, in ascending order.
template <int D>
struct SelectSmem {
    unsigned hist[4][16][257];
    unsigned q8[64][D / 4 + 1];
};

template <int D>
__global__ __launch_bounds__(256) void block_select_kernel(const uint16_t* __restrict__ q, int H, int Hkv, int n, int nbw, int top,
                                                           const int8_t* __restrict__ km, const float* __restrict__ kms,
                                                           int32_t* __restrict__ idx)
{
    __shared__ SelectSmem<D> sm;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int nbp = gridDim.x - 1 - blockIdx.x;   // blocks behind the chunk's own; long chunks first
    const int bg = blockIdx.y, b = bg / Hkv, g = bg % Hkv, G = H / Hkv;
    const int i0 = nbp * BT, rows = min(BT, n - i0);
    int32_t* out = idx + ((size_t)bg * n + i0) * top;
    if (nbp <= top) {   // everything behind the query
        for (int x = tid; x < rows * top; x += 256) out[x] = x % top < nbp ? x % top : -1;
        return;
    }
    // the group's queries, added up in fp64 and rounded: 4 threads per query
    {
        constexpr int DP = D / 4;
        const int r = tid >> 2, part = tid & 3, i = min(i0 + r, n - 1);
        float x[DP];
        float most = 0.0f;
#pragma unroll
        for (int c = 0; c < DP / 8; c++) {
            double s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            for (int h = 0; h < G; h++) {
                const u32x4 v = *(const u32x4*)(q + (((size_t)b * H + g * G + h) * n + i) * D + DP * part + 8 * c);
#pragma unroll
                for (int e = 0; e < 8; e++) s[e] += (double)__uint_as_float(e & 1 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16);
            }
#pragma unroll
            for (int e = 0; e < 8; e++) {
                x[8 * c + e] = (float)s[e];
                most = fmaxf(most, fabsf(x[8 * c + e]));
            }
        }
        most = fmaxf(most, __shfl_xor(most, 1, 64));
        most = fmaxf(most, __shfl_xor(most, 2, 64));
        const float f = code_factor(most, 127.0f);
#pragma unroll
        for (int c = 0; c < DP / 4; c++)
            sm.q8[r][DP / 4 * part + c] = pack4(code_i8(x[4 * c], f), code_i8(x[4 * c + 1], f), code_i8(x[4 * c + 2], f), code_i8(x[4 * c + 3], f));
    }
    __syncthreads();
    const int col = lane & 15, grp = lane >> 4;   // query of the wave, 16-byte piece of the operands / row group of the result
    i32x4 qf[D / 64];
#pragma unroll
    for (int s = 0; s < D / 64; s++)
#pragma unroll
        for (int e = 0; e < 4; e++) qf[s][e] = (int)sm.q8[16 * wv + col][16 * s + 4 * grp + e];
    const int8_t* kmr = km + (size_t)bg * nbw * D;
    const float* msr = kms + (size_t)bg * nbw;
    // the images of blocks 16 t + 4 grp .. + 3 for query col; 0 (below every score) beyond the last block
    auto keys = [&](int t, unsigned (&key)[4]) {
        const int row = min(16 * t + col, nbp - 1);
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < D / 64; s++) {
            const i32x4 a = *(const i32x4*)(kmr + (size_t)row * D + 64 * s + 16 * grp);
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, qf[s], acc, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const int j = 16 * t + 4 * grp + r;
            key[r] = j < nbp ? max(score_key((float)acc[r] * msr[min(j, nbp - 1)]), 1u) : 0u;
        }
    };
    const int nt = (nbp + 15) / 16;
    unsigned(*hist)[257] = sm.hist[wv];
    unsigned prefix = 0, need = top;   // the threshold's upper bits, and how many of the scores that share them are wanted
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int x = lane; x < 16 * 257; x += 64) (&hist[0][0])[x] = 0;
        __builtin_amdgcn_wave_barrier();
        for (int t = 0; t < nt; t++) {
            unsigned key[4];
            keys(t, key);
#pragma unroll
            for (int r = 0; r < 4; r++)
                if (shift == 24 || key[r] >> (shift + 8) == prefix) atomicAdd(&hist[col][key[r] >> shift & 255], 1u);
        }
        __builtin_amdgcn_wave_barrier();
        // lane (col, grp) adds up digits 64 grp .. 64 grp + 63; the threshold's digit is where the sum from the top reaches `need`
        unsigned mine = 0;
        for (int x = 0; x < 64; x++) mine += hist[col][64 * grp + x];
        unsigned above = 0;
#pragma unroll
        for (int y = 1; y < 4; y++) {
            const unsigned other = (unsigned)__shfl((int)mine, (col + 16 * (grp + y)) & 63, 64);
            if (grp + y < 4) above += other;
        }
        unsigned digit = 0, left = 0;
        const bool here = above < need && above + mine >= need;
        if (here) {
            unsigned sum = above;
            for (int x = 63; x >= 0; x--) {
                const unsigned c = hist[col][64 * grp + x];
                if (sum + c >= need) {
                    digit = 64 * grp + x;
                    left = need - sum;
                    break;
                }
                sum += c;
            }
        }
        // (one of a query's four lanes has found it)
        digit |= (unsigned)__shfl_xor((int)digit, 16, 64);
        left |= (unsigned)__shfl_xor((int)left, 16, 64);
        digit |= (unsigned)__shfl_xor((int)digit, 32, 64);
        left |= (unsigned)__shfl_xor((int)left, 32, 64);
        prefix = prefix << 8 | digit;
        need = left;
        __builtin_amdgcn_wave_barrier();
    }
    unsigned written = 0, equal = 0;   // so far, of this query
    const bool live = 16 * wv + col < rows;
    int32_t* mine = out + (size_t)(16 * wv + col) * top;
    for (int t = 0; t < nt; t++) {
        unsigned key[4];
        keys(t, key);
        unsigned gt = 0, eq = 0;   // bit 4 grp + r
#pragma unroll
        for (int r = 0; r < 4; r++) {
            gt |= (key[r] > prefix ? 1u : 0u) << (4 * grp + r);
            eq |= (key[r] == prefix ? 1u : 0u) << (4 * grp + r);
        }
        unsigned both = gt | eq << 16;
        both |= (unsigned)__shfl_xor((int)both, 16, 64);
        both |= (unsigned)__shfl_xor((int)both, 32, 64);
        gt = both & 0xFFFFu;
        eq = both >> 16;
        unsigned take = gt;
        for (unsigned e = eq; e && equal < need; e &= e - 1, equal++) take |= e & -e;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const unsigned bit = 1u << (4 * grp + r);
            if (live && (take & bit)) mine[written + __popc(take & (bit - 1))] = 16 * t + 4 * grp + r;
        }
        written += __popc(take);
    }
}

size_t block_select_ws_bytes(const sparsek_block_cfg& c)
{
    const size_t rows = (size_t)c.B * c.Hkv * (c.n / BT);
    return align_up(rows * c.d, 256) + align_up(rows * sizeof(float), 256);
}

int launch_block_select(const sparsek_block_cfg& c, const void* q, const void* k, int32_t* idx, void* ws, hipStream_t st)
{
    if (c.top == 0) return SPARSEK_OK;
    const int nbw = c.n / BT, BG = c.B * c.Hkv;
    int8_t* km = (int8_t*)ws;
    float* kms = (float*)((char*)ws + align_up((size_t)BG * nbw * c.d, 256));
    const dim3 all(block_count(c.n), BG);
#define SELECT(D)                                                                                                                  \
    if (nbw > c.top) hipLaunchKernelGGL((block_means_kernel<D>), dim3(nbw, BG), dim3(256), 0, st, (const uint16_t*)k, c.n, nbw, km, kms); \
    hipLaunchKernelGGL((block_select_kernel<D>), all, dim3(256), 0, st, (const uint16_t*)q, c.H, c.Hkv, c.n, nbw, c.top, km, kms, idx)
    if (c.d == 128) {
        SELECT(128);
    } else {
        SELECT(64);
    }
#undef SELECT
    return launch_status();
}

}  // namespace spk
