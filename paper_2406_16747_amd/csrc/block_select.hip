// Selection of key blocks by a cheap score, for every query (prefill and training).
//
// mean_j = the mean key of block j (summed in fp64, which is exact for bf16 keys within 2^39 of each other), held as whole
// numbers m8_j of at most 127 with a scale ms_j; the queries of a group are added up and rounded the same way.  The score of
// block j for query i is float(p8_i . m8_j) * ms_j: the product is exact in 32 bits whatever the order of its sums, so the
// choice has one answer.  v_mfma_i32_16x16x64_i8 does it, 16 blocks by 16 queries at a time.  What bounds it is the vector ALU, which
// counts the scores above a bound: 282 us for 8 heads of keys and 32768 queries (512 blocks), 136 for 64 and 8192 (128 blocks).
#include "block_parts.hpp"

namespace spk {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Scales of a head: whole tiles of 16.
__host__ __device__ inline size_t scale_row(int nbw) { return (size_t)(nbw + 15) / 16 * 16; }

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
    if (tid == 0) kms[bg * scale_row(nbw) + j] = code_scale(top, 127.0f);
}

// The sum and the largest over the four lanes col, col + 16, col + 32, col + 48.
__device__ __forceinline__ unsigned groups_sum(unsigned x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    const unsigned y = (unsigned)a[0] + (unsigned)a[1];
    const auto b = __builtin_amdgcn_permlane16_swap(y, y, false, false);
    return (unsigned)b[0] + (unsigned)b[1];
}
__device__ __forceinline__ unsigned groups_max(unsigned x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    const unsigned y = max((unsigned)a[0], (unsigned)a[1]);
    const auto b = __builtin_amdgcn_permlane16_swap(y, y, false, false);
    return max((unsigned)b[0], (unsigned)b[1]);
}

// One workgroup of 4 waves per (64 queries, batch and head), a wave per 16 queries: a lane holds the order-preserving images of
// the scores of every fourth group of 4 blocks for one query.  A threshold with exactly `top` scores at or above it is
// found by bisection, first halfway between values, then between images; where equal scores leave no such threshold the first of
// those that share the last place are taken.  (Between the logarithms of the counts instead: 10 % slower, the logarithms cost more than
// the steps they save.)  Counting a score costs two instructions; a radix pass in LDS counters
// cost 4 to 8 times as much.  NT: tiles of 16 blocks whose images stay in registers; 0: any number, formed again for every count.
template <int D, int NT>
__global__ __launch_bounds__(256) void block_select_kernel(const uint16_t* __restrict__ q, int H, int Hkv, int n, int nbw, int top,
                                                           const int8_t* __restrict__ km, const float* __restrict__ kms,
                                                           int32_t* __restrict__ idx)
{
    __shared__ unsigned q8[64][D / 4 + 1];
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
            q8[r][DP / 4 * part + c] = pack4(code_i8(x[4 * c], f), code_i8(x[4 * c + 1], f), code_i8(x[4 * c + 2], f), code_i8(x[4 * c + 3], f));
    }
    __syncthreads();
    if (16 * wv >= rows) return;
    const int col = lane & 15, grp = lane >> 4;   // query of the wave, 16-byte piece of the operands / row group of the result
    i32x4 qf[D / 64];
#pragma unroll
    for (int s = 0; s < D / 64; s++)
#pragma unroll
        for (int e = 0; e < 4; e++) qf[s][e] = (int)q8[16 * wv + col][16 * s + 4 * grp + e];
    const int8_t* kmr = km + (size_t)bg * nbw * D;
    const float* msr = kms + (size_t)bg * scale_row(nbw);
    const int nt = (nbp + 15) / 16;
    typedef unsigned keys4 __attribute__((ext_vector_type(4)));
    // the images of blocks 16 t + 4 grp .. + 3 for query col; 0 (below every score) beyond the last block
    auto form = [&](int t) -> keys4 {
        const int row = min(16 * t + col, nbp - 1);
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < D / 64; s++) {
            const i32x4 a = *(const i32x4*)(kmr + (size_t)row * D + 64 * s + 16 * grp);
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, qf[s], acc, 0, 0, 0);
        }
        const f32x4v ms = *(const f32x4v*)(msr + 16 * t + 4 * grp);   // (the scales' rows are whole tiles long)
        keys4 key;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const unsigned b = __float_as_uint((float)acc[r] * ms[r] + 0.0f);   // (as score_key; 1 at least, and below the largest)
            key[r] = min(max(b ^ ((unsigned)((int)b >> 31) | 0x80000000u), 1u), 0xFFFFFFFEu);
        }
        if (t == nt - 1)
#pragma unroll
            for (int r = 0; r < 4; r++) key[r] = 16 * t + 4 * grp + r < nbp ? key[r] : 0u;
        return key;
    };
    keys4 kept[NT ? NT : 1];
    // f(t, images) for every tile, the numbers of tiles known to the compiler where they stay in registers
    auto each = [&](auto&& f) {
        if constexpr (NT > 0) {
            static_for<0, NT>([&](auto t) {
                if (t < nt) f((int)t, kept[t]);
            });
        } else {
            for (int t = 0; t < nt; t++) f(t, form(t));
        }
    };
    if constexpr (NT > 0)
        static_for<0, NT>([&](auto t) {
            if (t < nt) kept[t] = form(t);
        });
    unsigned most = 0, least = ~0u;
    each([&](int t, const keys4& k) {
#pragma unroll
        for (int r = 0; r < 4; r++) {
            most = max(most, k[r]);
            least = min(least, k[r] ? k[r] : ~0u);
        }
    });
    // at least `top` images are >= lo, fewer are >= hi
    unsigned lo = ~groups_max(~least), hi = groups_max(most) + 1, above = 0;
    bool done = false;
    for (int it = 0; __any(!done); it++) {
        unsigned mid = lo + (hi - lo) / 2;
        if (it < 20) {   // halfway between the values: scores of one size are found apart in about ten steps
            const unsigned m = score_key(0.5f * __uint_as_float(score_key_inv(lo)) + 0.5f * __uint_as_float(score_key_inv(hi - 1)));
            mid = m > lo && m < hi ? m : mid;
        }
        unsigned c = 0;
        each([&](int t, const keys4& k) {
#pragma unroll
            for (int r = 0; r < 4; r++) c += k[r] >= mid ? 1u : 0u;
        });
        c = groups_sum(c);
        if (!done) {
            if (mid == lo) done = true;              // hi == lo + 1: what is equal to lo shares the last places
            else if (c >= (unsigned)top) lo = mid;
            else { hi = mid; above = c; }
            if (!done && c == (unsigned)top) { hi = lo; above = c; done = true; }
        }
    }
    unsigned need = (unsigned)top - above, written = 0;   // places left for images equal to lo; written so far
    const bool live = 16 * wv + col < rows;
    int32_t* mine = out + (size_t)(16 * wv + col) * top;
    const unsigned long long all = 0x0001000100010001ull << col, lower = all & ((1ull << (16 * grp)) - 1);
    const bool ties = __any(need > 0);
    each([&](int t, const keys4& k) {
        bool in[4];
#pragma unroll
        for (int r = 0; r < 4; r++) in[r] = k[r] >= hi;
        if (ties) {
            unsigned eq = 0;
#pragma unroll
            for (int r = 0; r < 4; r++) eq |= (need > 0 && k[r] == lo ? 1u : 0u) << (4 * grp + r);
            eq = groups_sum(eq);   // (each bit is one lane's)
            unsigned take = 0;
            for (; eq && need; eq &= eq - 1, need--) take |= eq & -eq;
#pragma unroll
            for (int r = 0; r < 4; r++) in[r] |= take >> (4 * grp + r) & 1;
        }
        unsigned place = written;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const unsigned long long m = __ballot(in[r]);
            place += __popcll(m & lower);
            written += __popcll(m & all);
        }
#pragma unroll
        for (int r = 0; r < 4; r++)
            if (in[r]) {
                if (live) mine[place] = 16 * t + 4 * grp + r;
                place++;
            }
    });
}

size_t block_select_ws_bytes(const sparsek_block_cfg& c)
{
    const size_t BG = (size_t)c.B * c.Hkv, nbw = c.n / BT;
    // (0 is what the size query says of a configuration that is refused; without a whole block there is nothing to keep)
    return std::max<size_t>(256, align_up(BG * nbw * c.d, 256) + align_up(BG * scale_row(nbw) * sizeof(float), 256));
}

int launch_block_select(const sparsek_block_cfg& c, const void* q, const void* k, int32_t* idx, void* ws, hipStream_t st)
{
    if (c.top == 0) return SPARSEK_OK;
    const int nbw = c.n / BT, BG = c.B * c.Hkv;
    int8_t* km = (int8_t*)ws;
    float* kms = (float*)((char*)ws + align_up((size_t)BG * nbw * c.d, 256));
    const dim3 all(block_count(c.n), BG);
    if (nbw > c.top) {
        if (c.d == 128) hipLaunchKernelGGL((block_means_kernel<128>), dim3(nbw, BG), dim3(256), 0, st, (const uint16_t*)k, c.n, nbw, km, kms);
        else hipLaunchKernelGGL((block_means_kernel<64>), dim3(nbw, BG), dim3(256), 0, st, (const uint16_t*)k, c.n, nbw, km, kms);
    }
#define SELECT(D, NT) hipLaunchKernelGGL((block_select_kernel<D, NT>), all, dim3(256), 0, st, (const uint16_t*)q, c.H, c.Hkv, c.n, nbw, c.top, km, kms, idx)
#define BY_LENGTH(D)                          \
    if (nbw <= 128) { SELECT(D, 8); }         \
    else if (nbw <= 512) { SELECT(D, 32); }   \
    else { SELECT(D, 0); }
    if (c.d == 128) {
        BY_LENGTH(128)
    } else {
        BY_LENGTH(64)
    }
#undef BY_LENGTH
#undef SELECT
    return launch_status();
}

}  // namespace spk
