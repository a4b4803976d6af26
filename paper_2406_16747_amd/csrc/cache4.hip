// Reading the cache in 4 bits back: tokens of every sequence as bf16, which holds their values exactly.  (Its append, attention, selection
// and eviction share their kernels with the cache in 8 bits.)
#include "cache4_parts.hpp"

namespace spk {

struct ReadArgs {
    sparsek_cache4 t;
    int Hkv, cap, pages, begin, n;
    const int32_t* lens;
    uint16_t *k, *v;   // [B,Hkv,n,D]
};

// One workgroup of 256 per (block that the range touches, batch and head).  What bounds it is writing: STREAM leaves the chip's caches out where
// much is written (a prefix of 4096 for 16 sequences, 8 heads of 128, 268 MB: 52 us, 6.0 TB/s, and 70 through them; for 8 of them 27 and 38, for 4 of
// them, 67 MB, 14.3 and 13.1).
template <int D, bool STREAM>
__global__ __launch_bounds__(256) void cache4_read_kernel(ReadArgs a)
{
    using P = Page4<D>;
    constexpr int C8 = D / 8;
    __shared__ __attribute__((aligned(16))) unsigned char codes[2][P::CODES], scales[2][P::SCALES];
    const int tid = threadIdx.x, bg = blockIdx.y, b = bg / a.Hkv;
    const int len = min(max(a.lens[b], 0), a.cap * BT + BT - 1);
    const int j = a.begin / BT + blockIdx.x, first = j * BT - a.begin;   // the block's first token, as a row of the outputs
    uint16_t *ko = a.k + (size_t)bg * a.n * D, *vo = a.v + (size_t)bg * a.n * D;
    auto out_row = [&](int s) { return first + s >= 0 && first + s < a.n; };
    auto put = [&](uint16_t* o, int s, int c8, u32x4 w) {
        u32x4* at = (u32x4*)(o + (size_t)(first + s) * D + 8 * c8);
        if (!out_row(s)) return;
        if constexpr (STREAM) __builtin_nontemporal_store(w, at);
        else *at = w;
    };
    const int live = min(len - j * BT, BT);                  // tokens of the block that are there
    const int page = live == BT && j < a.cap ? a.t.table[(size_t)bg * a.cap + j] : -1;
    if (live == BT && page >= 0 && page < a.pages) {
        if (tid < P::CODES / 16) {
            *(u32x4*)&codes[0][16 * tid] = *(const u32x4*)((const unsigned char*)a.t.k4 + (size_t)page * P::CODES + 16 * tid);
            *(u32x4*)&codes[1][16 * tid] = *(const u32x4*)((const unsigned char*)a.t.v4 + (size_t)page * P::CODES + 16 * tid);
        }
        if (tid < P::SCALES / 4) {
            *(unsigned*)&scales[0][4 * tid] = *(const unsigned*)(a.t.ke + (size_t)page * P::SCALES + 4 * tid);
            *(unsigned*)&scales[1][4 * tid] = *(const unsigned*)(a.t.ve + (size_t)page * P::SCALES + 4 * tid);
        }
        const float ks = a.t.ks[page], vs = a.t.vs[page];
        const u32x4 none = {0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};   // (a page with a value that is not finite)
        __syncthreads();
        for (int x = tid; x < BT * C8; x += 256) {
            const int s = x / C8, c8 = x % C8;
            const unsigned w = *(const unsigned*)&codes[0][P::key_at(s, c8)];
            const float scale = __uint_as_float((unsigned)scales[0][P::key_scale_at(s, c8 / 4)] << 23);
            u32x4 y;
            y[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
            y[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
            y[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
            y[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
            put(ko, s, c8, ks == ks ? y : none);
        }
        // 8 channels of 8 tokens to a thread: two tokens of a channel come together, and go to rows of their own
        for (int x = tid; x < 8 * C8; x += 256) {
            const int s8 = x / C8, c8 = x % C8;
            u32x4 y[8];
#pragma unroll
            for (int h = 0; h < 4; h++) {   // channels 8 c8 + 2 h and the next
                unsigned w[2];
                float scale[2];
#pragma unroll
                for (int z = 0; z < 2; z++) {
                    w[z] = *(const unsigned*)&codes[1][P::value_at(8 * c8 + 2 * h + z, s8)];
                    scale[z] = __uint_as_float((unsigned)scales[1][P::value_scale_at(8 * c8 + 2 * h + z, s8 / 4)] << 23);
                }
                auto two = [&](int e, unsigned lo, unsigned hi) {
                    y[2 * e][h] = (lo & 0xFFFFu) | hi << 16;
                    y[2 * e + 1][h] = lo >> 16 | (hi & 0xFFFF0000u);
                };
                two(0, __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale[0], 0)),
                    __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[1], scale[1], 0)));
                two(1, __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale[0], 1)),
                    __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[1], scale[1], 1)));
                two(2, __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale[0], 2)),
                    __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[1], scale[1], 2)));
                two(3, __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[0], scale[0], 3)),
                    __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[1], scale[1], 3)));
            }
#pragma unroll
            for (int e = 0; e < 8; e++) put(vo, 8 * s8 + e, c8, vs == vs ? y[e] : none);
        }
        return;
    }
    // the unfinished block's tokens as they were given; zeros behind the end, and where there is no page
    const bool tail = live > 0 && live < BT;
    const uint16_t *kt = (const uint16_t*)a.t.kt + (size_t)bg * BT * D, *vt = (const uint16_t*)a.t.vt + (size_t)bg * BT * D;
    for (int x = tid; x < BT * C8; x += 256) {
        const int s = x / C8, c8 = x % C8;
        if (!out_row(s)) continue;
        u32x4 y = {0, 0, 0, 0}, z = {0, 0, 0, 0};
        if (tail && s < live) {
            y = *(const u32x4*)(kt + s * D + 8 * c8);
#pragma unroll
            for (int e = 0; e < 4; e++) z[e] = (unsigned)vt[(8 * c8 + 2 * e) * BT + s] | (unsigned)vt[(8 * c8 + 2 * e + 1) * BT + s] << 16;
        }
        put(ko, s, c8, y);
        put(vo, s, c8, z);
    }
}

int launch_cache4_read(const sparsek_cache8_cfg& c, const sparsek_cache4& t, const int32_t* lens, int begin, int n, void* k, void* v, hipStream_t st)
{
    const ReadArgs a = {t, c.Hkv, c.cap, c.pages, begin, n, lens, (uint16_t*)k, (uint16_t*)v};
    const dim3 grid((unsigned)((begin + n - 1) / BT - begin / BT + 1), c.B * c.Hkv);
    const bool stream = 4.0 * c.B * c.Hkv * n * c.d > 100e6;
#define READ(D, S) hipLaunchKernelGGL((cache4_read_kernel<D, S>), grid, dim3(256), 0, st, a)
    if (c.d == 128) {
        if (stream) READ(128, true);
        else READ(128, false);
    } else {
        if (stream) READ(64, true);
        else READ(64, false);
    }
#undef READ
    return launch_status();
}

}  // namespace spk
