// Norms of queries and keys for each head, with the rotation by position in the same pass, forward and backward.
//
// Forward: y = x r w with r = 1 / sqrt(mean(x^2) + eps) (or y = x), then pair p of a head turns by a_p = pos[axis_p] freq_p:
//     (y1, y2) -> (y1 cos a - y2 sin a, y2 cos a + y1 sin a).
// Backward, of dout: g = the rotation by -a of dout, dw = sum over rows of x r g, dx = r (w g - x r^2 mean(x w g)).
//
// A row is one head of one token.  Its lanes have 8 channels each, four and the four that they turn with (pairs half a rotation apart), or
// eight neighbours, so a pair never leaves a lane; a token's lanes go through the heads, and the angles, which depend on the token
// alone, are made once.
#include "block_parts.hpp"

namespace spk {

struct RopeArgs {
    int B, H, Hkv, n, d, rot, axes, interleaved, norm;
    float eps, inv_d;
    sparsek_rope_strides qs, ks, dqs, dks;
    const void *q, *k, *dqo, *dko;
    void *qo, *ko, *dq, *dk;
    const int32_t *pos, *axis;
    const float *freq, *qw, *kw;
    float* part;     // [workgroups][2][d]: sums for dqw and dkw
    int heads;       // of a workgroup's share
    int tiles;       // of a workgroup's tokens
};

template <class T>
struct Four {   // 4 values of storage type T
    static __device__ __forceinline__ void load(const T* p, float (&x)[4]);
    static __device__ __forceinline__ void store(T* p, const float (&x)[4]);
};
template <>
struct Four<uint16_t> {
    static __device__ __forceinline__ void load(const uint16_t* p, float (&x)[4])
    {
        const u32x2 w = *(const u32x2*)p;
#pragma unroll
        for (int e = 0; e < 4; e++) x[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    }
    static __device__ __forceinline__ void store(uint16_t* p, const float (&x)[4])
    {
        u32x2 w;
#pragma unroll
        for (int e = 0; e < 2; e++) w[e] = (unsigned)f32_to_bf16(x[2 * e]) | (unsigned)f32_to_bf16(x[2 * e + 1]) << 16;
        *(u32x2*)p = w;
    }
};
template <>
struct Four<float> {
    static __device__ __forceinline__ void load(const float* p, float (&x)[4])
    {
        const u32x4 w = *(const u32x4*)p;
#pragma unroll
        for (int e = 0; e < 4; e++) x[e] = __uint_as_float(w[e]);
    }
    static __device__ __forceinline__ void store(float* p, const float (&x)[4])
    {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; e++) w[e] = __float_as_uint(x[e]);
        *(u32x4*)p = w;
    }
};

// The sum over LPR neighbouring lanes.
template <int LPR>
__device__ __forceinline__ float row_sum(float x)
{
    x += dpp_f32(x, 0);
    if constexpr (LPR > 2) x += dpp_f32(x, 1);
    if constexpr (LPR > 4) x += dpp_f32(x, 2);
    if constexpr (LPR > 8) x += dpp_f32(x, 3);
    if constexpr (LPR > 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return x;
}

// Which channels a lane has: four from a, four from b.
struct Chunk {
    int a, b, pair;   // pair: of a's first channel (interleaved: b's are two on), -1: they do not turn
};
__device__ __forceinline__ Chunk chunk_of(const RopeArgs& p, int c)
{
    if (8 * c >= p.rot) return Chunk{8 * c, 8 * c + 4, -1};
    if (p.interleaved) return Chunk{8 * c, 8 * c + 4, 4 * c};
    return Chunk{4 * c, p.rot / 2 + 4 * c, 4 * c};
}

// cos and sin of the lane's four pairs.  The angle in turns, pos freq / (2 pi), is made and reduced in 64 bits: at position 2^31 and a
// frequency of 1 it is off by 2^-24 of a turn.
__device__ __forceinline__ void angles(const RopeArgs& p, const Chunk& ch, unsigned token, float (&co)[4], float (&si)[4])
{
#pragma unroll
    for (int e = 0; e < 4; e++) {
        co[e] = 1.0f;
        si[e] = 0.0f;
    }
    if (ch.pair < 0) return;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const int x = ch.pair + e, ax = p.axis ? min(max(p.axis[x], 0), p.axes - 1) : 0;
        const double turns = (double)p.pos[(size_t)ax * p.B * p.n + token] * ((double)p.freq[x] * 0.15915494309189533577);
        const float t = (float)(turns - rint(turns));
        sincospif(2.0f * t, &si[e], &co[e]);
    }
}

// The four pairs of a lane turn (back: the other way).
__device__ __forceinline__ void turn(bool interleaved, bool back, const float (&co)[4], const float (&si)[4], float (&a)[4], float (&b)[4])
{
    auto one = [&](float& x, float& y, float c, float s) {
        s = back ? -s : s;
        const float z = x * c - y * s;
        y = y * c + x * s;
        x = z;
    };
    if (interleaved) {
        one(a[0], a[1], co[0], si[0]);
        one(a[2], a[3], co[1], si[1]);
        one(b[0], b[1], co[2], si[2]);
        one(b[2], b[3], co[3], si[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++) one(a[e], b[e], co[e], si[e]);
    }
}

struct Weights {
    float a[4], b[4];
    __device__ __forceinline__ void load(const float* w, const Chunk& ch, bool live)
    {
#pragma unroll
        for (int e = 0; e < 4; e++) {
            a[e] = w && live ? w[ch.a + e] : 1.0f;
            b[e] = w && live ? w[ch.b + e] : 1.0f;
        }
    }
};

template <class T, int LPR>
__global__ __launch_bounds__(256) void rope_fwd_kernel(RopeArgs p)
{
    constexpr int TOK = 256 / LPR;
    const int c = threadIdx.x % LPR;
    const unsigned token = blockIdx.x * TOK + threadIdx.x / LPR, all = (unsigned)p.B * p.n;   // (below 2^31)
    const bool live = token < all && 8 * c < p.d;
    const Chunk ch = chunk_of(p, live ? c : 0);
    const unsigned at = live ? token : 0, b = at / p.n, t = at - b * p.n;
    float co[4], si[4];
    angles(p, ch, at, co, si);
    const int h0 = blockIdx.y * p.heads, h1 = min(h0 + p.heads, p.H + p.Hkv);
    auto part = [&](const T* x, long long step, T* out, const float* wts, int from, int to) {   // x, out: of head 0
        Weights w;
        w.load(wts, ch, live);
        for (int h = from; h < to; h++) {
            float xa[4] = {0, 0, 0, 0}, xb[4] = {0, 0, 0, 0};
            if (live) {
                Four<T>::load(x + h * step + ch.a, xa);
                Four<T>::load(x + h * step + ch.b, xb);
            }
            if (p.norm) {
                float s = 0.0f;
#pragma unroll
                for (int e = 0; e < 4; e++) s = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], s));
                const float r = rsqrtf(row_sum<LPR>(s) * p.inv_d + p.eps);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    xa[e] *= r * w.a[e];
                    xb[e] *= r * w.b[e];
                }
            }
            if (ch.pair >= 0) turn(p.interleaved, false, co, si, xa, xb);
            if (live) {
                T* o = out + (long long)h * p.n * p.d;
                Four<T>::store(o + ch.a, xa);
                Four<T>::store(o + ch.b, xb);
            }
        }
    };
    part((const T*)p.q + b * p.qs.batch + t * p.qs.token, p.qs.head, (T*)p.qo + ((size_t)b * p.H * p.n + t) * p.d, p.qw, h0, min(h1, p.H));
    if (h1 > p.H) part((const T*)p.k + b * p.ks.batch + t * p.ks.token, p.ks.head, (T*)p.ko + ((size_t)b * p.Hkv * p.n + t) * p.d, p.kw, max(h0 - p.H, 0), h1 - p.H);
}

// A workgroup takes `tiles` groups of tokens one after another and all of its heads, and leaves its part of the sums for the weights.
template <class T, int LPR>
__global__ __launch_bounds__(256) void rope_bwd_kernel(RopeArgs p)
{
    constexpr int TOK = 256 / LPR;
    __shared__ float sums[TOK][8 * LPR + 1];
    const int c = threadIdx.x % LPR, row = threadIdx.x / LPR;
    const unsigned all = (unsigned)p.B * p.n;
    const int h0 = blockIdx.y * p.heads, h1 = min(h0 + p.heads, p.H + p.Hkv);
    const Chunk ch = chunk_of(p, 8 * c < p.d ? c : 0);
    float wsum[2][8];
#pragma unroll
    for (int e = 0; e < 8; e++) wsum[0][e] = wsum[1][e] = 0.0f;
    for (int tile = 0; tile < p.tiles; tile++) {
        const unsigned token = (blockIdx.x * p.tiles + tile) * TOK + row;   // (below 2^31 and a workgroup's share)
        const bool live = token < all && 8 * c < p.d;
        const unsigned at = live ? token : 0, b = at / p.n, t = at - b * p.n;
        float co[4], si[4];
        angles(p, ch, at, co, si);
        auto part = [&](const T* x, long long step, const T* dout, T* dx, long long dstep, const float* wts, float (&ws)[8], int from, int to) {
            Weights w;
            w.load(wts, ch, live);
            for (int h = from; h < to; h++) {
                float ga[4] = {0, 0, 0, 0}, gb[4] = {0, 0, 0, 0};
                if (live) {
                    const T* g = dout + (long long)h * p.n * p.d;
                    Four<T>::load(g + ch.a, ga);
                    Four<T>::load(g + ch.b, gb);
                }
                if (ch.pair >= 0) turn(p.interleaved, true, co, si, ga, gb);
                if (p.norm) {
                    float xa[4] = {0, 0, 0, 0}, xb[4] = {0, 0, 0, 0}, s = 0.0f, m = 0.0f;
                    if (live) {
                        Four<T>::load(x + h * step + ch.a, xa);
                        Four<T>::load(x + h * step + ch.b, xb);
                    }
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        s = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], s));
                        m = fmaf(xa[e] * w.a[e], ga[e], fmaf(xb[e] * w.b[e], gb[e], m));
                    }
                    const float r = rsqrtf(row_sum<LPR>(s) * p.inv_d + p.eps);
                    const float f = r * r * (row_sum<LPR>(m) * p.inv_d);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        ws[e] = fmaf(xa[e] * r, ga[e], ws[e]);
                        ws[4 + e] = fmaf(xb[e] * r, gb[e], ws[4 + e]);
                        ga[e] = r * (w.a[e] * ga[e] - xa[e] * f);
                        gb[e] = r * (w.b[e] * gb[e] - xb[e] * f);
                    }
                }
                if (live) {
                    Four<T>::store(dx + h * dstep + ch.a, ga);
                    Four<T>::store(dx + h * dstep + ch.b, gb);
                }
            }
        };
        part((const T*)p.q + b * p.qs.batch + t * p.qs.token, p.qs.head, (const T*)p.dqo + ((size_t)b * p.H * p.n + t) * p.d,
             (T*)p.dq + b * p.dqs.batch + t * p.dqs.token, p.dqs.head, p.qw, wsum[0], h0, min(h1, p.H));
        if (h1 > p.H)
            part((const T*)p.k + b * p.ks.batch + t * p.ks.token, p.ks.head, (const T*)p.dko + ((size_t)b * p.Hkv * p.n + t) * p.d,
                 (T*)p.dk + b * p.dks.batch + t * p.dks.token, p.dks.head, p.kw, wsum[1], max(h0 - p.H, 0), h1 - p.H);
    }
    if (!p.part) return;
    float* out = p.part + ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * p.d;
#pragma unroll
    for (int w = 0; w < 2; w++) {
        if (w) __syncthreads();
        if (8 * c < p.d)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                sums[row][ch.a + e] = wsum[w][e];
                sums[row][ch.b + e] = wsum[w][4 + e];
            }
        __syncthreads();
        for (int x = threadIdx.x; x < p.d; x += 256) {
            float y = 0.0f;
            for (int r = 0; r < TOK; r++) y += sums[r][x];
            out[w * p.d + x] = y;
        }
    }
}

// The workgroups' parts are added up in 64 bits, in an order of their own: 8 columns of dqw and dkw to a workgroup.
__global__ __launch_bounds__(256) void rope_weights_kernel(const float* __restrict__ part, int parts, int d, float* __restrict__ dqw, float* __restrict__ dkw)
{
    __shared__ double sums[32][8];
    const int row = threadIdx.x / 8, x = blockIdx.x * 8 + threadIdx.x % 8;
    double y = 0;
#pragma unroll 8
    for (int r = row; r < parts; r += 32) y += (double)part[(size_t)r * 2 * d + x];
    sums[row][threadIdx.x % 8] = y;
    __syncthreads();
    if (threadIdx.x >= 8) return;
    y = 0;
#pragma unroll
    for (int r = 0; r < 32; r++) y += sums[r][threadIdx.x];
    float* out = x < d ? dqw : dkw;
    if (out) out[x % d] = (float)y;
}

// ---- launches ----

struct RopeShape {
    int lpr, tok;        // lanes of a row, tokens of a workgroup
    long long groups;    // of tokens
};
static RopeShape rope_shape(const sparsek_rope_cfg& c)
{
    RopeShape s;
    s.lpr = 2;
    while (8 * s.lpr < c.d) s.lpr *= 2;
    s.tok = 256 / s.lpr;
    s.groups = ((long long)c.B * c.n + s.tok - 1) / s.tok;
    return s;
}
static RopeArgs rope_args(const sparsek_rope_cfg& c, const void* q, const void* k, const int32_t* pos, const float* freq, const int32_t* axis,
                          const float* qw, const float* kw)
{
    RopeArgs a = {};
    a.B = c.B; a.H = c.H; a.Hkv = c.Hkv; a.n = c.n; a.d = c.d; a.rot = c.rot; a.axes = c.axes;
    a.interleaved = c.interleaved; a.norm = c.norm;
    a.eps = c.eps; a.inv_d = 1.0f / (float)c.d;
    a.qs = c.q; a.ks = c.k; a.dqs = c.dq; a.dks = c.dk;
    a.q = q; a.k = k; a.pos = pos; a.freq = freq; a.axis = axis; a.qw = qw; a.kw = kw;
    return a;
}

#define BY_ROW(c, lpr, LAUNCH)                                       \
    if (c.dtype == SPARSEK_BF16) {                                   \
        if (lpr == 2) { LAUNCH(uint16_t, 2); }                       \
        else if (lpr == 4) { LAUNCH(uint16_t, 4); }                  \
        else if (lpr == 8) { LAUNCH(uint16_t, 8); }                  \
        else if (lpr == 16) { LAUNCH(uint16_t, 16); }                \
        else { LAUNCH(uint16_t, 32); }                               \
    } else {                                                         \
        if (lpr == 2) { LAUNCH(float, 2); }                          \
        else if (lpr == 4) { LAUNCH(float, 4); }                     \
        else if (lpr == 8) { LAUNCH(float, 8); }                     \
        else if (lpr == 16) { LAUNCH(float, 16); }                   \
        else { LAUNCH(float, 32); }                                  \
    }

// Workgroups that share a token's heads: as many as leave 2048 in all.
static int head_shares(long long groups, int heads) { return (int)std::max<long long>(1, std::min<long long>(heads, 2048 / std::max<long long>(groups, 1))); }

int launch_rope_fwd(const sparsek_rope_cfg& c, const void* q, const void* k, const int32_t* pos, const float* freq, const int32_t* axis,
                    const float* qw, const float* kw, void* qo, void* ko, hipStream_t st)
{
    const RopeShape s = rope_shape(c);
    RopeArgs a = rope_args(c, q, k, pos, freq, axis, qw, kw);
    a.qo = qo; a.ko = ko;
    const int heads = c.H + c.Hkv, shares = head_shares(s.groups, heads);
    a.heads = (heads + shares - 1) / shares;
    const dim3 grid((unsigned)s.groups, (heads + a.heads - 1) / a.heads);
#define FWD(T, L) hipLaunchKernelGGL((rope_fwd_kernel<T, L>), grid, dim3(256), 0, st, a)
    BY_ROW(c, s.lpr, FWD)
#undef FWD
    return launch_status();
}

struct RopeBwdShape {
    RopeShape s;
    int heads, tiles;
    unsigned gx, gy;
};
static RopeBwdShape rope_bwd_shape(const sparsek_rope_cfg& c)
{
    RopeBwdShape y;
    y.s = rope_shape(c);
    const int heads = c.H + c.Hkv, shares = head_shares(y.s.groups, heads);
    y.heads = (heads + shares - 1) / shares;
    y.gy = (heads + y.heads - 1) / y.heads;
    y.tiles = (int)((y.s.groups + 2047) / 2048);
    y.gx = (unsigned)((y.s.groups + y.tiles - 1) / y.tiles);
    return y;
}
size_t rope_bwd_ws_bytes(const sparsek_rope_cfg& c)
{
    const RopeBwdShape y = rope_bwd_shape(c);
    return c.norm ? align_up((size_t)y.gx * y.gy * 2 * c.d * 4, 256) : 256;
}

int launch_rope_bwd(const sparsek_rope_cfg& c, const void* q, const void* k, const int32_t* pos, const float* freq, const int32_t* axis,
                    const float* qw, const float* kw, const void* dqo, const void* dko, void* dq, void* dk, float* dqw, float* dkw, void* ws,
                    hipStream_t st)
{
    const RopeBwdShape y = rope_bwd_shape(c);
    RopeArgs a = rope_args(c, q, k, pos, freq, axis, qw, kw);
    a.dqo = dqo; a.dko = dko; a.dq = dq; a.dk = dk;
    a.heads = y.heads;
    a.tiles = y.tiles;
    a.part = dqw || dkw ? (float*)ws : nullptr;
#define BWD(T, L) hipLaunchKernelGGL((rope_bwd_kernel<T, L>), dim3(y.gx, y.gy), dim3(256), 0, st, a)
    BY_ROW(c, y.s.lpr, BWD)
#undef BWD
    if (a.part) hipLaunchKernelGGL(rope_weights_kernel, dim3(c.d / 4), dim3(256), 0, st, a.part, (int)(y.gx * y.gy), c.d, dqw, dkw);
    return launch_status();
}

}  // namespace spk
