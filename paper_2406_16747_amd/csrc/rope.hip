// Norms of queries and keys for each head, with the rotation by position in the same pass, forward and backward.
//
// Forward: y = x r w with r = 1 / sqrt(mean(x^2) + eps) (or y = x), then pair p of a head turns by a_p = pos[axis_p] freq_p:
//     (y1, y2) -> (y1 cos a - y2 sin a, y2 cos a + y1 sin a).
// Backward, of dout: g = the rotation by -a of dout, dw = sum over rows of x r g, dx = r (w g - x r^2 mean(x w g)).
//
// A row is one head of one token.  Its lanes have 8 channels each, four and the four that they turn with (pairs half a rotation apart), or
// four of either half (neighbours), so a pair never leaves a lane; a token's lanes go through the heads, and the angles, which depend on the
// token alone, are made once.  What bounds it is memory: a document of 32768, 32 + 8 heads of 128, is normed and turned in 136 us, at 4.9 TB/s
// (a copy of 1 GiB reaches 5.1), its vector instructions beside that for 60 % of the time; backward 4 x 8192 tokens of 32 heads take 170 us (4.7).
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

constexpr int W = 4;   // channels of a lane in either half (eight bf16 values, 16 bytes to a load, are no faster)

// W values of storage type T, as they lie and in fp32.
template <class T>
struct Some;
template <>
struct Some<uint16_t> {
    typedef u32x2 Raw;
    static __device__ __forceinline__ void widen(Raw w, float (&x)[W])
    {
#pragma unroll
        for (int e = 0; e < W; e++) x[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
    }
    static __device__ __forceinline__ Raw narrow(const float (&x)[W])
    {
        typedef __bf16 Four __attribute__((ext_vector_type(4)));   // (to the nearest, even on ties, two to an instruction)
        return __builtin_bit_cast(Raw, Four{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]});
    }
};
template <>
struct Some<float> {
    typedef u32x4 Raw;
    static __device__ __forceinline__ void widen(Raw w, float (&x)[W])
    {
#pragma unroll
        for (int e = 0; e < W; e++) x[e] = __uint_as_float(w[e]);
    }
    static __device__ __forceinline__ Raw narrow(const float (&x)[W])
    {
        return Raw{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
};
// What a call reads and writes goes past the chip's caches where it is more than the last of them holds.
template <bool STREAM, class Raw>
__device__ __forceinline__ Raw load(const void* p)
{
    if constexpr (STREAM) return __builtin_nontemporal_load((const Raw*)p);
    else return *(const Raw*)p;
}
template <bool STREAM, class Raw>
__device__ __forceinline__ void store(void* p, Raw x)
{
    if constexpr (STREAM) __builtin_nontemporal_store(x, (Raw*)p);
    else *(Raw*)p = x;
}

// The sum over LPR neighbouring lanes.
template <int LPR>
__device__ __forceinline__ float row_sum(float x)
{
    if constexpr (LPR > 1) x += dpp_f32(x, 0);
    if constexpr (LPR > 2) x += dpp_f32(x, 1);
    if constexpr (LPR > 4) x += dpp_f32(x, 2);
    if constexpr (LPR > 8) x += dpp_f32(x, 3);
    if constexpr (LPR > 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return x;
}

// Which channels a lane has: W from a, W from b, and which of the angles turn them.  A row's lanes have neighbouring ones, so each load or
// store of a row is one of whole lines (eight neighbours of fp32 in two loads to a lane: 82 us instead of 60, 16 x 2000 tokens forward).
struct Chunk {
    int a, b, pa, pb;   // the first pair of a's and of b's channels (not interleaved: of both), -1: they do not turn
};
__device__ __forceinline__ Chunk chunk_of(const RopeArgs& p, int c)
{
    if (p.interleaved) {
        const int a = W * c, b = p.d / 2 + W * c;
        return Chunk{a, b, a < p.rot ? a / 2 : -1, b < p.rot ? b / 2 : -1};
    }
    if (2 * W * c < p.rot) return Chunk{W * c, p.rot / 2 + W * c, W * c, W * c};
    const int a = p.rot / 2 + W * c;   // (rot + W (c - rot / 2W))
    return Chunk{a, a + (p.d - p.rot) / 2, -1, -1};
}

// cos and sin of the lane's W pairs.  The angle in turns, pos freq / (2 pi), is made and reduced in 64 bits: at position 2^31 and a
// frequency of 1 it is off by 2^-24 of a turn.
__device__ __forceinline__ void angles(const RopeArgs& p, const Chunk& ch, unsigned token, float (&co)[W], float (&si)[W])
{
#pragma unroll
    for (int e = 0; e < W; e++) {
        const bool second = p.interleaved && e >= W / 2;
        const int first = second ? ch.pb : ch.pa;
        co[e] = 1.0f;
        si[e] = 0.0f;
        if (first < 0) continue;
        const int x = first + e - (second ? W / 2 : 0), ax = p.axis ? min(max(p.axis[x], 0), p.axes - 1) : 0;
        const double turns = (double)p.pos[(size_t)ax * p.B * p.n + token] * ((double)p.freq[x] * 0.15915494309189533577);
        const float t = (float)(turns - rint(turns));
        sincospif(2.0f * t, &si[e], &co[e]);
    }
}

// The W pairs of a lane turn (back: the other way).
__device__ __forceinline__ void turn(bool interleaved, bool back, const Chunk& ch, const float (&co)[W], const float (&si)[W], float (&a)[W], float (&b)[W])
{
    auto one = [&](float& x, float& y, float c, float s) {
        s = back ? -s : s;
        const float z = x * c - y * s;
        y = y * c + x * s;
        x = z;
    };
    if (interleaved) {
        if (ch.pa >= 0)
#pragma unroll
            for (int e = 0; e < W / 2; e++) one(a[2 * e], a[2 * e + 1], co[e], si[e]);
        if (ch.pb >= 0)
#pragma unroll
            for (int e = 0; e < W / 2; e++) one(b[2 * e], b[2 * e + 1], co[W / 2 + e], si[W / 2 + e]);
    } else if (ch.pa >= 0) {
#pragma unroll
        for (int e = 0; e < W; e++) one(a[e], b[e], co[e], si[e]);
    }
}

// Rows of a token that are on their way together.  Four where much is streamed in bf16 (a document of 32768, 32 + 8 heads of 128: 136 us, one
// at a time 138; training on video, 4 x 8192 tokens, 286 and 303); one where the caches have it (a document of 8192 38.5 us, four 41.4) and in fp32,
// whose rows are twice as long (a training pass of 4 x 2000, 24 heads of 64: 57 us, four 70; of 16 x 2000 198 and 199).
template <class T, bool STREAM>
constexpr int rows_at_once() { return STREAM && sizeof(T) == 2 ? 4 : 1; }

struct Weights {
    float a[W], b[W];
    __device__ __forceinline__ void load(const float* w, const Chunk& ch, bool live)
    {
#pragma unroll
        for (int e = 0; e < W; e++) {
            a[e] = w && live ? w[ch.a + e] : 1.0f;
            b[e] = w && live ? w[ch.b + e] : 1.0f;
        }
    }
};

template <class T, int LPR, bool STREAM>
__global__ __launch_bounds__(256) void rope_fwd_kernel(RopeArgs p)
{
    constexpr int TOK = 256 / LPR, ROWS = rows_at_once<T, STREAM>();
    const int c = threadIdx.x % LPR;
    const unsigned token = blockIdx.x * TOK + threadIdx.x / LPR, all = (unsigned)p.B * p.n;   // (at most 2^26)
    const bool live = token < all && 2 * W * c < p.d;
    const Chunk ch = chunk_of(p, live ? c : 0);
    const unsigned at = live ? token : 0, b = at / p.n, t = at - b * p.n;
    float co[W], si[W];
    angles(p, ch, at, co, si);
    const int h0 = blockIdx.y * p.heads, h1 = min(h0 + p.heads, p.H + p.Hkv);
    auto part = [&](const T* x, long long step, T* out, const float* wts, int from, int to) {   // x, out: of head 0
        typedef typename Some<T>::Raw Raw;
        Weights w;
        w.load(wts, ch, live);
        for (int hr = from; hr < to; hr += ROWS) {
            Raw ra[ROWS], rb[ROWS];
#pragma unroll
            for (int u = 0; u < ROWS; u++) {   // (on their way together)
                const T* row = x + min(hr + u, to - 1) * step;
                ra[u] = load<STREAM, Raw>(row + ch.a);
                rb[u] = load<STREAM, Raw>(row + ch.b);
            }
#pragma unroll
            for (int u = 0; u < ROWS; u++) {
                float xa[W], xb[W];
                Some<T>::widen(ra[u], xa);
                Some<T>::widen(rb[u], xb);
                if (p.norm) {
                    float s = 0.0f;
#pragma unroll
                    for (int e = 0; e < W; e++) s = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], s));
                    const float r = rsqrtf(row_sum<LPR>(live ? s : 0.0f) * p.inv_d + p.eps);
#pragma unroll
                    for (int e = 0; e < W; e++) {
                        xa[e] *= r * w.a[e];
                        xb[e] *= r * w.b[e];
                    }
                }
                turn(p.interleaved, false, ch, co, si, xa, xb);
                if (live && hr + u < to) {
                    T* o = out + (size_t)(hr + u) * p.n * p.d;
                    store<STREAM, Raw>(o + ch.a, Some<T>::narrow(xa));
                    store<STREAM, Raw>(o + ch.b, Some<T>::narrow(xb));
                }
            }
        }
    };
    if (h0 < p.H) part((const T*)p.q + b * p.qs.batch + t * p.qs.token, p.qs.head, (T*)p.qo + ((size_t)b * p.H * p.n + t) * p.d, p.qw, h0, min(h1, p.H));
    if (h1 > p.H) part((const T*)p.k + b * p.ks.batch + t * p.ks.token, p.ks.head, (T*)p.ko + ((size_t)b * p.Hkv * p.n + t) * p.d, p.kw, max(h0 - p.H, 0), h1 - p.H);
}

// A workgroup takes `tiles` groups of tokens one after another and all of its heads, and leaves its part of the sums for the weights.
template <class T, int LPR, bool STREAM>
__global__ __launch_bounds__(256, 3) void rope_bwd_kernel(RopeArgs p)
{
    constexpr int TOK = 256 / LPR, ROWS = rows_at_once<T, STREAM>();
    __shared__ float sums[TOK][2 * W * LPR + 1];
    const int c = threadIdx.x % LPR, row = threadIdx.x / LPR;
    const unsigned all = (unsigned)p.B * p.n;
    const int h0 = blockIdx.y * p.heads, h1 = min(h0 + p.heads, p.H + p.Hkv);
    const Chunk ch = chunk_of(p, 2 * W * c < p.d ? c : 0);
    float wsum[2][2 * W];
#pragma unroll
    for (int e = 0; e < 2 * W; e++) wsum[0][e] = wsum[1][e] = 0.0f;
    for (int tile = 0; tile < p.tiles; tile++) {
        const unsigned token = (blockIdx.x * p.tiles + tile) * TOK + row;   // (at most 2^26 and a workgroup's share)
        const bool live = token < all && 2 * W * c < p.d;
        const unsigned at = live ? token : 0, b = at / p.n, t = at - b * p.n;
        float co[W], si[W];
        angles(p, ch, at, co, si);
        auto part = [&](const T* x, long long step, const T* dout, T* dx, long long dstep, const float* wts, float (&ws)[2 * W], int from, int to) {
            typedef typename Some<T>::Raw Raw;
            Weights w;
            w.load(wts, ch, live);
            for (int hr = from; hr < to; hr += ROWS) {
                Raw rga[ROWS], rgb[ROWS], rxa[ROWS], rxb[ROWS];
#pragma unroll
                for (int u = 0; u < ROWS; u++) {   // (on their way together)
                    const int h = min(hr + u, to - 1);
                    const T *g = dout + (size_t)h * p.n * p.d, *row = x + h * step;
                    rga[u] = load<STREAM, Raw>(g + ch.a);
                    rgb[u] = load<STREAM, Raw>(g + ch.b);
                    if (p.norm) {
                        rxa[u] = load<STREAM, Raw>(row + ch.a);
                        rxb[u] = load<STREAM, Raw>(row + ch.b);
                    }
                }
#pragma unroll
                for (int u = 0; u < ROWS; u++) {
                    const bool real = live && hr + u < to;
                    float ga[W], gb[W];
                    Some<T>::widen(rga[u], ga);
                    Some<T>::widen(rgb[u], gb);
                    turn(p.interleaved, true, ch, co, si, ga, gb);
                    if (p.norm) {
                        float xa[W], xb[W], s = 0.0f, m = 0.0f;
                        Some<T>::widen(rxa[u], xa);
                        Some<T>::widen(rxb[u], xb);
#pragma unroll
                        for (int e = 0; e < W; e++) {
                            s = fmaf(xa[e], xa[e], fmaf(xb[e], xb[e], s));
                            m = fmaf(xa[e] * w.a[e], ga[e], fmaf(xb[e] * w.b[e], gb[e], m));
                        }
                        const float r = rsqrtf(row_sum<LPR>(live ? s : 0.0f) * p.inv_d + p.eps);
                        const float f = r * r * (row_sum<LPR>(live ? m : 0.0f) * p.inv_d);
#pragma unroll
                        for (int e = 0; e < W; e++) {
                            ws[e] += real ? xa[e] * r * ga[e] : 0.0f;
                            ws[W + e] += real ? xb[e] * r * gb[e] : 0.0f;
                            ga[e] = r * (w.a[e] * ga[e] - xa[e] * f);
                            gb[e] = r * (w.b[e] * gb[e] - xb[e] * f);
                        }
                    }
                    if (real) {
                        T* o = dx + (hr + u) * dstep;
                        store<STREAM, Raw>(o + ch.a, Some<T>::narrow(ga));
                        store<STREAM, Raw>(o + ch.b, Some<T>::narrow(gb));
                    }
                }
            }
        };
        if (h0 < p.H)
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
        if (2 * W * c < p.d)
#pragma unroll
            for (int e = 0; e < W; e++) {
                sums[row][ch.a + e] = wsum[w][e];
                sums[row][ch.b + e] = wsum[w][W + e];
            }
        __syncthreads();
        for (int x = threadIdx.x; x < p.d; x += 256) {
            double y = 0;   // (in fp32 the weights' gradients of 8000 tokens are 1.8e-7 of their scale off, so 0.7e-7)
            for (int r = 0; r < TOK; r++) y += (double)sums[r][x];
            out[w * p.d + x] = (float)y;
        }
    }
}

// The workgroups' parts are added up in 64 bits, in an order of their own: COLS columns of dqw and dkw to a workgroup.
constexpr int COLS = 4;
__global__ __launch_bounds__(1024) void rope_weights_kernel(const float* __restrict__ part, int parts, int d, float* __restrict__ dqw, float* __restrict__ dkw)
{
    constexpr int ROWS = 1024 / COLS;
    __shared__ double sums[ROWS][COLS + 1];
    const int row = threadIdx.x / COLS, col = threadIdx.x % COLS, x = blockIdx.x * COLS + col;
    double y = 0;
#pragma unroll 8
    for (int r = row; r < parts; r += ROWS) y += (double)part[(size_t)r * 2 * d + x];
    sums[row][col] = y;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    y = 0;
#pragma unroll
    for (int r = 0; r < ROWS * COLS / 64; r++) y += sums[row + 64 / COLS * r][col];
#pragma unroll
    for (int z = COLS; z < 64; z *= 2) y += __shfl_xor(y, z, 64);
    float* out = x < d ? dqw : dkw;
    if (row == 0 && out) out[x % d] = (float)y;
}

// ---- launches ----

struct RopeShape {
    int lpr, tok;        // lanes of a row, tokens of a workgroup
    long long groups;    // of tokens
};
static RopeShape rope_shape(const sparsek_rope_cfg& c)
{
    RopeShape s;
    s.lpr = 1;
    while (2 * W * s.lpr < c.d) s.lpr *= 2;
    s.tok = 256 / s.lpr;
    s.groups = ((long long)c.B * c.n + s.tok - 1) / s.tok;
    return s;
}
// Whether a call that reads or writes every value `passes` times goes past the last cache, of 256 MB (streamed and not: a document of 32768, 671 MB,
// 136 and 149 us; of 12000, 246 MB, 51.6 and 58.4; of 8192, 168 MB, 37.7 and 38.5; two prompts of 5003, 92 MB, 28 and 17; forward of 16 x 2000 tokens
// in fp32, 393 MB, 75 and 81; of 4 x 2000, 98 MB, 20.6 and 19.3).
static bool rope_streams(const sparsek_rope_cfg& c, int passes)
{
    return (double)passes * c.B * c.n * (c.H + c.Hkv) * c.d * (c.dtype == SPARSEK_BF16 ? 2 : 4) > 200e6;
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

#define BY_LANES(T, lpr, stream, LAUNCH)                                                      \
    if (lpr == 1) { if (stream) { LAUNCH(T, 1, true); } else { LAUNCH(T, 1, false); } }        \
    else if (lpr == 2) { if (stream) { LAUNCH(T, 2, true); } else { LAUNCH(T, 2, false); } }   \
    else if (lpr == 4) { if (stream) { LAUNCH(T, 4, true); } else { LAUNCH(T, 4, false); } }   \
    else if (lpr == 8) { if (stream) { LAUNCH(T, 8, true); } else { LAUNCH(T, 8, false); } }   \
    else if (lpr == 16) { if (stream) { LAUNCH(T, 16, true); } else { LAUNCH(T, 16, false); } } \
    else { if (stream) { LAUNCH(T, 32, true); } else { LAUNCH(T, 32, false); } }
#define BY_ROW(c, lpr, stream, LAUNCH)                                     \
    if (c.dtype == SPARSEK_F32) { BY_LANES(float, lpr, stream, LAUNCH) }   \
    else { BY_LANES(uint16_t, lpr, stream, LAUNCH) }

// Workgroups that share a token's heads: as many as leave 1024 in all (training on 4 x 500 tokens, 16 + 16 heads of 128: 30.4 us, with 512 28.4, with
// 2048 39.1; on 4 x 2000: 79, 91 and 87; each share makes the angles anew).
static int head_shares(long long groups, int heads) { return (int)std::max<long long>(1, std::min<long long>(heads, 1024 / std::max<long long>(groups, 1))); }

int launch_rope_fwd(const sparsek_rope_cfg& c, const void* q, const void* k, const int32_t* pos, const float* freq, const int32_t* axis,
                    const float* qw, const float* kw, void* qo, void* ko, hipStream_t st)
{
    const RopeShape s = rope_shape(c);
    RopeArgs a = rope_args(c, q, k, pos, freq, axis, qw, kw);
    a.qo = qo; a.ko = ko;
    const int heads = c.H + c.Hkv, shares = head_shares(s.groups, heads);
    a.heads = (heads + shares - 1) / shares;
    const dim3 grid((unsigned)s.groups, (heads + a.heads - 1) / a.heads);
    const bool stream = rope_streams(c, 2);
#define FWD(T, L, S) hipLaunchKernelGGL((rope_fwd_kernel<T, L, S>), grid, dim3(256), 0, st, a)
    BY_ROW(c, s.lpr, stream, FWD)
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
    const bool stream = rope_streams(c, c.norm ? 3 : 2);
#define BWD(T, L, S) hipLaunchKernelGGL((rope_bwd_kernel<T, L, S>), dim3(y.gx, y.gy), dim3(256), 0, st, a)
    BY_ROW(c, y.s.lpr, stream, BWD)
#undef BWD
    if (a.part) hipLaunchKernelGGL(rope_weights_kernel, dim3(2 * c.d / COLS), dim3(1024), 0, st, a.part, (int)(y.gx * y.gy), c.d, dqw, dkw);
    return launch_status();
}

}  // namespace spk
