// Norms of queries and keys for each head, with the rotation by position in the same pass, forward and backward.
//
// Forward: y = x r w with r = 1 / sqrt(mean(x^2) + eps) (or y = x), then pair p of a head turns by a_p = pos[axis_p] freq_p:
//     (y1, y2) -> (y1 cos a - y2 sin a, y2 cos a + y1 sin a).
// Backward, of dout: g = the rotation by -a of dout, dw = sum over rows of x r g, dx = r (w g - x r^2 mean(x w g)).
//
// A row is one head of one token.  Its lanes have 8 channels each, four and the four that they turn with (pairs half a rotation apart), or
// four of either half (neighbours), so a pair never leaves a lane; a token's lanes go through the heads, and the angles, which depend on the
// token alone, are made once.  What bounds it is memory: a document of 32768, 32 + 8 heads of 128, is normed and turned in 135 us, at 5.0 TB/s
// (a copy of 1 GiB reaches 5.1), its vector instructions beside that for 43 % of the time; backward 4 x 8192 tokens of 32 heads take 170 us (4.7).
// In a call that is streamed every load and store takes whole lines: where a row's halves end inside one, its wave's lanes load what lies side by side
// and hand it over in LDS.
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
// frequency of 1 it is off by 2^-24 of a turn.  What its rounding to fp32 drops, up to 9e-8 radians where a cosine's own rounding is 3e-8, is added
// with the derivatives.
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
        const double t = 2.0 * (turns - rint(turns));
        const float hi = (float)t, lo = 3.14159265f * (float)(t - (double)hi);
        float s, c;
        sincospif(hi, &s, &c);
        co[e] = fmaf(-lo, s, c);
        si[e] = fmaf(lo, c, s);
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

// Rows of a token that are on their way together.  Four where much is streamed in bf16 (a document of 32768, 32 + 8 heads of 128: 132 us, one
// at a time 139; training on video, 4 x 8192 tokens of 16 + 16 heads, 280 and 305); one where the caches have it (training on 4 x 1250 of those tokens 53.9 us,
// four 59.7; on 4 x 500 29 and 31; forward two prompts of 5003, 16 + 2 heads, 17.3 and 17.8, but a document of 5000 24.0 and 22.1) and in fp32, whose rows are
// twice as long (a training pass of 4 x 2000, 24 heads of 64, its backward streamed: 50 us, four 62.5).
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

// Where a lane loads and stores: two pieces of W channels.  They are those that it turns, a and b; or, LINES, those that stand at its place
// among all of its wave's, token after token, and change hands in LDS, so that whole lines come and go where a's and b's are less.
struct Piece {
    unsigned b, t;
    int ch;
    bool live;
};
template <int LPR, bool LINES>
struct Pieces {
    Piece at[2];
    int a, b;   // LINES: where those that it turns lie among the wave's
    __device__ __forceinline__ Pieces(const RopeArgs& p, const Chunk& ch, unsigned token, unsigned all)
    {
        const int lane = threadIdx.x % 64, c = lane % LPR;
        if constexpr (LINES) {
            const int row = p.d / W, first = lane / LPR * row;
            a = first + ch.a / W;
            b = first + ch.b / W;
#pragma unroll
            for (int x = 0; x < 2; x++) {
                const int m = lane + 64 * x, of = m / row;
                const unsigned tk = token - lane / LPR + of;
                at[x].live = of < 64 / LPR && tk < all;
                at[x].ch = W * (m - of * row);
                at[x].b = at[x].live ? tk / p.n : 0;
                at[x].t = at[x].live ? tk - at[x].b * p.n : 0;
            }
        } else {
            at[0].live = token < all && 2 * W * c < p.d;
            at[0].b = at[0].live ? token / p.n : 0;
            at[0].t = at[0].live ? token - at[0].b * p.n : 0;
            at[1] = at[0];
            at[0].ch = ch.a;
            at[1].ch = ch.b;
        }
    }
    // From the pieces that were loaded to those that are turned, ROWS heads at once, and back (mine: the lane has some to turn).
    template <int ROWS, class Raw>
    __device__ __forceinline__ void take(Raw (*lds)[128], Raw (&x)[ROWS], Raw (&y)[ROWS]) const
    {
        if constexpr (LINES) {
            const int lane = threadIdx.x % 64;
            wave_lds_order();
#pragma unroll
            for (int u = 0; u < ROWS; u++) {
                lds[u][lane] = x[u];
                lds[u][lane + 64] = y[u];
            }
            wave_lds_order();
#pragma unroll
            for (int u = 0; u < ROWS; u++) {
                x[u] = lds[u][a];
                y[u] = lds[u][b];
            }
        }
    }
    template <int ROWS, class Raw>
    __device__ __forceinline__ void give(Raw (*lds)[128], bool mine, Raw (&x)[ROWS], Raw (&y)[ROWS]) const
    {
        if constexpr (LINES) {
            const int lane = threadIdx.x % 64;
            wave_lds_order();
            if (mine)
#pragma unroll
                for (int u = 0; u < ROWS; u++) {
                    lds[u][a] = x[u];
                    lds[u][b] = y[u];
                }
            wave_lds_order();
#pragma unroll
            for (int u = 0; u < ROWS; u++) {
                x[u] = lds[u][lane];
                y[u] = lds[u][lane + 64];
            }
        }
    }
};

template <class T, int LPR, bool STREAM, bool LINES>
__global__ __launch_bounds__(256) void rope_fwd_kernel(RopeArgs p)
{
    typedef typename Some<T>::Raw Raw;
    constexpr int TOK = 256 / LPR, ROWS = rows_at_once<T, STREAM>();
    __shared__ Raw pieces[LINES ? 4 * ROWS : 1][128];
    Raw(*lds)[128] = &pieces[LINES ? threadIdx.x / 64 * ROWS : 0];
    const int c = threadIdx.x % LPR;
    const unsigned token = blockIdx.x * TOK + threadIdx.x / LPR, all = (unsigned)p.B * p.n;   // (at most 2^26)
    const bool mine = 2 * W * c < p.d, live = token < all && mine;
    const Chunk ch = chunk_of(p, mine ? c : 0);
    float co[W], si[W];
    angles(p, ch, live ? token : 0, co, si);
    const Pieces<LPR, LINES> at(p, ch, token, all);
    const int h0 = blockIdx.y * p.heads, h1 = min(h0 + p.heads, p.H + p.Hkv);
    auto part = [&](const T* x, const sparsek_rope_strides& step, T* out, int heads, const float* wts, int from, int to) {
        const T* xs[2];
        T* os[2];
#pragma unroll
        for (int y = 0; y < 2; y++) {
            xs[y] = x + at.at[y].b * step.batch + at.at[y].t * step.token + at.at[y].ch;
            os[y] = out + ((size_t)at.at[y].b * heads * p.n + at.at[y].t) * p.d + at.at[y].ch;
        }
        Weights w;
        w.load(wts, ch, live);
        for (int hr = from; hr < to; hr += ROWS) {
            Raw ra[ROWS], rb[ROWS];
#pragma unroll
            for (int u = 0; u < ROWS; u++) {   // (on their way together)
                const long long h = min(hr + u, to - 1) * step.head;
                ra[u] = load<STREAM, Raw>(xs[0] + h);
                rb[u] = load<STREAM, Raw>(xs[1] + h);
            }
            at.take(lds, ra, rb);
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
                ra[u] = Some<T>::narrow(xa);
                rb[u] = Some<T>::narrow(xb);
            }
            at.give(lds, mine, ra, rb);
#pragma unroll
            for (int u = 0; u < ROWS; u++) {
                const size_t o = (size_t)(hr + u) * p.n * p.d;
                if (at.at[0].live && hr + u < to) store<STREAM, Raw>(os[0] + o, ra[u]);
                if (at.at[1].live && hr + u < to) store<STREAM, Raw>(os[1] + o, rb[u]);
            }
        }
    };
    if (h0 < p.H) part((const T*)p.q, p.qs, (T*)p.qo, p.H, p.qw, h0, min(h1, p.H));
    if (h1 > p.H) part((const T*)p.k, p.ks, (T*)p.ko, p.Hkv, p.kw, max(h0 - p.H, 0), h1 - p.H);
}

// A workgroup takes `tiles` groups of tokens one after another and all of its heads, and leaves its part of the sums for the weights.
template <class T, int LPR, bool STREAM, bool LINES>
__global__ __launch_bounds__(256, 3) void rope_bwd_kernel(RopeArgs p)
{
    typedef typename Some<T>::Raw Raw;
    constexpr int TOK = 256 / LPR, ROWS = rows_at_once<T, STREAM>();
    __shared__ float sums[TOK][2 * W * LPR + 1];
    __shared__ Raw pieces[LINES ? 4 * ROWS : 1][128];
    Raw(*lds)[128] = &pieces[LINES ? threadIdx.x / 64 * ROWS : 0];
    const int c = threadIdx.x % LPR, row = threadIdx.x / LPR;
    const unsigned all = (unsigned)p.B * p.n;
    const int h0 = blockIdx.y * p.heads, h1 = min(h0 + p.heads, p.H + p.Hkv);
    const bool mine = 2 * W * c < p.d;
    const Chunk ch = chunk_of(p, mine ? c : 0);
    float wsum[2][2 * W];
#pragma unroll
    for (int e = 0; e < 2 * W; e++) wsum[0][e] = wsum[1][e] = 0.0f;
    for (int tile = 0; tile < p.tiles; tile++) {
        const unsigned token = (blockIdx.x * p.tiles + tile) * TOK + row;   // (at most 2^26 and a workgroup's share)
        const bool live = token < all && mine;
        float co[W], si[W];
        angles(p, ch, live ? token : 0, co, si);
        const Pieces<LPR, LINES> at(p, ch, token, all);
        auto part = [&](const T* x, const sparsek_rope_strides& step, const T* dout, T* dx, const sparsek_rope_strides& dstep, int heads, const float* wts,
                        float (&ws)[2 * W], int from, int to) {
            const T *xs[2], *gs[2];
            T* os[2];
#pragma unroll
            for (int y = 0; y < 2; y++) {
                const Piece& l = at.at[y];
                xs[y] = x + l.b * step.batch + l.t * step.token + l.ch;
                gs[y] = dout + ((size_t)l.b * heads * p.n + l.t) * p.d + l.ch;
                os[y] = dx + l.b * dstep.batch + l.t * dstep.token + l.ch;
            }
            const long long between = os[1] - os[0];
            Weights w;
            w.load(wts, ch, live);
            for (int hr = from; hr < to; hr += ROWS) {
                Raw rga[ROWS], rgb[ROWS], rxa[ROWS], rxb[ROWS];
#pragma unroll
                for (int u = 0; u < ROWS; u++) {   // (on their way together)
                    const int h = min(hr + u, to - 1);
                    const size_t g = (size_t)h * p.n * p.d;
                    rga[u] = load<STREAM, Raw>(gs[0] + g);
                    rgb[u] = load<STREAM, Raw>(gs[1] + g);
                    if (p.norm) {
                        rxa[u] = load<STREAM, Raw>(xs[0] + h * step.head);
                        rxb[u] = load<STREAM, Raw>(xs[1] + h * step.head);
                    }
                }
                auto put = [&](int u) {
                    T* o = os[0] + (hr + u) * dstep.head;
                    if (at.at[0].live && hr + u < to) store<STREAM, Raw>(o, rga[u]);
                    if (at.at[1].live && hr + u < to) store<STREAM, Raw>(o + between, rgb[u]);
                };
                at.take(lds, rga, rgb);
                if (p.norm) at.take(lds, rxa, rxb);
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
                    rga[u] = Some<T>::narrow(ga);
                    rgb[u] = Some<T>::narrow(gb);
                    if (!LINES) put(u);
                }
                if (LINES) {
                    at.give(lds, mine, rga, rgb);
#pragma unroll
                    for (int u = 0; u < ROWS; u++) put(u);
                }
            }
        };
        if (h0 < p.H)
            part((const T*)p.q, p.qs, (const T*)p.dqo, (T*)p.dq, p.dqs, p.H, p.qw, wsum[0], h0, min(h1, p.H));
        if (h1 > p.H)
            part((const T*)p.k, p.ks, (const T*)p.dko, (T*)p.dk, p.dks, p.Hkv, p.kw, wsum[1], max(h0 - p.H, 0), h1 - p.H);
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
// Whether a call that reads or writes every value `passes` times goes past the last cache, of 256 MB.  Forward, streamed and not: a document of
// 32768, 671 MB, 135 and 149 us; of 9500, 195 MB, 43 and 52; of 8192, 168 MB, 35 and 39; 16 x 2000 tokens in fp32, 393 MB, 75 and 81; 8000 tokens of
// 32 heads of 128, 131 MB, with their backward, which finds less in the cache then, 80 and 77; 5003 of 64 heads of 64, 82 MB, 21.5 and 16.6.
// Backward, behind a forward that was not: 4 x 2000 in fp32, 147 MB, 50 and 55; 5500 tokens of 32 heads, 135 MB, 55 and 59; 5000, 123 MB, 54 and 51.
static bool rope_streams(const sparsek_rope_cfg& c, int passes)
{
    return (double)passes * c.B * c.n * (c.H + c.Hkv) * c.d * (c.dtype == SPARSEK_BF16 ? 2 : 4) > (passes == 3 ? 130e6 : 150e6);
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

// Whether what a row's lanes load and store at once ends inside a line of 128 bytes, in a call that is streamed: then LINES (without, every line
// goes twice: 22592 tokens, 64 heads of 64, forward 79 us, 96 otherwise, with the backward 213 and 236; 32 heads of 128 of which 64 turn 77 and 95, 203 and
// 229; 36 heads of 112 of which 96 turn 83 and 116, 222 and 290; whole lines anyway, 32 heads of 128: 77.5 and 76.5, 203 and 200).  Through the caches
// LDS costs more than it brings: two prompts of 5003, 18.4 us and 17.2.
static bool part_lines(const sparsek_rope_cfg& c)
{
    const int size = c.dtype == SPARSEK_BF16 ? 2 : 4;
    return c.interleaved ? c.d / 2 * size % 128 : c.rot / 2 * size % 128 || (c.d - c.rot) / 2 * size % 128;
}

#define BY_CACHES(T, lpr, c, stream, LAUNCH)           \
    if (!stream) { LAUNCH(T, lpr, false, false); }      \
    else if (part_lines(c)) { LAUNCH(T, lpr, true, true); } \
    else { LAUNCH(T, lpr, true, false); }
#define BY_LANES(T, lpr, c, stream, LAUNCH)                    \
    if (lpr == 1) { BY_CACHES(T, 1, c, stream, LAUNCH) }        \
    else if (lpr == 2) { BY_CACHES(T, 2, c, stream, LAUNCH) }   \
    else if (lpr == 4) { BY_CACHES(T, 4, c, stream, LAUNCH) }   \
    else if (lpr == 8) { BY_CACHES(T, 8, c, stream, LAUNCH) }   \
    else if (lpr == 16) { BY_CACHES(T, 16, c, stream, LAUNCH) } \
    else { BY_CACHES(T, 32, c, stream, LAUNCH) }
#define BY_ROW(c, lpr, stream, LAUNCH)                                        \
    if (c.dtype == SPARSEK_F32) { BY_LANES(float, lpr, c, stream, LAUNCH) }   \
    else { BY_LANES(uint16_t, lpr, c, stream, LAUNCH) }

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
#define FWD(T, L, S, N) hipLaunchKernelGGL((rope_fwd_kernel<T, L, S, N>), grid, dim3(256), 0, st, a)
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
#define BWD(T, L, S, N) hipLaunchKernelGGL((rope_bwd_kernel<T, L, S, N>), dim3(y.gx, y.gy), dim3(256), 0, st, a)
    BY_ROW(c, y.s.lpr, stream, BWD)
#undef BWD
    if (a.part) hipLaunchKernelGGL(rope_weights_kernel, dim3(2 * c.d / COLS), dim3(1024), 0, st, a.part, (int)(y.gx * y.gy), c.d, dqw, dkw);
    return launch_status();
}

}  // namespace spk
