// Norms of Q and K per head and their rotation by the token's (frame, height, width) position: forward, gradients, and both
// with the reorder (paper Sec. 4.1) and the block quantizer (Sec. 4.3 (1)) behind them.
//
// A row is the d channels of one token of one head.  d / 16 lanes share it, 16 channels each: eight from the front half of the
// row (8 L ..) and the eight that lie d / 2 behind them, so that both ways to pair channels find their pairs inside a lane.
// Row sums meet in two or three steps across neighbouring lanes (DPP); nothing goes through LDS.
//
// The angles' table separates by axis: some KB instead of some MB per layer, so it comes from the caches nearest to the compute
// unit.
//
// Sums and values are binary64 and rounded to binary32 once: the codes of the quantizing form then do not depend on the order of
// a sum (up to values within 2^-50 of a rounding border).
#include <math.h>
#include <string.h>

#include <algorithm>

#include "quantize_tile.h"

namespace paro {

constexpr int kThreads = 256;

// Channels turned by position: what the kernels need of a paro_rope_axes, its table and the grid.
struct Turning {
    const float2* table;
    int pairs[3];  // pairs per axis
    int base[3];   // first entry of an axis in the table
    int total;     // pairs that turn; pair p turns with the axis whose run of pairs holds it
    int n_img, Hg, Wg;
    double inv_hg, inv_wg;
    float sign;  // -1: turned back
    int halves;
};

// Norms: entry [tensor][text].
struct Norms {
    const float* w[2][2];
    const float* b[2][2];
    int kind;
    double eps;
};

template <typename T>
struct Rows {
    T* p;
    int64_t batch, head, token;
    __device__ T* row(int b, int h, int n) const { return p + b * batch + h * head + n * token; }
};

// floor(n / divisor) for 0 <= n < 2^24 and a divisor of at most that, inv = fl64(1 / divisor): (n + 1/2) inv lies 1 / (2 divisor)
// or more from the next integers, and is off by less than 2^-51 n / divisor.
__device__ inline int quotient_of(int n, double inv) { return (int)(((double)n + 0.5) * inv); }

// ---- the 16 channels of a lane -------------------------------------------------------------------------------------
// As loaded: 8 channels are 16 bytes of bf16 or 32 of binary32.
template <typename T>
struct LaneRow {
    static constexpr int Q = sizeof(T) / 2;  // 16-byte pieces per 8 channels
    uint4 q[2 * Q];
    template <int D>
    __device__ __forceinline__ void load(const T* row, int L) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < Q; ++i) q[half * Q + i] = ((const uint4*)(row + half * (D / 2) + 8 * L))[i];
    }
    __device__ __forceinline__ float operator[](int e) const {
        if constexpr (sizeof(T) == 2) {
            const uint4& v = q[e >> 3];
            const unsigned w = (e & 7) < 2 ? v.x : (e & 7) < 4 ? v.y : (e & 7) < 6 ? v.z : v.w;
            return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
        } else {
            const uint4& v = q[e >> 2];
            return __uint_as_float((e & 3) == 0 ? v.x : (e & 3) == 1 ? v.y : (e & 3) == 2 ? v.z : v.w);
        }
    }
};

typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ inline unsigned pack_bf16(float a, float b) { return __builtin_bit_cast(unsigned, __builtin_convertvector((float2v){a, b}, bf16x2)); }

template <int D>
__device__ __forceinline__ void store_lane(uint16_t* row, int L, const float (&y)[16]) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const float* v = y + 8 * half;
        *(uint4*)(row + half * (D / 2) + 8 * L) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
}
template <int D>
__device__ __forceinline__ void store_lane(float* row, int L, const float (&y)[16]) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float4* out = (float4*)(row + half * (D / 2) + 8 * L);
        const float* v = y + 8 * half;
        out[0] = make_float4(v[0], v[1], v[2], v[3]);
        out[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// A lane's channels of a float32 [d] vector, or `other` where there is none.
template <int D>
__device__ __forceinline__ void load_vector(const float* v, int L, float other, float (&x)[16]) {
    if (v) {
        LaneRow<float> r;
        r.load<D>(v, L);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = r[e];
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = other;
    }
}

// ---- row sums ------------------------------------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ int moved(int v) { return __builtin_amdgcn_mov_dpp(v, CTRL, 0xf, 0xf, true); }
template <int CTRL>
__device__ __forceinline__ double moved(double v) { return __hiloint2double(moved<CTRL>(__double2hiint(v)), moved<CTRL>(__double2loint(v))); }
template <int CTRL>
__device__ __forceinline__ float moved(float v) { return __int_as_float(moved<CTRL>(__float_as_int(v))); }
// Sum over the D / 16 neighbouring lanes of a row, in every one of them: the lane beside (quad_perm 1 0 3 2), the pair beside
// (2 3 0 1), the other four of eight (row_half_mirror).
template <int D, typename V>
__device__ __forceinline__ V row_sum(V v) {
    v += moved<0xB1>(v);
    v += moved<0x4E>(v);
    if constexpr (D == 128) v += moved<0x141>(v);
    return v;
}

// 1 / sqrt(v): the instruction's estimate and two Newton steps, y <- y + y (1/2 - v/2 y^2), which square its relative error.  The
// estimate stands where v is 0 or infinite.
__device__ __forceinline__ double rsqrt_of(double v) {
    const double y0 = __builtin_amdgcn_rsq(v);
    double y = y0;
#pragma unroll
    for (int i = 0; i < 2; ++i) y = fma(y, fma(-0.5 * v * y, y, 0.5), y);
    return v > 0.0 && v < __builtin_inf() ? y : y0;
}

// What a row is normalised by: value e becomes (x[e] - mean) r.
template <int D, typename T>
__device__ __forceinline__ void row_norm(const LaneRow<T>& x, int kind, double eps, double& mean, double& r) {
    mean = 0.0;
    if (kind == PARO_NORM_LAYER) {
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < 16; ++e) s += (double)x[e];
        mean = row_sum<D>(s) * (1.0 / D);
    }
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const double v = (double)x[e] - mean;
        s = fma(v, v, s);
    }
    r = rsqrt_of(fma(row_sum<D>(s), 1.0 / D, eps));
}

// ---- turning -------------------------------------------------------------------------------------------------------
// Pair e of a lane: channels (2e, 2e + 1) of its 16 (PARO_PAIRS_ADJACENT) or (e, 8 + e) (PARO_PAIRS_HALVES).  Pairs 0 .. 3 and 4 .. 7
// are four consecutive pairs of the row each.
struct LaneTurn {
    float c[8], s[8];
    unsigned turned;  // bit e: pair e turns
};

template <int D>
__device__ __forceinline__ LaneTurn load_turn(const Turning& t, int L, int f, int h, int w) {
    LaneTurn r;
    r.turned = 0;
    const int e0 = t.base[0] + f * t.pairs[0], e1 = t.base[1] + h * t.pairs[1] - t.pairs[0], e2 = t.base[2] + w * t.pairs[2] - t.pairs[0] - t.pairs[1];
    const int to1 = t.pairs[0], to2 = t.pairs[0] + t.pairs[1];
#pragma unroll
    for (int g = 0; g < 2; ++g) {
        const int p0 = t.halves ? 8 * L + 4 * g : g * (D / 4) + 4 * L;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = p0 + i, e = 4 * g + i;
            r.c[e] = 1.0f;
            r.s[e] = 0.0f;
            if (p < t.total) {
                const float2 v = t.table[(p < to1 ? e0 : p < to2 ? e1 : e2) + p];
                r.c[e] = v.x;
                r.s[e] = v.y * t.sign;
                r.turned |= 1u << e;
            }
        }
    }
    return r;
}

// One pair: values that do not turn stay as they are, whatever their partner holds.
template <typename V>
__device__ __forceinline__ void turn(V& x, V& y, float c, float s, bool turned) {
    const V a = fma(x, (V)c, -(y * (V)s)), b = fma(x, (V)s, y * (V)c);
    x = turned ? a : x;
    y = turned ? b : y;
}

template <typename V>
__device__ __forceinline__ void turn_lane(V (&u)[16], const LaneTurn& t, int halves) {
    if (halves) {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn(u[e], u[8 + e], t.c[e], t.s[e], t.turned >> e & 1);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn(u[2 * e], u[2 * e + 1], t.c[e], t.s[e], t.turned >> e & 1);
    }
}

// Grid coordinates of a token in default order; text tokens do not turn.
template <int D>
__device__ __forceinline__ LaneTurn turn_of_token(const Turning& t, int L, int n) {
    if (n >= t.n_img || t.total == 0) {
        LaneTurn r;
        r.turned = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) r.c[e] = 1.0f, r.s[e] = 0.0f;
        return r;
    }
    const int q = quotient_of(n, t.inv_wg), f = quotient_of(q, t.inv_hg);
    return load_turn<D>(t, L, f, q - f * t.Hg, n - q * t.Wg);
}

// The row behind norm and rotation, rounded to binary32.
template <int D, bool NORM, typename T>
__device__ __forceinline__ void normed_and_turned(const LaneRow<T>& x, const Norms& norm, const float (&w)[16], const float (&b)[16], const LaneTurn& t,
                                                  int halves, float (&y)[16]) {
    double u[16];
    if constexpr (NORM) {
        double mean, r;
        row_norm<D>(x, norm.kind, norm.eps, mean, r);
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] = fma(((double)x[e] - mean) * r, (double)w[e], (double)b[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) u[e] = (double)x[e];
    }
    turn_lane(u, t, halves);
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = (float)u[e];
}

// ---- forward -------------------------------------------------------------------------------------------------------
template <typename T>
struct RowsArgs {
    Rows<const T> in[2];
    Rows<T> out[2];
    int n_tokens, nh, heads;  // heads per workgroup
};

// grid: (token tiles, batches x groups of heads, tensors).  A lane keeps its token's angles and its channels' weights while it goes
// through the heads.
template <typename T, int D, bool NORM>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(RowsArgs<T> a, Turning t, Norms norm) {
    constexpr int LANES = D / 16, TOKENS = kThreads / LANES;
    const int L = threadIdx.x % LANES, n = blockIdx.x * TOKENS + threadIdx.x / LANES, z = blockIdx.z;
    if (n >= a.n_tokens) return;
    const int groups = (a.nh + a.heads - 1) / a.heads, b = blockIdx.y / groups, h0 = (blockIdx.y - b * groups) * a.heads;
    const int h1 = min(h0 + a.heads, a.nh);
    const LaneTurn angles = turn_of_token<D>(t, L, n);
    float w[16], bias[16];
    if constexpr (NORM) {
        const int text = n >= t.n_img;
        load_vector<D>(norm.w[z][text], L, 1.0f, w);
        load_vector<D>(norm.b[z][text], L, 0.0f, bias);
    }
    for (int h = h0; h < h1; ++h) {
        LaneRow<T> x;
        x.template load<D>(a.in[z].row(b, h, n), L);
        float y[16];
        normed_and_turned<D, NORM>(x, norm, w, bias, angles, t.halves, y);
        store_lane<D>(a.out[z].row(b, h, n), L, y);
    }
}

// ---- gradients -----------------------------------------------------------------------------------------------------
template <typename T>
struct GradArgs {
    Rows<const T> x[2], dy[2];
    Rows<T> dx[2];
    float* partial;  // [tensor][slot][weight, bias][D], or NULL
    int n_tokens, nh, heads, img_tiles;
};

// grid: (tiles of image tokens, then of text tokens; batches x groups of heads; tensors).  A tile holds tokens of one kind, so a
// workgroup's sums belong to one set of weights.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void norm_rope_grad_kernel(GradArgs<T> a, Turning t, Norms norm) {
    constexpr int LANES = D / 16, TOKENS = kThreads / LANES;
    const int L = threadIdx.x % LANES, row = threadIdx.x / LANES, z = blockIdx.z;
    const int text = (int)blockIdx.x >= a.img_tiles;
    const int n = text ? t.n_img + ((int)blockIdx.x - a.img_tiles) * TOKENS + row : blockIdx.x * TOKENS + row;
    const bool live = n < (text ? a.n_tokens : t.n_img);
    const int groups = (a.nh + a.heads - 1) / a.heads, b = blockIdx.y / groups, h0 = (blockIdx.y - b * groups) * a.heads;
    const int h1 = min(h0 + a.heads, a.nh);
    float dw[16], db[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[e] = db[e] = 0.0f;
    if (live) {
        const LaneTurn angles = turn_of_token<D>(t, L, n);
        float w[16];
        load_vector<D>(norm.w[z][text], L, 1.0f, w);
        for (int h = h0; h < h1; ++h) {
            LaneRow<T> x, dy;
            x.template load<D>(a.x[z].row(b, h, n), L);
            dy.template load<D>(a.dy[z].row(b, h, n), L);
            float g[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) g[e] = dy[e];
            turn_lane(g, angles, t.halves);
            float dx[16];
            if (norm.kind == PARO_NORM_NONE) {
#pragma unroll
                for (int e = 0; e < 16; ++e) dx[e] = g[e];
            } else {
                double mean, r;
                row_norm<D>(x, norm.kind, norm.eps, mean, r);
                float xhat[16], mv = 0.0f, mvh = 0.0f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    xhat[e] = (float)(((double)x[e] - mean) * r);
                    dw[e] = fmaf(g[e], xhat[e], dw[e]);
                    db[e] += g[e];
                    const float v = g[e] * w[e];
                    mv += v;
                    mvh = fmaf(v, xhat[e], mvh);
                }
                mv = norm.kind == PARO_NORM_LAYER ? row_sum<D>(mv) * (1.0f / D) : 0.0f;
                mvh = row_sum<D>(mvh) * (1.0f / D);
                const float rf = (float)r;
#pragma unroll
                for (int e = 0; e < 16; ++e) dx[e] = rf * (fmaf(g[e], w[e], -mv) - xhat[e] * mvh);
            }
            store_lane<D>(a.dx[z].row(b, h, n), L, dx);
        }
    }
    if (!a.partial) return;
    // the workgroup's sums: [weight, bias][channel][token row], one row more against bank conflicts
    __shared__ float meet[D][TOKENS + 1];
    const size_t slot = (size_t)blockIdx.x * gridDim.y + blockIdx.y, slots = (size_t)gridDim.x * gridDim.y;
    float* out = a.partial + (z * slots + slot) * (2 * D);
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 16; ++e) meet[(e >> 3) * (D / 2) + 8 * L + (e & 7)][row] = kind ? db[e] : dw[e];
        __syncthreads();
        if (threadIdx.x < D) {
            double s = 0.0;
            for (int i = 0; i < TOKENS; ++i) s += (double)meet[threadIdx.x][i];
            out[kind * D + threadIdx.x] = (float)s;
        }
    }
}

// One wanted gradient each: slots [first, last) of a tensor's weight or bias sums.
struct GradJob {
    float* out;
    int tensor, kind;
    int64_t first, last;
};
struct GradJobs {
    GradJob job[8];
};

template <int D>
__global__ __launch_bounds__(1024) void norm_grad_kernel(const float* __restrict__ partial, int64_t slots, GradJobs jobs) {
    constexpr int PARTS = 1024 / D;
    __shared__ double meet[PARTS][D];
    const GradJob j = jobs.job[blockIdx.x];
    const int c = threadIdx.x % D, part = threadIdx.x / D;
    double s = 0.0;
    for (int64_t i = j.first + part; i < j.last; i += PARTS) s += (double)partial[((j.tensor * slots + i) * 2 + j.kind) * D + c];
    meet[part][c] = s;
    __syncthreads();
    if (part == 0) {
        for (int i = 1; i < PARTS; ++i) s += meet[i][c];
        j.out[c] = (float)s;
    }
}

// ---- codes of a tile in registers ----------------------------------------------------------------------------------
// Rows of the staged transposed tile (one channel each) are 4 bytes longer than the block for the integer codes, so that the
// byte stores of the 8 lanes that hold one token's 64 channels fall into different LDS banks; bf16 takes 16-bit words.
template <int BITS, int BLK>
constexpr int stage_row() { return BITS == 16 ? BLK : BLK + 4; }
template <int BITS, int BLK, int D>
constexpr int stage_bytes() { return D * stage_row<BITS, BLK>() * (BITS == 16 ? 2 : 1); }

template <int BITS>
__device__ __forceinline__ void codes_of(const float (&x)[8], const GroupDivider& quotient, int (&q)[8]) {
    constexpr float QMAX = BITS == 4 ? 7.0f : 127.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float r = rintf(quotient(x[e]));  // v_rndne_f32: round half to even
        q[e] = (int)fminf(fmaxf(r, -QMAX), QMAX);
    }
}

// PARO_ROWS: the codes of eight channels, the chunk-th eight of the group at `out`.
template <int BITS>
__device__ __forceinline__ void store_codes(uint8_t* out, int chunk, const float (&x)[8], const GroupDivider& quotient) {
    if constexpr (BITS == 16) {
        unsigned h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = f32_to_bf16_bits(x[e]);
        uint4 w = make_uint4(h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16));
        *(uint4*)(out + (size_t)chunk * 16) = w;
    } else {
        int q[8];
        codes_of<BITS>(x, quotient, q);
        if constexpr (BITS == 8) {
            uint2 w;
            w.x = (q[0] & 0xff) | ((q[1] & 0xff) << 8) | ((q[2] & 0xff) << 16) | ((unsigned)q[3] << 24);
            w.y = (q[4] & 0xff) | ((q[5] & 0xff) << 8) | ((q[6] & 0xff) << 16) | ((unsigned)q[7] << 24);
            *(uint2*)(out + (size_t)chunk * 8) = w;
        } else {
            unsigned w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) w |= (unsigned)(q[e] & 0xf) << (4 * e);
            *(unsigned*)(out + (size_t)chunk * 4) = w;
        }
    }
}

// PARO_VT: channels c0 .. c0 + 7 of token `row` of the block, into the staged tile.
template <int BITS, int BLK>
__device__ __forceinline__ void stage_codes(uint8_t* stage, int row, int c0, const float (&x)[8], const GroupDivider& quotient) {
    if constexpr (BITS == 16) {
        unsigned h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = f32_to_bf16_bits(x[e]);
        uint16_t* st = (uint16_t*)stage;
        const int slot = vt_slot(row);
#pragma unroll
        for (int e = 0; e < 8; ++e) st[(c0 + e) * BLK + slot] = (uint16_t)h[e];
    } else {
        int q[8];
        codes_of<BITS>(x, quotient, q);
        const int slot = vt_slot(row);
#pragma unroll
        for (int e = 0; e < 8; ++e) stage[(c0 + e) * stage_row<BITS, BLK>() + slot] = (uint8_t)q[e];
    }
}

// The staged tile to memory, by THREADS threads, 16 bytes (4-bit codes: 4) each in turn.
template <int BITS, int BLK, int D, int THREADS>
__device__ __forceinline__ void store_staged(uint8_t* out, const uint8_t* stage, int tid) {
    constexpr int ELEMS = BLK * D, SSTR = stage_row<BITS, BLK>();
    if constexpr (BITS == 4) {
        // 8 consecutive slots of one channel -> 4 bytes: byte t = slot t | slot 4+t << 4
        constexpr int GROUPS = ELEMS / 8;
        for (int g = tid; g < GROUPS; g += THREADS) {
            const unsigned* src = (const unsigned*)(stage + (g / (BLK / 8)) * SSTR + (g % (BLK / 8)) * 8);
            *(unsigned*)(out + (size_t)g * 4) = (src[0] & 0x0f0f0f0fu) | ((src[1] & 0x0f0f0f0fu) << 4);
        }
    } else if constexpr (BITS == 8) {
        constexpr int VEC = ELEMS / 16;
        for (int v = tid; v < VEC; v += THREADS) {
            const unsigned* src = (const unsigned*)(stage + (v / (BLK / 16)) * SSTR + (v % (BLK / 16)) * 16);
            ((uint4*)out)[v] = make_uint4(src[0], src[1], src[2], src[3]);
        }
    } else {
        constexpr int VEC = ELEMS / 8;
        for (int v = tid; v < VEC; v += THREADS) ((uint4*)out)[v] = ((const uint4*)stage)[v];
    }
}

// ---- with reorder and quantizer ------------------------------------------------------------------------------------
template <typename T>
struct QuantArgs {
    Rows<const T> in[3];
    uint8_t* codes[3];
    float* scales[3];
    int n_tokens, kblocks, nh;
    double inv[6][2];  // per axis order: 1 / extent of the middle and of the fastest axis
    ReorderTable table;
};

// One workgroup owns one group of one tensor (grid: blocks, batches x heads, Q K V), one row per D / 16 lanes.
template <typename T, int BLK, int D, int BITS, int LAYOUT>
__device__ __forceinline__ void quantize_rows(const QuantArgs<T>& a, const Turning& t, const Norms& norm, int z) {
    constexpr int LANES = D / 16, THREADS = BLK * LANES, WAVES = THREADS / 64, OUT_BYTES = BLK * D * BITS / 8;
    constexpr float QMAX = BITS == 4 ? 7.0f : 127.0f;
    __shared__ __attribute__((aligned(16))) uint8_t stage[LAYOUT == PARO_VT ? stage_bytes<BITS, BLK, D>() : 16];
    __shared__ float wave_amax[WAVES];
    const int tid = threadIdx.x, L = tid % LANES, row = tid / LANES, blk = blockIdx.x, bh = blockIdx.y, b = bh / a.nh, h = bh - b * a.nh;
    const size_t group = (size_t)bh * a.kblocks + blk;
    const int n_new = blk * BLK + row;
    float y[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = 0.0f;
    if (n_new < a.n_tokens) {
        int n = n_new, f = 0, hg = 0, w = 0;
        if (n_new < t.n_img) {
            const int order = a.table.perm[h];
            const int* fwd = a.table.fwd[order];
            const int q = quotient_of(n_new, a.inv[order][1]), c2 = n_new - q * fwd[1], c0 = quotient_of(q, a.inv[order][0]), c1 = q - c0 * fwd[0];
            n = c0 * fwd[2] + c1 * fwd[3] + c2 * fwd[4];
            const AxisOrder axes = axis_order(order);
            f = axes.a[0] == 0 ? c0 : axes.a[1] == 0 ? c1 : c2;
            hg = axes.a[0] == 1 ? c0 : axes.a[1] == 1 ? c1 : c2;
            w = axes.a[0] == 2 ? c0 : axes.a[1] == 2 ? c1 : c2;
        }
        LaneRow<T> x;
        x.template load<D>(a.in[z].row(b, h, n), L);
        if (LAYOUT == PARO_VT) {
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = x[e];
        } else {
            LaneTurn angles;
            if (n_new < t.n_img && t.total) angles = load_turn<D>(t, L, f, hg, w);
            else angles = turn_of_token<D>(t, L, t.n_img);
            if (norm.kind == PARO_NORM_NONE) {
                normed_and_turned<D, false>(x, norm, y, y, angles, t.halves, y);
            } else {
                float weight[16], bias[16];
                const int text = n_new >= t.n_img;
                load_vector<D>(norm.w[z][text], L, 1.0f, weight);
                load_vector<D>(norm.b[z][text], L, 0.0f, bias);
                normed_and_turned<D, true>(x, norm, weight, bias, angles, t.halves, y);
            }
        }
    }
    float scale = 1.0f;
    if constexpr (BITS != 16) {
        float amax = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) amax = fmaxf(amax, fabsf(y[e]));
        amax = wave_max(amax);
        if ((tid & 63) == 0) wave_amax[tid >> 6] = amax;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < WAVES; ++i) amax = fmaxf(amax, wave_amax[i]);
        if (amax > 0.0f) scale = amax / QMAX;  // correctly rounded binary32 divide
    }
    if (tid == 0) a.scales[z][group] = scale;
    const GroupDivider quotient(scale);
    uint8_t* out = a.codes[z] + group * OUT_BYTES;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int c0 = half * (D / 2) + 8 * L;
        const float(&v)[8] = *(const float(*)[8])(y + 8 * half);
        if constexpr (LAYOUT == PARO_ROWS) store_codes<BITS>(out, row * (D / 8) + c0 / 8, v, quotient);
        else stage_codes<BITS, BLK>(stage, row, c0, v, quotient);
    }
    if constexpr (LAYOUT == PARO_VT) {
        __syncthreads();
        store_staged<BITS, BLK, D, THREADS>(out, stage, tid);
    }
}

template <typename T, int BLK, int D, int QKBITS, int PVBITS>
__global__ __launch_bounds__(BLK * D / 16) void norm_rope_quantize_kernel(QuantArgs<T> a, Turning t, Norms norm) {
    if (blockIdx.z < 2) quantize_rows<T, BLK, D, QKBITS, PARO_ROWS>(a, t, norm, blockIdx.z);
    else quantize_rows<T, BLK, D, PVBITS, PARO_VT>(a, t, norm, 2);
}

// ---- host ----------------------------------------------------------------------------------------------------------
static bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// Rows that every entry point takes: `what` names them in the error text.
static int check_rows(const paro_shape* s, int64_t n, paro_dtype dtype, const paro_strided* r, const char* what, bool written) {
    if (!r || !r->data) return fail(PARO_EINVAL, "%s is NULL", what);
    const int64_t size = dtype == PARO_F32 ? 4 : 2, extent[3] = {s->B, s->nh, n}, stride[3] = {r->batch, r->head, r->token};
    if (misaligned(r->data)) return fail(PARO_EINVAL, "%s must be 16-byte aligned", what);
    int64_t reach = s->d;
    for (int i = 0; i < 3; ++i) {
        if (extent[i] == 1) continue;
        if (stride[i] < 0 || stride[i] > ((int64_t)1 << 56) / extent[i])
            return fail(PARO_EINVAL, "%s: a stride of %lld elements is negative or out of range", what, (long long)stride[i]);
        if (stride[i] * size % 16) return fail(PARO_EINVAL, "%s: a stride of %lld elements is no multiple of 16 bytes", what, (long long)stride[i]);
    }
    if (!written) return PARO_OK;
    // the strides in ascending order: each must lie behind all that the smaller ones reach
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int x, int y) { return stride[x] < stride[y]; });
    for (int i : order) {
        if (extent[i] == 1) continue;
        if (stride[i] < reach) return fail(PARO_EINVAL, "%s: rows overlap (a stride of %lld elements inside %lld)", what, (long long)stride[i], (long long)reach);
        reach += (extent[i] - 1) * stride[i];
    }
    return PARO_OK;
}

static bool same_rows(const paro_shape* s, int64_t n, const paro_strided* x, const paro_strided* y) {
    return x->data == y->data && (s->B == 1 || x->batch == y->batch) && (s->nh == 1 || x->head == y->head) && (n == 1 || x->token == y->token);
}

static int make_turning(const paro_shape* s, const paro_rope_axes* axes, const float* table, bool back, Turning* t) {
    if (int st = check_axes(s, axes)) return st;
    t->total = (axes->dims[0] + axes->dims[1] + axes->dims[2]) / 2;
    if (t->total && !table) return fail(PARO_EINVAL, "table is NULL");
    if (misaligned(table)) return fail(PARO_EINVAL, "table must be 16-byte aligned");
    t->table = (const float2*)table;
    const int extent[3] = {s->F, s->Hg, s->Wg};
    int64_t at = 0;
    for (int a = 0; a < 3; ++a) {
        t->pairs[a] = axes->dims[a] / 2;
        t->base[a] = (int)at;
        at += (int64_t)extent[a] * t->pairs[a];
    }
    t->n_img = s->F * s->Hg * s->Wg;
    t->Hg = s->Hg;
    t->Wg = s->Wg;
    t->inv_hg = 1.0 / s->Hg;
    t->inv_wg = 1.0 / s->Wg;
    t->sign = back ? -1.0f : 1.0f;
    t->halves = axes->pairs == PARO_PAIRS_HALVES;
    return PARO_OK;
}

static int make_norms(const paro_qk_norm* norm, Norms* out) {
    if (!norm) return fail(PARO_EINVAL, "norm is NULL");
    if (norm->kind != PARO_NORM_NONE && norm->kind != PARO_NORM_RMS && norm->kind != PARO_NORM_LAYER)
        return fail(PARO_EINVAL, "norm kind=%d is not a paro_norm_kind", (int)norm->kind);
    if (norm->kind != PARO_NORM_NONE && !(norm->eps >= 0.0 && norm->eps < INFINITY)) return fail(PARO_EINVAL, "eps=%g must be finite and >= 0", norm->eps);
    out->kind = norm->kind;
    out->eps = norm->eps;
    for (int i = 0; i < 2; ++i) {
        if (norm->kind == PARO_NORM_NONE && (norm->weight[i] || norm->text_weight[i])) return fail(PARO_EINVAL, "weights need a norm");
        if (norm->kind != PARO_NORM_LAYER && (norm->bias[i] || norm->text_bias[i])) return fail(PARO_EINVAL, "biases need PARO_NORM_LAYER");
        for (const float* p : {norm->weight[i], norm->bias[i], norm->text_weight[i], norm->text_bias[i]})
            if (misaligned(p)) return fail(PARO_EINVAL, "weights and biases must be 16-byte aligned");
        out->w[i][0] = norm->weight[i];
        out->b[i][0] = norm->bias[i];
        out->w[i][1] = norm->text_weight[i] ? norm->text_weight[i] : norm->weight[i];
        out->b[i][1] = norm->text_bias[i] ? norm->text_bias[i] : norm->bias[i];
    }
    return PARO_OK;
}

template <typename T>
static Rows<T> rows_of(const paro_strided* r) { return {(T*)r->data, r->batch, r->head, r->token}; }

// Heads that a workgroup goes through: all of them as soon as there are 2048 workgroups without splitting them, else as few as it takes.
static int heads_per_group(const paro_shape* s, int64_t tiles, int tensors) {
    int heads = s->nh;
    while (heads > 1 && tiles * tensors * s->B * ((s->nh + heads - 1) / heads) < 2048) heads = (heads + 1) / 2;
    return heads;
}

static int tile_tokens(const paro_shape* s) { return kThreads / (s->d / 16); }

static int check_dtype(paro_dtype dtype) {
    if (dtype != PARO_F32 && dtype != PARO_BF16) return fail(PARO_EINVAL, "dtype=%d is not a paro_dtype", (int)dtype);
    return PARO_OK;
}

template <typename T, int D>
static void launch_rows(bool norm, dim3 grid, hipStream_t st, const RowsArgs<T>& a, const Turning& t, const Norms& n) {
    if (norm) hipLaunchKernelGGL((rotate_rows_kernel<T, D, true>), grid, dim3(kThreads), 0, st, a, t, n);
    else hipLaunchKernelGGL((rotate_rows_kernel<T, D, false>), grid, dim3(kThreads), 0, st, a, t, n);
}

template <typename T>
static void launch_forward(const paro_shape* s, int64_t n, int tensors, const paro_strided* const (&in)[2], const paro_strided* const (&out)[2],
                           const Turning& t, const Norms& norm, hipStream_t st) {
    RowsArgs<T> a;
    memset(&a, 0, sizeof(a));
    for (int i = 0; i < tensors; ++i) {
        a.in[i] = rows_of<const T>(in[i]);
        a.out[i] = rows_of<T>(out[i]);
    }
    const int64_t tiles = (n + tile_tokens(s) - 1) / tile_tokens(s);
    a.n_tokens = (int)n;
    a.nh = s->nh;
    a.heads = heads_per_group(s, tiles, tensors);
    const dim3 grid((unsigned)tiles, (unsigned)(s->B * ((s->nh + a.heads - 1) / a.heads)), (unsigned)tensors);
    if (s->d == 64) launch_rows<T, 64>(norm.kind != PARO_NORM_NONE, grid, st, a, t, norm);
    else launch_rows<T, 128>(norm.kind != PARO_NORM_NONE, grid, st, a, t, norm);
}

// What the gradient's partial sums take: tiles of image and of text tokens, and the groups of heads.
struct GradSplit {
    int64_t img_tiles, tiles;
    int heads, groups;
    int64_t slots(const paro_shape* s) const { return tiles * s->B * groups; }
};
static GradSplit grad_split(const paro_shape* s) {
    GradSplit g;
    const int64_t tile = tile_tokens(s), n_img = (int64_t)s->F * s->Hg * s->Wg;
    g.img_tiles = (n_img + tile - 1) / tile;
    g.tiles = g.img_tiles + (s->T_text + tile - 1) / tile;
    g.heads = heads_per_group(s, g.tiles, 2);
    g.groups = (s->nh + g.heads - 1) / g.heads;
    return g;
}

template <typename T>
static void launch_grad(const paro_shape* s, int64_t n, const GradSplit& split, const paro_strided* const (&x)[2], const paro_strided* const (&dy)[2],
                        const paro_strided* const (&dx)[2], float* partial, const Turning& t, const Norms& norm, hipStream_t st) {
    GradArgs<T> a;
    for (int i = 0; i < 2; ++i) {
        a.x[i] = rows_of<const T>(x[i]);
        a.dy[i] = rows_of<const T>(dy[i]);
        a.dx[i] = rows_of<T>(dx[i]);
    }
    a.partial = partial;
    a.n_tokens = (int)n;
    a.nh = s->nh;
    a.heads = split.heads;
    a.img_tiles = (int)split.img_tiles;
    const dim3 grid((unsigned)split.tiles, (unsigned)(s->B * split.groups), 2);
    if (s->d == 64) hipLaunchKernelGGL((norm_rope_grad_kernel<T, 64>), grid, dim3(kThreads), 0, st, a, t, norm);
    else hipLaunchKernelGGL((norm_rope_grad_kernel<T, 128>), grid, dim3(kThreads), 0, st, a, t, norm);
}

template <typename T, int BLK, int D>
static bool launch_quant_bits(int bits_qk, int bits_pv, dim3 grid, hipStream_t st, const QuantArgs<T>& a, const Turning& t, const Norms& norm) {
#define PARO_QKV_CASE(QK, PV)                                                                                                             \
    if (bits_qk == QK && bits_pv == PV) {                                                                                                 \
        hipLaunchKernelGGL((norm_rope_quantize_kernel<T, BLK, D, QK, PV>), grid, dim3(BLK * D / 16), 0, st, a, t, norm);                  \
        return true;                                                                                                                      \
    }
    PARO_QKV_CASE(8, 8)
    PARO_QKV_CASE(8, 4)
    PARO_QKV_CASE(4, 4)
    PARO_QKV_CASE(4, 8)
    PARO_QKV_CASE(16, 16)
#undef PARO_QKV_CASE
    return false;
}

template <typename T>
static bool launch_quant(const paro_shape* s, int bits_qk, int bits_pv, dim3 grid, hipStream_t st, const QuantArgs<T>& a, const Turning& t, const Norms& norm) {
    if (s->block == 64 && s->d == 64) return launch_quant_bits<T, 64, 64>(bits_qk, bits_pv, grid, st, a, t, norm);
    if (s->block == 64) return launch_quant_bits<T, 64, 128>(bits_qk, bits_pv, grid, st, a, t, norm);
    if (s->d == 64) return launch_quant_bits<T, 32, 64>(bits_qk, bits_pv, grid, st, a, t, norm);
    return launch_quant_bits<T, 32, 128>(bits_qk, bits_pv, grid, st, a, t, norm);
}

template <typename T>
static int quantize_entry(const paro_shape* s, int64_t n, int64_t kb, int bits_qk, int bits_pv, const uint8_t* h_perm_ids, const paro_strided* const (&in)[3],
                          void* const (&codes)[3], float* const (&scales)[3], const Turning& t, const Norms& norm, hipStream_t st) {
    QuantArgs<T> a;
    if (int e = make_reorder_table(s, h_perm_ids, &a.table)) return e;
    for (int p = 0; p < 6; ++p)
        for (int i = 0; i < 2; ++i) a.inv[p][i] = 1.0 / a.table.fwd[p][i];
    for (int i = 0; i < 3; ++i) {
        a.in[i] = rows_of<const T>(in[i]);
        a.codes[i] = (uint8_t*)codes[i];
        a.scales[i] = scales[i];
    }
    a.n_tokens = (int)n;
    a.kblocks = (int)kb;
    a.nh = s->nh;
    if (!launch_quant<T>(s, bits_qk, bits_pv, dim3((unsigned)kb, (unsigned)(s->B * s->nh), 3), st, a, t, norm))
        return fail(PARO_EINVAL, "bits (qk=%d, pv=%d): expected (8,8), (8,4), (4,4), (4,8) or (16,16)", bits_qk, bits_pv);
    return check_launch("paro_qk_norm_rope_quantize_qkv");
}

}  // namespace paro

using namespace paro;

extern "C" int paro_rope(const paro_shape* s, paro_dtype dtype, const paro_rope_axes* axes, const float* table, int inverse, const paro_strided* x,
                         const paro_strided* y, void* stream) {
    int64_t n;
    Turning t;
    if (int st = check_shape(s, &n, nullptr)) return st;
    if (int st = check_dtype(dtype)) return st;
    if (int st = make_turning(s, axes, table, inverse != 0, &t)) return st;
    if (int st = check_rows(s, n, dtype, x, "x", false)) return st;
    if (int st = check_rows(s, n, dtype, y, "y", true)) return st;
    if (x->data == y->data && !same_rows(s, n, x, y)) return fail(PARO_EINVAL, "y lies in the memory of x in another order");
    Norms none;
    memset(&none, 0, sizeof(none));
    if (dtype == PARO_F32) launch_forward<float>(s, n, 1, {x, nullptr}, {y, nullptr}, t, none, (hipStream_t)stream);
    else launch_forward<uint16_t>(s, n, 1, {x, nullptr}, {y, nullptr}, t, none, (hipStream_t)stream);
    return check_launch("paro_rope");
}

extern "C" int paro_qk_norm_rope(const paro_shape* s, paro_dtype dtype, const paro_rope_axes* axes, const float* table, const paro_qk_norm* norm,
                                 const paro_strided* q, const paro_strided* k, const paro_strided* q_out, const paro_strided* k_out, void* stream) {
    int64_t n;
    Turning t;
    Norms norms;
    if (int st = check_shape(s, &n, nullptr)) return st;
    if (int st = check_dtype(dtype)) return st;
    if (int st = make_turning(s, axes, table, false, &t)) return st;
    if (int st = make_norms(norm, &norms)) return st;
    if (int st = check_rows(s, n, dtype, q, "q", false)) return st;
    if (int st = check_rows(s, n, dtype, k, "k", false)) return st;
    if (int st = check_rows(s, n, dtype, q_out, "q_out", true)) return st;
    if (int st = check_rows(s, n, dtype, k_out, "k_out", true)) return st;
    if (q_out->data == k_out->data || q_out->data == k->data || k_out->data == q->data || (q_out->data == q->data && !same_rows(s, n, q, q_out)) ||
        (k_out->data == k->data && !same_rows(s, n, k, k_out)))
        return fail(PARO_EINVAL, "an output may be its own input in the same order, and none of the other tensors");
    if (dtype == PARO_F32) launch_forward<float>(s, n, 2, {q, k}, {q_out, k_out}, t, norms, (hipStream_t)stream);
    else launch_forward<uint16_t>(s, n, 2, {q, k}, {q_out, k_out}, t, norms, (hipStream_t)stream);
    return check_launch("paro_qk_norm_rope");
}

extern "C" int64_t paro_qk_norm_rope_backward_bytes(const paro_shape* s) {
    if (int st = check_shape(s, nullptr, nullptr)) return st;
    return grad_split(s).slots(s) * 2 * 2 * s->d * 4;
}

extern "C" int paro_qk_norm_rope_backward(const paro_shape* s, paro_dtype dtype, const paro_rope_axes* axes, const float* table, const paro_qk_norm* norm,
                                          const paro_strided* q, const paro_strided* k, const paro_strided* dq_out, const paro_strided* dk_out,
                                          const paro_strided* dq, const paro_strided* dk, const paro_qk_norm_grad* grad, void* scratch, void* stream) {
    int64_t n;
    Turning t;
    Norms norms;
    if (int st = check_shape(s, &n, nullptr)) return st;
    if (int st = check_dtype(dtype)) return st;
    if (int st = make_turning(s, axes, table, true, &t)) return st;
    if (int st = make_norms(norm, &norms)) return st;
    const paro_strided* const x[2] = {q, k};
    const paro_strided* const dy[2] = {dq_out, dk_out};
    const paro_strided* const dx[2] = {dq, dk};
    const char* const names[3][2] = {{"q", "k"}, {"dq_out", "dk_out"}, {"dq", "dk"}};
    for (int i = 0; i < 2; ++i) {
        if (int st = check_rows(s, n, dtype, x[i], names[0][i], false)) return st;
        if (int st = check_rows(s, n, dtype, dy[i], names[1][i], false)) return st;
        if (int st = check_rows(s, n, dtype, dx[i], names[2][i], true)) return st;
    }
    for (int i = 0; i < 2; ++i) {
        const void* mine = dx[i]->data;
        if (mine == dx[1 - i]->data || mine == x[1 - i]->data || mine == dy[1 - i]->data || (mine == x[i]->data && !same_rows(s, n, x[i], dx[i])) ||
            (mine == dy[i]->data && !same_rows(s, n, dy[i], dx[i])))
            return fail(PARO_EINVAL, "%s may be %s or %s in the same order, and none of the other tensors", names[2][i], names[0][i], names[1][i]);
    }
    const GradSplit split = grad_split(s);
    const int64_t slots = split.slots(s), img_slots = split.img_tiles * s->B * split.groups;
    GradJobs jobs;
    int count = 0;
    for (int i = 0; grad && i < 2; ++i)
        for (int kind = 0; kind < 2; ++kind) {
            float* const whole = kind ? grad->bias[i] : grad->weight[i];
            float* const text = kind ? grad->text_bias[i] : grad->text_weight[i];
            const bool own = (kind ? norm->text_bias[i] : norm->text_weight[i]) != nullptr;
            if ((whole || text) && norm->kind == PARO_NORM_NONE) return fail(PARO_EINVAL, "gradients of weights need a norm");
            if ((whole || text) && kind && norm->kind != PARO_NORM_LAYER) return fail(PARO_EINVAL, "gradients of biases need PARO_NORM_LAYER");
            if (text && !own) return fail(PARO_EINVAL, "a text gradient needs the text tokens' own %s", kind ? "bias" : "weight");
            if (misaligned(whole) || misaligned(text)) return fail(PARO_EINVAL, "gradients must be 16-byte aligned");
            if (whole) jobs.job[count++] = {whole, i, kind, 0, own ? img_slots : slots};
            if (text) jobs.job[count++] = {text, i, kind, img_slots, slots};
        }
    for (int i = 0; i < count; ++i)
        for (int j = 0; j < i; ++j)
            if (jobs.job[i].out == jobs.job[j].out) return fail(PARO_EINVAL, "two gradients must not share memory");
    if (count && (!scratch || misaligned(scratch))) return fail(PARO_EINVAL, "scratch must be a 16-byte aligned buffer");
    const auto st = (hipStream_t)stream;
    float* const partial = count ? (float*)scratch : nullptr;
    if (dtype == PARO_F32) launch_grad<float>(s, n, split, x, dy, dx, partial, t, norms, st);
    else launch_grad<uint16_t>(s, n, split, x, dy, dx, partial, t, norms, st);
    if (int e = check_launch("paro_qk_norm_rope_backward")) return e;
    if (count) {
        if (s->d == 64) hipLaunchKernelGGL((norm_grad_kernel<64>), dim3(count), dim3(1024), 0, st, partial, slots, jobs);
        else hipLaunchKernelGGL((norm_grad_kernel<128>), dim3(count), dim3(1024), 0, st, partial, slots, jobs);
    }
    return check_launch("paro_qk_norm_rope_backward");
}

extern "C" int paro_qk_norm_rope_quantize_qkv(const paro_shape* s, paro_dtype dtype, int bits_qk, int bits_pv, const uint8_t* h_perm_ids,
                                              const paro_rope_axes* axes, const float* table, const paro_qk_norm* norm, const paro_strided* q,
                                              const paro_strided* k, const paro_strided* v, void* q_codes, float* sq, void* k_codes, float* sk,
                                              void* v_codes, float* sv, void* stream) {
    int64_t n, kb;
    Turning t;
    Norms norms;
    if (int st = check_shape(s, &n, &kb)) return st;
    if (int st = check_dtype(dtype)) return st;
    if (!h_perm_ids) return fail(PARO_EINVAL, "perm_ids is NULL");
    if (int st = make_turning(s, axes, table, false, &t)) return st;
    if (int st = make_norms(norm, &norms)) return st;
    const paro_strided* const in[3] = {q, k, v};
    void* const codes[3] = {q_codes, k_codes, v_codes};
    float* const scales[3] = {sq, sk, sv};
    const char* const names[3] = {"q", "k", "v"};
    for (int i = 0; i < 3; ++i) {
        if (int st = check_rows(s, n, dtype, in[i], names[i], false)) return st;
        if (!codes[i] || !scales[i]) return fail(PARO_EINVAL, "codes and scales must not be NULL");
        if (misaligned(codes[i])) return fail(PARO_EINVAL, "codes must be 16-byte aligned");
    }
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < 3; ++j)
            if (codes[i] == in[j]->data || (i != j && codes[i] == codes[j]) || (i != j && scales[i] == scales[j]))
                return fail(PARO_EINVAL, "inputs and outputs must not alias");
    const auto st = (hipStream_t)stream;
    if (dtype == PARO_F32) return quantize_entry<float>(s, n, kb, bits_qk, bits_pv, h_perm_ids, in, codes, scales, t, norms, st);
    return quantize_entry<uint16_t>(s, n, kb, bits_qk, bits_pv, h_perm_ids, in, codes, scales, t, norms, st);
}
