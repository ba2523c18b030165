// Norms of Q and K per head and their rotation by the token's (frame, height, width) position: forward, gradients, and both
// with the reorder (paper Sec. 4.1) and the block quantizer (Sec. 4.3 (1)) behind them.
//
// A row is the d channels of one token of one head.  d / 8 lanes share it, eight channels each: for adjacent pairs the eight
// from 8 L on, for pairs across the halves four from 4 L on and the four that lie d / 2 behind them, so that a lane holds both
// channels of its pairs 4 L .. 4 L + 3.  Row sums meet across neighbouring lanes (DPP).  (16 channels a lane: 183 vector registers, two wavefronts
// per SIMD, 126 us where eight take 89.)
//
// The angles' table separates by axis: some KB instead of some MB per layer, so it comes from the caches nearest to the compute
// unit.
//
// Sums and values are binary64 and rounded to binary32 once: the codes of the quantizing form then do not depend on the order of
// a sum (up to values within 2^-45 of a rounding border), and the instructions cost what binary32 ones do.
//
// Everything but the 8- and 4-bit quantizing form is bound by HBM.  48 heads of 17550 bf16 tokens, d = 64, where a copy takes 5.2 TB/s: rotation 44
// us (216 MB, 4.9 TB/s) out of one projection's output and 39 from contiguous heads, norms and rotation of Q and K 89 (431 MB, 4.8) and 81,
// gradients 142 (647 MB, 4.6) and 130.  Stores past the caches take 5 to 15 % off these kernels by themselves, and add more than that to the next one, which
// reads what they wrote (copy, norms and rotation, quantizer: 323 -> 329 us; 24 heads of 4608 tokens, d = 128: 46.0 -> 47.8): not used.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "common.h"

namespace paro {

constexpr int kThreads = 256;

// Channels turned by position: what the kernels need of a paro_rope_axes, its table and the grid.
struct Turning {
    const float* table;
    int pairs[3];  // pairs per axis
    int base[3];   // first entry of an axis in the table
    int total;     // pairs that turn; pair p turns with the axis whose run of pairs holds it
    bool fours;    // there are pairs, a multiple of four per axis: four entries from a multiple of four on are one axis' and 32 aligned bytes
    int n_img, Hg, Wg;
    double inv_hg, inv_wg;
    float sign;  // -1: turned back
};

// Norms: entry [tensor][text].
struct Norms {
    const float* w[2][2];
    const float* b[2][2];
    double eps;
};

template <typename T>
struct Rows {
    T* p;
    int64_t batch, head;
    int token;
    __device__ T* row(int b, int h, int n) const { return p + b * batch + h * head + (int64_t)n * token; }
};

// floor(n / divisor) for 0 <= n < 2^24 and a divisor of at most that, inv = fl64(1 / divisor): (n + 1/2) inv lies 1 / (2 divisor)
// or more from the next integers, and is off by less than 2^-51 n / divisor.
__device__ inline int quotient_of(int n, double inv) { return (int)(((double)n + 0.5) * inv); }

// By value: a conditional between members would choose between their addresses, and every lane would load from there.
__device__ __forceinline__ int pick(int c0, int c1, int c2, int place) { return place == 0 ? c0 : place == 1 ? c1 : c2; }
__device__ __forceinline__ const float* pick(const float* image, const float* text, bool is_text) { return is_text ? text : image; }

// ---- the 8 channels of a lane --------------------------------------------------------------------------------------
typedef unsigned uint4v __attribute__((ext_vector_type(4)));
typedef unsigned uint2v __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ inline unsigned pack_bf16(float a, float b) { return __builtin_bit_cast(unsigned, __builtin_convertvector((float2v){a, b}, bf16x2)); }

// As in memory: 16 bytes of bf16 or 32 of binary32, in one piece or in two (HALVES).
template <typename T, int D, bool HALVES>
struct LaneRow {
    static constexpr int WORDS = 2 * sizeof(T);
    unsigned w[WORDS];
    // where the lane's second four channels lie behind its first
    static constexpr int SECOND = HALVES ? D / 2 : 4;
    static __device__ __forceinline__ int first(int L) { return HALVES ? 4 * L : 8 * L; }

    __device__ __forceinline__ void load(const T* row, int L) {
        const T* p = row + first(L);
        if constexpr (sizeof(T) == 2 && !HALVES) {
            const uint4v v = *(const uint4v*)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = v[i];
        } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if constexpr (sizeof(T) == 2) {
                    const uint2v v = *(const uint2v*)(p + half * SECOND);
                    w[2 * half] = v[0], w[2 * half + 1] = v[1];
                } else {
                    const uint4v v = *(const uint4v*)(p + half * SECOND);
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[4 * half + i] = v[i];
                }
            }
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0;
    }
    __device__ __forceinline__ float operator[](int e) const {
        if constexpr (sizeof(T) == 2) return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
        else return __uint_as_float(w[e]);
    }
    static __device__ __forceinline__ void store(T* row, int L, const float (&y)[8]) {
        T* p = row + first(L);
        if constexpr (sizeof(T) == 2) {
            const unsigned v[4] = {pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])};
            if constexpr (HALVES) {
                *(uint2v*)p = (uint2v){v[0], v[1]};
                *(uint2v*)(p + SECOND) = (uint2v){v[2], v[3]};
            } else {
                *(uint4v*)p = (uint4v){v[0], v[1], v[2], v[3]};
            }
        } else {
            ((float4*)p)[0] = make_float4(y[0], y[1], y[2], y[3]);
            *(float4*)(p + SECOND) = make_float4(y[4], y[5], y[6], y[7]);
        }
    }
};

// A lane's channels of a float32 [d] vector, or `other` where there is none.
template <int D, bool HALVES>
__device__ __forceinline__ void load_vector(const float* v, int L, float other, float (&x)[8]) {
    if (v) {
        LaneRow<float, D, HALVES> r;
        r.load(v, L);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = r[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = other;
    }
}

// ---- row sums ------------------------------------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ int moved(int v) { return __builtin_amdgcn_mov_dpp(v, CTRL, 0xf, 0xf, true); }
template <int CTRL>
__device__ __forceinline__ double moved(double v) { return __hiloint2double(moved<CTRL>(__double2hiint(v)), moved<CTRL>(__double2loint(v))); }
template <int CTRL>
__device__ __forceinline__ float moved(float v) { return __int_as_float(moved<CTRL>(__float_as_int(v))); }
// Sum over the D / 8 neighbouring lanes of a row, in every one of them: the lane beside (quad_perm 1 0 3 2), the pair beside
// (2 3 0 1), the other four of eight (row_half_mirror), the other eight of sixteen (row_mirror).
template <int D, typename V>
__device__ __forceinline__ V row_sum(V v) {
    v += moved<0xB1>(v);
    v += moved<0x4E>(v);
    v += moved<0x141>(v);
    if constexpr (D == 128) v += moved<0x140>(v);
    return v;
}

// Sum over the rows of a wavefront, lane by lane of a row: lanes 8 (d = 64), 16 and 32 apart.
template <int D>
__device__ __forceinline__ float rows_sum(float v) {
    if constexpr (D == 64) v += moved<0x128>(v);  // row_ror:8
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// 1 / sqrt(v): the instruction's estimate y (2^-24 off on this card at most) and one step of third order, y (1 + e/2 + 3/8 e^2) with
// e = 1 - v y^2, which leaves 5/16 e^3: the result is within 2^-52.  The estimate stands where v is 0 or infinite.
__device__ __forceinline__ double rsqrt_of(double v) {
    const double y = __builtin_amdgcn_rsq(v), e = fma(-v * y, y, 1.0);
    const double better = fma(y * e, fma(e, 0.375, 0.5), y);
    return __builtin_amdgcn_class(v, 0x264) ? y : better;  // zeros and infinities
}

// What a row is divided by; under PARO_NORM_LAYER its values lose their mean first.
template <int D>
__device__ __forceinline__ double row_norm(double (&u)[8], int kind, double eps) {
    if (kind == PARO_NORM_LAYER) {
        double s = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) s += u[e];
        s = row_sum<D>(s) * (1.0 / D);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] -= s;
    }
    double s = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fma(u[e], u[e], s);
    return rsqrt_of(fma(row_sum<D>(s), 1.0 / D, eps));
}

// ---- turning -------------------------------------------------------------------------------------------------------
// Pair e of a lane: its channels (2e, 2e + 1), or (e, 4 + e) with HALVES.
struct LaneTurn {
    float c[4], s[4];
    unsigned turned;  // bit e: pair e turns
    __device__ __forceinline__ void none() {
        turned = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = 1.0f, s[e] = 0.0f;
    }
};

__device__ __forceinline__ void load_turn(const Turning& t, int L, int f, int h, int w, LaneTurn& r) {
    const int to1 = t.pairs[0], to2 = t.pairs[0] + t.pairs[1], p0 = 4 * L;
    const int e0 = t.base[0] + f * t.pairs[0], e1 = t.base[1] + h * t.pairs[1] - to1, e2 = t.base[2] + w * t.pairs[2] - to2;
    r.none();
    if (t.fours) {
        if (p0 >= t.total) return;
        const float4* v = (const float4*)(t.table + 2 * (int64_t)((p0 < to1 ? e0 : p0 < to2 ? e1 : e2) + p0));
        const float4 a = v[0], b = v[1];
        r.c[0] = a.x, r.c[1] = a.z, r.c[2] = b.x, r.c[3] = b.z;
        r.s[0] = a.y * t.sign, r.s[1] = a.w * t.sign, r.s[2] = b.y * t.sign, r.s[3] = b.w * t.sign;
        r.turned = 15;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int p = p0 + e;
        if (p < t.total) {
            const float2 v = *(const float2*)(t.table + 2 * (int64_t)((p < to1 ? e0 : p < to2 ? e1 : e2) + p));
            r.c[e] = v.x;
            r.s[e] = v.y * t.sign;
            r.turned |= 1u << e;
        }
    }
}

// Grid coordinates of a token in default order; text tokens do not turn.
__device__ __forceinline__ void turn_of_token(const Turning& t, int L, int n, LaneTurn& r) {
    if (n < t.n_img && t.total) {
        const int q = quotient_of(n, t.inv_wg), f = quotient_of(q, t.inv_hg);
        load_turn(t, L, f, q - f * t.Hg, n - q * t.Wg, r);
    } else {
        r.none();
    }
}

template <typename V>
__device__ __forceinline__ void turn_pair(V& x, V& y, V c, V s) {
    const V a = fma(x, c, -(y * s));
    y = fma(x, s, y * c);
    x = a;
}
// A value that does not turn stays as it is, whatever its partner holds.
template <bool HALVES, typename V>
__device__ __forceinline__ void turn_lane(V (&u)[8], const LaneTurn& t) {
    if (t.turned == 15) {
#pragma unroll
        for (int e = 0; e < 4; ++e) turn_pair<V>(HALVES ? u[e] : u[2 * e], HALVES ? u[4 + e] : u[2 * e + 1], t.c[e], t.s[e]);
    } else if (t.turned) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (t.turned >> e & 1) turn_pair<V>(HALVES ? u[e] : u[2 * e], HALVES ? u[4 + e] : u[2 * e + 1], t.c[e], t.s[e]);
    }
}

// The row behind norm and rotation, rounded to binary32.  w and b: 1 and 0 where there is nothing, in every kernel: a row that is its mean then
// leaves +0 under any weights.
template <typename T, int D, bool HALVES, typename W>
__device__ __forceinline__ void normed_and_turned(const LaneRow<T, D, HALVES>& x, int kind, double eps, const W& w, const W& b, const LaneTurn& t,
                                                  float (&y)[8]) {
    double u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = (double)x[e];
    if (kind != PARO_NORM_NONE) {
        const double r = row_norm<D>(u, kind, eps);
        if (kind == PARO_NORM_LAYER) {
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = fma(u[e] * r, (double)w[e], (double)b[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = u[e] * r * (double)w[e];
        }
    }
    turn_lane<HALVES>(u, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (float)u[e];
}

// ---- forward -------------------------------------------------------------------------------------------------------
template <typename T>
struct RowsArgs {
    Rows<const T> in[2];
    Rows<T> out[2];
    int n_tokens, nh, heads;  // heads per workgroup
};

// grid: (token tiles, batches x groups of heads, tensors).  A lane keeps its token's angles and its channels' weights while it goes
// through the heads, and reads a row while it works on the one before.
template <typename T, int D, int KIND, bool HALVES>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(RowsArgs<T> a, Turning t, Norms norm) {
    constexpr int LANES = D / 8, TOKENS = kThreads / LANES;
    const int L = threadIdx.x % LANES, n = blockIdx.x * TOKENS + threadIdx.x / LANES, z = blockIdx.z;
    if (n >= a.n_tokens) return;
    const int groups = (a.nh + a.heads - 1) / a.heads, b = blockIdx.y / groups, h0 = (blockIdx.y - b * groups) * a.heads;
    const int h1 = min(h0 + a.heads, a.nh);
    LaneRow<T, D, HALVES> next;
    next.load(a.in[z].row(b, h0, n), L);
    LaneTurn angles;
    turn_of_token(t, L, n, angles);
    float w[8], bias[8];
    const bool text = n >= t.n_img;
    if constexpr (KIND != PARO_NORM_NONE) load_vector<D, HALVES>(pick(norm.w[z][0], norm.w[z][1], text), L, 1.0f, w);
    if constexpr (KIND == PARO_NORM_LAYER) load_vector<D, HALVES>(pick(norm.b[z][0], norm.b[z][1], text), L, 0.0f, bias);
    for (int h = h0; h < h1; ++h) {
        const LaneRow<T, D, HALVES> x = next;
        if (h + 1 < h1) next.load(a.in[z].row(b, h + 1, n), L);
        float y[8];
        normed_and_turned(x, KIND, norm.eps, w, bias, angles, y);
        LaneRow<T, D, HALVES>::store(a.out[z].row(b, h, n), L, y);
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
template <typename T, int D, int KIND, bool HALVES>
__global__ __launch_bounds__(kThreads) void norm_rope_grad_kernel(GradArgs<T> a, Turning t, Norms norm) {
    constexpr int LANES = D / 8, TOKENS = kThreads / LANES;
    typedef LaneRow<T, D, HALVES> Lane;
    const int L = threadIdx.x % LANES, row = threadIdx.x / LANES, z = blockIdx.z;
    const int text = (int)blockIdx.x >= a.img_tiles;
    const int n = text ? t.n_img + ((int)blockIdx.x - a.img_tiles) * TOKENS + row : blockIdx.x * TOKENS + row;
    const bool live = n < (text ? a.n_tokens : t.n_img);
    const int groups = (a.nh + a.heads - 1) / a.heads, b = blockIdx.y / groups, h0 = (blockIdx.y - b * groups) * a.heads;
    const int h1 = min(h0 + a.heads, a.nh);
    float dw[8], db[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[e] = db[e] = 0.0f;
    if (live) {
        Lane next_x, next_dy;
        next_x.load(a.x[z].row(b, h0, n), L);
        next_dy.load(a.dy[z].row(b, h0, n), L);
        LaneTurn angles;
        turn_of_token(t, L, n, angles);
        float w[8];
        load_vector<D, HALVES>(norm.w[z][text], L, 1.0f, w);
        for (int h = h0; h < h1; ++h) {
            const Lane x = next_x, dy = next_dy;
            if (h + 1 < h1) {
                next_x.load(a.x[z].row(b, h + 1, n), L);
                next_dy.load(a.dy[z].row(b, h + 1, n), L);
            }
            float g[8], dx[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] = dy[e];
            turn_lane<HALVES>(g, angles);
            if constexpr (KIND == PARO_NORM_NONE) {
#pragma unroll
                for (int e = 0; e < 8; ++e) dx[e] = g[e];
            } else {
                double u[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = (double)x[e];
                const double r = row_norm<D>(u, KIND, norm.eps);
                float xhat[8], mv = 0.0f, mvh = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    xhat[e] = (float)(u[e] * r);
                    dw[e] = fmaf(g[e], xhat[e], dw[e]);
                    db[e] += g[e];
                    const float v = g[e] * w[e];
                    mv += v;
                    mvh = fmaf(v, xhat[e], mvh);
                }
                mv = KIND == PARO_NORM_LAYER ? row_sum<D>(mv) * (1.0f / D) : 0.0f;
                mvh = row_sum<D>(mvh) * (1.0f / D);
                const float rf = (float)r;
#pragma unroll
                for (int e = 0; e < 8; ++e) dx[e] = rf * (fmaf(g[e], w[e], -mv) - xhat[e] * mvh);
            }
            Lane::store(a.dx[z].row(b, h, n), L, dx);
        }
    }
    if (KIND == PARO_NORM_NONE || !a.partial) return;
    // the workgroup's sums: over the rows of a wavefront, then over the wavefronts
    constexpr int KINDS = KIND == PARO_NORM_LAYER ? 2 : 1, WAVES = kThreads / 64;
    __shared__ float meet[WAVES][KINDS][D];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int kind = 0; kind < KINDS; ++kind)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float s = rows_sum<D>(kind ? db[e] : dw[e]);
            if (lane < LANES) meet[wave][kind][Lane::first(L) + (e >> 2) * Lane::SECOND + (e & 3)] = s;
        }
    __syncthreads();
    const size_t slot = (size_t)blockIdx.x * gridDim.y + blockIdx.y, slots = (size_t)gridDim.x * gridDim.y;
    float* out = a.partial + (z * slots + slot) * (2 * D);
    if (threadIdx.x < KINDS * D) {
        const int kind = threadIdx.x / D, c = threadIdx.x % D;
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) s += (double)meet[i][kind][c];
        out[threadIdx.x] = (float)s;
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

// grid: (jobs, D / 16).  A workgroup adds up 16 channels of a job's slots, 64 slots at a time, in binary64 and in a fixed order; four loads a
// thread are in flight.
template <int D>
__global__ __launch_bounds__(1024) void norm_grad_kernel(const float* __restrict__ partial, int64_t slots, GradJobs jobs) {
    constexpr int PARTS = 64;
    __shared__ double meet[PARTS][16];
    const GradJob j = jobs.job[blockIdx.x];
    const int c = threadIdx.x % 16, part = threadIdx.x / 16;
    const float* mine = partial + (j.tensor * slots * 2 + j.kind) * D + blockIdx.y * 16 + c;
    double s = 0.0;
#pragma unroll 4
    for (int64_t i = j.first + part; i < j.last; i += PARTS) s += (double)mine[i * (2 * D)];
    meet[part][c] = s;
    __syncthreads();
    if (part < 8) {
        for (int i = 8; i < PARTS; i += 8) s += meet[part + i][c];
        meet[part][c] = s;  // no other thread reads this entry before the barrier
    }
    __syncthreads();
    if (part == 0) {
        for (int i = 1; i < 8; ++i) s += meet[i][c];
        j.out[blockIdx.y * 16 + c] = (float)s;
    }
}

// ---- codes of a tile in registers ----------------------------------------------------------------------------------
// Rows of the staged transposed tile (one channel each) are 4 bytes longer than the block, so that the stores of lanes that hold one token's
// channels fall into different LDS banks (bf16, 24 heads of 4608 tokens, d = 128: 44 -> 38 us); bf16 takes 16-bit words.
template <int BITS, int BLK>
constexpr int stage_row() { return BITS == 16 ? BLK + 2 : BLK + 4; }
template <int BITS, int BLK, int D>
constexpr int stage_bytes() { return D * stage_row<BITS, BLK>() * (BITS == 16 ? 2 : 1); }

// The largest of a value over a wavefront, in every lane: as row_sum and rows_sum.
__device__ __forceinline__ float wavefront_max(float v) {
    v = fmaxf(v, moved<0xB1>(v));
    v = fmaxf(v, moved<0x4E>(v));
    v = fmaxf(v, moved<0x141>(v));
    v = fmaxf(v, moved<0x140>(v));
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The largest magnitude of a lane's values: past every NaN, or NaN where there is one (v_maximum3_f32, which needs its operands in no
// canonical form first).
template <bool NANS, int N>
__device__ __forceinline__ float lane_max(const float (&y)[N][8]) {
    float m = 0.0f;
#pragma unroll
    for (int it = 0; it < N; ++it)
#pragma unroll
        for (int e = 0; e < 8; ++e) m = NANS ? __builtin_elementwise_maximum(m, fabsf(y[it][e])) : fmaxf(m, fabsf(y[it][e]));
    return m;
}

__device__ __forceinline__ float uniform(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }

// x / scale for a group as GroupDivider has it, correctly rounded, with short ways to the scale amax / QMAX (the same theorem, with the constant's
// reciprocal) and to 1 / scale: from the instruction's estimate y, within a unit in the last place, 1 - scale y is exact, and y + y (1 - scale y)
// rounds correctly for every significand but all ones.  Both equal the divide for each amax of the range (all 10^9 compared).
// nans: there are some among the wavefront's values; its quotients then take the divide and its clamps.
template <int BITS>
struct GroupQuotient {
    static constexpr float QMAX = BITS == 4 ? 7.0f : 127.0f;
    float scale, inv;
    bool generic;
    __device__ __forceinline__ GroupQuotient(float amax, bool nans) {
        constexpr float INV = 1.0f / QMAX;
        if (amax > 1e-18f && amax < 1e20f) {
            const float q0 = amax * INV;
            scale = fmaf(fmaf(-q0, QMAX, amax), INV, q0);
            const float y = __builtin_amdgcn_rcpf(scale);
            inv = fmaf(fmaf(-scale, y, 1.0f), y, y);
            generic = nans || (__float_as_uint(scale) & 0x7fffffu) == 0x7fffffu;
        } else {
            scale = amax > 0.0f ? amax / QMAX : 1.0f;
            inv = 0.0f;
            generic = true;
        }
    }
};

// Codes of a lane's values, each in the low byte (4-bit codes: the low four bits) of its word.  A quotient of numbers is at most QMAX (1 + 2^-22) in
// magnitude where the scale is a normal number, which rounds to QMAX: only the generic divide clamps, in groups whose scale lost bits or is
// infinite, and NaN.  Adding 1.5 2^23 rounds to an integer, halves to even, and leaves it as two's complement in the low bits.
template <int BITS>
__device__ __forceinline__ void codes_of(const float (&x)[8], const GroupQuotient<BITS>& quotient, unsigned (&q)[8]) {
    constexpr float QMAX = GroupQuotient<BITS>::QMAX;
    float r[8];
    if (quotient.generic) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = fminf(fmaxf(x[e] / quotient.scale, -QMAX), QMAX);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float q0 = x[e] * quotient.inv;
            r[e] = fmaf(fmaf(-q0, quotient.scale, x[e]), quotient.inv, q0);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = __float_as_uint(r[e] + 12582912.0f);
}

// The low bytes of four words.
__device__ __forceinline__ unsigned low_bytes(unsigned a, unsigned b, unsigned c, unsigned d) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400), __builtin_amdgcn_perm(b, a, 0x0c0c0400), 0x05040100);
}

// PARO_ROWS: a lane's codes into its row of the group.
template <int BITS, int D, bool HALVES>
__device__ __forceinline__ void store_codes(uint8_t* row, int L, const float (&x)[8], const GroupQuotient<BITS>& quotient) {
    typedef LaneRow<float, D, HALVES> Lane;
    const int first = Lane::first(L), second = first + Lane::SECOND;
    if constexpr (BITS == 16) {
        const unsigned v[4] = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
        if constexpr (HALVES) {
            *(uint2v*)(row + 2 * first) = (uint2v){v[0], v[1]};
            *(uint2v*)(row + 2 * second) = (uint2v){v[2], v[3]};
        } else {
            *(uint4v*)(row + 2 * first) = (uint4v){v[0], v[1], v[2], v[3]};
        }
    } else {
        unsigned q[8];
        codes_of<BITS>(x, quotient, q);
        unsigned v[2] = {low_bytes(q[0], q[1], q[2], q[3]), low_bytes(q[4], q[5], q[6], q[7])};
        if constexpr (BITS == 8) {
            if constexpr (HALVES) {
                *(unsigned*)(row + first) = v[0];
                *(unsigned*)(row + second) = v[1];
            } else {
                *(uint2v*)(row + first) = (uint2v){v[0], v[1]};
            }
        } else {
            // bytes 0 and 2 of each word take their upper neighbour's code as upper half
#pragma unroll
            for (int i = 0; i < 2; ++i) v[i] = (v[i] & 0x000f000f) | (v[i] >> 4 & 0x00f000f0);
            const unsigned all = __builtin_amdgcn_perm(v[1], v[0], 0x06040200);
            if constexpr (HALVES) {
                *(uint16_t*)(row + first / 2) = (uint16_t)all;
                *(uint16_t*)(row + second / 2) = (uint16_t)(all >> 16);
            } else {
                *(unsigned*)(row + first / 2) = all;
            }
        }
    }
}

// PARO_VT: a lane's channels of token `token` of the block, into the staged tile.
template <int BITS, int BLK, int D, bool HALVES>
__device__ __forceinline__ void stage_codes(uint8_t* stage, int token, int L, const float (&x)[8], const GroupQuotient<BITS>& quotient) {
    typedef LaneRow<float, D, HALVES> Lane;
    const int slot = vt_slot(token);
    const auto at = [&](int e) { return (Lane::first(L) + (e >> 2) * Lane::SECOND + (e & 3)) * stage_row<BITS, BLK>() + slot; };
    if constexpr (BITS == 16) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const unsigned two = pack_bf16(x[e], x[e + 1]);
            ((uint16_t*)stage)[at(e)] = (uint16_t)two;
            ((uint16_t*)stage)[at(e + 1)] = (uint16_t)(two >> 16);
        }
    } else {
        unsigned q[8];
        codes_of<BITS>(x, quotient, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) stage[at(e)] = (uint8_t)q[e];
    }
}

// The staged tile to memory, by the workgroup, 16 bytes (4-bit codes: 4) each in turn.
template <int BITS, int BLK, int D>
__device__ __forceinline__ void store_staged(uint8_t* out, const uint8_t* stage, int tid) {
    constexpr int ELEMS = BLK * D, SSTR = stage_row<BITS, BLK>();
    if constexpr (BITS == 4) {
        // 8 consecutive slots of one channel -> 4 bytes: byte t = slot t | slot 4+t << 4
        constexpr int GROUPS = ELEMS / 8;
        for (int g = tid; g < GROUPS; g += kThreads) {
            const unsigned* src = (const unsigned*)(stage + (g / (BLK / 8)) * SSTR + (g % (BLK / 8)) * 8);
            *(unsigned*)(out + (size_t)g * 4) = (src[0] & 0x0f0f0f0fu) | ((src[1] & 0x0f0f0f0fu) << 4);
        }
    } else {
        constexpr int BYTES = BITS / 8, PIECES = BLK * BYTES / 16;  // 16-byte pieces per channel
        for (int v = tid; v < D * PIECES; v += kThreads) {
            const unsigned* src = (const unsigned*)(stage + (v / PIECES) * SSTR * BYTES + (v % PIECES) * 16);
            ((uint4*)out)[v] = make_uint4(src[0], src[1], src[2], src[3]);
        }
    }
}

// ---- with reorder and quantizer ------------------------------------------------------------------------------------
// The six axis orders, as the kernels below use them.
struct Orders {
    uint32_t ids[kMaxHeads / 4];  // a head's order id, a byte each
    int extent[6][2];             // of the middle and of the fastest axis
    int stride[6][3];             // default-order strides of the slowest, middle and fastest axis
    int place[6][3];              // which of the three the frame, height and width axis is
    double inv[6][2];             // 1 / extent
};

template <typename T>
struct QuantArgs {
    Rows<const T> in[3];
    uint8_t* codes[3];
    float* scales[3];
    int n_tokens, kblocks, nh, kind, span;  // blocks per workgroup
    Orders orders;
};

// A head's order, and where a token of its sequence comes from.
struct HeadOrder {
    int e1, e2, s0, s1, s2, place0, place1, place2;
    double i1, i2;
    __device__ __forceinline__ HeadOrder(const Orders& o, int h) {
        const int id = o.ids[h >> 2] >> 8 * (h & 3) & 255;
        e1 = o.extent[id][0], e2 = o.extent[id][1], s0 = o.stride[id][0], s1 = o.stride[id][1], s2 = o.stride[id][2];
        i1 = o.inv[id][0], i2 = o.inv[id][1];
        place0 = o.place[id][0], place1 = o.place[id][1], place2 = o.place[id][2];
    }
    // The coordinates along the order's axes of the image token at n_new; returns its position in default order.  Factors are below 2^24, or
    // are 2^24 (an extent or a stride of all tokens) beside a 0.
    __device__ __forceinline__ int source(int n_new, int& c0, int& c1, int& c2) const {
        const int q = quotient_of(n_new, i2);
        c2 = n_new - __umul24(q, e2);
        c0 = quotient_of(q, i1);
        c1 = q - __umul24(c0, e1);
        return __umul24(c0, s0) + __umul24(c1, s1) + __umul24(c2, s2);
    }
};

// Where a lane's angles lie in the table when its four pairs belong to one axis (Turning::fours).
struct LaneAxis {
    int place, pairs, base;  // base < 0: the lane's pairs do not turn
    __device__ __forceinline__ LaneAxis(const Turning& t, const HeadOrder& o, int L) {
        const int to1 = t.pairs[0], to2 = to1 + t.pairs[1], p0 = 4 * L, a = p0 < to1 ? 0 : p0 < to2 ? 1 : 2;
        place = pick(o.place0, o.place1, o.place2, a);
        pairs = pick(t.pairs[0], t.pairs[1], t.pairs[2], a);
        base = p0 >= t.total ? -1 : pick(t.base[0], t.base[1] - to1, t.base[2] - to2, a) + p0;
    }
};


// Where the rows of a workgroup's blocks come from, in LDS: position in default order and the coordinates along the order's axes (the first -1
// for a token that does not turn).  A row has 8 or 16 lanes; one thread finds its place for all of them.
constexpr int kSpan = 8;  // blocks per workgroup at most
template <int BLK>
struct Places {
    int4 row[kSpan * BLK];
    template <typename T>
    __device__ __forceinline__ void fill(const QuantArgs<T>& a, const Turning& t, const HeadOrder& order, int blk0, int blocks) {
        for (int i = threadIdx.x; i < blocks * BLK; i += kThreads) {
            const int n_new = blk0 * BLK + i;
            int4 p;
            p.x = order.source(min(n_new, t.n_img - 1), p.y, p.z, p.w);
            if (n_new >= t.n_img) p.x = min(n_new, a.n_tokens - 1), p.y = -1;
            row[i] = p;
        }
    }
};

// Weights and biases of a tensor as binary64 in LDS, of image and of text tokens: a row's lanes read those of their channels without a conversion and
// without registers that hold them.  Pair i of all lanes lies in one piece, so that a read of 16 bytes per lane meets no bank twice.
template <int D, bool HALVES>
struct Vectors {
    double v[2][2][D];  // [text][weight, bias][pair of a lane][lane][2]
    static constexpr int LANES = D / 8;
    __device__ __forceinline__ void fill(const Norms& norm, int z) {
#pragma unroll
        for (int j = 0; j < 4 * D / kThreads; ++j) {
            // a wavefront fills one vector (or half of one): which is a scalar, and so is its address
            const int which = __builtin_amdgcn_readfirstlane((threadIdx.x + j * kThreads) / D), c = threadIdx.x % D, bias = which & 1, text = which >> 1;
            const float* p = bias ? norm.b[z][text] : norm.w[z][text];
            const int L = HALVES ? c % (D / 2) / 4 : c / 8, e = HALVES ? c % 4 + (c >= D / 2 ? 4 : 0) : c % 8;
            v[text][bias][((e >> 1) * LANES + L) * 2 + (e & 1)] = p ? (double)p[c] : bias ? 0.0 : 1.0;
        }
    }
};
// A lane's eight of them.
template <int D>
struct LaneVector {
    const double* p;  // behind the lane's first two
    __device__ __forceinline__ double operator[](int e) const { return p[(e >> 1) * (D / 8) * 2 + (e & 1)]; }
};

// What a workgroup holds in LDS: for Q and K, and for V.
template <int BLK, int D, bool HALVES>
struct RowsLds {
    Places<BLK> places;
    Vectors<D, HALVES> vectors;
    float amax[2][kThreads / 64];
};
template <int BLK, int D, int BITS>
struct TransposedLds {
    Places<BLK> places;
    __attribute__((aligned(16))) uint8_t stage[stage_bytes<BITS, BLK, D>()];
    float amax[kThreads / 64];
};

// Q (z = 0) or K: one workgroup goes through `span` blocks of a head and reads a block while it works on the one before; the block stays in
// registers between the pass for the largest value and the codes.
//
// Bound by vector instructions with 8-bit codes (some 180 for the eight channels of a lane, V's among them; a third binary64), by HBM with bf16.
// 48 heads of 17550 bf16 tokens, d = 64, layer norms, out of one projection's output: 117 us with 8-bit codes (485 MB, 4.1 TB/s), 133 with bf16 (647 MB, 4.9 TB/s); one
// block per workgroup, no reading ahead, each row's place found by all of its lanes, weights in registers: 192 and 190.  Q and K in one
// workgroup, for their common places and angles: 116 registers in place of 90, 3 % slower.
template <typename T, int BLK, int D, int BITS, bool HALVES, bool FOURS>
__device__ __forceinline__ void quantize_rows(const QuantArgs<T>& a, const Turning& t, const Norms& norm, int z, uint8_t* lds) {
    constexpr int LANES = D / 8, ROWS = kThreads / LANES, IT = BLK / ROWS, OUT_BYTES = BLK * D * BITS / 8, WAVES = kThreads / 64;
    RowsLds<BLK, D, HALVES>& s = *(RowsLds<BLK, D, HALVES>*)lds;
    const int tid = threadIdx.x, L = tid % LANES, row = tid / LANES, bh = blockIdx.y, b = bh / a.nh, h = bh - b * a.nh;
    const int blk0 = blockIdx.x * a.span, blk1 = min(blk0 + a.span, a.kblocks);
    const HeadOrder order(a.orders, h);
    const LaneAxis axis(t, order, L);
    const T* const base = a.in[z].row(b, h, 0);
    const int stride = a.in[z].token;
    LaneRow<T, D, HALVES> next[IT];
    int next_at[IT];  // FOURS: where the row's angles lie in the table, < 0: it does not turn
    const auto read = [&](int blk) {
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int4 p = s.places.row[(blk - blk0) * BLK + it * ROWS + row];
            next[it].load(base + (int64_t)p.x * stride, L);
            if constexpr (FOURS) next_at[it] = (p.y | axis.base) >= 0 ? axis.base + (int)__umul24(pick(p.y, p.z, p.w, axis.place), axis.pairs) : -1;
        }
    };
    s.places.fill(a, t, order, blk0, blk1 - blk0);
    __syncthreads();
    read(blk0);
    s.vectors.fill(norm, z);
    __syncthreads();
    for (int blk = blk0; blk < blk1; ++blk) {
        LaneRow<T, D, HALVES> x[IT];
        LaneTurn turn[IT];
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            x[it] = next[it];
            LaneTurn& r = turn[it];
            if constexpr (FOURS) {
                r.turned = next_at[it] >= 0 ? 15 : 0;
                const float4* v = (const float4*)(t.table + 2 * (int64_t)max(next_at[it], 0));
                const float4 p = v[0], q = v[1];
                r.c[0] = p.x, r.s[0] = p.y, r.c[1] = p.z, r.s[1] = p.w, r.c[2] = q.x, r.s[2] = q.y, r.c[3] = q.z, r.s[3] = q.w;
            } else {
                const int4 p = s.places.row[(blk - blk0) * BLK + it * ROWS + row];
                if (p.y >= 0) load_turn(t, L, pick(p.y, p.z, p.w, order.place0), pick(p.y, p.z, p.w, order.place1), pick(p.y, p.z, p.w, order.place2), r);
                else r.none();
            }
        }
        if (blk + 1 < blk1) read(blk + 1);
        float y[IT][8], amax = 0.0f;
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            const int n_new = blk * BLK + it * ROWS + row;
            const double* v = s.vectors.v[n_new >= t.n_img][0] + 2 * L;
            normed_and_turned(x[it], a.kind, norm.eps, LaneVector<D>{v}, LaneVector<D>{v + D}, turn[it], y[it]);
            if (n_new >= a.n_tokens) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[it][e] = 0.0f;
            }
        }
        bool nans = false;
        if constexpr (BITS != 16) {
            amax = lane_max<true>(y);
            nans = __any(amax != amax);
            if (nans) amax = lane_max<false>(y);
            amax = wavefront_max(amax);
            float* meet = s.amax[blk & 1];  // of two in turn: this one was read before the last block's barrier
            if ((tid & 63) == 0) meet[tid >> 6] = amax;
            __syncthreads();
#pragma unroll
            for (int wave = 0; wave < WAVES; ++wave) amax = fmaxf(amax, meet[wave]);
            amax = uniform(amax);
        }
        const size_t group = (size_t)bh * a.kblocks + blk;
        const GroupQuotient<BITS> quotient(amax, nans);
        if (tid == 0) a.scales[z][group] = quotient.scale;
        uint8_t* out = a.codes[z] + group * OUT_BYTES;
#pragma unroll
        for (int it = 0; it < IT; ++it) store_codes<BITS, D, HALVES>(out + (it * ROWS + row) * (D * BITS / 8), L, y[it], quotient);
    }
}

// V: a block's codes are transposed through LDS.
template <typename T, int BLK, int D, int BITS>
__device__ __forceinline__ void quantize_transposed(const QuantArgs<T>& a, const Turning& t, uint8_t* lds) {
    constexpr int LANES = D / 8, ROWS = kThreads / LANES, IT = BLK / ROWS, OUT_BYTES = BLK * D * BITS / 8, WAVES = kThreads / 64;
    TransposedLds<BLK, D, BITS>& s = *(TransposedLds<BLK, D, BITS>*)lds;
    const int tid = threadIdx.x, L = tid % LANES, row = tid / LANES, bh = blockIdx.y, b = bh / a.nh, h = bh - b * a.nh;
    const int blk0 = blockIdx.x * a.span, blk1 = min(blk0 + a.span, a.kblocks);
    const HeadOrder order(a.orders, h);
    const T* const base = a.in[2].row(b, h, 0);
    const int stride = a.in[2].token;
    LaneRow<T, D, false> next[IT];
    const auto read = [&](int blk) {
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            next[it].load(base + (int64_t)s.places.row[(blk - blk0) * BLK + it * ROWS + row].x * stride, L);
            if (blk * BLK + it * ROWS + row >= a.n_tokens) next[it].zero();
        }
    };
    s.places.fill(a, t, order, blk0, blk1 - blk0);
    __syncthreads();
    read(blk0);
    for (int blk = blk0; blk < blk1; ++blk) {
        float y[IT][8], amax = 0.0f;
        bool nans = false;
#pragma unroll
        for (int it = 0; it < IT; ++it)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[it][e] = next[it][e];
        if (blk + 1 < blk1) read(blk + 1);
        if constexpr (BITS != 16) {
            amax = lane_max<true>(y);
            nans = __any(amax != amax);
            if (nans) amax = lane_max<false>(y);
            amax = wavefront_max(amax);
            if ((tid & 63) == 0) s.amax[tid >> 6] = amax;
        }
        __syncthreads();  // also: the block before has left the staged tile
        if constexpr (BITS != 16) {
#pragma unroll
            for (int wave = 0; wave < WAVES; ++wave) amax = fmaxf(amax, s.amax[wave]);
            amax = uniform(amax);
        }
        const size_t group = (size_t)bh * a.kblocks + blk;
        const GroupQuotient<BITS> quotient(amax, nans);
        if (tid == 0) a.scales[2][group] = quotient.scale;
#pragma unroll
        for (int it = 0; it < IT; ++it) stage_codes<BITS, BLK, D, false>(s.stage, it * ROWS + row, L, y[it], quotient);
        __syncthreads();
        store_staged<BITS, BLK, D>(a.codes[2] + group * OUT_BYTES, s.stage, tid);
    }
}

// grid: spans of blocks; batches x heads; Q, K, V
template <typename T, int BLK, int D, int QKBITS, int PVBITS, bool HALVES, bool FOURS>
__global__ __launch_bounds__(kThreads) void norm_rope_quantize_kernel(QuantArgs<T> a, Turning t, Norms norm) {
    constexpr size_t rows = sizeof(RowsLds<BLK, D, HALVES>), transposed = sizeof(TransposedLds<BLK, D, PVBITS>);
    __shared__ __attribute__((aligned(16))) uint8_t lds[rows > transposed ? rows : transposed];
    if (blockIdx.z < 2) quantize_rows<T, BLK, D, QKBITS, HALVES, FOURS>(a, t, norm, blockIdx.z, lds);
    else quantize_transposed<T, BLK, D, PVBITS>(a, t, lds);
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
        if (i == 2 && stride[i] > INT32_MAX) return fail(PARO_EUNSUPPORTED, "%s: a token stride of %lld elements exceeds 2^31", what, (long long)stride[i]);
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
    t->table = table;
    t->fours = t->total > 0;  // kernels may read four entries for a lane that does not turn
    const int extent[3] = {s->F, s->Hg, s->Wg};
    int64_t at = 0;
    for (int a = 0; a < 3; ++a) {
        t->pairs[a] = axes->dims[a] / 2;
        t->fours = t->fours && t->pairs[a] % 4 == 0;
        t->base[a] = (int)at;
        at += (int64_t)extent[a] * t->pairs[a];
    }
    t->n_img = s->F * s->Hg * s->Wg;
    t->Hg = s->Hg;
    t->Wg = s->Wg;
    t->inv_hg = 1.0 / s->Hg;
    t->inv_wg = 1.0 / s->Wg;
    t->sign = back ? -1.0f : 1.0f;
    return PARO_OK;
}

static int make_norms(const paro_qk_norm* norm, Norms* out) {
    if (!norm) return fail(PARO_EINVAL, "norm is NULL");
    if (norm->kind != PARO_NORM_NONE && norm->kind != PARO_NORM_RMS && norm->kind != PARO_NORM_LAYER)
        return fail(PARO_EINVAL, "norm kind=%d is not a paro_norm_kind", (int)norm->kind);
    if (norm->kind != PARO_NORM_NONE && !(norm->eps >= 0.0 && norm->eps < INFINITY)) return fail(PARO_EINVAL, "eps=%g must be finite and >= 0", norm->eps);
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
static Rows<T> rows_of(const paro_strided* r) { return {(T*)r->data, r->batch, r->head, (int)r->token}; }

// Heads that a workgroup goes through: so few that there are `least` workgroups (below that a launch lasts as long as a workgroup), and
// not more than three while there are fewer than `enough`.
static int heads_per_group(const paro_shape* s, int64_t tiles, int tensors, int least, int enough) {
    int heads = s->nh;
    const auto workgroups = [&] { return tiles * tensors * s->B * ((s->nh + heads - 1) / heads); };
    while (heads > 1 && workgroups() < least) heads = (heads + 1) / 2;
    while (heads > 3 && workgroups() < enough) heads = (heads + 1) / 2;
    return heads;
}

// Forward: four workgroups for each compute unit before anything else.  With fewer heads a workgroup's angles and weights cost more than
// its rows (24 heads of 4608 tokens, d = 128, rotation: one head 15.1 us, three 11.9, six 11.5), with more a launch ends unevenly (48
// heads of 17550 tokens, d = 64, rotation: three 44.8, six 46.2, twelve 49.8; Q and K with root-mean-square norms six 86.8, twelve 88.0, 24
// 90.6; with layer norms, which hold more per lane, in the form of the day six 93.8, twelve 91.5, 24 94.6).
static int forward_heads(const paro_shape* s, int64_t tiles, int tensors, int kind) {
    return heads_per_group(s, tiles, tensors, 1024, kind == PARO_NORM_LAYER ? 4096 : 8192);
}

static int tile_tokens(const paro_shape* s) { return kThreads / (s->d / 8); }

static int check_dtype(paro_dtype dtype) {
    if (dtype != PARO_F32 && dtype != PARO_BF16) return fail(PARO_EINVAL, "dtype=%d is not a paro_dtype", (int)dtype);
    return PARO_OK;
}

// f(T, D, KIND, HALVES) of a call, as compile-time constants.
template <typename F>
static void with_kernel(const paro_shape* s, paro_dtype dtype, int kind, int pairs, F&& f) {
    auto of_pairs = [&](auto t, auto d, auto k) {
        if (pairs == PARO_PAIRS_HALVES) f(t, d, k, std::true_type());
        else f(t, d, k, std::false_type());
    };
    auto of_kind = [&](auto t, auto d) {
        if (kind == PARO_NORM_NONE) of_pairs(t, d, std::integral_constant<int, PARO_NORM_NONE>());
        else if (kind == PARO_NORM_RMS) of_pairs(t, d, std::integral_constant<int, PARO_NORM_RMS>());
        else of_pairs(t, d, std::integral_constant<int, PARO_NORM_LAYER>());
    };
    auto of_d = [&](auto t) {
        if (s->d == 64) of_kind(t, std::integral_constant<int, 64>());
        else of_kind(t, std::integral_constant<int, 128>());
    };
    if (dtype == PARO_F32) of_d(float());
    else of_d(uint16_t());
}

static void launch_forward(const paro_shape* s, int64_t n, paro_dtype dtype, int kind, int pairs, int tensors, const paro_strided* const (&in)[2],
                           const paro_strided* const (&out)[2], const Turning& t, const Norms& norm, hipStream_t st) {
    const int64_t tiles = (n + tile_tokens(s) - 1) / tile_tokens(s);
    const int heads = forward_heads(s, tiles, tensors, kind);
    const dim3 grid((unsigned)tiles, (unsigned)(s->B * ((s->nh + heads - 1) / heads)), (unsigned)tensors);
    with_kernel(s, dtype, kind, pairs, [&](auto t0, auto d, auto k, auto halves) {
        typedef decltype(t0) T;
        RowsArgs<T> a;
        memset(&a, 0, sizeof(a));
        for (int i = 0; i < tensors; ++i) {
            a.in[i] = rows_of<const T>(in[i]);
            a.out[i] = rows_of<T>(out[i]);
        }
        a.n_tokens = (int)n;
        a.nh = s->nh;
        a.heads = heads;
        hipLaunchKernelGGL((rotate_rows_kernel<T, d(), k(), halves()>), grid, dim3(kThreads), 0, st, a, t, norm);
    });
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
    // fewer workgroups than forward: each leaves partial sums (12 fp32 heads of 1955 tokens: at least 256 workgroups 12.9 us, 1024 16.1;
    // 24 bf16 heads of 4608, d = 128: 1024 38.4, 2048 39.5; 48 of 17550, d = 64: the same within 2 %)
    g.heads = heads_per_group(s, g.tiles, 2, 256, 1024);
    g.groups = (s->nh + g.heads - 1) / g.heads;
    return g;
}

static void launch_grad(const paro_shape* s, int64_t n, paro_dtype dtype, int kind, int pairs, const GradSplit& split, const paro_strided* const (&x)[2],
                        const paro_strided* const (&dy)[2], const paro_strided* const (&dx)[2], float* partial, const Turning& t, const Norms& norm,
                        hipStream_t st) {
    const dim3 grid((unsigned)split.tiles, (unsigned)(s->B * split.groups), 2);
    with_kernel(s, dtype, kind, pairs, [&](auto t0, auto d, auto k, auto halves) {
        typedef decltype(t0) T;
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
        hipLaunchKernelGGL((norm_rope_grad_kernel<T, d(), k(), halves()>), grid, dim3(kThreads), 0, st, a, t, norm);
    });
}

template <typename T, int BLK, int D, bool HALVES, bool FOURS>
static bool launch_quant_bits(int bits_qk, int bits_pv, dim3 grid, hipStream_t st, const QuantArgs<T>& a, const Turning& t, const Norms& norm) {
#define PARO_QKV_CASE(QK, PV)                                                                                                             \
    if (bits_qk == QK && bits_pv == PV) {                                                                                                 \
        hipLaunchKernelGGL((norm_rope_quantize_kernel<T, BLK, D, QK, PV, HALVES, FOURS>), grid, dim3(kThreads), 0, st, a, t, norm); \
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

template <typename T, bool HALVES, bool FOURS>
static bool launch_quant(const paro_shape* s, int bits_qk, int bits_pv, dim3 grid, hipStream_t st, const QuantArgs<T>& a, const Turning& t, const Norms& norm) {
    if (s->block == 64 && s->d == 64) return launch_quant_bits<T, 64, 64, HALVES, FOURS>(bits_qk, bits_pv, grid, st, a, t, norm);
    if (s->block == 64) return launch_quant_bits<T, 64, 128, HALVES, FOURS>(bits_qk, bits_pv, grid, st, a, t, norm);
    if (s->d == 64) return launch_quant_bits<T, 32, 64, HALVES, FOURS>(bits_qk, bits_pv, grid, st, a, t, norm);
    return launch_quant_bits<T, 32, 128, HALVES, FOURS>(bits_qk, bits_pv, grid, st, a, t, norm);
}

template <typename T>
static int quantize_entry(const paro_shape* s, int64_t n, int64_t kb, int kind, int pairs, int bits_qk, int bits_pv, const uint8_t* h_perm_ids, const paro_strided* const (&in)[3],
                          void* const (&codes)[3], float* const (&scales)[3], const Turning& t, const Norms& norm, hipStream_t st) {
    QuantArgs<T> a;
    ReorderTable table;
    if (int e = make_reorder_table(s, h_perm_ids, &table)) return e;
    memset(&a.orders, 0, sizeof(a.orders));
    for (int h = 0; h < s->nh; ++h) a.orders.ids[h >> 2] |= (uint32_t)table.perm[h] << 8 * (h & 3);
    for (int p = 0; p < 6; ++p) {
        for (int i = 0; i < 2; ++i) {
            a.orders.extent[p][i] = table.fwd[p][i];
            a.orders.inv[p][i] = 1.0 / table.fwd[p][i];
        }
        for (int i = 0; i < 3; ++i) {
            a.orders.stride[p][i] = table.fwd[p][2 + i];
            a.orders.place[p][axis_order(p).a[i]] = i;
        }
    }
    for (int i = 0; i < 3; ++i) {
        a.in[i] = rows_of<const T>(in[i]);
        a.codes[i] = (uint8_t*)codes[i];
        a.scales[i] = scales[i];
    }
    a.n_tokens = (int)n;
    a.kblocks = (int)kb;
    a.nh = s->nh;
    a.kind = kind;
    // As many blocks per workgroup as leave 2048 workgroups, eight for each compute unit: what a workgroup sets up is shared and all but its first
    // block is read ahead (48 heads of 275 blocks, 8 bit: one block 182 us, two 160, eight 145 with an earlier form; 24 heads of 72, d = 128: with 4096
    // workgroups 37.3, 2048 36.0, 1024 36.7).
    a.span = 1;
    while (a.span < kSpan && 3 * (int64_t)s->B * s->nh * ((kb + a.span) / (a.span + 1)) >= 2048) ++a.span;
    const auto run = pairs == PARO_PAIRS_HALVES ? (t.fours ? launch_quant<T, true, true> : launch_quant<T, true, false>)
                                                : (t.fours ? launch_quant<T, false, true> : launch_quant<T, false, false>);
    if (!run(s, bits_qk, bits_pv, dim3((unsigned)((kb + a.span - 1) / a.span), (unsigned)(s->B * s->nh), 3), st, a, t, norm))
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
    launch_forward(s, n, dtype, PARO_NORM_NONE, axes->pairs, 1, {x, nullptr}, {y, nullptr}, t, none, (hipStream_t)stream);
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
    launch_forward(s, n, dtype, norm->kind, axes->pairs, 2, {q, k}, {q_out, k_out}, t, norms, (hipStream_t)stream);
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
    launch_grad(s, n, dtype, norm->kind, axes->pairs, split, x, dy, dx, partial, t, norms, st);
    if (int e = check_launch("paro_qk_norm_rope_backward")) return e;
    if (count) {
        if (s->d == 64) hipLaunchKernelGGL((norm_grad_kernel<64>), dim3(count, 4), dim3(1024), 0, st, partial, slots, jobs);
        else hipLaunchKernelGGL((norm_grad_kernel<128>), dim3(count, 8), dim3(1024), 0, st, partial, slots, jobs);
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
    if (dtype == PARO_F32) return quantize_entry<float>(s, n, kb, norm->kind, axes->pairs, bits_qk, bits_pv, h_perm_ids, in, codes, scales, t, norms, st);
    return quantize_entry<uint16_t>(s, n, kb, norm->kind, axes->pairs, bits_qk, bits_pv, h_perm_ids, in, codes, scales, t, norms, st);
}
