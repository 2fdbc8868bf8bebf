// norm.hip -- root-mean-square norm of the residual stream (forward with the
// residual's addition and an optional 8-bit output, backward) and the 8-bit
// row quantiser.
//
//   s = x + r,  rho = (mean s^2 + eps)^(-1/2),  y_j = s_j rho w_j
//   dx_j = rho (w_j dy_j - s_j rho^2 mean(w dy s)) + ds_j,  dw_j = sum_rows dy_j s_j rho
//
// Everything here is bound by memory: about ten operations for 4 to 8 bytes.
// A row is read once, stays in the registers of the threads that share it
// (a wave, or a workgroup of 2 to 8 waves) and is written once; its sums are the only exchange.  Workgroups walk the rows
// with a fixed stride, so the weight is read once a workgroup and the weight
// gradient is summed in registers, left as one partial row a workgroup and
// added up by a second launch in a fixed order (no atomics).
#include <float.h>

#include "common.hpp"
#include "elsaa.h"
#include "internal.hpp"

namespace elsaa {
namespace {

constexpr int kMaxCols = 16384;

// V consecutive elements of the storage type: as loaded, as float32, stored.
template <class T, int V> struct Piece;
template <> struct Piece<BF16, 8> {
    using raw = uint4;
    __device__ static __forceinline__ raw ld(const uint16_t* p) { return *(const uint4*)p; }
    __device__ static __forceinline__ void val(raw v, float* x)
    {
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
    __device__ static __forceinline__ void st(uint16_t* p, const float* x)
    {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = (uint32_t)f32_to_bf16(x[2 * i]) | ((uint32_t)f32_to_bf16(x[2 * i + 1]) << 16);
        *(uint4*)p = make_uint4(u[0], u[1], u[2], u[3]);
    }
};
template <> struct Piece<F32, 4> {
    using raw = f32x4;
    __device__ static __forceinline__ raw ld(const float* p) { return *(const f32x4*)p; }
    __device__ static __forceinline__ void val(raw v, float* x)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[i];
    }
    __device__ static __forceinline__ void st(float* p, const float* x) { *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]}; }
};
template <class T> struct Piece<T, 1> {
    using raw = typename T::store_t;
    __device__ static __forceinline__ raw ld(const raw* p) { return *p; }
    __device__ static __forceinline__ void val(raw v, float* x) { x[0] = T::load(v); }
    __device__ static __forceinline__ void st(raw* p, const float* x) { *p = T::store(x[0]); }
};

// V 8-bit values in one store.
template <int V>
__device__ __forceinline__ void store_i8(int8_t* p, const int (&q)[V])
{
    if constexpr (V == 1) {
        *p = (int8_t)q[0];
    } else {
        uint32_t u[V / 4];
#pragma unroll
        for (int i = 0; i < V / 4; ++i)
            u[i] = (q[4 * i] & 255) | ((q[4 * i + 1] & 255) << 8) | ((q[4 * i + 2] & 255) << 16) | ((uint32_t)q[4 * i + 3] << 24);
        if constexpr (V == 4) *(uint32_t*)p = u[0];
        else *(uint2*)p = make_uint2(u[0], u[1]);
    }
}

__device__ __forceinline__ float wave_sum(float v) { return wave_sum16(row_sum16(v)); }

__device__ __forceinline__ uint32_t wave_umax(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x128, 0xf, 0xf, true));   // row_ror:8, 4, 2, 1
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x124, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x122, 0xf, 0xf, true));
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x121, 0xf, 0xf, true));
    const LanePair a = xpair16(__uint_as_float(v));
    v = max(__float_as_uint(a.lo), __float_as_uint(a.hi));
    const LanePair b = xpair32(__uint_as_float(v));
    return max(__float_as_uint(b.lo), __float_as_uint(b.hi));
}

// The TPR threads that share a row (a wave, or the whole workgroup) add up
// one or two values, or take a largest one.  `red` holds two sets of slots,
// used in turn by the calls of a row, so one barrier a call is enough: a
// wave writes a set again only behind a barrier that every wave reached after
// reading it.
template <int TPR>
struct Row {
    static constexpr int W = TPR / 64;
    float (*red)[2 * W];
    int set = 0;
    __device__ __forceinline__ void sum2(float& a, float& b)
    {
        a = wave_sum(a);
        b = wave_sum(b);
        if constexpr (W > 1) {
            float* s = red[set];
            set ^= 1;
            const int w = threadIdx.x >> 6;
            if ((threadIdx.x & 63) == 0) {
                s[w] = a;
                s[W + w] = b;
            }
            __syncthreads();
            a = b = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                a += s[i];
                b += s[W + i];
            }
        }
    }
    __device__ __forceinline__ float sum(float a)
    {
        a = wave_sum(a);
        if constexpr (W > 1) {
            float* s = red[set];
            set ^= 1;
            if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = a;
            __syncthreads();
            a = 0;
#pragma unroll
            for (int i = 0; i < W; ++i) a += s[i];
        }
        return a;
    }
    __device__ __forceinline__ uint32_t umax(uint32_t v)
    {
        v = wave_umax(v);
        if constexpr (W > 1) {
            float* s = red[set];
            set ^= 1;
            if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = __uint_as_float(v);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < W; ++i) v = max(v, __float_as_uint(s[i]));
        }
        return v;
    }
};

// 8-bit values of a row held E a thread, y[], largest |y| at `top` (as bits,
// which order like the values; infinities and NaN come last).  The quotient
// 127 y / top is formed as y c times 1 / (top f) with one correction, so a value
// halfway between two steps (which 127 y, exact for bfloat16 y, can be) comes
// out halfway and goes to the even step.  f is 1 for rows between 2^-64 and 2^64, 2^64 below (whose
// reciprocal would overflow) and 2^-64 above (where 127 y would, from 2.68e36 on, and
// the reciprocal would be subnormal); what the latter makes subnormal is far below half a step.
struct Quant {
    float c, inv, top, scale;
    __device__ __forceinline__ explicit Quant(uint32_t bits)
    {
        const bool ok = bits < 0x7f800000u;
        const float t = ok ? __uint_as_float(bits) : 0.f;
        const float f = t < 0x1p-64f ? 0x1p64f : t > 0x1p64f ? 0x1p-64f : 1.f;
        c = 127.f * f;
        top = t * f;
        inv = t > 0.f ? 1.f / top : 0.f;
        scale = ok ? t / 127.f : __uint_as_float(0x7fc00000u);
    }
    __device__ __forceinline__ int operator()(float y) const
    {
        const float n = y * c;
        float q = n * inv;
        q = fmaf(fmaf(-q, top, n), inv, q);
        return inv > 0.f ? (int)rintf(q) : 0;      // (a row with an infinity or NaN: 0)
    }
};

struct NormArgs {
    const void *x, *r, *dy;
    const float* w;
    void *s, *y;
    float* scale;
    float* part;         // backward: [blocks][cols] partial weight gradients, or null
    int64_t rows, ldx, ldr, lds, ldy;
    int cols;
    float eps;
};

template <class T, int V, int E, int TPR, bool I8>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void rms_norm_fwd_kernel(NormArgs a)
{
    using S = typename T::store_t;
    using P = Piece<T, V>;
    constexpr int NC = E / V, NT = TPR == 64 ? 256 : TPR, RPB = NT / TPR;
    __shared__ float red[2][2 * (TPR / 64)];
    Row<TPR> row{red};
    const int t = threadIdx.x % TPR;
    float w[E];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = (c * TPR + t) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) w[c * V + i] = col < a.cols ? a.w[col + i] : 0.f;
    }
    const float mean = 1.f / (float)a.cols;
    // (whole waves share a row, so this loop is uniform in a wave, and in the
    // workgroup where the workgroup shares one)
    for (int64_t rw = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; rw < a.rows; rw += (int64_t)gridDim.x * RPB) {
        const S* x = (const S*)a.x + rw * a.ldx;
        typename P::raw xr[NC], rr[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * TPR + t) * V;
            xr[c] = typename P::raw{};
            rr[c] = typename P::raw{};
            if (col < a.cols) {
                xr[c] = P::ld(x + col);
                if (a.r) rr[c] = P::ld((const S*)a.r + rw * a.ldr + col);
            }
        }
        float s[E], ss = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float rv[V];
            P::val(xr[c], &s[c * V]);
            P::val(rr[c], rv);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[c * V + i] += a.r ? rv[i] : 0.f;
                ss = fmaf(s[c * V + i], s[c * V + i], ss);
            }
        }
        if (a.s) {
            S* so = (S*)a.s + rw * a.lds;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = (c * TPR + t) * V;
                if (col < a.cols) P::st(so + col, &s[c * V]);
            }
        }
        ss = row.sum(ss);
        const float rho = 1.f / sqrtf(fmaf(ss, mean, a.eps));
        if constexpr (!I8) {
            S* y = (S*)a.y + rw * a.ldy;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = (c * TPR + t) * V;
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = s[c * V + i] * rho * w[c * V + i];
                if (col < a.cols) P::st(y + col, o);
            }
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                // (a thread's places behind the last column hold 0 * 0)
                s[e] = s[e] * rho * w[e];
                const bool in = ((e / V) * TPR + t) * V < a.cols;
                top = max(top, in ? __float_as_uint(s[e]) & 0x7fffffffu : 0u);
            }
            const Quant qz(row.umax(top));
            int8_t* y = (int8_t*)a.y + rw * a.ldy;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = (c * TPR + t) * V;
                int q[V];
#pragma unroll
                for (int i = 0; i < V; ++i) q[i] = qz(s[c * V + i]);
                if (col < a.cols) store_i8<V>(y + col, q);
            }
            if (t == 0) a.scale[rw] = qz.scale;
        }
    }
}

template <class T, int V, int E, int TPR>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void rms_norm_bwd_kernel(NormArgs a)
{
    using S = typename T::store_t;
    using P = Piece<T, V>;
    constexpr int NC = E / V, NT = TPR == 64 ? 256 : TPR, RPB = NT / TPR;
    __shared__ float red[2][2 * (TPR / 64)];
    __shared__ float acc[RPB > 1 ? E * TPR : 1];
    Row<TPR> row{red};
    const int t = threadIdx.x % TPR;
    float w[E], dw[E];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = (c * TPR + t) * V;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            w[c * V + i] = col < a.cols ? a.w[col + i] : 0.f;
            dw[c * V + i] = 0.f;
        }
    }
    const float mean = 1.f / (float)a.cols;
    for (int64_t rw = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; rw < a.rows; rw += (int64_t)gridDim.x * RPB) {
        typename P::raw xr[NC], gr[NC], rr[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * TPR + t) * V;
            xr[c] = gr[c] = rr[c] = typename P::raw{};
            if (col < a.cols) {
                xr[c] = P::ld((const S*)a.x + rw * a.ldx + col);
                gr[c] = P::ld((const S*)a.dy + rw * a.ldy + col);
                if (a.r) rr[c] = P::ld((const S*)a.r + rw * a.ldr + col);
            }
        }
        float ss = 0.f, ps = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float s[V], g[V];
            P::val(xr[c], s);
            P::val(gr[c], g);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                ss = fmaf(s[i], s[i], ss);
                ps = fmaf(w[c * V + i] * g[i], s[i], ps);
            }
        }
        row.sum2(ss, ps);
        const float rho = 1.f / sqrtf(fmaf(ss, mean, a.eps));
        const float k = rho * (rho * (ps * mean));      // (rho^2 alone passes float32's range where eps is below 3e-39)
        S* dx = (S*)a.s + rw * a.lds;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * TPR + t) * V;
            float s[V], g[V], r[V];
            P::val(xr[c], s);
            P::val(gr[c], g);
            P::val(rr[c], r);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                dw[c * V + i] = fmaf(g[i], s[i] * rho, dw[c * V + i]);
                const float d = rho * (w[c * V + i] * g[i] - s[i] * k);
                s[i] = a.r ? d + r[i] : d;
            }
            if (col < a.cols) P::st(dx + col, s);
        }
    }
    if (!a.part) return;
    float* out = a.part + (int64_t)blockIdx.x * a.cols;
    if constexpr (RPB > 1) {
        // the waves' sums, added in wave order
        for (int v = 0; v < RPB; ++v) {
            if ((int)threadIdx.x / TPR == v) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if (v) dw[e] += acc[e * TPR + t];
                    acc[e * TPR + t] = dw[e];
                }
            }
            __syncthreads();
        }
        if ((int)threadIdx.x / TPR != RPB - 1) return;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = (c * TPR + t) * V;
        if (col < a.cols) {
#pragma unroll
            for (int i = 0; i < V; ++i) out[col + i] = dw[c * V + i];
        }
    }
}

// dw[c] = sum of the partial rows: 16 groups of rows a column, then the groups.
__global__ __launch_bounds__(1024) void rms_norm_dw_kernel(const float* part, float* dw, int cols, int parts)
{
    __shared__ float acc[16][64];
    const int col = blockIdx.x * 64 + (threadIdx.x & 63), grp = threadIdx.x >> 6;
    float v = 0.f;
    if (col < cols) {
#pragma unroll 8
        for (int p = grp; p < parts; p += 16) v += part[(int64_t)p * cols + col];
    }
    acc[grp][threadIdx.x & 63] = v;
    __syncthreads();
    if (grp == 0 && col < cols) {
        v = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) v += acc[i][threadIdx.x & 63];
        dw[col] = v;
    }
}

struct QuantArgs {
    const void* x;
    int8_t* q;
    float* scale;
    int64_t rows, ld, ldq;
    int cols, heads, seq, dh_shift;
};

template <class T, int V, int E, int TPR>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void quantize_rows_kernel(QuantArgs a)
{
    using S = typename T::store_t;
    using P = Piece<T, V>;
    constexpr int NC = E / V, NT = TPR == 64 ? 256 : TPR, RPB = NT / TPR;
    __shared__ float red[2][2 * (TPR / 64)];
    Row<TPR> row{red};
    const int t = threadIdx.x % TPR;
    for (int64_t rw = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; rw < a.rows; rw += (int64_t)gridDim.x * RPB) {
        // element of column 0, and of column c behind it (a piece lies in one head)
        int64_t base, plane = 0;
        if (a.heads) {
            const int64_t b = rw / a.seq;
            base = (b * (a.heads - 1) * a.seq + rw) << a.dh_shift;
            plane = (int64_t)(a.seq - 1) << a.dh_shift;
        } else {
            base = rw * a.ld;
        }
        typename P::raw xr[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * TPR + t) * V;
            xr[c] = typename P::raw{};
            if (col < a.cols) xr[c] = P::ld((const S*)a.x + base + (a.heads ? (col >> a.dh_shift) * plane : 0) + col);
        }
        float s[E];
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            P::val(xr[c], &s[c * V]);
#pragma unroll
            for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(s[c * V + i]) & 0x7fffffffu);
        }
        const Quant qz(row.umax(top));
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (c * TPR + t) * V;
            int q[V];
#pragma unroll
            for (int i = 0; i < V; ++i) q[i] = qz(s[c * V + i]);
            if (col < a.cols) store_i8<V>(a.q + rw * a.ldq + col, q);
        }
        if (t == 0) a.scale[rw] = qz.scale;
    }
}

// Threads a row and values a thread.
struct Fit {
    int tpr, e;
    int rows() const { return tpr == 64 ? 4 : 1; }                 // a workgroup
    int waves() const { return tpr == 64 ? 4 : tpr / 64; }
};
// The norm: eight values (one 16-byte piece in bfloat16) a thread as long as 256
// threads reach, so that reads, sums and writes of many rows overlap on a
// compute unit: 4096 rows of 2048 in 16.3 us with four waves a row against
// 23.6 with one (32 values a thread), 32768 rows 98 against 101.
Fit norm_fit(int cols)
{
    if (cols <= 64 * 8) return {64, 8};
    if (cols <= 128 * 8) return {128, 8};
    if (cols <= 256 * 8) return {256, 8};
    if (cols <= 256 * 16) return {256, 16};
    if (cols <= 256 * 32) return {256, 32};
    return {512, 32};
}
// The quantiser has no weight to read and one sum less: a wave a row up to
// 2048 columns (32768 rows of 2048 in 38 us, with four waves 42).
Fit quant_fit(int cols)
{
    if (cols <= 64 * 8) return {64, 8};
    if (cols <= 64 * 16) return {64, 16};
    if (cols <= 64 * 32) return {64, 32};
    if (cols <= 256 * 16) return {256, 16};
    if (cols <= 256 * 32) return {256, 32};
    return {512, 32};
}

// Workgroups of a pass over the rows, about `waves` waves: a workgroup walks
// several rows and reads the weight once (a workgroup for each four rows of 2048
// took 145 us where 101 do: the float32 weight is as many bytes as x and r).
int64_t blocks_of(int64_t rows, const Fit& f, int waves)
{
    const int64_t need = (rows + f.rows() - 1) / f.rows(), most = waves / f.waves();
    return need < most ? need : most;
}
constexpr int kNormWaves = 4096, kBwdWaves = 2048, kQuantWaves = 8192;
// The backward leaves a partial row a workgroup for the sum over them (32768 rows
// of 1024: 57 us with 2048 waves, 84 with half and 62 with twice as many).
int64_t bwd_blocks(int64_t rows, int cols)
{
    const Fit f = norm_fit(cols);
    return blocks_of(rows, f, kBwdWaves);
}

bool aligned(const void* p, int n) { return ((uintptr_t)p & (n - 1)) == 0; }
// (multiples of 8 elements; 8-bit buffers in pieces of 8 bytes)
bool vec_ok(const void* p, int64_t ld, bool i8 = false) { return !p || (aligned(p, i8 ? 8 : 16) && ld % 8 == 0); }

int check_norm(const elsaa_norm_desc* d)
{
    if (!d) return api_fail(ELSAA_ERR_INVALID_ARG, "desc is NULL");
    if (d->rows < 1 || d->cols < 1)
        return api_fail(ELSAA_ERR_INVALID_ARG, "rows and cols must be >= 1 (got %lld, %d)", (long long)d->rows, d->cols);
    if (d->cols > kMaxCols) return api_fail(ELSAA_ERR_UNSUPPORTED, "cols must be <= %d (got %d)", kMaxCols, d->cols);
    if (d->dtype != ELSAA_F32 && d->dtype != ELSAA_BF16) return api_fail(ELSAA_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
    if (!(d->eps > 0.f)) return api_fail(ELSAA_ERR_INVALID_ARG, "eps must be > 0");
    return ELSAA_OK;
}

// a buffer of rows: aligned to its element, with room for a row
int check_rows(const char* name, const void* p, int64_t ld, int cols, int elem)
{
    if (!aligned(p, elem)) return api_fail(ELSAA_ERR_INVALID_ARG, "%s must be aligned to its element", name);
    if (ld < cols) return api_fail(ELSAA_ERR_INVALID_ARG, "%s: row stride %lld is below %d columns", name, (long long)ld, cols);
    return ELSAA_OK;
}

// an output at an input's address: its rows must be the input's
int check_in_place(const char* name, const void* out, int64_t ldo, const void* in, int64_t ldi, int64_t rows)
{
    if (out && out == in && ldo != ldi && rows > 1)
        return api_fail(ELSAA_ERR_INVALID_ARG, "%s is written over an input with another row stride (%lld, %lld)", name, (long long)ldo,
                        (long long)ldi);
    return ELSAA_OK;
}

template <class T, int V>
void launch_fwd(const NormArgs& a, bool i8, hipStream_t st)
{
    const Fit f = norm_fit(a.cols);
    const dim3 grid((unsigned)blocks_of(a.rows, f, kNormWaves)), block(64 * f.waves());
#define GO(E, TPR)                                                                                                  \
    if (f.e == E && f.tpr == TPR) {                                                                                 \
        if (i8) ELSAA_LAUNCH("rms_norm_i8", (rms_norm_fwd_kernel<T, V, E, TPR, true>), grid, block, 0, st, a);      \
        else ELSAA_LAUNCH("rms_norm_fwd", (rms_norm_fwd_kernel<T, V, E, TPR, false>), grid, block, 0, st, a);       \
    }
    GO(8, 64) GO(8, 128) GO(8, 256) GO(16, 256) GO(32, 256) GO(32, 512)
#undef GO
}
template <class T, int V>
void launch_bwd(const NormArgs& a, hipStream_t st)
{
    const Fit f = norm_fit(a.cols);
    const dim3 grid((unsigned)bwd_blocks(a.rows, a.cols)), block(64 * f.waves());
#define GO(E, TPR) \
    if (f.e == E && f.tpr == TPR) ELSAA_LAUNCH("rms_norm_bwd", (rms_norm_bwd_kernel<T, V, E, TPR>), grid, block, 0, st, a);
    GO(8, 64) GO(8, 128) GO(8, 256) GO(16, 256) GO(32, 256) GO(32, 512)
#undef GO
}
template <class T, int V>
void launch_quant(const QuantArgs& a, hipStream_t st)
{
    const Fit f = quant_fit(a.cols);
    const dim3 grid((unsigned)blocks_of(a.rows, f, kQuantWaves)), block(64 * f.waves());
#define GO(E, TPR) \
    if (f.e == E && f.tpr == TPR) ELSAA_LAUNCH("quantize_rows", (quantize_rows_kernel<T, V, E, TPR>), grid, block, 0, st, a);
    GO(8, 64) GO(16, 64) GO(32, 64) GO(16, 256) GO(32, 256) GO(32, 512)
#undef GO
}

}  // namespace
}  // namespace elsaa

using namespace elsaa;

extern "C" {

int elsaa_rms_norm_fwd(const elsaa_norm_desc* d, const void* X, const void* residual, const float* weight, void* sum,
                       void* Y, float* scale, hipStream_t stream)
{
    int rc = check_norm(d);
    if (rc) return rc;
    if (d->y_dtype != d->dtype && d->y_dtype != ELSAA_I8)
        return api_fail(ELSAA_ERR_INVALID_ARG, "y_dtype must be dtype or ELSAA_I8 (got %d)", d->y_dtype);
    const bool i8 = d->y_dtype == ELSAA_I8;
    if (!X || !weight || !Y || (i8 && !scale)) return api_fail(ELSAA_ERR_INVALID_ARG, "a required pointer is NULL");
    const int el = d->dtype == ELSAA_BF16 ? 2 : 4;
    if ((rc = check_rows("X", X, d->ldx, d->cols, el)) || (rc = check_rows("Y", Y, d->ldy, d->cols, i8 ? 1 : el)) ||
        (residual && (rc = check_rows("residual", residual, d->ldr, d->cols, el))) ||
        (sum && (rc = check_rows("sum", sum, d->lds, d->cols, el))))
        return rc;
    if (!aligned(weight, 4) || (i8 && !aligned(scale, 4)))
        return api_fail(ELSAA_ERR_INVALID_ARG, "weight and scale must be 4-byte aligned");
    if (sum == Y) return api_fail(ELSAA_ERR_INVALID_ARG, "sum and Y must be different buffers");
    if (i8 && (Y == X || Y == residual)) return api_fail(ELSAA_ERR_INVALID_ARG, "8-bit Y must not be X or the residual");
    if ((rc = check_in_place("sum", sum, d->lds, X, d->ldx, d->rows)) ||
        (rc = check_in_place("sum", sum, d->lds, residual, d->ldr, d->rows)) || (rc = check_in_place("Y", Y, d->ldy, X, d->ldx, d->rows)) ||
        (rc = check_in_place("Y", Y, d->ldy, residual, d->ldr, d->rows)))
        return rc;
    NormArgs a = {};
    a.x = X; a.r = residual; a.w = weight; a.s = sum; a.y = Y; a.scale = scale;
    a.rows = d->rows; a.ldx = d->ldx; a.ldr = d->ldr; a.lds = d->lds; a.ldy = d->ldy;
    a.cols = d->cols; a.eps = d->eps;
    const bool vec = d->cols % 8 == 0 && vec_ok(X, d->ldx) && vec_ok(residual, d->ldr) && vec_ok(sum, d->lds) &&
                     vec_ok(Y, d->ldy, i8);
    if (d->dtype == ELSAA_BF16) vec ? launch_fwd<BF16, 8>(a, i8, stream) : launch_fwd<BF16, 1>(a, i8, stream);
    else vec ? launch_fwd<F32, 4>(a, i8, stream) : launch_fwd<F32, 1>(a, i8, stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ELSAA_OK : api_hip_fail(e, "rms norm launch");
}

int elsaa_rms_norm_workspace_bytes(const elsaa_norm_desc* d, size_t* bytes)
{
    const int rc = check_norm(d);
    if (rc) return rc;
    if (!bytes) return api_fail(ELSAA_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = (size_t)bwd_blocks(d->rows, d->cols) * d->cols * sizeof(float);
    return ELSAA_OK;
}

int elsaa_rms_norm_bwd(const elsaa_norm_desc* d, const void* X, const float* weight, const void* dY, const void* dS,
                       void* dX, float* dweight, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    int rc = check_norm(d);
    if (rc) return rc;
    if (!X || !weight || !dY || !dX || (dweight && !workspace))
        return api_fail(ELSAA_ERR_INVALID_ARG, "a required pointer is NULL");
    const int el = d->dtype == ELSAA_BF16 ? 2 : 4;
    if ((rc = check_rows("X", X, d->ldx, d->cols, el)) || (rc = check_rows("dY", dY, d->ldy, d->cols, el)) ||
        (dS && (rc = check_rows("dS", dS, d->ldr, d->cols, el))) || (rc = check_rows("dX", dX, d->lds, d->cols, el)))
        return rc;
    if (!aligned(weight, 4) || !aligned(dweight, 4) || !aligned(workspace, 4))
        return api_fail(ELSAA_ERR_INVALID_ARG, "weight, dweight and workspace must be 4-byte aligned");
    if ((rc = check_in_place("dX", dX, d->lds, X, d->ldx, d->rows)) || (rc = check_in_place("dX", dX, d->lds, dY, d->ldy, d->rows)) ||
        (rc = check_in_place("dX", dX, d->lds, dS, d->ldr, d->rows)))
        return rc;
    const int64_t parts = bwd_blocks(d->rows, d->cols);
    const size_t need = (size_t)parts * d->cols * sizeof(float);
    if (dweight && workspace_bytes < need)
        return api_fail(ELSAA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
    NormArgs a = {};
    a.x = X; a.r = dS; a.dy = dY; a.w = weight; a.s = dX; a.part = dweight ? (float*)workspace : nullptr;
    a.rows = d->rows; a.ldx = d->ldx; a.ldr = d->ldr; a.lds = d->lds; a.ldy = d->ldy;
    a.cols = d->cols; a.eps = d->eps;
    const bool vec = d->cols % 8 == 0 && vec_ok(X, d->ldx) && vec_ok(dS, d->ldr) && vec_ok(dX, d->lds) && vec_ok(dY, d->ldy);
    if (d->dtype == ELSAA_BF16) vec ? launch_bwd<BF16, 8>(a, stream) : launch_bwd<BF16, 1>(a, stream);
    else vec ? launch_bwd<F32, 4>(a, stream) : launch_bwd<F32, 1>(a, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return api_hip_fail(e, "rms norm backward launch");
    if (dweight) {
        ELSAA_LAUNCH("rms_norm_dw", rms_norm_dw_kernel, dim3((d->cols + 63) / 64), dim3(1024), 0, stream, a.part, dweight,
                     d->cols, (int)parts);
        if ((e = hipGetLastError()) != hipSuccess) return api_hip_fail(e, "rms norm weight gradient launch");
    }
    return ELSAA_OK;
}

int elsaa_quantize_rows(const elsaa_quant_desc* d, const void* X, int8_t* Q, float* scale, hipStream_t stream)
{
    if (!d) return api_fail(ELSAA_ERR_INVALID_ARG, "desc is NULL");
    if (d->rows < 1 || d->cols < 1)
        return api_fail(ELSAA_ERR_INVALID_ARG, "rows and cols must be >= 1 (got %lld, %d)", (long long)d->rows, d->cols);
    if (d->cols > kMaxCols) return api_fail(ELSAA_ERR_UNSUPPORTED, "cols must be <= %d (got %d)", kMaxCols, d->cols);
    if (d->dtype != ELSAA_F32 && d->dtype != ELSAA_BF16) return api_fail(ELSAA_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
    if (!X || !Q || !scale) return api_fail(ELSAA_ERR_INVALID_ARG, "a required pointer is NULL");
    if (d->heads < 0) return api_fail(ELSAA_ERR_INVALID_ARG, "heads must be >= 0 (got %d)", d->heads);
    const int el = d->dtype == ELSAA_BF16 ? 2 : 4;
    QuantArgs a = {};
    int rc;
    if ((rc = check_rows("X", X, d->heads ? d->cols : d->ld, d->cols, el)) ||
        (rc = check_rows("Q", Q, d->ldq, d->cols, 1)))
        return rc;
    if (!aligned(scale, 4)) return api_fail(ELSAA_ERR_INVALID_ARG, "scale must be 4-byte aligned");
    if (d->heads) {
        if (d->cols % d->heads != 0)
            return api_fail(ELSAA_ERR_INVALID_ARG, "%d columns do not split into %d heads", d->cols, d->heads);
        const int dh = d->cols / d->heads;
        if (dh < 8 || (dh & (dh - 1)) != 0)
            return api_fail(ELSAA_ERR_UNSUPPORTED, "head width %d must be a power of two >= 8", dh);
        if (d->seq < 1 || d->rows % d->seq != 0)
            return api_fail(ELSAA_ERR_INVALID_ARG, "%lld rows are not a whole number of sequences of %d",
                            (long long)d->rows, d->seq);
        while ((1 << a.dh_shift) < dh) ++a.dh_shift;
    }
    a.x = X; a.q = Q; a.scale = scale;
    a.rows = d->rows; a.ld = d->ld; a.ldq = d->ldq; a.cols = d->cols; a.heads = d->heads; a.seq = d->seq;
    const bool vec = d->cols % 8 == 0 && vec_ok(X, d->heads ? 0 : d->ld) && vec_ok(Q, d->ldq, true);
    if (d->dtype == ELSAA_BF16) vec ? launch_quant<BF16, 8>(a, stream) : launch_quant<BF16, 1>(a, stream);
    else vec ? launch_quant<F32, 4>(a, stream) : launch_quant<F32, 1>(a, stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ELSAA_OK : api_hip_fail(e, "quantize rows launch");
}

}  // extern "C"
