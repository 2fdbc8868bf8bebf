// gemm_i8.hip -- product of 8-bit rows and 8-bit weights with a float32 scale for
// each row and each output channel:
//     C_ij = a_i b_j sum_k A_ik B_jk
//
// The sums are 32-bit integers (v_mfma_i32_16x16x64_i8: twice the rate of the
// bfloat16 instruction on operands half as wide), so they are exact whatever
// the order, and one scaling and rounding at the end is all that differs from
// the definition.  Both operands are stored with k contiguous (tokens and output
// channels are rows), so every operand fragment is 16 contiguous bytes of a
// row; which k each lane holds does not matter as long as A and B agree.
//
// gemm_i8_rows_kernel (few tokens): bound by the weights' bytes.  A workgroup
// takes 16 channels and all tokens, its waves share out k, operands go from
// memory to registers, and the waves' sums meet in LDS.
//
// gemm_i8_big_kernel (tiles of 256 rows by 256, 192 or 128 channels, K-tiles of 128
// bytes, one workgroup of four waves a compute unit, the sums in the accumulation
// registers): per 64 bytes of k a wave of 128 x 128 reads 16 operand fragments
// for 64 matrix-core operations.
//
// gemm_i8_kernel (128 x 128 tiles, K-tiles of 128 bytes, four waves in a 2 x 2
// grid): operands staged through LDS, loads two K-tiles ahead in
// registers.  Products with few tiles split K over workgroups; the partial
// sums (32-bit integers) are added by gemm_i8_reduce_kernel.
#include <cstring>

#include "common.hpp"
#include "elsaa.h"
#include "gemm_index.hpp"
#include "internal.hpp"

namespace elsaa {

using gemm::Mat;

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxK = 131071;          // 2^14 K < 2^31
constexpr int kMaxRows = 1 << 30;      // M and N: positions up to a tile behind them fit 32 bits
constexpr int BM = 128, BN = 128;
constexpr int BKB = 128;               // bytes of k in a K-tile
constexpr int kThreads = 256;
// LDS place (bytes) of 16-byte chunk c of row r of an operand tile.  A 16-byte
// read serves lanes 0-3, 12-15, 20-23 and 24-27 together (then 4-11, 16-19 and
// 28-31, and the same 32 lanes on): rows 0-3 and 12-15 of one chunk and 4-11 of
// its neighbour.  With the chunks of a row exchanged by the row pair's number these
// 256 bytes lie in 64 different banks; padding of 16 bytes a row or a row pair leaves two of them
// in one bank, which adds half to the read (1000 x 2048 x 2048: 19.9 us padded, 19.0 exchanged;
// 16384 x 6144 x 2048: 226 either way, the matrix cores and the card's power set its pace).
__device__ __forceinline__ constexpr int lds_at(int r, int c) { return r * BKB + 16 * (c ^ ((r >> 1) & 7)); }
constexpr int kGroupM = 8;

struct IArgs {
    const int8_t *A, *B;
    const float *as, *bs;
    int64_t lda, ldb;
    Mat C;
    int M, N, K;
    int vec;                           // C takes four columns in one store
    int tiles_m, tiles_n, splits, kper;
    int32_t* part;                     // [splits][M][np] when splits > 1
    int np;                            // N rounded up to 4
};

__device__ __forceinline__ i32x4 mma(i32x4 a, i32x4 b, i32x4 c)
{
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// 16 bytes at the uniform address q plus a per-lane byte offset < 2^31.
__device__ __forceinline__ i32x4 ldb16(const int8_t* q, uint32_t off)
{
    const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(q), (short)0, 0x7fffffff, 0x00027000);
    return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0));
}

// The first n of 16 bytes, the rest zero.
__device__ __forceinline__ i32x4 keep_bytes(i32x4 v, int n)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int left = n - 4 * i;
        v[i] = left >= 4 ? v[i] : left <= 0 ? 0 : v[i] & ((1 << (8 * left)) - 1);
    }
    return v;
}

// Columns n .. n + 3 of row m, scaled, rounded once and stored.
template <bool OUT_BF16>
__device__ __forceinline__ void store_c(const IArgs& a, int m, int n, i32x4 v)
{
    const float s = a.as[m];
    if (a.vec && n + 3 < a.N) {
        const f32x4 b = {a.bs[n], a.bs[n + 1], a.bs[n + 2], a.bs[n + 3]};
        f32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = (float)v[i] * s * b[i];
        const int64_t off = mat_offset(a.C, m, n);
        if (OUT_BF16) store4<BF16>((uint16_t*)a.C.p + off, o);
        else store4<F32>((float*)a.C.p + off, o);
        return;
    }
    for (int i = 0; i < 4 && n + i < a.N; ++i) {
        const float o = (float)v[i] * s * a.bs[n + i];
        const int64_t off = mat_offset(a.C, m, n + i);
        if (OUT_BF16) ((uint16_t*)a.C.p)[off] = f32_to_bf16(o);
        else ((float*)a.C.p)[off] = o;
    }
}

// ---------------------------------------------------------------- few tokens
// MT groups of 16 tokens, NW waves.  Per step a wave covers 128 bytes of k:
// lane (row i = lane % 16, g = lane / 16) holds bytes 32 g .. 32 g + 31, two
// fragments, so a row is read as one 128-byte line.
template <int MT, int NW, bool OUT_BF16>
__global__ __launch_bounds__(64 * NW) void gemm_i8_rows_kernel(IArgs a)
{
    __shared__ __attribute__((aligned(16))) i32x4 sums[NW][MT][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int g = lane >> 4, i = lane & 15;
    const int n0 = blockIdx.x * 16;
    // rows past the matrix repeat its last one and are not stored
    const int8_t* pb = a.B + (int64_t)min(n0 + i, a.N - 1) * a.ldb + 32 * g;
    const int8_t* pa[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) pa[t] = a.A + (int64_t)min(16 * t + i, a.M - 1) * a.lda + 32 * g;
    i32x4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = i32x4{0, 0, 0, 0};
    // whole steps of this wave, then (last wave) the short one
    const int steps = a.K / BKB, per = (steps + NW - 1) / NW;
    const int s0 = min(w * per, steps), s1 = min(s0 + per, steps);
    constexpr int U = 4;
    int s = s0;
    for (; s + U <= s1; s += U) {
        i32x4 fb[U][2], fa[U][MT][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = (s + u) * BKB;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                fb[u][h] = *(const i32x4*)(pb + k + 16 * h);
#pragma unroll
                for (int t = 0; t < MT; ++t) fa[u][t][h] = *(const i32x4*)(pa[t] + k + 16 * h);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < MT; ++t) acc[t] = mma(fb[u][h], fa[u][t][h], acc[t]);
    }
    // one step of which only the bytes before K count: weights past K are zero,
    // so what stands there in A does not matter
    auto masked = [&](int k) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int left = a.K - (k + 32 * g + 16 * h);
            i32x4 b = {0, 0, 0, 0}, x[MT];
            if (left > 0) b = keep_bytes(*(const i32x4*)(pb + k + 16 * h), left);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                x[t] = i32x4{0, 0, 0, 0};
                if (left > 0) x[t] = *(const i32x4*)(pa[t] + k + 16 * h);
                acc[t] = mma(b, x[t], acc[t]);
            }
        }
    };
    for (; s < s1; ++s) masked(s * BKB);
    if (w == NW - 1 && steps * BKB < a.K) masked(steps * BKB);
#pragma unroll
    for (int t = 0; t < MT; ++t) sums[w][t][lane] = acc[t];
    __syncthreads();
    if (w >= MT) return;
    i32x4 v = sums[0][w][lane];
#pragma unroll
    for (int j = 1; j < NW; ++j) v += sums[j][w][lane];
    const int m = 16 * w + i, n = n0 + 4 * g;
    if (m < a.M && n < a.N) store_c<OUT_BF16>(a, m, n, v);
}

// ---------------------------------------------------------------- tiles
// Tile coordinates of this workgroup: ids dealt so that each of the eight
// XCDs works on a contiguous run, in groups of kGroupM row tiles swept along
// the channels.
__device__ __forceinline__ void tile_of(const IArgs& a, int& sp, int& tm, int& tn)
{
    const int total = a.tiles_m * a.tiles_n * a.splits;
    int id = blockIdx.x;
    const int full = total & ~7;
    if (id < full) id = (id & 7) * (full >> 3) + (id >> 3);
    const int per = a.tiles_m * a.tiles_n;
    sp = id / per;
    const int t = id - sp * per;
    const int group = t / (kGroupM * a.tiles_n);
    const int m0 = group * kGroupM;
    const int gm = min(kGroupM, a.tiles_m - m0);
    const int r = t - group * kGroupM * a.tiles_n;
    tm = m0 + r % gm;
    tn = r / gm;
}

// Rows x0 + tx / 8 + 32 c of an operand, 16-byte chunk tx % 8 of a K-tile.
// Rows past the matrix repeat its last one.
template <int C>
struct Loader {
    const int8_t* p;        // row x0
    uint32_t off[C];
    int kc;                 // first k of the thread's chunk in a K-tile
    __device__ __forceinline__ void init(const int8_t* m, int64_t ld, int x0, int rows)
    {
        p = m + (int64_t)x0 * ld;
        kc = 16 * (threadIdx.x & 7);
#pragma unroll
        for (int c = 0; c < C; ++c) off[c] = (uint32_t)((min(x0 + (int)(threadIdx.x >> 3) + 32 * c, rows - 1) - x0) * ld) + kc;
    }
    __device__ __forceinline__ i32x4 chunk(int k0, int c) const { return ldb16(p + k0, off[c]); }
    __device__ __forceinline__ void load(int k0, i32x4 (&r)[C]) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c) r[c] = chunk(k0, c);
    }
    // a K-tile whose values from ke on are zero
    __device__ __forceinline__ void load_short(int k0, int ke, i32x4 (&r)[C]) const
    {
        const int left = ke - (k0 + kc);
#pragma unroll
        for (int c = 0; c < C; ++c) r[c] = left > 0 ? keep_bytes(chunk(k0, c), left) : i32x4{0, 0, 0, 0};
    }
};

__device__ __forceinline__ void store_tile(int8_t* s, const i32x4 (&r)[4])
{
#pragma unroll
    for (int c = 0; c < 4; ++c) *(i32x4*)&s[32 * BKB * c + lds_at(threadIdx.x >> 3, threadIdx.x & 7)] = r[c];
}

// Operand fragment of rows x0 .. x0 + 15, bytes 64 ks .. 64 ks + 63 of k.
__device__ __forceinline__ i32x4 frag(const int8_t* s, int x0, int ks)
{
    const int lane = threadIdx.x & 63;
    return *(const i32x4*)&s[x0 * BKB + lds_at(lane & 15, 4 * ks + (lane >> 4))];
}

template <bool OUT_BF16>
__global__ __launch_bounds__(kThreads, 2) void gemm_i8_kernel(IArgs a)
{
    __shared__ __attribute__((aligned(16))) int8_t sa[2][BM * BKB];
    __shared__ __attribute__((aligned(16))) int8_t sb[2][BN * BKB];
    int sp, tm, tn;
    tile_of(a, sp, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN;
    const int kb = sp * a.kper, ke = min(a.K, kb + a.kper);
    const int nkt = (ke - kb + BKB - 1) / BKB;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int wm = w & 1, wn = w >> 1;
    const int g = lane >> 4, col = lane & 15;

    i32x4 acc[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = i32x4{0, 0, 0, 0};

    Loader<4> gA, gB;
    gA.init(a.A, a.lda, m0, a.M);
    gB.init(a.B, a.ldb, n0, a.N);
    auto fetch = [&](int t, i32x4 (&ra)[4], i32x4 (&rb)[4]) {
        const int k0 = kb + t * BKB;
        if (k0 + BKB <= ke) {
            gA.load(k0, ra);
            gB.load(k0, rb);
        } else {
            gA.load_short(k0, ke, ra);
            gB.load_short(k0, ke, rb);
        }
    };
    // LDS buffer t & 1 holds K-tile t, register set (t + 1) & 1 K-tile t + 1,
    // and iteration t requests K-tile t + 2.
    i32x4 ra[2][4], rb[2][4];
    fetch(0, ra[0], rb[0]);
    if (nkt > 1) fetch(1, ra[1], rb[1]);
    store_tile(sa[0], ra[0]);
    store_tile(sb[0], rb[0]);
    __syncthreads();
    auto step = [&](int t, auto parity) {
        constexpr int P = decltype(parity)::value;        // t & 1
        if (t + 2 < nkt) fetch(t + 2, ra[P], rb[P]);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            i32x4 xf[4], yf[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) xf[j] = frag(sb[P], 64 * wn + 16 * j, ks);
#pragma unroll
            for (int i = 0; i < 4; ++i) yf[i] = frag(sa[P], 64 * wm + 16 * i, ks);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] = mma(xf[j], yf[i], acc[j][i]);
        }
        if (t + 1 < nkt) {
            store_tile(sa[1 - P], ra[1 - P]);
            store_tile(sb[1 - P], rb[1 - P]);
        }
        __syncthreads();
    };
    for (int t = 0; t < nkt; t += 2) {
        step(t, std::integral_constant<int, 0>{});
        if (t + 1 < nkt) step(t + 1, std::integral_constant<int, 1>{});
    }

    // lane holds C[m0 + 64 wm + 16 i + col][n0 + 64 wn + 16 j + 4 g + (0..3)]
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int m = m0 + 64 * wm + 16 * i + col;
        if (m >= a.M) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = n0 + 64 * wn + 16 * j + 4 * g;
            if (n >= a.N) continue;
            if (a.splits > 1) *(i32x4*)(a.part + ((int64_t)sp * a.M + m) * a.np + n) = acc[j][i];
            else store_c<OUT_BF16>(a, m, n, acc[j][i]);
        }
    }
}

// ---------------------------------------------------------------- large tiles
namespace big {

constexpr int BT = 256;                              // rows of a tile; 32 NJ channels, 16 NJ a wave
constexpr int kChunks = BT * BKB / 16 / kThreads;    // 16-byte chunks a thread loads of A's K-tile (NJ of B's)
static_assert(kChunks == 8, "one chunk of A per group of operations");

__device__ __forceinline__ void store1(int8_t* s, i32x4 v, int c)
{
    *(i32x4*)&s[32 * BKB * c + lds_at(threadIdx.x >> 3, threadIdx.x & 7)] = v;
}

// acc += a x b with acc tied to accumulation registers: the 64 accumulators
// fill all 256 of them, and with the builtin the register allocator moves some
// through vector registers on every iteration.  The compiler does not see this
// as a matrix-core instruction: the statements keep program order (an
// accumulator is used again only after the 63 others), and what reads acc after the
// last one is behind the wait states of mfma_drain.
__device__ __forceinline__ void mfma_acc(i32x4& acc, i32x4 a, i32x4 b)
{
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
__device__ __forceinline__ void mfma_drain()
{
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15\n\ts_nop 15" ::: "memory");
}

// K a multiple of 16, at least 128.  K ranges that are no multiple of 128 begin
// with their short K-tile (zeros behind its end), so that the loop runs on
// whole ones.
template <bool OUT_BF16, int NJ>
__global__ __launch_bounds__(kThreads, 1) void gemm_i8_big_kernel(IArgs a)
{
    constexpr int BTN = 32 * NJ, WN = 16 * NJ;       // channels of a tile and of a wave
    constexpr int A_TILE = BT * BKB, B_TILE = BTN * BKB;
    constexpr int LDS = 2 * (A_TILE + B_TILE) > 4 * 64 * (WN + 4) * 4 ? 2 * (A_TILE + B_TILE) : 4 * 64 * (WN + 4) * 4;
    __shared__ __attribute__((aligned(16))) int8_t lds[LDS];
    int8_t(*sa)[A_TILE] = (int8_t(*)[A_TILE])lds;
    int8_t(*sb)[B_TILE] = (int8_t(*)[B_TILE])(lds + 2 * A_TILE);
    int sp, tm, tn;
    tile_of(a, sp, tm, tn);
    const int m0 = tm * BT, n0 = tn * BTN;
    const int kb = sp * a.kper, ke = min(a.K, kb + a.kper);
    const int nkt = (ke - kb + BKB - 1) / BKB;
    // first k of K-tile t >= 1; past the end the last one again (loaded, never read)
    auto whole = [&](int t) { return ke - (nkt - min(t, nkt - 1)) * BKB; };
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int wm = w & 1, wn = w >> 1;
    const int g = lane >> 4, col = lane & 15;

    i32x4 acc[NJ][8];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[j][i] = i32x4{0, 0, 0, 0};

    Loader<kChunks> gA;
    Loader<NJ> gB;
    gA.init(a.A, a.lda, m0, a.M);
    gB.init(a.B, a.ldb, n0, a.N);
    // Pipeline: LDS buffer t & 1 holds K-tile t, the registers K-tile t + 1.
    // The first half of an iteration runs k-step 0 of tile t (fragments
    // already read) in eight groups of NJ operations; before group i it
    // reads fragment pair i of k-step 1, stores chunk i of both operands of
    // tile t + 1 to the other buffer and reloads those registers with chunk i
    // of tile t + 2.  After the one barrier, the second half runs k-step 1 the
    // same way, reading k-step 0 of tile t + 1.  Each load has an iteration
    // to arrive, and no burst of memory instructions stalls the in-order wave.
    i32x4 ra[kChunks], rb[NJ];
    gA.load_short(kb, ke - (nkt - 1) * BKB, ra);
    gB.load_short(kb, ke - (nkt - 1) * BKB, rb);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        store1(sa[0], ra[i], i);
        if (i < NJ) store1(sb[0], rb[i], i);
    }
    {
        const int k1 = whole(1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            ra[i] = gA.chunk(k1, i);
            if (i < NJ) rb[i] = gB.chunk(k1, i);
        }
    }
    __syncthreads();
    i32x4 x0[NJ], y0[8], x1[NJ], y1[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (j < NJ) x0[j] = frag(sb[0], WN * wn + 16 * j, 0);
        y0[j] = frag(sa[0], 128 * wm + 16 * j, 0);
    }
    for (int t = 0; t < nkt; ++t) {
        const int8_t *A_ = sa[t & 1], *B_ = sb[t & 1];
        int8_t *An = sa[(t + 1) & 1], *Bn = sb[(t + 1) & 1];
        const int k2 = whole(t + 2);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i < NJ) x1[i] = frag(B_, WN * wn + 16 * i, 1);
            y1[i] = frag(A_, 128 * wm + 16 * i, 1);
            store1(An, ra[i], i);
            if (i < NJ) store1(Bn, rb[i], i);
            ra[i] = gA.chunk(k2, i);
            if (i < NJ) rb[i] = gB.chunk(k2, i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NJ; ++j) mfma_acc(acc[j][i], x0[j], y0[i]);
            __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i < NJ) x0[i] = frag(Bn, WN * wn + 16 * i, 0);
            y0[i] = frag(An, 128 * wm + 16 * i, 0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NJ; ++j) mfma_acc(acc[j][i], x1[j], y1[i]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    __syncthreads();
    mfma_drain();

    if (a.splits > 1) {
        // lane holds C[m0 + 128 wm + 16 i + col][n0 + WN wn + 16 j + 4 g + (0..3)]
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int m = m0 + 128 * wm + 16 * i + col;
            if (m >= a.M) continue;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int n = n0 + WN * wn + 16 * j + 4 * g;
                if (n < a.N) *(i32x4*)(a.part + ((int64_t)sp * a.M + m) * a.np + n) = acc[j][i];
            }
        }
        return;
    }
    // The sums pass through LDS (each wave its own 64 x WN block per half, four
    // values of padding a row) and leave as 8 columns of a row a lane.  Accumulators
    // are only ever stored, never operated on, so they stay in the accumulation registers.
    constexpr int kLdC = WN + 4, PR = WN / 8;        // pieces of 8 columns a row: as many passes over 64 rows
    int32_t* cs = (int32_t*)lds + w * 64 * kLdC;
    static_assert(4 * 64 * kLdC * 4 <= LDS, "the waves' blocks fit");
    // A lane's columns repeat every SETS passes.
    constexpr int SETS = PR % 3 == 0 ? 3 : 1;
    static_assert(64 * SETS % PR == 0, "the columns repeat");
    float bs[SETS][8];
#pragma unroll
    for (int q = 0; q < SETS; ++q)
#pragma unroll
        for (int i = 0; i < 8; ++i) bs[q][i] = a.bs[min(n0 + WN * wn + 8 * ((lane + 64 * q) % PR) + i, a.N - 1)];
    // a whole tile inside one sequence: rows of C equally spaced, whole vectors, no bounds
    const bool all = a.vec && m0 + BT <= a.M && n0 + BTN <= a.N && (a.C.heads == 0 || m0 / a.C.seq == (m0 + BT - 1) / a.C.seq);
    auto epilogue = [&](auto whole_tile) {
        constexpr bool WHOLE = decltype(whole_tile)::value;
        using O = typename std::conditional<OUT_BF16, BF16, F32>::type;
        using S = typename O::store_t;
        const int64_t cs_ = row_stride(a.C);
        S* c_first[SETS];
#pragma unroll
        for (int q = 0; q < SETS; ++q)
            c_first[q] = (S*)a.C.p + (WHOLE ? row_part(a.C, m0 + 128 * wm + (lane + 64 * q) / PR) +
                                                  col_part(a.C, n0 + WN * wn + 8 * ((lane + 64 * q) % PR)) : 0);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            float as[PR];
#pragma unroll
            for (int it = 0; it < PR; ++it) {
                const int m = m0 + 128 * wm + 64 * hh + (lane + 64 * it) / PR;
                as[it] = a.as[WHOLE ? m : min(m, a.M - 1)];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < NJ; ++j) *(i32x4*)&cs[(16 * i + col) * kLdC + 16 * j + 4 * g] = acc[j][4 * hh + i];
            __builtin_amdgcn_wave_barrier();      // (a wave reads what it wrote itself)
#pragma unroll
            for (int it = 0; it < PR; ++it) {
                const int r = (lane + 64 * it) / PR, c8 = 8 * ((lane + 64 * it) % PR);
                const int m = m0 + 128 * wm + 64 * hh + r, n = n0 + WN * wn + c8;
                const i32x4 x = *(const i32x4*)&cs[r * kLdC + c8];
                const i32x4 y = *(const i32x4*)&cs[r * kLdC + c8 + 4];
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    o[i] = (float)(i < 4 ? x[i & 3] : y[i & 3]) * as[it] * bs[it % SETS][i];
                if (WHOLE) {
                    store8<O>(c_first[it % SETS] + (64 * hh + it / SETS * (64 * SETS / PR)) * cs_, o);
                } else if (m < a.M && n < a.N) {
                    if (a.vec && n + 8 <= a.N) {
                        store8<O>((S*)a.C.p + mat_offset(a.C, m, n), o);
                    } else {
                        for (int i = 0; i < 8 && n + i < a.N; ++i) ((S*)a.C.p)[mat_offset(a.C, m, n + i)] = O::store(o[i]);
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    };
    if (all) epilogue(std::true_type{});
    else epilogue(std::false_type{});
}

}  // namespace big

// C from the sum of the splits' partial sums.
template <bool OUT_BF16>
__global__ __launch_bounds__(256) void gemm_i8_reduce_kernel(IArgs a)
{
    const int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int n4 = a.np / 4;
    if (q >= (int64_t)a.M * n4) return;
    const int m = (int)(q / n4), n = (int)(q - (int64_t)m * n4) * 4;
    const int64_t plane = (int64_t)a.M * a.np;
    i32x4 v = *(const i32x4*)(a.part + 4 * q);
    for (int s = 1; s < a.splits; ++s) v += *(const i32x4*)(a.part + s * plane + 4 * q);
    store_c<OUT_BF16>(a, m, n, v);
}

constexpr int kRowsMax = 64;           // tokens that gemm_i8_rows_kernel takes
constexpr int64_t kGridThreads = (int64_t)1 << 32;      // a launch has fewer threads in a dimension

struct Plan {
    bool rows;
    bool fits;                         // there are tiles that one launch holds
    int nj;                            // large tiles of 32 nj channels; 0: 128 x 128
    int tiles_m, tiles_n, splits, kper;
    size_t ws_bytes;
};

Plan plan_of(const elsaa_gemm_i8_desc* d)
{
    auto parts = [](int64_t n, int64_t per) { return (n + per - 1) / per; };
    Plan p = {};
    // (a workgroup of 256 threads for 16 channels; tiles take the rest)
    p.rows = d->M <= kRowsMax && parts(d->N, 16) * 256 < kGridThreads;
    p.fits = p.rows;
    const int64_t ktiles = parts(d->K, BKB);
    p.splits = 1;
    if (!p.rows) {
        // Estimated microseconds of a tile size and split count, a round being
        // the workgroups resident at once (256 large tiles or 512 small ones): a
        // cost for each K-tile and one for a round's first loads and last stores, fitted to
        // products of one to six rounds.  Small tiles take three quarters where they fill at most half the
        // chip; splitting K costs a launch and the partial sums' way to memory and back.
        // The lines this draws, measured (us with 256 x 256, 256 x 192, 256 x 128 and 128 x 128 tiles):
        // 16384 x 6144 x 2048 226, 250, 270, 298; 8002 x 2048 x 2048 39, 59, 47, 53;
        // 4096 x 6144 x 2048 70, 64, 69, 80; 4096 x 2048 x 2048 34, 32, 24.5, 29; 2048 x 2048 x 2048 32, 29,
        // 21.0, 20.3.
        auto estimate = [&](int nj, int64_t tiles, int splits) {
            const int fill = nj ? 256 : 512;
            const int64_t per = parts(ktiles, splits);
            const int64_t wgs = tiles * parts(ktiles, per), rem = wgs % fill;
            const double rounds = wgs / fill + (rem == 0 ? 0. : !nj && 2 * rem <= fill ? 0.75 : 1.);
            const double reduce = splits > 1 ? 5. + 2e-6 * splits * (double)d->M * d->N * 4 / 6. : 0.;
            const double step = nj == 8 ? 1.8 : nj == 6 ? 1.62 : nj == 4 ? 1.18 : 1.25;
            const double rest = nj == 8 ? 12.5 : nj == 6 ? 8.3 : nj == 4 ? 7. : 9.;
            return rounds * (per * step + rest) + reduce;
        };
        double best = 0.;
        for (int nj : {0, 4, 6, 8}) {
            if (nj && (d->K < BKB || d->K % 16 != 0)) continue;
            const int64_t tiles = parts(d->M, nj ? big::BT : BM) * parts(d->N, nj ? 32 * nj : BN), fill = nj ? 256 : 512;
            if (tiles * kThreads >= kGridThreads) continue;
            p.fits = true;
            // at least four K-tiles a split, at most one round of workgroups
            int64_t most = tiles < fill ? fill / tiles : 1;
            if (most > ktiles / 4) most = ktiles / 4;
            for (int splits = 1; splits <= (most < 1 ? 1 : most); ++splits) {
                const double e = estimate(nj, tiles, splits);
                if (best == 0. || e < best) {
                    best = e;
                    p.nj = nj;
                    p.splits = splits;
                }
            }
        }
    }
    p.tiles_m = (int)parts(d->M, p.nj ? big::BT : BM);
    p.tiles_n = (int)parts(d->N, p.nj ? 32 * p.nj : BN);
    p.kper = (int)parts(ktiles, p.splits) * BKB;
    p.splits = (int)parts(d->K, p.kper);
    p.ws_bytes = p.splits > 1 ? (size_t)p.splits * d->M * (parts(d->N, 4) * 4) * sizeof(int32_t) : 0;
    return p;
}

int validate(const elsaa_gemm_i8_desc* d)
{
    if (!d) return api_fail(ELSAA_ERR_INVALID_ARG, "desc is NULL");
    if (d->M < 1 || d->N < 1 || d->K < 1)
        return api_fail(ELSAA_ERR_INVALID_ARG, "M, N, K must be >= 1 (got %d, %d, %d)", d->M, d->N, d->K);
    if (d->M > kMaxRows || d->N > kMaxRows)
        return api_fail(ELSAA_ERR_UNSUPPORTED, "M and N must be <= 2^30 (got %d, %d)", d->M, d->N);
    if (d->K > kMaxK) return api_fail(ELSAA_ERR_UNSUPPORTED, "K must be <= %d (got %d)", kMaxK, d->K);
    if (d->c_dtype != ELSAA_F32 && d->c_dtype != ELSAA_BF16)
        return api_fail(ELSAA_ERR_INVALID_ARG, "unknown c_dtype %d", d->c_dtype);
    return ELSAA_OK;
}

int too_large(const elsaa_gemm_i8_desc* d)
{
    return api_fail(ELSAA_ERR_UNSUPPORTED, "M x N is too large (%d x %d)", d->M, d->N);
}

int check_operand(const char* name, const void* p, int K, int64_t ld)
{
    if (!p) return api_fail(ELSAA_ERR_INVALID_ARG, "%s is NULL", name);
    if (((uintptr_t)p & 15) != 0) return api_fail(ELSAA_ERR_INVALID_ARG, "%s must be 16-byte aligned", name);
    if (ld < K || ld % 16 != 0)
        return api_fail(ELSAA_ERR_INVALID_ARG, "%s: the row stride must be >= %d and a multiple of 16 (got %lld)", name, K,
                        (long long)ld);
    if (ld > (1 << 23))      // a tile's rows lie within 32-bit offsets of its first
        return api_fail(ELSAA_ERR_UNSUPPORTED, "%s: row strides above 2^23 are not supported (got %lld)", name, (long long)ld);
    return ELSAA_OK;
}

}  // namespace
}  // namespace elsaa

using namespace elsaa;

extern "C" {

int elsaa_gemm_i8_workspace_bytes(const elsaa_gemm_i8_desc* d, size_t* bytes)
{
    const int rc = validate(d);
    if (rc) return rc;
    if (!bytes) return api_fail(ELSAA_ERR_INVALID_ARG, "bytes is NULL");
    const Plan p = plan_of(d);
    if (!p.fits) return too_large(d);
    *bytes = p.ws_bytes;
    return ELSAA_OK;
}

int elsaa_gemm_i8(const elsaa_gemm_i8_desc* d, const int8_t* A, const float* a_scale, const int8_t* B,
                  const float* b_scale, void* C, void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    int rc = validate(d);
    if (rc) return rc;
    if ((rc = check_operand("A", A, d->K, d->lda)) || (rc = check_operand("B", B, d->K, d->ldb))) return rc;
    if (!a_scale || !b_scale || !C) return api_fail(ELSAA_ERR_INVALID_ARG, "a required pointer is NULL");
    const bool bf16 = d->c_dtype == ELSAA_BF16;
    const unsigned el = bf16 ? 2 : 4;
    if (((uintptr_t)a_scale & 3) || ((uintptr_t)b_scale & 3) || ((uintptr_t)C & (el - 1)))
        return api_fail(ELSAA_ERR_INVALID_ARG, "the scales and C must be aligned to their element");
    IArgs a;
    std::memset(&a, 0, sizeof a);
    a.C.p = C;
    a.C.ld = d->ldc;
    a.C.heads = d->c_heads;
    a.C.seq = d->seq;
    if (d->c_heads < 0) return api_fail(ELSAA_ERR_INVALID_ARG, "c_heads must be >= 0 (got %d)", d->c_heads);
    if (d->c_heads == 0) {
        if (d->ldc < d->N)
            return api_fail(ELSAA_ERR_INVALID_ARG, "ldc must be >= %d (got %lld)", d->N, (long long)d->ldc);
    } else {
        if (d->N % d->c_heads != 0)
            return api_fail(ELSAA_ERR_INVALID_ARG, "%d columns do not split into %d heads", d->N, d->c_heads);
        const int dh = d->N / d->c_heads;
        if (dh < 8 || (dh & (dh - 1)) != 0)
            return api_fail(ELSAA_ERR_UNSUPPORTED, "head width %d must be a power of two >= 8", dh);
        if (d->seq < 1 || d->M % d->seq != 0)
            return api_fail(ELSAA_ERR_INVALID_ARG, "%d rows are not a whole number of sequences of %d", d->M, d->seq);
        while ((1 << a.C.dh_shift) < dh) ++a.C.dh_shift;
    }
    const Plan p = plan_of(d);
    if (!p.fits) return too_large(d);
    if (p.ws_bytes > 0) {
        if (!workspace) return api_fail(ELSAA_ERR_INVALID_ARG, "workspace is NULL (%zu bytes needed)", p.ws_bytes);
        if (workspace_bytes < p.ws_bytes)
            return api_fail(ELSAA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, p.ws_bytes);
        if (((uintptr_t)workspace & 15) != 0) return api_fail(ELSAA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    }
    a.A = A; a.B = B; a.as = a_scale; a.bs = b_scale;
    a.lda = d->lda; a.ldb = d->ldb;
    a.M = d->M; a.N = d->N; a.K = d->K;
    a.tiles_m = p.tiles_m; a.tiles_n = p.tiles_n; a.splits = p.splits; a.kper = p.kper;
    a.part = (int32_t*)workspace;
    a.np = (d->N + 3) / 4 * 4;
    // (columns that one store takes: four here, eight behind large tiles)
    const int cv = p.nj ? 8 : 4;
    a.vec = ((uintptr_t)C & ((cv * el < 16 ? cv * el : 16) - 1)) == 0 && (d->c_heads > 0 || d->ldc % cv == 0);
    hipError_t e;
    if (p.rows) {
        const dim3 grid((d->N + 15) / 16);
        // (16 waves where four a workgroup leave the chip short of loads in flight)
        const bool wide = grid.x < 256 && d->K >= 16 * BKB;
#define ELSAA_I8_ROWS(MT, NW, OB) ELSAA_LAUNCH("gemm_i8_rows", (gemm_i8_rows_kernel<MT, NW, OB>), grid, dim3(64 * NW), 0, stream, a)
#define ELSAA_I8_MT(MT)                                                                          \
    do {                                                                                         \
        if (wide) { if (bf16) ELSAA_I8_ROWS(MT, 16, true); else ELSAA_I8_ROWS(MT, 16, false); }   \
        else { if (bf16) ELSAA_I8_ROWS(MT, 4, true); else ELSAA_I8_ROWS(MT, 4, false); }          \
    } while (0)
        if (d->M <= 16) ELSAA_I8_MT(1);
        else if (d->M <= 32) ELSAA_I8_MT(2);
        else ELSAA_I8_MT(4);
#undef ELSAA_I8_MT
#undef ELSAA_I8_ROWS
        e = hipGetLastError();
        return e == hipSuccess ? ELSAA_OK : api_hip_fail(e, "gemm_i8 launch");
    }
    const dim3 grid((unsigned)(p.tiles_m * p.tiles_n * p.splits));
    const char* big_name = p.nj == 8 ? "gemm_i8_256x256" : p.nj == 6 ? "gemm_i8_256x192" : "gemm_i8_256x128";
#define ELSAA_I8_BIG(NJ)                                                                                                      \
    do {                                                                                                                      \
        if (bf16) ELSAA_LAUNCH(big_name, (big::gemm_i8_big_kernel<true, NJ>), grid, dim3(kThreads), 0, stream, a);            \
        else ELSAA_LAUNCH(big_name, (big::gemm_i8_big_kernel<false, NJ>), grid, dim3(kThreads), 0, stream, a);                \
    } while (0)
    if (p.nj == 8) ELSAA_I8_BIG(8);
    else if (p.nj == 6) ELSAA_I8_BIG(6);
    else if (p.nj == 4) ELSAA_I8_BIG(4);
    else if (bf16) ELSAA_LAUNCH("gemm_i8", gemm_i8_kernel<true>, grid, dim3(kThreads), 0, stream, a);
    else ELSAA_LAUNCH("gemm_i8", gemm_i8_kernel<false>, grid, dim3(kThreads), 0, stream, a);
#undef ELSAA_I8_BIG
    if ((e = hipGetLastError()) != hipSuccess) return api_hip_fail(e, "gemm_i8 launch");
    if (p.splits > 1) {
        const dim3 rgrid((unsigned)(((int64_t)d->M * (a.np / 4) + 255) / 256));
        if (bf16) ELSAA_LAUNCH("gemm_i8_reduce", gemm_i8_reduce_kernel<true>, rgrid, dim3(256), 0, stream, a);
        else ELSAA_LAUNCH("gemm_i8_reduce", gemm_i8_reduce_kernel<false>, rgrid, dim3(256), 0, stream, a);
        if ((e = hipGetLastError()) != hipSuccess) return api_hip_fail(e, "gemm_i8 reduce launch");
    }
    return ELSAA_OK;
}

}  // extern "C"
