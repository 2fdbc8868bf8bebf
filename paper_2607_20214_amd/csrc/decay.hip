// decay.hip -- linear attention with a decay for each head: chunked forward,
// backward, and one token from the running state.
//
//   S_t = lambda S_{t-1} + k_t v_t^T,   o_t = tau q_t^T S_t
//
// For a chunk of n tokens (rows r = 0 .. n - 1) behind the state S:
//   O = P V + tau lambda^(r+1) Q S,  P_rc = tau lambda^(r-c) q_r.k_c  (c <= r)
//   S' = lambda^n S + sum_c lambda^(n-1-c) k_c v_c^T
// All exponents of lambda are >= 0, so nothing overflows, and no exponent is larger than a
// chunk's or a segment's length.
//
// The gradients are the same operator over other operands:
//   dQ_t = tau sum_{j<=t} lambda^(t-j) (dO_t.V_j) K_j + ..  query dO, key V, value K, state S^T
//   dK_j = tau sum_{t>=j} lambda^(t-j) (V_j.dO_t) Q_t       query V, key dO, value Q, reversed time
//   dV_j = tau sum_{t>=j} lambda^(t-j) (K_j.Q_t) dO_t       query K, key Q, value dO, reversed time
// the last two with one state, R_j = tau sum_{t>=j} lambda^(t-j) q_t dO_t^T + lambda^(N-j) dS_N
// (and its transpose).  In reversed time the state carries one factor of lambda more
// and the readout one less (`shift`), so that it starts as dS_N and ends as dS_0
// without a division by lambda.
//
// A sequence is cut into segments so that the chip is full: a pass sums each
// segment's own state, a scan adds up the states before each segment, and the
// readout walks a segment's 64-token chunks with the state in registers.
// States, scores and outputs are float32; operands of the matrix cores are
// in the storage type, those formed here (weighted values, scores, states) as sums of two or three
// bfloat16 parts, so that nothing but a row's output is rounded to 8 bits.
#include "common.hpp"
#include "elsaa.h"
#include "internal.hpp"
#include "tile.hpp"

namespace elsaa {
namespace {

constexpr int kChunk = tile::kRows;      // 64 tokens

constexpr int kThreads = 256;
// One operator over rows [B, H, N, D]: `rev` walks the tokens last to first.
struct StateRole {
    const void *k, *v;
    int64_t kb, vb;          // batch strides (elements)
    int rev, shift;
    float s_tok;             // factor of a token's product
    float* slots;            // [BH][nseg + 1] states (slot_index): slot s holds the state before segment s
    const float* init;       // state before the first token, or null
    float* fin;              // state behind the last token, or null
};
struct OutRole {
    const void *q, *k, *v;
    void* o;
    int64_t qb, kb, vb, ob;
    int rev, shift;
    float s_tok, s_out;      // factors of a token's product in the state and of the state's readout
    const float* slots;      // states before the segments (or their transposes)
    const float* first;      // state before segment 0, [BH][D][D], where there is no slot for it; null: zero
    int slot0;               // slot 0 holds it
    int trans;
};
struct DecayArgs {
    StateRole st[2];
    OutRole out[3];
    const float* log_decay;
    const int32_t* lengths;
    int H, N, nseg, seg_len;
    float tau;
    int zero_tail;           // rows behind a sequence's length are set to zero
};

__device__ __forceinline__ int length_of(const DecayArgs& a, int b)
{
    return a.lengths ? min(max(a.lengths[b], 0), a.N) : a.N;
}

// Four consecutive values of a row in the storage type, one store (in
// bfloat16 two conversions, each of two values).
template <class T>
__device__ __forceinline__ void put4(typename T::store_t* p, f32x4 v)
{
    if constexpr (T::bytes == 2) *(bf16x4*)p = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    else *(f32x4*)p = v;
}

// log2 of the head's decay.  Minus infinity would give NaN at distance 0;
// 2^-10000 is zero at every other distance as well.
__device__ __forceinline__ float log2_decay(const DecayArgs& a, int h)
{
    const float l = a.log_decay[h] * kLog2e;
    return l < -1e4f ? -1e4f : l;
}

__device__ __forceinline__ float power(float lg, int n) { return fast_exp2(lg * (float)n); }

// Token of position t of a walk over `len` tokens.
__device__ __forceinline__ int token_of(int t, int len, int rev) { return rev ? len - 1 - t : t; }

// Rows of a chunk through registers, C columns from c0 on: the byte offsets of
// the pieces this thread stages, the same in every operand.  Rows behind the chunk's n repeat
// its last one (every load is in the sequence and none is behind a branch, so
// the waits count exactly); put() clears them.
template <class T, int D, int C>
struct Rows {
    using TL = tile::Tile<T, C, kThreads>;
    using S = typename T::store_t;
    static constexpr int P = TL::PER_THREAD;
    uint32_t off[P];
    __device__ __forceinline__ void at(int t0, int n, int len, int rev, int c0 = 0)
    {
#pragma unroll
        for (int j = 0; j < P; ++j)
            off[j] = (uint32_t)token_of(t0 + min(TL::row_of(j), n - 1), len, rev) * (uint32_t)(D * T::bytes) +
                     (uint32_t)TL::chunk_of(j) * 16u + (uint32_t)(c0 * T::bytes);
    }
    __device__ __forceinline__ void get(const S* X, uint4 (&r)[P]) const
    {
#pragma unroll
        for (int j = 0; j < P; ++j) r[j] = ldg16((const char*)X + off[j]);
    }
    __device__ static __forceinline__ void put(S* t, const uint4 (&r)[P], int n)
    {
        if (n == kChunk) {
            TL::store(t, r);
        } else {
#pragma unroll
            for (int j = 0; j < P; ++j)
                *(uint4*)&t[TL::off(TL::row_of(j), TL::chunk_of(j))] = TL::row_of(j) < n ? r[j] : make_uint4(0, 0, 0, 0);
        }
    }
};

// Sign bits of the bfloat16 halves (of the float32 words) set where a value is
// an infinity or NaN; the other bits mean nothing.
template <class T>
__device__ __forceinline__ uint32_t not_finite(uint4 v)
{
    constexpr uint32_t E = T::bytes == 2 ? 0x7f807f80u : 0x7f800000u, ONE = T::bytes == 2 ? 0x00800080u : 0x00800000u;
    return ((v.x & E) + ONE) | ((v.y & E) + ONE) | ((v.z & E) + ONE) | ((v.w & E) + ONE);
}
template <class T> constexpr uint32_t kSigns = T::bytes == 2 ? 0x80008000u : 0x80000000u;

// Q is kept in LDS with the four-element units 0 .. 7 of every 32 columns in
// the order 0 4 1 5 2 6 3 7: the readout's operand of lane group g, columns 4 g .. and 16 + 4 g ..
// (the state's rows as its accumulators hold them), is then 16 contiguous bytes.
template <class T, int D>
__device__ __forceinline__ void put_q(typename T::store_t* t, const uint4 (&r)[Rows<T, D, D>::P], int n)
{
    using TL = typename Rows<T, D, D>::TL;
#pragma unroll
    for (int j = 0; j < Rows<T, D, D>::P; ++j) {
        const uint4 v = n == kChunk || TL::row_of(j) < n ? r[j] : make_uint4(0, 0, 0, 0);
        typename T::store_t* row = t + TL::row(TL::row_of(j));
        const int c = TL::chunk_of(j);
        if constexpr (T::bytes == 2) {
            const int pos = 32 * (c >> 2) + 16 * (c & 1) + 4 * ((c >> 1) & 1);
            *(uint2*)(row + pos) = make_uint2(v.x, v.y);
            *(uint2*)(row + pos + 8) = make_uint2(v.z, v.w);
        } else {
            *(uint4*)(row + 32 * (c >> 3) + 8 * (c & 3) + 4 * ((c >> 2) & 1)) = v;
        }
    }
}
// Columns 32 s + 8 g .. + 7 of row r of such a tile.
template <class T, int D>
__device__ __forceinline__ typename T::frag_t row8_q(const typename T::store_t* t, int r, int s, int g)
{
    const typename T::store_t* p = t + Rows<T, D, D>::TL::row(r) + 32 * s + 16 * (g & 1) + 4 * (g >> 1);
    return T::ld44(p, p + 8);
}

// States between the passes are kept as 16 x 16 blocks of 64 lanes' four
// values, the accumulator layout: lane (g, i) of block (row / 16, column / 16) holds rows 4 g + r
// of column i.
template <int D>
__device__ __forceinline__ int slot_index(int row, int col)
{
    return ((((col >> 4) * (D / 16) + (row >> 4)) * 64) + ((row >> 2) & 3) * 16 + (col & 15)) * 4 + (row & 3);
}

// The part of a state that a wave holds: 16 NV columns from c on, lane (g, i)
// rows 16 a + 4 g + r of columns c + 16 n + i, r = 0 .. 3.
template <int D, int NV>
struct State {
    static constexpr int NA = D / 16;
    f32x4 s[NA][NV];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int n = 0; n < NV; ++n) s[a][n] = f32x4{0, 0, 0, 0};
    }
    // from a slot, or from the transpose of one
    __device__ __forceinline__ void load(const float* p, int c, int trans)
    {
        const int lane = threadIdx.x & 63, row = 4 * (lane >> 4), col = c + (lane & 15);
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                if (!trans) {
                    s[a][n] = *(const f32x4*)(p + slot_index<D>(16 * a + row, col + 16 * n));
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[a][n][r] = p[slot_index<D>(col + 16 * n, 16 * a + row + r)];
                }
            }
    }
    // from a row-major state
    __device__ __forceinline__ void load_rows(const float* p, int c, int trans)
    {
        const int lane = threadIdx.x & 63, row = 4 * (lane >> 4), col = c + (lane & 15);
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                if (trans) {
                    s[a][n] = *(const f32x4*)(p + (col + 16 * n) * D + 16 * a + row);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[a][n][r] = p[(16 * a + row + r) * D + col + 16 * n];
                }
            }
    }
    __device__ __forceinline__ void store(float* p, int c) const
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int n = 0; n < NV; ++n)
                *(f32x4*)(p + slot_index<D>(16 * a + 4 * (lane >> 4), c + 16 * n + (lane & 15))) = s[a][n];
    }
};

// Workgroup -> (item, part of the columns).  Workgroups go to the eight XCDs
// in turn, so the parts of an item are eight ids apart: they read the same rows of Q
// and K at about the same time, through one XCD's L2.
template <int P>
__device__ __forceinline__ bool item_of(int items, int& item, int& part)
{
    part = (blockIdx.x / 8) % P;
    item = blockIdx.x / (8 * P) * 8 + blockIdx.x % 8;
    return item < items;
}

// Weights of the tokens of a chunk of n rows in a lane's k-slots: token 32 ks + 8 g + j.
__device__ __forceinline__ void token_weights(float lg, int n, int shift, float s_tok, float (&wt)[2][8])
{
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int t = 32 * ks + 8 * g + j;
            wt[ks][j] = t < n ? s_tok * power(lg, n - 1 - t + shift) : 0.f;
        }
}

// x rounded to an operand of the storage type, x left with what is missing.
template <class T>
__device__ __forceinline__ typename T::frag_t take_part(float (&x)[8], bool more)
{
    const typename T::frag_t f = T::pack(x);
    if constexpr (T::bytes == 2) {
        typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
        const u32x4_t u = __builtin_bit_cast(u32x4_t, f);
#pragma unroll
        for (int j = 0; more && j < 4; ++j) {
            x[2 * j] -= __uint_as_float(u[j] << 16);
            x[2 * j + 1] -= __uint_as_float(u[j] & 0xffff0000u);
        }
    }
    return f;
}

// S = keep S + K^T (wt V) over a chunk in LDS.  The weighted values are float32;
// in bfloat16 storage they become the sum of PARTS bfloat16 operands (8 bits each).
template <class T, int D, int PARTS, int NV>
__device__ __forceinline__ void update_state(State<D, NV>& st, const typename T::store_t* Ks, const typename T::store_t* Vs,
                                             float keep, const float (&wt)[2][8])
{
    using TK = tile::Tile<T, D, kThreads>;
    using TV = tile::Tile<T, 64 * NV, kThreads>;
    using F = typename T::frag_t;
    constexpr int NA = State<D, NV>::NA;
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int n = 0; n < NV; ++n) st.s[a][n] *= keep;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        F part[NV][PARTS];
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const F v = TV::col8(Vs, 32 * ks, 16 * NV * (threadIdx.x >> 6) + 16 * n);
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (float)v[j] * wt[ks][j];
#pragma unroll
            for (int p = 0; p < PARTS; ++p) part[n][p] = take_part<T>(x, p + 1 < PARTS);
        }
        // (four rows' operands at a time, the next four requested ahead: left
        // to itself the compiler requests all of them and spills)
        F k[2][4];
#pragma unroll
        for (int a = 0; a < 4; ++a) k[0][a] = TK::col8(Ks, 32 * ks, 16 * a);
#pragma unroll
        for (int a0 = 0; a0 < NA; a0 += 4) {
            if (a0 + 4 < NA) {
#pragma unroll
                for (int a = 0; a < 4; ++a) k[(a0 / 4 + 1) & 1][a] = TK::col8(Ks, 32 * ks, 16 * (a0 + 4 + a));
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
#pragma unroll
                for (int a = 0; a < 4; ++a)
#pragma unroll
                    for (int n = 0; n < NV; ++n) st.s[a0 + a][n] = T::mma(k[(a0 / 4) & 1][a], part[n][p], st.s[a0 + a][n]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Segment's own state, COLS columns of it, to the slot behind it.
template <class T, int D, int COLS>
__global__ __launch_bounds__(kThreads, T::bytes == 4 ? 1 : COLS == 128 ? 2 : D == 128 ? 3 : 4) void decay_state_kernel(DecayArgs a, int count, int items)
{
    using RK = Rows<T, D, D>;
    constexpr int NV = COLS / 64;
    using RV = Rows<T, D, COLS>;
    using S = typename T::store_t;
    constexpr int PARTS = T::kSplit ? 3 : 1;           // (a state is a float32 result)
    __shared__ __attribute__((aligned(16))) S Ks[2][RK::TL::elems(kChunk)], Vs[2][RV::TL::elems(kChunk)];
    const StateRole& ro = a.st[blockIdx.y];
    int item, part;
    if (!item_of<D / COLS>(items, item, part)) return;
    const int bh = item / count, seg = item - bh * count;
    const int b = bh / a.H, h = bh - b * a.H;
    const int len = length_of(a, b), t0 = seg * a.seg_len, t1 = min(len, t0 + a.seg_len);
    const float lg = log2_decay(a, h);
    const S* K = (const S*)ro.k + b * ro.kb + (int64_t)h * a.N * D;
    const S* V = (const S*)ro.v + b * ro.vb + (int64_t)h * a.N * D;
    State<D, NV> st;
    st.zero();
    if (t0 < t1) {
        const int last = t0 + (t1 - 1 - t0) / kChunk * kChunk;
        uint4 kr[RK::P], vr[RV::P];
        auto fetch = [&](int t) {
            RK rk;
            RV rv;
            t = min(t, last);
            rk.at(t, t1 - t, len, ro.rev);
            rv.at(t, t1 - t, len, ro.rev, COLS * part);
            rk.get(K, kr);
            rv.get(V, vr);
        };
        float wt[2][8];
        const float keep = power(lg, kChunk);
        token_weights(lg, kChunk, ro.shift, ro.s_tok, wt);
        fetch(t0);
        for (int t = t0, buf = 0; t < t1; t += kChunk, buf ^= 1) {
            const int n = min(kChunk, t1 - t);
            RK::put(Ks[buf], kr, n);
            RV::put(Vs[buf], vr, n);
            fetch(t + kChunk);
            __syncthreads();       // (the buffer's last readers are behind the barrier of the chunk between)
            if (n < kChunk) token_weights(lg, n, ro.shift, ro.s_tok, wt);
            update_state<T, D, PARTS>(st, Ks[buf], Vs[buf], n < kChunk ? power(lg, n) : keep, wt);
        }
    }
    st.store(ro.slots + ((int64_t)bh * (a.nseg + 1) + seg + 1) * D * D, COLS * part + 16 * NV * (threadIdx.x >> 6));
}

// Slots of segment states -> states before each segment; the last sum is the
// state behind the last token.  Eight slots are requested at a time: their
// addresses do not depend on the sum.  A workgroup takes 1024 values of a
// state, and further ones where there are more than the launch has workgroups
// (a launch holds 2^24 of them, fewer than 2^20 states of 128 x 128).
constexpr int kScanGroups = 1 << 16;
template <int D>
__global__ __launch_bounds__(256) void decay_scan_kernel(DecayArgs a, int count, int total)
{
    const StateRole& ro = a.st[blockIdx.y];
    constexpr int PER = D * D / 4 / 256;               // workgroups a (b, h)
    for (int wg = blockIdx.x; wg < total; wg += gridDim.x) {
        const int bh = wg / PER, e = (wg - bh * PER) * 256 + threadIdx.x;
        const int b = bh / a.H, h = bh - b * a.H;
        const int len = length_of(a, b);
        const float lg = log2_decay(a, h);
        f32x4* slot = (f32x4*)(ro.slots + (int64_t)bh * (a.nseg + 1) * D * D) + e;
        constexpr int64_t step = D * D / 4;
        // (row, column) of the first of this thread's four values (rows row .. row + 3)
        const int lane = e & 63, blk = e >> 6;
        const int row = 16 * (blk % (D / 16)) + 4 * (lane >> 4), col = 16 * (blk / (D / 16)) + (lane & 15);
        const int64_t user = (int64_t)bh * D * D + row * D + col;
        f32x4 run = {0, 0, 0, 0};
        if (ro.init) {
#pragma unroll
            for (int r = 0; r < 4; ++r) run[r] = ro.init[user + r * D];
            slot[0] = run;                                  // (`fin` may be `init`)
        }
        constexpr int U = 8;
        for (int s0 = 0; s0 < count; s0 += U) {
            f32x4 own[U];
#pragma unroll
            for (int u = 0; u < U; ++u) own[u] = slot[min(s0 + u + 1, count) * step];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int s = s0 + u;
                if (s >= count) break;
                run = run * power(lg, min(max(len - s * a.seg_len, 0), a.seg_len)) + own[u];
                if (s + 1 < a.nseg) slot[(s + 1) * step] = run;
            }
        }
        if (ro.fin) {
#pragma unroll
            for (int r = 0; r < 4; ++r) ro.fin[user + r * D] = run[r];
        }
    }
}

// The readout of a segment's rows from position t on, token by token, for
// segments with an infinity or NaN among the values: in a chunk it would meet
// the zeros of P in the rows before its token, and 0 x infinity is NaN.  The recurrence
// from the segment's first token, float32 throughout, 1.2 to 1.8 us a token (16
// heads of 16384 x 128 with one NaN, segments of 512 tokens: 0.85 ms where the chunks alone
// take 0.12).  Thread (i, c): rows i, i + RT, .. of four columns, sums over the rows in `red`.
template <class T, int D, int COLS>
__device__ void decay_walk(const DecayArgs& a, const OutRole& ro, const float* slot, const float* first, const typename T::store_t* Q,
                           const typename T::store_t* K, const typename T::store_t* V, typename T::store_t* O, int c0, float lg, int len,
                           int t0, int t, int t1, f32x4* red)
{
    constexpr int CG = COLS / 4, RT = kThreads / CG;
    const int c = threadIdx.x % CG, i = threadIdx.x / CG, col = c0 + 4 * c;
    f32x4 s[D / RT];
    auto load = [&](auto at) {
#pragma unroll
        for (int j = 0; j < D / RT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[j][e] = at(ro.trans ? col + e : i + j * RT, ro.trans ? i + j * RT : col + e);
    };
    if (slot) load([&](int x, int y) { return slot[slot_index<D>(x, y)]; });
    else if (first) load([&](int x, int y) { return first[x * D + y]; });
    else load([](int, int) { return 0.f; });
    const float before = power(lg, 1 - ro.shift), behind = power(lg, ro.shift);
    for (int x = t0; x < t1; ++x) {
        const int64_t row = (int64_t)token_of(x, len, ro.rev) * D;
        const f32x4 v = load4<T>(V + row + 4 * c);
        f32x4 o = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < D / RT; ++j) {
            s[j] = s[j] * before + v * (ro.s_tok * T::load(K[row + i + j * RT]));
            o += s[j] * T::load(Q[row + i + j * RT]);
            s[j] *= behind;
        }
        if (x < t) continue;
        __syncthreads();
        red[i * CG + c] = o;
        __syncthreads();
        if (i == 0) {
            for (int j = 1; j < RT; ++j) o += red[j * CG + c];
            store4<T>(O + row + 4 * c, o * ro.s_out);
        }
    }
}

// Readout of one segment, COLS columns.
template <class T, int D, int COLS>
__global__ __launch_bounds__(kThreads, T::bytes == 4 ? 128 / D : D == 128 ? 2 : 3) void decay_out_kernel(DecayArgs a, int items)
{
    using RK = Rows<T, D, D>;
    constexpr int NV = COLS / 64;
    using RV = Rows<T, D, COLS>;
    using TK = typename RK::TL;
    using TV = typename RV::TL;
    using TP = tile::Tile<T, kChunk, kThreads>;
    using S = typename T::store_t;
    using F = typename T::frag_t;
    __shared__ __attribute__((aligned(16))) S Qs[TK::elems(kChunk)], Ks[TK::elems(kChunk)], Vs[TV::elems(kChunk)];
    // Scores and the state are operands in two bfloat16 parts (float32: one), so
    // that a row is as exact as its own rounding: error against exact sums 1.66e-3
    // of a bfloat16 tensor's norm, and 2.35e-3 with one part of each.  (16 heads of 16384 x
    // 128: 131 us, and 122 with one part, backward 270 and 242; 64 heads of 4096 x 64: 54 and 50,
    // backward 110 and 102.)
    constexpr int PARTS = T::kSplit ? 2 : 1;
    __shared__ __attribute__((aligned(16))) S Ps[PARTS][TP::elems(kChunk)];
    __shared__ int special;                            // a value of V is an infinity or NaN
    const OutRole& ro = a.out[blockIdx.y];
    int item, part;
    if (!item_of<D / COLS>(items, item, part)) return;
    const int bh = item / a.nseg, seg = item - bh * a.nseg;
    const int b = bh / a.H, h = bh - b * a.H;
    const int len = length_of(a, b), t0 = seg * a.seg_len, t1 = min(len, t0 + a.seg_len);
    const float lg = log2_decay(a, h);
    const int64_t head = (int64_t)h * a.N * D;
    const S* Q = (const S*)ro.q + b * ro.qb + head;
    const S* K = (const S*)ro.k + b * ro.kb + head;
    const S* V = (const S*)ro.v + b * ro.vb + head;
    S* O = (S*)ro.o + b * ro.ob + head + COLS * part;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, g = lane >> 4, i = lane & 15;

    if (a.zero_tail) {
        // rows of this segment's positions behind the sequence (the same tokens in either direction)
        const int z0 = max(len, t0), z1 = min(a.N, t0 + a.seg_len);
        for (int x = threadIdx.x; x < (z1 - z0) * TV::CPR; x += kThreads)
            stg16(O + (int64_t)(z0 + x / TV::CPR) * D + x % TV::CPR * TV::EPC, make_uint4(0, 0, 0, 0));
    }
    if (t0 >= t1) return;
    if (threadIdx.x == 0) special = 0;

    const int last = t0 + (t1 - 1 - t0) / kChunk * kChunk;
    uint4 qr[RK::P], kr[RK::P], vr[RV::P];
    auto fetch_q = [&](int t) {
        RK rk;
        t = min(t, last);
        rk.at(t, t1 - t, len, ro.rev);
        rk.get(Q, qr);
    };
    auto fetch_kv = [&](int t) {
        RK rk;
        RV rv;
        t = min(t, last);
        rk.at(t, t1 - t, len, ro.rev);
        rv.at(t, t1 - t, len, ro.rev, COLS * part);
        rk.get(K, kr);
        rv.get(V, vr);
    };
    // At 128 columns a workgroup 256 registers do not hold the next rows and both
    // parts of the state: K and V are requested behind its readout, and what depends on the
    // lane alone is formed in every chunk (all at its start, with registers
    // spilled: the same 16 heads 154 us, backward 330).
    constexpr bool LATE = T::bytes == 2;
    fetch_q(t0);
    fetch_kv(t0);
    State<D, NV> st;
    const int c0 = COLS * part + 16 * NV * w;
    if (seg || ro.slot0) st.load(ro.slots + ((int64_t)bh * (a.nseg + 1) + seg) * D * D, c0, ro.trans);
    else if (ro.first) st.load_rows(ro.first + (int64_t)bh * D * D, c0, ro.trans);
    else st.zero();

    // factors that are the same in every chunk: scores of row 16 w + i with
    // rows 16 kt + 4 g + r, readout of rows 16 qt + i, tokens in the state
    float fp[4][4], fq[4], wt[2][8];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int gap = 16 * w + i - (16 * kt + 4 * g + r);
            fp[kt][r] = gap >= 0 ? a.tau * power(lg, gap) : 0.f;
        }
#pragma unroll
    for (int qt = 0; qt < 4; ++qt) fq[qt] = ro.s_out * power(lg, 16 * qt + i + 1 - ro.shift);
    token_weights(lg, kChunk, ro.shift, ro.s_tok, wt);
    const float keep = power(lg, kChunk);

    // One chunk; whole ones carry no conditions, so that the waits for the
    // next rows do not wait for this chunk's stores as well.  False, and
    // nothing written, where the values are not all finite.
    auto chunk = [&](int t, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        const int n = WHOLE ? kChunk : t1 - t;
        uint32_t nf = 0;
#pragma unroll
        for (int j = 0; j < RV::P; ++j) nf |= not_finite<T>(vr[j]);
        __syncthreads();
        if (nf & kSigns<T>) special = 1;
        put_q<T, D>(Qs, qr, n);
        RK::put(Ks, kr, n);
        RV::put(Vs, vr, n);
        fetch_q(t + kChunk);
        if (!LATE) fetch_kv(t + kChunk);
        __syncthreads();
        int lane = threadIdx.x & 63;
        if (LATE) asm volatile("" : "+v"(lane));
        const int g = lane >> 4, i = lane & 15;
        // scores of this wave's 16 rows with rows 16 kt .. on, and a tile of zeros where
        // the readout, in steps of 32 rows, reads past the diagonal
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) {
            if (kt > (w | 1)) break;
            f32x4 p = {0, 0, 0, 0};
            if (kt <= w) {
#pragma unroll
                for (int s = 0; s < D / 32; ++s)
                    p = T::mma(TK::row8(Ks, 16 * kt + i, 32 * s + 8 * g), row8_q<T, D>(Qs, 16 * w + i, s, g), p);
            }
            // (by selection on the diagonal: an infinite score there would give NaN)
            if (kt < w) {
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] *= fp[kt][r];
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] = kt == w && i >= 4 * g + r ? p[r] * fp[kt][r] : 0.f;
            }
            const int at = TP::row(16 * w + i) + 16 * kt + 4 * g;
            put4<T>(&Ps[0][at], p);
            if constexpr (PARTS == 2) {
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] -= (float)(__bf16)p[r];
                put4<T>(&Ps[1][at], p);
            }
        }
        // O^T = S^T Q^T, rows of O^T in this wave's columns
        f32x4 o[NV][4];
#pragma unroll
        for (int m = 0; m < NV; ++m)
#pragma unroll
            for (int qt = 0; qt < 4; ++qt) o[m][qt] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            F sf[PARTS][NV];
#pragma unroll
            for (int m = 0; m < NV; ++m) {
                float x[8];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[r] = st.s[2 * s][m][r];
                    x[4 + r] = st.s[2 * s + 1][m][r];
                }
#pragma unroll
                for (int p = 0; p < PARTS; ++p) sf[p][m] = take_part<T>(x, p + 1 < PARTS);
            }
#pragma unroll
            for (int qt = 0; qt < 4; ++qt) {
                const F q = TK::row8(Qs, 16 * qt + i, 32 * s + 8 * g);
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int m = 0; m < NV; ++m) o[m][qt] = T::mma(sf[p][m], q, o[m][qt]);
            }
        }
#pragma unroll
        for (int m = 0; m < NV; ++m)
#pragma unroll
            for (int qt = 0; qt < 4; ++qt) o[m][qt] *= fq[qt];
        if (LATE) fetch_kv(t + kChunk);
        const int stop = special;
        __syncthreads();
        if (__builtin_amdgcn_readfirstlane(stop)) return false;
        // O^T += V^T P^T
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            F v[NV];
#pragma unroll
            for (int m = 0; m < NV; ++m) v[m] = TV::col8(Vs, 32 * ks, 16 * NV * w + 16 * m);
#pragma unroll
            for (int qt = 2 * ks; qt < 4; ++qt) {
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    const F pf = TP::row8(Ps[p], 16 * qt + i, 32 * ks + 8 * g);
#pragma unroll
                    for (int m = 0; m < NV; ++m) o[m][qt] = T::mma(v[m], pf, o[m][qt]);
                }
            }
        }
#pragma unroll
        for (int qt = 0; qt < 4; ++qt) {
            const int r = 16 * qt + i;
            if (WHOLE || r < n) {
                S* row = O + (int64_t)token_of(t + r, len, ro.rev) * D + 16 * NV * w + 4 * g;
#pragma unroll
                for (int m = 0; m < NV; ++m) put4<T>(row + 16 * m, o[m][qt]);
            }
        }
        // (a short chunk is the last one)
        if (WHOLE) update_state<T, D, PARTS>(st, Ks, Vs, keep, wt);
        return true;
    };
    int t = t0;
    bool done = true;
    for (; done && t + kChunk <= t1; t += done ? kChunk : 0) done = chunk(t, std::true_type{});
    if (done && t < t1) done = chunk(t, std::false_type{});
    if (!done)
        decay_walk<T, D, COLS>(a, ro, seg || ro.slot0 ? ro.slots + ((int64_t)bh * (a.nseg + 1) + seg) * D * D : nullptr,
                               ro.first ? ro.first + (int64_t)bh * D * D : nullptr, Q, K, V + COLS * part, O, COLS * part, lg, len, t0, t,
                               t1, (f32x4*)Qs);
}

// One token: state columns [16 blockIdx.y, +16) of one (b, h).  Thread (i, c):
// rows i, i + RT, .. of column group c (4 floats); partial sums over rows meet in LDS.
template <class T, int D>
__global__ __launch_bounds__(256) void decay_step_kernel(DecayArgs a, const float* state, float* state_out)
{
    using S = typename T::store_t;
    const OutRole& ro = a.out[0];
    constexpr int CG = 8, CW = 4 * CG, RT = 256 / CG;          // 32 columns a workgroup, 32 rows at a time
    __shared__ f32x4 red[RT][CG];
    const int bh = blockIdx.x, b = bh / a.H, h = bh - b * a.H;
    const int c = blockIdx.y * CW + 4 * (threadIdx.x % CG), r0 = threadIdx.x / CG;
    const int64_t head = (int64_t)h * D;
    const S* q = (const S*)ro.q + b * ro.qb + head;
    const S* k = (const S*)ro.k + b * ro.kb + head;
    const S* v = (const S*)ro.v + b * ro.vb + head;
    const float lam = power(log2_decay(a, h), 1);
    const int64_t base = (int64_t)bh * D * D + c;
    f32x4 s[D / RT];
#pragma unroll
    for (int j = 0; j < D / RT; ++j) s[j] = *(const f32x4*)(state + base + (int64_t)(r0 + j * RT) * D);
    const f32x4 vv = load4<T>(v + c);
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < D / RT; ++j) {
        const int r = r0 + j * RT;
        s[j] = s[j] * lam + vv * T::load(k[r]);
        *(f32x4*)(state_out + base + (int64_t)r * D) = s[j];
        o += s[j] * T::load(q[r]);
    }
    red[r0][threadIdx.x % CG] = o;
    __syncthreads();
    if (threadIdx.x < CG) {
        f32x4 t = red[0][threadIdx.x];
#pragma unroll
        for (int j = 1; j < RT; ++j) t += red[j][threadIdx.x];
        store4<T>((S*)ro.o + b * ro.ob + head + c, t * a.tau);
    }
}

struct Plan {
    int nseg, seg_len;
    size_t slots;            // floats of one set of slots
};

// Segments of whole chunks.  More segments fill the chip better and cost
// states written, scanned and read.  Forward: two workgroups a compute unit from eight chunks a
// segment on (64 heads of 4096 x 64: 54 us with 512 workgroups, 64 with 256; 16 heads of 16384 x
// 128: 127 and 126), one below (16 heads of 4096 x 128: 46 with 256, 56 with 512).
// Backward: its three readouts in one round of what is resident (16 heads of 16384 x 128: 269 us with
// 3 x 160 workgroups, 290 with 3 x 512; 128 heads of 2048: 209 with one segment a head, no
// state pass, and 266 with four), three a compute unit at 64 in bfloat16 (64
// heads of 4096: 111 with four segments, 139 with two).  Float32 at 128 takes two workgroups a
// segment.
Plan plan_of(const elsaa_decay_desc* d, bool backward)
{
    Plan p;
    const bool f32 = d->dtype == ELSAA_F32;
    const int64_t bh = (int64_t)d->B * d->H, chunks = (d->N + kChunk - 1) / kChunk;
    auto most = [](int64_t x) { return x < 1 ? (int64_t)1 : x; };
    const int64_t room = (!f32 && d->d_h == 64 && backward ? 768 : 512) / (f32 ? d->d_h / 64 : 1);
    int64_t n;
    if (backward) {
        n = most(room / (3 * bh));
    } else {
        n = most(room / bh);
        if (chunks < 8 * n) n = most(room / 2 / bh);
    }
    int64_t per = (chunks + n - 1) / n;
    if (per < 2 && (backward || !f32)) per = 2;      // (a float32 chunk costs more than its state)
    p.seg_len = (int)per * kChunk;
    p.nseg = (int)((chunks + per - 1) / per);
    p.slots = (size_t)bh * (p.nseg + 1) * d->d_h * d->d_h;
    return p;
}

int validate(const elsaa_decay_desc* d, int64_t (&batch)[7])
{
    if (!d) return api_fail(ELSAA_ERR_INVALID_ARG, "desc is NULL");
    if (d->B < 1 || d->H < 1 || d->N < 1)
        return api_fail(ELSAA_ERR_INVALID_ARG, "B, H, N must be >= 1 (got %d, %d, %d)", d->B, d->H, d->N);
    if (d->d_h != 64 && d->d_h != 128) return api_fail(ELSAA_ERR_UNSUPPORTED, "d_h must be 64 or 128 (got %d)", d->d_h);
    if (d->dtype != ELSAA_F32 && d->dtype != ELSAA_BF16) return api_fail(ELSAA_ERR_INVALID_ARG, "unknown dtype %d", d->dtype);
    const int64_t el = d->dtype == ELSAA_BF16 ? 2 : 4, per = (int64_t)d->N * d->d_h;
    if (per * el >= ((int64_t)1 << 32)) return api_fail(ELSAA_ERR_UNSUPPORTED, "N * d_h * element bytes must be below 2^32");
    if ((int64_t)d->B * d->H > (1 << 22))
        return api_fail(ELSAA_ERR_UNSUPPORTED, "B * H must be at most 2^22 (got %lld)", (long long)d->B * d->H);
    const int64_t in[7] = {d->q_batch, d->k_batch, d->v_batch, d->o_batch, d->dq_batch, d->dk_batch, d->dv_batch};
    for (int i = 0; i < 7; ++i) {
        batch[i] = in[i] ? in[i] : per * d->H;
        if (batch[i] < per * d->H || batch[i] % 8 != 0)
            return api_fail(ELSAA_ERR_INVALID_ARG, "batch strides must be >= H * N * d_h and multiples of 8 (got %lld)",
                            (long long)in[i]);
    }
    return ELSAA_OK;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

int check_workspace(const void* ws, size_t have, size_t need)
{
    if (need == 0) return ELSAA_OK;
    if (!ws) return api_fail(ELSAA_ERR_INVALID_ARG, "workspace is NULL (%zu bytes needed)", need);
    if (have < need) return api_fail(ELSAA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", have, need);
    if (!aligned16(ws)) return api_fail(ELSAA_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    return ELSAA_OK;
}

// Segment states of `states` operators and their scan, then `outs` readouts.  The
// last segment's own state is only needed for a state behind the last token.
//
// A workgroup takes all columns of a state where that is 64 or (bfloat16) 128,
// or 64 of the 128.  Each wave reads the whole of Q and of K from LDS whatever its
// width, and LDS is what halves are slower by where the chip is full (16K
// tokens, 16 heads of 128: 134 us against 122).  Where it is not (up to one
// workgroup a compute unit in the readout, 1.25 in the state pass) they bring twice the
// waves (4K tokens: forward 50 -> 46 us, backward 94 -> 91).  In float32 only
// tiles of 64 columns fit LDS.
template <class T, int D>
hipError_t launch(const DecayArgs& a, int bh, int states, int outs, hipStream_t st)
{
    constexpr int WIDE = T::bytes == 2 ? D : 64;
    bool fin = false;
    for (int i = 0; i < states; ++i) fin |= a.st[i].fin != nullptr;
    const int count = fin ? a.nseg : a.nseg - 1;
    auto grid = [&](int items, int roles, int cols) { return dim3((items + 7) / 8 * 8 * (D / cols), roles); };
    auto narrow = [](int items, int roles, int lim) { return WIDE > 64 && (int64_t)items * roles <= lim; };
    if (count > 0) {
        const int items = bh * count;
        if (narrow(items, states, 320))
            ELSAA_LAUNCH("decay_state_half", (decay_state_kernel<T, D, 64>), grid(items, states, 64), dim3(kThreads), 0, st, a, count, items);
        else
            ELSAA_LAUNCH("decay_state", (decay_state_kernel<T, D, WIDE>), grid(items, states, WIDE), dim3(kThreads), 0, st, a, count,
                         items);
        const int total = bh * (D * D / 1024);
        ELSAA_LAUNCH("decay_scan", decay_scan_kernel<D>, dim3(total < kScanGroups ? total : kScanGroups, states), dim3(256), 0, st, a,
                     count, total);
    }
    const int items = bh * a.nseg;
    if (narrow(items, outs, 256))
        ELSAA_LAUNCH("decay_out_half", (decay_out_kernel<T, D, 64>), grid(items, outs, 64), dim3(kThreads), 0, st, a, items);
    else
        ELSAA_LAUNCH("decay_out", (decay_out_kernel<T, D, WIDE>), grid(items, outs, WIDE), dim3(kThreads), 0, st, a, items);
    return hipGetLastError();
}

hipError_t launch_any(const elsaa_decay_desc* d, const DecayArgs& a, int states, int outs, hipStream_t st)
{
    const int bh = d->B * d->H;
    if (d->dtype == ELSAA_BF16)
        return d->d_h == 128 ? launch<BF16, 128>(a, bh, states, outs, st) : launch<BF16, 64>(a, bh, states, outs, st);
    return d->d_h == 128 ? launch<F32, 128>(a, bh, states, outs, st) : launch<F32, 64>(a, bh, states, outs, st);
}

DecayArgs common_args(const elsaa_decay_desc* d, const Plan& p, const float* log_decay, const int32_t* lengths)
{
    DecayArgs a = {};
    a.log_decay = log_decay;
    a.lengths = lengths;
    a.H = d->H; a.N = d->N; a.nseg = p.nseg; a.seg_len = p.seg_len;
    a.tau = d->scale > 0.f ? d->scale : 1.f / sqrtf((float)d->d_h);
    return a;
}

// Where the readout of segment 0 finds its state: slot 0 where the scan ran
// (it copied the caller's there), else the caller's.
void set_first(OutRole& o, const StateRole& s, bool scanned)
{
    o.slots = s.slots;
    o.first = s.init;
    o.slot0 = s.init && scanned;
}

}  // namespace
}  // namespace elsaa

using namespace elsaa;

extern "C" {

int elsaa_decay_workspace_bytes(const elsaa_decay_desc* d, int pass, size_t* bytes)
{
    int64_t batch[7];
    const int rc = validate(d, batch);
    if (rc) return rc;
    if (!bytes) return api_fail(ELSAA_ERR_INVALID_ARG, "bytes is NULL");
    if (pass != 0 && pass != 1) return api_fail(ELSAA_ERR_INVALID_ARG, "pass must be 0 or 1 (got %d)", pass);
    *bytes = plan_of(d, pass == 1).slots * sizeof(float) * (pass ? 2 : 1);
    return ELSAA_OK;
}

int elsaa_decay_fwd(const elsaa_decay_desc* d, const void* Q, const void* K, const void* V, const float* log_decay,
                    const float* state, const int32_t* lengths, void* O, float* state_out,
                    void* workspace, size_t workspace_bytes, hipStream_t stream)
{
    int64_t batch[7];
    int rc = validate(d, batch);
    if (rc) return rc;
    if (!Q || !K || !V || !log_decay || !O) return api_fail(ELSAA_ERR_INVALID_ARG, "a required pointer is NULL");
    if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(state) || !aligned16(state_out))
        return api_fail(ELSAA_ERR_INVALID_ARG, "Q, K, V, O and the states must be 16-byte aligned");
    if (O == Q || O == K || O == V)
        return api_fail(ELSAA_ERR_INVALID_ARG, "O must not be Q, K or V: rows are read by several workgroups");
    const Plan p = plan_of(d, false);
    if ((rc = check_workspace(workspace, workspace_bytes, p.slots * sizeof(float)))) return rc;
    DecayArgs a = common_args(d, p, log_decay, lengths);
    a.st[0] = StateRole{K, V, batch[1], batch[2], 0, 0, 1.f, (float*)workspace, state, state_out};
    a.out[0] = OutRole{Q, K, V, O, batch[0], batch[1], batch[2], batch[3], 0, 0, 1.f, a.tau, nullptr, nullptr, 0, 0};
    set_first(a.out[0], a.st[0], p.nseg > 1 || state_out);
    a.zero_tail = lengths && d->zero_tail;
    const hipError_t e = launch_any(d, a, 1, 1, stream);
    return e == hipSuccess ? ELSAA_OK : api_hip_fail(e, "decay forward");
}

int elsaa_decay_bwd(const elsaa_decay_desc* d, const void* Q, const void* K, const void* V, const float* log_decay,
                    const void* dO, const float* state, const float* dstate_out, const int32_t* lengths,
                    void* dQ, void* dK, void* dV, float* dstate, void* workspace, size_t workspace_bytes,
                    hipStream_t stream)
{
    int64_t batch[7];
    int rc = validate(d, batch);
    if (rc) return rc;
    if (!Q || !K || !V || !log_decay || !dO || !dQ || !dK || !dV)
        return api_fail(ELSAA_ERR_INVALID_ARG, "a required pointer is NULL");
    if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(dO) || !aligned16(dQ) || !aligned16(dK) ||
        !aligned16(dV) || !aligned16(state) || !aligned16(dstate_out) || !aligned16(dstate))
        return api_fail(ELSAA_ERR_INVALID_ARG, "Q, K, V, dO, dQ, dK, dV and the states must be 16-byte aligned");
    const void* in[4] = {Q, K, V, dO};
    for (const void* x : in)
        if (dQ == x || dK == x || dV == x)
            return api_fail(ELSAA_ERR_INVALID_ARG, "dQ, dK and dV must not be Q, K, V or dO: rows are read again behind their gradients");
    if (dQ == dK || dQ == dV || dK == dV || (dstate && dstate == state))
        return api_fail(ELSAA_ERR_INVALID_ARG, "dQ, dK, dV must be different buffers, and dstate not the state");
    const Plan p = plan_of(d, true);
    if ((rc = check_workspace(workspace, workspace_bytes, 2 * p.slots * sizeof(float)))) return rc;
    DecayArgs a = common_args(d, p, log_decay, lengths);
    a.zero_tail = lengths != nullptr;
    float* ws = (float*)workspace;
    a.st[0] = StateRole{K, V, batch[1], batch[2], 0, 0, 1.f, ws, state, nullptr};
    a.st[1] = StateRole{Q, dO, batch[0], batch[3], 1, 1, a.tau, ws + p.slots, dstate_out, dstate};
    a.out[0] = OutRole{dO, V, K, dQ, batch[3], batch[2], batch[1], batch[4], 0, 0, 1.f, a.tau, nullptr, nullptr, 0, 1};
    a.out[1] = OutRole{V, dO, Q, dK, batch[2], batch[3], batch[0], batch[5], 1, 1, a.tau, 1.f, nullptr, nullptr, 0, 1};
    a.out[2] = OutRole{K, Q, dO, dV, batch[1], batch[0], batch[3], batch[6], 1, 1, a.tau, 1.f, nullptr, nullptr, 0, 0};
    const bool scanned = p.nseg > 1 || dstate;
    set_first(a.out[0], a.st[0], scanned);
    set_first(a.out[1], a.st[1], scanned);
    set_first(a.out[2], a.st[1], scanned);
    const hipError_t e = launch_any(d, a, 2, 3, stream);
    return e == hipSuccess ? ELSAA_OK : api_hip_fail(e, "decay backward");
}

int elsaa_decay_step(const elsaa_decay_desc* d, const void* Q, const void* K, const void* V,
                     const float* log_decay, const float* state, void* O, float* state_out, hipStream_t stream)
{
    int64_t batch[7];
    const int rc = validate(d, batch);
    if (rc) return rc;
    if (d->N != 1) return api_fail(ELSAA_ERR_INVALID_ARG, "a step takes one token a sequence (N = 1, got %d)", d->N);
    if (!Q || !K || !V || !log_decay || !state || !O || !state_out)
        return api_fail(ELSAA_ERR_INVALID_ARG, "a required pointer is NULL");
    if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(state) || !aligned16(state_out))
        return api_fail(ELSAA_ERR_INVALID_ARG, "Q, K, V, O and the states must be 16-byte aligned");
    if (O == Q || O == K || O == V)
        return api_fail(ELSAA_ERR_INVALID_ARG, "O must not be Q, K or V: other columns' workgroups read them");
    DecayArgs a = common_args(d, plan_of(d, false), log_decay, nullptr);
    a.out[0].q = Q; a.out[0].k = K; a.out[0].v = V; a.out[0].o = O;
    a.out[0].qb = batch[0]; a.out[0].kb = batch[1]; a.out[0].vb = batch[2]; a.out[0].ob = batch[3];
    const dim3 grid(d->B * d->H, d->d_h / 32);
#define ELSAA_STEP(T, D) ELSAA_LAUNCH("decay_step", (decay_step_kernel<T, D>), grid, dim3(256), 0, stream, a, state, state_out)
    if (d->dtype == ELSAA_BF16) {
        if (d->d_h == 128) ELSAA_STEP(BF16, 128);
        else ELSAA_STEP(BF16, 64);
    } else {
        if (d->d_h == 128) ELSAA_STEP(F32, 128);
        else ELSAA_STEP(F32, 64);
    }
#undef ELSAA_STEP
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? ELSAA_OK : api_hip_fail(e, "decay step");
}

}  // extern "C"
