// Causal attention of runs of new tokens over the paged cache.
#include <cfloat>
#include <type_traits>

#include "cache8.h"
#include "decoder_internal.h"
#include "device_util.h"

namespace npas {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;

template <int DT> __device__ __forceinline__ f32x16 mfma32(uint4 a, uint4 b, f32x16 c)
{
    if constexpr (DT == NPAS_BF16) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Four rows of sixteen 16-bit numbers in LDS, turned round: lane i of sixteen names the four numbers 4 (i & 3) .. of row i >> 2 and gets column i.
__device__ __forceinline__ uint2 read_columns(const uint8_t *p)
{
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p));
}

// Whether one of the two numbers is an infinity or a NaN.
template <int DT> __device__ __forceinline__ bool not_finite2(uint32_t w)
{
    constexpr uint32_t e = DT == NPAS_BF16 ? 0x7f80u : 0x7c00u;
    return (w & e) == e || (w >> 16 & e) == e;
}

// Tile of a workgroup: BM rows (token, query head of the key head) of one sequence.
struct Tile {
    int s, token0, row0, rows; // sequence, its first row of q, first row of the tile and rows from there on within the run
    int at0;                   // position of the run's first token
    int length;
};
// Sequence s owns the places [start G / BM] + s .. of the grid: as many as its rows need, whatever the parting.
template <int BM> __device__ __forceinline__ bool find_tile(const ChunkArgs &a, int place, int group, Tile &t)
{
    auto start = [&](int s) { return max(0, min(a.start[s], a.T)); };
    auto first = [&](int s) { return (int)((long)start(s) * group / BM) + s; };
    const int lane = threadIdx.x & 63;
    int count = 0; // sequences that begin at or before this place
    for (int s0 = 0; s0 < a.c.sequences; s0 += 64) {
        const int s = s0 + lane;
        const int here = __popcll(__ballot(s < a.c.sequences && first(s) <= place));
        count += here;
        if (here < 64) break;
    }
    if (!count) return false;
    t.s = count - 1;
    t.token0 = start(t.s);
    const int run = max(0, start(t.s + 1) - t.token0);
    t.row0 = (place - first(t.s)) * BM;
    t.rows = run * group - t.row0;
    const long room = (long)a.c.table_stride * a.c.page_size;
    int n = max(0, min(a.length[t.s], a.max_length));
    if (n > room) n = (int)room;
    t.length = n;
    t.at0 = n - run;
    return t.rows > 0;
}

// One workgroup a (tile of BM = 32 WM rows, key head, cut).  A wave has 32 rows as columns of 32 x 32 x 16 matrix instructions and walks the tokens in steps of
// 32 NSUB: scores S = K Q^T (row operand: keys from LDS as they lie), running maximum and sum a column, O^T = V^T P^T, where the weights
// are the column operand as the first product leaves them, if a step's tokens are counted so that a lane's half h has tokens 4 h .. 4 h + 3 of
// each eight; the values come out of LDS turned round.  WK waves side by side take different tokens of a step and are joined at the end.
// Keys and values of a step come through registers into one of two places in LDS (16-byte pieces in an order that spreads rows over the banks; 8-bit
// floats become 16-bit numbers on the way) while the other is multiplied; the cache rows of the tokens are looked up two steps ahead.
template <int DT, bool E8, int ND, int NSUB, int WM, int WK>
__global__ __launch_bounds__(64 * WM * WK, ND <= 4 && WK == 1 ? 2 : 1) void chunk_attention_kernel(ChunkArgs a, int places)
{
    constexpr int DP = 32 * ND, BM = 32 * WM, BN = 32 * NSUB * WK, THREADS = 64 * WM * WK, PIECES = DP / 8, STRIDE = DP * 2;
    constexpr int UNITS = E8 ? BN * PIECES / 2 : BN * PIECES, PER = (UNITS + THREADS - 1) / THREADS, IN_ROW = E8 ? PIECES / 2 : PIECES;
    constexpr float TOP = DT == NPAS_BF16 ? 0.f : 15.f; // the largest weight is 2^TOP: fp16 reaches down to 2^-24 only
    __shared__ __align__(16) uint8_t kv[2][2][BN * STRIDE]; // [place][keys, values]
    __shared__ uint32_t ring[3][BN];
    __shared__ uint32_t gone[3][(BN + 63) / 64 * 2]; // a bit a token: not there
    __shared__ float stat[2][WK][32];
    auto swizzle = [](int row) { return ND == 2 ? (row >> 1 & 3) * 2 : ND == 3 ? (row >> 2 & 1) * 2 : (row & 7) * 2; };
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, wm = wave % WM, wk = wave / WM, r = lane & 31, h = lane >> 5, D = a.c.head_dim;
    const int group = a.heads / a.c.kv_heads;
    uint32_t id = blockIdx.x;
    const int head0 = id % a.c.kv_heads * group, kvh = id % a.c.kv_heads;
    id /= a.c.kv_heads;
    const int cut = id % a.splits, place = places - 1 - (int)(id / a.splits); // (the last tiles of a run have most to do)
    Tile t;
    if (!find_tile<BM>(a, place, group, t)) return;

    // the lane's row
    const int row = 32 * wm + r;
    const bool real = row < t.rows;
    const int in_run = t.row0 + (real ? row : 0), token = in_run / group, head = head0 + in_run - token * group;
    const int at = t.at0 + token; // its position
    const size_t out_row = (size_t)(t.token0 + token) * a.heads + head;
    // tokens that some row of the tile sees, and this cut's share
    const int last_row = min(t.rows, BM) - 1;
    const int end = max(0, t.at0 + (t.row0 + last_row) / group + 1), from0 = a.window > 0 ? max(0, t.at0 + t.row0 / group - a.window + 1) : 0;
    const long skip = (long)cut * a.chunk;
    const int from = (int)min((long)end, from0 + skip), to = (int)min((long)end, (long)from + a.chunk);
    const int steps = (to - from + BN - 1) / BN;

    uint4 qf[2 * ND];
#pragma unroll
    for (int c = 0; c < 2 * ND; ++c) {
        const int d = 16 * c + 8 * h;
        qf[c] = make_uint4(0, 0, 0, 0);
        if (real && d < D) {
            struct __attribute__((packed, aligned(2))) Words { uint32_t w[4]; };
            const Words x = *reinterpret_cast<const Words *>(reinterpret_cast<const uint16_t *>(a.q) + (size_t)(t.token0 + token) * a.q_stride + (size_t)head * D + d);
            qf[c] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
        }
    }
    const float to2 = a.scale * 1.4426950408889634f; // scores in powers of two
    f32x16 o[ND] = {};
    float m = -INFINITY, l = 0.f;

    // Tokens of step i: the cache rows of those that are there.
    auto page_of = [&](int i) __attribute__((always_inline)) {
        const long j = (long)from + (long)i * BN + threadIdx.x;
        return threadIdx.x < BN && j < to ? a.c.table[(size_t)t.s * a.c.table_stride + (uint32_t)j / (uint32_t)a.c.page_size] : -1;
    };
    auto look_up = [&](int i, int page) __attribute__((always_inline)) {
        if (threadIdx.x >= (BN + 63) / 64 * 64) return;
        const uint32_t j = (uint32_t)from + (uint32_t)i * BN + threadIdx.x;
        const bool there = (uint32_t)page < (uint32_t)a.c.pages;
        if (threadIdx.x < BN) ring[i % 3][threadIdx.x] = there ? ((uint32_t)page * a.c.kv_heads + kvh) * a.c.page_size + j % (uint32_t)a.c.page_size : kAbsent;
        const uint64_t none = ~__ballot(there);
        if (lane == 0) gone[i % 3][2 * wave] = (uint32_t)none, gone[i % 3][2 * wave + 1] = (uint32_t)(none >> 32);
    };
    uint4 in[2][PER];
    uint32_t scale8[2][E8 ? PER : 1], absent; // absent: a bit a unit
    auto load = [&](int i) __attribute__((always_inline)) {
        absent = 0;
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int n = threadIdx.x + u * THREADS, key = n / IN_ROW, d = (n - key * IN_ROW) * (E8 ? 16 : 8);
            const bool used = UNITS % THREADS == 0 || n < UNITS;
            const uint32_t row = used ? ring[i % 3][key] : kAbsent;
            const bool there = row != kAbsent && d < D;
            if (!there) absent |= 1u << u;
            const uint64_t at = (uint64_t)(there ? row : 0u) * D + (there ? d : 0);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                in[x][u] = *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint8_t *>(x ? a.c.v : a.c.k) + at * (E8 ? 1 : 2));
                if constexpr (E8) scale8[x][u] = (x ? a.c.v_scale : a.c.k_scale)[(uint64_t)(there ? row : 0u) * ((uint32_t)(D + 31) >> 5) + (there ? d >> 5 : 0)];
            }
        }
    };
    auto store = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int n = threadIdx.x + u * THREADS, key = n / IN_ROW, p = (n - key * IN_ROW) * (E8 ? 2 : 1);
            if (UNITS % THREADS && n >= UNITS) continue;
            const bool none = absent >> u & 1;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                uint8_t *row = kv[i & 1][x] + key * STRIDE;
                uint4 w = in[x][u];
                if (none) w = make_uint4(0, 0, 0, 0);
                if constexpr (E8) {
                    const uint32_t byte = none ? 127u : scale8[x][u];
                    *reinterpret_cast<uint4 *>(row + ((p ^ swizzle(key)) << 4)) = from_e4m3x8<DT>(make_uint2(w.x, w.y), byte);
                    *reinterpret_cast<uint4 *>(row + (((p + 1) ^ swizzle(key)) << 4)) = from_e4m3x8<DT>(make_uint2(w.z, w.w), byte);
                } else *reinterpret_cast<uint4 *>(row + ((p ^ swizzle(key)) << 4)) = w;
            }
        }
    };
    auto value_columns = [&](const uint8_t *vb, int key0, int dt, int part) __attribute__((always_inline)) {
        const int key = key0 + 8 * part + 4 * h + (lane >> 2 & 3), p = 4 * dt + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
        return read_columns(vb + key * STRIDE + ((p ^ swizzle(key)) << 4) + (lane & 1) * 8);
    };
    auto compute = [&](int i) __attribute__((always_inline)) {
        const uint8_t *kb = kv[i & 1][0], *vb = kv[i & 1][1];
        f32x16 sc[NSUB];
#pragma unroll
        for (int u = 0; u < NSUB; ++u) {
            sc[u] = f32x16{};
            const int key = 32 * (wk * NSUB + u) + r;
#pragma unroll
            for (int c = 0; c < 2 * ND; ++c) {
                const uint4 kf = *reinterpret_cast<const uint4 *>(kb + key * STRIDE + (((2 * c + h) ^ swizzle(key)) << 4));
                sc[u] = mfma32<DT>(kf, qf[c], sc[u]);
            }
        }
        float top = -INFINITY;
        uint32_t seen[NSUB]; // a bit a token of the 32
        bool all = true;
#pragma unroll
        for (int u = 0; u < NSUB; ++u) {
            const int sub = wk * NSUB + u;
            const long base = (long)from + (long)i * BN + 32 * sub, past = at - base, before = a.window > 0 ? at - a.window + 1 - base : 0;
            uint32_t bits = ~gone[i % 3][sub];
            if (past < 31) bits &= past < 0 ? 0u : (2u << past) - 1u;
            if (before > 0) bits &= before > 31 ? 0u : ~0u << before;
            seen[u] = bits;
            all = all && bits == ~0u;
        }
        const bool whole = __all(all);
#pragma unroll
        for (int u = 0; u < NSUB; ++u)
#pragma unroll
            for (int k = 0; k < 16; ++k) sc[u][k] *= to2;
        if (!whole)
#pragma unroll
            for (int u = 0; u < NSUB; ++u) {
                const uint32_t bits = seen[u] >> 4 * h;
#pragma unroll
                for (int k = 0; k < 16; ++k) sc[u][k] = bits >> (8 * (k >> 2) + (k & 3)) & 1 ? sc[u][k] : -INFINITY;
            }
#pragma unroll
        for (int u = 0; u < NSUB; ++u)
#pragma unroll
            for (int k = 0; k < 16; ++k) top = fmaxf(top, sc[u][k]);
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > m)) { // (an infinite score has an infinite weight, and so has the sum: finite maxima keep these from being NaN)
            const float now = fminf(fmaxf(m, top), FLT_MAX), c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= c;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) o[dt] *= c;
        }
        const float base = m == -INFINITY ? 0.f : m - TOP;
        uint4 pf[2 * NSUB];
#pragma unroll
        for (int u = 0; u < NSUB; ++u) {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                sc[u][k] = __builtin_amdgcn_exp2f(sc[u][k] - base);
                l += sc[u][k];
            }
#pragma unroll
            for (int x = 0; x < 2; ++x)
                pf[2 * u + x] = make_uint4(pack2<DT>(sc[u][8 * x], sc[u][8 * x + 1]), pack2<DT>(sc[u][8 * x + 2], sc[u][8 * x + 3]),
                                           pack2<DT>(sc[u][8 * x + 4], sc[u][8 * x + 5]), pack2<DT>(sc[u][8 * x + 6], sc[u][8 * x + 7]));
        }
        // A weight of zero times an infinity would be NaN in rows that do not see the token: such values are added one by one.
        bool odd = false;
        if (!whole)
#pragma unroll
            for (int u = 0; u < 2 * NSUB; ++u)
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const uint2 v = value_columns(vb, 32 * wk * NSUB + 16 * u, dt, x);
                        odd = odd || not_finite2<DT>(v.x) || not_finite2<DT>(v.y);
                    }
        if (!__any(odd)) {
#pragma unroll
            for (int u = 0; u < 2 * NSUB; ++u)
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) {
                    const uint2 v0 = value_columns(vb, 32 * wk * NSUB + 16 * u, dt, 0), v1 = value_columns(vb, 32 * wk * NSUB + 16 * u, dt, 1);
                    o[dt] = mfma32<DT>(make_uint4(v0.x, v0.y, v1.x, v1.y), pf[u], o[dt]);
                }
        } else {
#pragma unroll
            for (int u = 0; u < NSUB; ++u)
#pragma unroll 1
                for (int n = 0; n < 32; ++n) {
                    float p = 0.f; // the weight of token n: in half n >> 2 & 1, register 4 (n >> 3) + (n & 3)
#pragma unroll
                    for (int k = 0; k < 16; ++k) p = k == 4 * (n >> 3) + (n & 3) ? sc[u][k] : p;
                    p = __shfl(p, r + 32 * (n >> 2 & 1));
                    const bool see = seen[u] >> n & 1;
                    const int key = 32 * (wk * NSUB + u) + n;
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const uint2 v = *reinterpret_cast<const uint2 *>(vb + key * STRIDE + (((4 * dt + g) ^ swizzle(key)) << 4) + 8 * h);
                            const uint32_t w[2] = {v.x, v.y};
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const float x = from_storage<DT>((uint16_t)(w[k >> 1] >> 16 * (k & 1)));
                                o[dt][4 * g + k] += see ? p * x : 0.f;
                            }
                        }
                }
        }
    };

    if (steps > 0) {
        look_up(0, page_of(0));
        look_up(1, page_of(1));
        __syncthreads();
        load(0);
        store(0);
        for (int i = 0; i < steps; ++i) {
            __syncthreads();
            const int page = page_of(i + 2);
            if (i + 1 < steps) load(i + 1);
            compute(i);
            if (i + 1 < steps) store(i + 1);
            look_up(i + 2, page);
        }
    }
    l += __shfl_xor(l, 32);
    if constexpr (WK > 1) {
        // the side-by-side waves' sums, rescaled to the largest maximum and added in the waves' order; columns lie in LDS
        static_assert(WM * WK * 32 * DP * 4 <= sizeof(kv), "the sums fit where keys and values were");
        auto sums = [&](int w, int dt, int g) { // four of the lane's, in an order that spreads columns over the banks
            return reinterpret_cast<float4 *>(kv) + (w * 32 + r) * (DP / 4) + ((8 * dt + 2 * g + h) ^ (r & 7));
        };
        __syncthreads(); // (the last step's readers are done)
        if (h == 0) stat[0][wave][r] = m;
        __syncthreads();
        float top = stat[0][wm][r];
#pragma unroll
        for (int w = 1; w < WK; ++w) top = fmaxf(top, stat[0][w * WM + wm][r]);
        const float c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *sums(wave, dt, g) = make_float4(c * o[dt][4 * g], c * o[dt][4 * g + 1], c * o[dt][4 * g + 2], c * o[dt][4 * g + 3]);
        if (h == 0) stat[1][wave][r] = c * l;
        __syncthreads();
        if (wk) return;
        m = top;
        l = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) l += stat[1][w * WM + wm][r];
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < WK; ++w) {
                    const float4 v = *sums(w * WM + wm, dt, g);
                    sum.x += v.x, sum.y += v.y, sum.z += v.z, sum.w += v.w;
                }
                o[dt][4 * g] = sum.x, o[dt][4 * g + 1] = sum.y, o[dt][4 * g + 2] = sum.z, o[dt][4 * g + 3] = sum.w;
            }
        }
    }
    if (!real) return;
    if (a.splits > 1) {
        float *part = a.part + (out_row * a.splits + cut) * D;
        if (m != -INFINITY)
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int d = 32 * dt + 8 * g + 4 * h;
                    if (d < D) *reinterpret_cast<float4 *>(part + d) = make_float4(o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]);
                }
        if (h == 0) a.part_stat[out_row * a.splits + cut] = make_float2(m, l);
        return;
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * dt + 8 * g + 4 * h;
            struct __attribute__((packed, aligned(2))) Words { uint32_t w[2]; };
            if (d < D)
                *reinterpret_cast<Words *>(reinterpret_cast<uint16_t *>(a.y) + out_row * D + d) =
                    Words{{pack2<DT>(o[dt][4 * g] * inv, o[dt][4 * g + 1] * inv), pack2<DT>(o[dt][4 * g + 2] * inv, o[dt][4 * g + 3] * inv)}};
        }
    if (h == 0 && a.lse) a.lse[out_row] = l != 0.f ? (m - TOP + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// One wave a row: the cuts' sums, rescaled to the largest maximum and added in their order.
template <int DT> __global__ __launch_bounds__(256) void chunk_attention_join_kernel(ChunkArgs a)
{
    constexpr float TOP = DT == NPAS_BF16 ? 0.f : 15.f;
    const size_t row = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, D = a.c.head_dim;
    if (row >= (size_t)a.T * a.heads) return;
    const int token = (int)(row / a.heads);
    if (token < a.start[0] || token >= a.start[a.c.sequences]) return; // no sequence's
    const float2 *stat = a.part_stat + row * a.splits;
    float m = -INFINITY;
    for (int i = lane; i < a.splits; i += 64) m = fmaxf(m, stat[i].x);
#pragma unroll
    for (int w = 32; w; w >>= 1) m = fmaxf(m, __shfl_xor(m, w));
    float l = 0.f;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = 0; i < a.splits; ++i) {
        const float2 x = stat[i];
        if (x.x == -INFINITY) continue;
        const float c = __builtin_amdgcn_exp2f(x.x - m);
        l += c * x.y;
        if (lane * 4 < D) {
            const float4 v = *reinterpret_cast<const float4 *>(a.part + (row * a.splits + i) * D + lane * 4);
            y.x += c * v.x, y.y += c * v.y, y.z += c * v.z, y.w += c * v.w;
        }
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    struct __attribute__((packed, aligned(2))) Words { uint32_t w[2]; };
    if (lane * 4 < D)
        *reinterpret_cast<Words *>(reinterpret_cast<uint16_t *>(a.y) + row * D + lane * 4) = Words{{pack2<DT>(y.x * inv, y.y * inv), pack2<DT>(y.z * inv, y.w * inv)}};
    if (lane == 0 && a.lse) a.lse[row] = l != 0.f ? (m - TOP + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

int chunk_tile_rows(int head_dim, int few) { return few ? (head_dim <= 128 ? 32 : 64) : 128; }

int launch_chunk_attention(int dt, const ChunkArgs &a, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    const int group = a.heads / a.c.kv_heads, D = a.c.head_dim;
    const long places = (long)a.T * group / chunk_tile_rows(D, a.few) + a.c.sequences;
    if (int rc = check_grid("chunk attention", (uint64_t)places * a.splits * a.c.kv_heads, 256)) return rc;
    const dim3 grid((unsigned)(places * a.splits * a.c.kv_heads)), block(256);
    auto run = [&](auto dtc, auto e8c) {
        constexpr int DT = decltype(dtc)::value;
        constexpr bool E8 = decltype(e8c)::value;
        auto width = [&](auto ndc) {
            constexpr int ND = decltype(ndc)::value;
            if (!a.few) hipLaunchKernelGGL((chunk_attention_kernel<DT, E8, ND, ND <= 4 ? 2 : 1, 4, 1>), grid, block, 0, st, a, (int)places);
            else if constexpr (ND <= 4) hipLaunchKernelGGL((chunk_attention_kernel<DT, E8, ND, 1, 1, 4>), grid, block, 0, st, a, (int)places);
            else hipLaunchKernelGGL((chunk_attention_kernel<DT, E8, ND, 1, 2, 2>), grid, block, 0, st, a, (int)places);
        };
        if (D <= 64) width(std::integral_constant<int, 2>{});
        else if (D <= 96) width(std::integral_constant<int, 3>{});
        else if (D <= 128) width(std::integral_constant<int, 4>{});
        else width(std::integral_constant<int, 8>{});
        if (a.splits > 1) hipLaunchKernelGGL((chunk_attention_join_kernel<DT>), dim3((unsigned)(((size_t)a.T * a.heads + 3) / 4)), dim3(256), 0, st, a);
    };
    auto cache = [&](auto dtc) {
        if (a.c.k_scale) run(dtc, std::true_type{});
        else run(dtc, std::false_type{});
    };
    if (dt == NPAS_BF16) cache(std::integral_constant<int, NPAS_BF16>{});
    else cache(std::integral_constant<int, NPAS_F16>{});
    return launched("chunk attention");
}

} // namespace npas
