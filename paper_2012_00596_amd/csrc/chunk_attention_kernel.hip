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

// The largest of three, one instruction; a NaN is left out, as fmaxf leaves it.
__device__ __forceinline__ float max3(float x, float y, float z)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(y), "v"(z));
    return r;
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

// One workgroup a (tile of BM = 32 WAVES rows, key head, cut).  A wave has 32 rows as columns of 32 x 32 x 16 matrix instructions and walks the tokens in steps of
// BN = 32 NSUB: scores S = K Q^T (row operand: keys from LDS as they lie), running maximum and sum a column, O^T = V^T P^T, where the weights
// are the column operand as the first product leaves them, if a step's tokens are counted so that a lane's half h has tokens 4 h .. 4 h + 3 of
// each eight; the values come out of LDS turned round.
// Keys and values of a step come through registers into one of two places in LDS (16-byte pieces in an order that spreads rows over the banks; 8-bit
// floats become 16-bit numbers on the way) while the other is multiplied; the cache rows of the tokens are looked up two steps ahead.
// The maximum in use follows a row's scores only where one exceeds it by 2^GROW, so that sums are hardly ever rescaled.
template <int DT, bool E8, int ND, int NSUB, int WAVES, int OCC> __global__ __launch_bounds__(64 * WAVES, OCC) void chunk_attention_kernel(ChunkArgs a, int places)
{
    constexpr int DP = 32 * ND, BM = 32 * WAVES, BN = 32 * NSUB, THREADS = 64 * WAVES, PIECES = DP / 8, STRIDE = DP * 2;
    constexpr int UNITS = E8 ? BN * PIECES / 2 : BN * PIECES, PER = (UNITS + THREADS - 1) / THREADS, IN_ROW = E8 ? PIECES / 2 : PIECES;
    constexpr float GROW = DT == NPAS_BF16 ? 8.f : 4.f, TOP = DT == NPAS_BF16 ? 0.f : 11.f; // a weight is at most 2^(TOP + GROW)
    __shared__ __align__(16) uint8_t kbuf[2][BN * STRIDE], vbuf[2][BN * STRIDE];
    __shared__ uint32_t ring[3][BN], gone[3][NSUB]; // cache rows of a step's tokens; a bit a token that is not there
    __shared__ uint32_t odd[2]; // values of a step hold an infinity or a NaN, and not every row sees every token
    // Where a row's pieces lie, so that what a read takes at once is spread over all banks: keys are read one piece of 16 rows, values two or four of 4 or 8.
    auto key_piece = [](int row, int p) { return (p ^ (ND == 2 ? row >> 1 & 7 : ND == 3 ? row >> 2 & 3 : row & 15)) << 4; };
    auto value_piece = [](int row, int p) { return (p ^ ((ND == 2 ? (row >> 1 & 1) * 4 : ND == 3 ? 0 : (row & 3) * 4) + (row >> 2 & 1) * 2)) << 4; };
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5, D = a.c.head_dim;
    const int group = a.heads / a.c.kv_heads;
    uint32_t id = blockIdx.x;
    const int kvh = id % a.c.kv_heads, head0 = kvh * group;
    id /= a.c.kv_heads;
    const int cut = id % a.splits, place = places - 1 - (int)(id / a.splits); // (the last tiles of a run have most to do)
    Tile t;
    if (!find_tile<BM>(a, place, group, t)) return;

    // the lane's row
    const int row = 32 * wave + r;
    const bool real = row < t.rows;
    const int in_run = t.row0 + (real ? row : 0), token = in_run / group, head = head0 + in_run - token * group;
    const int at = t.at0 + token; // its position
    const size_t out_row = (size_t)(t.token0 + token) * a.heads + head;
    // tokens that some row of the tile sees, and this cut's share
    const int last_row = min(t.rows, BM) - 1, at_first = t.at0 + t.row0 / group, at_last = t.at0 + (t.row0 + last_row) / group;
    const int end = max(0, at_last + 1), from0 = a.window > 0 ? max(0, at_first - a.window + 1) : 0;
    const int from = (int)min((long)end, from0 + (long)cut * a.chunk), to = (int)min((long)end, (long)from + a.chunk);
    const int steps = (to - from + BN - 1) / BN;

    uint4 qf[2 * ND];
    const uint32_t sign = a.scale < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int c = 0; c < 2 * ND; ++c) {
        const int d = 16 * c + 8 * h;
        qf[c] = make_uint4(0, 0, 0, 0);
        if (real && d < D) {
            struct __attribute__((packed, aligned(2))) Words { uint32_t w[4]; };
            const Words x = *reinterpret_cast<const Words *>(reinterpret_cast<const uint16_t *>(a.q) + (size_t)(t.token0 + token) * a.q_stride + (size_t)head * D + d);
            qf[c] = make_uint4(x.w[0] ^ sign, x.w[1] ^ sign, x.w[2] ^ sign, x.w[3] ^ sign);
        }
    }
    // scores in powers of two; positive, so that a score that is left out can be minus infinity throughout
    const float to2 = fmaxf(fabsf(a.scale) * 1.4426950408889634f, FLT_MIN);
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
        if (lane == 0) {
            gone[i % 3][2 * wave] = (uint32_t)none;
            if (NSUB > 1) gone[i % 3][2 * wave + 1] = (uint32_t)(none >> 32);
        }
    };
    // whether a row of the workgroup does not see a token of step i that another sees
    auto parted = [&](int i) __attribute__((always_inline)) {
        const long base = (long)from + (long)i * BN;
        return base + BN - 1 > at_first || (a.window > 0 && base <= (long)at_last - a.window);
    };
    uint4 in[2][PER];
    uint32_t scale8[2][E8 ? PER : 1], absent; // absent: a bit a unit
    auto load = [&](int i) __attribute__((always_inline)) {
        absent = 0;
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int n = threadIdx.x + u * THREADS, key = n / IN_ROW, d = (n - key * IN_ROW) * (E8 ? 16 : 8);
            const uint32_t row = UNITS % THREADS == 0 || n < UNITS ? ring[i % 3][key] : kAbsent;
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
        if (__any(absent)) { // another's row, or the padding of a head
            asm volatile("" : : : "memory");
#pragma unroll
            for (int u = 0; u < PER; ++u)
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (absent >> u & 1) {
                        in[x][u] = make_uint4(0, 0, 0, 0);
                        if constexpr (E8) scale8[x][u] = 127;
                    }
        }
        if (parted(i)) {
            bool bad = false;
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const uint4 w = in[1][u];
                if constexpr (E8) bad = bad || scale8[1][u] == 255;
                else bad = bad || not_finite2<DT>(w.x) || not_finite2<DT>(w.y) || not_finite2<DT>(w.z) || not_finite2<DT>(w.w);
            }
            if (bad) odd[i & 1] = 1;
        }
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int n = threadIdx.x + u * THREADS, key = n / IN_ROW, p = (n - key * IN_ROW) * (E8 ? 2 : 1);
            if (UNITS % THREADS && n >= UNITS) continue;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                uint8_t *to = (x ? vbuf : kbuf)[i & 1] + key * STRIDE;
                auto piece = [&](int p) { return x ? value_piece(key, p) : key_piece(key, p); };
                const uint4 w = in[x][u];
                if constexpr (E8) {
                    *reinterpret_cast<uint4 *>(to + piece(p)) = from_e4m3x8<DT>(make_uint2(w.x, w.y), scale8[x][u]);
                    *reinterpret_cast<uint4 *>(to + piece(p + 1)) = from_e4m3x8<DT>(make_uint2(w.z, w.w), scale8[x][u]);
                } else *reinterpret_cast<uint4 *>(to + piece(p)) = w;
            }
        }
    };
    // the tokens of 32 from step i's sub-step u that the lane's row sees, a bit each
    auto seen = [&](int i, int u) __attribute__((always_inline)) {
        const long base = (long)from + (long)i * BN + 32 * u, past = at - base, before = a.window > 0 ? at - a.window + 1 - base : 0;
        uint32_t bits = ~gone[i % 3][u];
        if (past < 31) bits &= past < 0 ? 0u : (2u << past) - 1u;
        if (before > 0) bits &= before > 31 ? 0u : ~0u << before;
        return bits;
    };
    // Values that are infinite or NaN in a step that not every row sees, where a weight of zero would make them NaN: added to the rows that see them, and zero for the products.
    auto part_values = [&](int i) __attribute__((always_inline)) {
        uint8_t *buf = vbuf[i & 1];
#pragma unroll 1
        for (int n = 0; n < BN; ++n) {
            const bool see = seen(i, n >> 5) >> (n & 31) & 1;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const uint2 v = *reinterpret_cast<const uint2 *>(buf + n * STRIDE + value_piece(n, 4 * dt + x) + 8 * h);
                    const uint32_t w[2] = {v.x, v.y};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float y = from_storage<DT>((uint16_t)(w[k >> 1] >> 16 * (k & 1)));
                        o[dt][4 * x + k] += see && !(fabsf(y) < INFINITY) ? y : 0.f;
                    }
                }
        }
        __syncthreads();
        for (int n = threadIdx.x; n < BN * STRIDE / 4; n += THREADS) {
            uint32_t &w = reinterpret_cast<uint32_t *>(buf)[n];
            constexpr uint32_t e = DT == NPAS_BF16 ? 0x7f80u : 0x7c00u;
            if ((w & e) == e) w &= 0xffff0000u;
            if ((w >> 16 & e) == e) w &= 0xffffu;
        }
        if (threadIdx.x == 0) odd[i & 1] = 0;
        __syncthreads();
    };
    auto compute = [&](int i) __attribute__((always_inline)) {
        const uint8_t *kb = kbuf[i & 1], *vb = vbuf[i & 1];
        f32x16 sc[NSUB];
#pragma unroll
        for (int u = 0; u < NSUB; ++u) sc[u] = f32x16{};
#pragma unroll
        for (int c = 0; c < 2 * ND; ++c)
#pragma unroll
            for (int u = 0; u < NSUB; ++u) {
                const int key = 32 * u + r;
                sc[u] = mfma32<DT>(*reinterpret_cast<const uint4 *>(kb + key * STRIDE + key_piece(key, 2 * c + h)), qf[c], sc[u]);
            }
        uint32_t none = 0;
#pragma unroll
        for (int u = 0; u < NSUB; ++u) none |= gone[i % 3][u];
        if (parted(i) || __builtin_amdgcn_readfirstlane(none)) {
            asm volatile("" : : : "memory");
#pragma unroll
            for (int u = 0; u < NSUB; ++u) {
                const uint32_t bits = seen(i, u) >> 4 * h;
#pragma unroll
                for (int k = 0; k < 16; ++k) sc[u][k] = bits >> (8 * (k >> 2) + (k & 3)) & 1 ? sc[u][k] : -INFINITY;
            }
        }
        float top = -INFINITY;
#pragma unroll
        for (int u = 0; u < NSUB; ++u)
#pragma unroll
            for (int k = 0; k < 16; k += 2) top = max3(top, sc[u][k], sc[u][k + 1]);
        top = fmaxf(top, __shfl_xor(top, 32)) * to2;
        float mul = to2;
        if (__any(fabsf(top) > 0x1p20f && top != -INFINITY)) { // (where a product's rounding would count in the exponent)
            asm volatile("" : : : "memory");
#pragma unroll
            for (int u = 0; u < NSUB; ++u) sc[u] *= to2;
            mul = 1.f;
        }
        if (__any(top > m + GROW)) { // (an infinite score has an infinite weight, and so has the sum: finite maxima keep these from being NaN)
            const float now = fminf(fmaxf(m, top), FLT_MAX), c = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= c;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) o[dt] *= c;
        }
        const float base = m == -INFINITY ? 0.f : m - TOP;
#pragma unroll
        for (int u = 0; u < NSUB; ++u)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                float p[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    p[k] = __builtin_amdgcn_exp2f(fmaf(sc[u][8 * x + k], mul, -base));
                    l += p[k];
                }
                const uint4 pf = make_uint4(pack2<DT>(p[0], p[1]), pack2<DT>(p[2], p[3]), pack2<DT>(p[4], p[5]), pack2<DT>(p[6], p[7]));
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) {
                    uint2 v[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int key = 32 * u + 16 * x + 8 * y + 4 * h + (lane >> 2 & 3), piece = 4 * dt + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
                        v[y] = read_columns(vb + key * STRIDE + value_piece(key, piece) + (lane & 1) * 8);
                    }
                    o[dt] = mfma32<DT>(make_uint4(v[0].x, v[0].y, v[1].x, v[1].y), pf, o[dt]);
                }
            }
    };

    if (steps > 0) {
        if (threadIdx.x < 2) odd[threadIdx.x] = 0;
        look_up(0, page_of(0));
        look_up(1, page_of(1));
        __syncthreads();
        load(0);
        store(0);
        for (int i = 0; i < steps; ++i) {
            __syncthreads();
            if (__builtin_amdgcn_readfirstlane(odd[i & 1])) part_values(i);
            const int page = page_of(i + 2);
            if (i + 1 < steps) load(i + 1);
            compute(i);
            if (i + 1 < steps) store(i + 1);
            look_up(i + 2, page);
        }
    }
    l += __shfl_xor(l, 32);
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
        if (h == 0) a.part_stat[out_row * a.splits + cut] = make_float2(m - TOP, l);
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
    if (lane == 0 && a.lse) a.lse[row] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

int chunk_tile_rows(int head_dim, int few) { return 128; }

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
            if constexpr (ND <= 4) hipLaunchKernelGGL((chunk_attention_kernel<DT, E8, ND, 2, 4, 2>), grid, block, 0, st, a, (int)places);
            else hipLaunchKernelGGL((chunk_attention_kernel<DT, E8, ND, 1, 4, 1>), grid, block, 0, st, a, (int)places);
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
