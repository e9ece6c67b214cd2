// Causal attention of runs of new tokens over the paged cache.
#include <cfloat>
#include <type_traits>

#include "cache8.h"
#include "decoder_internal.h"
#include "device_util.h"
#include "join_cuts.h"
#include "run_tiles.h"
#include "weight_parts.h"

namespace npas {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;

// Zeros, as 8-bit numbers and as 16-bit ones; the first byte as a scale too.
__device__ const uint4 kNothing = {};

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

// The largest of three; a NaN is left out.  (Becomes one instruction.  Not an asm statement: the compiler would not keep its distance from the matrix
// instruction whose results it reads.)
__device__ __forceinline__ float max3(float x, float y, float z) { return fmaxf(fmaxf(x, y), z); }

// The larger of a lane's and its partner's in the other half of the wave.
__device__ __forceinline__ float over_halves(float x)
{
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}

// One workgroup a (tile of BM = 32 WAVES rows, key head, cut).  A wave has 32 rows as columns of 32 x 32 x 16 matrix instructions and walks the tokens in steps of
// BN = 32 NSUB: scores S = K Q^T (row operand: keys from LDS as they lie), running maximum and sum a column, O^T = V^T P^T, where the weights
// are the column operand as the first product leaves them, if a step's tokens are counted so that a lane's half h has tokens 4 h .. 4 h + 3 of
// each eight; the values come out of LDS turned round.
// Keys and values of a step come into one of two places in LDS while the other is multiplied, 16-byte pieces in an order that spreads rows over the banks:
// 16-bit numbers straight from memory, 8-bit floats through registers, where they become 16-bit numbers.  Loads are issued a part at a time between the
// products.  The cache rows of 4 or 8 steps' tokens are looked up at once, a token a thread, in the step before they are needed.
// The maximum in use follows a row's scores only where one exceeds it by 2^GROW, so that sums are hardly ever rescaled.  A weight enters the second product as
// 16-bit numbers whose sum it is, three in bf16 and two in fp16 (22 bits), so that results are those of fp32 weights (one rounded number: 160 us for the
// prompts below, 2.33 ms for the long sequence).  Masks, absent tokens and values that are not finite are branches that the steps which every
// row sees whole do not have.
// (Measured with one number a weight: the banks, 2048 tokens on 63000 2.41 -> 2.34 ms; loads by parts, 8191 prompt tokens 182 -> 172 us; branches for selects,
// 343 -> 183.)
// Bound by the matrix cores: one sequence's 2048 tokens on 63000, 32 query and 8 key heads of 128 in 8 bits: 3.65 to 3.86 ms, its instructions at 1110 to 1180 TFLOP/s
// (a large library product 1250); 8191 tokens of five prompts in 16 bits 245 to 275 us (800 to 900 TFLOP/s), where the diagonal's half-empty steps and the order
// and the last, partial round of workgroups count.
// BN is 64 tokens for heads of up to 128, two workgroups a compute unit; 32 for longer ones, whose tiles fill LDS and registers.
template <int DT, bool E8, int ND, int NSUB, int WAVES, int OCC, bool FULL> __global__ __launch_bounds__(64 * WAVES, OCC) void chunk_attention_kernel(ChunkArgs a)
{
    constexpr int DP = 32 * ND, BM = 32 * WAVES, BN = 32 * NSUB, THREADS = 64 * WAVES, PIECES = DP / 8, STRIDE = DP * 2;
    constexpr int UNITS = E8 ? BN * PIECES / 2 : BN * PIECES, PER = (UNITS + THREADS - 1) / THREADS, IN_ROW = E8 ? PIECES / 2 : PIECES;
    constexpr float GROW = RunWeight<DT>::grow, UNIT = RunWeight<DT>::unit;
    constexpr int PARTS = DT == NPAS_BF16 ? 3 : 2; // 16-bit numbers that a weight is taken apart into
    __shared__ __align__(16) uint8_t kbuf[2][BN * STRIDE], vbuf[2][BN * STRIDE];
    constexpr int AHEAD = THREADS / BN; // steps whose tokens are looked up at once, one a thread
    __shared__ uint32_t ring[2 * THREADS], gone[2 * THREADS / 32], holes[2 * AHEAD]; // cache rows of tokens; a bit a token that is not there; whether a step has such
    __shared__ uint32_t odd[2]; // values of a step hold an infinity or a NaN, and not every row sees every token
    // Where a row's pieces lie, so that what a read takes at once is spread over all banks: keys are read one piece of 16 rows, values two or four of 4 or 8.
    auto key_piece = [](int row, int p) { return (p ^ (ND == 2 ? row >> 1 & 7 : ND == 3 ? row >> 2 & 3 : row & 15)) << 4; };
    auto value_piece = [](int row, int p) { return (p ^ ((ND == 2 ? (row >> 1 & 1) * 4 : ND == 3 ? 0 : (row & 3) * 4) + (row >> 2 & 1) * 2)) << 4; };
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5, D = FULL ? DP : a.c.head_dim;
    const int group = a.heads / a.c.kv_heads;
    uint32_t id = blockIdx.x;
    const int kvh = id % a.c.kv_heads, head0 = kvh * group;
    id /= a.c.kv_heads;
    const int cut = id % a.splits, place = a.places - 1 - (int)(id / a.splits); // (the last tiles of a run have most to do)
    RunTile t;
    if (!find_run_tile<BM>(a, place, group, t)) return;

    // the lane's row
    const int row = 32 * wave + r;
    const bool real = row < t.rows;
    const int in_run = t.row0 + (real ? row : 0), token = in_run / group, head = head0 + in_run - token * group;
    const int at = t.at0 + token; // its position
    const size_t out_row = (size_t)(t.token0 + token) * a.heads + head;
    // tokens that some row of the tile sees, and this cut's share
    const int last_row = min(t.rows, BM) - 1, at_first = t.at0 + t.row0 / group, at_last = t.at0 + (t.row0 + last_row) / group;
    const int end = max(0, at_last + 1), from0 = a.window > 0 ? (int)max(0l, (long)at_first - a.window + 1) : 0;
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

    // Tokens of the steps AHEAD n .. : the cache rows of those that are there.
    auto page_of = [&](int n) __attribute__((always_inline)) {
        const long j = (long)from + (long)n * THREADS + threadIdx.x;
        return j < to ? a.c.table[(size_t)t.s * a.c.table_stride + (uint32_t)j / (uint32_t)a.c.page_size] : -1;
    };
    auto look_up = [&](int n, int page) __attribute__((always_inline)) {
        const uint32_t j = (uint32_t)from + (uint32_t)n * THREADS + threadIdx.x;
        const bool there = (uint32_t)page < (uint32_t)a.c.pages;
        ring[(n & 1) * THREADS + threadIdx.x] = there ? ((uint32_t)page * a.c.kv_heads + kvh) * a.c.page_size + j % (uint32_t)a.c.page_size : 0;
        const uint64_t none = ~__ballot(there);
        if (lane == 0) {
            gone[(n & 1) * (THREADS / 32) + 2 * wave] = (uint32_t)none;
            gone[(n & 1) * (THREADS / 32) + 2 * wave + 1] = (uint32_t)(none >> 32);
            if (BN == 64) holes[(n & 1) * AHEAD + wave] = none != 0;
            else holes[(n & 1) * AHEAD + 2 * wave] = (uint32_t)none, holes[(n & 1) * AHEAD + 2 * wave + 1] = (uint32_t)(none >> 32);
        }
    };
    auto rows_of = [&](int i) { return ring + i % (2 * AHEAD) * BN; };
    // Every row sees every token of the steps lo .. hi - 1.
    const int hi = (int)max(0l, min((long)steps, ((long)at_first + 1 - from) >> (BN == 64 ? 6 : 5)));
    const long behind_all = (long)at_last - a.window - from; // the last token that some row has left behind
    const int lo = a.window > 0 && behind_all >= 0 ? (int)min((long)steps, behind_all / BN + 1) : 0;
    auto parted = [&](int i) { return i >= hi || i < lo; };
    auto hole = [&](int i) { return __builtin_amdgcn_readfirstlane(holes[i % (2 * AHEAD)]) != 0; };
    // The next step's keys and values are asked for a part at a time, between the products: a wave that asks for all at once stands still while the compute unit
    // takes them in, 64 bytes a cycle.  A part is 64 pieces of the wave, or 64 sixteens of 8-bit floats; its address is one multiplication and addition.
    // 16 bits: straight into LDS as the pieces lie there, a lane taking the one that belongs in its place.  A token that is not there is row 0 of the cache: it
    // has no score, and no value but where holes are looked after.
    const int wave0 = __builtin_amdgcn_readfirstlane(wave);
    auto key_of = [&](int u) { return THREADS % IN_ROW == 0 ? (int)threadIdx.x / IN_ROW + u * (THREADS / IN_ROW) : ((int)threadIdx.x + u * THREADS) / IN_ROW; };
    auto slot_of = [&](int u) { return THREADS % IN_ROW == 0 ? (int)threadIdx.x % IN_ROW : ((int)threadIdx.x + u * THREADS) % IN_ROW; };
    const uint32_t row_bytes = (uint32_t)D * (E8 ? 1 : 2), blocks = (uint32_t)(D + 31) >> 5;
    uint32_t rows[PER];
    auto rows_of_step = [&](int i) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < PER; ++u) rows[u] = rows_of(i)[UNITS % THREADS == 0 || key_of(u) < BN ? key_of(u) : 0];
    };
    typedef __attribute__((address_space(3))) uint8_t lds_u8;
    uint4 in[2][E8 ? PER : 1];
    uint32_t scale8[2][E8 ? PER : 1];
    auto load = [&](auto place, int u, int x) __attribute__((always_inline)) {
        const int slot = slot_of(u), p = E8 ? 2 * slot : (x ? value_piece(key_of(u), slot) : key_piece(key_of(u), slot)) >> 4; // (an exclusive or: its own inverse)
        const uint8_t *from = reinterpret_cast<const uint8_t *>(x ? a.c.v : a.c.k) + p * (E8 ? 8 : 16) + (uint64_t)rows[u] * row_bytes;
        const bool behind = !FULL && p * 8 >= D; // the end of the head
        if (behind) from = reinterpret_cast<const uint8_t *>(&kNothing);
        if constexpr (E8) {
            const uint8_t *scale = ((x ? a.c.v_scale : a.c.k_scale) + (p >> 2)) + (uint64_t)rows[u] * blocks;
            in[x][u] = *reinterpret_cast<const uint4 *>(from);
            scale8[x][u] = *(behind ? from : scale);
        } else lds_dma16(from, (uint32_t)(uintptr_t)(lds_u8 *)(x ? vbuf : kbuf)[place] + (uint32_t)(wave0 * 64 + u * THREADS) * 16);
    };
    auto store = [&](int i) __attribute__((always_inline)) {
        if constexpr (!E8) return;
        if (hole(i))
#pragma unroll
            for (int u = 0; u < PER; ++u)
                if ((UNITS % THREADS == 0 || key_of(u) < BN) && gone[i % (2 * AHEAD) * NSUB + (key_of(u) >> 5)] >> (key_of(u) & 31) & 1) {
                    in[0][u] = in[1][u] = make_uint4(0, 0, 0, 0);
                    scale8[0][u] = scale8[1][u] = 127;
                }
        if (parted(i)) {
            bool bad = false;
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const uint4 w = in[1][u];
                const uint32_t byte = scale8[1][u];
                bad = bad || (nan_codes(w.x, byte) | nan_codes(w.y, byte) | nan_codes(w.z, byte) | nan_codes(w.w, byte)) != 0;
            }
            if (bad) odd[i & 1] = 1;
        }
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int key = key_of(u), p = slot_of(u) * 2;
            if (UNITS % THREADS && key >= BN) continue;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                uint8_t *to = (x ? vbuf : kbuf)[i & 1] + key * STRIDE;
                auto piece = [&](int p) { return x ? value_piece(key, p) : key_piece(key, p); };
                const uint4 w = in[x][u];
                *reinterpret_cast<uint4 *>(to + piece(p)) = from_e4m3x8<DT>(make_uint2(w.x, w.y), scale8[x][u]);
                *reinterpret_cast<uint4 *>(to + piece(p + 1)) = from_e4m3x8<DT>(make_uint2(w.z, w.w), scale8[x][u]);
            }
        }
    };
    // the tokens of 32 from step i's sub-step u that the lane's row sees, a bit each
    auto seen = [&](int i, int u) __attribute__((always_inline)) {
        const long base = (long)from + (long)i * BN + 32 * u, past = at - base, before = a.window > 0 ? (long)at - a.window + 1 - base : 0;
        uint32_t bits = ~gone[i % (2 * AHEAD) * NSUB + u];
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
    // 16 bits: whether there are such values is looked up where they lie, in the steps where it matters.
    auto look_for_odd = [&](int i) __attribute__((always_inline)) {
        bool bad = false;
        for (int n = threadIdx.x; n < BN * PIECES; n += THREADS) {
            const uint4 w = reinterpret_cast<const uint4 *>(vbuf[i & 1])[n];
            bad = bad || not_finite2<DT>(w.x) || not_finite2<DT>(w.y) || not_finite2<DT>(w.z) || not_finite2<DT>(w.w);
        }
        if (bad) odd[i & 1] = 1;
        __syncthreads();
    };
    auto compute = [&](int i, auto parity, bool some_hidden, auto morec) __attribute__((always_inline)) {
        constexpr bool more = decltype(morec)::value;
        const uint8_t *kb = kbuf[parity], *vb = vbuf[parity];
        f32x16 sc[NSUB];
#pragma unroll
        for (int u = 0; u < NSUB; ++u) sc[u] = f32x16{};
        uint4 kf[3][NSUB];
        auto read_keys = [&](int c) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < NSUB; ++u) kf[c % 3][u] = *reinterpret_cast<const uint4 *>(kb + (32 * u + r) * STRIDE + key_piece(32 * u + r, 2 * c + h));
        };
        read_keys(0);
        read_keys(1);
#pragma unroll
        for (int c = 0; c < 2 * ND; ++c) {
            if (c + 2 < 2 * ND) read_keys(c + 2);
#pragma unroll
            for (int u = 0; u < NSUB; ++u) sc[u] = mfma32<DT>(kf[c % 3][u], qf[c], sc[u]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < PER; ++u)
                if (more && u * 2 * ND / PER == c) load(1 - parity, u, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (some_hidden) {
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
        top = over_halves(top) * to2;
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
        const float base = m == -INFINITY ? 0.f : m;
        // 16 tokens at a time; between the products of one such part the next one's weights are formed, and its values read as soon as these have been multiplied
        constexpr int STRETCHES = 2 * NSUB;
        uint32_t pf[2][PARTS][4];
        uint4 vf[ND];
        // two weights of a stretch: formed, then taken apart, a part a step
        float rest[8];
        auto weigh = [&](int x, int pair) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 2 * pair; k < 2 * pair + 2; ++k) {
                rest[k] = __builtin_amdgcn_exp2f(fmaf(sc[x >> 1][8 * (x & 1) + k], mul, -base)) * UNIT;
                l += rest[k];
            }
        };
        auto take = [&](int x, int pair, int n) __attribute__((always_inline)) {
            float &a = rest[2 * pair], &b = rest[2 * pair + 1];
            pf[x & 1][n][pair] = n < PARTS - 1 ? part_below2<DT>(a, b) : pack2<DT>(a, b);
        };
        auto read = [&](int x, int dt) __attribute__((always_inline)) {
            uint2 v[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int key = 16 * x + 8 * y + 4 * h + (lane >> 2 & 3), piece = 4 * dt + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
                v[y] = read_columns(vb + key * STRIDE + value_piece(key, piece) + (lane & 1) * 8);
            }
            vf[dt] = make_uint4(v[0].x, v[0].y, v[1].x, v[1].y);
        };
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) read(0, dt);
#pragma unroll
        for (int pair = 0; pair < 4; ++pair) {
            weigh(0, pair);
#pragma unroll
            for (int n = 0; n < PARTS; ++n) take(0, pair, n);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < STRETCHES; ++x) {
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) {
#pragma unroll
                for (int n = 0; n < PARTS; ++n) {
                    const uint32_t (&w)[4] = pf[x & 1][n];
                    o[dt] = mfma32<DT>(vf[dt], make_uint4(w[0], w[1], w[2], w[3]), o[dt]);
                    if (x + 1 < STRETCHES) {
#pragma unroll
                        for (int pair = 4 * dt / ND; pair < 4 * (dt + 1) / ND; ++pair) {
                            if (n == 0) weigh(x + 1, pair);
                            take(x + 1, pair, n);
                        }
                        if (n + 1 == PARTS) read(x + 1, dt);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
#pragma unroll
                for (int u = 0; u < PER; ++u)
                    if (more && u * STRETCHES * ND / PER / 2 == x * ND + dt) {
                        load(1 - parity, u, 1);
                        __builtin_amdgcn_sched_barrier(0);
                    }
            }
        }
        asm volatile("" : "+v"(l)); // (its additions belong here)
    };

    if (steps > 0) {
        if (threadIdx.x < 2) odd[threadIdx.x] = 0;
        look_up(0, page_of(0));
        __syncthreads();
        rows_of_step(0);
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            load(0, u, 0);
            load(0, u, 1);
        }
        store(0);
        if (!E8) asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        if (steps > 1) rows_of_step(1);
        uint32_t hole_next = holes[0];
        auto step = [&](int i, auto parity, auto morec) __attribute__((always_inline)) {
            constexpr bool more = decltype(morec)::value; // another follows
            __syncthreads();
            const bool hidden = parted(i) || __builtin_amdgcn_readfirstlane(hole_next);
            if (hidden) {
                if (!E8) look_for_odd(i);
                if (__builtin_amdgcn_readfirstlane(odd[i & 1])) part_values(i);
            }
            // the next tokens are looked up in the first step of the last that were
            const int next = i / AHEAD + 1;
            const bool ask = more && i % AHEAD == 0 && (long)next * AHEAD < steps;
            const int page = ask ? page_of(next) : -1;
            compute(i, parity, hidden, morec);
            if (more) {
                store(i + 1);
                rows_of_step(i + 2); // (where there is such a step; the tokens were looked up at least a step ago)
                hole_next = holes[(i + 1) % (2 * AHEAD)];
            }
            if (ask) look_up(next, page);
            if (!E8) asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); // what is on its way into LDS
        };
        int i = 0;
        for (; i + 1 < steps; ++i) step(i, i & 1, std::true_type{});
        step(i, i & 1, std::false_type{});
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
    if (h == 0 && a.lse) a.lse[out_row] = l != 0.f ? (m + log2f(l * (1.f / UNIT))) * 0.6931471805599453f : -INFINITY;
}

// One wave a row, for up to 16 cuts: their sums, rescaled to the largest maximum and added in their order (64 tokens of 32 heads in 4 to 11 cuts: the whole call,
// with weights of one number, 18 to 22 us, with a workgroup a row as more cuts have it 20 to 25; in 118 cuts, read in this way, 61, in that 28).  The bytes of the
// sums bound it.
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
    constexpr int SIDE = 4; // cuts on their way
    for (int i0 = 0; i0 < a.splits; i0 += SIDE) {
        float2 x[SIDE];
        float4 v[SIDE];
#pragma unroll
        for (int k = 0; k < SIDE; ++k) x[k] = stat[min(i0 + k, a.splits - 1)];
#pragma unroll
        for (int k = 0; k < SIDE; ++k) {
            if (i0 + k >= a.splits) x[k] = make_float2(-INFINITY, 0.f);
            v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (x[k].x != -INFINITY && lane * 4 < D) v[k] = *reinterpret_cast<const float4 *>(a.part + (row * a.splits + i0 + k) * D + lane * 4);
        }
#pragma unroll
        for (int k = 0; k < SIDE; ++k) {
            const float c = x[k].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[k].x - m);
            l += c * x[k].y; // (zero, or NaN from a cut whose scores all are)
            y.x += c * v[k].x, y.y += c * v[k].y, y.z += c * v[k].z, y.w += c * v[k].w;
        }
    }
    const float inv = l != 0.f ? 1.f / l : 0.f;
    struct __attribute__((packed, aligned(2))) Words { uint32_t w[2]; };
    if (lane * 4 < D)
        *reinterpret_cast<Words *>(reinterpret_cast<uint16_t *>(a.y) + row * D + lane * 4) = Words{{pack2<DT>(y.x * inv, y.y * inv), pack2<DT>(y.z * inv, y.w * inv)}};
    if (lane == 0 && a.lse) a.lse[row] = l != 0.f ? (m + log2f(l * (1.f / RunWeight<DT>::unit))) * 0.6931471805599453f : -INFINITY;
}

int launch_chunk_attention(int dt, const ChunkArgs &a, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    const int D = a.c.head_dim;
    const uint64_t workgroups = (uint64_t)a.places * a.splits * a.c.kv_heads;
    if (int rc = check_grid("chunk attention", workgroups, 2 * kChunkRows)) return rc;
    const dim3 grid((unsigned)workgroups), block(2 * kChunkRows);
    auto run = [&](auto dtc, auto e8c) {
        constexpr int DT = decltype(dtc)::value;
        constexpr bool E8 = decltype(e8c)::value;
        auto width = [&](auto ndc) {
            constexpr int ND = decltype(ndc)::value, OCC = ND <= 4 ? 2 : 1, NSUB = ND <= 4 ? 2 : 1;
            if (D == 32 * ND) hipLaunchKernelGGL((chunk_attention_kernel<DT, E8, ND, NSUB, kChunkRows / 32, OCC, true>), grid, block, 0, st, a);
            else hipLaunchKernelGGL((chunk_attention_kernel<DT, E8, ND, NSUB, kChunkRows / 32, OCC, false>), grid, block, 0, st, a);
        };
        if (D <= 64) width(std::integral_constant<int, 2>{});
        else if (D <= 96) width(std::integral_constant<int, 3>{});
        else if (D <= 128) width(std::integral_constant<int, 4>{});
        else width(std::integral_constant<int, 8>{});
    };
    auto cache = [&](auto dtc) {
        if (a.c.k_scale) run(dtc, std::true_type{});
        else run(dtc, std::false_type{});
    };
    if (dt == NPAS_BF16) cache(std::integral_constant<int, NPAS_BF16>{});
    else cache(std::integral_constant<int, NPAS_F16>{});
    return launched("chunk attention");
}

int launch_chunk_join(int dt, const ChunkArgs &a, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    if (a.splits > 16) return launch_join("chunk attention", dt, a, (uint64_t)a.T * a.heads, st);
    const uint64_t workgroups = ((uint64_t)a.T * a.heads + 3) / 4;
    if (int rc = check_grid("chunk attention", workgroups, 256)) return rc;
    const dim3 grid((unsigned)workgroups), block(256);
    if (dt == NPAS_BF16) hipLaunchKernelGGL((chunk_attention_join_kernel<NPAS_BF16>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((chunk_attention_join_kernel<NPAS_F16>), grid, block, 0, st, a);
    return launched("chunk attention");
}

} // namespace npas
