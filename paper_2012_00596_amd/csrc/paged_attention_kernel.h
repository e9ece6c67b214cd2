// The kernel of attention of one new token a sequence, or of short runs of them, over the paged cache: it walks the tokens once with running maximum
// and sum; long sequences are cut over workgroups.
#pragma once
#include <cfloat>
#include <type_traits>

#include "cache8.h"
#include "decoder_internal.h"
#include "run_tiles.h"
#include "device_util.h"
#include "join_cuts.h"
#include "weight_parts.h"

namespace npas {

constexpr int kRows = 2048; // tokens whose cache rows are looked up at once

// One workgroup a (sequence, key head, 16 of its query heads, cut): its four waves take tiles of 32 tokens in turn.
// Both products run on 16 x 16 x 32 matrix instructions with the query heads as columns, so that a key or value is read once for all
// heads of its group.  Scores: row operand = keys as they lie in the cache (lane 16 q + r: token r, 8 elements), result register i of
// lane 16 q + n = token 4 q + i, head n.  The weights are the second product's column operand as they stand, if its 32 tokens are
// counted so that quarter q holds tokens 4 q .. 4 q + 3 of both 16-token tiles; its row operand, values by element, comes from rows of
// the cache read whole (lane 16 q + r: VW consecutive elements of those eight tokens) and turned round in registers, two elements an
// instruction: row r of tile j is element VW r + j.  Nothing passes through LDS but the cache rows of the tokens.
// A weight goes in as three 16-bit numbers whose sum it is: the matrix cores have time for them (the kernel waits for memory).  The first two
// are taken below what there is to represent, so that all three are positive and an infinite value comes out as itself.  fp16 reaches
// down to 2^-24 only, so there the largest weight is 2^15: what is below 2^-39 of it is lost.
// Memory bound: 64 sequences of up to 8192 tokens, 8 key heads of 128, 1.07 GB in 205 us with the join (5.2 TB/s); one of 131071, 4 key heads, 55 us
// (4.9 TB/s).  Few short sequences are a chain of latencies: a launch, the length, the pages, then 1.1-1.8 us a round of tiles.
// E8: the cache holds 8-bit floats with a power of two for 32 elements.  A lane keeps the bytes and the scales of its next tile and makes 16-bit numbers of
// them, exactly, when they are multiplied: keys as the first product's operand (where head_dim is DP a lane takes 16 consecutive elements of 64, so that a load
// has 16 bytes; the query's elements are taken in the same order), values before they are turned round.  Half the bytes for more instructions, still bound by
// memory where there is enough of it: the 64 sequences, 0.55 GB, 116 to 123 us with the join (4.5 to 4.8 TB/s), the one of 131071 33 us
// (4.2 TB/s).
// RUNS: columns are the rows (token, query head of the key head) of a run of new tokens, 16 in each of RUNS groups (0: one token a sequence): a key or value is read
// once for all of them.  Where not every row sees every token of a tile, scores are left out by their positions, and values that are infinite or NaN, which a
// weight of zero would spread, are added one by one to the rows that see them.  A bf16 weight goes in as three 16-bit numbers here too, a fp16 one as two (22 bits).
// 32 sequences, 163 new tokens, 8 key heads of 128, up to 4096 tokens before them in 8 bits (0.15 GB): 65 us with the join (with bf16 weights of 17 bits, two
// numbers, 61; the same tokens over 16 bits, 0.28 GB, 69 to 78).  Not bound by memory: some 650 workgroups have work and 512 fit at once, so that the last ones
// run alone.  Two groups of rows at head_dim up to 64: three waves a SIMD with some 6 registers in memory (32 sequences of 5 tokens on 4000, 4
// key heads, in 8 bits 35 us, in 16 35; 64 of 6 on 2000, 8 key heads, 53 and 58) for two without (42, 38; 61 and 62).
template <int DT, int NC, bool FULL, int NW, bool E8, int RUNS = 0> __global__ __launch_bounds__(64 * NW, RUNS ? (NC == 2 ? 3 : NC == 4 ? 2 : 1) : NC == 2 ? 4 : NC == 4 ? (NW == 4 && FULL ? 3 : 2) : 1) void paged_attention_kernel(AttentionArgs a)
{
    constexpr int G = RUNS ? RUNS : 1; // groups of 16 columns
    constexpr int DP = 32 * NC, VW = DP / 16, VP = VW < 8 ? 1 : VW / 8, VD = VW / VP / 2; // a lane's value row: VP pieces of VD words
    constexpr int PITCH = DP + 4, PARTS = RUNS && DT == NPAS_F16 ? 2 : 3;
    constexpr float GROW = RUNS ? RunWeight<DT>::grow : 0.f; // the maximum in use follows a row's scores where one exceeds it by 2^GROW
    constexpr float TOP = RUNS ? RunWeight<DT>::unit : DT == NPAS_BF16 ? 1.f : 32768.f; // the largest weight is TOP 2^GROW
    constexpr float LEAVE = RUNS ? 1.f : 1.f / TOP, UNIT = RUNS ? TOP : 1.f; // factor of the sums that leave the kernel, and of the weights in them
    __shared__ __align__(16) uint32_t rows[kRows];
    __shared__ float sm[NW][16], sl[NW][16];
    __shared__ __align__(16) float so[NW * 16 * PITCH];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, D = FULL ? DP : a.c.head_dim;
    const int group = a.heads / a.c.kv_heads, head_tiles = (group + 15) >> 4;
    uint32_t id = blockIdx.x;
    const int kv = id % a.c.kv_heads;
    id /= a.c.kv_heads;
    // Workgroups go to the compute units in turn, so the cuts of a sequence start at one or another: in their order, the last, often empty ones would all meet
    // the same units
    // (64 sequences of up to 8192 tokens, 8 key heads of 128, two ragged batches, a launch without its join: in their order 129 and 122 us and so 116 and 106 in 8
    // bits, 229 and 213, 209 and 194 in 16).
    auto turned = [&](uint32_t n) { return (int)((id % a.splits + (n * 0x9e3779b1u >> 16)) % a.splits); };
    int h0 = 0, split, s, first, count; // h0: first of the group's heads here
    RunTile tile_of_run{};
    int at_first = 0, at_last = 0; // positions of the first and the last row
    if constexpr (RUNS) {
        split = turned(id / a.splits);
        if (!find_run_tile<16 * G>(a, (int)(id / a.splits), group, tile_of_run)) return;
        s = tile_of_run.s;
        at_first = tile_of_run.at0 + tile_of_run.row0 / group;
        at_last = tile_of_run.at0 + (tile_of_run.row0 + min(tile_of_run.rows, 16 * G) - 1) / group;
        first = a.window > 0 ? (int)max(0l, (long)at_first - a.window + 1) : 0;
        count = max(0, at_last + 1 - first);
    } else {
        h0 = id % head_tiles * 16;
        id /= head_tiles;
        s = id / a.splits;
        split = turned(s);
        token_range(a, s, first, count);
    }
    const long from = (long)split * a.chunk;
    if (!RUNS && from >= count && (split > 0 || a.splits > 1)) return;
    const int t0 = first + (int)min(from, (long)count), cnt = min(a.chunk, count - (int)min(from, (long)count));
    // where column n of group g is a row: its place in y
    auto row_of = [&](int g, int n, size_t &row, int &token) __attribute__((always_inline)) {
        if constexpr (RUNS) {
            const int in_run = tile_of_run.row0 + 16 * g + n;
            token = in_run / group;
            row = (size_t)(tile_of_run.token0 + token) * a.heads + kv * group + in_run - token * group;
            return 16 * g + n < tile_of_run.rows;
        } else {
            row = (size_t)s * a.heads + kv * group + h0 + n;
            return h0 + n < group;
        }
    };
    int at[G]; // positions of the lane's rows
    // first of the eight elements that a lane has in the first product's step c
    auto key_element = [&](int c) __attribute__((always_inline)) { return E8 && FULL ? (c >> 1) * 64 + 16 * q + 8 * (c & 1) : 32 * c + 8 * q; };
    uint4 qf[G][NC];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        size_t row = 0;
        int token = 0;
        const bool real = row_of(g, r, row, token);
        at[g] = real ? tile_of_run.at0 + token : at_last;
        const size_t q_at = RUNS ? (size_t)(tile_of_run.token0 + token) * a.q_stride + (row - (size_t)(tile_of_run.token0 + token) * a.heads) * D
                                 : (size_t)s * a.q_stride + (size_t)(kv * group + h0 + r) * D;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int d = key_element(c);
            qf[g][c] = make_uint4(0, 0, 0, 0);
            if (real && d < D) {
                struct __attribute__((packed, aligned(2))) Words { uint32_t w[4]; };
                const Words x = *reinterpret_cast<const Words *>(reinterpret_cast<const uint16_t *>(a.q) + q_at + d);
                qf[g][c] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
            }
        }
    }
    const uint8_t *kb = reinterpret_cast<const uint8_t *>(a.c.k), *vb = reinterpret_cast<const uint8_t *>(a.c.v);
    const uint32_t row_bytes = (uint32_t)D * (E8 ? 1 : 2), blocks = (uint32_t)(D + 31) >> 5;
    const float to2 = a.scale * 1.4426950408889634f; // scores in powers of two
    f32x4 o[G][VW] = {};
    float m[G], l[G] = {};
#pragma unroll
    for (int g = 0; g < G; ++g) m[g] = -INFINITY;

    // A tile's keys and values have one place each: the next tile's keys are asked for as soon as the scores are formed, its values as soon as
    // they have been multiplied, so that one tile is on its way all the time and the registers leave room for more waves.
    constexpr int VR = E8 ? VP * VD / 2 : VP * VD; // words of a lane's value row
    std::conditional_t<E8, uint2, uint4> kt[2][NC];
    uint32_t vt[8][VR], absent;
    uint32_t ks[2][E8 ? NC : 1], vs[E8 ? 8 : 1]; // scales: of each step's elements, of each token's
    auto load_keys = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t row = rows[tile * 32 + 16 * h + r], at = row == kAbsent ? 0u : row;
            const uint8_t *p = kb + (uint64_t)at * row_bytes;
            if constexpr (E8) {
                const uint8_t *sp = a.c.k_scale + (uint64_t)at * blocks;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const int d = key_element(c);
                    if constexpr (FULL) {
                        if (c % 2 == 0) {
                            const uint4 w = *reinterpret_cast<const uint4 *>(p + d);
                            kt[h][c] = make_uint2(w.x, w.y), kt[h][c + 1] = make_uint2(w.z, w.w);
                            ks[h][c] = ks[h][c + 1] = sp[d >> 5];
                        }
                    } else if (d < D) {
                        kt[h][c] = *reinterpret_cast<const uint2 *>(p + d);
                        ks[h][c] = sp[d >> 5];
                    } else {
                        kt[h][c] = make_uint2(0, 0);
                        ks[h][c] = 127;
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const int d = 32 * c + 8 * q;
                    if (FULL || d < D) kt[h][c] = *reinterpret_cast<const uint4 *>(p + 2 * d);
                    else kt[h][c] = make_uint4(0, 0, 0, 0);
                }
            }
        }
    };
    auto keys = [&](int h, int c) __attribute__((always_inline)) {
        if constexpr (E8) return from_e4m3x8<DT>(kt[h][c], ks[h][c]);
        else return kt[h][c];
    };
    auto load_values = [&](int tile) __attribute__((always_inline)) {
        absent = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 four = *reinterpret_cast<const uint4 *>(rows + tile * 32 + 16 * h + 4 * q);
            const uint32_t row[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool none = row[i] == kAbsent;
                if (none) absent |= 1u << (4 * h + i);
                const uint8_t *p = vb + (uint64_t)(none ? 0u : row[i]) * row_bytes;
                if constexpr (E8) vs[4 * h + i] = a.c.v_scale[(uint64_t)(none ? 0u : row[i]) * blocks + (FULL || VW * r < D ? VW * r >> 5 : 0)];
#pragma unroll
                for (int e = 0; e < VP; ++e) {
                    const int d = VW * r + 8 * e;
                    const uint8_t *x = p + (E8 ? 1 : 2) * (FULL || d < D ? d : 0); // elements past the head: their results are not kept
                    uint32_t *v = &vt[4 * h + i][e * VR / VP];
                    if constexpr (VR / VP == 1) v[0] = *reinterpret_cast<const uint32_t *>(x);
                    else if constexpr (VR / VP == 4) {
                        const uint4 w = *reinterpret_cast<const uint4 *>(x);
                        v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w;
                    } else {
                        const uint2 w = *reinterpret_cast<const uint2 *>(x);
                        v[0] = w.x, v[1] = w.y;
                    }
                }
            }
        }
    };
    // Whether row r of group g sees the token t of the lane's quarter in tile `j0` (its first token's position).
    auto sees = [&](int g, long j) __attribute__((always_inline)) { return j <= at[g] && (a.window <= 0 || j > (long)at[g] - a.window); };
    // Values that are infinite or NaN: added to the rows that see them, zero for the products.
    auto part_values = [&](long j0) __attribute__((always_inline)) {
        constexpr uint32_t e = DT == NPAS_BF16 ? 0x7f80u : 0x7c00u;
        auto odd16 = [](uint32_t v) __attribute__((always_inline)) { return (v & e) == e; };
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int w = 0; w < VR; ++w) odd = odd || (E8 ? nan_codes(vt[i][w], vs[E8 ? i : 0]) != 0 : odd16(vt[i][w]) || odd16(vt[i][w] >> 16));
        if (!__any(odd)) return;
        // the tile's values by token, in the wave's part of LDS; a lane reads those of its results
        uint16_t *tile = reinterpret_cast<uint16_t *>(so + wave * 16 * PITCH);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int w = 0; w < VW / 2; ++w) {
                uint32_t mine = vt[i][E8 ? w >> 1 : w]; // (8 bits: the NaN alone)
                if constexpr (E8) {
                    const uint32_t n = nan_codes(mine, vs[i]) >> 16 * (w & 1);
                    mine = (n & 0x80u ? 0xffffu : 0u) | (n & 0x8000u ? 0xffff0000u : 0u);
                }
                *reinterpret_cast<uint32_t *>(tile + (16 * (i >> 2) + 4 * q + (i & 3)) * DP + VW * r + 2 * w) = mine;
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll 1
        for (int k = 0; k < 32; ++k)
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    const float y = from_storage<DT>(tile[k * DP + VW * (4 * q + c) + w]);
#pragma unroll
                    for (int g = 0; g < G; ++g) o[g][w][c] += sees(g, j0 + k) && !(fabsf(y) < INFINITY) ? y : 0.f;
                }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (E8) {
#pragma unroll
                for (int w = 0; w < VR; ++w) vt[i][w] &= ~((nan_codes(vt[i][w], vs[i]) >> 7) * 255u);
                vs[i] = vs[i] == 255 ? 127u : vs[i]; // (its codes are zero now)
            } else
#pragma unroll
                for (int w = 0; w < VR; ++w) vt[i][w] &= (odd16(vt[i][w]) ? 0xffff0000u : ~0u) & (odd16(vt[i][w] >> 16) ? 0xffffu : ~0u);
        }
    };
    // One tile; MORE: another follows.
    auto tile_step = [&](int next, long j0, auto morec) __attribute__((always_inline)) { // j0: position of the tile's first token
        constexpr bool MORE = decltype(morec)::value;
        f32x4 c0[G] = {}, c1[G] = {};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint4 k0 = keys(0, c), k1 = keys(1, c);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                c0[g] = mfma16<DT>(k0, qf[g][c], c0[g]);
                c1[g] = mfma16<DT>(k1, qf[g][c], c1[g]);
            }
        }
        if (MORE) load_keys(next);
        __builtin_amdgcn_sched_barrier(0);
        const bool parted = RUNS && (j0 + 31 > at_first || (a.window > 0 && j0 <= (long)at_last - a.window)); // not every row sees every token
        uint32_t part[G][PARTS][4];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            uint32_t hidden = absent;
            if (parted) {
                asm volatile("" : : : "memory");
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (!sees(g, j0 + 16 * (i >> 2) + 4 * q + (i & 3))) hidden |= 1u << i;
            }
            float x[8], top = -INFINITY;
            if constexpr (RUNS) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = (i < 4 ? c0[g][i] : c1[g][i - 4]) * to2;
                if (__any(hidden != 0)) {
                    asm volatile("" : : : "memory");
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = hidden >> i & 1 ? -INFINITY : x[i];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, x[i]);
            } else
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] = hidden >> i & 1 ? -INFINITY : (i < 4 ? c0[g][i] : c1[g][i - 4]) * to2;
                    top = fmaxf(top, x[i]);
                }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (__any(top > m[g] + GROW)) { // (an infinite score has an infinite weight, and so has the sum: finite maxima keep these from being NaN)
                const float now = fminf(fmaxf(m[g], top), FLT_MAX), c = m[g] == -INFINITY ? (RUNS ? 1.f : 0.f) : __builtin_amdgcn_exp2f(m[g] - now);
                m[g] = now;
                l[g] *= c;
#pragma unroll
                for (int j = 0; j < VW; ++j) o[g][j] *= c;
            }
            const float base = m[g] == -INFINITY ? 0.f : m[g];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float p0 = __builtin_amdgcn_exp2f(x[2 * i] - base) * TOP, p1 = __builtin_amdgcn_exp2f(x[2 * i + 1] - base) * TOP;
                l[g] += p0 + p1;
#pragma unroll
                for (int n = 0; n < PARTS; ++n) {
                    if constexpr (RUNS) part[g][n][i] = n < PARTS - 1 ? part_below2<DT>(p0, p1) : pack2<DT>(p0, p1);
                    else {
                        part[g][n][i] = n < PARTS - 1 ? below2<DT>(p0, p1) : pack2<DT>(p0, p1);
                        p0 -= from_storage<DT>((uint16_t)part[g][n][i]);
                        p1 -= from_storage<DT>((uint16_t)(part[g][n][i] >> 16));
                    }
                }
            }
        }
        if (__any(absent != 0)) // an absent token's row is another's: it must not bring in an infinity or a NaN
#pragma unroll
            for (int i = 0; i < 8; ++i) {
#pragma unroll
                for (int w = 0; w < VR; ++w) vt[i][w] = absent >> i & 1 ? 0u : vt[i][w];
                if constexpr (E8) vs[i] = absent >> i & 1 ? 127u : vs[i];
            }
        if (parted) part_values(j0);
#pragma unroll
        for (int w = 0; w < VW / 2; ++w) {
            uint32_t even[4], odd[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t lo, hi; // two elements of two tokens
                if constexpr (E8) {
                    lo = w & 1 ? from_e4m3x2<DT, true>(vt[2 * i][w >> 1], vs[2 * i]) : from_e4m3x2<DT, false>(vt[2 * i][w >> 1], vs[2 * i]);
                    hi = w & 1 ? from_e4m3x2<DT, true>(vt[2 * i + 1][w >> 1], vs[2 * i + 1]) : from_e4m3x2<DT, false>(vt[2 * i + 1][w >> 1], vs[2 * i + 1]);
                } else lo = vt[2 * i][w], hi = vt[2 * i + 1][w];
                even[i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
                odd[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
            }
            const uint4 ve = make_uint4(even[0], even[1], even[2], even[3]), vo = make_uint4(odd[0], odd[1], odd[2], odd[3]);
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int n = 0; n < PARTS; ++n) {
                    const uint4 p = make_uint4(part[g][n][0], part[g][n][1], part[g][n][2], part[g][n][3]);
                    o[g][2 * w] = mfma16<DT>(ve, p, o[g][2 * w]);
                    o[g][2 * w + 1] = mfma16<DT>(vo, p, o[g][2 * w + 1]);
                }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (MORE) load_values(next);
        __builtin_amdgcn_sched_barrier(0);
    };

    for (int base = 0; base < cnt; base += kRows) {
        const int here = min(kRows, cnt - base), tiles = (here + 31) >> 5;
        if (base) __syncthreads();
        for (int i = threadIdx.x; i < tiles * 32; i += 64 * NW) {
            uint32_t row = kAbsent;
            if (i < here) {
                const uint32_t j = (uint32_t)(t0 + base + i), column = j / (uint32_t)a.c.page_size;
                const uint32_t page = (uint32_t)a.c.table[(size_t)s * a.c.table_stride + column];
                if (page < (uint32_t)a.c.pages) row = (page * a.c.kv_heads + kv) * a.c.page_size + (j - column * a.c.page_size);
            }
            rows[i] = row;
        }
        __syncthreads();
        if (wave < tiles) {
            int tile = wave;
            load_keys(tile);
            load_values(tile);
            const long j0 = (long)t0 + base;
            for (; tile + NW < tiles; tile += NW) tile_step(tile + NW, j0 + 32 * tile, std::true_type{});
            tile_step(0, j0 + 32 * tile, std::false_type{}); // (the last by itself: a branch around the loads would make the counted waits wait for all of them)
        }
    }

    // Join of the waves: maxima, then rescaled sums, in the waves' order.
#pragma unroll
    for (int g = 0; g < G; ++g) {
        if (g) __syncthreads();
        l[g] += __shfl_xor(l[g], 16);
        l[g] += __shfl_xor(l[g], 32);
        if (q == 0) {
            sm[wave][r] = m[g];
            sl[wave][r] = l[g];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float *p = so + (wave * 16 + r) * PITCH + VW * (4 * q + i);
#pragma unroll
            for (int j = 0; j < VW; j += 4) *reinterpret_cast<float4 *>(p + j) = make_float4(o[g][j][i], o[g][j + 1][i], o[g][j + 2][i], o[g][j + 3][i]);
        }
        __syncthreads();
        for (int u = threadIdx.x; u < 16 * (DP / 4); u += 64 * NW) {
            const int n = u / (DP / 4), d = (u - n * (DP / 4)) * 4;
            size_t row;
            int token;
            if (!row_of(g, n, row, token) || d >= D) continue;
            float top = sm[0][n], sum = 0.f;
#pragma unroll
            for (int w = 1; w < NW; ++w) top = fmaxf(top, sm[w][n]);
            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float c = sm[w][n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[w][n] - top) * LEAVE;
                const float4 v = *reinterpret_cast<const float4 *>(so + (w * 16 + n) * PITCH + d);
                sum += c * sl[w][n];
                y.x += c * v.x, y.y += c * v.y, y.z += c * v.z, y.w += c * v.w;
            }
            if (a.splits > 1) {
                *reinterpret_cast<float4 *>(a.part + (row * a.splits + split) * D + d) = y;
                if (d == 0) a.part_stat[row * a.splits + split] = make_float2(top, sum);
            } else {
                const float inv = sum != 0.f ? 1.f / sum : 0.f;
                uint16_t *out = reinterpret_cast<uint16_t *>(a.y) + row * D + d;
                const float v[4] = {y.x * inv, y.y * inv, y.z * inv, y.w * inv};
#pragma unroll
                for (int k = 0; k < 4; ++k) out[k] = to_storage<DT>(v[k]);
                if (d == 0 && a.lse) a.lse[row] = sum != 0.f ? (top + log2f(sum * (1.f / UNIT))) * 0.6931471805599453f : -INFINITY;
            }
        }
    }
}

} // namespace npas
