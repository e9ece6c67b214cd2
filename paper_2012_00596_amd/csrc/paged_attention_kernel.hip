// Attention of one new token a sequence over the paged cache: a split kernel that walks the tokens once with running maximum and
// sum, and a joining kernel for sequences that were cut over several workgroups.
#include <cfloat>
#include <type_traits>

#include "decoder_internal.h"
#include "device_util.h"

namespace npas {

constexpr uint32_t kAbsent = 0xffffffffu;
constexpr int kRows = 2048; // tokens whose cache rows are looked up at once

// The tokens of sequence s that take part: [first, first + count).
__device__ __forceinline__ void token_range(const AttentionArgs &a, int s, int &first, int &count)
{
    const long room = (long)a.c.table_stride * a.c.page_size;
    int n = max(0, min(a.length[s], a.max_length));
    if (n > room) n = (int)room;
    first = a.window > 0 ? max(0, n - a.window) : 0;
    count = n - first;
}

// Two 16-bit numbers below the weights a and b, next to them or nearly so; zero for zero.
template <int DT> __device__ __forceinline__ uint32_t below2(float a, float b)
{
    const uint32_t u = __builtin_elementwise_sub_sat(__float_as_uint(a), 1u), w = __builtin_elementwise_sub_sat(__float_as_uint(b), 1u);
    if constexpr (DT == NPAS_BF16) return __builtin_amdgcn_perm(w, u, 0x07060302u);
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(__uint_as_float(u), __uint_as_float(w)));
}

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
// Memory bound: 64 sequences of up to 8192 tokens, 8 key heads of 128, 1.07 GB in 227 us (4.7 TB/s); one of 131071, 4 key heads, 55 us
// (4.9 TB/s).  Few short sequences are a chain of latencies: a launch, the length, the pages, then 1.1-1.8 us a round of tiles.
template <int DT, int NC, bool FULL, int NW> __global__ __launch_bounds__(64 * NW, NC == 2 ? 4 : NC == 4 ? (NW == 4 && FULL ? 3 : 2) : 1) void paged_attention_kernel(AttentionArgs a)
{
    constexpr int DP = 32 * NC, VW = DP / 16, VP = VW < 8 ? 1 : VW / 8, VD = VW / VP / 2; // a lane's value row: VP pieces of VD words
    constexpr int PITCH = DP + 4, PARTS = 3;
    constexpr float TOP = DT == NPAS_BF16 ? 1.f : 32768.f; // the largest weight
    __shared__ __align__(16) uint32_t rows[kRows];
    __shared__ float sm[NW][16], sl[NW][16];
    __shared__ __align__(16) float so[NW * 16 * PITCH];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4, D = FULL ? DP : a.c.head_dim;
    const int group = a.heads / a.c.kv_heads, head_tiles = (group + 15) >> 4;
    uint32_t id = blockIdx.x;
    const int kv = id % a.c.kv_heads;
    id /= a.c.kv_heads;
    const int h0 = id % head_tiles * 16; // first of the group's heads here
    id /= head_tiles;
    const int split = id % a.splits, s = id / a.splits;
    int first, count;
    token_range(a, s, first, count);
    const long from = (long)split * a.chunk;
    if (from >= count && (split > 0 || a.splits > 1)) return;
    const int t0 = first + (int)from, cnt = min(a.chunk, count - (int)from);
    const bool real = h0 + r < group;
    uint4 qf[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int d = 32 * c + 8 * q;
        qf[c] = make_uint4(0, 0, 0, 0);
        if (real && d < D) {
            struct __attribute__((packed, aligned(2))) Words { uint32_t w[4]; };
            const Words x = *reinterpret_cast<const Words *>(reinterpret_cast<const uint16_t *>(a.q) + (size_t)s * a.q_stride +
                                                             (size_t)(kv * group + h0 + r) * D + d);
            qf[c] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
        }
    }
    const uint8_t *kb = reinterpret_cast<const uint8_t *>(a.c.k), *vb = reinterpret_cast<const uint8_t *>(a.c.v);
    const uint32_t row_bytes = (uint32_t)D * 2;
    const float to2 = a.scale * 1.4426950408889634f; // scores in powers of two
    f32x4 o[VW] = {};
    float m = -INFINITY, l = 0.f;

    // A tile's keys and values have one place each: the next tile's keys are asked for as soon as the scores are formed, its values as soon as
    // they have been multiplied, so that one tile is on its way all the time and the registers leave room for more waves.
    uint4 kt[2][NC];
    uint32_t vt[8][VP * VD], absent;
    auto load_keys = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t row = rows[tile * 32 + 16 * h + r];
            const uint8_t *p = kb + (uint64_t)(row == kAbsent ? 0u : row) * row_bytes;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int d = 32 * c + 8 * q;
                if (FULL || d < D) kt[h][c] = *reinterpret_cast<const uint4 *>(p + 2 * d);
                else kt[h][c] = make_uint4(0, 0, 0, 0);
            }
        }
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
#pragma unroll
                for (int e = 0; e < VP; ++e) {
                    const int d = VW * r + 8 * e;
                    const uint8_t *x = p + 2 * (FULL || d < D ? d : 0); // elements past the head: their results are not kept
                    uint32_t *v = &vt[4 * h + i][e * VD];
                    if constexpr (VD == 4) {
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
    // One tile; MORE: another follows.
    auto tile_step = [&](int next, auto morec) __attribute__((always_inline)) {
        constexpr bool MORE = decltype(morec)::value;
        f32x4 c0 = {}, c1 = {};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            c0 = mfma16<DT>(kt[0][c], qf[c], c0);
            c1 = mfma16<DT>(kt[1][c], qf[c], c1);
        }
        if (MORE) load_keys(next);
        __builtin_amdgcn_sched_barrier(0);
        float x[8], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = absent >> i & 1 ? -INFINITY : (i < 4 ? c0[i] : c1[i - 4]) * to2;
            top = fmaxf(top, x[i]);
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > m)) { // (an infinite score has an infinite weight, and so has the sum: finite maxima keep these from being NaN)
            const float now = fminf(fmaxf(m, top), FLT_MAX), c = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= c;
#pragma unroll
            for (int j = 0; j < VW; ++j) o[j] *= c;
        }
        const float base = m == -INFINITY ? 0.f : m;
        uint32_t part[PARTS][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float p0 = __builtin_amdgcn_exp2f(x[2 * i] - base) * TOP, p1 = __builtin_amdgcn_exp2f(x[2 * i + 1] - base) * TOP;
            l += p0 + p1;
#pragma unroll
            for (int n = 0; n < PARTS; ++n) {
                part[n][i] = n < PARTS - 1 ? below2<DT>(p0, p1) : pack2<DT>(p0, p1);
                p0 -= from_storage<DT>((uint16_t)part[n][i]);
                p1 -= from_storage<DT>((uint16_t)(part[n][i] >> 16));
            }
        }
        if (__any(absent != 0)) // an absent token's row is another's: it must not bring in an infinity or a NaN
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int w = 0; w < VW / 2; ++w) vt[i][w] = absent >> i & 1 ? 0u : vt[i][w];
#pragma unroll
        for (int w = 0; w < VW / 2; ++w) {
            uint32_t even[4], odd[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                even[i] = __builtin_amdgcn_perm(vt[2 * i + 1][w], vt[2 * i][w], 0x05040100u);
                odd[i] = __builtin_amdgcn_perm(vt[2 * i + 1][w], vt[2 * i][w], 0x07060302u);
            }
            const uint4 ve = make_uint4(even[0], even[1], even[2], even[3]), vo = make_uint4(odd[0], odd[1], odd[2], odd[3]);
#pragma unroll
            for (int n = 0; n < PARTS; ++n) {
                const uint4 p = make_uint4(part[n][0], part[n][1], part[n][2], part[n][3]);
                o[2 * w] = mfma16<DT>(ve, p, o[2 * w]);
                o[2 * w + 1] = mfma16<DT>(vo, p, o[2 * w + 1]);
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
            for (; tile + NW < tiles; tile += NW) tile_step(tile + NW, std::true_type{});
            tile_step(0, std::false_type{}); // (the last by itself: a branch around the loads would make the counted waits wait for all of them)
        }
    }

    // Join of the four waves: maxima, then rescaled sums, in the waves' order.
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (q == 0) {
        sm[wave][r] = m;
        sl[wave][r] = l;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float *p = so + (wave * 16 + r) * PITCH + VW * (4 * q + i);
#pragma unroll
        for (int j = 0; j < VW; j += 4) *reinterpret_cast<float4 *>(p + j) = make_float4(o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]);
    }
    __syncthreads();
    for (int u = threadIdx.x; u < 16 * (DP / 4); u += 64 * NW) {
        const int n = u / (DP / 4), d = (u - n * (DP / 4)) * 4;
        if (h0 + n >= group || d >= D) continue;
        const int head = kv * group + h0 + n;
        float top = sm[0][n], sum = 0.f;
#pragma unroll
        for (int w = 1; w < NW; ++w) top = fmaxf(top, sm[w][n]);
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float c = sm[w][n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[w][n] - top) * (1.f / TOP);
            const float4 v = *reinterpret_cast<const float4 *>(so + (w * 16 + n) * PITCH + d);
            sum += c * sl[w][n];
            y.x += c * v.x, y.y += c * v.y, y.z += c * v.z, y.w += c * v.w;
        }
        const size_t row = (size_t)s * a.heads + head;
        if (a.splits > 1) {
            *reinterpret_cast<float4 *>(a.part + (row * a.splits + split) * D + d) = y;
            if (d == 0) a.part_stat[row * a.splits + split] = make_float2(top, sum);
        } else {
            const float inv = sum != 0.f ? 1.f / sum : 0.f;
            uint16_t *out = reinterpret_cast<uint16_t *>(a.y) + row * D + d;
            const float v[4] = {y.x * inv, y.y * inv, y.z * inv, y.w * inv};
#pragma unroll
            for (int k = 0; k < 4; ++k) out[k] = to_storage<DT>(v[k]);
            if (d == 0 && a.lse) a.lse[row] = sum != 0.f ? (top + log2f(sum)) * 0.6931471805599453f : -INFINITY;
        }
    }
}

// One workgroup a (sequence, head): the cuts' sums, rescaled to the largest maximum and added; LANES lanes hold a cut's row, four elements
// each, so that THREADS / LANES cuts are read side by side.  One wave for up to 16 cuts (2048 rows of two cuts: 3 us, with eight
// waves 8.5), eight for more (32 rows of 128 cuts 4.8 us; 512 cuts read one after the other by four waves 37).
template <int DT, int LANES, int THREADS> __global__ __launch_bounds__(THREADS) void paged_attention_join_kernel(AttentionArgs a)
{
    constexpr int SIDE = THREADS / LANES, WAVES = THREADS / 64;
    __shared__ float weight[THREADS], part[WAVES], total[WAVES];
    __shared__ __align__(16) float so[SIDE][LANES * 4];
    const int s = blockIdx.x / a.heads, D = a.c.head_dim, tid = threadIdx.x, side = tid / LANES, d = tid % LANES * 4;
    const size_t row = blockIdx.x;
    int first, count;
    token_range(a, s, first, count);
    const int cuts = (int)(((uint32_t)count + (uint32_t)a.chunk - 1) / (uint32_t)a.chunk); // (count and chunk together pass 2^31)
    const float2 x = tid < cuts ? a.part_stat[row * a.splits + tid] : make_float2(-INFINITY, 0.f); // no more cuts than threads
    float m = x.x;
#pragma unroll
    for (int w = 32; w; w >>= 1) m = fmaxf(m, __shfl_xor(m, w));
    if ((tid & 63) == 0) part[tid >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, part[w]);
    const float c = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.x - m);
    float l = c * x.y;
    weight[tid] = c;
#pragma unroll
    for (int w = 32; w; w >>= 1) l += __shfl_xor(l, w);
    if ((tid & 63) == 0) total[tid >> 6] = l;
    __syncthreads();
    l = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) l += total[w];
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    if (d < D)
#pragma unroll 4
        for (int i = side; i < cuts; i += SIDE) {
            const float k = weight[i];
            const float4 v = *reinterpret_cast<const float4 *>(a.part + (row * a.splits + i) * D + d);
            y.x += k * v.x, y.y += k * v.y, y.z += k * v.z, y.w += k * v.w;
        }
    *reinterpret_cast<float4 *>(&so[side][d]) = y;
    __syncthreads();
    for (int i = tid; i < D; i += THREADS) {
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < SIDE; ++k) sum += so[k][i];
        reinterpret_cast<uint16_t *>(a.y)[row * D + i] = to_storage<DT>(l != 0.f ? sum / l : 0.f);
    }
    if (tid == 0 && a.lse) a.lse[row] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

int launch_paged_attention(int dt, const AttentionArgs &a, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    const int group = a.heads / a.c.kv_heads;
    const dim3 grid((unsigned)((size_t)a.c.sequences * a.splits * ((group + 15) / 16) * a.c.kv_heads));
    const unsigned joiners = a.splits <= 16 ? 64 : kMaxSplits; // threads of a workgroup that joins
    if (int rc = check_grid("paged attention", grid.x, 64 * a.waves)) return rc;
    if (a.splits > 1)
        if (int rc = check_grid("paged attention", (uint64_t)a.c.sequences * a.heads, joiners)) return rc;
    auto pick = [&](auto dtc) {
        constexpr int DT = decltype(dtc)::value;
        auto run = [&](auto ncc) {
            constexpr int NC = decltype(ncc)::value;
            auto form = [&](auto nwc) {
                constexpr int NW = decltype(nwc)::value;
                if (a.c.head_dim == 32 * NC) hipLaunchKernelGGL((paged_attention_kernel<DT, NC, true, NW>), grid, dim3(64 * NW), 0, st, a);
                else hipLaunchKernelGGL((paged_attention_kernel<DT, NC, false, NW>), grid, dim3(64 * NW), 0, st, a);
            };
            if constexpr (NC <= 4) {
                if (a.waves == 8) return form(std::integral_constant<int, 8>{});
            }
            form(std::integral_constant<int, 4>{});
        };
        if (a.c.head_dim <= 64) run(std::integral_constant<int, 2>{});
        else if (a.c.head_dim <= 128) run(std::integral_constant<int, 4>{});
        else run(std::integral_constant<int, 8>{});
        if (a.splits == 1) return;
        auto join = [&](auto lanesc) {
            constexpr int LANES = decltype(lanesc)::value;
            const dim3 rows((unsigned)(a.c.sequences * a.heads));
            if (joiners == 64) hipLaunchKernelGGL((paged_attention_join_kernel<DT, LANES, 64>), rows, dim3(joiners), 0, st, a);
            else hipLaunchKernelGGL((paged_attention_join_kernel<DT, LANES, kMaxSplits>), rows, dim3(joiners), 0, st, a);
        };
        if (a.c.head_dim <= 64) join(std::integral_constant<int, 16>{});
        else if (a.c.head_dim <= 128) join(std::integral_constant<int, 32>{});
        else join(std::integral_constant<int, 64>{});
    };
    if (dt == NPAS_BF16) pick(std::integral_constant<int, NPAS_BF16>{});
    else pick(std::integral_constant<int, NPAS_F16>{});
    return launched("paged attention");
}

} // namespace npas
