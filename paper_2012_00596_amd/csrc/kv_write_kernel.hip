// Rows in and out of the paged cache: per-head norms, rotation and the write of keys and values in 16-bit or 8-bit numbers, and 8-bit numbers back.
#include <type_traits>

#include "cache8.h"
#include "decoder_internal.h"
#include "row_vectors.h"

namespace npas {

// Where token t lies in the cache: whether it is a token at all, whether it is stored, and the cache row of its first head.
struct Place {
    bool token, stored;
    size_t row;
    int position;
};
__device__ __forceinline__ Place place_of(const CacheArgs &c, const int32_t *sequence, const int32_t *position, int t, uint32_t positions)
{
    const int s = sequence ? sequence[t] : t, pos = position[t];
    Place p;
    p.token = (uint32_t)s < (uint32_t)c.sequences && (uint32_t)pos < positions;
    const int column = p.token ? pos / c.page_size : 0, slot = p.token ? pos - column * c.page_size : 0;
    const int page = p.token && column < c.table_stride ? c.table[(size_t)s * c.table_stride + column] : -1;
    p.stored = (uint32_t)page < (uint32_t)c.pages;
    p.row = p.stored ? (size_t)page * c.kv_heads * c.page_size + slot : 0;
    p.position = p.token ? pos : 0;
    return p;
}

// Another lane's value by a fixed pattern within 16 lanes, without LDS.
template <int CTRL> __device__ __forceinline__ uint32_t lane16(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true); }
template <int CTRL> __device__ __forceinline__ float lane16(float x) { return __uint_as_float(lane16<CTRL>(__float_as_uint(x))); }
constexpr int kLaneXor1 = 0xb1, kLaneXor2 = 0x4e, kQuadMirror = 0x1b, kMirror8 = 0x141, kMirror16 = 0x140, kTurn8 = 0x128;
// Sum over P lanes, the same bits in each: a tree whose steps add what both sides add.
template <int P> __device__ __forceinline__ float lanes_sum(float s)
{
    s += lane16<kLaneXor1>(s);
    s += lane16<kLaneXor2>(s);
    s += lane16<kMirror8>(s);
    if constexpr (P >= 16) s += lane16<kMirror16>(s);
    if constexpr (P >= 32) s += __shfl_xor(s, 16);
    return s;
}
// The value of the lane P / 2 away, of P.
template <int P> __device__ __forceinline__ float far_half(float x)
{
    if constexpr (P == 8) return lane16<kQuadMirror>(lane16<kMirror8>(x));
    else if constexpr (P == 16) return lane16<kTurn8>(x);
    else return __shfl_xor(x, 16);
}

// How a rotation's partners are found: in the lane itself (PAIRS), half a head away, some lanes away, or through LDS.
enum { PAIRS, FAR_HALF, LANES, LDS };

// One workgroup a token.  P lanes, a power of two, hold a head, eight consecutive elements each; heads follow each other (queries, keys, values), four of a
// lane's on their way at once.  A lane's elements are the same in every head, so that its angles and weights are read once.
// The sum of squares is a tree over the P lanes, of lane patterns where 16 lanes hold a head (through LDS 49.6 us of the prompt below, so 47.5).  A block of
// 8-bit floats is four lanes.
// Bound by memory for long calls: 8191 tokens of 32 query and 8 key heads of 128, 206 MB, 46 us between other launches (4.4 TB/s; a large copy 5.0), 34 where
// the caches still hold what it reads.  5003 tokens of 20 query and 5 key heads of 80 elements into 8 bits 15.8 us of a row of calls (2.5 TB/s), into 16 15.4, keys and
// values alone 11.3 and 11.0: what 8 bits save in bytes, and what their conversion costs, hardly show.  Vector instructions take 60 % of that time, 40000 tokens go
// at 3.7 TB/s; what bounds the short call beside its latencies is not known.  For single tokens a launch and a chain of latencies, position, page, row: 24 tokens
// 10 us from call to call.
template <int DT, bool E8, int ROT, int P> __global__ __launch_bounds__(256) void kv_write_kernel(WriteArgs a)
{
    constexpr int SIDE = 4; // heads of a lane on their way
    __shared__ __align__(16) float pass[ROT == LDS ? 2048 : 1];
    constexpr bool WHOLE = ROT == FAR_HALF || ROT == LANES; // half of rot_dim is a multiple of eight
    const int t = blockIdx.x, D = a.c.head_dim, half = a.rot_dim / 2, in_head = threadIdx.x % P, d = in_head * 8, groups = blockDim.x / P;
    const Place at = place_of(a.c, a.sequence, a.position, t, a.rot_dim ? (uint32_t)a.positions : 0x80000000u);
    const bool mine = d < D, rotated = mine && d < a.rot_dim; // (WHOLE or not, a vector may pass the end of the rotated part)
    const int nq = a.q ? a.heads : 0, units = nq + 2 * a.c.kv_heads; // (all are read: that need not wait for the page)
    float cs[8] = {}, sn[8] = {}, wq[8] = {}, wk[8] = {};
    if (rotated) {
        const float *row = a.cos_sin + (size_t)at.position * a.rot_dim;
        if constexpr (ROT == PAIRS) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = d / 2 + k;
                cs[k] = i < half ? row[i] : 1.f;
                sn[k] = i < half ? row[half + i] : 0.f;
            }
        } else if constexpr (WHOLE) {
            const int i = d < half ? d : d - half;
            load8<NPAS_F32>(row, i, 8, cs);
            load8<NPAS_F32>(row, half + i, 8, sn);
        } else
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int e = d + k, i = e < half ? e : e - half;
                cs[k] = e < a.rot_dim ? row[i] : 1.f;
                sn[k] = e < a.rot_dim ? row[half + i] : 0.f;
            }
        if constexpr (ROT != PAIRS)
#pragma unroll
            for (int k = 0; k < 8; ++k) sn[k] = d + k < half ? -sn[k] : sn[k];
    }
    if (a.q_weight && mine) load8<NPAS_F32>(a.q_weight, d, 8, wq);
    if (a.k_weight && mine) load8<NPAS_F32>(a.k_weight, d, 8, wk);
    for (int first = threadIdx.x / P; first < units; first += SIDE * groups) {
        float x[SIDE][8];
#pragma unroll
        for (int j = 0; j < SIDE; ++j) {
            const int u = first + j * groups;
#pragma unroll
            for (int k = 0; k < 8; ++k) x[j][k] = 0.f;
            if (u >= units || !mine) continue;
            const bool is_q = u < nq, is_k = !is_q && u < nq + a.c.kv_heads;
            const int head = is_q ? u : is_k ? u - nq : u - nq - a.c.kv_heads;
            load8<DT>(is_q ? a.q : is_k ? a.k : a.v, (size_t)t * (is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride) + (size_t)head * D + d, 8, x[j]);
        }
#pragma unroll
        for (int j = 0; j < SIDE; ++j) {
            const int u = first + j * groups;
            if (u >= units) continue; // (all lanes of a head alike)
            const bool is_q = u < nq, is_k = !is_q && u < nq + a.c.kv_heads, normed = is_q ? a.q_weight != nullptr : is_k && a.k_weight;
            const int head = is_q ? u : is_k ? u - nq : u - nq - a.c.kv_heads;
            if (normed) {
                float s = 0.f;
#pragma unroll
                for (int k = 0; k < 8; ++k) s = fmaf(x[j][k], x[j][k], s);
                const float mean = fmaf(lanes_sum<P>(s), a.inv_d, a.eps);
                const bool small = mean < 0x1p-100f; // (the instruction takes a subnormal number for zero)
                const float r = __builtin_amdgcn_rsqf(small ? mean * 0x1p64f : mean) * (small ? 0x1p32f : 1.f); // (an ulp; what lies behind the head is zero and stays so)
                if (is_q) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[j][k] *= r * wq[k];
                } else {
                    asm volatile(""); // (two paths, one of which a wave mostly takes, not a choice for every weight)
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[j][k] *= r * wk[k];
                }
            }
            if (a.rot_dim && (is_q || is_k)) {
                if constexpr (ROT == PAIRS) {
                    if (rotated)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float u0 = x[j][2 * k], u1 = x[j][2 * k + 1];
                            x[j][2 * k] = u0 * cs[k] - u1 * sn[k];
                            x[j][2 * k + 1] = u1 * cs[k] + u0 * sn[k];
                        }
                } else {
                    float p[8];
                    if constexpr (ROT == FAR_HALF) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) p[k] = far_half<P>(x[j][k]);
                    } else if constexpr (ROT == LANES) {
                        const int from = (d < half ? in_head + half / 8 : in_head - half / 8) & (P - 1);
#pragma unroll
                        for (int k = 0; k < 8; ++k) p[k] = __shfl(x[j][k], from, P);
                    } else {
                        // (a wave's own part of LDS: its lanes meet, other waves do not matter)
                        float *row = pass + (threadIdx.x / P) * P * 8;
#pragma unroll
                        for (int k = 0; k < 8; ++k) row[d + k] = x[j][k];
                        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                        __builtin_amdgcn_wave_barrier();
                        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const int e = d + k, o = e < half ? e + half : e - half;
                            p[k] = e < a.rot_dim ? row[o] : 0.f;
                        }
                        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                        __builtin_amdgcn_wave_barrier();
                        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                    }
                    if (rotated)
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (WHOLE || d + k < a.rot_dim) x[j][k] = x[j][k] * cs[k] + p[k] * sn[k];
                }
            }
            if (is_q) {
                if (!at.token)
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[j][k] = 0.f;
                if (mine) store8<DT>(a.q_out, ((size_t)t * a.heads + head) * D + d, 8, x[j]);
                continue;
            }
            if (!at.stored) continue;
            const size_t row = at.row + (size_t)head * a.c.page_size;
            if constexpr (E8) {
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(x[j][k]) & 0x7fffffffu);
                top = max(top, lane16<kLaneXor1>(top));
                top = max(top, lane16<kLaneXor2>(top));
                const uint32_t byte = scale8_of<DT>(top);
                const uint2 codes = to_e4m3x8<DT>(x[j], byte);
                if (mine) {
                    *reinterpret_cast<uint2 *>(reinterpret_cast<uint8_t *>(is_k ? a.c.k : a.c.v) + row * D + d) = codes;
                    if ((in_head & 3) == 0) (is_k ? a.c.k_scale : a.c.v_scale)[row * ((D + 31) >> 5) + (d >> 5)] = (uint8_t)byte;
                }
            } else if (mine) store8<DT>(is_k ? a.c.k : a.c.v, row * D + d, 8, x[j]);
        }
    }
}

int launch_kv_write(int dt, const WriteArgs &a, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    const int lanes = a.c.head_dim <= 64 ? 8 : a.c.head_dim <= 128 ? 16 : 32;
    const long threads = ((a.q ? a.heads : 0) + 2l * a.c.kv_heads) * lanes;
    const dim3 grid((unsigned)a.T), block(threads <= 64 ? 64 : threads <= 128 ? 128 : 256);
    if (int rc = check_grid("cache write", grid.x, block.x)) return rc;
    auto form = [&](auto dtc, auto e8c, auto lanesc) {
        constexpr int DT = decltype(dtc)::value, P = decltype(lanesc)::value;
        constexpr bool E8 = decltype(e8c)::value;
        if (a.pairs) hipLaunchKernelGGL((kv_write_kernel<DT, E8, PAIRS, P>), grid, block, 0, st, a);
        else if (a.rot_dim == 8 * P) hipLaunchKernelGGL((kv_write_kernel<DT, E8, FAR_HALF, P>), grid, block, 0, st, a);
        else if (a.rot_dim % 16 == 0) hipLaunchKernelGGL((kv_write_kernel<DT, E8, LANES, P>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((kv_write_kernel<DT, E8, LDS, P>), grid, block, 0, st, a);
    };
    auto width = [&](auto dtc, auto e8c) {
        if (lanes == 8) form(dtc, e8c, std::integral_constant<int, 8>{});
        else if (lanes == 16) form(dtc, e8c, std::integral_constant<int, 16>{});
        else form(dtc, e8c, std::integral_constant<int, 32>{});
    };
    auto cache = [&](auto dtc) {
        if (a.c.k_scale) width(dtc, std::true_type{});
        else width(dtc, std::false_type{});
    };
    if (dt == NPAS_BF16) cache(std::integral_constant<int, NPAS_BF16>{});
    else cache(std::integral_constant<int, NPAS_F16>{});
    return launched("cache write");
}

// One workgroup a token; a thread has eight elements of a key or value: a code is its value times a power of two, so nothing is rounded.
// 5003 tokens of 5 key heads of 80 5 us, 2.4 TB/s: one round of workgroups, the chain position, page, row; 40000 tokens 27 us, 3.6 TB/s.
template <int DT> __global__ __launch_bounds__(256) void kv_read_kernel(ReadArgs a)
{
    const int t = blockIdx.x, D = a.c.head_dim, vectors = D >> 3, heads = a.c.kv_heads, blocks = (D + 31) >> 5;
    const Place at = place_of(a.c, a.sequence, a.position, t, 0x80000000u);
    const int parts = (a.k_out != nullptr) + (a.v_out != nullptr);
    for (int u = threadIdx.x; u < parts * heads * vectors; u += blockDim.x) {
        const int unit = u / vectors, d = (u - unit * vectors) * 8;
        const bool is_k = a.k_out && unit < heads;
        const int head = unit < heads ? unit : unit - heads;
        uint4 y = make_uint4(0, 0, 0, 0);
        if (at.stored) {
            const size_t row = at.row + (size_t)head * a.c.page_size;
            const uint2 codes = *reinterpret_cast<const uint2 *>(reinterpret_cast<const uint8_t *>(is_k ? a.c.k : a.c.v) + row * D + d);
            y = from_e4m3x8<DT>(codes, (is_k ? a.c.k_scale : a.c.v_scale)[row * blocks + (d >> 5)]);
        }
        const u32x4_any out = {y.x, y.y, y.z, y.w};
        __builtin_nontemporal_store(out, reinterpret_cast<u32x4_any *>(reinterpret_cast<uint16_t *>(is_k ? a.k_out : a.v_out) + ((size_t)t * heads + head) * D + d));
    }
}

int launch_kv_read(int dt, const ReadArgs &a, void *stream)
{
    hipStream_t st = (hipStream_t)stream;
    const long units = ((a.k_out != nullptr) + (a.v_out != nullptr)) * (long)a.c.kv_heads * (a.c.head_dim >> 3);
    const dim3 grid((unsigned)a.T), block(units <= 64 ? 64 : units <= 128 ? 128 : 256);
    if (int rc = check_grid("cache read", grid.x, block.x)) return rc;
    if (dt == NPAS_BF16) hipLaunchKernelGGL((kv_read_kernel<NPAS_BF16>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((kv_read_kernel<NPAS_F16>), grid, block, 0, st, a);
    return launched("cache read");
}

} // namespace npas
