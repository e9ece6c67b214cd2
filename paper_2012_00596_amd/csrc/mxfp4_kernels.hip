// Microscaled 4-bit floats: rows to codes and scales and back, and the product of quantised activations and packed weights on the
// scaled matrix instructions.
#include <type_traits>

#include "mxfp4_internal.h"
#include "row_vectors.h"

namespace npas {

// A quarter of a block: 8 elements as they are stored (fp32: as they are, 16-bit types: four words).
template <int DT> struct Quarter {
    uint32_t w[DT == NPAS_F32 ? 8 : 4];
};
template <int DT> __device__ __forceinline__ void load_quarter(const void *p, size_t i, int n, Quarter<DT> &q)
{
    if constexpr (DT == NPAS_F32) {
        float v[8];
        load8<DT>(p, i, n, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) q.w[k] = __float_as_uint(v[k]);
    } else if (n >= 8) {
        const Words16 x = *reinterpret_cast<const Words16 *>(reinterpret_cast<const uint16_t *>(p) + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) q.w[k] = x.w[k];
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t lo = 2 * k < n ? reinterpret_cast<const uint16_t *>(p)[i + 2 * k] : 0;
            const uint32_t hi = 2 * k + 1 < n ? reinterpret_cast<const uint16_t *>(p)[i + 2 * k + 1] : 0;
            q.w[k] = lo | hi << 16;
        }
    }
}

// A quarter's codes; the four lanes of a block are neighbours and agree on its scale byte.  Magnitudes are compared as bits (16-bit types two at
// a time): a NaN is above an infinity, an infinity above every number.  The conversions round to nearest, ties to the even code, and stop
// at 6; x / 2^e is exact in them for 16-bit types (checked for every value with every scale that a block of it can have), as is x times
// 2^-e in fp32 (down to the smallest numbers).
template <int DT> __device__ __forceinline__ uint32_t encode8(const Quarter<DT> &q, uint32_t &scale)
{
    uint32_t e, c = 0;
    if constexpr (DT == NPAS_F32) {
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = max(top, q.w[k] & 0x7fffffffu);
        top = max(top, (uint32_t)__shfl_xor((int)top, 1));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2));
        e = top >> 23;
    } else {
        typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
        u16x2 top = {0, 0};
#pragma unroll
        for (int k = 0; k < 4; ++k) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, q.w[k] & 0x7fff7fffu));
#pragma unroll
        for (int x = 1; x < 3; ++x) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, __shfl_xor(__builtin_bit_cast(int, top), x)));
        const uint16_t m = top[0] > top[1] ? top[0] : top[1];
        e = (__float_as_uint(from_storage<DT>(m)) & 0x7fffffffu) >> 23;
    }
    scale = e == 255 ? 255u : e > 2 ? e - 2 : 0u;
    if (e == 255) return 0u;
    if constexpr (DT == NPAS_F32) {
        const float inv = __uint_as_float((254u - scale) << 23);
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = __builtin_amdgcn_fmed3f(__uint_as_float(q.w[k]) * inv, -6.f, 6.f);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[0], w[1], 1.f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[2], w[3], 1.f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[4], w[5], 1.f, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, w[6], w[7], 1.f, 3);
    } else {
        const float unit = __uint_as_float(scale ? scale << 23 : 0x00400000u);
        typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
        typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
#define NPAS_PAIR(k)                                                                                                                  \
    if constexpr (DT == NPAS_BF16) c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, q.w[k]), unit, k);     \
    else c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, q.w[k]), unit, k);
        NPAS_PAIR(0) NPAS_PAIR(1) NPAS_PAIR(2) NPAS_PAIR(3)
#undef NPAS_PAIR
    }
    return c;
}

// Canonical rows: four neighbouring lanes a block, blocks counted through all rows of a slab (blockIdx.y), so that a row that ends in the
// middle of a workgroup leaves no lane idle; two blocks' quarters a thread, both asked for before the first is used.
// Memory bound: 8192 x 4100 bf16 in 15 us (5.6 TB/s; a workgroup a row's piece of 64 blocks 23).
template <int DT> __global__ __launch_bounds__(256) void mxfp4_quantize_kernel(QuantizeArgs a)
{
    const int row0 = blockIdx.y * a.slab, part = threadIdx.x & 3;
    const uint32_t end = (uint32_t)min(a.slab, a.rows - row0) * a.blocks;
    Quarter<DT> v[2];
    uint32_t n[2];
    size_t row[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        n[i] = blockIdx.x * 128 + i * 64 + (threadIdx.x >> 2);
        const uint32_t m = n[i] < end ? n[i] : end - 1, r = fastdiv_wide(m, a.by_blocks);
        row[i] = row0 + r;
        const int k0 = (int)(m - r * a.blocks) * 32 + part * 8;
        load_quarter<DT>(a.x, row[i] * a.x_stride + k0, a.K - k0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t scale;
        const uint32_t c = encode8<DT>(v[i], scale);
        if (n[i] >= end) continue;
        const size_t b = (size_t)row0 * a.blocks + n[i];
        reinterpret_cast<uint32_t *>(a.codes)[b * 4 + part] = c;
        if (part == 0) a.scales[b] = (uint8_t)scale;
    }
}

// Operand images: a workgroup takes a step of a tile, four neighbouring lanes a block; what it writes is one image.  4096 x 4096 bf16 in 9.0-10
// us (4.2-4.7 TB/s).
template <int DT> __global__ __launch_bounds__(256) void mxfp4_quantize_images_kernel(QuantizeArgs a)
{
    const int step = blockIdx.x % a.steps, tile = blockIdx.x / a.steps, h = threadIdx.x >> 7, r = threadIdx.x >> 2 & 31, part = threadIdx.x & 3;
    const int row = tile * 32 + r, k0 = step * 64 + h * 32 + part * 8;
    Quarter<DT> v;
    load_quarter<DT>(a.x, (size_t)(row < a.rows ? row : 0) * a.x_stride + k0, row < a.rows ? a.K - k0 : 0, v);
    uint32_t scale;
    const uint32_t c = encode8<DT>(v, scale);
    reinterpret_cast<uint32_t *>(a.codes)[((size_t)tile * a.steps + step) * 256 + threadIdx.x] = c;
    if (part == 0) a.scales[(((size_t)tile * a.quads + (step >> 2)) * 64 + h * 32 + r) * 4 + (step & 3)] = (uint8_t)scale;
}

// The way back, counted through like the rows above, eight values a thread: 8192 x 4100 bf16 in 14.7 us (5.8 TB/s).
template <int DT> __global__ __launch_bounds__(256) void mxfp4_dequantize_kernel(DequantizeArgs a)
{
    const int row0 = blockIdx.y * a.slab, part = threadIdx.x & 3;
    const uint32_t end = (uint32_t)min(a.slab, a.rows - row0) * a.blocks;
    uint32_t c[2], s[2], n[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        n[i] = blockIdx.x * 128 + i * 64 + (threadIdx.x >> 2);
        const size_t b = (size_t)row0 * a.blocks + (n[i] < end ? n[i] : end - 1);
        c[i] = reinterpret_cast<const uint32_t *>(a.codes)[b * 4 + part];
        s[i] = a.scales[b];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (n[i] >= end) return;
        const uint32_t r = fastdiv_wide(n[i], a.by_blocks);
        const int k0 = (int)(n[i] - r * a.blocks) * 32 + part * 8;
        const float unit = __uint_as_float(s[i] == 255 ? 0x7fc00000u : s[i] ? s[i] << 23 : 0x00400000u);
        float v[8];
#define NPAS_PAIR(k)                                                             \
    {                                                                            \
        const auto p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], 1.f, k);   \
        v[2 * k] = p[0] * unit;                                                  \
        v[2 * k + 1] = p[1] * unit;                                              \
    }
        NPAS_PAIR(0) NPAS_PAIR(1) NPAS_PAIR(2) NPAS_PAIR(3)
#undef NPAS_PAIR
        store8<DT>(a.y, (size_t)(row0 + r) * a.K + k0, a.K - k0, v);
    }
}

// ---- product --------------------------------------------------------------------

typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
__device__ __forceinline__ i32x8 operand(uint4 v) { return i32x8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0}; }
// 32 x 32 x 64 of two 4-bit images; byte S of each lane's scale word is its block's scale.  (A loop of nothing but this instruction runs at
// 6.7 PFLOP/s on random codes, of 16 x 16 x 128 with scales at 4.6-5.2.)
template <int S> __device__ __forceinline__ f32x16 mfma_mx(uint4 a, uint32_t sa, uint4 b, uint32_t sb, f32x16 c)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(a), operand(b), c, 4, 4, S, (int)sa, S, (int)sb);
}
// Row of a tile that result register i of lane 32 h + n holds (its column is n: outputs 2 n and 2 n + 1 of the group in its two images).
__device__ __forceinline__ int result_row(int i, int lane) { return 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3); }

// The activation with NaN passed on (rows whose blocks stand for NaN stay NaN).
template <int ACT> __device__ __forceinline__ float activate(float v)
{
    if constexpr (ACT == NPAS_ACT_RELU) return v < 0.f ? 0.f : v;
    if constexpr (ACT == NPAS_ACT_RELU6) {
        const float w = v < 0.f ? 0.f : v;
        return w > 6.f ? 6.f : w;
    }
    if constexpr (ACT == NPAS_ACT_HARDSWISH) return v * __builtin_amdgcn_fmed3f(v + 3.f, 0.f, 6.f) * (1.f / 6.f);
    return v;
}
// Calls f with the launch's activation as a constant: chosen once, not per value.
template <typename F> __device__ __forceinline__ void with_activation(int act, F &&f)
{
    if (act == NPAS_ACT_NONE) f(std::integral_constant<int, NPAS_ACT_NONE>{});
    else if (act == NPAS_ACT_RELU) f(std::integral_constant<int, NPAS_ACT_RELU>{});
    else if (act == NPAS_ACT_RELU6) f(std::integral_constant<int, NPAS_ACT_RELU6>{});
    else f(std::integral_constant<int, NPAS_ACT_HARDSWISH>{});
}
// What a wave's lanes have written to or read from LDS is done before its other lanes read or write there (one wave's accesses are in order in
// the hardware; this keeps the compiler, to which they are of unlike types, from moving them).
__device__ __forceinline__ void wave_meets()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}
// A lane's two biases of a group.
__device__ __forceinline__ float2 group_bias(const FcMxArgs &a, int o)
{
    return make_float2(a.bias && o < a.OUT ? a.bias[o] : 0.f, a.bias && o + 1 < a.OUT ? a.bias[o + 1] : 0.f);
}

// Few rows: a workgroup takes 32 rows and J of a group's two images (32 outputs each), its W waves every W-th run of four steps; their sums
// are added through LDS, in the waves' order.  Nothing passes through LDS on the way in: all of a run's loads are asked for at once.
// FUSED (few enough rows that quantising them again in every workgroup costs less than a launch): the workgroup brings its rows to
// codes in LDS, four lanes a block, while its first weights are on their way.
// One row of 4096 x 4096 4.2-4.9 us (8.9 MB: launch, one round trip to memory, the exchange of the sums; 1.8 us at the rate of a copy), 256 rows
// of 1280 x 1000 4.0 us and 2.6 for their images.
template <int DT, int W, int J, bool FUSED> __global__ __launch_bounds__(64 * W) void fc_mxfp4_split_kernel(FcMxArgs a)
{
    constexpr int PARTS = 2 / J;
    __shared__ __align__(16) uint8_t lds[W * J * 4096]; // codes and scale bytes of at most 512 steps (34 bytes each), then the sums
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, h = lane >> 5;
    const int part = blockIdx.x % PARTS, group = blockIdx.x / PARTS % a.groups, tile = blockIdx.x / PARTS / a.groups;
    const uint4 *x = reinterpret_cast<const uint4 *>(a.x_images) + (size_t)tile * a.steps * 64 + lane;
    const uint4 *w = reinterpret_cast<const uint4 *>(a.w_images) + ((size_t)group * a.steps * 2 + part) * 64 + lane;
    const uint32_t *ws = a.w_scales + ((size_t)group * a.quads * 2 + part) * 64 + lane;
    const int rows = min(32, a.B - tile * 32);
    f32x16 c[J] = {};
    uint4 wv[4][J], xv[4];
    uint32_t sw[J], sx = 0;
    auto load = [&](int quad) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < J; ++j) sw[j] = ws[(quad * 2 + j) * 64];
#pragma unroll
        for (int s = 0; s < 4; ++s)
            if (quad * 4 + s < a.steps)
#pragma unroll
                for (int j = 0; j < J; ++j) wv[s][j] = w[((quad * 4 + s) * 2 + j) * 64];
        if constexpr (!FUSED) {
            sx = a.x_scales[((size_t)tile * a.quads + quad) * 64 + lane];
#pragma unroll
            for (int s = 0; s < 4; ++s)
                if (quad * 4 + s < a.steps) xv[s] = x[(quad * 4 + s) * 64];
        }
    };
    auto multiply = [&](int quad) __attribute__((always_inline)) {
        auto step = [&](auto sc) __attribute__((always_inline)) {
            constexpr int S = decltype(sc)::value;
            const int s = quad * 4 + S;
            if (s >= a.steps) return;
            uint4 xo;
            uint32_t so = sx;
            if constexpr (FUSED) { // rows are a multiple of 16 bytes long in LDS, their scale bytes behind all of them
                const int block = 2 * s + h;
                xo = make_uint4(0, 0, 0, 0);
                so = 0;
                if (r < rows) {
                    xo = *reinterpret_cast<const uint4 *>(lds + ((size_t)r * a.steps * 2 + block) * 16);
                    so = (uint32_t)lds[(size_t)rows * a.steps * 32 + r * a.steps * 2 + block] << 8 * S;
                }
            } else xo = xv[S];
#pragma unroll
            for (int j = 0; j < J; ++j) c[j] = mfma_mx<S>(xo, so, wv[S][j], sw[j], c[j]);
        };
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
    };
    int quad = wave;
    if (quad < a.quads) load(quad);
    if constexpr (FUSED) {
        const int quarters = a.steps * 8; // of a row, up to the last step's end
        for (int u = threadIdx.x; u < rows * quarters; u += 64 * W) {
            const int row = u / quarters, k = u - row * quarters;
            Quarter<DT> v;
            load_quarter<DT>(a.x, (size_t)(tile * 32 + row) * a.x_stride + k * 8, a.IN - k * 8, v);
            uint32_t scale;
            const uint32_t code = encode8<DT>(v, scale);
            reinterpret_cast<uint32_t *>(lds)[row * quarters + k] = code;
            if ((k & 3) == 0) lds[(size_t)rows * a.steps * 32 + row * a.steps * 2 + (k >> 2)] = (uint8_t)scale;
        }
        __syncthreads();
    }
    for (; quad < a.quads; quad += W) {
        multiply(quad);
        if (quad + W < a.quads) load(quad + W);
    }
    // [wave][image][row][output]: lane 32 h + n holds rows of its half, output n of the image
    if constexpr (FUSED) __syncthreads();
    float *part_sum = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (result_row(i, lane) < rows) part_sum[((wave * J + j) * 32 + result_row(i, lane)) * 32 + r] = c[j][i];
    __syncthreads();
    const int waves = min(W, a.quads);
    with_activation(a.act, [&](auto act) __attribute__((always_inline)) {
        for (int u = threadIdx.x; u < rows * 32 * J; u += 64 * W) { // consecutive threads, consecutive outputs
            const int row = u / (32 * J), k = u % (32 * J), j = J == 2 ? k & 1 : 0, n = J == 2 ? k >> 1 : k, o = group * 64 + 2 * n + (J == 2 ? j : part);
            float v = 0.f;
            for (int i = 0; i < waves; ++i) v += part_sum[((i * J + j) * 32 + row) * 32 + n];
            if (o < a.OUT) st_act<DT>(a.y, (size_t)(tile * 32 + row) * a.OUT + o, activate<decltype(act)::value>(v + (a.bias ? a.bias[o] : 0.f)));
        }
    });
}

// Many rows: a workgroup of 2 x 2 waves, each RR row tiles by RC weight images, walks the stages (two steps) together.  Operand images and
// scale words come to LDS lane by lane as they lie in memory (direct loads, nothing held in registers, three stages in a ring), so that
// an operand read is one 16-byte LDS read without bank conflicts.  A wave reads stage t + 1's operands while it multiplies stage t's: a
// row tile's take the place of this stage's as soon as the row has been multiplied; weights, used by all rows, and the last row's (so
// that no read is young when the wave reaches the barrier) have two places.  One barrier a stage: before it a wave waits until its own
// loads of stage t + 1 have landed (all but those of the stage behind it may be outstanding) and its reads of stage t are done; behind
// it stage t is free for stage t + 3.
// 4096 x 4096 -> 8192 in 67-75 us (4.1-3.7 PFLOP/s), about 18 of them launch, first stages and 67 MB of results; the loop runs at 5-5.7
// PFLOP/s of the 6.7 that nothing but such instructions reach.  With zeros for codes the whole call takes 63-66 us instead of 82-92: so much
// is power.  The rest above the 41 of the instructions is those 18, which two rounds of workgroups do not cover, and 9 for the codes.
// LDS: a stage's operand reads and direct loads take as many cycles as its multiplications (128 x 128 tiles 1.33 times as many); 256 x 256
// tiles of four waves, 0.67, had no second workgroup to cover their stores (71.9 us).
template <int DT, int RR, int RC> struct MxTile {
    static constexpr int XI = 4 * RR, WI = 4 * RC, STAGE = (XI + WI) * 1024, RING = 3;  // images of a stage: activations, then weights
    static constexpr int SCALES = (2 * RR + 2 * RC) * 256, LOADS = RR + RC;              // scale words of two stages; loads of a wave, a stage
    // results on their way out: PASS row tiles of a wave at a time, rows far enough apart that the halves of a wave meet other banks
    static constexpr int ESIZE = DT == NPAS_F32 ? 4 : 2, PASS = RR / 2, PITCH = RC * 32 * ESIZE + 32;
    static constexpr int LOOP = RING * STAGE + 2 * SCALES, OUT = 4 * PASS * 32 * PITCH, LDS = LOOP > OUT ? LOOP : OUT;
};
template <int N> __device__ __forceinline__ void wait_and_meet() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory"); }

template <int DT, int RR, int RC> __global__ __launch_bounds__(256, 2) void fc_mxfp4_tile_kernel(FcMxArgs a)
{
    using L = MxTile<DT, RR, RC>;
    constexpr int NT = 2 * RR, NG = RC; // row tiles and groups of 64 outputs of the workgroup
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const uint32_t lbase = (uint32_t)(uintptr_t)lds;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave >> 1, wc = wave & 1;
    // Workgroups of an XCD: runs of 8 row blocks by as many output blocks, so that what they read together stays in its L2.
    const uint32_t id = xcd_remap(blockIdx.x, gridDim.x), rb = (a.tiles + NT - 1) / NT, cb = (a.groups + NG - 1) / NG, band = id / (8 * cb);
    const uint32_t high = rb - band * 8 < 8 ? rb - band * 8 : 8, in = id - band * 8 * cb;
    const int tile0 = (int)(band * 8 + in % high) * NT, group0 = (int)(in / high) * NG, stages = a.steps >> 1;
    const int tiles = min(NT, a.tiles - tile0), groups = min(NG, a.groups - group0); // blocks at the edge read the last one's again
    const uint32_t lane16 = lane * 16u;

    // What a wave fetches of a stage: RR images of activations and RC of weights, and of two stages' scale words one kilobyte (the
    // activations' RR / 2 by the first waves, the weights' by the others, some of them the same).  In LDS activations lie [tile][step],
    // weights [group][step][image].
    const uint32_t xs = (uint32_t)a.steps * 1024u, ws = (uint32_t)a.steps * 2048u, xq = (uint32_t)a.quads * 256u, wq = (uint32_t)a.quads * 512u;
    const u32x4 xsrc = buffer_of((const uint8_t *)a.x_images + (size_t)tile0 * xs, tiles * xs);
    const u32x4 wsrc = buffer_of((const uint8_t *)a.w_images + (size_t)group0 * ws, groups * ws);
    const bool scales_of_x = wave < RR / 2;
    const u32x4 ssrc = scales_of_x ? buffer_of((const uint8_t *)a.x_scales + (size_t)tile0 * xq, tiles * xq)
                                   : buffer_of((const uint8_t *)a.w_scales + (size_t)group0 * wq, groups * wq);
    const int part = scales_of_x ? wave : min(wave - RR / 2, RC / 2 - 1); // four tiles, or two groups
    const uint32_t sat = scales_of_x ? (uint32_t)min(part * 4 + (lane >> 4), tiles - 1) * xq + (lane & 15) * 16u
                                     : (uint32_t)min(part * 2 + (lane >> 5), groups - 1) * wq + (lane & 31) * 16u;
    const uint32_t sstep = scales_of_x ? 256u : 512u, sdst = lbase + L::RING * L::STAGE + (scales_of_x ? 0u : NT * 256u) + part * 1024u;
    uint32_t xat[RR], wat[RC];
#pragma unroll
    for (int k = 0; k < RR; ++k) xat[k] = (uint32_t)min((wave * RR + k) >> 1, tiles - 1) * xs + ((wave * RR + k) & 1) * 1024u;
#pragma unroll
    for (int k = 0; k < RC; ++k) wat[k] = (uint32_t)min((wave * RC + k) >> 2, groups - 1) * ws + ((wave * RC + k) & 3) * 1024u;
    auto fetch = [&](int t, uint32_t slot, int k) __attribute__((always_inline)) {
        if (k < RR) lds_buffer16(xsrc, lane16, xat[k < RR ? k : 0] + (uint32_t)t * 2048u, lbase + slot + (wave * RR + k) * 1024u);
        else lds_buffer16(wsrc, lane16, wat[k < RR ? 0 : k - RR] + (uint32_t)t * 4096u, lbase + slot + (L::XI + wave * RC + k - RR) * 1024u);
    };
    auto fetch_scales = [&](int quad) __attribute__((always_inline)) {
        lds_buffer16(ssrc, sat, (uint32_t)quad * sstep, sdst + (uint32_t)(quad & 1) * L::SCALES);
    };

    uint4 x0[RR], x1[RR - 1], xl[2], w0[RC], w1[2][RC]; // of a stage's first step, and of its second: all but the last row tile, the last
    uint32_t sx[RR], sw[RC], nsw[RC];
    f32x16 c[RR][RC] = {};
    auto read_x = [&](uint32_t slot, int i, int u) __attribute__((always_inline)) {
        return *reinterpret_cast<const uint4 *>(lds + slot + lane16 + (wr * RR * 2 + i * 2 + u) * 1024);
    };
    auto read_w = [&](uint32_t slot, int j, int u) __attribute__((always_inline)) {
        return *reinterpret_cast<const uint4 *>(lds + slot + lane16 + (L::XI + wc * RC * 2 + (j / 2) * 4 + u * 2 + (j & 1)) * 1024);
    };
    auto read_sx = [&](int quad, int i) __attribute__((always_inline)) {
        return *reinterpret_cast<const uint32_t *>(lds + L::RING * L::STAGE + (quad & 1) * L::SCALES + (wr * RR + i) * 256 + lane * 4);
    };
    auto read_sw = [&](int quad, int j) __attribute__((always_inline)) {
        return *reinterpret_cast<const uint32_t *>(lds + L::RING * L::STAGE + (quad & 1) * L::SCALES + (NT + wc * RC + j) * 256 + lane * 4);
    };

    for (int t = 0; t < 3 && t < stages; ++t) {
        if ((t & 1) == 0) fetch_scales(t >> 1);
#pragma unroll
        for (int k = 0; k < L::LOADS; ++k) fetch(t, t * L::STAGE, k);
    }
    if (stages >= 3) wait_and_meet<2 * L::LOADS + 1>(); // (stage 2's scale words)
    else wait_and_meet<0>();
    uint32_t slot = 0, slot1 = L::STAGE, slot2 = 2 * L::STAGE; // of stages t, t + 1, t + 2
#pragma unroll
    for (int i = 0; i < RR; ++i) {
        sx[i] = read_sx(0, i);
        x0[i] = read_x(0, i, 0);
        if (i < RR - 1) x1[i] = read_x(0, i, 1);
        else xl[0] = read_x(0, i, 1);
    }
#pragma unroll
    for (int j = 0; j < RC; ++j) {
        sw[j] = read_sw(0, j);
        w0[j] = read_w(0, j, 0);
        w1[0][j] = read_w(0, j, 1);
    }

    // Stage t (P: odd).  MAIN: stages up to t + 3 exist, nothing is asked.
    auto stage = [&](int t, auto pc, auto mainc) __attribute__((always_inline)) {
        constexpr int P = decltype(pc)::value;
        constexpr bool MAIN = decltype(mainc)::value;
        const bool far = MAIN || t + 3 < stages;
        if (MAIN || t + 2 < stages) wait_and_meet<L::LOADS + (P == 0)>(); // (of stage t + 2, with scale words where it is even)
        else wait_and_meet<0>();
        if (far && P == 1) fetch_scales((t + 3) >> 1);
        if (!MAIN && far)
#pragma unroll
            for (int k = 0; k < L::LOADS; ++k) fetch(t + 3, slot, k);
        // where there is no next stage the reads bring what lies there, and nothing uses it
        xl[P ^ 1] = read_x(slot1, RR - 1, 1);
#pragma unroll
        for (int i = 0; i < RR; ++i) {
            if (MAIN && i < L::LOADS) fetch(t + 3, slot, i);
            if (i < RC) w1[P ^ 1][i < RC ? i : 0] = read_w(slot1, i, 1);
#pragma unroll
            for (int j = 0; j < RC; ++j) c[i][j] = mfma_mx<2 * P>(x0[i], sx[i], w0[j], sw[j], c[i][j]);
            x0[i] = read_x(slot1, i, 0);
        }
#pragma unroll
        for (int i = 0; i < RR; ++i) {
            if (MAIN && RR + i < L::LOADS) fetch(t + 3, slot, RR + i);
            if (i < RC) {
                w0[i < RC ? i : 0] = read_w(slot1, i, 0);
                if (P == 1) nsw[i < RC ? i : 0] = read_sw((t + 1) >> 1, i);
            }
            const uint4 x = i < RR - 1 ? x1[i < RR - 1 ? i : 0] : xl[P];
#pragma unroll
            for (int j = 0; j < RC; ++j) c[i][j] = mfma_mx<2 * P + 1>(x, sx[i], w1[P][j], sw[j], c[i][j]);
            if (i < RR - 1) x1[i] = read_x(slot1, i, 1);
            if (P == 1) sx[i] = read_sx((t + 1) >> 1, i);
        }
        if (P == 1)
#pragma unroll
            for (int j = 0; j < RC; ++j) sw[j] = nsw[j];
        const uint32_t first = slot;
        slot = slot1, slot1 = slot2, slot2 = first;
    };
    static_assert(RC <= RR && L::LOADS <= 2 * RR, "reads and fetches are spread over the row tiles");
    int t = 0;
    for (; t + 4 < stages; t += 2) {
        stage(t, std::integral_constant<int, 0>{}, std::true_type{});
        stage(t + 1, std::integral_constant<int, 1>{}, std::true_type{});
    }
    for (; t < stages; t += 2) {
        stage(t, std::integral_constant<int, 0>{}, std::false_type{});
        if (t + 1 < stages) stage(t + 1, std::integral_constant<int, 1>{}, std::false_type{});
    }

    // Results through the wave's own part of LDS, so that rows leave in runs of 16 bytes a lane.
    const int o0 = (group0 + wc * (RC / 2)) * 64, r0 = (tile0 + wr * RR) * 32, n = lane & 31;
    float2 b[RC / 2];
#pragma unroll
    for (int j = 0; j < RC / 2; ++j) {
        b[j] = group_bias(a, o0 + j * 64 + 2 * n);
        asm volatile("" : "+v"(b[j].x), "+v"(b[j].y)); // the wait for the loads stands here, not at every store
    }
    uint8_t *own = lds + wave * (L::PASS * 32 * L::PITCH);
    __syncthreads();
#pragma unroll
    for (int i0 = 0; i0 < RR; i0 += L::PASS) {
        if (i0) wave_meets(); // the pass before has been read
        with_activation(a.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < L::PASS; ++i)
#pragma unroll
                for (int k = 0; k < 16; ++k)
#pragma unroll
                    for (int j = 0; j < RC / 2; ++j) {
                        const float v0 = activate<decltype(act)::value>(c[i0 + i][2 * j][k] + b[j].x);
                        const float v1 = activate<decltype(act)::value>(c[i0 + i][2 * j + 1][k] + b[j].y);
                        uint8_t *p = own + (i * 32 + result_row(k, lane)) * L::PITCH + (j * 64 + 2 * n) * L::ESIZE;
                        if constexpr (DT == NPAS_F32) *reinterpret_cast<float2 *>(p) = make_float2(v0, v1);
                        else *reinterpret_cast<uint32_t *>(p) = pack2<DT>(v0, v1);
                    }
        });
        wave_meets();
        constexpr int LANES = RC * 32 / 8; // lanes of a row, 8 results each
#pragma unroll 4
        for (int u = lane; u < L::PASS * 32 * LANES; u += 64) {
            const int r = u / LANES, o = u % LANES * 8, row = r0 + i0 * 32 + r, left = a.OUT - o0 - o;
            if (row >= a.B || left <= 0) continue;
            const size_t at = (size_t)row * a.OUT + o0 + o;
            const uint8_t *p = own + r * L::PITCH + o * L::ESIZE;
            if (left >= 8) store_vectors<8 * L::ESIZE>((uint8_t *)a.y + at * L::ESIZE, p);
            else
#pragma unroll
                for (int k = 0; k < 7; ++k)
                    if (k < left) {
                        if constexpr (DT == NPAS_F32) reinterpret_cast<uint32_t *>(a.y)[at + k] = reinterpret_cast<const uint32_t *>(p)[k];
                        else reinterpret_cast<uint16_t *>(a.y)[at + k] = reinterpret_cast<const uint16_t *>(p)[k];
                    }
        }
    }
}

// ---- launches -------------------------------------------------------------------

template <typename F> static int with_dtype(int dt, const char *what, F &&f)
{
    if (dt == NPAS_F32) f(std::integral_constant<int, NPAS_F32>{});
    else if (dt == NPAS_BF16) f(std::integral_constant<int, NPAS_BF16>{});
    else f(std::integral_constant<int, NPAS_F16>{});
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return NPAS_OK;
    set_error("%s launch failed: %s", what, hipGetErrorString(e));
    return NPAS_E_HIP;
}

// 128 blocks a workgroup, by slabs.  (In 64 bits: rows and a slab together pass 2^31.)
static dim3 slab_grid(int rows, int slab, int blocks)
{
    return dim3((unsigned)(((long)slab * blocks + 127) / 128), (unsigned)(((long)rows + slab - 1) / slab));
}

int launch_mxfp4_quantize(int dt, const QuantizeArgs &a, void *stream)
{
    const dim3 grid = slab_grid(a.rows, a.slab, a.blocks);
    return with_dtype(dt, "4-bit quantisation", [&](auto dtc) {
        hipLaunchKernelGGL((mxfp4_quantize_kernel<decltype(dtc)::value>), grid, dim3(256), 0, (hipStream_t)stream, a);
    });
}

int launch_mxfp4_quantize_images(int dt, const QuantizeArgs &a, void *stream)
{
    const dim3 grid((unsigned)((a.rows + 31L) / 32 * a.steps));
    return with_dtype(dt, "4-bit quantisation", [&](auto dtc) {
        hipLaunchKernelGGL((mxfp4_quantize_images_kernel<decltype(dtc)::value>), grid, dim3(256), 0, (hipStream_t)stream, a);
    });
}

int launch_mxfp4_dequantize(int dt, const DequantizeArgs &a, void *stream)
{
    const dim3 grid = slab_grid(a.rows, a.slab, a.blocks);
    return with_dtype(dt, "4-bit dequantisation", [&](auto dtc) {
        hipLaunchKernelGGL((mxfp4_dequantize_kernel<decltype(dtc)::value>), grid, dim3(256), 0, (hipStream_t)stream, a);
    });
}

// Pieces of 32 rows x 32 outputs; with one workgroup each on 256 compute units they take (pieces + 255) / 256 rounds.
static long pieces_of(int B, int groups) { return (long)((B + 31L) / 32) * groups * 2; }

// Few elements are quantised again in every workgroup rather than by a launch of their own: what counts is how often a compute unit does it.
// bf16, us replayed from a graph, so / by two launches: 4096 x 4096 1 row 4.2 / 6.1, 4 rows 5.3 / 6.1, 8 rows 6.7 / 6.2, 16 rows 9.7 / 6.2;
// 1280 x 1000 16 rows 4.9 / 5.4, 32 rows 6.5 / 5.5; 2048 -> 16384 4 rows 6.0 / 6.8, 8 rows 7.1 / 6.9; 4096 -> 32000 2 rows 15.0 / 15.1, 4 rows
// 17.8 / 15.2; 512 -> 512 512 rows 5.4 / 5.5.  A launch takes 1.6 to 2.4 us to issue on top.
bool fc_mxfp4_quantises(int B, int steps, int groups)
{
    return (long)(B < 32 ? B : 32) * steps * ((pieces_of(B, groups) + 255) / 256) <= 512;
}

// Which kernel, by how many pieces of 32 rows x 32 outputs there are (us for 2048 -> 8192; sixteen waves on each piece / eight on two / tiles
// of 128 x 128: 256 pieces 6.9 / 7.6 / 9.3, 512 8.3 / 8.4 / 10.3, 1024 12.7 / 9.3 / 10.2, 2048 22.8 / 14.7 / 10.8; for 8192 -> 1024 512
// pieces 15.9 / 14.5 / 24.1, 1024 27.0 / 21.6 / 27.4, 2048 47 / 33.7 / 30.0), and tiles of 256 x 128 where two of them come to a compute
// unit (4096 x 4096 -> 8192 67.5 us, with 128 x 128 70.8; 2048 x 4096 -> 4096, 256 tiles, 31.2 and 30.5).
int launch_fc_mxfp4(int dt, const FcMxArgs &a, void *stream)
{
    using std::integral_constant;
    auto tiled = [&](auto dtc, auto rrc) {
        constexpr int DT = decltype(dtc)::value, RR = decltype(rrc)::value;
        using L = MxTile<DT, RR, 2>;
        static std::once_flag once;
        allow_lds_once(once, fc_mxfp4_tile_kernel<DT, RR, 2>, L::LDS);
        const unsigned grid = (unsigned)((a.tiles + 2 * RR - 1) / (2 * RR)) * (unsigned)((a.groups + 1) / 2);
        hipLaunchKernelGGL((fc_mxfp4_tile_kernel<DT, RR, 2>), dim3(grid), dim3(256), L::LDS, (hipStream_t)stream, a);
    };
    auto split = [&](auto dtc, auto wc, auto jc, auto fc) {
        constexpr int DT = decltype(dtc)::value, W = decltype(wc)::value, J = decltype(jc)::value;
        constexpr bool FUSED = decltype(fc)::value;
        hipLaunchKernelGGL((fc_mxfp4_split_kernel<DT, W, J, FUSED>), dim3((unsigned)(a.tiles * a.groups * (2 / J))), dim3(64 * W), 0, (hipStream_t)stream, a);
    };
    const long pieces = pieces_of(a.B, a.groups), large = (long)((a.tiles + 7) / 8) * ((a.groups + 1) / 2);
    return with_dtype(dt, "4-bit product", [&](auto dtc) {
        if (!a.x_images && pieces <= 256) split(dtc, integral_constant<int, 16>{}, integral_constant<int, 1>{}, std::true_type{});
        else if (!a.x_images) split(dtc, integral_constant<int, 8>{}, integral_constant<int, 2>{}, std::true_type{});
        else if (pieces <= 256) split(dtc, integral_constant<int, 16>{}, integral_constant<int, 1>{}, std::false_type{});
        else if (pieces <= 1024) split(dtc, integral_constant<int, 8>{}, integral_constant<int, 2>{}, std::false_type{});
        else if (large < 512) tiled(dtc, integral_constant<int, 2>{});
        else tiled(dtc, integral_constant<int, 4>{});
    });
}

} // namespace npas
