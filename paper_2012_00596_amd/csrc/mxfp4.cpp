// C-ABI calls of the linear layers in microscaled 4-bit floats: packing on the host, argument checks, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <memory>
#include <exception>
#include <thread>

#include "mxfp4_internal.h"

using namespace npas;

namespace {

bool misaligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

int check_dtype(int dt)
{
    if (dt == NPAS_F32 || dt == NPAS_BF16 || dt == NPAS_F16) return NPAS_OK;
    set_error("unknown storage type %d", dt);
    return NPAS_E_DTYPE;
}

float bits(uint32_t u)
{
    float v;
    memcpy(&v, &u, 4);
    return v;
}

// n elements of a row to fp32 bit patterns.
void widen(const void *w, size_t i, int n, int dt, uint32_t *u)
{
    if (dt == NPAS_F32) memcpy(u, (const uint32_t *)w + i, (size_t)n * 4);
    else if (dt == NPAS_BF16)
        for (int k = 0; k < n; ++k) u[k] = (uint32_t)((const uint16_t *)w)[i + k] << 16;
    else
        for (int k = 0; k < n; ++k) {
            const uint32_t h = ((const uint16_t *)w)[i + k], sign = (h & 0x8000u) << 16, e = h >> 10 & 31, m = h & 1023;
            float v = (float)m * 0x1p-24f; // zero or subnormal
            uint32_t b;
            memcpy(&b, &v, 4);
            u[k] = sign | (e == 0 ? b : e == 31 ? 0x7f800000u | m << 13 : (e + 112) << 23 | m << 13);
        }
}

// One block of 32 values (fp32 bit patterns, zeros past the row's end) to 16 bytes of codes and the scale byte; false where one is not finite.
bool encode_block(const uint32_t u[32], uint8_t codes[16], uint8_t *scale)
{
    uint32_t top = 0;
    for (int i = 0; i < 32; ++i) top = std::max(top, u[i] & 0x7fffffffu);
    const uint32_t e = top >> 23;
    if (e == 255) return false;
    *scale = (uint8_t)(e > 2 ? e - 2 : 0);
    const float inv = bits((254u - *scale) << 23); // 2^-(scale - 127), exact
    uint8_t c[32];
    for (int i = 0; i < 32; ++i) {
        const float a = bits(u[i] & 0x7fffffffu) * inv; // exact; between two neighbouring values the even code takes the middle
        const int code = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.0f);
        c[i] = (uint8_t)(code | u[i] >> 28 & 8u);
    }
    for (int i = 0; i < 16; ++i) codes[i] = (uint8_t)(c[2 * i] | c[2 * i + 1] << 4);
    return true;
}

// Rows [lo, hi) of the weights to codes and scales, and to their places in the images (blob, where there is one).  Returns the first block
// (row * blocks + block) that holds a number that is not finite, or -1.
int64_t pack_rows(npas_mxfp4 *p, const void *w, int lo, int hi, uint8_t *blob)
{
    uint8_t *words = blob ? blob + (size_t)p->groups * p->steps * 2048 : nullptr;
    for (int o = lo; o < hi; ++o) {
        const int g = o >> 6, r = (o & 63) >> 1, j = o & 1;
        for (int b = 0; b < p->blocks; ++b) {
            const size_t at = (size_t)o * p->blocks + b;
            uint32_t v[32] = {};
            widen(w, (size_t)o * p->IN + b * 32, std::min(32, p->IN - b * 32), p->dtype, v);
            if (!encode_block(v, &p->codes[at * 16], &p->scales[at])) return (int64_t)at;
            if (!blob) continue;
            const int step = b >> 1, lane = (b & 1) * 32 + r;
            memcpy(blob + (((size_t)g * p->steps + step) * 2 + j) * 1024 + lane * 16, &p->codes[at * 16], 16);
            words[((((size_t)g * p->quads + (step >> 2)) * 2 + j) * 64 + lane) * 4 + (step & 3)] = p->scales[at];
        }
    }
    return -1;
}

// The same over all rows, large layers by up to eight threads (8192 x 4096 bf16: 75 ms by one).
int64_t pack_all(npas_mxfp4 *p, const void *w, uint8_t *blob)
{
    const int64_t per = (int64_t)1 << 21; // elements that are worth a thread
    const int n = (int)std::min<int64_t>(std::min(8u, std::max(1u, std::thread::hardware_concurrency())), (int64_t)p->OUT * p->IN / per + 1);
    // bounds between threads at whole groups: no two write one word of scales
    auto bound = [&](int i) { return (int)std::min<int64_t>(p->OUT, (int64_t)p->groups * i / n * 64); };
    std::vector<int64_t> bad(n, -1);
    std::vector<std::thread> workers;
    workers.reserve(n);
    int started = 1;
    try {
        for (; started < n; ++started)
            workers.emplace_back([&, i = started] { bad[i] = pack_rows(p, w, bound(i), bound(i + 1), blob); });
    } catch (const std::exception &) { // no more threads: the rest here
    }
    bad[0] = pack_rows(p, w, 0, bound(1), blob);
    for (int i = started; i < n; ++i) bad[i] = pack_rows(p, w, bound(i), bound(i + 1), blob);
    for (std::thread &t : workers) t.join();
    for (int64_t b : bad)
        if (b >= 0) return b;
    return -1;
}

bool on_gpu(int *dev)
{
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) == hipSuccess && ndev > 0 && hipGetDevice(dev) == hipSuccess) return true;
    (void)hipGetLastError();
    return false;
}

int upload(npas_mxfp4 *p, const std::vector<uint8_t> &blob, int dev, void *hip_stream)
{
    void *ptr = nullptr;
    hipError_t e = hipMalloc(&ptr, blob.size());
    if (e != hipSuccess) {
        (void)hipGetLastError(); // reported here, not by the next launch
        set_error("hipMalloc(%zu) failed: %s", blob.size(), hipGetErrorString(e));
        return NPAS_E_HIP;
    }
    // on the caller's stream; the source is the caller's buffer, so wait for the copy before it goes away
    e = hipMemcpyAsync(ptr, blob.data(), blob.size(), hipMemcpyHostToDevice, (hipStream_t)hip_stream);
    if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)hip_stream);
    if (e != hipSuccess) {
        (void)hipFree(ptr);
        (void)hipGetLastError();
        set_error("hipMemcpy to device failed: %s", hipGetErrorString(e));
        return NPAS_E_HIP;
    }
    p->device = dev;
    p->blob = ptr;
    p->bytes = blob.size();
    p->images = ptr;
    p->image_scales = (const uint32_t *)((const uint8_t *)ptr + (size_t)p->groups * p->steps * 2048);
    return NPAS_OK;
}

int check_rows(const void *a, const void *b, const void *c, int rows, int K, int dt)
{
    if (!a || !b || !c) {
        set_error("NULL argument");
        return NPAS_E_NULL;
    }
    if (int rc = check_dtype(dt)) return rc;
    if (rows <= 0 || K <= 0 || K > 1 << 24) {
        set_error("bad shape rows=%d K=%d", rows, K);
        return NPAS_E_SHAPE;
    }
    return NPAS_OK;
}

// Rows whose blocks are counted through in one go: fewer than 2^30 blocks, so that a reciprocal divides exactly.
int row_slab(int rows, int blocks) { return std::min(rows, std::max(1, (1 << 30) / blocks)); }

// Activations in the workspace: images of 32 rows, then their scale words.
int row_tiles(int B) { return (int)(((int64_t)B + 31) / 32); }
size_t image_bytes(const npas_mxfp4 *p, int B) { return (size_t)row_tiles(B) * p->steps * 1024; }

} // namespace

extern "C" {

int npas_mxfp4_quantize(const void *x_dev, int64_t x_stride, void *codes_dev, void *scales_dev, int rows, int K, npas_dtype dt,
                        void *hip_stream)
{
    if (int rc = check_rows(x_dev, codes_dev, scales_dev, rows, K, dt)) return rc;
    if (x_stride < K || x_stride > (int64_t)1 << 40 || misaligned(x_dev, dtype_size(dt)) || misaligned(codes_dev, 4)) {
        set_error("row stride %lld of %d elements, or a pointer that is not aligned (x to its element, codes to 4 bytes)", (long long)x_stride, K);
        return NPAS_E_SHAPE;
    }
    const int blocks = (K + 31) / 32;
    QuantizeArgs a{x_dev, (uint8_t *)codes_dev, (uint8_t *)scales_dev, x_stride, rows, K, blocks, 0, 0, magic_div_wide(blocks), row_slab(rows, blocks)};
    return launch_mxfp4_quantize(dt, a, hip_stream);
}

int npas_mxfp4_dequantize(const void *codes_dev, const void *scales_dev, void *y_dev, int rows, int K, npas_dtype dt,
                          void *hip_stream)
{
    if (int rc = check_rows(codes_dev, scales_dev, y_dev, rows, K, dt)) return rc;
    if (misaligned(y_dev, dtype_size(dt)) || misaligned(codes_dev, 4)) {
        set_error("a pointer that is not aligned (y to its element, codes to 4 bytes)");
        return NPAS_E_SHAPE;
    }
    const int blocks = (K + 31) / 32;
    DequantizeArgs a{(const uint8_t *)codes_dev, (const uint8_t *)scales_dev, y_dev, rows, K, blocks, magic_div_wide(blocks), row_slab(rows, blocks)};
    return launch_mxfp4_dequantize(dt, a, hip_stream);
}

int npas_pack_fc_mxfp4(const void *w_host, int OUT, int IN, npas_dtype dt, void *hip_stream, npas_mxfp4 **out)
{
    if (!w_host || !out) {
        set_error("NULL argument (w_host=%p out=%p)", w_host, (void *)out);
        return NPAS_E_NULL;
    }
    *out = nullptr;
    if (OUT <= 0 || IN <= 0 || OUT > 1 << 24 || IN > 1 << 24) {
        set_error("bad shape OUT=%d IN=%d", OUT, IN);
        return NPAS_E_SHAPE;
    }
    if (int rc = check_dtype(dt)) return rc;
    try {
        std::unique_ptr<npas_mxfp4> p(new npas_mxfp4);
        p->dtype = dt; p->OUT = OUT; p->IN = IN;
        p->blocks = (IN + 31) / 32; p->steps = (p->blocks + 3) / 4 * 2; p->quads = (p->steps + 3) / 4; p->groups = (OUT + 63) / 64;
        p->codes.resize((size_t)OUT * p->blocks * 16);
        p->scales.resize((size_t)OUT * p->blocks);
        int dev = 0;
        const bool gpu = on_gpu(&dev); // otherwise a host-only handle: export works, run calls fail loudly
        std::vector<uint8_t> blob(gpu ? (size_t)p->groups * (p->steps * 2048 + p->quads * 512) : 0, 0);
        const int64_t bad = pack_all(p.get(), w_host, gpu ? blob.data() : nullptr);
        if (bad >= 0) {
            const int b = (int)(bad % p->blocks);
            set_error("a weight of output %d, inputs %d .. %d, is not finite", (int)(bad / p->blocks), b * 32, std::min(IN, b * 32 + 32) - 1);
            return NPAS_E_SHAPE;
        }
        if (gpu)
            if (int rc = upload(p.get(), blob, dev, hip_stream)) return rc;
        *out = p.release();
        return NPAS_OK;
    } catch (const std::exception &e) { // no host memory for so large a layer
        set_error("packing %d x %d weights: %s", OUT, IN, e.what());
        return NPAS_E_SHAPE;
    }
}

int npas_mxfp4_info(const npas_mxfp4 *p, int64_t info[8])
{
    if (!p || !info) {
        set_error("NULL argument");
        return NPAS_E_NULL;
    }
    const int64_t v[8] = {p->dtype, p->OUT, p->IN, p->blocks, p->device >= 0, (int64_t)p->bytes, 0, 0};
    memcpy(info, v, sizeof(v));
    return NPAS_OK;
}

int npas_mxfp4_export(const npas_mxfp4 *p, uint8_t *codes_host, uint8_t *scales_host)
{
    if (!p) {
        set_error("NULL handle");
        return NPAS_E_NULL;
    }
    if (codes_host) memcpy(codes_host, p->codes.data(), p->codes.size());
    if (scales_host) memcpy(scales_host, p->scales.data(), p->scales.size());
    return NPAS_OK;
}

void npas_mxfp4_free(npas_mxfp4 *p)
{
    if (!p) return;
    if (p->blob) (void)hipFree(p->blob);
    delete p;
}

size_t npas_fc_mxfp4_workspace_bytes(const npas_mxfp4 *p, int B)
{
    if (!p || B <= 0 || fc_mxfp4_quantises(B, p->steps, p->groups)) return 0;
    return image_bytes(p, B) + (size_t)row_tiles(B) * p->quads * 256;
}

int npas_fc_mxfp4(const npas_mxfp4 *p, const void *x_dev, int64_t x_stride, void *y_dev, int B, const void *bias_dev, npas_act act,
                  void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    if (!p || !x_dev || !y_dev) {
        set_error("NULL argument (handle=%p x_dev=%p y_dev=%p)", (const void *)p, x_dev, y_dev);
        return NPAS_E_NULL;
    }
    if (B <= 0 || x_stride < p->IN || x_stride > (int64_t)1 << 40 || (row_tiles(B) / 8 + 1.0) * (p->groups / 2 + 1.0) * 256 > 4294967295.0 ||
        (double)row_tiles(B) * p->steps * 256 > 4294967295.0) { // (threads of its launches)
        set_error("bad shape B=%d, row stride %lld of %d elements", B, (long long)x_stride, p->IN);
        return NPAS_E_SHAPE;
    }
    if (!valid_act(act)) {
        set_error("unknown activation %d", (int)act);
        return NPAS_E_SHAPE;
    }
    if (misaligned(x_dev, dtype_size(p->dtype)) || misaligned(y_dev, dtype_size(p->dtype)) || misaligned(bias_dev, 4)) {
        set_error("a pointer is not aligned to its element type");
        return NPAS_E_SHAPE;
    }
    const size_t need = npas_fc_mxfp4_workspace_bytes(p, B);
    if (need && (!workspace_dev || workspace_bytes < need || misaligned(workspace_dev, 16))) {
        set_error("the layer needs %zu bytes of workspace at a multiple of 16 for %d rows, got %zu at %p", need, B, workspace_bytes, workspace_dev);
        return NPAS_E_WORKSPACE;
    }
    if (p->device < 0) {
        set_error("packed layer has no device copy (packed on a machine without a GPU)");
        return NPAS_E_HIP;
    }
    FcMxArgs a{x_dev, x_stride, nullptr, nullptr, p->images, p->image_scales, (const float *)bias_dev, y_dev, B, p->IN, p->OUT, p->blocks, p->steps,
               p->quads, p->groups, row_tiles(B), act};
    if (!fc_mxfp4_quantises(B, p->steps, p->groups)) {
        uint8_t *images = (uint8_t *)workspace_dev, *words = images + image_bytes(p, B);
        QuantizeArgs q{x_dev, images, words, x_stride, B, p->IN, p->blocks, p->steps, p->quads, WideDiv{}, 0};
        if (int rc = launch_mxfp4_quantize_images(p->dtype, q, hip_stream)) return rc;
        a.x_images = images;
        a.x_scales = (const uint32_t *)words;
    }
    return launch_fc_mxfp4(p->dtype, a, hip_stream);
}

} // extern "C"
