// Patch rows: resize (two-tap bilinear or antialiased) + normalize + cut into patches, fused (gfx950).
//
// An output value is sum_j wy[j] sum_k wx[k] src[j][k]: per axis a window of source samples around
// the output sample's centre c = (i + 1/2) in / out - 1/2, two taps or a triangle of half-width s = max(in / out, 1).
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <cmath>
#include <stdint.h>

#include <new>

#include "../../include/prep.h"
#include "kernels.h"
#include "tokens.h"

namespace prep {

namespace {

constexpr int kThreads = 256;
constexpr int kClips = 32;  // clips of one launch: their records are kernel arguments (2 KB), so that a call has
                            // no workspace, calls may overlap and a captured call keeps its own

// One clip as the kernels see it.
struct PatchClip {
    uint64_t src_off;       // first byte of its first frame
    uint64_t frame_stride;  // bytes
    int64_t row0;           // its first row
    uint32_t pitch;
    int32_t width, height, out_w, out_h;  // pixels
    int32_t frames;
    int32_t image;          // index into `status`
    uint32_t block0;        // first workgroup of the launch that takes it
};
struct ClipPack {
    PatchClip c[kClips];
};
struct PatchGeometry {
    int32_t patch, merge, group;  // pixels, patches, frames
    int32_t antialias;
    float scale[3], bias[3];      // 1 / (255 std), -mean / std
};

// The taps of one output sample of one axis.
struct Taps {
    int first, end;
    float centre;  // c - floor(c - 1/2 ...) relative to `first`
    float inv;     // 1 / s
    int size;
};
__device__ __forceinline__ Taps make_taps(int i, int size, int out, bool antialias)
{
    // in 64 bits: a coordinate near 2000 would leave a float 13 bits of fraction
    const double scale = (double)size / (double)out;
    const double c = ((double)i + 0.5) * scale - 0.5;
    Taps t;
    const double s = antialias && scale > 1.0 ? scale : 1.0;
    t.first = (int)floor(c - s) + 1;  // weight 0 at c - s itself
    t.end = (int)ceil(c + s);
    t.centre = (float)(c - (double)t.first);
    t.inv = (float)(1.0 / s);
    t.size = size;
    return t;
}

// One thread produces the three channels of one pixel, pixels in the order of the rows.
template <typename T>
__global__ __launch_bounds__(kThreads) void patch_rows_kernel(const uint8_t *__restrict__ rgb, ClipPack pack, int n, PatchGeometry g,
                                                              const int32_t *__restrict__ status, T *__restrict__ out, int64_t out_stride)
{
    int i = 0;
    while (i + 1 < n && pack.c[i + 1].block0 <= blockIdx.x) i++;
    const PatchClip C = pack.c[i];
    const int area = g.patch * g.patch;
    const int cols = C.out_w / g.patch, rows = C.out_h / g.patch;
    const int64_t per_frame = (int64_t)C.out_w * C.out_h;
    const int64_t item = (int64_t)(blockIdx.x - C.block0) * kThreads + threadIdx.x;
    const int groups = (C.frames + g.group - 1) / g.group;
    if (item >= per_frame * g.group * groups) return;
    const int slot = (int)(item / per_frame), e = (int)(item - slot * per_frame);
    const int f = min(slot, C.frames - 1);
    const int row = e / area, in_patch = e - row * area;  // row of the group
    const int band = row / (g.merge * cols), r1 = row - band * g.merge * cols;
    const int window = r1 / (g.merge * g.merge), r2 = r1 - window * g.merge * g.merge;
    const int py = band * g.merge + r2 / g.merge, px = window * g.merge + r2 % g.merge;
    const int y = py * g.patch + in_patch / g.patch, x = px * g.patch + in_patch % g.patch;
    float v[3] = {0.0f, 0.0f, 0.0f};
    if (status == nullptr || status[C.image] == PREP_OK) {
        const Taps ty = make_taps(y, C.height, C.out_h, g.antialias), tx = make_taps(x, C.width, C.out_w, g.antialias);
        const uint8_t *src = rgb + C.src_off + (uint64_t)f * C.frame_stride;
        float sum = 0.0f;
        for (int j = ty.first; j < ty.end; j++) {
            // a two-tap window reaches over the border, where the border's sample counts; a triangle ends there
            if (ty.inv < 1.0f && (j < 0 || j >= C.height)) continue;
            const float wy = fmaxf(0.0f, 1.0f - fabsf((float)(j - ty.first) - ty.centre) * ty.inv);
            const uint8_t *line = src + (uint64_t)min(max(j, 0), C.height - 1) * C.pitch;
            for (int k = tx.first; k < tx.end; k++) {
                if (tx.inv < 1.0f && (k < 0 || k >= C.width)) continue;
                const float w = wy * fmaxf(0.0f, 1.0f - fabsf((float)(k - tx.first) - tx.centre) * tx.inv);
                const uint8_t *p = line + (int64_t)min(max(k, 0), C.width - 1) * 3;
                sum += w;
#pragma unroll
                for (int c = 0; c < 3; c++) v[c] = fmaf(w, (float)p[c], v[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < 3; c++) v[c] = fmaf(v[c] / sum, g.scale[c], g.bias[c]);
    }
    T *o = out + (C.row0 + (int64_t)(slot / g.group) * rows * cols + row) * out_stride + (int64_t)(slot % g.group) * area + in_patch;
#pragma unroll
    for (int c = 0; c < 3; c++) o[(int64_t)c * g.group * area] = from_float<T>(v[c]);
}

uint64_t floor_sqrt(uint64_t v)
{
    uint64_t r = 0;
    for (int b = 31; b >= 0; b--) {
        const uint64_t t = r | (1ull << b);
        if (t * t <= v) r = t;
    }
    return r;
}

bool patch_params_ok(const prep_patch_params *p)
{
    if (!p || p->patch < 1 || p->patch > 64 || p->merge < 1 || p->merge > 16 || p->frames_per_patch < 1 || p->frames_per_patch > 16 ||
        !float_type(p->out_dtype) || p->reserved != 0 || p->min_pixels < 0 || p->max_pixels < 0)
        return false;
    if (p->filter != PREP_FILTER_BILINEAR && p->filter != PREP_FILTER_ANTIALIAS) return false;
    for (int c = 0; c < 3; c++)
        if (!(p->std[c] > 0.0f) || !std::isfinite(p->std[c]) || !std::isfinite(p->mean[c])) return false;
    return true;
}

bool patch_size(const prep_patch_params *p, int32_t width, int32_t height, int32_t *rows, int32_t *cols)
{
    if (width < 1 || height < 1 || width > 65535 || height > 65535) return false;
    const uint64_t u = (uint64_t)p->patch * (uint64_t)p->merge, w = (uint64_t)width, h = (uint64_t)height;
    uint64_t kw = (2 * w + u) / (2 * u), kh = (2 * h + u) / (2 * u);
    if (kw == 0) kw = 1;
    if (kh == 0) kh = 1;
    const uint64_t pixels = kw * kh * u * u;
    // (a bound of 2^40 bounds nothing that fits the sides, and keeps the products in 64 bits)
    const uint64_t bound = 1ull << 40, least = (uint64_t)p->min_pixels, most = (uint64_t)p->max_pixels < bound ? (uint64_t)p->max_pixels : bound;
    if (most != 0 && pixels > most) {
        // k u <= side sqrt(most / (w h)), in whole numbers
        kw = floor_sqrt(w * most / (h * u * u));
        kh = floor_sqrt(h * most / (w * u * u));
        if (kw == 0) kw = 1;
        if (kh == 0) kh = 1;
    } else if (pixels < least) {
        if (least > 0xFFFFFFFFull) return false;
        auto up = [](uint64_t a, uint64_t b) {  // the smallest k with k k b >= a
            const uint64_t k = floor_sqrt(a / b);
            return k * k * b >= a ? k : k + 1;
        };
        kw = up(w * least, h * u * u);
        kh = up(h * least, w * u * u);
    }
    if (kw * u > 65535 || kh * u > 65535) return false;
    *cols = (int32_t)(kw * (uint64_t)p->merge);
    *rows = (int32_t)(kh * (uint64_t)p->merge);
    return true;
}

template <typename T>
void launch_for(const uint8_t *rgb, const ClipPack &pack, int n, uint32_t blocks, const PatchGeometry &g, const int32_t *status, T *out,
                int64_t out_stride, hipStream_t stream)
{
    hipLaunchKernelGGL((patch_rows_kernel<T>), dim3(blocks), dim3(kThreads), 0, stream, rgb, pack, n, g, status, out, out_stride);
}

// status: DEVICE, per PatchClip::image, or nullptr = all PREP_OK (others get rows of zeros).  clips: HOST, n of them,
// all but block0 filled in.
int launch_patch_rows(const uint8_t *rgb, const PatchClip *clips, int32_t n, const prep_patch_params *params, const int32_t *status, void *out,
                      int64_t out_stride, hipStream_t stream)
{
    PatchGeometry g;
    g.patch = params->patch;
    g.merge = params->merge;
    g.group = params->frames_per_patch;
    g.antialias = params->filter == PREP_FILTER_ANTIALIAS;
    for (int c = 0; c < 3; c++) {
        g.scale[c] = (float)(1.0 / (255.0 * (double)params->std[c]));
        g.bias[c] = (float)(-(double)params->mean[c] / (double)params->std[c]);
    }
    int32_t at = 0;
    while (at < n) {
        ClipPack pack;
        uint64_t blocks = 0;
        int m = 0;
        while (at < n && m < kClips) {
            const PatchClip &c = clips[at];
            const uint64_t groups = (uint64_t)((c.frames + g.group - 1) / g.group);
            const uint64_t mine = ((uint64_t)c.out_w * (uint64_t)c.out_h * groups * (uint64_t)g.group + kThreads - 1) / kThreads;
            if (blocks + mine > 0x7FFFFFFFull) break;
            pack.c[m] = c;
            pack.c[m].block0 = (uint32_t)blocks;
            blocks += mine;
            m++;
            at++;
        }
        for (int k = m; k < kClips; k++) pack.c[k] = pack.c[0];
        if (params->out_dtype == PREP_F16) launch_for(rgb, pack, m, (uint32_t)blocks, g, status, (__half *)out, out_stride, stream);
        else if (params->out_dtype == PREP_BF16) launch_for(rgb, pack, m, (uint32_t)blocks, g, status, (__hip_bfloat16 *)out, out_stride, stream);
        else launch_for(rgb, pack, m, (uint32_t)blocks, g, status, (float *)out, out_stride, stream);
    }
    return PREP_OK;
}

// The clips of a call: geometry, rows, and whether they fit.
class PatchCall {
public:
    PatchCall(const prep_patch_params *params, int32_t n, void *out, int64_t out_stride, int64_t out_rows, int64_t *row_starts)
        : params_(params), out_(out), out_stride_(out_stride), out_rows_(out_rows), row_starts_(row_starts), n_(n)
    {
    }
    ~PatchCall() { delete[] clips_; }
    PatchCall(const PatchCall &) = delete;
    PatchCall &operator=(const PatchCall &) = delete;

    int check()
    {
        if (n_ < 0 || !patch_params_ok(params_) || !row_starts_ || out_rows_ < 0 || (n_ > 0 && !out_)) return PREP_E_INVALID_ARG;
        const int64_t row = 3ll * params_->frames_per_patch * params_->patch * params_->patch;
        if (out_stride_ == 0) out_stride_ = row;
        if (out_stride_ < row || !aligned(out_, (uintptr_t)element_bytes(params_->out_dtype))) return PREP_E_INVALID_ARG;
        row_starts_[0] = 0;
        if (n_ > 0 && !(clips_ = new (std::nothrow) PatchClip[(size_t)n_])) return PREP_E_NOMEM;
        return PREP_OK;
    }
    // Clips come in ascending order; those left out have no rows.
    bool add(int32_t i, int32_t width, int32_t height, uint64_t src_off, uint32_t pitch, int32_t frames, uint64_t frame_stride)
    {
        int32_t rows, cols;
        skip_to(i);
        if (frames < 1 || !patch_size(params_, width, height, &rows, &cols)) return false;
        const int64_t groups = ((int64_t)frames - 1) / params_->frames_per_patch + 1;
        // a launch has fewer than 2^31 workgroups
        if (groups * params_->frames_per_patch * rows * cols * params_->patch * params_->patch > (int64_t)0x7FFFFFFF * kThreads) return false;
        PatchClip &c = clips_[count_++];
        c.src_off = src_off;
        c.frame_stride = frame_stride;
        c.row0 = row_starts_[i];
        c.pitch = pitch;
        c.width = width;
        c.height = height;
        c.out_w = cols * params_->patch;
        c.out_h = rows * params_->patch;
        c.frames = frames;
        c.image = i;
        c.block0 = 0;
        row_starts_[i + 1] = row_starts_[i] + groups * rows * cols;
        next_ = i + 1;
        return true;
    }
    int finish()
    {
        skip_to(n_);
        return row_starts_[n_] > out_rows_ ? PREP_E_TOO_LARGE : PREP_OK;
    }
    int launch(const uint8_t *rgb, const int32_t *status, hipStream_t stream)
    {
        return launch_patch_rows(rgb, clips_, count_, params_, status, out_, out_stride_, stream);
    }

private:
    void skip_to(int32_t i)
    {
        for (; next_ < i; next_++) row_starts_[next_ + 1] = row_starts_[next_];
    }
    const prep_patch_params *params_;
    void *out_;
    int64_t out_stride_, out_rows_, *row_starts_;
    int32_t n_, count_ = 0, next_ = 0;
    PatchClip *clips_ = nullptr;
};

// Behind the JPEG decoder.
struct PatchStage final : OutputStage {
    explicit PatchStage(PatchCall *call) : call_(call) {}
    bool add(int32_t image, int w, int h, uint64_t src_off, uint32_t pitch) override { return call_->add(image, w, h, src_off, pitch, 1, 0); }
    int ready() override { return call_->finish(); }
    int launch(const uint8_t *rgb, const int32_t *status, hipStream_t stream) override { return call_->launch(rgb, status, stream); }
    PatchCall *call_;
};

}  // namespace

}  // namespace prep

using namespace prep;

extern "C" {

int prep_patch_grid(const prep_patch_params *params, int32_t width, int32_t height, int32_t frames, int32_t grid[3])
{
    if (!patch_params_ok(params) || !grid || frames < 1) return PREP_E_INVALID_ARG;
    int32_t rows, cols;
    if (!patch_size(params, width, height, &rows, &cols)) return PREP_E_INVALID_ARG;
    grid[0] = (int32_t)(((int64_t)frames - 1) / params->frames_per_patch + 1);
    grid[1] = rows;
    grid[2] = cols;
    return PREP_OK;
}

int prep_patch_rows(int32_t device, const uint8_t *rgb, const uint64_t *rgb_offsets, const int32_t *widths, const int32_t *heights,
                    const int32_t *pitches, const int32_t *frames, const uint64_t *frame_strides, int32_t n, const prep_patch_params *params,
                    void *out, int64_t out_stride, int64_t out_rows, int64_t *row_starts, void *stream)
{
    if ((frames == nullptr) != (frame_strides == nullptr) || (n > 0 && (!rgb || !rgb_offsets || !widths || !heights || !pitches)))
        return PREP_E_INVALID_ARG;
    PatchCall call(params, n, out, out_stride, out_rows, row_starts);
    int rc = call.check();
    if (rc != PREP_OK) return rc;
    for (int32_t i = 0; i < n; i++) {
        const int32_t f = frames ? frames[i] : 1;
        if (widths[i] < 1 || heights[i] < 1 || widths[i] > 65535 || heights[i] > 65535 || pitches[i] < widths[i] * 3) return PREP_E_INVALID_ARG;
        if (f > 1 && frame_strides[i] < (uint64_t)pitches[i] * (uint64_t)(heights[i] - 1) + (uint64_t)widths[i] * 3) return PREP_E_INVALID_ARG;
        if (!call.add(i, widths[i], heights[i], rgb_offsets[i], (uint32_t)pitches[i], f, frame_strides ? frame_strides[i] : 0))
            return PREP_E_INVALID_ARG;
    }
    rc = call.finish();
    if (rc != PREP_OK || n == 0) return rc;
    DeviceScope scope(device);
    if (!scope.ok()) return PREP_E_HIP;
    rc = call.launch(rgb, nullptr, (hipStream_t)stream);
    if (hipGetLastError() != hipSuccess) return PREP_E_HIP;
    return rc;
}

int prep_decode_patches_batch(prep_handle *h, const uint8_t *bitstreams, const uint8_t *bitstreams_device, const uint64_t *offsets, int32_t n,
                              const prep_patch_params *params, void *out, int64_t out_stride, int64_t out_rows, int64_t *row_starts,
                              void *stream)
{
    if (!h || !bitstreams || !offsets) return PREP_E_INVALID_ARG;
    PatchCall call(params, n, out, out_stride, out_rows, row_starts);
    const int rc = call.check();
    if (rc != PREP_OK) return rc;
    PatchStage stage(&call);
    return decode_batch(h, bitstreams, bitstreams_device, offsets, n, &stage, (hipStream_t)stream);
}

}  // extern "C"
