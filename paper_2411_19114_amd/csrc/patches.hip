// Patch rows: resize (two-tap bilinear or antialiased) + normalize + cut into patches, fused (gfx950).
//
// An output value is sum_j wy[j] sum_k wx[k] src[j][k]: per axis a window of source samples around the output sample's
// centre c = (i + 1/2) in / out - 1/2, weights max(0, 1 - |j - c| / s) scaled to sum 1 over the samples inside the image, s =
// max(in / out, 1) (antialiased) or 1, which is two taps; a tap that the border would clamp counts for the border's sample either way.
//
// A workgroup makes a tile of patches: the source samples under the tile go to LDS, every wave sums a row's samples over the
// rows of its window (weights by row, whole bytes eight at a time), then over the columns, and leaves the values in LDS in the order
// of the patch rows, from where they are written in runs.
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

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kClips = 32;  // clips of one launch: their records are kernel arguments (3 KB), so that a call has
                            // no workspace, calls may overlap and a captured call keeps its own

// A tile's limits: pixels a side, pixels in all by element size, bytes of source samples, source samples of a row, taps of a row.
constexpr int kTileCols = 64, kTileRows = 32, kRawBytes = 18 << 10, kSpan = 150, kTaps = 32;
constexpr int stage_pixels(int element) { return element == 2 ? 2048 : 1024; }
constexpr int kPatches = 1024;      // of a tile (patches of few pixels)
constexpr int kLoads = 5;           // 16-byte reads of a thread that go out together
constexpr int kNarrowest = 6;       // narrowest image whose rows hold a read of 16 bytes

// One clip as the kernels see it.
struct PatchClip {
    uint64_t src_off;       // first byte of its first frame
    uint64_t frame_stride;  // bytes
    int64_t row0;           // its first row
    double scale_x, scale_y;  // source samples per output sample
    uint32_t pitch;
    int32_t width, height, out_w, out_h;  // pixels
    int32_t frames;
    int32_t image;          // index into `status`
    // tiles: patches across and down, rows of a patch in it (fewer than the patch has where that is tall: `parts` tiles
    // share a patch then), tiles across and down
    int32_t across, down, part_rows, parts, tiles_x, tiles_y;
};
struct ClipPack {
    uint32_t block0[kClips];  // first workgroup of each clip; of those that the launch lacks 2^32 - 1
    PatchClip c[kClips];
};
struct PatchGeometry {
    int32_t patch, merge, group;  // pixels, patches, frames
    int32_t antialias;
    float scale[3], bias[3];      // 1 / (255 std), -mean / std
};

// The window of one output sample of one axis, cut at the image's edge.
struct Taps {
    int first, end;
    float centre;  // relative to `first`
    float inv;     // 1 / s
    __device__ __forceinline__ float weight(int k) const { return fmaxf(0.0f, fmaf(-fabsf((float)k - centre), inv, 1.0f)); }
};
__host__ __device__ __forceinline__ Taps make_taps(int i, int size, double scale, bool antialias)
{
    // in 64 bits: a coordinate near 2000 would leave a float 13 bits of fraction
    const double c = ((double)i + 0.5) * scale - 0.5, s = antialias && scale > 1.0 ? scale : 1.0;
    Taps t;
    t.first = max((int)floor(c - s) + 1, 0);  // (weight 0 at c - s itself)
    t.end = min((int)ceil(c + s), size);
    t.centre = (float)(c - (double)t.first);
    t.inv = (float)(1.0 / s);
    return t;
}

// (without a branch: scalar loads of the whole list go out together)
__device__ __forceinline__ int clip_of(const ClipPack &pack, uint32_t block)
{
    int i = 0;
#pragma unroll
    for (int k = 1; k < kClips; k++) i += pack.block0[k] <= block ? 1 : 0;
    return i;
}

// Row, inside its group of frames, of patch (py, px).
__device__ __forceinline__ int row_of_patch(int py, int px, int cols, int merge)
{
    const int band = py / merge, window = px / merge;
    return band * merge * cols + window * merge * merge + (py - band * merge) * merge + (px - window * merge);
}

// What a wave's lanes have written to LDS is there for all of them.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 16 bytes at `at` of a row of `bytes` (at least 16) bytes, those behind the row's end 0: nothing outside the row is read.
__device__ __forceinline__ uint4 load_inside(const uint8_t *row, int at, int bytes)
{
    uint64_t lo, hi;
    const int from = min(at, bytes - 16), back = at - from;
    __builtin_memcpy(&lo, row + from, 8);
    __builtin_memcpy(&hi, row + from + 8, 8);
    if (back != 0) {
        if (back >= 8) {
            lo = hi;
            hi = 0;
        }
        const int bits = 8 * (back & 7);
        if (bits != 0) {
            lo = lo >> bits | hi << (64 - bits);
            hi >>= bits;
        }
    }
    return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
}

template <int kBytes> struct Chunk;
template <> struct Chunk<16> { typedef uint4 type; };
template <> struct Chunk<8> { typedef uint2 type; };
template <> struct Chunk<4> { typedef uint32_t type; };
template <> struct Chunk<2> { typedef uint16_t type; };

// A frame's runs of `run` elements, `n` of them (three of a patch), from the stage to the patches' rows, kBytes at a time.
template <typename T, int kBytes>
__device__ __forceinline__ void write_runs(const T *stage, const int32_t *row, int n, int run, T *out, int64_t out_stride, int64_t channel_stride)
{
    typedef typename Chunk<kBytes>::type C;
    constexpr int kElements = kBytes / (int)sizeof(T);
    const int chunks = run / kElements, by = kThreads / chunks, rest = kThreads - by * chunks;
    int r = (int)threadIdx.x / chunks, at = (int)threadIdx.x - r * chunks;
    while (r < n) {
        const int patch = r / 3, channel = r - 3 * patch;
        T *o = out + row[patch] * out_stride + channel * channel_stride + at * kElements;
        *reinterpret_cast<C *>(o) = *reinterpret_cast<const C *>(stage + r * run + at * kElements);
        r += by;
        at += rest;
        if (at >= chunks) {
            at -= chunks;
            r++;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void patch_rows_tiled(const uint8_t *__restrict__ rgb, ClipPack pack, PatchGeometry g,
                                                             const int32_t *__restrict__ status, T *__restrict__ out, int64_t out_stride,
                                                             int chunk)
{
    __shared__ alignas(16) uint8_t raw[kRawBytes];                      // the tile's source samples, rows 16-byte multiples apart
    __shared__ alignas(16) float summed[kWaves][kSpan * 3 + 6];         // a row's samples summed over its window, of each wave
    __shared__ alignas(16) T stage[stage_pixels((int)sizeof(T)) * 3];   // values by patch, channel, pixel
    __shared__ alignas(16) float row_weight[kTileRows][kTaps];          // scaled to sum 1, then 0
    __shared__ int32_t row_first[kTileRows], row_taps[kTileRows], row_stage[kTileRows];
    __shared__ int32_t col_first[kTileCols], col_taps[kTileCols], col_stage[kTileCols];
    __shared__ float col_centre[kTileCols], col_norm[kTileCols];
    __shared__ int32_t patch_row[kPatches];

    const int clip = clip_of(pack, blockIdx.x);
    const PatchClip &C = pack.c[clip];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t tile = blockIdx.x - pack.block0[clip];
    const int frames_group = (int)(tile / (uint32_t)(C.tiles_x * C.tiles_y));
    tile -= (uint32_t)frames_group * (uint32_t)(C.tiles_x * C.tiles_y);
    const int tile_y = (int)(tile / (uint32_t)C.tiles_x), tile_x = (int)(tile - (uint32_t)tile_y * (uint32_t)C.tiles_x);
    const int cols = C.out_w / g.patch, rows = C.out_h / g.patch;
    // the tile's patches, and its rows of pixels
    const int px0 = tile_x * C.across, across = min(C.across, cols - px0);
    const int py0 = tile_y / C.parts * C.down, down = min(C.down, rows - py0);
    const int part_y0 = tile_y % C.parts * C.part_rows;
    const int part_rows = C.parts > 1 ? min(C.part_rows, g.patch - part_y0) : g.patch;
    const int tile_w = across * g.patch, tile_h = down * part_rows, x0 = px0 * g.patch, y0 = py0 * g.patch + part_y0;
    const int run = part_rows * g.patch;  // of a patch's channel
    // the source samples under it; at least kNarrowest columns, so that a row holds a read of 16 bytes
    const bool antialias = g.antialias != 0;
    int c_end = make_taps(x0 + tile_w - 1, C.width, C.scale_x, antialias).end;
    const int c0 = max(min(make_taps(x0, C.width, C.scale_x, antialias).first, C.width - kNarrowest), 0);
    c_end = max(c_end, min(c0 + kNarrowest, C.width));
    const int r0 = make_taps(y0, C.height, C.scale_y, antialias).first, r_end = make_taps(y0 + tile_h - 1, C.height, C.scale_y, antialias).end;
    const int bytes = (c_end - c0) * 3, units = (bytes + 15) / 16, raw_pitch = units * 16;

    for (int t = threadIdx.x; t < tile_h; t += kThreads) {
        const Taps w = make_taps(y0 + t, C.height, C.scale_y, antialias);
        const int taps = w.end - w.first;
        float sum = 0.0f;
        for (int k = 0; k < taps; k++) sum += w.weight(k);
        for (int k = 0; k < taps; k++) row_weight[t][k] = w.weight(k) / sum;
        if (taps & 1) row_weight[t][taps] = 0.0f;
        row_first[t] = w.first - r0;
        row_taps[t] = taps;
        const int patch = t / part_rows;
        row_stage[t] = patch * across * 3 * run + (t - patch * part_rows) * g.patch;
    }
    for (int t = (int)threadIdx.x - 64; t < tile_w; t += kThreads) {
        if (t < 0) continue;
        const Taps w = make_taps(x0 + t, C.width, C.scale_x, antialias);
        float sum = 0.0f;
        for (int k = 0; k < w.end - w.first; k++) sum += w.weight(k);
        col_first[t] = (w.first - c0) * 3;
        col_taps[t] = w.end - w.first;
        col_centre[t] = w.centre;
        col_norm[t] = 1.0f / sum;
        const int patch = t / g.patch;
        col_stage[t] = patch * 3 * run + (t - patch * g.patch);
    }
    for (int t = threadIdx.x; t < down * across; t += kThreads) {
        const int a = t / across;
        patch_row[t] = row_of_patch(py0 + a, px0 + t - a * across, cols, g.merge);
    }
    const bool ok = status == nullptr || status[C.image] == PREP_OK;
    const float inv_x = (float)(1.0 / (antialias && C.scale_x > 1.0 ? C.scale_x : 1.0));
    const int distinct = min(g.group, C.frames - frames_group * g.group);  // the last frame stands in for the others
    out += (C.row0 + (int64_t)frames_group * rows * cols) * out_stride + (int64_t)part_y0 * g.patch;
    const int64_t area = (int64_t)g.patch * g.patch;

    for (int f = 0; f < distinct; f++) {
        const uint8_t *src = rgb + C.src_off + (uint64_t)(frames_group * g.group + f) * C.frame_stride + (uint64_t)r0 * C.pitch + (uint64_t)c0 * 3;
        if (ok) {
            const int total = (r_end - r0) * units;
            for (int u0 = 0; u0 < total; u0 += kLoads * kThreads) {
                uint4 v[kLoads];
#pragma unroll
                for (int k = 0; k < kLoads; k++) {
                    const int u = u0 + k * kThreads + (int)threadIdx.x;
                    if (u < total) {
                        const int r = u / units;
                        v[k] = load_inside(src + (uint64_t)r * C.pitch, (u - r * units) * 16, bytes);
                    }
                }
#pragma unroll
                for (int k = 0; k < kLoads; k++) {
                    const int u = u0 + k * kThreads + (int)threadIdx.x;
                    if (u < total) *reinterpret_cast<uint4 *>(raw + u * 16) = v[k];
                }
            }
        }
        __syncthreads();  // (the tables too)
        for (int t = wave; t < tile_h; t += kWaves) {
            if (ok) {
                const uint8_t *first = raw + row_first[t] * raw_pitch;
                const int taps = row_taps[t];
                for (int at = lane * 8; at < bytes; at += 64 * 8) {
                    float a[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
                    const uint8_t *p = first + at;
                    for (int k = 0; k < taps; k += 2) {
                        // (an odd window's last row is read twice, the second time with weight 0)
                        const uint2 v0 = *reinterpret_cast<const uint2 *>(p), v1 = *reinterpret_cast<const uint2 *>(k + 1 < taps ? p + raw_pitch : p);
                        const float w0 = row_weight[t][k], w1 = row_weight[t][k + 1];
                        p += 2 * raw_pitch;
#pragma unroll
                        for (int i = 0; i < 8; i++) {
                            const uint32_t b0 = i < 4 ? v0.x : v0.y, b1 = i < 4 ? v1.x : v1.y;
                            a[i] = fmaf(w0, (float)(b0 >> (8 * (i & 3)) & 255u), fmaf(w1, (float)(b1 >> (8 * (i & 3)) & 255u), a[i]));
                        }
                    }
                    float4 *s = reinterpret_cast<float4 *>(&summed[wave][at]);
                    s[0] = make_float4(a[0], a[1], a[2], a[3]);
                    s[1] = make_float4(a[4], a[5], a[6], a[7]);
                }
                wave_sync();
            }
            for (int x = lane; x < tile_w; x += 64) {
                float v[3] = {0.0f, 0.0f, 0.0f};
                if (ok) {
                    const float *s = &summed[wave][col_first[x]];
                    const float centre = col_centre[x], norm = col_norm[x];
                    const int taps = col_taps[x];
                    for (int k = 0; k < taps; k++) {
                        const float w = fmaxf(0.0f, fmaf(-fabsf((float)k - centre), inv_x, 1.0f));
#pragma unroll
                        for (int c = 0; c < 3; c++) v[c] = fmaf(w, s[3 * k + c], v[c]);
                    }
#pragma unroll
                    for (int c = 0; c < 3; c++) v[c] = fmaf(v[c] * norm, g.scale[c], g.bias[c]);
                }
                T *o = stage + row_stage[t] + col_stage[x];
#pragma unroll
                for (int c = 0; c < 3; c++) o[c * run] = from_float<T>(v[c]);
            }
            if (ok) wave_sync();
        }
        __syncthreads();
        for (int slot = f; slot < (f + 1 == distinct ? g.group : f + 1); slot++) {
            T *o = out + slot * area;
            const int64_t channel = g.group * area;
            if (chunk == 16) write_runs<T, 16>(stage, patch_row, down * across * 3, run, o, out_stride, channel);
            else if (chunk == 8) write_runs<T, 8>(stage, patch_row, down * across * 3, run, o, out_stride, channel);
            else if (chunk == 4) write_runs<T, 4>(stage, patch_row, down * across * 3, run, o, out_stride, channel);
            else write_runs<T, (int)sizeof(T)>(stage, patch_row, down * across * 3, run, o, out_stride, channel);
        }
        // (raw is not read any more, and the barrier before the next frame's sums ends the stage's reads)
    }
}

// Any sizes: one thread produces the three channels of one pixel, pixels in the order of the rows.  For images narrower than a
// tile's reads and reductions so strong that a tile's samples do not fit its LDS.
template <typename T>
__global__ __launch_bounds__(kThreads) void patch_rows_direct(const uint8_t *__restrict__ rgb, ClipPack pack, PatchGeometry g,
                                                              const int32_t *__restrict__ status, T *__restrict__ out, int64_t out_stride)
{
    const int clip = clip_of(pack, blockIdx.x);
    const PatchClip &C = pack.c[clip];
    const int area = g.patch * g.patch;
    const int cols = C.out_w / g.patch, rows = C.out_h / g.patch;
    const int64_t per_frame = (int64_t)C.out_w * C.out_h;
    const int64_t item = (int64_t)(blockIdx.x - pack.block0[clip]) * kThreads + threadIdx.x;
    const int groups = (C.frames - 1) / g.group + 1;
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
        const Taps ty = make_taps(y, C.height, C.scale_y, g.antialias), tx = make_taps(x, C.width, C.scale_x, g.antialias);
        const uint8_t *src = rgb + C.src_off + (uint64_t)f * C.frame_stride;
        float sum_x = 0.0f, sum_y = 0.0f;
        for (int k = 0; k < tx.end - tx.first; k++) sum_x += tx.weight(k);
        for (int j = 0; j < ty.end - ty.first; j++) {
            const float wy = ty.weight(j);
            const uint8_t *p = src + (uint64_t)(ty.first + j) * C.pitch + (uint64_t)tx.first * 3;
            float a[3] = {0.0f, 0.0f, 0.0f};
            for (int k = 0; k < tx.end - tx.first; k++, p += 3) {
                const float w = tx.weight(k);
#pragma unroll
                for (int c = 0; c < 3; c++) a[c] = fmaf(w, (float)p[c], a[c]);
            }
            sum_y += wy;
#pragma unroll
            for (int c = 0; c < 3; c++) v[c] = fmaf(wy, a[c], v[c]);
        }
        const float norm = 1.0f / (sum_x * sum_y);
#pragma unroll
        for (int c = 0; c < 3; c++) v[c] = fmaf(v[c] * norm, g.scale[c], g.bias[c]);
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

// How a clip is cut into tiles; false = it is not (see patch_rows_direct).
bool cut_into_tiles(PatchClip *c, const PatchGeometry &g, int element)
{
    if (c->width < kNarrowest) return false;
    const double sx = g.antialias && c->scale_x > 1.0 ? c->scale_x : 1.0, sy = g.antialias && c->scale_y > 1.0 ? c->scale_y : 1.0;
    if (2.0 * sy + 2.0 > (double)kTaps) return false;
    const int cols = c->out_w / g.patch, rows = c->out_h / g.patch;
    // the most source columns and rows under `n` output samples in a row
    auto span = [](int n, double scale, double s) { return (n - 1) * scale + 2.0 * s + 2.0; };
    auto fits = [&](int across, int tall) {
        const int w = across * g.patch;
        const double x = fmax(span(w, c->scale_x, sx), (double)kNarrowest), y = span(tall, c->scale_y, sy);
        return w <= kTileCols && tall <= kTileRows && w * tall <= stage_pixels(element) && x <= (double)kSpan && y * (3.0 * x + 16.0) <= (double)kRawBytes;
    };
    c->parts = 1;
    c->part_rows = g.patch;
    while (!fits(1, c->part_rows)) {
        if (c->part_rows <= 4) return false;
        c->parts++;
        c->part_rows = (g.patch + c->parts - 1) / c->parts;
    }
    c->parts = (g.patch + c->part_rows - 1) / c->part_rows;
    c->across = c->down = 1;
    while (c->across < cols && fits(c->across + 1, c->part_rows)) c->across++;
    if (c->parts == 1)
        while (c->down < rows && (c->down + 1) * c->across <= kPatches && fits(c->across, (c->down + 1) * g.patch)) c->down++;
    c->tiles_x = (cols + c->across - 1) / c->across;
    c->tiles_y = (rows + c->down - 1) / c->down * c->parts;
    return true;
}

uint64_t blocks_of(const PatchClip &c, const PatchGeometry &g, bool tiled)
{
    const uint64_t groups = (uint64_t)((c.frames - 1) / g.group + 1);
    if (tiled) return groups * (uint64_t)c.tiles_x * (uint64_t)c.tiles_y;
    return ((uint64_t)c.out_w * (uint64_t)c.out_h * groups * (uint64_t)g.group + kThreads - 1) / kThreads;
}

// Bytes that all runs can be written by at a time.
int chunk_bytes(const prep_patch_params *params, const ClipPack &pack, int n, const void *out, int64_t out_stride)
{
    const uint64_t element = (uint64_t)element_bytes(params->out_dtype), p = (uint64_t)params->patch;
    uint64_t all = (uint64_t)(uintptr_t)out | (uint64_t)out_stride * element | p * p * element;
    for (int i = 0; i < n; i++)
        if (pack.c[i].parts > 1) all |= (uint64_t)pack.c[i].part_rows * p * element;
    const uint64_t low = all & (~all + 1);
    return (int)(low < 16 ? low : 16);
}

template <typename T>
void launch_for(const uint8_t *rgb, const ClipPack &pack, uint32_t blocks, const PatchGeometry &g, bool tiled, int chunk, const int32_t *status,
                T *out, int64_t out_stride, hipStream_t stream)
{
    if (tiled)
        hipLaunchKernelGGL((patch_rows_tiled<T>), dim3(blocks), dim3(kThreads), 0, stream, rgb, pack, g, status, out, out_stride, chunk);
    else
        hipLaunchKernelGGL((patch_rows_direct<T>), dim3(blocks), dim3(kThreads), 0, stream, rgb, pack, g, status, out, out_stride);
}

// status: DEVICE, per PatchClip::image, or nullptr = all PREP_OK (others get rows of zeros).  clips: HOST, n of them, all but
// the tiles filled in.  Every clip is taken by a launch of one kind or the other.
int launch_patch_rows(const uint8_t *rgb, PatchClip *clips, int32_t n, const prep_patch_params *params, const int32_t *status, void *out,
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
    bool any[2] = {false, false};
    for (int32_t i = 0; i < n; i++) {
        if (!cut_into_tiles(&clips[i], g, element_bytes(params->out_dtype))) clips[i].tiles_x = 0;
        any[clips[i].tiles_x != 0] = true;
    }
    for (int kind = 0; kind < 2; kind++) {
        const bool tiled = kind == 1;
        if (!any[kind]) continue;
        for (int32_t at = 0; at < n;) {
            ClipPack pack;
            uint64_t blocks = 0;
            int m = 0;
            for (; at < n && m < kClips; at++) {
                if ((clips[at].tiles_x != 0) != tiled) continue;
                const uint64_t mine = blocks_of(clips[at], g, tiled);
                if (blocks + mine > 0x7FFFFFFFull) break;
                pack.c[m] = clips[at];
                pack.block0[m] = (uint32_t)blocks;
                blocks += mine;
                m++;
            }
            if (m == 0) continue;
            for (int k = m; k < kClips; k++) {
                pack.c[k] = pack.c[0];
                pack.block0[k] = 0xFFFFFFFFu;
            }
            const int chunk = tiled ? chunk_bytes(params, pack, m, out, out_stride) : 0;
            if (params->out_dtype == PREP_F16)
                launch_for(rgb, pack, (uint32_t)blocks, g, tiled, chunk, status, (__half *)out, out_stride, stream);
            else if (params->out_dtype == PREP_BF16)
                launch_for(rgb, pack, (uint32_t)blocks, g, tiled, chunk, status, (__hip_bfloat16 *)out, out_stride, stream);
            else
                launch_for(rgb, pack, (uint32_t)blocks, g, tiled, chunk, status, (float *)out, out_stride, stream);
        }
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
        c.scale_x = (double)width / (double)c.out_w;
        c.scale_y = (double)height / (double)c.out_h;
        c.frames = frames;
        c.image = i;
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
