// Patch rows: resize (two-tap bilinear or antialiased) + normalize + cut into patches, fused (gfx950).
//
// An output value is sum_j wy[j] sum_k wx[k] src[j][k]: per axis a window of source samples around the output sample's
// centre c = (i + 1/2) in / out - 1/2, weights max(0, 1 - |j - c| / s) scaled to sum 1 over the samples inside the image, s =
// max(in / out, 1) (antialiased) or 1, which is two taps; a tap that the border would clamp counts for the border's sample either way.
//
// A workgroup makes a tile of patches, up to 16 x 64 pixels.  The source samples under it go to LDS.  The sums over rows are a
// product (16 output rows) x (source rows) x (bytes of a row) on the matrix cores: a byte is a half exactly, a weight is two halves,
// 2^15 w = hi + lo with 22 bits, and sums are fp32; with vector instructions (a conversion and a multiply-add per tap and byte) that part alone
// took as long as the rest of the kernel.  The sums over columns are vector instructions, a lane an output column whose weights stay in registers.
// The values go to LDS in the order of the patch rows, from where they are written in runs.
//
// Measured, us a pass among passes over other data: 48 frames of 1920 x 1080 to 400 000 pixels, bf16, antialiased 191 (their bytes at 5.2 TB/s: 78; a thread a
// pixel, patch_rows_direct, 519); 64 frames of some 560 x 420, two taps, fp32 75 (30; 94); 32 photographs, fp16 27 (9.5; 59).  Neither unit is
// full: in the first the vector ALU is busy 45 % of the time, LDS 45 %, and waves wait 53 % of theirs.
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <cmath>
#include <stdint.h>

#include <new>

#include "../../include/prep.h"
#include "kernels.h"
#include "matrix.h"
#include "tokens.h"

namespace prep {

namespace {

constexpr int kThreads = 256;
constexpr int kClips = 64;  // clips of one launch: their records are kernel arguments (4 KB), so that a call has
                            // no workspace, calls may overlap and a captured call keeps its own

// Division by a number that the host knows: the quotient by a multiplication is right or one too large.
struct Divisor {
    uint32_t d, m;  // m = 2^32 / d, rounded up (d = 1: not looked at)
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const
    {
        const uint32_t q = __umulhi(n, m);
        return d == 1 ? n : q - (q * d > n ? 1u : 0u);
    }
};
// (2^32 - 1) / d + 1 = 2^32 / d rounded up, modulo 2^32
__host__ __device__ __forceinline__ Divisor divisor(int d) { return {(uint32_t)d, 0xFFFFFFFFu / (uint32_t)d + 1u}; }

// A tile's limits, for clips whose windows hold at most kFewTaps columns (kWide = false) and for the others.
constexpr int kTileCols = 64, kTileRows = 16, kPatches = 128;
constexpr int kStrip = 4;                          // tiles one below the other that a workgroup takes, at most (2: 201 us for 191, 85 for 75)
constexpr int kNarrowest = 6;                      // narrowest image whose rows hold a read of 16 bytes
constexpr int kFewTaps = 3, kMostTaps = 6;          // columns of a window whose weights stay in registers
constexpr int kSomeTaps = 5;                       // fewer than kMostTaps, where a window has no more
constexpr float kWeightScale = 32768.0f;
template <bool kWide, int kElement>
struct Limits {
    static constexpr int span_bytes = kWide ? 448 : 256, sum_pitch = span_bytes + 4;  // of a source row
    static constexpr int steps = kWide ? 2 : 1, source_rows = 32 * steps;  // products over 32 source rows each
    static constexpr int raw_bytes = kWide ? 16 << 10 : 8 << 10;           // source samples, rows 16-byte multiples apart
    static constexpr int threads = kWide ? 512 : 256, waves = threads / 64;
    static constexpr int loads = raw_bytes / (16 * threads);               // 16-byte reads of a thread
    static constexpr int workgroups = kWide ? 2 : kElement == 2 ? 4 : 3;   // that a compute unit's LDS holds
};

// One clip as the kernels see it.
struct PatchClip {
    uint64_t src_off;       // first byte of its first frame
    uint64_t frame_stride;  // bytes
    int64_t row0;           // its first row
    uint32_t pitch;
    int32_t frames;
    int32_t image;          // index into `status`
    uint32_t strips_m;      // Divisors' m: strips of a frame group, and of a row of them
    uint32_t strips_x_m;
    uint16_t width, height; // pixels
    uint16_t cols, rows;    // patches
    // tiles: patches across and down, rows of a patch in it (fewer than the patch has where that is tall: `parts` tiles
    // share a patch then)
    uint8_t across, down, part_rows, parts;
    __host__ __device__ int tiles_x() const { return (cols + across - 1) / across; }
    __host__ __device__ int tiles_y() const { return (rows + down - 1) / down * parts; }
    // source samples per output sample
    __host__ __device__ double scale_x(int patch) const { return (double)width / (double)(cols * patch); }
    __host__ __device__ double scale_y(int patch) const { return (double)height / (double)(rows * patch); }
};
struct ClipPack {
    uint32_t block0[kClips];  // first workgroup of each clip; of those that the launch lacks 2^32 - 1
    PatchClip c[kClips];
};
static_assert(sizeof(ClipPack) <= 3976, "kernel arguments are 4 KB at most");
struct PatchGeometry {
    int32_t patch, merge, group;  // pixels, patches, frames
    int32_t antialias;
    int32_t strip;                // tiles of a workgroup
    int32_t chunk;                // bytes written at a time
    uint32_t block0;              // first workgroup of the launch
    Divisor by_patch, by_merge, by_chunks;  // (chunks of a patch's channel)
    float scale[3], bias[3];      // 1 / (255 std), -mean / std
};

// The window of one output sample of one axis, cut at the image's edge.
struct Taps {
    int first, end;
    float centre;  // relative to `first`
    float inv;     // 1 / s
    __device__ __forceinline__ float weight(int k) const { return fmaxf(0.0f, fmaf(-fabsf((float)k - centre), inv, 1.0f)); }
};
__host__ __device__ __forceinline__ Taps make_taps(int i, int size, double scale, float inv, bool antialias)
{
    // in 64 bits: a coordinate near 2000 would leave a float 13 bits of fraction
    const double c = ((double)i + 0.5) * scale - 0.5, s = antialias && scale > 1.0 ? scale : 1.0;
    Taps t;
    t.first = max((int)floor(c - s) + 1, 0);  // (weight 0 at c - s itself)
    t.end = min((int)ceil(c + s), size);
    t.centre = (float)(c - (double)t.first);
    t.inv = inv;
    return t;
}

// (eight entries at a time without a branch: their scalar loads go out together)
__device__ __forceinline__ int clip_of(const ClipPack &pack, uint32_t block)
{
    static_assert(kClips == 64, "two steps of eight");
    int i = 0, k = 0;
#pragma unroll
    for (int e = 1; e < 8; e++) i += pack.block0[8 * e] <= block ? 8 : 0;
#pragma unroll
    for (int e = 1; e < 8; e++) k += pack.block0[i + e] <= block ? 1 : 0;
    return i + k;
}

// Row, inside its group of frames, of patch (py, px): row_of_line(py) + row_of_column(px).
__device__ __forceinline__ int row_of_line(const PatchGeometry &g, int py, int cols)
{
    const int band = (int)g.by_merge.quotient((uint32_t)py);
    return band * g.merge * cols + (py - band * g.merge) * g.merge;
}
__device__ __forceinline__ int row_of_column(const PatchGeometry &g, int px)
{
    const int window = (int)g.by_merge.quotient((uint32_t)px);
    return window * g.merge * g.merge + (px - window * g.merge);
}

// A value that all lanes of a wave hold alike.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// The most columns (or rows) that a window holds.
__host__ __device__ __forceinline__ int columns_of_window(double scale, bool antialias) { return antialias && scale > 1.0 ? (int)(2.0 * scale) + 1 : 2; }

// 16 bytes of a row that were read `back` bytes early, so as to end with the row: those behind the row's end become 0.
__device__ __forceinline__ uint4 moved_back(uint4 v, int back)
{
    uint64_t lo = v.x | (uint64_t)v.y << 32, hi = v.z | (uint64_t)v.w << 32;
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

// A frame's runs, `n` of them (three of a patch), from the stage to the patches' rows, kBytes at a time; of `chunks` each.  Offsets from
// `out` stay below 2^31 elements (see cut_into_tiles).
template <typename T, int kBytes, int kThreads>
__device__ __forceinline__ void write_runs(const T *stage, const int32_t *row, int n, const Divisor &chunks, T *out, int stride, int channel_stride)
{
    typedef typename Chunk<kBytes>::type C;
    constexpr int kElements = kBytes / (int)sizeof(T);
    for (uint32_t u = threadIdx.x; u < (uint32_t)n * chunks.d; u += kThreads) {
        const uint32_t r = chunks.quotient(u), patch = r / 3, channel = r - 3 * patch;
        const int at = row[patch] * stride + (int)(channel * (uint32_t)channel_stride + (u - r * chunks.d) * kElements);
        *reinterpret_cast<C *>(out + at) = *reinterpret_cast<const C *>(stage + u * kElements);
    }
}

// A lane's output column: its window in the row's sums, at most kTaps samples wide, and their weights; kTaps = 0: any width, weights formed for
// every row.
template <int kTaps>
struct Column {
    int at;      // first sample
    int taps;    // kTaps = 0
    float centre, inv, norm;
    float w[kTaps != 0 ? kTaps : 1];
    // `used` samples are summed, at most kTaps: a window starts earlier where they would end behind the row's sums; what is not under the
    // triangle has weight 0
    __device__ __forceinline__ Column(int first, int taps_, float centre_, float inv_, float norm_, int most, int used)
        : at(kTaps != 0 ? min(first, most - used) : first), taps(taps_), centre(centre_), inv(inv_), norm(norm_)
    {
#pragma unroll
        for (int k = 0; k < kTaps; k++) {
            const int tap = at + k - first;
            w[k] = tap >= 0 && tap < taps ? fmaxf(0.0f, fmaf(-fabsf((float)tap - centre), inv, 1.0f)) * norm : 0.0f;
        }
    }
    template <int kUsed>
    __device__ __forceinline__ void sum(const float *summed, float v[3]) const
    {
        const float *s = summed + at * 3;
        v[0] = v[1] = v[2] = 0.0f;
        if (kTaps != 0) {
#pragma unroll
            for (int k = 0; k < kUsed; k++)
#pragma unroll
                for (int c = 0; c < 3; c++) v[c] = fmaf(w[k], s[3 * k + c], v[c]);
        } else {
            for (int k = 0; k < taps; k++) {
                const float wk = fmaxf(0.0f, fmaf(-fabsf((float)k - centre), inv, 1.0f)) * norm;
#pragma unroll
                for (int c = 0; c < 3; c++) v[c] = fmaf(wk, s[3 * k + c], v[c]);
            }
        }
    }
};
template <typename T, int kUsed, int kTaps, int kSumPitch, int kWaves>
__device__ __forceinline__ void sum_columns(const Column<kTaps> &column, const float *summed, T *stage, const int32_t *row_stage, int tile_h, int x_stage,
                                            int run, const PatchGeometry &g)
{
    for (int t = uniform((int)threadIdx.x >> 6); t < tile_h; t += kWaves) {
        float v[3];
        column.template sum<kUsed>(summed + t * kSumPitch, v);
        T *o = stage + uniform(row_stage[t]) + x_stage;
#pragma unroll
        for (int c = 0; c < 3; c++) o[c * run] = from_float<T>(fmaf(v[c], g.scale[c], g.bias[c]));
    }
}

template <typename T, bool kWide>
__global__ __launch_bounds__((Limits<kWide, (int)sizeof(T)>::threads), (Limits<kWide, (int)sizeof(T)>::waves / 4 * Limits<kWide, (int)sizeof(T)>::workgroups)) void patch_rows_tiled(const uint8_t *__restrict__ rgb, ClipPack pack, PatchGeometry g,
                                                             const int32_t *__restrict__ status, T *__restrict__ out, int64_t out_stride)
{
    typedef Limits<kWide, (int)sizeof(T)> Most;
    constexpr int kSumPitch = Most::sum_pitch, kLoads = Most::loads, kThreads = Most::threads, kWaves = Most::waves;
    __shared__ alignas(16) uint8_t raw[Most::raw_bytes + 64];    // (a product's last columns may lie behind the last row)
    __shared__ alignas(16) float summed[kTileRows * kSumPitch];  // sums over rows, by output row and byte of a source row
    __shared__ alignas(16) T stage[kTileRows * kTileCols * 3];   // values by patch, channel, pixel
    __shared__ uint4 weight[Most::steps][2][64];                 // hi and lo as the product's lanes hold them
    __shared__ int32_t row_first[kStrip * kTileRows], row_taps[kStrip * kTileRows], row_stage[kStrip * kTileRows];
    __shared__ float row_centre[kStrip * kTileRows], row_norm[kStrip * kTileRows];
    __shared__ int32_t col_first[kTileCols], col_taps[kTileCols], line_row[kStrip * kTileRows], column_row[kTileCols];
    __shared__ float col_centre[kTileCols], col_norm[kTileCols];
    __shared__ int32_t patch_row[2][kPatches], tile_down[kStrip], tile_part_rows[kStrip], tile_part_y0[kStrip];

    const uint32_t block = g.block0 + blockIdx.x;
    const int clip = clip_of(pack, block);
    const PatchClip &C = pack.c[clip];
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const int tiles_x = C.tiles_x(), tiles_y = C.tiles_y();
    const Divisor strips = {(uint32_t)(tiles_x * ((tiles_y + g.strip - 1) / g.strip)), C.strips_m}, strips_x = {(uint32_t)tiles_x, C.strips_x_m};
    const uint32_t strip = block - pack.block0[clip], frames_group = strips.quotient(strip);
    const uint32_t in_group = strip - frames_group * strips.d, strip_y = strips_x.quotient(in_group);
    const int tile_x = (int)(in_group - strip_y * strips_x.d), tile_y0 = (int)strip_y * g.strip;
    const int tiles = min(g.strip, tiles_y - tile_y0);
    const int px0 = tile_x * C.across, across = min((int)C.across, C.cols - px0);  // patches
    const int tile_w = across * g.patch, x0 = px0 * g.patch;
    const bool antialias = g.antialias != 0;
    // 1 / s
    const float inv_x = antialias ? fminf((float)(C.cols * g.patch) / (float)C.width, 1.0f) : 1.0f;
    const float inv_y = antialias ? fminf((float)(C.rows * g.patch) / (float)C.height, 1.0f) : 1.0f;

    if (wave == 0) {
        if (lane < tile_w) {
            const Taps w = make_taps(x0 + lane, C.width, C.scale_x(g.patch), inv_x, antialias);
            float sum = 0.0f;
            for (int k = 0; k < w.end - w.first; k++) sum += w.weight(k);
            col_first[lane] = w.first;
            col_taps[lane] = w.end - w.first;
            col_centre[lane] = w.centre;
            col_norm[lane] = 1.0f / (sum * (kWeightScale * kBytePairScale));
        }
    } else if (wave == 1) {
        // row t of tile i
        const int i = lane / kTileRows, t = lane - i * kTileRows;
        int line = tile_y0 + i, part = 0;
        if (C.parts > 1) {
            line = (tile_y0 + i) / C.parts;
            part = tile_y0 + i - line * C.parts;
        }
        const int py0 = line * C.down, down = min((int)C.down, C.rows - py0), part_y0 = part * C.part_rows, part_rows = min((int)C.part_rows, g.patch - part_y0);
        if (i < tiles) {
            if (t < down) line_row[lane] = row_of_line(g, py0 + t, C.cols);
            if (t < down * part_rows) {
                const Taps w = make_taps(py0 * g.patch + part_y0 + t, C.height, C.scale_y(g.patch), inv_y, antialias);
                float sum = 0.0f;
                for (int k = 0; k < w.end - w.first; k++) sum += w.weight(k);
                row_first[lane] = w.first;
                row_taps[lane] = w.end - w.first;
                row_centre[lane] = w.centre;
                row_norm[lane] = kWeightScale / sum;
                const int a = down == 1 ? 0 : (int)g.by_patch.quotient((uint32_t)t);  // (several lines of patches are whole ones)
                row_stage[lane] = a * across * 3 * part_rows * g.patch + (t - a * part_rows) * g.patch;
            }
            if (t == 0) {
                tile_down[i] = down;
                tile_part_rows[i] = part_rows;
                tile_part_y0[i] = part_y0;
            }
        }
    } else if (wave == 2) {
        if (lane < across) column_row[lane] = row_of_column(g, px0 + lane);
    }
    __syncthreads();
    // the samples under the strip's columns, in sixteens (48 bytes, whole reads of 16) unless the image is narrower
    const int c_end = uniform(col_first[tile_w - 1] + col_taps[tile_w - 1]), sixteens = (c_end - uniform(col_first[0]) + 15) / 16;
    const int span = min(16 * sixteens, (int)C.width), c0 = min(uniform(col_first[0]), C.width - span);
    const int bytes = span * 3, units = (bytes + 15) / 16, raw_pitch = units * 16;
    const bool whole = span == 16 * sixteens;
    const bool ok = status == nullptr || status[C.image] == PREP_OK;
    const int distinct = min(g.group, C.frames - (int)frames_group * g.group);  // the last frame stands in for the others
    const uint8_t *src = rgb + C.src_off + (uint64_t)frames_group * (uint64_t)g.group * C.frame_stride + (uint64_t)c0 * 3;
    out += (C.row0 + (int64_t)frames_group * C.rows * C.cols) * out_stride;
    const int area = g.patch * g.patch;
    const int groups = (bytes + 63) / 64;
    // the thread's reads of a frame: row and column of each
    int read_row[kLoads], read_at[kLoads];
    uint4 read[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; k++) {
        const int u = k * kThreads + (int)threadIdx.x;
        read_row[k] = u / units;
        read_at[k] = (u - read_row[k] * units) * 16;
    }

    // the lane's output column
    // (48 full-HD frames, bf16, us.  Windows of up to 5 samples, with 5 and with 6 summed: reduced 1.6 times 277 and 285, 2.3 times 180 and 181.
    // Windows of 6, with weights kept and with weights formed for every row, as larger ones have them: 2.5 times 200 and 221, 2.7 times 180
    // and 197, 2.9 times 222 and 248.)
    constexpr int kColumnTaps = kWide ? kMostTaps : kFewTaps;
    const int x = min(lane, tile_w - 1), patch = (int)g.by_patch.quotient((uint32_t)x);
    const bool any_taps = kWide && antialias && 2 * (int)C.width >= kMostTaps * C.cols * g.patch;  // (columns_of_window > kMostTaps)
    const bool some_taps = kWide && !(antialias && 2 * (int)C.width >= kSomeTaps * C.cols * g.patch);
    const Column<kColumnTaps> column(col_first[x] - c0, col_taps[x], col_centre[x], inv_x, col_norm[x], groups * 64 / 3, some_taps ? kSomeTaps : kColumnTaps);

    // what is written at a time, of a patch's channel in a tile, and in the last tile of a patch that several share
    Divisor whole_part = g.by_chunks, last_part = g.by_chunks;
    if (C.parts > 1) {
        whole_part = divisor(C.part_rows * g.patch * (int)sizeof(T) / g.chunk);
        last_part = divisor((g.patch - (C.parts - 1) * C.part_rows) * g.patch * (int)sizeof(T) / g.chunk);
    }

    // Tile i, frame f is worked on while the frame after it is read; before the first, nothing is.
    int i = 0, f = -1, n_rows = 0, down = 0, part_rows = 0, part_y0 = 0;
    for (;;) {
        if (f >= 0) {
            if (ok) {
                // sums over rows: a wave takes 64 bytes of all rows, four products of 16 (bytes 4 n + j)
                for (int group = wave; group < groups; group += kWaves) {
                    const int at = group * 64 + 4 * (lane & 15);
                    float4 sum[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) sum[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 1
                    for (int step = 0; step < Most::steps && 32 * step < n_rows; step++) {
                        // (pairs of rows behind the last one are left out; a row behind it in a pair has weight 0)
                        uint32_t pair[4][4];
#pragma unroll
                        for (int p = 0; p < 4; p++) {
                            pair[0][p] = pair[1][p] = pair[2][p] = pair[3][p] = 0;
                            if (32 * step + 8 * p < n_rows) {
                                const int k = 32 * step + 8 * p + (lane >> 4);
                                const uint32_t r0 = *reinterpret_cast<const uint32_t *>(raw + min(k, n_rows - 1) * raw_pitch + at);
                                const uint32_t r1 = *reinterpret_cast<const uint32_t *>(raw + min(k + 4, n_rows - 1) * raw_pitch + at);
#pragma unroll
                                for (int j = 0; j < 4; j++) pair[j][p] = byte_pair(r0, r1, j);
                            }
                        }
                        const uint4 hi = weight[step][0][lane], lo = weight[step][1][lane];
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            const uint4 column = make_uint4(pair[j][0], pair[j][1], pair[j][2], pair[j][3]);
                            sum[j] = multiply_add_16x16x32(lo, column, multiply_add_16x16x32(hi, column, sum[j]));
                        }
                    }
                    float *s = summed + 4 * (lane >> 4) * kSumPitch + at;
                    *reinterpret_cast<float4 *>(s) = make_float4(sum[0].x, sum[1].x, sum[2].x, sum[3].x);
                    *reinterpret_cast<float4 *>(s + kSumPitch) = make_float4(sum[0].y, sum[1].y, sum[2].y, sum[3].y);
                    *reinterpret_cast<float4 *>(s + 2 * kSumPitch) = make_float4(sum[0].z, sum[1].z, sum[2].z, sum[3].z);
                    *reinterpret_cast<float4 *>(s + 3 * kSumPitch) = make_float4(sum[0].w, sum[1].w, sum[2].w, sum[3].w);
                }
            }
            __syncthreads();
        }
        // what comes next
        const int i_next = f + 1 == distinct ? i + 1 : i, f_next = f + 1 == distinct ? 0 : f + 1;
        const bool more = i_next < tiles;
        int n_next = n_rows, down_next = down, part_rows_next = part_rows, part_y0_next = part_y0;
        if (more) {
            const int row = i_next * kTileRows, r0 = uniform(row_first[row]);
            if (f_next == 0) {
                down_next = uniform(tile_down[i_next]);
                part_rows_next = uniform(tile_part_rows[i_next]);
                part_y0_next = uniform(tile_part_y0[i_next]);
                const int end = row + down_next * part_rows_next - 1;
                n_next = uniform(row_first[end] + row_taps[end]) - r0;
            }
            if (ok) {
                // (all reads go out before the first is waited for)
                const uint8_t *frame = src + (uint64_t)f_next * C.frame_stride + (uint64_t)(uint32_t)r0 * C.pitch;
#pragma unroll
                for (int k = 0; k < kLoads; k++)
                    if (k * kThreads < n_next * units)
                        __builtin_memcpy(&read[k], frame + ((uint32_t)min(read_row[k], n_next - 1) * C.pitch + (uint32_t)min(read_at[k], bytes - 16)), 16);
            }
            if (f_next == 0) {
                // Weights for 32 source rows a wave, the last ones (which have fewer rows to finish where these do not divide
                // evenly): lane l of a product holds rows 4 j + l / 16, j = 0 .. 7.
                const int m = lane & 15, step = kWaves - 1 - wave;
                if (32 * step < n_next) {
                    uint32_t hi[4] = {0, 0, 0, 0}, lo[4] = {0, 0, 0, 0};
                    if (m < down_next * part_rows_next) {
                        const int begin = row_first[row + m] - r0 - 32 * step - (lane >> 4), n = row_taps[row + m];
                        const float centre = row_centre[row + m], scale = row_norm[row + m];
#pragma unroll
                        for (int j = 0; j < 8; j++) {
                            const int tap = 4 * j - begin;
                            const float w = tap >= 0 && tap < n ? fmaxf(0.0f, fmaf(-fabsf((float)tap - centre), inv_y, 1.0f)) * scale : 0.0f;
                            const __half h = __float2half_rn(w);
                            const __half r = __float2half_rn(w - __half2float(h));
                            uint16_t hb, rb;
                            __builtin_memcpy(&hb, &h, 2);
                            __builtin_memcpy(&rb, &r, 2);
                            hi[j >> 1] |= (uint32_t)hb << (16 * (j & 1));
                            lo[j >> 1] |= (uint32_t)rb << (16 * (j & 1));
                        }
                    }
                    weight[step][0][lane] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    weight[step][1][lane] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
                for (int p = threadIdx.x; p < down_next * across; p += kThreads) {
                    const int a = down_next == 1 ? 0 : p / across;
                    patch_row[i_next & 1][p] = line_row[row + a] + column_row[p - a * across];
                }
            }
        }
        if (f >= 0) {
            const int run = part_rows * g.patch, tile_h = down * part_rows;  // of a patch's channel
            if (ok) {
                if (lane < tile_w) {
                    const int x_stage = patch * 3 * run + (x - patch * g.patch);
                    const int32_t *rows = row_stage + i * kTileRows;
                    if (some_taps) {
                        sum_columns<T, kSomeTaps < kColumnTaps ? kSomeTaps : kColumnTaps, kColumnTaps, kSumPitch, kWaves>(column, summed, stage, rows, tile_h, x_stage, run, g);
                    } else if (!any_taps) {
                        sum_columns<T, kColumnTaps, kColumnTaps, kSumPitch, kWaves>(column, summed, stage, rows, tile_h, x_stage, run, g);
                    } else {
                        const Column<0> wide(col_first[x] - c0, col_taps[x], col_centre[x], inv_x, col_norm[x], 0, 0);
                        sum_columns<T, 0, 0, kSumPitch, kWaves>(wide, summed, stage, rows, tile_h, x_stage, run, g);
                    }
                }
            } else {
                for (int e = threadIdx.x; e < tile_w * tile_h * 3; e += kThreads) stage[e] = from_float<T>(0.0f);
            }
        }
        if (more && ok) {
            // (the sums over rows are done with the samples before these)
#pragma unroll
            for (int k = 0; k < kLoads; k++) {
                const int u = k * kThreads + (int)threadIdx.x;
                if (!whole) read[k] = moved_back(read[k], max(read_at[k] - (bytes - 16), 0));
                if (u < n_next * units) *reinterpret_cast<uint4 *>(raw + u * 16) = read[k];
            }
        }
        __syncthreads();
        if (f >= 0) {
            // nothing waits for these: the next sums over columns follow a barrier, by which the values here are read
            for (int slot = f; slot < (f + 1 == distinct ? g.group : f + 1); slot++) {
                T *o = out + slot * area + part_y0 * g.patch;
                const int channel = g.group * area, runs = down * across * 3, stride = (int)out_stride;
                const int32_t *rows = patch_row[i & 1];
                const Divisor &chunks = part_rows == C.part_rows ? whole_part : last_part;
                if (g.chunk == 16) write_runs<T, 16, kThreads>(stage, rows, runs, chunks, o, stride, channel);
                else if (g.chunk == 8) write_runs<T, 8, kThreads>(stage, rows, runs, chunks, o, stride, channel);
                else if (g.chunk == 4) write_runs<T, 4, kThreads>(stage, rows, runs, chunks, o, stride, channel);
                else write_runs<T, (int)sizeof(T), kThreads>(stage, rows, runs, chunks, o, stride, channel);
            }
        }
        if (!more) break;
        i = i_next;
        f = f_next;
        n_rows = n_next;
        down = down_next;
        part_rows = part_rows_next;
        part_y0 = part_y0_next;
    }
}

// Any sizes: one thread produces the three channels of one pixel, pixels in the order of the rows.  For images narrower than a
// tile's reads, reductions so strong that a tile's samples do not fit its LDS, and what a tile's 32-bit offsets do not reach.
template <typename T>
__global__ __launch_bounds__(kThreads) void patch_rows_direct(const uint8_t *__restrict__ rgb, ClipPack pack, PatchGeometry g,
                                                              const int32_t *__restrict__ status, T *__restrict__ out, int64_t out_stride)
{
    const uint32_t block = g.block0 + blockIdx.x;
    const int clip = clip_of(pack, block);
    const PatchClip &C = pack.c[clip];
    // (a frame's pixels and rows are below 2^32, sides being at most 65535, but not below 2^31)
    const uint32_t area = (uint32_t)(g.patch * g.patch), cols = C.cols, rows = C.rows, merge = (uint32_t)g.merge;
    const int64_t per_frame = (int64_t)(cols * rows * area);
    const int64_t item = (int64_t)(block - pack.block0[clip]) * kThreads + threadIdx.x;
    const int64_t groups = (C.frames - 1) / g.group + 1;
    if (item >= per_frame * g.group * groups) return;
    const int64_t slot = item / per_frame;
    const uint32_t e = (uint32_t)(item - slot * per_frame);
    const int64_t f = min(slot, (int64_t)C.frames - 1);
    const uint32_t row = e / area, in_patch = e - row * area;  // row of the group
    const uint32_t band = row / (merge * cols), r1 = row - band * merge * cols;
    const uint32_t window = r1 / (merge * merge), r2 = r1 - window * merge * merge;
    const uint32_t py = band * merge + r2 / merge, px = window * merge + r2 % merge;
    const int y = (int)(py * (uint32_t)g.patch + in_patch / (uint32_t)g.patch), x = (int)(px * (uint32_t)g.patch + in_patch % (uint32_t)g.patch);
    float v[3] = {0.0f, 0.0f, 0.0f};
    if (status == nullptr || status[C.image] == PREP_OK) {
        const float inv_y = g.antialias ? fminf((float)(C.rows * g.patch) / (float)C.height, 1.0f) : 1.0f;
        const float inv_x = g.antialias ? fminf((float)(C.cols * g.patch) / (float)C.width, 1.0f) : 1.0f;
        const Taps ty = make_taps(y, C.height, C.scale_y(g.patch), inv_y, g.antialias), tx = make_taps(x, C.width, C.scale_x(g.patch), inv_x, g.antialias);
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
    T *o = out + (C.row0 + slot / g.group * (int64_t)(rows * cols) + row) * out_stride + slot % g.group * (int64_t)area + in_patch;
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

// How a clip is cut into tiles, one way or the other; false = it is not.
template <typename Most>
bool cut_into_tiles(PatchClip *c, const PatchGeometry &g, int64_t out_stride)
{
    // (offsets inside a frame group are 32-bit, and so are those inside the samples under a tile)
    if (c->width < kNarrowest || (int64_t)c->cols * c->rows * out_stride > INT32_MAX || (uint64_t)c->pitch * Most::source_rows > UINT32_MAX) return false;
    const double scale_x = c->scale_x(g.patch), scale_y = c->scale_y(g.patch);
    const double sx = g.antialias && scale_x > 1.0 ? scale_x : 1.0, sy = g.antialias && scale_y > 1.0 ? scale_y : 1.0;
    // Under n output samples in a row lie fewer than (n - 1) scale + 2 s + 1 source samples; columns come in sixteens.
    const auto rows_under = [&](int n) { return (n - 1) * scale_y + 2.0 * sy + 1.0; };
    // the most output samples over at most `most` source samples
    const auto over = [](double most, double scale, double s) {
        const double n = floor((most - 2.0 * s - 1.0) / scale) + 1.0;
        return n < 0.0 ? 0 : n > 65535.0 ? 65535 : (int)n;
    };
    const auto columns_over = [&](int tall) {  // pixels across where the tile is `tall` pixels high; 0 = too many rows lie under it
        const double y = rows_under(tall);
        if (tall > kTileRows || y > (double)Most::source_rows) return 0;
        const double most = fmin(Most::span_bytes / 48 * 16.0, 16.0 * floor(Most::raw_bytes / (48.0 * y)));
        const int w = over(most, scale_x, sx);
        return w < kTileCols ? w : kTileCols;
    };
    c->parts = 1;
    c->part_rows = (uint8_t)g.patch;
    int across;
    while ((across = columns_over(c->part_rows) / g.patch) < 1) {
        if (c->part_rows <= 4) return false;
        c->parts++;
        c->part_rows = (uint8_t)((g.patch + c->parts - 1) / c->parts);
    }
    c->parts = (uint8_t)((g.patch + c->part_rows - 1) / c->part_rows);
    c->across = (uint8_t)(across < c->cols ? across : c->cols);
    if (c->across > kPatches) c->across = kPatches;
    c->down = 1;
    if (c->parts == 1) {
        const double x = 16.0 * ceil(((c->across * g.patch - 1) * scale_x + 2.0 * sx + 1.0) / 16.0);
        const int tall = over(fmin((double)Most::source_rows, Most::raw_bytes / (3.0 * x)), scale_y, sy);
        int down = (tall < kTileRows ? tall : kTileRows) / g.patch;
        if (down > kPatches / c->across) down = kPatches / c->across;
        if (down > c->rows) down = c->rows;
        if (down > 1) c->down = (uint8_t)down;
    }
    return true;
}

// The kernels: patch_rows_direct, patch_rows_tiled with kWide = false and true.
enum { kDirect = 0, kNarrow = 1, kWide = 2, kKinds = 3 };

// Cuts the clips of a call into tiles.  The narrow kind is for clips whose tiles are as large there as the wide kind's: it keeps four
// workgroups on a compute unit where the wide one keeps two.  Clips of both kinds take a launch each if the narrow ones have 2^22 pixels or
// more, some four rounds of the chip; with fewer the wait for one launch's last workgroups costs more, and one launch of the wide kind takes all.  us in one
// launch and in two, antialiased, fp16: photographs of 400 x 365 with one picture of 4000 x 3000 reduced to 2^20 pixels, 4 of them 54 and 59, 16 of them 61 and
// 62, 32 of them 76 and 72, 128 of them 180 and 132; frames of 380 x 285 up to 520 x 390 reduced to 147 456 pixels where they have more, 96 of them
// 106 and 90, 256 of them 263 and 193; two taps, fp32, of 300 x 225 up to 900 x 675, 64 of them 77 and 84, 96 of them 125 and 114.
// Threads of a workgroup, 256 and 512, us: narrow 29 and 36 (32 photographs), wide 260 and 191 (48 full-HD frames).
constexpr uint64_t kOwnLaunchPixels = 1 << 22;
template <int kElement>
void cut_clips(PatchClip *clips, uint8_t *kinds, int32_t n, const PatchGeometry &g, int64_t out_stride)
{
    const auto few_taps = [&](const PatchClip &c) { return columns_of_window(c.scale_x(g.patch), g.antialias) <= kFewTaps; };
    const auto pixels = [&](const PatchClip &c) { return (uint64_t)c.frames * c.cols * c.rows * (uint64_t)(g.patch * g.patch); };
    uint64_t few = 0, narrow = 0;
    for (int32_t i = 0; i < n; i++)
        if (few_taps(clips[i])) few += pixels(clips[i]);
    const bool may_part = few >= kOwnLaunchPixels;
    bool all = true;  // those looked at so far are of the narrow kind
    for (int32_t i = 0; i < n; i++) {
        PatchClip &c = clips[i], other = c;
        kinds[i] = cut_into_tiles<Limits<true, kElement>>(&c, g, out_stride) ? kWide : kDirect;
        if (kinds[i] == kDirect || (!may_part && !all)) continue;
        if (few_taps(c) && cut_into_tiles<Limits<false, kElement>>(&other, g, out_stride) &&
            other.across * other.down * other.part_rows >= c.across * c.down * c.part_rows) {
            c = other;
            kinds[i] = kNarrow;
            narrow += pixels(c);
        } else {
            all = false;
        }
    }
    if (all || narrow >= kOwnLaunchPixels) return;
    for (int32_t i = 0; i < n; i++)
        if (kinds[i] == kNarrow && cut_into_tiles<Limits<true, kElement>>(&clips[i], g, out_stride)) kinds[i] = kWide;
}

uint64_t groups_of(const PatchClip &c, const PatchGeometry &g) { return (uint64_t)((c.frames - 1) / g.group + 1); }
int strips_of(const PatchClip &c, const PatchGeometry &g) { return c.tiles_x() * ((c.tiles_y() + g.strip - 1) / g.strip); }
uint64_t blocks_of(const PatchClip &c, const PatchGeometry &g, int kind)
{
    if (kind != kDirect) return groups_of(c, g) * (uint64_t)strips_of(c, g);
    return ((uint64_t)c.cols * (uint64_t)c.rows * (uint64_t)(g.patch * g.patch) * groups_of(c, g) * (uint64_t)g.group + kThreads - 1) / kThreads;
}

// Bytes that all runs can be written by at a time.
int chunk_bytes(const prep_patch_params *params, const PatchClip *clips, int32_t n, const void *out, int64_t out_stride)
{
    const uint64_t element = (uint64_t)element_bytes(params->out_dtype), p = (uint64_t)params->patch;
    uint64_t all = (uint64_t)(uintptr_t)out | (uint64_t)out_stride * element | p * p * element;
    for (int32_t i = 0; i < n; i++)
        if (clips[i].parts > 1) all |= (uint64_t)clips[i].part_rows * p * element;
    const uint64_t low = all & (~all + 1);
    return (int)(low < 16 ? low : 16);
}

template <typename T>
void launch_for(const uint8_t *rgb, const ClipPack &pack, uint32_t blocks, PatchGeometry g, int kind, const int32_t *status,
                T *out, int64_t out_stride, hipStream_t stream)
{
    const int threads = kind == kWide ? Limits<true, (int)sizeof(T)>::threads : kind == kNarrow ? Limits<false, (int)sizeof(T)>::threads : kThreads;
    in_launches(blocks, threads, [&](uint32_t first, uint32_t n) {
        const dim3 grid(n), block(threads);
        g.block0 = first;
        if (kind == kWide) hipLaunchKernelGGL((patch_rows_tiled<T, true>), grid, block, 0, stream, rgb, pack, g, status, out, out_stride);
        else if (kind == kNarrow) hipLaunchKernelGGL((patch_rows_tiled<T, false>), grid, block, 0, stream, rgb, pack, g, status, out, out_stride);
        else hipLaunchKernelGGL((patch_rows_direct<T>), grid, block, 0, stream, rgb, pack, g, status, out, out_stride);
    });
}

// status: DEVICE, per PatchClip::image, or nullptr = all PREP_OK (others get rows of zeros).  clips, kinds: HOST, n of them; the tiles
// and kinds are found here.  Every clip is taken by a launch of its kind.
int launch_patch_rows(const uint8_t *rgb, PatchClip *clips, uint8_t *kinds, int32_t n, const prep_patch_params *params, const int32_t *status,
                      void *out, int64_t out_stride, hipStream_t stream)
{
    PatchGeometry g;
    g.block0 = 0;
    g.patch = params->patch;
    g.merge = params->merge;
    g.group = params->frames_per_patch;
    g.antialias = params->filter == PREP_FILTER_ANTIALIAS;
    g.by_patch = divisor(g.patch);
    g.by_merge = divisor(g.merge);
    for (int c = 0; c < 3; c++) {
        g.scale[c] = (float)(1.0 / (255.0 * (double)params->std[c]));
        g.bias[c] = (float)(-(double)params->mean[c] / (double)params->std[c]);
    }
    if (element_bytes(params->out_dtype) == 2) cut_clips<2>(clips, kinds, n, g, out_stride);
    else cut_clips<4>(clips, kinds, n, g, out_stride);
    g.chunk = chunk_bytes(params, clips, n, out, out_stride);
    g.by_chunks = divisor(g.patch * g.patch * element_bytes(params->out_dtype) / g.chunk);
    bool any[kKinds] = {false, false, false};
    uint64_t tiles = 0;
    for (int32_t i = 0; i < n; i++) {
        PatchClip &c = clips[i];
        if (kinds[i] != kDirect) tiles += groups_of(c, g) * (uint64_t)c.tiles_x() * (uint64_t)c.tiles_y();
    }
    // a workgroup takes a strip of tiles where there are plenty, so that it can read one while it works on another
    g.strip = (int)(tiles / 1536 < 1 ? 1 : tiles / 1536 > kStrip ? kStrip : tiles / 1536);
    for (int32_t i = 0; i < n; i++) {
        PatchClip &c = clips[i];
        if (kinds[i] != kDirect && blocks_of(c, g, kinds[i]) > 0x7FFFFFFFull) kinds[i] = kDirect;  // (which add() has bounded)
        any[kinds[i]] = true;
        if (kinds[i] == kDirect) continue;
        c.strips_x_m = divisor(c.tiles_x()).m;
        c.strips_m = divisor(strips_of(c, g)).m;
    }
    for (int kind = 0; kind < kKinds; kind++) {
        if (!any[kind]) continue;
        for (int32_t at = 0; at < n;) {
            ClipPack pack;
            uint64_t blocks = 0;
            int m = 0;
            for (; at < n && m < kClips; at++) {
                if (kinds[at] != kind) continue;
                const uint64_t mine = blocks_of(clips[at], g, kind);
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
            if (params->out_dtype == PREP_F16)
                launch_for(rgb, pack, (uint32_t)blocks, g, kind, status, (__half *)out, out_stride, stream);
            else if (params->out_dtype == PREP_BF16)
                launch_for(rgb, pack, (uint32_t)blocks, g, kind, status, (__hip_bfloat16 *)out, out_stride, stream);
            else
                launch_for(rgb, pack, (uint32_t)blocks, g, kind, status, (float *)out, out_stride, stream);
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
    ~PatchCall()
    {
        delete[] clips_;
        delete[] kinds_;
    }
    PatchCall(const PatchCall &) = delete;
    PatchCall &operator=(const PatchCall &) = delete;

    int check()
    {
        if (n_ < 0 || !patch_params_ok(params_) || !row_starts_ || out_rows_ < 0 || (n_ > 0 && !out_)) return PREP_E_INVALID_ARG;
        const int64_t row = 3ll * params_->frames_per_patch * params_->patch * params_->patch;
        if (out_stride_ == 0) out_stride_ = row;
        if (out_stride_ < row || !aligned(out_, (uintptr_t)element_bytes(params_->out_dtype))) return PREP_E_INVALID_ARG;
        row_starts_[0] = 0;
        if (n_ > 0 && (!(clips_ = new (std::nothrow) PatchClip[(size_t)n_]) || !(kinds_ = new (std::nothrow) uint8_t[(size_t)n_]))) return PREP_E_NOMEM;
        return PREP_OK;
    }
    // Clips come in ascending order; those left out have no rows.
    bool add(int32_t i, int32_t width, int32_t height, uint64_t src_off, uint32_t pitch, int32_t frames, uint64_t frame_stride)
    {
        int32_t rows, cols;
        skip_to(i);
        if (frames < 1 || !patch_size(params_, width, height, &rows, &cols)) return false;
        const int64_t groups = ((int64_t)frames - 1) / params_->frames_per_patch + 1;
        // fewer than 2^31 workgroups
        if (groups * params_->frames_per_patch * rows * cols * params_->patch * params_->patch > (int64_t)0x7FFFFFFF * kThreads) return false;
        PatchClip &c = clips_[count_++];
        c.src_off = src_off;
        c.frame_stride = frame_stride;
        c.row0 = row_starts_[i];
        c.pitch = pitch;
        c.width = (uint16_t)width;
        c.height = (uint16_t)height;
        c.cols = (uint16_t)cols;
        c.rows = (uint16_t)rows;
        c.across = c.down = c.part_rows = c.parts = 1;  // (direct)
        c.frames = frames;
        c.image = i;
        if (__builtin_add_overflow(row_starts_[i], groups * rows * cols, &row_starts_[i + 1])) row_starts_[i + 1] = INT64_MAX;
        next_ = i + 1;
        return true;
    }
    int finish()
    {
        skip_to(n_);
        return row_starts_[n_] > out_rows_ || row_starts_[n_] == INT64_MAX ? PREP_E_TOO_LARGE : PREP_OK;
    }
    int launch(const uint8_t *rgb, const int32_t *status, hipStream_t stream)
    {
        return launch_patch_rows(rgb, clips_, kinds_, count_, params_, status, out_, out_stride_, stream);
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
    uint8_t *kinds_ = nullptr;
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
