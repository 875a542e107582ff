// Places and cache slots of the tokens of a packed batch (gfx950): whole-number work on lists of
// lengths that lie on the GPU.  Both operators are a prefix sum over the list (segments of
// sequences, or requests) and then a search in it for every token.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "../../include/prep.h"
#include "tokens.h"

namespace prep {

namespace {

constexpr int kThreads = 256;
constexpr int kScanThreads = 1024, kWaves = kScanThreads / 64;
constexpr int32_t kMaxEntries = 1 << 20;

// Inclusive sums of v over the lanes up to one's own, in a workgroup of kScanThreads; *total = over all.
template <typename T>
__device__ T scan_block(T v, T *total)
{
    __shared__ T wave_sum[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = 1; d < 64; d *= 2) {
        const T u = __shfl_up(v, (unsigned)d);
        if (lane >= d) v += u;
    }
    if (lane == 63) wave_sum[wave] = v;
    __syncthreads();
    T before = 0, all = 0;
    for (int w = 0; w < kWaves; w++) {
        if (w < wave) before += wave_sum[w];
        all += wave_sum[w];
    }
    __syncthreads();
    *total = all;
    return v + before;
}

__device__ __forceinline__ int32_t clip31(uint64_t v) { return v > 0x7FFFFFFFull ? 0x7FFFFFFF : (int32_t)v; }

// Index of the last of n + 1 ascending entries (the first is taken to be <= v) that is <= v, at most n - 1.
__device__ __forceinline__ int last_not_above(const int32_t *list, int n, int64_t v)
{
    int lo = 0, hi = n;  // list[lo] <= v, and hi = n or list[hi] > v
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (list[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

// ---- places --------------------------------------------------------------------------------------

struct SegmentList {
    const prep_segment *segments;
    const int32_t *seq_segments;
    const int32_t *first;
    int32_t n_segments, n_seq;
};
__device__ __forceinline__ int32_t seq_bound(const SegmentList &L, int i) { return min(max(L.seq_segments[i], 0), L.n_segments); }

__device__ __forceinline__ void segment_size(const prep_segment &s, uint64_t *tokens, uint32_t *advance)
{
    constexpr int32_t kMost = 32767;
    *tokens = 0;
    *advance = 0;
    if (s.h == 0 && s.w == 0) {
        if (s.t > 0 && s.step == 0) *tokens = *advance = (uint32_t)s.t;
        return;
    }
    if (s.t < 1 || s.h < 1 || s.w < 1 || s.step < 0 || s.t > kMost || s.h > kMost || s.w > kMost || s.step > kMost) return;
    *tokens = (uint64_t)s.t * (uint64_t)s.h * (uint64_t)s.w;
    *advance = (uint32_t)(max(max((s.t - 1) * s.step, s.h - 1), s.w - 1) + 1);
}

// starts[j]: first token of segment j (at most 2^31 - 1); moved[j]: how far places have moved on before it, over all
// segments (modulo 2^32).  n_segments + 1 entries each.
__global__ __launch_bounds__(kScanThreads) void sum_segments(SegmentList L, int32_t *__restrict__ starts, uint32_t *__restrict__ moved)
{
    const int32_t lo = seq_bound(L, 0), hi = seq_bound(L, L.n_seq);
    uint64_t tokens_before = 0;
    uint32_t moved_before = 0;
    for (int32_t at = 0; at < L.n_segments; at += kScanThreads) {
        const int32_t j = at + (int32_t)threadIdx.x;
        uint64_t tokens = 0, tokens_all;
        uint32_t advance = 0, moved_all;
        if (j >= lo && j < hi) segment_size(L.segments[j], &tokens, &advance);
        const uint64_t tokens_to = scan_block<uint64_t>(tokens, &tokens_all);
        const uint32_t moved_to = scan_block<uint32_t>(advance, &moved_all);
        if (j < L.n_segments) {
            starts[j] = clip31(tokens_before + tokens_to - tokens);
            moved[j] = moved_before + moved_to - advance;
        }
        tokens_before += tokens_all;
        moved_before += moved_all;
    }
    if (threadIdx.x == 0) {
        starts[L.n_segments] = clip31(tokens_before);
        moved[L.n_segments] = moved_before;
    }
}

__global__ __launch_bounds__(kThreads) void place_tokens(SegmentList L, int32_t merge, const int32_t *__restrict__ starts,
                                                         const uint32_t *__restrict__ moved, int32_t *__restrict__ positions,
                                                         int64_t capacity, int32_t *__restrict__ token_starts, int32_t *__restrict__ next)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i <= L.n_seq) {
        const int32_t b = seq_bound(L, (int)i);
        token_starts[i] = starts[b];
        if (next != nullptr && i < L.n_seq)
            next[i] = (int32_t)((L.first ? (uint32_t)L.first[i] : 0u) + moved[seq_bound(L, (int)i + 1)] - moved[b]);
    }
    if (i >= capacity) return;
    uint32_t pt = 0, ph = 0, pw = 0;
    if (i < starts[L.n_segments]) {
        const int j = last_not_above(starts, L.n_segments, i);
        const int q = last_not_above(L.seq_segments, L.n_seq, j);
        const prep_segment s = L.segments[j];
        const uint32_t base = (L.first ? (uint32_t)L.first[q] : 0u) + moved[j] - moved[seq_bound(L, q)];
        const uint32_t r = (uint32_t)i - (uint32_t)starts[j];
        if (s.h == 0) {
            pt = ph = pw = base + r;
        } else {
            const uint32_t h = (uint32_t)s.h, w = (uint32_t)s.w, m = (uint32_t)merge;
            const uint32_t a = r / (h * w), r1 = r - a * (h * w);
            // bands of m rows, windows of m columns in a band, both shorter at the edge
            const uint32_t band = r1 / (m * w), r2 = r1 - band * (m * w);
            const uint32_t tall = min(m, h - band * m);
            const uint32_t window = r2 / (tall * m), r3 = r2 - window * (tall * m);
            const uint32_t wide = min(m, w - window * m);
            const uint32_t y = r3 / wide;
            pt = base + a * (uint32_t)s.step;
            ph = base + band * m + y;
            pw = base + window * m + (r3 - y * wide);
        }
    }
    positions[i] = (int32_t)pt;
    positions[capacity + i] = (int32_t)ph;
    positions[2 * capacity + i] = (int32_t)pw;
}

// ---- slots ---------------------------------------------------------------------------------------

// Blocks that hold v tokens (v < 2^31)
__device__ __forceinline__ uint32_t blocks_of(uint32_t v, uint32_t block_size)
{
    const uint32_t whole = v / block_size;
    return whole + (whole * block_size != v ? 1u : 0u);
}

// starts[i]: first token of request i, n + 1 entries; taken[i]: blocks off the stack before its own, or -1: it is refused.
__global__ __launch_bounds__(kScanThreads) void sum_requests(prep_block_args A, int32_t *__restrict__ starts, int32_t *__restrict__ taken)
{
    __shared__ uint32_t used;  // blocks that go
    if (threadIdx.x == 0) used = 0;
    const int32_t on_stack = min(max(*A.free_count, 0), A.free_capacity);
    uint64_t tokens_before = 0, needed_before = 0;
    for (int32_t at = 0; at < A.n; at += kScanThreads) {
        const int32_t i = at + (int32_t)threadIdx.x;
        int32_t cached = 0, fresh = 0;
        bool sound = i < A.n;
        if (sound) {
            cached = A.cached[i];
            fresh = A.fresh[i];
            sound = cached >= 0 && fresh >= 0;
            if (!sound) cached = fresh = 0;
        }
        uint64_t tokens_all, needed_all;
        const uint64_t tokens_to = tokens_before + scan_block<uint64_t>((uint64_t)fresh, &tokens_all);
        const uint32_t after = (uint32_t)cached + (uint32_t)fresh;
        const uint32_t had = blocks_of((uint32_t)cached, (uint32_t)A.block_size), want = blocks_of(after, (uint32_t)A.block_size);
        const bool fits = sound && after <= (uint32_t)INT32_MAX && want <= (uint32_t)A.table_width && tokens_to <= (uint64_t)A.capacity;
        const uint32_t need = fits ? want - had : 0;
        const uint64_t needed_to = needed_before + scan_block<uint64_t>(need, &needed_all);
        const bool granted = fits && (need == 0 || needed_to <= (uint64_t)on_stack);
        if (granted && need != 0) atomicMax(&used, (uint32_t)needed_to);  // (sums only grow)
        if (i < A.n) {
            starts[i] = A.token_starts[i] = clip31(tokens_to - (uint64_t)fresh);
            taken[i] = !granted ? -1 : need == 0 ? 0 : (int32_t)(needed_to - need);
            A.lengths[i] = granted ? (int32_t)after : cached;
            A.status[i] = granted ? PREP_OK : sound ? PREP_E_TOO_LARGE : PREP_E_INVALID_ARG;
        }
        tokens_before += tokens_all;
        needed_before += needed_all;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        starts[A.n] = A.token_starts[A.n] = clip31(tokens_before);
        *A.free_left = on_stack - (int32_t)used;
    }
}

__global__ __launch_bounds__(kThreads) void place_slots(prep_block_args A, const int32_t *__restrict__ starts, const int32_t *__restrict__ taken)
{
    const int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (t >= A.capacity) return;
    int64_t slot = -1;
    if (t < starts[A.n]) {
        const int i = last_not_above(starts, A.n, t);
        if (taken[i] >= 0) {
            const uint32_t cached = (uint32_t)A.cached[i], size = (uint32_t)A.block_size;
            const uint32_t place = cached + (uint32_t)t - (uint32_t)starts[i];
            const uint32_t block = place / size, had = blocks_of(cached, size), offset = place - block * size;
            int32_t *entry = A.table + (int64_t)i * A.table_stride + block;
            int32_t id;
            if (block < had) {
                id = *entry;
            } else {
                const int32_t on_stack = min(max(*A.free_count, 0), A.free_capacity);
                id = A.free_blocks[on_stack - 1 - (taken[i] + (int32_t)(block - had))];
                if (offset == 0) *entry = id;  // the block's first token is a new one
            }
            if (id >= 0 && (int64_t)id < A.n_blocks) slot = (int64_t)id * size + offset;
        }
    }
    A.slots[t] = slot;
}

}  // namespace

}  // namespace prep

using namespace prep;

extern "C" {

uint64_t prep_token_positions_workspace(int32_t n_segments)
{
    return n_segments < 0 || n_segments > kMaxEntries ? 0 : ((uint64_t)n_segments + 1) * 8;
}

int prep_token_positions(int32_t device, const prep_segment *segments, int32_t n_segments, const int32_t *seq_segments, int32_t n_seq,
                         const int32_t *first, int32_t merge, int32_t *positions, int64_t capacity, int32_t *token_starts, int32_t *next,
                         void *workspace, uint64_t workspace_bytes, void *stream_ptr)
{
    hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
    if (n_segments < 0 || n_segments > kMaxEntries || n_seq < 0 || n_seq > 65535 || merge < 1 || merge > 32767 || capacity < 0 ||
        capacity > 0x7FFFFFFF || (n_segments > 0 && !segments) || !seq_segments || (capacity > 0 && !positions) || !token_starts || !workspace)
        return PREP_E_INVALID_ARG;
    if (!aligned(segments, 4) || !aligned(seq_segments, 4) || !aligned(first, 4) || !aligned(positions, 4) || !aligned(token_starts, 4) ||
        !aligned(next, 4) || !aligned(workspace, 16))
        return PREP_E_INVALID_ARG;
    if (workspace_bytes < prep_token_positions_workspace(n_segments)) return PREP_E_TOO_LARGE;
    DeviceScope scope(device);
    if (!scope.ok()) return PREP_E_HIP;
    const SegmentList L = {segments, seq_segments, first, n_segments, n_seq};
    int32_t *starts = static_cast<int32_t *>(workspace);
    uint32_t *moved = reinterpret_cast<uint32_t *>(starts + n_segments + 1);
    hipLaunchKernelGGL(sum_segments, dim3(1), dim3(kScanThreads), 0, stream, L, starts, moved);
    const int64_t items = capacity > n_seq + 1 ? capacity : n_seq + 1;
    hipLaunchKernelGGL(place_tokens, dim3((uint32_t)((items + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, L, merge,
                       (const int32_t *)starts, (const uint32_t *)moved, positions, capacity, token_starts, next);
    return hipGetLastError() == hipSuccess ? PREP_OK : PREP_E_HIP;
}

uint64_t prep_block_slots_workspace(int32_t n) { return n < 0 || n > kMaxEntries ? 0 : ((uint64_t)n + 1) * 8; }

int prep_block_slots(int32_t device, const prep_block_args *args, void *stream_ptr)
{
    hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
    if (!args) return PREP_E_INVALID_ARG;
    const prep_block_args A = *args;
    if (A.n < 0 || A.n > kMaxEntries || A.block_size < 1 || A.block_size > 65536 || A.n_blocks < 0 || A.n_blocks > 0x7FFFFFFF ||
        A.free_capacity < 0 || A.table_width < 0 || A.table_stride < A.table_width || A.capacity < 0 || A.capacity > 0x7FFFFFFF)
        return PREP_E_INVALID_ARG;
    if ((A.n > 0 && (!A.cached || !A.fresh || !A.lengths || !A.status || (A.table_width > 0 && !A.table))) ||
        (A.free_capacity > 0 && !A.free_blocks) || !A.free_count || !A.free_left || A.free_left == A.free_count || !A.token_starts ||
        (A.capacity > 0 && !A.slots) || !A.workspace)
        return PREP_E_INVALID_ARG;
    if (!aligned(A.cached, 4) || !aligned(A.fresh, 4) || !aligned(A.free_blocks, 4) || !aligned(A.free_count, 4) || !aligned(A.table, 4) ||
        !aligned(A.slots, 8) || !aligned(A.token_starts, 4) || !aligned(A.lengths, 4) || !aligned(A.status, 4) || !aligned(A.free_left, 4) ||
        !aligned(A.workspace, 16))
        return PREP_E_INVALID_ARG;
    if (A.workspace_bytes < prep_block_slots_workspace(A.n)) return PREP_E_TOO_LARGE;
    DeviceScope scope(device);
    if (!scope.ok()) return PREP_E_HIP;
    int32_t *starts = static_cast<int32_t *>(A.workspace), *taken = starts + A.n + 1;
    hipLaunchKernelGGL(sum_requests, dim3(1), dim3(kScanThreads), 0, stream, A, starts, taken);
    if (A.capacity > 0)
        hipLaunchKernelGGL(place_slots, dim3((uint32_t)((A.capacity + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, A,
                           (const int32_t *)starts, (const int32_t *)taken);
    return hipGetLastError() == hipSuccess ? PREP_OK : PREP_E_HIP;
}

}  // extern "C"
