// Places and cache slots of the tokens of a packed batch (gfx950): whole-number work on lists of
// lengths that lie on the GPU.  Both operators are a prefix sum over the list (segments of
// sequences, or requests) and then a search in it for every token.
//
// Up to kListed entries one launch does both: every workgroup sums the whole list in LDS, which costs it a few
// microseconds beside the others, and places a share of the tokens.  Longer lists are summed by one workgroup into
// the workspace, and a second launch searches there.
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
// One launch: a workgroup's threads, the longest list, entries and tokens of a thread.
constexpr int kListThreads = 512, kListWaves = kListThreads / 64, kListed = 4096, kPerThread = kListed / kListThreads;
constexpr int kTokensPerThread = 4, kTokensPerWg = kListThreads * kTokensPerThread;

// What a prefix sum carries: whole numbers that add up, and one of which the largest counts.
struct Sums {
    uint64_t tokens;
    uint64_t blocks;
    uint32_t moved;
    uint32_t sequence;
};
__device__ __forceinline__ Sums operator+(const Sums &a, const Sums &b)
{
    return {a.tokens + b.tokens, a.blocks + b.blocks, a.moved + b.moved, max(a.sequence, b.sequence)};
}
// The members that kPlaces names (places) or does not (slots) are left out.
template <bool kPlaces>
__device__ __forceinline__ Sums from_lane_before(const Sums &v, unsigned d)
{
    Sums r = {__shfl_up(v.tokens, d), 0, 0, 0};
    if (kPlaces) {
        r.moved = __shfl_up(v.moved, d);
        r.sequence = __shfl_up(v.sequence, d);
    } else {
        r.blocks = __shfl_up(v.blocks, d);
    }
    return r;
}
// v of the lanes before one's own taken together, in a workgroup of kScanWaves waves; *total = of all.
template <int kScanWaves, bool kPlaces>
__device__ Sums scan_block(Sums v, Sums *total)
{
    __shared__ Sums wave_sum[kScanWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const Sums u = from_lane_before<kPlaces>(v, (unsigned)d);
        if (lane >= d) v = u + v;
    }
    const Sums left = from_lane_before<kPlaces>(v, 1u);
    if (lane == 63) wave_sum[wave] = v;
    __syncthreads();
    Sums before = {0, 0, 0, 0}, all = {0, 0, 0, 0};
    for (int w = 0; w < kScanWaves; w++) {
        if (w < wave) before = before + wave_sum[w];
        all = all + wave_sum[w];
    }
    __syncthreads();
    *total = all;
    return lane == 0 ? before : before + left;
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

// The same for kTokens values at once: the searches' reads go out together.  top = the highest power of two below n (0 for
// n <= 1).
template <int kTokens>
__device__ __forceinline__ void search_together(const int32_t *list, int n, int top, const int64_t *v, int *at)
{
#pragma unroll
    for (int k = 0; k < kTokens; k++) at[k] = 0;
    for (int step = top; step > 0; step >>= 1) {
#pragma unroll
        for (int k = 0; k < kTokens; k++) {
            const int c = at[k] + step;
            if (c < n && list[min(c, n - 1)] <= v[k]) at[k] = c;
        }
    }
}
__device__ __forceinline__ int top_step(int n) { return n <= 1 ? 0 : 1 << (31 - __clz(n - 1)); }

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
    Sums before = {0, 0, 0, 0};
    for (int32_t at = 0; at < L.n_segments; at += kScanThreads) {
        const int32_t j = at + (int32_t)threadIdx.x;
        Sums mine = {0, 0, 0, 0}, all;
        if (j >= lo && j < hi) segment_size(L.segments[j], &mine.tokens, &mine.moved);
        const Sums here = before + scan_block<kWaves, true>(mine, &all);
        if (j < L.n_segments) {
            starts[j] = clip31(here.tokens);
            moved[j] = here.moved;
        }
        before = before + all;
    }
    if (threadIdx.x == 0) {
        starts[L.n_segments] = clip31(before.tokens);
        moved[L.n_segments] = before.moved;
    }
}

// Place of token r of a segment that starts at place `base`.
struct Place {
    uint32_t t, h, w;
};
__device__ __forceinline__ Place place_in_segment(const prep_segment &s, uint32_t base, uint32_t r, int32_t merge)
{
    Place p;
    p.t = p.h = p.w = base + r;
    if (s.h != 0) {
        const uint32_t h = (uint32_t)s.h, w = (uint32_t)s.w, m = (uint32_t)merge;
        const uint32_t a = r / (h * w), r1 = r - a * (h * w);
        p.t = base + a * (uint32_t)s.step;
        if (merge == 1) {
            const uint32_t y = r1 / w;
            p.h = base + y;
            p.w = base + (r1 - y * w);
        } else {
            // bands of m rows, windows of m columns in a band, both shorter at the edge
            const uint32_t band = r1 / (m * w), r2 = r1 - band * (m * w);
            const uint32_t tall = min(m, h - band * m);
            const uint32_t window = r2 / (tall * m), r3 = r2 - window * (tall * m);
            const uint32_t wide = min(m, w - window * m);
            const uint32_t y = r3 / wide;
            p.h = base + band * m + y;
            p.w = base + window * m + (r3 - y * wide);
        }
    }
    return p;
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
    Place p = {0, 0, 0};
    if (i < starts[L.n_segments]) {
        const int j = last_not_above(starts, L.n_segments, i);
        const int q = last_not_above(L.seq_segments, L.n_seq, j);
        const uint32_t base = (L.first ? (uint32_t)L.first[q] : 0u) + moved[j] - moved[seq_bound(L, q)];
        p = place_in_segment(L.segments[j], base, (uint32_t)i - (uint32_t)starts[j], merge);
    }
    positions[i] = (int32_t)p.t;
    positions[capacity + i] = (int32_t)p.h;
    positions[2 * capacity + i] = (int32_t)p.w;
}

// The same in one launch, for lists of at most kListed segments and as many sequences.
__global__ __launch_bounds__(kListThreads) void place_listed(SegmentList L, int32_t merge, int32_t *__restrict__ positions,
                                                             int64_t capacity, int32_t *__restrict__ token_starts,
                                                             int32_t *__restrict__ next)
{
    // of the segments: the first token (before: tokens), how far places have moved before it (before: its own share),
    // and its sequence + 1 (before: the sequence that begins there, 0 = none); of the sequences: where places
    // would start if all of the list's segments were theirs
    __shared__ alignas(16) int32_t starts[kListed + kPerThread];
    __shared__ alignas(16) uint32_t moved[kListed + kPerThread], sequence[kListed + kPerThread], origin[kListed];
    const int32_t n = L.n_segments, lo = seq_bound(L, 0), hi = seq_bound(L, L.n_seq);
    // what is read goes out together
    prep_segment segment[kPerThread];
    int32_t begins[kPerThread];
#pragma unroll
    for (int k = 0; k < kPerThread; k++) {
        const int32_t e = k * kListThreads + (int32_t)threadIdx.x;
        segment[k] = prep_segment{0, 0, 0, 0};
        if (e < n) segment[k] = L.segments[e];
        if (e < L.n_seq) begins[k] = seq_bound(L, e);
    }
    for (int32_t j = threadIdx.x; j <= n; j += kListThreads) sequence[j] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPerThread; k++) {
        const int32_t e = k * kListThreads + (int32_t)threadIdx.x;
        if (e < L.n_seq) atomicMax(&sequence[begins[k]], (uint32_t)e + 1);
        if (e < n) {
            uint64_t tokens = 0;
            uint32_t advance = 0;
            if (e >= lo && e < hi) segment_size(segment[k], &tokens, &advance);
            starts[e] = clip31(tokens);
            moved[e] = advance;
        }
    }
    __syncthreads();
    const int32_t j0 = (int32_t)threadIdx.x * kPerThread;
    Sums mine = {0, 0, 0, 0}, all;
#pragma unroll
    for (int k = 0; k < kPerThread; k++)
        if (j0 + k < n) mine = mine + Sums{(uint64_t)(uint32_t)starts[j0 + k], 0, moved[j0 + k], sequence[j0 + k]};
    Sums here = scan_block<kListWaves, true>(mine, &all);
#pragma unroll
    for (int k = 0; k < kPerThread; k++) {
        if (j0 + k < n) {
            const Sums own = {(uint64_t)(uint32_t)starts[j0 + k], 0, moved[j0 + k], sequence[j0 + k]};
            starts[j0 + k] = clip31(here.tokens);
            moved[j0 + k] = here.moved;
            here = here + own;
            sequence[j0 + k] = here.sequence;
        }
    }
    if (threadIdx.x == 0) {
        starts[n] = clip31(all.tokens);
        moved[n] = all.moved;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPerThread; k++) {
        const int32_t q = k * kListThreads + (int32_t)threadIdx.x;
        if (q < L.n_seq) origin[q] = (L.first ? (uint32_t)L.first[q] : 0u) - moved[begins[k]];
    }
    // the sequences' own results, dealt to the workgroups
    for (int32_t q = (int32_t)(blockIdx.x * kListThreads + threadIdx.x); q <= L.n_seq; q += (int32_t)(gridDim.x * kListThreads)) {
        const int32_t b = seq_bound(L, q);
        token_starts[q] = starts[b];
        if (next != nullptr && q < L.n_seq) next[q] = (int32_t)((L.first ? (uint32_t)L.first[q] : 0u) + moved[seq_bound(L, q + 1)] - moved[b]);
    }
    __syncthreads();
    const int64_t token0 = (int64_t)blockIdx.x * kTokensPerWg + threadIdx.x;
    int64_t token[kTokensPerThread];
    int at[kTokensPerThread];
#pragma unroll
    for (int k = 0; k < kTokensPerThread; k++) token[k] = token0 + k * kListThreads;
    search_together<kTokensPerThread>(starts, n, top_step(n), token, at);
    const int32_t total = starts[n];
#pragma unroll
    for (int k = 0; k < kTokensPerThread; k++) segment[k] = token[k] < total ? L.segments[at[k]] : prep_segment{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < kTokensPerThread; k++) {
        if (token[k] >= capacity) break;
        Place p = {0, 0, 0};
        if (token[k] < total) {
            const int j = at[k];
            const uint32_t q = sequence[j];  // (not 0 where a segment has tokens)
            const uint32_t base = (q != 0 ? origin[q - 1] : 0u) + moved[j];
            p = place_in_segment(segment[k], base, (uint32_t)token[k] - (uint32_t)starts[j], merge);
        }
        positions[token[k]] = (int32_t)p.t;
        positions[capacity + token[k]] = (int32_t)p.h;
        positions[2 * capacity + token[k]] = (int32_t)p.w;
    }
}
static_assert(kTokensPerThread <= kPerThread, "place_listed keeps the tokens' segments where it kept the list's");

// ---- slots ---------------------------------------------------------------------------------------

// Blocks that hold v tokens (v < 2^31)
__device__ __forceinline__ uint32_t blocks_of(uint32_t v, uint32_t block_size)
{
    const uint32_t whole = v / block_size;
    return whole + (whole * block_size != v ? 1u : 0u);
}

// Tokens of request i, and the blocks that it needs; false = it cannot be served whatever there is (or is no request).
// Of the requests before, all count: once a sum of tokens is beyond the capacity, or a sum of blocks beyond the stack, so
// are the later ones, and what is refused changes nothing for them.
__device__ __forceinline__ bool request_needs(const prep_block_args &A, int32_t cached, int32_t fresh, uint32_t *tokens, uint32_t *blocks)
{
    *tokens = *blocks = 0;
    if (cached < 0 || fresh < 0) return false;
    *tokens = (uint32_t)fresh;
    const uint32_t after = (uint32_t)cached + (uint32_t)fresh;
    const uint32_t want = blocks_of(after, (uint32_t)A.block_size);
    if (after > (uint32_t)INT32_MAX || want > (uint32_t)A.table_width) return false;
    *blocks = want - blocks_of((uint32_t)cached, (uint32_t)A.block_size);
    return true;
}
// Blocks off the stack before a request's own, or -1: it is refused.
__device__ __forceinline__ int32_t grant(const prep_block_args &A, const Sums &before, uint32_t tokens, uint32_t blocks, int32_t on_stack)
{
    if (before.tokens + tokens > (uint64_t)A.capacity) return -1;
    if (blocks == 0) return 0;
    return before.blocks + blocks <= (uint64_t)on_stack ? (int32_t)before.blocks : -1;
}
__device__ __forceinline__ void report_request(const prep_block_args &A, int32_t i, int32_t cached, int32_t fresh, bool granted)
{
    const bool sound = cached >= 0 && fresh >= 0;
    A.lengths[i] = granted ? cached + fresh : sound ? cached : 0;
    A.status[i] = granted ? PREP_OK : sound ? PREP_E_TOO_LARGE : PREP_E_INVALID_ARG;
}

// starts[i]: first token of request i, n + 1 entries; taken[i]: as grant gives it.
__global__ __launch_bounds__(kScanThreads) void sum_requests(prep_block_args A, int32_t *__restrict__ starts, int32_t *__restrict__ taken)
{
    __shared__ uint32_t used;  // blocks that go
    if (threadIdx.x == 0) used = 0;
    const int32_t on_stack = min(max(*A.free_count, 0), A.free_capacity);
    Sums before = {0, 0, 0, 0};
    for (int32_t at = 0; at < A.n; at += kScanThreads) {
        const int32_t i = at + (int32_t)threadIdx.x;
        const int32_t cached = i < A.n ? A.cached[i] : -1, fresh = i < A.n ? A.fresh[i] : -1;
        uint32_t tokens, blocks;
        const bool fits = request_needs(A, cached, fresh, &tokens, &blocks);
        Sums all;
        const Sums here = before + scan_block<kWaves, false>(Sums{tokens, blocks, 0, 0}, &all);
        const int32_t given = fits ? grant(A, here, tokens, blocks, on_stack) : -1;
        if (given >= 0 && blocks != 0) atomicMax(&used, (uint32_t)given + blocks);  // (sums only grow)
        if (i < A.n) {
            starts[i] = A.token_starts[i] = clip31(here.tokens);
            taken[i] = given;
            report_request(A, i, cached, fresh, given >= 0);
        }
        before = before + all;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        starts[A.n] = A.token_starts[A.n] = clip31(before.tokens);
        *A.free_left = on_stack - (int32_t)used;
    }
}

// Slot of token t of a request that is served: blocks taken before its own, its first token.
__device__ __forceinline__ int64_t slot_of(const prep_block_args &A, int32_t i, uint32_t cached, uint32_t r, int32_t taken, int32_t on_stack)
{
    const uint32_t size = (uint32_t)A.block_size, place = cached + r;
    const uint32_t block = place / size, had = blocks_of(cached, size), offset = place - block * size;
    int32_t *entry = A.table + (int64_t)i * A.table_stride + block;
    int32_t id;
    if (block < had) {
        id = *entry;
    } else {
        id = A.free_blocks[on_stack - 1 - (taken + (int32_t)(block - had))];
        if (offset == 0) *entry = id;  // the block's first token is a new one
    }
    return id >= 0 && (int64_t)id < A.n_blocks ? (int64_t)id * size + offset : -1;
}

__global__ __launch_bounds__(kThreads) void place_slots(prep_block_args A, const int32_t *__restrict__ starts, const int32_t *__restrict__ taken)
{
    const int64_t t = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (t >= A.capacity) return;
    int64_t slot = -1;
    if (t < starts[A.n]) {
        const int i = last_not_above(starts, A.n, t);
        if (taken[i] >= 0)
            slot = slot_of(A, i, (uint32_t)A.cached[i], (uint32_t)t - (uint32_t)starts[i], taken[i], min(max(*A.free_count, 0), A.free_capacity));
    }
    A.slots[t] = slot;
}

// Both in one launch, for at most kListed requests.
__global__ __launch_bounds__(kListThreads) void place_slots_listed(prep_block_args A)
{
    // of the requests: the first token (before: tokens), and blocks taken before its own or -1 (before: the blocks
    // that it needs or -1)
    __shared__ alignas(16) int32_t starts[kListed + kPerThread], taken[kListed + kPerThread];
    __shared__ uint32_t used;
    const int32_t n = A.n, i0 = (int32_t)threadIdx.x * kPerThread;
    const int32_t on_stack = min(max(*A.free_count, 0), A.free_capacity);
    if (threadIdx.x == 0) used = 0;
    int32_t cached[kPerThread], fresh[kPerThread];  // (the reads go out together)
#pragma unroll
    for (int k = 0; k < kPerThread; k++) {
        const int32_t i = k * kListThreads + (int32_t)threadIdx.x;
        cached[k] = i < n ? A.cached[i] : -1;
        fresh[k] = i < n ? A.fresh[i] : -1;
    }
#pragma unroll
    for (int k = 0; k < kPerThread; k++) {
        const int32_t i = k * kListThreads + (int32_t)threadIdx.x;
        if (i < n) {
            uint32_t tokens, blocks;
            const bool fits = request_needs(A, cached[k], fresh[k], &tokens, &blocks);
            starts[i] = (int32_t)tokens;
            taken[i] = fits ? (int32_t)blocks : -1;
        }
    }
    __syncthreads();
    Sums mine = {0, 0, 0, 0}, all;
#pragma unroll
    for (int k = 0; k < kPerThread; k++)
        if (i0 + k < n) mine = mine + Sums{(uint64_t)(uint32_t)starts[i0 + k], (uint64_t)(uint32_t)max(taken[i0 + k], 0), 0, 0};
    Sums here = scan_block<kListWaves, false>(mine, &all);
    uint32_t most = 0;  // blocks off the stack after the thread's last request that takes some
#pragma unroll
    for (int k = 0; k < kPerThread; k++) {
        if (i0 + k < n) {
            const uint32_t tokens = (uint32_t)starts[i0 + k], blocks = (uint32_t)max(taken[i0 + k], 0);
            const int32_t given = taken[i0 + k] >= 0 ? grant(A, here, tokens, blocks, on_stack) : -1;
            if (given >= 0 && blocks != 0) most = (uint32_t)given + blocks;
            starts[i0 + k] = clip31(here.tokens);
            taken[i0 + k] = given;
            here = here + Sums{tokens, blocks, 0, 0};
        }
    }
    if (most != 0) atomicMax(&used, most);
    if (threadIdx.x == 0) starts[n] = clip31(all.tokens);
    __syncthreads();
    const int64_t token0 = (int64_t)blockIdx.x * kTokensPerWg + threadIdx.x;
    int64_t token[kTokensPerThread];
    int at[kTokensPerThread];
    int32_t length[kTokensPerThread];
#pragma unroll
    for (int k = 0; k < kTokensPerThread; k++) token[k] = token0 + k * kListThreads;
    search_together<kTokensPerThread>(starts, n, top_step(n), token, at);
    const int32_t total = starts[n];
#pragma unroll
    for (int k = 0; k < kTokensPerThread; k++) length[k] = token[k] < total ? A.cached[at[k]] : 0;
#pragma unroll
    for (int k = 0; k < kTokensPerThread; k++) {
        if (token[k] >= A.capacity) break;
        int64_t slot = -1;
        if (token[k] < total && taken[at[k]] >= 0)
            slot = slot_of(A, at[k], (uint32_t)length[k], (uint32_t)token[k] - (uint32_t)starts[at[k]], taken[at[k]], on_stack);
        A.slots[token[k]] = slot;
    }
    // the requests' own results, dealt to the workgroups
    for (int32_t i = (int32_t)(blockIdx.x * kListThreads + threadIdx.x); i <= n; i += (int32_t)(gridDim.x * kListThreads)) {
        A.token_starts[i] = starts[i];
        if (i < n) report_request(A, i, A.cached[i], A.fresh[i], taken[i] >= 0);
        else *A.free_left = on_stack - (int32_t)used;
    }
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
    if (n_segments <= kListed && n_seq <= kListed) {
        const int64_t blocks = capacity > kTokensPerWg ? (capacity + kTokensPerWg - 1) / kTokensPerWg : 1;
        hipLaunchKernelGGL(place_listed, dim3((uint32_t)blocks), dim3(kListThreads), 0, stream, L, merge, positions, capacity, token_starts, next);
        return hipGetLastError() == hipSuccess ? PREP_OK : PREP_E_HIP;
    }
    hipLaunchKernelGGL(sum_segments, dim3(1), dim3(kScanThreads), 0, stream, L, starts, moved);
    const int64_t items = capacity > n_seq + 1 ? capacity : n_seq + 1;
    hipLaunchKernelGGL(place_tokens, dim3((uint32_t)((items + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, L, merge,
                       (const int32_t *)starts, (const uint32_t *)moved, positions, capacity, token_starts, next);
    return hipGetLastError() == hipSuccess ? PREP_OK : PREP_E_HIP;
}

uint64_t prep_block_slots_workspace(int32_t n) { return n < 0 || n > kMaxEntries ? 0 : ((uint64_t)n + 1) * 8; }

static_assert(sizeof(prep_block_args) == 136, "as the binding packs it");

int prep_block_slots(int32_t device, const prep_block_args *args, void *stream_ptr)
{
    hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
    if (!args) return PREP_E_INVALID_ARG;
    const prep_block_args A = *args;
    if (A.n < 0 || A.n > kMaxEntries || A.block_size < 1 || A.block_size > 65536 || A.n_blocks < 0 || A.n_blocks > 0x7FFFFFFF ||
        A.free_capacity < 0 || A.table_width < 0 || A.table_stride < A.table_width || A.capacity < 0 || A.capacity > 0x7FFFFFFF)
        return PREP_E_INVALID_ARG;
    if ((A.n > 0 && (!A.cached || !A.fresh || !A.lengths || !A.status || (A.table_width > 0 && !A.table))) ||
        (A.free_capacity > 0 && !A.free_blocks) || !A.free_count || !A.free_left || A.free_left == A.free_count || (A.n > 0 && (A.lengths == A.cached || A.lengths == A.fresh || A.status == A.cached || A.status == A.fresh)) || !A.token_starts ||
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
    if (A.n <= kListed) {
        const int64_t blocks = A.capacity > kTokensPerWg ? (A.capacity + kTokensPerWg - 1) / kTokensPerWg : 1;
        hipLaunchKernelGGL(place_slots_listed, dim3((uint32_t)blocks), dim3(kListThreads), 0, stream, A);
        return hipGetLastError() == hipSuccess ? PREP_OK : PREP_E_HIP;
    }
    hipLaunchKernelGGL(sum_requests, dim3(1), dim3(kScanThreads), 0, stream, A, starts, taken);
    if (A.capacity > 0)
        hipLaunchKernelGGL(place_slots, dim3((uint32_t)((A.capacity + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, A,
                           (const int32_t *)starts, (const int32_t *)taken);
    return hipGetLastError() == hipSuccess ? PREP_OK : PREP_E_HIP;
}

}  // extern "C"
