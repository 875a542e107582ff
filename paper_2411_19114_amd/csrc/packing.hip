// Places and cache slots of the tokens of a packed batch (gfx950): whole-number work on lists of
// lengths that lie on the GPU.  Both operators are a prefix sum over the list (segments of
// sequences, or requests) and then a search in it for every token.
//
// Neither moves much (5 MB for the places of 400 000 tokens): what counts is the chain of reads that wait for one another.
// Lists of up to 4096 entries take one launch: every workgroup sums the whole list in LDS, entries of a thread adjacent and
// all reads sent at once, and places a share of the tokens.  Longer lists are summed by one workgroup into the workspace,
// and a second launch searches there.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "../../include/prep.h"
#include "tokens.h"

namespace prep {

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kTokens = 4;                 // of a thread
constexpr int kWgTokens = kThreads * kTokens;
constexpr int kSumEntries = 8;             // entries of a thread at a time in the launch that sums a long list
constexpr int32_t kMaxEntries = 1 << 20;

// What a prefix sum carries.
struct Sums {
    uint64_t tokens;
    uint64_t more;  // by how much places move on (modulo 2^32), or blocks
};
__device__ __forceinline__ Sums operator+(const Sums &a, const Sums &b) { return {a.tokens + b.tokens, a.more + b.more}; }

// v of the threads before one's own taken together; *total = of all.
__device__ Sums scan_workgroup(Sums v, Sums *total)
{
    __shared__ Sums wave_sum[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const Sums u = {__shfl_up(v.tokens, (unsigned)d), __shfl_up(v.more, (unsigned)d)};
        if (lane >= d) v = u + v;
    }
    const Sums left = {__shfl_up(v.tokens, 1u), __shfl_up(v.more, 1u)};
    if (lane == 63) wave_sum[wave] = v;
    __syncthreads();
    Sums before = {0, 0}, all = {0, 0};
#pragma unroll
    for (int w = 0; w < kWaves; w++) {
        if (w < wave) before = before + wave_sum[w];
        all = all + wave_sum[w];
    }
    __syncthreads();
    *total = all;
    return lane == 0 ? before : before + left;
}

__device__ __forceinline__ int32_t clip31(uint64_t v) { return v > 0x7FFFFFFFull ? 0x7FFFFFFF : (int32_t)v; }

// For kTokens values at once: the index of the last entry that is <= v[k] among list[lo] .. list[hi - 1], ascending; lo if there is
// none.  Written without branches, so that a step's reads go out together: with a wait for each of them a step in LDS
// takes 0.25 us.
__device__ __forceinline__ void search_together(const int32_t *list, int lo, int hi, const int32_t *v, int *at)
{
    const int n = hi - lo;
#pragma unroll
    for (int k = 0; k < kTokens; k++) at[k] = lo;
    for (int step = n <= 1 ? 0 : 1 << (31 - __clz(n - 1)); step > 0; step >>= 1) {
        int32_t entry[kTokens];
#pragma unroll
        for (int k = 0; k < kTokens; k++) entry[k] = list[min(at[k] + step, hi - 1)];
#pragma unroll
        for (int k = 0; k < kTokens; k++) at[k] += (at[k] + step < hi) & (entry[k] <= v[k]) ? step : 0;
    }
}
// For a workgroup whose values lie in v0 .. v1: the part *lo .. *hi - 1 of a list in memory that they can be found in, by one
// read of a thread each.  To be called by all threads.
__device__ void narrow(const int32_t *list, int n, int32_t v0, int32_t v1, int *lo, int *hi)
{
    __shared__ uint32_t bounds[2];  // pivots not above v0; and v1
    if (threadIdx.x == 0) bounds[0] = bounds[1] = 0;
    __syncthreads();
    const int stride = (n + kThreads - 1) / kThreads, at = (int)threadIdx.x * stride;
    if (at < n) {
        const int32_t v = list[at];
        if (v <= v0) atomicMax(&bounds[0], threadIdx.x);
        if (v <= v1) atomicMax(&bounds[1], threadIdx.x);
    }
    __syncthreads();
    *lo = (int)bounds[0] * stride;
    *hi = min(((int)bounds[1] + 1) * stride, n);
    __syncthreads();
}

// ---- places --------------------------------------------------------------------------------------

struct SegmentList {
    const prep_segment *segments;
    const int32_t *seq_segments;
    const int32_t *first;
    int32_t n_segments, n_seq, merge;
    int64_t capacity;
    int32_t *positions, *token_starts, *next;
};
__device__ __forceinline__ int32_t seq_bound(const SegmentList &L, int i) { return min(max(L.seq_segments[i], 0), L.n_segments); }

// Tokens of a segment (2^31 stand for more, so that sums over 2^20 segments stay in 64 bits: what lies behind that many tokens is beyond any
// capacity), and how far places move on; both 0 for one that is not valid.
__device__ __forceinline__ Sums segment_size(const prep_segment &s)
{
    constexpr int32_t kMost = 32767;
    if (s.h == 0 && s.w == 0) {
        const uint32_t n = s.t > 0 && s.step == 0 ? (uint32_t)s.t : 0;
        return {n, n};
    }
    if (s.t < 1 || s.h < 1 || s.w < 1 || s.step < 0 || s.t > kMost || s.h > kMost || s.w > kMost || s.step > kMost) return {0, 0};
    return {min((uint64_t)s.t * (uint32_t)(s.h * s.w), (uint64_t)1 << 31), (uint64_t)(uint32_t)(max(max((s.t - 1) * s.step, s.h - 1), s.w - 1) + 1)};
}

// Place of token r of a segment that starts at place `base`; h = 0: text.
struct Place {
    uint32_t t, h, w;
};
__device__ __forceinline__ Place place_in_segment(uint32_t h, uint32_t w, uint32_t step, uint32_t base, uint32_t r, uint32_t m)
{
    Place p;
    p.t = p.h = p.w = base + r;
    if (h != 0) {
        const uint32_t a = r / (h * w), r1 = r - a * (h * w);
        p.t = base + a * step;
        if (m == 1) {
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
__device__ __forceinline__ void store_place(const SegmentList &L, int64_t i, const Place &p)
{
    L.positions[i] = (int32_t)p.t;
    L.positions[L.capacity + i] = (int32_t)p.h;
    L.positions[2 * L.capacity + i] = (int32_t)p.w;
}

// Long lists, first launch.  starts[j]: first token of segment j (at most 2^31 - 1); moved[j]: how far places have moved on
// before it, over all segments.  n_segments + 1 entries each.
__global__ __launch_bounds__(kThreads) void sum_segments(SegmentList L, int32_t *__restrict__ starts, uint32_t *__restrict__ moved)
{
    const int32_t n = L.n_segments, lo = seq_bound(L, 0), hi = seq_bound(L, L.n_seq);
    Sums before = {0, 0};
    for (int32_t at = 0; at < n; at += kThreads * kSumEntries) {
        const int32_t j0 = at + (int32_t)threadIdx.x * kSumEntries;
        Sums own[kSumEntries], mine = {0, 0}, all;
#pragma unroll
        for (int k = 0; k < kSumEntries; k++) {
            const int32_t j = j0 + k;
            own[k] = j >= lo && j < hi ? segment_size(L.segments[j]) : Sums{0, 0};
        }
#pragma unroll
        for (int k = 0; k < kSumEntries; k++) mine = mine + own[k];
        Sums here = before + scan_workgroup(mine, &all);
#pragma unroll
        for (int k = 0; k < kSumEntries; k++) {
            if (j0 + k < n) {
                starts[j0 + k] = clip31(here.tokens);
                moved[j0 + k] = (uint32_t)here.more;
            }
            here = here + own[k];
        }
        before = before + all;
    }
    if (threadIdx.x == 0) {
        starts[n] = clip31(before.tokens);
        moved[n] = (uint32_t)before.more;
    }
}

// Second launch.
__global__ __launch_bounds__(kThreads) void place_tokens(SegmentList L, const int32_t *__restrict__ starts, const uint32_t *__restrict__ moved)
{
    for (int64_t q = (int64_t)blockIdx.x * kThreads + threadIdx.x; q <= L.n_seq; q += (int64_t)gridDim.x * kThreads) {
        const int32_t b = seq_bound(L, (int)q);
        L.token_starts[q] = starts[b];
        if (L.next != nullptr && q < L.n_seq)
            L.next[q] = (int32_t)((L.first ? (uint32_t)L.first[q] : 0u) + moved[seq_bound(L, (int)q + 1)] - moved[b]);
    }
    const int64_t token0 = (int64_t)blockIdx.x * kWgTokens;
    const int32_t total = starts[L.n_segments];
    int j_lo = 0, j_hi = 0, q_lo = 0, q_hi = 0;
    if (token0 < total) {
        narrow(starts, L.n_segments, (int32_t)token0, (int32_t)min(token0 + kWgTokens, (int64_t)total) - 1, &j_lo, &j_hi);
        narrow(L.seq_segments, L.n_seq, j_lo, j_hi - 1, &q_lo, &q_hi);
    }
    int32_t token[kTokens], segment[kTokens], sequence[kTokens];
#pragma unroll
    for (int k = 0; k < kTokens; k++) token[k] = (int32_t)min(token0 + k * kThreads + (int64_t)threadIdx.x, (int64_t)total - 1);
    search_together(starts, j_lo, j_hi, token, segment);
    search_together(L.seq_segments, q_lo, q_hi, segment, sequence);
#pragma unroll
    for (int k = 0; k < kTokens; k++) {
        const int64_t i = token0 + k * kThreads + threadIdx.x;
        if (i >= L.capacity) break;
        Place p = {0, 0, 0};
        if (i < total) {
            const int j = segment[k], q = sequence[k];
            const prep_segment s = L.segments[j];
            const uint32_t base = (L.first ? (uint32_t)L.first[q] : 0u) + moved[j] - moved[seq_bound(L, q)];
            p = place_in_segment((uint32_t)s.h, (uint32_t)s.w, (uint32_t)s.step, base, (uint32_t)i - (uint32_t)starts[j], (uint32_t)L.merge);
        }
        store_place(L, i, p);
    }
}

// One launch, for at most kThreads * kEntries segments and sequences.  In a graph 4.6 us for 64 sequences of a token, 9.1 for 2048
// segments of 400 000 tokens and 10.7 for 2200 (eight entries a thread, not four); bound by the chain of reads, sum and search, not by the 5 MB.  At 4096
// segments 9 to 12 us by the number of tokens; the two launches take 20 to 27 at 4097, 56 at 20 000, 0.21 ms at 100 000 and 2.1 ms at 2^20.
template <int kEntries>
__global__ __launch_bounds__(kThreads) void place_listed(SegmentList L)
{
    constexpr int kList = kThreads * kEntries;
    // of the segments: first token, places moved on before, sides (15 bits each), step; of the sequences: first token, and where
    // places would start if all segments before were theirs
    __shared__ alignas(16) int32_t starts[kList + 4], seq_tokens[kList];
    __shared__ alignas(16) uint32_t moved[kList + 4], sides[kList], steps[kList], origin[kList];
    const int32_t n = L.n_segments, j0 = (int32_t)threadIdx.x * kEntries;
    const int32_t lo = seq_bound(L, 0), hi = seq_bound(L, L.n_seq);
    prep_segment segment[kEntries];
    int32_t begins[kEntries], ends[kEntries];
    uint32_t first[kEntries];
#pragma unroll
    for (int k = 0; k < kEntries; k++) {
        const int32_t j = j0 + k, q = k * kThreads + (int32_t)threadIdx.x;
        segment[k] = j < n ? L.segments[j] : prep_segment{0, 0, 0, 0};
        begins[k] = q < L.n_seq ? seq_bound(L, q) : 0;
        ends[k] = q < L.n_seq ? seq_bound(L, q + 1) : 0;
        first[k] = L.first != nullptr && q < L.n_seq ? (uint32_t)L.first[q] : 0u;
    }
    Sums own[kEntries], mine = {0, 0}, all;
#pragma unroll
    for (int k = 0; k < kEntries; k++) {
        own[k] = j0 + k >= lo && j0 + k < hi ? segment_size(segment[k]) : Sums{0, 0};
        mine = mine + own[k];
    }
    Sums here = scan_workgroup(mine, &all);
#pragma unroll
    for (int k = 0; k < kEntries; k++) {
        starts[j0 + k] = clip31(here.tokens);
        moved[j0 + k] = (uint32_t)here.more;
        sides[j0 + k] = (uint32_t)segment[k].h << 16 | ((uint32_t)segment[k].w & 0xFFFFu);
        steps[j0 + k] = (uint32_t)segment[k].step;
        here = here + own[k];
    }
    if (threadIdx.x == 0) {
        // (where the list fills the threads' entries, nobody else writes these)
        starts[kList] = clip31(all.tokens);
        moved[kList] = (uint32_t)all.more;
    }
    __syncthreads();
    const int32_t total = clip31(all.tokens);
#pragma unroll
    for (int k = 0; k < kEntries; k++) {
        const int32_t q = k * kThreads + (int32_t)threadIdx.x;
        if (q < L.n_seq) {
            seq_tokens[q] = starts[begins[k]];
            origin[q] = first[k] - moved[begins[k]];
            // a share of the sequences' own results
            if (((int)threadIdx.x >> 6) % (int)gridDim.x == (int)blockIdx.x) {
                L.token_starts[q] = starts[begins[k]];
                if (L.next != nullptr) L.next[q] = (int32_t)(first[k] + moved[ends[k]] - moved[begins[k]]);
            }
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) L.token_starts[L.n_seq] = starts[hi];
    __syncthreads();
    const int64_t token0 = (int64_t)blockIdx.x * kWgTokens + threadIdx.x;
    int32_t token[kTokens];
    int at[kTokens], seq[kTokens];
#pragma unroll
    for (int k = 0; k < kTokens; k++) token[k] = (int32_t)min(token0 + k * kThreads, (int64_t)total - 1);
    search_together(starts, 0, n, token, at);
    search_together(seq_tokens, 0, L.n_seq, token, seq);
#pragma unroll
    for (int k = 0; k < kTokens; k++) {
        if (token0 + k * kThreads >= L.capacity) break;
        Place p = {0, 0, 0};
        if (token0 + k * kThreads < total) {
            const int j = at[k];
            p = place_in_segment(sides[j] >> 16, sides[j] & 0xFFFFu, steps[j], origin[seq[k]] + moved[j], (uint32_t)(token[k] - starts[j]),
                                 (uint32_t)L.merge);
        }
        store_place(L, token0 + k * kThreads, p);
    }
}

// ---- slots ---------------------------------------------------------------------------------------

// v / size for a block size, by a shift where it is a power of two.
struct BlockSize {
    uint32_t size;
    int32_t shift;  // -1: no power of two
    __device__ __forceinline__ uint32_t quotient(uint32_t v) const { return shift >= 0 ? v >> shift : v / size; }
    // blocks that hold v tokens
    __device__ __forceinline__ uint32_t holding(uint32_t v) const
    {
        const uint32_t whole = quotient(v);
        return whole + (whole * size != v ? 1u : 0u);
    }
};

// Tokens of a request and the blocks that it needs; false = it cannot be served whatever there is (or is no request).
// All requests before one's own count: once a sum of tokens is beyond the capacity, or a sum of blocks beyond the stack, so
// are the later ones, so that what is refused changes nothing for them.
__device__ __forceinline__ bool request_needs(const prep_block_args &A, const BlockSize &B, int32_t cached, int32_t fresh, Sums *needs)
{
    *needs = Sums{0, 0};
    if (cached < 0 || fresh < 0) return false;
    needs->tokens = (uint32_t)fresh;
    const uint32_t after = (uint32_t)cached + (uint32_t)fresh, want = B.holding(after);
    if (after > (uint32_t)INT32_MAX || want > (uint32_t)A.table_width) return false;
    needs->more = want - B.holding((uint32_t)cached);
    return true;
}
// Blocks off the stack before a request's own, or -1: it is refused.
__device__ __forceinline__ int32_t grant(const prep_block_args &A, const Sums &before, const Sums &needs, int32_t on_stack)
{
    if (before.tokens + needs.tokens > (uint64_t)A.capacity) return -1;
    if (needs.more == 0) return 0;
    return before.more + needs.more <= (uint64_t)on_stack ? (int32_t)before.more : -1;
}
__device__ __forceinline__ void report_request(const prep_block_args &A, int32_t i, uint64_t start, int32_t cached, int32_t fresh, bool granted)
{
    const bool sound = cached >= 0 && fresh >= 0;
    A.token_starts[i] = clip31(start);
    A.lengths[i] = granted ? cached + fresh : sound ? cached : 0;
    A.status[i] = granted ? PREP_OK : sound ? PREP_E_TOO_LARGE : PREP_E_INVALID_ARG;
}
__device__ __forceinline__ int32_t stack_height(const prep_block_args &A) { return min(max(*A.free_count, 0), A.free_capacity); }

// Slot of token r of request i, which is served.
__device__ __forceinline__ int64_t slot_of(const prep_block_args &A, const BlockSize &B, int32_t i, uint32_t cached, uint32_t r, int32_t taken,
                                           int32_t on_stack)
{
    const uint32_t place = cached + r, block = B.quotient(place), had = B.holding(cached), offset = place - block * B.size;
    int32_t *entry = A.table + (int64_t)i * A.table_stride + block;
    int32_t id;
    if (block < had) {
        id = *entry;
    } else {
        id = A.free_blocks[on_stack - 1 - (taken + (int32_t)(block - had))];
        if (offset == 0) *entry = id;  // the block's first token is a new one
    }
    return id >= 0 && (int64_t)id < A.n_blocks ? (int64_t)id * B.size + offset : -1;
}

// Long lists, first launch.  starts[i]: first token of request i, n + 1 entries; taken[i]: as grant gives it.
__global__ __launch_bounds__(kThreads) void sum_requests(prep_block_args A, BlockSize B, int32_t *__restrict__ starts, int32_t *__restrict__ taken)
{
    __shared__ uint32_t used;  // blocks that go
    if (threadIdx.x == 0) used = 0;
    const int32_t on_stack = stack_height(A);
    Sums before = {0, 0};
    for (int32_t at = 0; at < A.n; at += kThreads * kSumEntries) {
        const int32_t i0 = at + (int32_t)threadIdx.x * kSumEntries;
        int32_t cached[kSumEntries], fresh[kSumEntries];
#pragma unroll
        for (int k = 0; k < kSumEntries; k++) {
            cached[k] = i0 + k < A.n ? A.cached[i0 + k] : -1;
            fresh[k] = i0 + k < A.n ? A.fresh[i0 + k] : -1;
        }
        Sums mine = {0, 0}, all, own;
#pragma unroll
        for (int k = 0; k < kSumEntries; k++) {
            (void)request_needs(A, B, cached[k], fresh[k], &own);
            mine = mine + own;
        }
        Sums here = before + scan_workgroup(mine, &all);
        uint32_t most = 0;  // (sums only grow)
#pragma unroll
        for (int k = 0; k < kSumEntries; k++) {
            const bool fits = request_needs(A, B, cached[k], fresh[k], &own);
            const int32_t given = fits ? grant(A, here, own, on_stack) : -1;
            if (given >= 0 && own.more != 0) most = (uint32_t)given + (uint32_t)own.more;
            if (i0 + k < A.n) {
                starts[i0 + k] = clip31(here.tokens);
                taken[i0 + k] = given;
                report_request(A, i0 + k, here.tokens, cached[k], fresh[k], given >= 0);
            }
            here = here + own;
        }
        if (most != 0) atomicMax(&used, most);
        before = before + all;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        starts[A.n] = A.token_starts[A.n] = clip31(before.tokens);
        *A.free_left = on_stack - (int32_t)used;
    }
}

// Second launch.
__global__ __launch_bounds__(kThreads) void place_slots(prep_block_args A, BlockSize B, const int32_t *__restrict__ starts,
                                                        const int32_t *__restrict__ taken)
{
    const int64_t token0 = (int64_t)blockIdx.x * kWgTokens;
    const int32_t total = starts[A.n], on_stack = stack_height(A);
    int lo = 0, hi = 0;
    if (token0 < total) narrow(starts, A.n, (int32_t)token0, (int32_t)min(token0 + kWgTokens, (int64_t)total) - 1, &lo, &hi);
    int32_t token[kTokens], request[kTokens];
#pragma unroll
    for (int k = 0; k < kTokens; k++) token[k] = (int32_t)min(token0 + k * kThreads + (int64_t)threadIdx.x, (int64_t)total - 1);
    search_together(starts, lo, hi, token, request);
#pragma unroll
    for (int k = 0; k < kTokens; k++) {
        const int64_t t = token0 + k * kThreads + threadIdx.x;
        if (t >= A.capacity) break;
        int64_t slot = -1;
        if (t < total) {
            const int i = request[k];
            if (taken[i] >= 0) slot = slot_of(A, B, i, (uint32_t)A.cached[i], (uint32_t)t - (uint32_t)starts[i], taken[i], on_stack);
        }
        A.slots[t] = slot;
    }
}

// One launch, for at most kThreads * kEntries requests.  In a graph 4.1 us for 128 requests of a token, 10 for 2000 of 300 000 tokens.  At 4096
// requests 14 to 16 us by the number of tokens; the two launches take 20 to 32 at 4097, 71 to 90 at 20 000, 0.34 to 0.38 ms at 100 000 and 3.5 to 3.9 ms at 2^20.
template <int kEntries>
__global__ __launch_bounds__(kThreads) void place_slots_listed(prep_block_args A, BlockSize B)
{
    constexpr int kList = kThreads * kEntries;
    __shared__ alignas(16) int32_t starts[kList], taken[kList], lengths[kList];
    __shared__ uint32_t used;
    const int32_t n = A.n, i0 = (int32_t)threadIdx.x * kEntries;
    int32_t cached[kEntries], fresh[kEntries];
#pragma unroll
    for (int k = 0; k < kEntries; k++) {
        cached[k] = i0 + k < n ? A.cached[i0 + k] : -1;
        fresh[k] = i0 + k < n ? A.fresh[i0 + k] : -1;
    }
    const int32_t on_stack = stack_height(A);
    if (threadIdx.x == 0) used = 0;
    Sums own[kEntries], mine = {0, 0}, all;
    bool fits[kEntries];
#pragma unroll
    for (int k = 0; k < kEntries; k++) {
        fits[k] = request_needs(A, B, cached[k], fresh[k], &own[k]);
        mine = mine + own[k];
    }
    Sums here = scan_workgroup(mine, &all);
    uint32_t most = 0;  // blocks off the stack after the thread's last request that takes some (sums only grow)
    const bool reports = ((int)threadIdx.x >> 6) % (int)gridDim.x == (int)blockIdx.x;  // a share of the requests' own results
#pragma unroll
    for (int k = 0; k < kEntries; k++) {
        const int32_t given = fits[k] ? grant(A, here, own[k], on_stack) : -1;
        if (given >= 0 && own[k].more != 0) most = (uint32_t)given + (uint32_t)own[k].more;
        starts[i0 + k] = clip31(here.tokens);
        taken[i0 + k] = given;
        lengths[i0 + k] = cached[k];
        if (reports && i0 + k < n) report_request(A, i0 + k, here.tokens, cached[k], fresh[k], given >= 0);
        here = here + own[k];
    }
    if (most != 0) atomicMax(&used, most);
    __syncthreads();
    const int32_t total = clip31(all.tokens);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        A.token_starts[n] = total;
        *A.free_left = on_stack - (int32_t)used;
    }
    const int64_t token0 = (int64_t)blockIdx.x * kWgTokens + threadIdx.x;
    int32_t token[kTokens];
    int at[kTokens];
#pragma unroll
    for (int k = 0; k < kTokens; k++) token[k] = (int32_t)min(token0 + k * kThreads, (int64_t)total - 1);
    search_together(starts, 0, n, token, at);
#pragma unroll
    for (int k = 0; k < kTokens; k++) {
        if (token0 + k * kThreads >= A.capacity) break;
        int64_t slot = -1;
        if (token0 + k * kThreads < total && taken[at[k]] >= 0)
            slot = slot_of(A, B, at[k], (uint32_t)lengths[at[k]], (uint32_t)(token[k] - starts[at[k]]), taken[at[k]], on_stack);
        A.slots[token0 + k * kThreads] = slot;
    }
}

uint32_t workgroups(int64_t capacity) { return capacity > kWgTokens ? (uint32_t)((capacity + kWgTokens - 1) / kWgTokens) : 1u; }

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
        capacity > 0x7FFFFFFF || (n_segments > 0 && !segments) || !seq_segments || (capacity > 0 && !positions) || !token_starts || !workspace ||
        (next && next == first) || token_starts == seq_segments || (const void *)token_starts == (const void *)first)
        return PREP_E_INVALID_ARG;
    if (!aligned(segments, 4) || !aligned(seq_segments, 4) || !aligned(first, 4) || !aligned(positions, 4) || !aligned(token_starts, 4) ||
        !aligned(next, 4) || !aligned(workspace, 16))
        return PREP_E_INVALID_ARG;
    if (workspace_bytes < prep_token_positions_workspace(n_segments)) return PREP_E_TOO_LARGE;
    DeviceScope scope(device);
    if (!scope.ok()) return PREP_E_HIP;
    const SegmentList L = {segments, seq_segments, first, n_segments, n_seq, merge, capacity, positions, token_starts, next};
    const dim3 grid(workgroups(capacity)), block(kThreads);
    const int32_t longest = n_segments > n_seq ? n_segments : n_seq;
    if (longest <= kThreads) {
        hipLaunchKernelGGL((place_listed<1>), grid, block, 0, stream, L);
    } else if (longest <= 4 * kThreads) {
        hipLaunchKernelGGL((place_listed<4>), grid, block, 0, stream, L);
    } else if (longest <= 8 * kThreads) {
        hipLaunchKernelGGL((place_listed<8>), grid, block, 0, stream, L);
    } else {
        int32_t *starts = static_cast<int32_t *>(workspace);
        uint32_t *moved = reinterpret_cast<uint32_t *>(starts + n_segments + 1);
        hipLaunchKernelGGL(sum_segments, dim3(1), block, 0, stream, L, starts, moved);
        hipLaunchKernelGGL(place_tokens, grid, block, 0, stream, L, (const int32_t *)starts, (const uint32_t *)moved);
    }
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
        (A.free_capacity > 0 && !A.free_blocks) || !A.free_count || !A.free_left || A.free_left == A.free_count ||
        (A.n > 0 && (A.lengths == A.cached || A.lengths == A.fresh || A.status == A.cached || A.status == A.fresh)) || !A.token_starts ||
        (A.capacity > 0 && !A.slots) || !A.workspace)
        return PREP_E_INVALID_ARG;
    if (!aligned(A.cached, 4) || !aligned(A.fresh, 4) || !aligned(A.free_blocks, 4) || !aligned(A.free_count, 4) || !aligned(A.table, 4) ||
        !aligned(A.slots, 8) || !aligned(A.token_starts, 4) || !aligned(A.lengths, 4) || !aligned(A.status, 4) || !aligned(A.free_left, 4) ||
        !aligned(A.workspace, 16))
        return PREP_E_INVALID_ARG;
    if (A.workspace_bytes < prep_block_slots_workspace(A.n)) return PREP_E_TOO_LARGE;
    DeviceScope scope(device);
    if (!scope.ok()) return PREP_E_HIP;
    BlockSize B = {(uint32_t)A.block_size, -1};
    for (int32_t s = 0; s <= 16; s++)
        if (A.block_size == 1 << s) B.shift = s;
    const dim3 grid(workgroups(A.capacity)), block(kThreads);
    if (A.n <= kThreads) {
        hipLaunchKernelGGL((place_slots_listed<1>), grid, block, 0, stream, A, B);
    } else if (A.n <= 4 * kThreads) {
        hipLaunchKernelGGL((place_slots_listed<4>), grid, block, 0, stream, A, B);
    } else if (A.n <= 8 * kThreads) {
        hipLaunchKernelGGL((place_slots_listed<8>), grid, block, 0, stream, A, B);
    } else {
        int32_t *starts = static_cast<int32_t *>(A.workspace), *taken = starts + A.n + 1;
        hipLaunchKernelGGL(sum_requests, dim3(1), block, 0, stream, A, B, starts, taken);
        if (A.capacity > 0) hipLaunchKernelGGL(place_slots, grid, block, 0, stream, A, B, (const int32_t *)starts, (const int32_t *)taken);
    }
    return hipGetLastError() == hipSuccess ? PREP_OK : PREP_E_HIP;
}

}  // extern "C"
