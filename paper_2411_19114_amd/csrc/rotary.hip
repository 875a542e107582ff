// Rotary embedding of queries and keys by places on up to three axes, with the store of keys and
// values into a paged cache (gfx950).
//
// A pair (a, b) of a head becomes (a cos u - b sin u, a sin u + b cos u) with u = place * f.  The angle is formed as a
// 64-bit fraction of a turn, place * (f / 2 pi * 2^64) modulo 2^64: the multiplication wraps exactly where
// the angle does, so a far place loses nothing, and the two top bits are the quadrant.
#include <hip/hip_runtime.h>
#include <cmath>
#include <stdint.h>

#include <new>

#include "../../include/prep.h"
#include "tokens.h"

struct prep_rotary {
    int32_t device, head_dim, pairs, dtype, pairing;
    uint64_t *d_turns;  // per pair: turns a place, as a fraction of 2^64, to the nearest multiple of four: the two lowest bits hold
                        // the axis (so it is off by 2^-63 of a turn at most, and 2^-32 at the farthest place)
};

namespace prep {

namespace {

constexpr int kThreads = 256;
constexpr int kTrig = 1024;  // angles of a workgroup
constexpr int kMaxTokens = 8;  // tokens of a workgroup

struct RotaryShape {
    int32_t head_dim, pairs;
    int32_t tokens;  // of a workgroup
    uint32_t block0;  // first workgroup of the launch
};

// cos and sin of a fraction of a turn.  Reduced to an eighth of a turn either side of a quadrant's middle
// axis; there Taylor's series up to x^9 and x^10 leave 2e-9 and 1.2e-10.  The angle is the sum of its upper 32 bits, rounded, and of the
// rest, with its sign, so that a small one (a slow pair's at a near place) has all the bits of a float.
__device__ __forceinline__ float2 cos_sin(uint64_t phase)
{
    const uint32_t turn = (uint32_t)((phase + 0x80000000ull) >> 32);
    const uint32_t quadrant = (turn + 0x20000000u) >> 30;
    const float x = fmaf((float)(int32_t)(turn - (quadrant << 30)), 4294967296.0f, (float)(int32_t)(uint32_t)phase) * 3.4061215800865545e-19f;  // 2 pi / 2^64
    const float z = x * x;
    const float s = x * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), 1.0f);
    const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
    const bool swap = (quadrant & 1u) != 0;
    const float a = swap ? s : c, b = swap ? c : s;
    float2 r;
    r.x = ((quadrant + 1u) & 2u) != 0 ? -a : a;
    r.y = (quadrant & 2u) != 0 ? -b : b;
    return r;
}

// Where the cache has token i's row, in elements, or -1.
__device__ __forceinline__ int64_t cache_row(const prep_rotary_args &A, int64_t i)
{
    const int64_t slot = A.slots[i];
    if (slot < 0 || slot >= A.n_blocks * A.block_size) return -1;
    // (a 64-bit division takes some 100 instructions, and hardly any cache has 2^32 slots)
    const int64_t block = slot <= 0xFFFFFFFF ? (int64_t)((uint32_t)slot / (uint32_t)A.block_size) : slot / A.block_size;
    return block * A.block_stride + (slot - block * A.block_size) * A.slot_stride;
}

// Any alignment and any number of pairs: one thread a pair, or a value behind the rotated ones.
template <typename T, bool kHalves>
__global__ __launch_bounds__(kThreads) void rotary_pairs(prep_rotary_args A, RotaryShape S, const uint64_t *__restrict__ turns)
{
    __shared__ float2 trig[kTrig];
    const int64_t token0 = (int64_t)(S.block0 + blockIdx.x) * S.tokens;
    const int n = (int)min((int64_t)S.tokens, A.n_tokens - token0);
    for (int e = threadIdx.x; e < n * S.pairs; e += kThreads) {
        const int t = e / S.pairs, p = e - t * S.pairs;
        const uint64_t f = turns[p];
        const int64_t place = A.positions[(int64_t)(f & 3u) * A.axis_stride + token0 + t];
        float2 cs = cos_sin((uint64_t)place * (f & ~(uint64_t)3));
        if (A.inverse) cs.y = -cs.y;
        trig[e] = cs;
    }
    __syncthreads();
    const bool store = A.k_cache != nullptr;
    const int units = S.head_dim - S.pairs;  // pairs, then single values
    const int heads = A.q_heads + A.k_heads * (store ? 2 : 1);
    for (int e = threadIdx.x; e < n * heads * units; e += kThreads) {
        const int row = e / units, u = e - row * units;
        const int t = row / heads, head = row - t * heads;
        const int64_t i = token0 + t;
        const bool paired = u < S.pairs;
        const int ia = paired && !kHalves ? 2 * u : paired ? u : u + S.pairs, ib = kHalves ? u + S.pairs : 2 * u + 1;
        const int of_k = head - A.q_heads, of_v = of_k - A.k_heads;
        const prep_heads &in = of_k < 0 ? A.q : of_v < 0 ? A.k : A.v;
        const int h = of_k < 0 ? head : of_v < 0 ? of_k : of_v;
        const T *src = (const T *)in.data + i * in.token_stride + (int64_t)h * in.head_stride;
        T a = src[ia], b = paired ? src[ib] : a;
        if (paired && of_v < 0) {
            const float2 cs = trig[t * S.pairs + u];
            const float x = to_float(a), y = to_float(b);
            a = from_float<T>(fmaf(x, cs.x, -y * cs.y));
            b = from_float<T>(fmaf(x, cs.y, y * cs.x));
        }
        if (of_v < 0) {
            const prep_heads &out = of_k < 0 ? A.q_out : A.k_out;
            if (out.data != nullptr) {
                T *dst = (T *)out.data + i * out.token_stride + (int64_t)h * out.head_stride;
                dst[ia] = a;
                if (paired) dst[ib] = b;
            }
        }
        if (store && of_k >= 0) {
            const int64_t at = cache_row(A, i);
            if (at >= 0) {
                T *dst = (T *)(of_v < 0 ? A.k_cache : A.v_cache) + at + (int64_t)h * A.cache_head_stride;
                dst[ia] = a;
                if (paired) dst[ib] = b;
            }
        }
    }
}

// Aligned rows.  A lane takes 32 bytes of a head's row in two loads of 16 (kHalves: values i.. and i + n.., whose pairs meet in
// the lane), always the same places of a row, and kRows rows whose loads go out together, before the
// angles are formed.  A token's angles are formed once per workgroup and shared by all its heads.  (All arguments take 256 bytes: with
// the call's number of rows among them, 264, 19321 tokens of 16 + 16 heads of 80 took 43.8 us where they take 42.3.)
struct RowShape {
    int32_t units;           // lanes of a row
    int32_t step;            // rows that a workgroup holds at a time
    int32_t heads;           // of q, k and (with a cache) v
    int32_t tokens;          // most of a workgroup
    int32_t head_dim, pairs;
    uint32_t block0;         // first workgroup of the launch
};

// Angles and tokens of a workgroup: 18 KB of LDS, which leaves a compute unit its eight workgroups.
constexpr int kMostAngles = 2048, kMostTokens = 256;

template <typename T>
union Vec {
    uint4 raw;
    T v[16 / sizeof(T)];
};

// 16 bytes; kStream: past the caches (launch_rows has the rule).
template <bool kStream>
__device__ __forceinline__ uint4 load16(const void *p)
{
    typedef uint32_t Four __attribute__((vector_size(16)));
    if (!kStream) return *static_cast<const uint4 *>(p);
    const Four v = __builtin_nontemporal_load(static_cast<const Four *>(p));
    return make_uint4(v[0], v[1], v[2], v[3]);
}
template <bool kStream>
__device__ __forceinline__ void store16(void *p, uint4 v)
{
    typedef uint32_t Four __attribute__((vector_size(16)));
    const Four f = {v.x, v.y, v.z, v.w};
    if (kStream) __builtin_nontemporal_store(f, static_cast<Four *>(p));
    else *static_cast<uint4 *>(p) = v;
}

// Bound by memory: 29 us for 8192 tokens of 28 + 4 heads of 128 in bf16 with the store into the cache (5.2 TB/s), 42 for 19321 of 16 + 16 heads
// of 80 in fp16 (4.7), 58 for 16384 of 32 + 8 heads of 64 in fp32, backwards (5.8, part of it from the last-level cache); a thread a pair takes 166, 191 and 146.
template <typename T, bool kHalves, int kRows, bool kStream>
__global__ __launch_bounds__(kThreads) void rotary_rows(prep_rotary_args A, RowShape S, const uint64_t *__restrict__ turns)
{
    constexpr int kV = 16 / (int)sizeof(T);
    __shared__ alignas(16) float cosine[kMostAngles], sine[kMostAngles];
    __shared__ int64_t place_in_cache[kMostTokens];

    const int64_t rows = A.n_tokens * S.heads;
    const int64_t row0 = (int64_t)(S.block0 + blockIdx.x) * (S.step * kRows);
    const int64_t token0 = rows <= 0xFFFFFFFF ? (int64_t)((uint32_t)row0 / (uint32_t)S.heads) : row0 / S.heads;
    const int head0 = (int)(row0 - token0 * S.heads);
    const int lane_row = (int)threadIdx.x / S.units, u = (int)threadIdx.x - lane_row * S.units;
    const bool works = lane_row < S.step;
    // the lane's places in a row
    const int rotated = 2 * S.pairs, rotary_units = S.pairs / kV;
    int at_a, at_b;
    if (kHalves) {
        const int tail = u - rotary_units;
        at_a = tail < 0 ? u * kV : rotated + 2 * tail * kV;
        at_b = tail < 0 ? u * kV + S.pairs : at_a + kV;
    } else {
        at_a = u * kV;
        at_b = (u + S.units) * kV;
    }
    const bool has_b = at_b < S.head_dim;
    const bool store = A.k_cache != nullptr;

    Vec<T> a[kRows], b[kRows];
    int token[kRows], head[kRows];  // of the rows; token -1: none
    {
        const int step_t = S.step / S.heads, step_h = S.step - step_t * S.heads;
        int t = (head0 + lane_row) / S.heads, h = head0 + lane_row - t * S.heads;
#pragma unroll
        for (int k = 0; k < kRows; k++) {
            const bool mine = works && row0 + lane_row + k * S.step < rows;
            token[k] = mine ? t : -1;
            head[k] = h;
            if (mine) {
                const int of_k = h - A.q_heads, of_v = of_k - A.k_heads;
                const T *base = (const T *)(of_k < 0 ? A.q.data : of_v < 0 ? A.k.data : A.v.data);
                const int64_t ts = of_k < 0 ? A.q.token_stride : of_v < 0 ? A.k.token_stride : A.v.token_stride;
                const int64_t hs = of_k < 0 ? A.q.head_stride : of_v < 0 ? A.k.head_stride : A.v.head_stride;
                const T *src = base + (token0 + t) * ts + (of_k < 0 ? h : of_v < 0 ? of_k : of_v) * hs;
                a[k].raw = load16<kStream>(src + at_a);
                if (has_b) b[k].raw = load16<kStream>(src + at_b);
            }
            t += step_t;
            h += step_h;
            if (h >= S.heads) {
                h -= S.heads;
                t++;
            }
        }
    }
    const int n = (int)min((int64_t)S.tokens, A.n_tokens - token0);
    for (int e = threadIdx.x; e < n * S.pairs; e += kThreads) {
        const int t = e / S.pairs, p = e - t * S.pairs;
        const uint64_t f = turns[p];
        const int64_t place = A.positions[(int64_t)(f & 3u) * A.axis_stride + token0 + t];
        const float2 cs = cos_sin((uint64_t)place * (f & ~(uint64_t)3));
        cosine[e] = cs.x;
        sine[e] = A.inverse ? -cs.y : cs.y;
    }
    if (store)
        for (int t = threadIdx.x; t < n; t += kThreads) place_in_cache[t] = cache_row(A, token0 + t);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kRows; k++) {
        if (token[k] < 0) continue;
        const int h = head[k], of_k = h - A.q_heads, of_v = of_k - A.k_heads;
        if (of_v < 0) {
            const float *c = cosine + token[k] * S.pairs, *s = sine + token[k] * S.pairs;
            if (kHalves) {
                if (u < rotary_units) {
#pragma unroll
                    for (int j = 0; j < kV; j++) {
                        const float x = to_float(a[k].v[j]), y = to_float(b[k].v[j]), cj = c[at_a + j], sj = s[at_a + j];
                        a[k].v[j] = from_float<T>(fmaf(x, cj, -y * sj));
                        b[k].v[j] = from_float<T>(fmaf(x, sj, y * cj));
                    }
                }
            } else {
#pragma unroll
                for (int half = 0; half < 2; half++) {
                    Vec<T> &w = half == 0 ? a[k] : b[k];
                    const int at = half == 0 ? at_a : at_b;
                    if (at < rotated) {
#pragma unroll
                        for (int j = 0; j < kV / 2; j++) {
                            const float x = to_float(w.v[2 * j]), y = to_float(w.v[2 * j + 1]), cj = c[at / 2 + j], sj = s[at / 2 + j];
                            w.v[2 * j] = from_float<T>(fmaf(x, cj, -y * sj));
                            w.v[2 * j + 1] = from_float<T>(fmaf(x, sj, y * cj));
                        }
                    }
                }
            }
            T *out = (T *)(of_k < 0 ? A.q_out.data : A.k_out.data);
            if (out != nullptr) {
                out += (token0 + token[k]) * (of_k < 0 ? A.q_out.token_stride : A.k_out.token_stride) +
                       (of_k < 0 ? h * A.q_out.head_stride : of_k * A.k_out.head_stride);
                store16<kStream>(out + at_a, a[k].raw);
                if (has_b) store16<kStream>(out + at_b, b[k].raw);
            }
        }
        if (store && of_k >= 0) {
            const int64_t at = place_in_cache[token[k]];
            if (at >= 0) {
                T *out = (T *)(of_v < 0 ? A.k_cache : A.v_cache) + at + (of_v < 0 ? of_k : of_v) * A.cache_head_stride;
                store16<kStream>(out + at_a, a[k].raw);
                if (has_b) store16<kStream>(out + at_b, b[k].raw);
            }
        }
    }
}

// Whether all rows of a call start at multiples of `bytes`.
bool rows_aligned(const prep_rotary &R, const prep_rotary_args &A, int64_t bytes)
{
    const int64_t v = bytes / element_bytes(R.dtype);
    auto fits = [&](const void *p, int64_t s, int64_t t) { return aligned(p, (uintptr_t)bytes) && s % v == 0 && t % v == 0; };
    auto rows = [&](const prep_heads &x) { return x.data == nullptr || fits(x.data, x.token_stride, x.head_stride); };
    if (A.q_heads > 0 && !(rows(A.q) && rows(A.q_out))) return false;
    if (A.k_heads > 0 && !(rows(A.k) && rows(A.k_out))) return false;
    if (A.k_cache != nullptr)
        return rows(A.v) && fits(A.k_cache, A.block_stride, A.slot_stride) && fits(A.v_cache, A.cache_head_stride, 0);
    return true;
}
// Whether all rows can be read and written 16 bytes at a time, pairs whole.
bool rows_in_16(const prep_rotary &R, const prep_rotary_args &A)
{
    const int64_t v = 16 / element_bytes(R.dtype);
    return R.head_dim % v == 0 && (R.pairing == PREP_PAIR_HALVES ? R.pairs : 2 * R.pairs) % v == 0 && rows_aligned(R, A, 16);
}

// Rows of a lane in large calls, from some two rounds of a full chip on.  Passes over fresh data, us, with 1, 2, 4, 8 rows: 8192
// tokens of 28 + 4 heads of 128 in bf16 into the cache 36, 34, 36, 39; 19321 of 16 + 16 of 80 in fp16 in a fused projection
// 43, 44, 49, 52; 16384 of 32 + 8 of 64 in fp32 63, 64, 67, 71.
constexpr int kManyRows = 2;

template <typename T, bool kHalves>
int launch_rows(const prep_rotary &R, const prep_rotary_args &A, hipStream_t stream)
{
    const int v = 16 / (int)sizeof(T);
    RowShape S;
    S.head_dim = R.head_dim;
    S.pairs = R.pairs;
    S.units = kHalves ? R.pairs / v + ((R.head_dim - 2 * R.pairs) / v + 1) / 2 : (R.head_dim / v + 1) / 2;
    S.heads = A.q_heads + A.k_heads * (A.k_cache != nullptr ? 2 : 1);
    const int64_t rows = A.n_tokens * S.heads;
    S.step = kThreads / S.units;
    auto tokens_of = [&](int n) { return (n + S.heads - 2) / S.heads + 1; };
    int per_lane = rows >= (int64_t)S.step * kManyRows * 512 ? kManyRows : 1;
    auto fit = [&](int n) { return tokens_of(n) <= kMostTokens && tokens_of(n) * S.pairs <= kMostAngles; };
    if (!fit(S.step * per_lane)) per_lane = 1;
    while (S.step > 1 && !fit(S.step)) S.step--;  // (one row is of one token, and a head has at most 512 pairs)
    S.tokens = tokens_of(S.step * per_lane);
    const int64_t blocks = (rows + S.step * per_lane - 1) / (S.step * per_lane);
    if (blocks > 0x7FFFFFFF) return PREP_E_TOO_LARGE;
    // Past the caches where what a load takes of a row is whole 128-byte lines: then 34 -> 30 us and 64 -> 58 us (the first and the last
    // of the calls above), 35 -> 29 for rows of 256 in bf16; pieces of 64 bytes 34 -> 34, of 80 and 96 bytes 44 -> 55 and 35 -> 39.
    // Who reads the outputs at once does not lose by it: with a copy of q and of the caches behind the first call both take 73.5 -> 72, with one of the
    // outputs behind the last 143 -> 129, the copies alone 43 and 71.
    const bool lines = S.units * 16 % 128 == 0 && rows_aligned(R, A, 128);
    in_launches((uint32_t)blocks, kThreads, [&](uint32_t first, uint32_t n) {
        const dim3 grid(n);
        S.block0 = first;
        if (per_lane == 1)
            hipLaunchKernelGGL((rotary_rows<T, kHalves, 1, false>), grid, dim3(kThreads), 0, stream, A, S, (const uint64_t *)R.d_turns);
        else if (!lines)
            hipLaunchKernelGGL((rotary_rows<T, kHalves, kManyRows, false>), grid, dim3(kThreads), 0, stream, A, S, (const uint64_t *)R.d_turns);
        else
            hipLaunchKernelGGL((rotary_rows<T, kHalves, kManyRows, true>), grid, dim3(kThreads), 0, stream, A, S, (const uint64_t *)R.d_turns);
    });
    return PREP_OK;
}

template <typename T>
int launch_for(const prep_rotary &R, const prep_rotary_args &A, hipStream_t stream)
{
    const bool halves = R.pairing == PREP_PAIR_HALVES;
    if (rows_in_16(R, A)) return halves ? launch_rows<T, true>(R, A, stream) : launch_rows<T, false>(R, A, stream);
    RotaryShape S;
    S.head_dim = R.head_dim;
    S.pairs = R.pairs;
    S.tokens = kTrig / R.pairs < kMaxTokens ? kTrig / R.pairs : kMaxTokens;
    const int64_t blocks = (A.n_tokens + S.tokens - 1) / S.tokens;
    if (blocks > 0x7FFFFFFF) return PREP_E_TOO_LARGE;
    in_launches((uint32_t)blocks, kThreads, [&](uint32_t first, uint32_t n) {
        const dim3 grid(n);
        S.block0 = first;
        if (halves)
            hipLaunchKernelGGL((rotary_pairs<T, true>), grid, dim3(kThreads), 0, stream, A, S, (const uint64_t *)R.d_turns);
        else
            hipLaunchKernelGGL((rotary_pairs<T, false>), grid, dim3(kThreads), 0, stream, A, S, (const uint64_t *)R.d_turns);
    });
    return PREP_OK;
}

// Rows of head_dim elements, n[a] of them stride[a] apart along each of the axes, lie apart from one another.
bool distinct_rows(int64_t head_dim, const int64_t *stride, const int64_t *n, int axes)
{
    int64_t span = head_dim;  // of the axes taken so far
    bool used[3] = {false, false, false};
    for (int step = 0; step < axes; step++) {
        int best = -1;
        for (int a = 0; a < axes; a++)
            if (!used[a] && (best < 0 || stride[a] < stride[best])) best = a;
        used[best] = true;
        if (n[best] <= 1) continue;
        if (stride[best] < span) return false;
        if (stride[best] > (INT64_MAX >> 4) / n[best]) return false;
        span += stride[best] * (n[best] - 1);
    }
    return true;
}

}  // namespace

}  // namespace prep

using namespace prep;

extern "C" {

int prep_rotary_create(prep_rotary **out, const prep_rotary_config *cfg)
{
    if (!out) return PREP_E_INVALID_ARG;
    *out = nullptr;
    if (!cfg || cfg->head_dim < 2 || cfg->head_dim > 1024 || !float_type(cfg->dtype) || cfg->reserved != 0 ||
        (cfg->pairing != PREP_PAIR_HALVES && cfg->pairing != PREP_PAIR_ADJACENT) ||
        (cfg->order != PREP_SECTIONS_BLOCKS && cfg->order != PREP_SECTIONS_INTERLEAVED) || (cfg->flags & ~(uint32_t)PREP_ROTARY_PER_AXIS) != 0)
        return PREP_E_INVALID_ARG;
    int32_t n = 0;
    for (int a = 0; a < 3; a++) {
        if (cfg->sections[a] < 0 || cfg->sections[a] > 512) return PREP_E_INVALID_ARG;
        n += cfg->sections[a];
    }
    if (n < 1 || n > cfg->head_dim / 2) return PREP_E_INVALID_ARG;
    if (!cfg->frequencies && !(cfg->base > 0.0 && std::isfinite(cfg->base))) return PREP_E_INVALID_ARG;
    uint64_t turns[512];
    int32_t seen[3] = {0, 0, 0};
    for (int32_t i = 0; i < n; i++) {
        int axis;
        if (cfg->order == PREP_SECTIONS_BLOCKS)
            axis = i < cfg->sections[0] ? 0 : i < cfg->sections[0] + cfg->sections[1] ? 1 : 2;
        else
            axis = i % 3 != 0 && i < 3 * cfg->sections[i % 3] ? i % 3 : 0;
        long double f;
        if (cfg->frequencies) {
            if (!std::isfinite(cfg->frequencies[i])) return PREP_E_INVALID_ARG;
            f = cfg->frequencies[i];
        } else if (cfg->flags & PREP_ROTARY_PER_AXIS) {
            f = cfg->sections[axis] == 0 ? 0.0L : powl((long double)cfg->base, -(long double)seen[axis] / (long double)cfg->sections[axis]);
        } else {
            f = powl((long double)cfg->base, -(long double)i / (long double)n);
        }
        seen[axis]++;
        long double t = f / (2.0L * acosl(-1.0L));
        if (!(t > -1e15L && t < 1e15L)) return PREP_E_INVALID_ARG;
        t -= floorl(t);
        // to the nearest multiple of four (two bits are the axis'); a fraction that rounds up to a whole turn is none
        const long double quarter = floorl(t * 4611686018427387904.0L + 0.5L);
        const uint64_t q = quarter >= 4611686018427387904.0L ? 0 : (uint64_t)quarter;
        turns[i] = (q << 2) | (uint64_t)axis;
    }
    for (int a = 0; a < 3; a++)
        if (seen[a] != cfg->sections[a]) return PREP_E_INVALID_ARG;
    int ndev = 0;
    if (hipGetDeviceCount(&ndev) != hipSuccess || cfg->device < 0 || cfg->device >= ndev) {
        (void)hipGetLastError();
        return PREP_E_HIP;
    }
    DeviceScope scope(cfg->device);
    if (!scope.ok()) return PREP_E_HIP;
    prep_rotary *r = new (std::nothrow) prep_rotary;
    if (!r) return PREP_E_NOMEM;
    *r = prep_rotary{cfg->device, cfg->head_dim, n, cfg->dtype, cfg->pairing, nullptr};
    if (hipMalloc((void **)&r->d_turns, sizeof(uint64_t) * (size_t)n) != hipSuccess ||
        hipMemcpy(r->d_turns, turns, sizeof(uint64_t) * (size_t)n, hipMemcpyHostToDevice) != hipSuccess) {
        (void)hipGetLastError();
        (void)hipFree(r->d_turns);
        delete r;
        return PREP_E_NOMEM;
    }
    *out = r;
    return PREP_OK;
}

int prep_rotary_destroy(prep_rotary *r)
{
    if (!r) return PREP_E_INVALID_ARG;
    {
        DeviceScope scope(r->device);
        (void)hipDeviceSynchronize();
        (void)hipFree(r->d_turns);
        (void)hipGetLastError();
    }
    delete r;
    return PREP_OK;
}

static_assert(sizeof(prep_rotary_args) == 216, "as the binding packs it");

int prep_rotary_apply(prep_rotary *r, const prep_rotary_args *args, void *stream_ptr)
{
    hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
    if (!r || !args) return PREP_E_INVALID_ARG;
    prep_rotary_args A = *args;
    if (A.n_tokens < 0 || A.n_tokens > 0x7FFFFFFF || A.q_heads < 0 || A.k_heads < 0 || A.q_heads > 65535 || A.k_heads > 65535 || A.q_heads + A.k_heads == 0 ||
        A.axis_stride < 0 || (A.inverse != 0 && A.inverse != 1))
        return PREP_E_INVALID_ARG;
    const bool store = A.k_cache != nullptr;
    if (store != (A.v_cache != nullptr)) return PREP_E_INVALID_ARG;
    if (A.n_tokens == 0) return PREP_OK;
    const uintptr_t size = (uintptr_t)element_bytes(r->dtype);
    auto input = [&](const prep_heads &x) { return x.data && aligned(x.data, size) && x.token_stride >= 0 && x.head_stride >= 0; };
    auto output = [&](const prep_heads &x, const prep_heads &from, int64_t heads) {
        const int64_t stride[2] = {x.token_stride, x.head_stride}, n[2] = {A.n_tokens, heads};
        if (!input(x) || !distinct_rows(r->head_dim, stride, n, 2)) return false;
        // in place: every value goes back where it came from
        return x.data != from.data || ((A.n_tokens == 1 || x.token_stride == from.token_stride) && (heads == 1 || x.head_stride == from.head_stride));
    };
    if (!A.positions || !aligned(A.positions, 4)) return PREP_E_INVALID_ARG;
    if (A.q_heads > 0 && (!input(A.q) || !output(A.q_out, A.q, A.q_heads))) return PREP_E_INVALID_ARG;
    if (A.k_heads > 0) {
        if (!input(A.k)) return PREP_E_INVALID_ARG;
        if (!(store && !A.k_out.data) && !output(A.k_out, A.k, A.k_heads)) return PREP_E_INVALID_ARG;
    }
    if (store) {
        if (A.k_heads == 0 || !input(A.v) || !A.slots || !aligned(A.slots, 8) || A.block_size < 1 || A.n_blocks < 0 || A.n_blocks > 0x7FFFFFFF ||
            A.k_cache == A.v_cache || !aligned(A.k_cache, size) || !aligned(A.v_cache, size))
            return PREP_E_INVALID_ARG;
        const int64_t stride[3] = {A.block_stride, A.slot_stride, A.cache_head_stride}, n[3] = {A.n_blocks, A.block_size, A.k_heads};
        for (int64_t s : stride)
            if (s < 0) return PREP_E_INVALID_ARG;
        if (!distinct_rows(r->head_dim, stride, n, 3)) return PREP_E_INVALID_ARG;
    }
    DeviceScope scope(r->device);
    if (!scope.ok()) return PREP_E_HIP;
    const int rc = r->dtype == PREP_F32   ? launch_for<float>(*r, A, stream)
                   : r->dtype == PREP_F16 ? launch_for<__half>(*r, A, stream)
                                          : launch_for<__hip_bfloat16>(*r, A, stream);
    if (rc != PREP_OK) return rc;
    return hipGetLastError() == hipSuccess ? PREP_OK : PREP_E_HIP;
}

}  // extern "C"
