// dq8 kernels: plan of a decoding step (slots, positions, pages) and verification of drafted tokens.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

constexpr uint32_t kPlanWg = 1024, kPlanMost = 4096;  // lanes of the plan's workgroup, sequences at most
constexpr uint32_t kRun = kPlanMost / kPlanWg;         // sequences of a lane, at most

// Sums over the lanes up to and with each.
template <typename T>
__device__ __forceinline__ T scan_wave(T v, uint32_t lane)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const T o = __shfl_up(v, d);
        if (lane >= (uint32_t)d) v += o;
    }
    return v;
}

// Sums over the lanes before each in a workgroup of WAVES wavefronts; all: the sum of everything.  `spare` is LDS of WAVES numbers.
template <int WAVES, typename T>
__device__ __forceinline__ T sum_before(T v, T *spare, T &all)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v = scan_wave(v, lane);
    __syncthreads();
    if (lane == 63) spare[wave] = v;
    __syncthreads();
    v = __shfl_up(v, 1);
    if (lane == 0) v = 0;
    T before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const T o = spare[w];
        if ((uint32_t)w < wave) before += o;
        all += o;
    }
    return v + before;
}

// How many of the n ascending numbers are <= v.
__device__ __forceinline__ uint32_t not_above(const uint32_t *p, uint32_t n, uint32_t v)
{
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (p[mid] <= v)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

// ---------------------------------------------------------------- plan

struct PlanArgs {
    const int32_t *lens, *new_tokens, *drop;
    int32_t *pages, *free_pages;
    const int32_t *n_free;
    int64_t *slots, *positions;
    int32_t *starts, *lens_out, *granted, *n_free_out;
    uint32_t batch, max_pages, tokens, capacity, page_shift;
    int finish;  // whether k_cache_plan writes slots and positions too
};

// What a sequence asks for.
struct Request {
    uint32_t len, kept;  // cached tokens before, and without what is dropped
    uint32_t more;       // new tokens
};

__device__ __forceinline__ Request request_of(const PlanArgs &a, uint32_t b)
{
    const int32_t len = a.lens[b], more = a.new_tokens[b], drop = a.drop ? a.drop[b] : 0;
    const uint32_t most = a.max_pages << a.page_shift;
    Request r;
    r.len = len < 0 ? 0 : (uint32_t)len < most ? (uint32_t)len : most;
    r.kept = drop <= 0 ? r.len : (uint32_t)drop < r.len ? r.len - (uint32_t)drop : 0;
    r.more = more < 0 ? 0 : (uint32_t)more;
    return r;
}

__device__ __forceinline__ uint32_t pages_of(const PlanArgs &a, uint32_t tokens) { return (tokens + (1u << a.page_shift) - 1) >> a.page_shift; }

// Token i of the step: its sequence is the first whose end is behind it.
__device__ __forceinline__ void place_token(const PlanArgs &a, uint32_t i, const uint32_t *ends, const int32_t *lens, bool ok_by_len)
{
    int64_t slot = -1, position = -1;
    const uint32_t b = not_above(ends, a.batch, i);
    if (b < a.batch) {
        const int32_t len = ok_by_len ? lens[b] : a.granted[b] < 0 ? -1 : lens[b];
        if (len >= 0) {
            const uint32_t p = (uint32_t)len - (ends[b] - i);
            position = p;
            slot = ((int64_t)a.pages[(size_t)b * a.max_pages + (p >> a.page_shift)] << a.page_shift) + (p & ((1u << a.page_shift) - 1));
        }
    }
    a.slots[i] = slot;
    a.positions[i] = position;
}

// One workgroup: three sums over the sequences (new tokens; pages given back and taken), then the pages that move, one lane each whatever
// sequence they belong to.
__global__ __launch_bounds__(kPlanWg) void k_cache_plan(PlanArgs a)
{
    __shared__ uint32_t ends[kPlanMost], gone_upto[kPlanMost], need_upto[kPlanMost], had_pages[kPlanMost];
    __shared__ int32_t lens[kPlanMost];  // after the step, -1 for refused sequences
    __shared__ uint64_t spare[kPlanWg / 64];
    __shared__ uint32_t taken_all;
    const uint32_t t = threadIdx.x, run = (a.batch + kPlanWg - 1) / kPlanWg, b0 = t * run;
    if (t == 0) taken_all = 0;
    const int32_t valid = *a.n_free;
    const uint32_t have = valid < 0 ? 0 : (uint32_t)valid < a.capacity ? (uint32_t)valid : a.capacity;

    Request r[kRun];
    uint64_t mine = 0;
#pragma unroll
    for (uint32_t i = 0; i < kRun; ++i) {
        r[i] = Request{0, 0, 0};
        if (i < run && b0 + i < a.batch) r[i] = request_of(a, b0 + i);
        mine += r[i].more;
    }
    uint64_t all;
    uint64_t before = sum_before<kPlanWg / 64>(mine, spare, all);
    bool fits[kRun];
    uint64_t moved = 0;  // pages given back, in the upper half pages taken
    const uint32_t most = a.max_pages << a.page_shift;
#pragma unroll
    for (uint32_t i = 0; i < kRun; ++i) {
        const uint32_t b = b0 + i;
        fits[i] = false;
        if (i >= run || b >= a.batch) continue;
        before += r[i].more;
        fits[i] = r[i].more <= most - r[i].kept && before <= a.tokens;
        ends[b] = before < a.tokens ? (uint32_t)before : a.tokens;
        a.starts[b + 1] = (int32_t)ends[b];
        const uint32_t had = pages_of(a, r[i].len), wanted = fits[i] ? pages_of(a, r[i].kept + r[i].more) : had;
        had_pages[b] = had;
        moved += had > wanted ? (uint64_t)(had - wanted) : (uint64_t)(wanted - had) << 32;
    }
    if (t == 0) a.starts[0] = 0;
    uint64_t upto = sum_before<kPlanWg / 64>(moved, spare, all);
    const uint32_t back = (uint32_t)all, room = a.capacity - have, stock = have + (back < room ? back : room);
    uint32_t taken = 0;
#pragma unroll
    for (uint32_t i = 0; i < kRun; ++i) {
        const uint32_t b = b0 + i;
        if (i >= run || b >= a.batch) continue;
        const uint32_t had = had_pages[b], wanted = fits[i] ? pages_of(a, r[i].kept + r[i].more) : had;
        upto += had > wanted ? (uint64_t)(had - wanted) : (uint64_t)(wanted - had) << 32;
        gone_upto[b] = (uint32_t)upto;
        need_upto[b] = (uint32_t)(upto >> 32);
        const bool ok = fits[i] && (wanted <= had || need_upto[b] <= stock);
        if (ok && wanted > had) taken = need_upto[b];
        const int32_t len = (int32_t)(ok ? r[i].kept + r[i].more : r[i].len);
        a.lens_out[b] = len;
        a.granted[b] = ok ? (int32_t)r[i].more : -1;
        lens[b] = ok ? len : -1;
    }
    if (taken) atomicMax(&taken_all, taken);
    __syncthreads();
    for (uint32_t i = t; i < stock - have; i += kPlanWg) {
        const uint32_t b = not_above(gone_upto, a.batch, i), count = gone_upto[b] - (b ? gone_upto[b - 1] : 0);
        const uint32_t page = had_pages[b] - count + (i - (b ? gone_upto[b - 1] : 0));
        a.free_pages[have + i] = a.pages[(size_t)b * a.max_pages + page];
    }
    __syncthreads();
    const uint32_t take = taken_all;
    for (uint32_t i = t; i < take; i += kPlanWg) {
        const uint32_t b = not_above(need_upto, a.batch, i);
        a.pages[(size_t)b * a.max_pages + had_pages[b] + (i - (b ? need_upto[b - 1] : 0))] = a.free_pages[stock - 1 - i];
    }
    if (t == 0) *a.n_free_out = (int32_t)(stock - take);
    if (!a.finish) return;
    __syncthreads();
    for (uint32_t i = t; i < a.tokens; i += kPlanWg) place_token(a, i, ends, lens, true);
}

// Slots and positions of many tokens, behind k_cache_plan.
constexpr uint32_t kPlaceWg = 256, kPlacePer = 4;

__global__ __launch_bounds__(kPlaceWg) void k_cache_place(PlanArgs a)
{
    __shared__ uint32_t ends[kPlanMost];
    for (uint32_t b = threadIdx.x; b < a.batch; b += kPlaceWg) ends[b] = (uint32_t)a.starts[b + 1];
    __syncthreads();
#pragma unroll
    for (uint32_t k = 0; k < kPlacePer; ++k) {
        const uint32_t i = (blockIdx.x * kPlacePer + k) * kPlaceWg + threadIdx.x;
        if (i < a.tokens) place_token(a, i, ends, a.lens_out, false);
    }
}

// ---------------------------------------------------------------- verification

struct VerifyArgs {
    const void *target, *draft;
    size_t target_stride, draft_stride;
    const int64_t *ids;
    const float *uniform, *sample;
    const int32_t *starts;
    int64_t *out;
    int32_t *accepted, *rejected;
    uint32_t tokens, batch, each, vocab;
    uint32_t chunk, chunks;  // probabilities that a wavefront adds up, and how many such
    double2 *sums;           // workspace [batch][chunks]: of the weights, and of the target alone (null: there is none)
};

// A probability: what is no positive number counts as none.
template <typename T>
__device__ __forceinline__ float probability(T v)
{
    const float f = (float)v;
    return f > 0.0f && f < __builtin_inff() ? f : 0.0f;
}

// Where a sequence ends: rows first .. first + n - 1, `row` of them accepted; refused: whether row `row` refused its draft `token`.
struct Verdict {
    uint32_t first, n, row;
    bool refused;
    int64_t token;
};

// Every wavefront that needs it finds it by itself: a lane per draft.
template <typename T>
__device__ __forceinline__ Verdict verdict_of(const VerifyArgs &a, uint32_t b)
{
    const uint32_t lane = threadIdx.x & 63;
    Verdict v;
    uint32_t end;
    if (a.starts) {
        const int32_t s0 = a.starts[b], s1 = a.starts[b + 1];
        v.first = s0 < 0 ? 0 : (uint32_t)s0 < a.tokens ? (uint32_t)s0 : a.tokens;
        end = s1 < 0 ? 0 : (uint32_t)s1 < a.tokens ? (uint32_t)s1 : a.tokens;
        if (end < v.first) end = v.first;
    } else {
        v.first = b * a.each;
        end = v.first + a.each;
    }
    v.n = end - v.first;
    v.row = v.n ? v.n - 1 : 0;
    v.refused = false;
    v.token = -1;
    for (uint32_t i0 = 0; i0 + 1 < v.n; i0 += 64) {
        const uint32_t i = i0 + lane;
        bool no = false;
        int64_t d = -1;
        if (i + 1 < v.n) {
            const size_t row = v.first + i;
            d = a.ids[row + 1];
            no = true;
            if (d >= 0 && d < (int64_t)a.vocab) {
                const double p = probability(static_cast<const T *>(a.target)[row * a.target_stride + d]);
                const double q = a.draft ? probability(static_cast<const T *>(a.draft)[row * a.draft_stride + d]) : 1.0f;
                no = !((double)a.uniform[row] * q < p);  // 24 times 24 bits: exact
            }
        }
        const uint64_t votes = __builtin_amdgcn_ballot_w64(no);
        if (votes) {
            const int l = __builtin_ctzll(votes);
            v.row = i0 + (uint32_t)l;
            v.refused = true;
            v.token = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(d >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)d, l));
            break;
        }
    }
    return v;
}

// The row from which a sequence's token is drawn.
template <typename T>
struct Row {
    const T *p, *q;  // q: what is taken off (null: nothing)
    int64_t less;    // the token that has no weight (-1: all have theirs)

    __device__ __forceinline__ Row(const VerifyArgs &a, const Verdict &v)
    {
        const size_t row = v.first + v.row;
        p = static_cast<const T *>(a.target) + row * a.target_stride;
        q = v.refused && a.draft ? static_cast<const T *>(a.draft) + row * a.draft_stride : nullptr;
        less = v.refused && !a.draft ? v.token : -1;
    }

    __device__ __forceinline__ double weight(float pt, float qt, uint32_t t) const
    {
        const double w = (double)pt - (double)qt;
        return (int64_t)t == less || !(w > 0.0) ? 0.0 : w;
    }
};

__device__ __forceinline__ double sum_wave(double v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    return v;
}

// A wavefront's sums over a chunk: of the weights and of the target's probabilities alone.
template <typename T>
__device__ __forceinline__ double2 sum_chunk(const VerifyArgs &a, const Row<T> &row, uint32_t c)
{
    typedef T V __attribute__((ext_vector_type(4)));
    typedef V VA __attribute__((aligned(sizeof(T))));
    const uint32_t lane = threadIdx.x & 63, begin = c * a.chunk, end = a.vocab - begin < a.chunk ? a.vocab : begin + a.chunk;
    double w = 0.0, all = 0.0;
#pragma unroll 4
    for (uint32_t t = begin + 4 * lane; t < end; t += 256) {
        V p = {}, q = {};
        if (t + 4 <= end) {
            p = *reinterpret_cast<const VA *>(row.p + t);
            if (row.q) q = *reinterpret_cast<const VA *>(row.q + t);
        } else {
            for (int e = 0; e < 4; ++e)
                if (t + e < end) {
                    p[e] = row.p[t + e];
                    if (row.q) q[e] = row.q[t + e];
                }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float f = probability(p[e]);
            w += row.weight(f, probability(q[e]), t + e);
            all += f;
        }
    }
    return double2{sum_wave(w), sum_wave(all)};
}

constexpr uint32_t kVerifyWg = 256, kVerifyWaves = kVerifyWg / 64, kChunksMost = 2048, kChunk = 1024;

template <typename T>
__global__ __launch_bounds__(kVerifyWg) void k_verify_sums(VerifyArgs a)
{
    const uint32_t b = blockIdx.y, c = blockIdx.x * kVerifyWaves + (threadIdx.x >> 6);
    if (c >= a.chunks) return;
    const Verdict v = verdict_of<T>(a, b);
    if (v.n == 0) return;
    const double2 s = sum_chunk(a, Row<T>(a, v), c);
    if ((threadIdx.x & 63) == 0) a.sums[(size_t)b * a.chunks + c] = s;
}

// One workgroup per sequence: the chunk in which the sum passes its mark, then the token in it.
template <typename T>
__global__ __launch_bounds__(kVerifyWg) void k_verify_pick(VerifyArgs a)
{
    __shared__ double2 sums[kChunksMost];
    __shared__ double spare[kVerifyWaves];
    __shared__ uint32_t found, last;
    const uint32_t b = blockIdx.x, t = threadIdx.x, lane = t & 63;
    const Verdict v = verdict_of<T>(a, b);
    if (t == 0) {
        a.accepted[b] = v.n ? (int32_t)v.row : -1;
        a.rejected[b] = v.n ? (int32_t)(v.n - 1 - v.row) : 0;
    }
    if (v.n == 0) return;
    const Row<T> row(a, v);
    if (a.sums) {
        for (uint32_t c = t; c < a.chunks; c += kVerifyWg) sums[c] = a.sums[(size_t)b * a.chunks + c];
    } else {
        for (uint32_t c = t >> 6; c < a.chunks; c += kVerifyWaves) {
            const double2 s = sum_chunk(a, row, c);
            if (lane == 0) sums[c] = s;
        }
    }
    if (t == 0) {
        found = 0xFFFFFFFFu;
        last = 0;
    }
    __syncthreads();
    // a lane has a run of chunks
    const uint32_t run = (a.chunks + kVerifyWg - 1) / kVerifyWg, c0 = t * run < a.chunks ? t * run : a.chunks, c1 = c0 + run < a.chunks ? c0 + run : a.chunks;
    double w = 0.0, all = 0.0, total, total_all;
    for (uint32_t c = c0; c < c1; ++c) {
        w += sums[c].x;
        all += sums[c].y;
    }
    const double before = sum_before<kVerifyWaves>(w, spare, total), before_all = sum_before<kVerifyWaves>(all, spare, total_all);
    const bool plain = !(total > 0.0);  // the target's own
    if (plain) total = total_all;
    const float r = a.sample[b];
    const double mark = (r > 0.0f ? (double)r : 0.0) * total;
    // the first chunk that passes the mark, else the last with a weight
    double sum = plain ? before_all : before;
    for (uint32_t c = c0; c < c1; ++c) {
        const double s = plain ? sums[c].y : sums[c].x, next = sum + s;
        if (s > 0.0) {
            atomicMax(&last, c);
            if (next > mark) {
                atomicMin(&found, c);
                break;
            }
        }
        sum = next;
    }
    __syncthreads();
    int64_t token = -1;
    if (total > 0.0) {
        const uint32_t c = found != 0xFFFFFFFFu ? found : last;
        __syncthreads();
        if (t == 0) found = 0xFFFFFFFFu, last = 0;
        // the sum before it, as that lane has it
        if (c >= c0 && c < c1) {
            double s = plain ? before_all : before;
            for (uint32_t k = c0; k < c; ++k) s += plain ? sums[k].y : sums[k].x;
            spare[0] = s;
        }
        __syncthreads();
        double base = spare[0];
        const uint32_t begin = c * a.chunk, end = a.vocab - begin < a.chunk ? a.vocab : begin + a.chunk;
        for (uint32_t i0 = begin; i0 < end; i0 += kVerifyWg * 4) {
            double x[4], mine = 0.0, some;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t i = i0 + 4 * t + e;
                x[e] = 0.0;
                if (i < end) {
                    const float p = probability(row.p[i]);
                    x[e] = plain ? (double)p : row.weight(p, row.q ? probability(row.q[i]) : 0.0f, i);
                }
                mine += x[e];
            }
            double s = base + sum_before<kVerifyWaves>(mine, spare, some);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s += x[e];
                if (x[e] > 0.0) {
                    atomicMax(&last, i0 + 4 * t + e);
                    if (s > mark) atomicMin(&found, i0 + 4 * t + e);
                }
            }
            __syncthreads();
            if (found != 0xFFFFFFFFu) break;
            base += some;
        }
        token = found != 0xFFFFFFFFu ? found : last;
    }
    for (uint32_t i = t; i < v.n; i += kVerifyWg) a.out[v.first + i] = i < v.row ? a.ids[v.first + i + 1] : i == v.row ? token : -1;
}

}  // namespace
