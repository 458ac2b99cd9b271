// dq8 kernels: plan of a decoding step (slots, positions, pages) and verification of drafted tokens.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

constexpr uint32_t kPlanWg = 1024, kPlanMost = 4096;  // lanes of the plan's workgroup, sequences at most
constexpr uint32_t kRun = kPlanMost / kPlanWg;         // sequences of a lane, at most

// A number of another lane (data-parallel primitives: no LDS, 8 cycles; a shuffle takes a hundred), zero where the pattern has none for a lane.
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T from_lane(T v)
{
    if constexpr (sizeof(T) == 8) {
        uint64_t u;
        __builtin_memcpy(&u, &v, 8);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, CTRL, ROWS, 0xF, false);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, ROWS, 0xF, false);
        u = (uint64_t)hi << 32 | lo;
        __builtin_memcpy(&v, &u, 8);
        return v;
    } else {
        return (T)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
    }
}

// Sums over the lanes up to and with each: 1, 2, 4, 8 lanes back inside rows of 16, then lane 15 of a row into the next and lane 31 into the upper half.
template <typename T>
__device__ __forceinline__ T scan_wave(T v)
{
    v += from_lane<0x111, 0xF>(v);
    v += from_lane<0x112, 0xF>(v);
    v += from_lane<0x114, 0xF>(v);
    v += from_lane<0x118, 0xF>(v);
    v += from_lane<0x142, 0xA>(v);
    v += from_lane<0x143, 0xC>(v);
    return v;
}

// A lane's wavefront, in a scalar register.
__device__ __forceinline__ uint32_t wave_of(uint32_t thread) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)(thread >> 6)); }

// The number of a lane that is the same for all.
template <typename T>
__device__ __forceinline__ T of_lane(T v, int lane)
{
    uint64_t all = 0;
    __builtin_memcpy(&all, &v, sizeof(T));
    uint64_t u = (uint32_t)__builtin_amdgcn_readlane((int)all, lane);
    if constexpr (sizeof(T) == 8) u |= (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(all >> 32), lane) << 32;
    __builtin_memcpy(&v, &u, sizeof(T));
    return v;
}

// The number of the lane before (zero for the first).
template <typename T>
__device__ __forceinline__ T before_lane(T v)
{
    return from_lane<0x138, 0xF>(v);
}

// Sums over the lanes before each in a workgroup of WAVES wavefronts; all: the sum of everything.  `spare` is LDS of WAVES numbers.
template <int WAVES, typename T>
__device__ __forceinline__ T sum_before(T v, T *spare, T &all)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T upto = scan_wave(v);
    __syncthreads();
    if (lane == 63) spare[wave] = upto;
    __syncthreads();
    v = before_lane(upto);
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

// Tokens i0, i0 + step .. of the step, N of them at once: their searches and loads run side by side.  A token's sequence is the first whose end is behind it.
// len(b): its length after the step, -1 where it is refused.
template <int N, typename F>
__device__ __forceinline__ void place_tokens(const PlanArgs &a, uint32_t i0, uint32_t step, const uint32_t *ends, F len)
{
    uint32_t b[N];
#pragma unroll
    for (int k = 0; k < N; ++k) b[k] = 0;
    for (uint32_t s = 1u << (31 - __builtin_clz(a.batch)); s != 0; s >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint32_t at = b[k] + s;
            if (at <= a.batch && ends[at - 1] <= i0 + k * step) b[k] = at;
        }
    int64_t position[N];
    int32_t page[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t c = b[k] < a.batch ? b[k] : a.batch - 1;
        const int32_t n = len(c);
        const bool there = b[k] < a.batch && n >= 0;
        position[k] = there ? (int64_t)n - (ends[c] - (i0 + k * step)) : -1;
        page[k] = a.pages[(size_t)c * a.max_pages + (there ? (uint32_t)position[k] >> a.page_shift : 0)];
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t i = i0 + k * step;
        if (i >= a.tokens) continue;
        a.slots[i] = position[k] < 0 ? -1 : ((int64_t)page[k] << a.page_shift) + (position[k] & ((1u << a.page_shift) - 1));
        a.positions[i] = position[k];
    }
}

// One workgroup: three sums over the sequences (new tokens; pages given back and taken), then the pages that move, one lane each whatever
// sequence they belong to, then slots and positions of up to a few thousand tokens.  256 sequences of five new tokens: 6.7 us, of which start, end and
// four dependent round trips to memory (requests; pages given back; pages taken; page numbers of the tokens) are 4.6, and the instructions of the tokens' searches and stores the
// rest: one compute unit, 0.6 to 1.2 us per thousand tokens.  So k_cache_place has many.  (512 lanes: 8.1 us; the top of the stack loaded ahead: 7.0.)
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
    for (uint32_t i = t; i < a.tokens; i += kPlanWg) place_tokens<1>(a, i, kPlanWg, ends, [&](uint32_t b) { return lens[b]; });
}

// Slots and positions of many tokens, behind k_cache_plan.
constexpr uint32_t kPlaceWg = 256;
constexpr int kPlacePer = 4;  // tokens of a lane

__global__ __launch_bounds__(kPlaceWg) void k_cache_place(PlanArgs a)
{
    __shared__ uint32_t ends[kPlanMost];
    __shared__ int32_t lens[kPlanMost];
    for (uint32_t b = threadIdx.x; b < a.batch; b += kPlaceWg) {
        ends[b] = (uint32_t)a.starts[b + 1];
        const int32_t granted = a.granted[b], len = a.lens_out[b];
        lens[b] = granted < 0 ? -1 : len;
    }
    __syncthreads();
    const uint32_t i = blockIdx.x * kPlacePer * kPlaceWg + threadIdx.x;
    if (i < a.tokens) place_tokens<kPlacePer>(a, i, kPlaceWg, ends, [&](uint32_t b) { return lens[b]; });
}

// ---------------------------------------------------------------- verification
//
// A sequence's drafts are judged by single numbers; only the row behind the accepted ones is read as a whole, the draft's too where one was
// refused.  A row is cut into chunks; a wavefront adds up one at a time.  The chunk in which the sum passes its mark is found from the
// chunks' sums and read once more by one wavefront, which finds the token in it.  All sums are binary64: each addition is off
// by 2^-53 of the whole at most.  A number is in 10 of them on its way into a chunk's sum (4 of a lane, 6 of lanes), 37 more into the whole's (31 of a lane's chunks at most,
// 6 of lanes), or 68 into the sum before a chunk (31 again) and 17 to a token's border in it; with the mark's product and the differences fewer than 150, so that no border
// moves by 2^-45 of the whole, 2^-21 of the step between two random numbers of 24 bits.  (Up to a vocabulary of 2^21; then chunks have more than 1024 numbers, one addition for
// each 1024 more.)

struct Verdict;

// 128 bytes, two cache lines of a launch's arguments: with 152 a row of 32000 took 6.40 us in a graph, so 6.33.
struct VerifyArgs {
    const void *target, *draft;
    size_t target_stride, draft_stride;
    const int64_t *ids;
    const float *uniform, *sample;
    union {
        const int32_t *starts;
        uint64_t each;  // rows of every sequence, with kEven
    };
    int64_t *out;
    int32_t *accepted, *rejected;
    const int32_t *granted, *drop;  // of the plan (null: nobody was refused, nothing was dropped)
    double *sums;                   // workspace [batch][chunks], and behind it [batch] verdicts
    uint32_t tokens, batch, vocab;
    uint32_t flags;                 // the logarithm of a chunk's probabilities, kEven, kFill

    static constexpr uint32_t kEven = 256, kFill = 512;  // kFill: rows of no sequence get -1

    __host__ __device__ uint32_t chunk() const { return 1u << (flags & 31); }  // probabilities that a wavefront adds up at a time
    __host__ __device__ uint32_t chunks() const { return (vocab + chunk() - 1) >> (flags & 31); }
    __host__ __device__ Verdict *verdicts() const { return reinterpret_cast<Verdict *>(sums + (size_t)batch * chunks()); }
};
static_assert(sizeof(VerifyArgs) == 128, "two cache lines");

// A probability: what is no positive number counts as none.
template <typename T>
__device__ __forceinline__ float probability(T v)
{
    const float f = (float)v;
    return __builtin_amdgcn_classf(f, 0x180) ? f : 0.0f;  // positive, subnormal or normal
}

// Where a sequence ends: rows first .. first + n - 1, `row` of them accepted; refused: whether row `row` refused its draft `token`.
struct Verdict {
    uint32_t first, n, row, refused;
    int64_t token;
};

__device__ __forceinline__ uint32_t start_of(const VerifyArgs &a, uint32_t b)
{
    const int32_t s = a.starts[b];
    return s < 0 ? 0 : (uint32_t)s < a.tokens ? (uint32_t)s : a.tokens;
}

// Whether the plan refused a sequence: its rows hold no tokens.
__device__ __forceinline__ bool without_places(const VerifyArgs &a, uint32_t b) { return a.granted && a.granted[b] < 0; }

// Every wavefront finds it by itself: a lane per draft.
template <typename T>
__device__ __forceinline__ Verdict verdict_of(const VerifyArgs &a, uint32_t b)
{
    const uint32_t lane = threadIdx.x & 63;
    Verdict v;
    uint32_t end;
    if (!(a.flags & VerifyArgs::kEven)) {
        v.first = start_of(a, b);
        end = start_of(a, b + 1);
        if (end < v.first) end = v.first;
    } else {
        v.first = b * (uint32_t)a.each;
        end = v.first + (uint32_t)a.each;
    }
    v.n = end - v.first;
    v.row = v.n ? v.n - 1 : 0;
    v.refused = 0;
    v.token = -1;
    for (uint32_t i0 = 0; i0 + 1 < v.n; i0 += 64) {
        const uint32_t i = i0 + lane;
        bool no = false;
        int64_t d = -1;
        if (i + 1 < v.n) {
            const size_t row = v.first + i;
            const float u = a.uniform[row];
            d = a.ids[row + 1];
            no = true;
            if (d >= 0 && d < (int64_t)a.vocab) {
                const double p = probability(static_cast<const T *>(a.target)[row * a.target_stride + d]);
                const double q = a.draft ? probability(static_cast<const T *>(a.draft)[row * a.draft_stride + d]) : 1.0f;
                no = !((double)u * q < p);  // 24 times 24 bits: exact
            }
        }
        const uint64_t votes = __builtin_amdgcn_ballot_w64(no);
        if (votes) {
            const int l = __builtin_ctzll(votes);
            v.row = i0 + (uint32_t)l;
            v.refused = 1;
            v.token = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(d >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)d, l));
            break;
        }
    }
    v.first = (uint32_t)__builtin_amdgcn_readfirstlane((int)v.first);
    v.n = (uint32_t)__builtin_amdgcn_readfirstlane((int)v.n);
    v.row = (uint32_t)__builtin_amdgcn_readfirstlane((int)v.row);
    return v;
}

// Wavefront `mine` of `all` writes its part of the rows of no sequence.  Wavefronts do it that nobody waits for (0.08 of 6.3 us).
__device__ __forceinline__ void fill_others(const VerifyArgs &a, uint32_t mine, uint32_t all)
{
    if (!(a.flags & VerifyArgs::kFill)) return;
    const uint32_t s0 = start_of(a, 0), s1 = start_of(a, a.batch), at = mine * 64 + (threadIdx.x & 63);
    for (uint32_t i = at; i < s0; i += all * 64) a.out[i] = -1;
    for (uint32_t i = s1 + at; i < a.tokens; i += all * 64) a.out[i] = -1;
}

constexpr uint32_t kSumsWaves = 4, kAloneWaves = 16, kPickWaves = 2, kChunksMost = 2048, kChunk = 1024;
constexpr int kPer = kChunk / 64;  // numbers of a lane: neighbours

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

    // The weights of the lane's kPer tokens of kChunk from `begin` on, zeros behind `end`: neighbours, or where only their sum counts (APART) 16 bytes from each of
    // the loads, whose lanes then lie side by side (a row of 32000 in one compute unit: 7.9 -> 7.15 us).  What a compute unit does for a number counts where it has a
    // whole row, so each kind of row has its own steps.  (A branch around each load would make the next wait for it: 16 round trips to memory.)
    template <bool APART>
    __device__ __forceinline__ void weights(uint32_t begin, uint32_t end, double (&w)[kPer]) const
    {
        constexpr int W = 16 / sizeof(T);  // numbers of a load
        typedef T V __attribute__((ext_vector_type(W)));
        typedef V VA __attribute__((aligned(sizeof(T))));
        constexpr uint32_t STEP = APART ? 64 * W : W;
        const uint32_t t = begin + (threadIdx.x & 63) * (APART ? W : kPer);
        auto at = [&](int k) { return t + (uint32_t)(k / W) * STEP + (uint32_t)(k % W); };
        V x[kPer / W], y[kPer / W];
        if (end - begin >= kChunk) {
#pragma unroll
            for (int k = 0; k < kPer; k += W) x[k / W] = *reinterpret_cast<const VA *>(p + at(k));
            if (q) {
#pragma unroll
                for (int k = 0; k < kPer; k += W) y[k / W] = *reinterpret_cast<const VA *>(q + at(k));
            }
        } else {
#pragma unroll
            for (int k = 0; k < kPer; ++k) x[k / W][k % W] = p[at(k) < end ? at(k) : end - 1];
            if (q) {
#pragma unroll
                for (int k = 0; k < kPer; ++k) y[k / W][k % W] = q[at(k) < end ? at(k) : end - 1];
            }
#pragma unroll
            for (int k = 0; k < kPer; ++k)
                if (at(k) >= end) x[k / W][k % W] = (T)0.0f;
        }
        if (q) {
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                const double d = (double)probability(x[k / W][k % W]) - (double)probability(y[k / W][k % W]);
                w[k] = __builtin_fmax(d, 0.0);
            }
        } else {
#pragma unroll
            for (int k = 0; k < kPer; ++k) w[k] = (double)probability(x[k / W][k % W]);
            if (less >= (int64_t)begin && less < (int64_t)end) {
#pragma unroll
                for (int k = 0; k < kPer; ++k)
                    if ((int64_t)at(k) == less) w[k] = 0.0;
            }
        }
    }
};

// A wavefront's sum of the weights of a chunk, in its last lane.
template <typename T>
__device__ __forceinline__ double sum_chunk(const VerifyArgs &a, const Row<T> &row, uint32_t c)
{
    const uint32_t begin = c * a.chunk(), end = a.vocab - begin < a.chunk() ? a.vocab : begin + a.chunk();
    double sum = 0.0;
    for (uint32_t i = begin; i < end; i += kChunk) {
        double w[kPer];
        row.template weights<true>(i, end, w);
#pragma unroll
        for (int d = kPer / 2; d > 0; d /= 2)
#pragma unroll
            for (int k = 0; k < d; ++k) w[k] += w[k + d];
        sum += w[0];
    }
    return scan_wave(sum);
}

template <typename T>
__global__ __launch_bounds__(kSumsWaves * 64) void k_verify_sums(VerifyArgs a)
{
    const uint32_t b = blockIdx.y, first = blockIdx.x * kSumsWaves + wave_of(threadIdx.x), lane = threadIdx.x & 63;
    if (first >= a.chunks()) return;
    const Verdict v = verdict_of<T>(a, b);
    if (first == 0 && lane == 0) a.verdicts()[b] = v;
    if (v.n == 0 || without_places(a, b)) return;
    const Row<T> row(a, v);
    for (uint32_t c = first; c < a.chunks(); c += gridDim.x * kSumsWaves) {
        const double s = sum_chunk(a, row, c);
        if (lane == 63) a.sums[(size_t)b * a.chunks() + c] = s;
    }
}

// Numbers of a wavefront, `run` of a lane in the order of the lanes; next(i): the lane's number i.  The sum before the lane's first one, and of all.
template <typename F>
__device__ __forceinline__ double sums_of(uint32_t run, double &total, F next)
{
    double mine = 0.0;
    for (uint32_t i = 0; i < run; ++i) mine += next(i);
    const double upto = scan_wave(mine);
    total = of_lane(upto, 63);
    return before_lane(upto);
}

// The first of them up to and with which their sum is above the mark, or the last positive one where none is; `sum` is the sum before the
// lane's first one, and then the one before that number.
template <typename F>
__device__ __forceinline__ uint32_t first_above(uint32_t run, double mark, double &sum, F next)
{
    uint32_t at = 0xFFFFFFFFu, last = 0xFFFFFFFFu;
    double held = 0.0, held_last = 0.0;
    for (uint32_t i = 0; i < run; ++i) {
        const double x = next(i);
        if (x > 0.0) {
            last = i;
            held_last = sum;
            if (at == 0xFFFFFFFFu && sum + x > mark) {
                at = i;
                held = sum;
            }
        }
        sum += x;
    }
    const uint64_t votes = __builtin_amdgcn_ballot_w64(at != 0xFFFFFFFFu), some = __builtin_amdgcn_ballot_w64(last != 0xFFFFFFFFu);
    const int l = votes ? __builtin_ctzll(votes) : 63 - __builtin_clzll(some);
    sum = of_lane(votes ? held : held_last, l);
    return (uint32_t)l * run + (uint32_t)__builtin_amdgcn_readlane((int)(votes ? at : last), l);
}

// One workgroup per sequence.  ALONE: its wavefronts add up the chunks themselves; otherwise it is one wavefront behind k_verify_sums, and a
// second one for the rows of no sequence.
// 32000 probabilities, ALONE: 6.3 us, of which binary64 instructions of one compute unit are half; 64 sequences of 131072: k_verify_sums 11.5 us (4.7 TB/s of what it
// needs), then 4.
template <typename T, bool ALONE>
__global__ __launch_bounds__((ALONE ? kAloneWaves : kPickWaves) * 64) void k_verify_pick(VerifyArgs a)
{
    __shared__ double sums[kChunksMost];
    constexpr uint32_t OTHERS = (ALONE ? kAloneWaves : kPickWaves) - 1;
    const uint32_t b = blockIdx.x, lane = threadIdx.x & 63, wave = wave_of(threadIdx.x);
    const float r = a.sample[b];
    const bool no_places = without_places(a, b);
    const Verdict v = ALONE ? verdict_of<T>(a, b) : a.verdicts()[b];
    if constexpr (!ALONE)
        for (uint32_t c = threadIdx.x; c < a.chunks(); c += kPickWaves * 64) sums[c] = a.sums[(size_t)b * a.chunks() + c];
    if (v.n == 0 || no_places) {
        if (wave != 0) {
            fill_others(a, b * OTHERS + wave - 1, a.batch * OTHERS);
            return;
        }
        if (lane == 0) {
            const int32_t owed = no_places && a.drop ? a.drop[b] : 0;  // what the plan was asked to take back is still to be taken
            a.accepted[b] = -1;
            a.rejected[b] = owed > 0 ? owed : 0;
        }
        for (uint32_t i = lane; i < v.n; i += 64) a.out[v.first + i] = -1;
        return;
    }
    if (threadIdx.x == 0) {
        a.accepted[b] = (int32_t)v.row;
        a.rejected[b] = (int32_t)(v.n - 1 - v.row);
    }
    Row<T> row(a, v);
    if constexpr (ALONE)
        for (uint32_t c = wave; c < a.chunks(); c += kAloneWaves) {
            const double s = sum_chunk(a, row, c);
            if (lane == 63) sums[c] = s;
        }
    __syncthreads();
    if (wave != 0) {
        fill_others(a, b * OTHERS + wave - 1, a.batch * OTHERS);
        return;
    }
    const uint32_t run = (a.chunks() + 63) / 64;
    auto chunk_sum = [&](uint32_t i) { return lane * run + i < a.chunks() ? sums[lane * run + i] : 0.0; };
    double total, sum = sums_of(run, total, chunk_sum);
    if (!(total > 0.0)) {  // nothing is left of the difference: the target's own
        row.q = nullptr;
        row.less = -1;
        for (uint32_t c = 0; c < a.chunks(); ++c) {
            const double s = sum_chunk(a, row, c);
            if (lane == 63) sums[c] = s;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        sum = sums_of(run, total, chunk_sum);
    }
    int64_t token = -1;
    if (total > 0.0) {
        // (of one and more: above all sums, for a running one may round to more than the whole's, which is taken in another order)
        const double mark = r >= 1.0f ? __builtin_inf() : (r > 0.0f ? (double)r : 0.0) * total;
        const uint32_t c = first_above(run, mark, sum, chunk_sum);
        const uint32_t begin = c * a.chunk(), end = a.vocab - begin < a.chunk() ? a.vocab : begin + a.chunk();
        for (uint32_t i0 = begin; i0 < end; i0 += kChunk) {
            double x[kPer], mine = 0.0;
            row.template weights<false>(i0, end, x);
#pragma unroll
            for (int k = 0; k < kPer; ++k) mine += x[k];
            const double upto = scan_wave(mine);
            double s = sum + before_lane(upto);
            uint32_t at = 0xFFFFFFFFu, last = 0xFFFFFFFFu;
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                s += x[k];
                if (x[k] > 0.0) {
                    last = k;
                    if (at == 0xFFFFFFFFu && s > mark) at = k;
                }
            }
            const uint64_t votes = __builtin_amdgcn_ballot_w64(at != 0xFFFFFFFFu), some = __builtin_amdgcn_ballot_w64(last != 0xFFFFFFFFu);
            if (some) {  // (the last one with a weight, if the rounding of sums leaves none above the mark)
                const int l = votes ? __builtin_ctzll(votes) : 63 - __builtin_clzll(some);
                token = i0 + (uint32_t)l * kPer + (uint32_t)__builtin_amdgcn_readlane((int)(votes ? at : last), l);
            }
            if (votes) break;
            sum += of_lane(upto, 63);
        }
    }
    for (uint32_t i = lane; i < v.n; i += 64) a.out[v.first + i] = i < v.row ? a.ids[v.first + i + 1] : i == v.row ? token : -1;
}

}  // namespace
