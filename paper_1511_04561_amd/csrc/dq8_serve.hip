// dq8: plan of a decoding step and verification of drafted tokens (include/dq8_serve.h): checks of arguments and launches.  The kernels
// are in dq8_kernels_serve.hpp.  Built with the flags of dq8.hip.
#include "dq8_serve.h"

#include "dq8_cache_check.hpp"
#include "dq8_kernels_serve.hpp"

namespace {

using dq8::failed;
using dq8::kCacheLimit;

static_assert(kPlanMost == DQ8_PLAN_MAX_BATCH, "LDS of the plan");

// Tokens up to which the plan's own workgroup writes slots and positions; more take a second launch.  us, 16 sequences of 256 tokens each: 6.8 in one (two: 7.7), of 512 9
// (8.1); 256 sequences of 16 9.4 (10.5), of 32 14 (11).
constexpr size_t kPlanTokens = 6144;

struct Array {
    const void *p;
    size_t n;
};

// Whether an array that is written overlaps another one.
template <int W, int R>
bool overlap(const Array (&written)[W], const Array (&read)[R])
{
    for (int i = 0; i < W; ++i) {
        for (int j = i + 1; j < W; ++j)
            if (dq8::meet(written[i].p, written[i].n, written[j].p, written[j].n)) return true;
        for (const Array &r : read)
            if (dq8::meet(written[i].p, written[i].n, r.p, r.n)) return true;
    }
    return false;
}

int check_verify(const char *who, const dq8_verify *in)
{
    if (!in) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    const dq8_verify &v = *in;
    if (v.type != DQ8_FLOAT32 && v.type != DQ8_BFLOAT16 && v.type != DQ8_FLOAT16) return failed(DQ8_ERR_ARG, "%s: unknown type %d", who, v.type);
    if (v.batch > 65535 || v.tokens >= kCacheLimit) return failed(DQ8_ERR_ARG, "%s: too many tokens or sequences", who);
    if (v.batch && !v.starts && v.tokens % v.batch != 0) return failed(DQ8_ERR_ARG, "%s: %zu tokens are not as many for each of %zu sequences", who, v.tokens, v.batch);
    if (!v.batch && !v.starts && v.tokens) return failed(DQ8_ERR_ARG, "%s: %zu tokens of no sequence", who, v.tokens);
    if (v.vocab < 1 || v.vocab >= kCacheLimit - 4096) return failed(DQ8_ERR_ARG, "%s: a vocabulary of %zu", who, v.vocab);
    if (!dq8::sane(v.target_stride, v.tokens) || (v.draft && !dq8::sane(v.draft_stride, v.tokens))) return failed(DQ8_ERR_ARG, "%s: a stride is too large", who);
    return DQ8_OK;
}

// Chunks of a row: of 1024 probabilities, more where there would be more chunks than the LDS of the last step holds.
void cut(const dq8_verify &v, uint32_t &chunk, uint32_t &chunks)
{
    chunk = kChunk;
    while ((v.vocab + chunk - 1) / chunk > kChunksMost) chunk *= 2;
    chunks = (uint32_t)((v.vocab + chunk - 1) / chunk);
}

// Whether one workgroup reads a sequence's whole row, in one launch, or the whole chip and then a wavefront per sequence, in two: ns that each takes.  What a compute unit
// needs for a row grows with its numbers, what the chip needs with all of them.  us from Python, in one | in two launches, four tokens of each sequence:
//   binary32 with the draft's probabilities, 8 sequences of 32768 7.8 | 7.9, 50021 9.8 | 7.9, 65536 11.0 | 8.1; 64 of 100000 16.7 | 12.9, 131072 19.9 | 15.8; 128 of 131072
//   22.7 | 23.0, bfloat16 20.7 | 17.2; binary32 without, 8 of 50021 7.7 | 7.8, 65536 8.5 | 8.0, 131072 12.9 | 8.0; 64 of 131072 14.0 | 11.2.  (In a graph two launches of few
//   sequences are a microsecond cheaper: one of 32768 with draft 6.2 | 6.2, of 65536 bfloat16 without 8.4 | 6.4; 256 of 131072 bfloat16 without 16.0 | 19.7.)
bool alone(const dq8_verify &v, int cus)
{
    uint32_t chunk, chunks;
    cut(v, chunk, chunks);
    const size_t bytes = (v.type == DQ8_FLOAT32 ? 4 : 2) * (v.draft ? 2 : 1), waves = v.batch * chunks;
    const size_t one = (v.draft ? 4500 + v.vocab / 10 : 4200 + v.vocab * 13 / 200) + waves * bytes / 28, two = 8000 + (waves > 2048 ? (waves - 2048) * (bytes + 1) / 8 : 0);
    return one <= two || v.batch >= (size_t)cus;
}

size_t workspace_of(const dq8_verify &v)
{
    uint32_t chunk, chunks;
    cut(v, chunk, chunks);
    return v.batch * (sizeof(Verdict) + chunks * sizeof(double));
}

template <typename T>
int verify(const VerifyArgs &k, int cus, hipStream_t stream)
{
    if (!k.sums) {
        hipLaunchKernelGGL((k_verify_pick<T, true>), dim3(k.batch), dim3(kAloneWaves * 64), 0, stream, k);
        return dq8::after_launch_of("k_verify_pick", stream);
    }
    // wavefronts for the whole chip, a chunk at least for each
    unsigned groups = (k.chunks() + kSumsWaves - 1) / kSumsWaves;
    const unsigned most = (unsigned)cus * 32 / (kSumsWaves * k.batch) + 1;
    if (groups > most) groups = most;
    hipLaunchKernelGGL(k_verify_sums<T>, dim3(groups, k.batch), dim3(kSumsWaves * 64), 0, stream, k);
    const int rc = dq8::after_launch_of("k_verify_sums", stream);
    if (rc) return rc;
    hipLaunchKernelGGL((k_verify_pick<T, false>), dim3(k.batch), dim3(kPickWaves * 64), 0, stream, k);
    return dq8::after_launch_of("k_verify_pick", stream);
}

}  // namespace

extern "C" {

int dq8_cache_plan(const dq8_plan *in, void *hip_stream)
{
    static const char who[] = "dq8_cache_plan";
    if (!in) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    const dq8_plan &p = *in;
    if (p.page_size < 16 || p.page_size > DQ8_CACHE_MAX_PAGE || (p.page_size & (p.page_size - 1)) != 0)
        return failed(DQ8_ERR_ARG, "%s: page_size %d is not a power of two from 16 to %d", who, p.page_size, DQ8_CACHE_MAX_PAGE);
    if (p.batch > DQ8_PLAN_MAX_BATCH) return failed(DQ8_ERR_ARG, "%s: %zu sequences are more than %d", who, p.batch, DQ8_PLAN_MAX_BATCH);
    if (p.max_pages < 1 || p.max_pages >= kCacheLimit / (size_t)p.page_size || p.batch * p.max_pages >= kCacheLimit)
        return failed(DQ8_ERR_ARG, "%s: %zu pages per sequence", who, p.max_pages);
    if (p.tokens >= kCacheLimit || p.free_capacity >= kCacheLimit) return failed(DQ8_ERR_ARG, "%s: too many tokens or pages", who);
    if (p.batch == 0) return failed(DQ8_ERR_ARG, "%s: no sequences", who);
    if (!p.lens || !p.new_tokens || !p.pages || !p.n_free || !p.starts || !p.lens_out || !p.granted || !p.n_free_out || (p.free_capacity && !p.free_pages) ||
        (p.tokens && (!p.slots || !p.positions)))
        return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    if ((((uintptr_t)p.lens | (uintptr_t)p.new_tokens | (uintptr_t)p.drop | (uintptr_t)p.pages | (uintptr_t)p.free_pages | (uintptr_t)p.n_free | (uintptr_t)p.starts |
          (uintptr_t)p.lens_out | (uintptr_t)p.granted | (uintptr_t)p.n_free_out) & 3) != 0 ||
        (((uintptr_t)p.slots | (uintptr_t)p.positions) & 7) != 0)
        return failed(DQ8_ERR_ARG, "%s: an array does not start at a multiple of its element's size", who);
    const size_t b4 = p.batch * 4;
    const Array written[] = {{p.pages, b4 * p.max_pages}, {p.free_pages, p.free_capacity * 4}, {p.slots, p.tokens * 8}, {p.positions, p.tokens * 8},
                             {p.starts, b4 + 4}, {p.lens_out, b4}, {p.granted, b4}, {p.n_free_out, 4}};
    const Array read[] = {{p.lens, p.lens == p.lens_out ? 0 : b4}, {p.new_tokens, b4}, {p.drop, p.drop ? b4 : 0}, {p.n_free, p.n_free == p.n_free_out ? 0 : (size_t)4}};
    if (overlap(written, read)) return failed(DQ8_ERR_ARG, "%s: an output overlaps another array", who);
    PlanArgs k;
    k.lens = p.lens, k.new_tokens = p.new_tokens, k.drop = p.drop, k.pages = p.pages, k.free_pages = p.free_pages, k.n_free = p.n_free;
    k.slots = p.slots, k.positions = p.positions, k.starts = p.starts, k.lens_out = p.lens_out, k.granted = p.granted, k.n_free_out = p.n_free_out;
    k.batch = (uint32_t)p.batch, k.max_pages = (uint32_t)p.max_pages, k.tokens = (uint32_t)p.tokens, k.capacity = (uint32_t)p.free_capacity;
    k.page_shift = (uint32_t)__builtin_ctz((unsigned)p.page_size);
    k.finish = p.tokens <= kPlanTokens;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipLaunchKernelGGL(k_cache_plan, dim3(1), dim3(kPlanWg), 0, stream, k);
    const int rc = dq8::after_launch_of("k_cache_plan", stream);
    if (rc || k.finish) return rc;
    constexpr size_t per = kPlaceWg * kPlacePer;
    hipLaunchKernelGGL(k_cache_place, dim3((unsigned)((p.tokens + per - 1) / per)), dim3(kPlaceWg), 0, stream, k);
    return dq8::after_launch_of("k_cache_place", stream);
}

size_t dq8_draft_verify_workspace_bytes(const dq8_verify *v)
{
    if (check_verify("dq8_draft_verify_workspace_bytes", v) || v->batch == 0 || v->tokens == 0) return 0;
    dq8::DeviceTables dev;
    return dq8::device_tables(0, &dev) || alone(*v, dev.cus) ? 0 : workspace_of(*v);
}

int dq8_draft_verify(const dq8_verify *in, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    static const char who[] = "dq8_draft_verify";
    const int rc = check_verify(who, in);
    if (rc) return rc;
    const dq8_verify &v = *in;
    if (v.batch == 0) return DQ8_OK;
    if (!v.accepted || !v.rejected || !v.sample || (v.tokens && (!v.target || !v.ids || !v.uniform || !v.out))) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    const size_t size = v.type == DQ8_FLOAT32 ? 4 : 2;
    if ((((uintptr_t)v.target | (uintptr_t)v.draft) & (size - 1)) != 0 || (((uintptr_t)v.ids | (uintptr_t)v.out) & 7) != 0 ||
        (((uintptr_t)v.uniform | (uintptr_t)v.sample | (uintptr_t)v.starts | (uintptr_t)v.accepted | (uintptr_t)v.rejected | (uintptr_t)v.granted |
          (uintptr_t)v.drop) & 3) != 0 || ((uintptr_t)workspace & 15) != 0)
        return failed(DQ8_ERR_ARG, "%s: an array does not start at a multiple of its element's size (workspace: 16 bytes)", who);
    auto extent = [&](size_t stride) { return v.tokens ? ((v.tokens - 1) * stride + v.vocab) * size : 0; };
    const Array written[] = {{v.out, v.tokens * 8}, {v.accepted, v.batch * 4}, {v.rejected, v.batch * 4}, {workspace, workspace ? workspace_bytes : 0}};
    const Array read[] = {{v.target, extent(v.target_stride)}, {v.draft, v.draft ? extent(v.draft_stride) : 0}, {v.ids, v.tokens * 8}, {v.uniform, v.tokens * 4},
                          {v.sample, v.batch * 4}, {v.starts, v.starts ? (v.batch + 1) * 4 : 0}, {v.granted, v.granted ? v.batch * 4 : 0},
                          {v.drop, v.granted && v.drop && v.drop != v.rejected ? v.batch * 4 : 0}};
    if (overlap(written, read)) return failed(DQ8_ERR_ARG, "%s: an output or the workspace overlaps another array", who);
    VerifyArgs k;
    k.target = v.target, k.draft = v.draft, k.target_stride = v.target_stride, k.draft_stride = v.draft_stride;
    k.ids = v.ids, k.uniform = v.uniform, k.sample = v.sample, k.starts = v.starts, k.out = v.out, k.accepted = v.accepted, k.rejected = v.rejected;
    k.granted = v.granted, k.drop = v.drop;
    k.tokens = (uint32_t)v.tokens, k.batch = (uint32_t)v.batch, k.vocab = (uint32_t)v.vocab;
    uint32_t chunk, chunks;
    cut(v, chunk, chunks);
    k.flags = (uint32_t)__builtin_ctz(chunk) | (v.starts ? 0 : VerifyArgs::kEven) | (v.fill && v.starts ? VerifyArgs::kFill : 0);
    if (!v.starts) k.each = v.tokens / v.batch;
    dq8::DeviceTables dev;
    const int found = dq8::device_tables(0, &dev);
    if (found) return found;
    const bool some = v.tokens && workspace && !alone(v, dev.cus) && workspace_bytes >= workspace_of(v);
    k.sums = some ? static_cast<double *>(workspace) : nullptr;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (v.type == DQ8_FLOAT32) return verify<float>(k, dev.cus, stream);
    return v.type == DQ8_BFLOAT16 ? verify<__bf16>(k, dev.cus, stream) : verify<_Float16>(k, dev.cus, stream);
}

}  // extern "C"
