// dq8: attention of new tokens over a paged cache of 8-bit keys and values (dq8_cache_attention of include/dq8_cache.h).
//
// The kernels are in dq8_kernels_attend.hpp (few query rows per cached head: decoding; and the join of parts) and
// dq8_kernels_attend_chunk.hpp (many: prompts); this file chooses between them.  Built with the flags of dq8.hip.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "dq8_cache_check.hpp"
#include "dq8_kernels_attend.hpp"
#include "dq8_kernels_attend_chunk.hpp"

namespace {

// What a call launches.
struct Shape {
    int dp;            // padded head length
    bool chunk;        // the kernel for many query rows
    unsigned rows16;   // otherwise: groups of 16 query rows of a job
    unsigned groups;   // workgroups
    unsigned splits;   // chunk: workgroups per job
    size_t jobs, work; // jobs and tiles, at most
    size_t records;    // of jobs that may be cut into parts
    unsigned rows;     // query rows of a job, at most
    size_t parts;      // that can be written
    bool few;          // whether the join has few rows
};

// Which kernel has the query rows of a cached head and sequence, up to 16 of them the one for few.  us, 8 cached heads of 128 (in
// parentheses of 64), few | many:
//   one sequence of 8192, 20 rows 28 | 24 (22 | 20), 64 rows 35 | 28 (28 | 21);  of 1024, 20 rows 18 | 18, 96 rows 24 | 20;
//   of 400, 20 rows 17 | 21, 96 rows 21 | 22;  2 of 16384, 20 rows 38 | 52 (25 | 41), 96 rows 61 | 59 (40 | 44);
//   16 of 4096, 20 rows 42 | 91 (28 | 72), 96 rows 93 | 100 (57 | 78), 128 rows 106 | 104 (67 | 80), 192 rows 150 | 112 (95 | 87)
// A tile costs the one for many as much whatever the rows, but it leaves a part per workgroup to the join and not one per wavefront: it has
// them above 128 rows, and fewer where its workgroups have a few tiles each of sequences that are not short.  Heads of 256, whose keys
// and values the one for few reads again for every 16 rows: 16 of 4096, 64 rows 291 | 378, 68 rows 402 | 379.
bool for_many(size_t rows, int dp, size_t jobs, size_t tiles, int cus)
{
    if (dp == 256) return rows > 64;
    return rows > 128 || (rows > 16 && tiles >= 16 && jobs <= 4 * (size_t)cus / tiles);
}

Shape shape_of(const dq8_cache *c, const dq8_attention &a, int cus)
{
    Shape s;
    s.dp = c->dim <= 64 ? 64 : c->dim <= 128 ? 128 : 256;
    const size_t group = (size_t)(a.heads / c->kv_heads);
    size_t new_tokens = a.starts ? (a.max_new ? a.max_new : a.tokens) : a.tokens / a.batch;
    if (new_tokens > a.tokens) new_tokens = a.tokens;
    const size_t rows = new_tokens * group;
    const size_t capacity = a.max_pages * (size_t)c->page_size, tiles64 = (capacity + 63) / 64;
    s.chunk = for_many(rows, s.dp, a.batch * (size_t)c->kv_heads, tiles64, cus);
    s.rows16 = rows <= 16 || s.dp == 256 ? 1 : 2;  // (16 sequences of 4096, 64 rows: 101 us with groups of 16, 66 of 32; 16 rows 36, 48)
    const size_t per = s.chunk ? 32 * kChunkWaves : 16 * (size_t)s.rows16;
    s.jobs = (a.starts ? a.tokens * group / per + a.batch : a.batch * ((rows + per - 1) / per)) * (size_t)c->kv_heads;
    s.rows = (unsigned)(!a.starts && rows < per ? rows : per);
    if (s.chunk) {
        // Idle compute units take parts of jobs, of two tiles at least (two sequences' heads, 256 rows, 2048 tokens: 94 us undivided, 28 with
        // parts of four tiles, 25 of two; 512 tokens 32, 27, 22).
        size_t splits = s.jobs ? (size_t)cus / s.jobs : 1;
        if (splits > tiles64 / 2) splits = tiles64 / 2;
        s.splits = splits < 1 ? 1 : (unsigned)splits;
        s.groups = (unsigned)(s.jobs * s.splits);
        s.parts = s.splits > 1 ? s.groups : 0;
        s.work = s.jobs * s.splits;
        s.records = s.jobs;
        s.few = s.records * s.rows <= (size_t)cus;
        return s;
    }
    s.splits = 1;
    const size_t tiles = (capacity + kTile - 1) / kTile;
    s.work = s.jobs > SIZE_MAX / 2 / tiles ? SIZE_MAX / 2 : s.jobs * tiles;
    // One table per compute unit, eight wavefronts of 256 registers, a tile at least for each (one sequence of 1337: 14 us; two tiles: 16,
    // four: 22).
    size_t groups = (size_t)cus;
    if (groups > (s.work + kAttendWaves - 1) / kAttendWaves) groups = (s.work + kAttendWaves - 1) / kAttendWaves;
    s.groups = (unsigned)groups;
    s.parts = groups * kAttendWaves * 2;
    s.records = s.jobs < groups * kAttendWaves ? s.jobs : groups * kAttendWaves;  // a wavefront leaves one job at most to others
    s.few = s.records * s.rows <= (size_t)cus;
    return s;
}

size_t record_bytes(const Shape &s) { return s.parts ? (1 + s.records) * sizeof(int4) : 0; }  // their number takes the first
size_t sums_bytes(const Shape &s) { return (s.parts * s.rows * sizeof(float2) + 15) / 16 * 16; }
size_t parts_bytes(const Shape &s) { return s.parts * s.rows * s.dp * sizeof(float); }
size_t workspace_bytes_of(const Shape &s) { return record_bytes(s) + sums_bytes(s) + parts_bytes(s); }

// What does not look at the arrays of the call.  0 tokens or sequences pass: such a call launches nothing.
int check_shape(const char *who, int kind, const dq8_cache *cache, const dq8_attention *in)
{
    using dq8::failed;
    const int rc = dq8::check_cache(who, kind, cache);
    if (rc) return rc;
    if (!in) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    const dq8_attention &a = *in;
    if (a.type != DQ8_BFLOAT16 && a.type != DQ8_FLOAT16) return failed(DQ8_ERR_ARG, "%s: type %d is neither bfloat16 nor float16", who, a.type);
    if (a.heads < 1 || a.heads > 65535 || a.heads % cache->kv_heads != 0)
        return failed(DQ8_ERR_ARG, "%s: %d query heads are no multiple of %d cached heads", who, a.heads, cache->kv_heads);
    if (a.batch >= dq8::kCacheLimit || a.tokens >= dq8::kCacheLimit || a.tokens * (size_t)a.heads >= dq8::kCacheLimit)
        return failed(DQ8_ERR_ARG, "%s: too many tokens or sequences", who);
    if (!a.starts && (a.batch ? a.tokens % a.batch : a.tokens) != 0)
        return failed(DQ8_ERR_ARG, "%s: %zu tokens are not as many for each of %zu sequences", who, a.tokens, a.batch);
    if (a.tokens == 0 || a.batch == 0) return DQ8_OK;
    if (a.max_pages < 1 || a.max_pages >= dq8::kCacheLimit / (size_t)cache->page_size || a.batch > ((size_t)1 << 40) / a.max_pages)
        return failed(DQ8_ERR_ARG, "%s: %zu pages per sequence", who, a.max_pages);
    if (a.window < 0) return failed(DQ8_ERR_ARG, "%s: window %d", who, a.window);
    if (!(a.softmax_scale >= -FLT_MAX && a.softmax_scale <= FLT_MAX)) return failed(DQ8_ERR_ARG, "%s: softmax_scale is not finite", who);
    if (!dq8::sane(a.q_token_stride, a.tokens) || !dq8::sane(a.out_token_stride, a.tokens) || !dq8::sane(a.q_head_stride, (size_t)a.heads) ||
        !dq8::sane(a.out_head_stride, (size_t)a.heads))
        return failed(DQ8_ERR_ARG, "%s: a stride is too large", who);
    return DQ8_OK;
}

int check_arrays(const char *who, const dq8_cache *cache, const dq8_attention &a, const void *workspace, size_t workspace_bytes)
{
    using dq8::failed;
    using dq8::meet;
    if (!a.q || !a.out || !a.pages || !a.lens) return failed(DQ8_ERR_NULL, "%s: NULL pointer", who);
    if ((((uintptr_t)a.q | (uintptr_t)a.out) & 1) != 0 || (((uintptr_t)a.pages | (uintptr_t)a.lens | (uintptr_t)a.starts) & 3) != 0 ||
        ((uintptr_t)workspace & 15) != 0)
        return failed(DQ8_ERR_ARG, "%s: an array does not start at a multiple of its element's size (workspace: 16 bytes)", who);
    const size_t n_out = dq8::extent(a.tokens, a.out_token_stride, a.heads, a.out_head_stride, cache->dim, 2);
    const struct {
        const void *p;
        size_t n;
    } read[] = {{a.q, dq8::extent(a.tokens, a.q_token_stride, a.heads, a.q_head_stride, cache->dim, 2)},
                {cache->codes, dq8::cache_rows(cache) * cache->dim},
                {cache->scales, dq8::cache_rows(cache) * 4},
                {a.pages, a.batch * a.max_pages * 4},
                {a.lens, a.batch * 4},
                {a.starts, a.starts ? (a.batch + 1) * 4 : 0}};
    bool bad = workspace && meet(a.out, n_out, workspace, workspace_bytes);
    for (const auto &r : read) bad = bad || meet(a.out, n_out, r.p, r.n) || (workspace && meet(workspace, workspace_bytes, r.p, r.n));
    if (bad || !dq8::apart(a.tokens, a.out_token_stride, a.heads, a.out_head_stride, cache->dim))
        return failed(DQ8_ERR_ARG, "%s: out or workspace overlaps another array or itself", who);
    return DQ8_OK;
}

template <int DP, uint32_t ROWS, typename T>
int launch_join(const AttendArgs &k, const Shape &s, hipStream_t stream)
{
    // Few rows leave most compute units idle: a workgroup of sixteen wavefronts for each, to have its parts on their way at once (one sequence
    // of 16384: 22 us, with the other 33; 80 rows of each of 16 sequences of 4096: 55, with the other 44).
    if (s.few)
        hipLaunchKernelGGL((k_cache_join<DP, ROWS, 1, 1024, T>), dim3((unsigned)s.records, s.rows), dim3(1024), 0, stream, k);
    else
        hipLaunchKernelGGL((k_cache_join<DP, ROWS, 4, 256, T>), dim3((unsigned)s.records, (s.rows + 3) / 4), dim3(256), 0, stream, k);
    return dq8::after_launch_of("k_cache_join", stream);
}

template <int DP, int NT, typename T>
int launch_rows(const uint32_t *tab, const AttendArgs &k, const Shape &s, hipStream_t stream)
{
    hipLaunchKernelGGL((k_cache_attend<DP, NT, T>), dim3(s.groups), dim3(kAttendWg), 0, stream, tab, k);
    const int rc = dq8::after_launch_of("k_cache_attend", stream);
    return rc || !k.parts ? rc : launch_join<DP, 16 * NT, T>(k, s, stream);
}

template <int DP, int TH, typename T>
int launch_chunk(const uint32_t *tab, const AttendArgs &k, const Shape &s, hipStream_t stream)
{
    const unsigned splits = k.parts ? s.splits : 1;
    hipLaunchKernelGGL((k_cache_attend_chunk<DP, TH, T>), dim3((unsigned)s.jobs * splits), dim3(kChunkWg), 0, stream, tab, k, splits);
    const int rc = dq8::after_launch_of("k_cache_attend_chunk", stream);
    return rc || !k.parts ? rc : launch_join<DP, ChunkShape<DP, TH>::kRows, T>(k, s, stream);
}

template <typename T>
int launch(const uint32_t *tab, const AttendArgs &k, const Shape &s, hipStream_t stream)
{
    if (s.chunk) return s.dp == 64 ? launch_chunk<64, 2, T>(tab, k, s, stream) : s.dp == 128 ? launch_chunk<128, 2, T>(tab, k, s, stream) : launch_chunk<256, 1, T>(tab, k, s, stream);
    if (s.dp == 64) return s.rows16 == 1 ? launch_rows<64, 1, T>(tab, k, s, stream) : launch_rows<64, 2, T>(tab, k, s, stream);
    if (s.dp == 128) return s.rows16 == 1 ? launch_rows<128, 1, T>(tab, k, s, stream) : launch_rows<128, 2, T>(tab, k, s, stream);
    return launch_rows<256, 1, T>(tab, k, s, stream);
}

}  // namespace

extern "C" {

size_t dq8_cache_attention_workspace_bytes(const dq8_cache *cache, const dq8_attention *a)
{
    static const char who[] = "dq8_cache_attention_workspace_bytes";
    if (check_shape(who, 0, cache, a) || a->tokens == 0 || a->batch == 0) return 0;
    dq8::DeviceTables dev;
    if (dq8::device_tables(0, &dev)) return 0;
    const Shape s = shape_of(cache, *a, dev.cus);
    return workspace_bytes_of(s);
}

int dq8_cache_attention(int kind, const dq8_cache *cache, const dq8_attention *in, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    static const char who[] = "dq8_cache_attention";
    int rc = check_shape(who, kind, cache, in);
    if (rc) return rc;
    const dq8_attention &a = *in;
    if (a.tokens == 0 || a.batch == 0) return DQ8_OK;
    rc = check_arrays(who, cache, a, workspace, workspace_bytes);
    if (rc) return rc;
    dq8::DeviceTables dev;
    rc = dq8::device_tables(kind, &dev);
    if (rc) return rc;
    const Shape s = shape_of(cache, a, dev.cus);
    if (s.work >= dq8::kCacheLimit || s.jobs >= dq8::kCacheLimit / 256)  // the join's workgroups are of 256, a chunk's of 512 lanes
        return dq8::failed(DQ8_ERR_ARG, "%s: too much work for one call (tokens, heads and pages)", who);
    AttendArgs k;
    k.q = a.q, k.out = a.out, k.q_ts = a.q_token_stride, k.q_hs = a.q_head_stride, k.o_ts = a.out_token_stride, k.o_hs = a.out_head_stride;
    const size_t half = dq8::cache_rows(cache) / 2;
    k.k_codes = cache->codes, k.v_codes = cache->codes + half * cache->dim;
    k.k_scales = cache->scales, k.v_scales = cache->scales + half;
    k.pages = a.pages, k.lens = a.lens, k.starts = a.starts;
    k.tokens = (uint32_t)a.tokens, k.batch = (uint32_t)a.batch, k.each = a.starts ? 0 : (uint32_t)(a.tokens / a.batch);
    k.heads = (uint32_t)a.heads, k.kv_heads = (uint32_t)cache->kv_heads, k.group = k.heads / k.kv_heads, k.dim = (uint32_t)cache->dim;
    k.n_pages = (uint32_t)cache->pages, k.max_pages = (uint32_t)a.max_pages;
    k.page_shift = (uint32_t)__builtin_ctz((unsigned)cache->page_size);
    k.window = a.window;
    k.entry = kind == DQ8_LINEAR ? 127.0f * 256.0f : 1280.0f * 32.0f;
    k.factor = (float)((double)a.softmax_scale * 1.44269504088896340736 / (double)k.entry);  // (the product alone may leave binary32)
    k.rows = s.rows, k.in_a_row = s.chunk, k.by_wave = !s.chunk && s.records < s.jobs;
    k.n_records = nullptr, k.records = nullptr, k.sums = nullptr, k.parts = nullptr;
    if (s.parts && workspace && workspace_bytes >= workspace_bytes_of(s)) {
        char *w = static_cast<char *>(workspace);
        k.n_records = reinterpret_cast<uint32_t *>(w);
        k.records = reinterpret_cast<int4 *>(w) + 1;
        k.sums = reinterpret_cast<float2 *>(w + record_bytes(s));
        k.parts = reinterpret_cast<float *>(w + record_bytes(s) + sums_bytes(s));
    }
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    return a.type == DQ8_BFLOAT16 ? launch<__bf16>(dev.tab, k, s, stream) : launch<_Float16>(dev.tab, k, s, stream);
}

}  // extern "C"
