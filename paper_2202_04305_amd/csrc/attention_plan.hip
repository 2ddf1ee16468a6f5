// The inspector of attention over a stored pattern: which distinct columns the rows of a block store, and which of the pairs.
//
// A workgroup takes a block of rows and a window of columns.  It marks the columns that any of the rows stores in a bitmap in
// LDS, ranks them by a prefix sum over the bitmap's words, and, in its second run, writes the columns at their ranks and ORs a bit
// for every stored entry into the words of its row.  The counts of all (block, window) pairs are scanned in between.  Everything
// is a set or an OR, so the result does not depend on the order in which anything runs.
#include "attention.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWindow = 8192;            // columns of a window: a 32-bit word of the bitmap for each thread, times 2^wlog

template <typename PT, typename CT>
__global__ __launch_bounds__(kThreads) void rowptr_kernel(const PT *__restrict__ pos, const CT *__restrict__ rowid, int64_t stored, int64_t m,
                                                          int32_t *__restrict__ rowptr)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i > m) return;
    if (!rowid) { rowptr[i] = (int32_t)pos[i]; return; }
    int64_t lo = 0, hi = stored;                         // the first stored row at or behind i
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if ((int64_t)rowid[mid] < i) lo = mid + 1; else hi = mid;
    }
    rowptr[i] = (int32_t)pos[lo];
}

__global__ __launch_bounds__(kThreads) void crd32_kernel(const int64_t *__restrict__ crd, int64_t n, int32_t *__restrict__ out)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i < n) out[i] = (int32_t)crd[i];
}

__global__ __launch_bounds__(kThreads) void fill_kernel(uint32_t *__restrict__ p, int64_t n, uint32_t v)
{
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) p[i] = v;
}

__device__ int32_t first_at_least(const int32_t *__restrict__ crd, int32_t s, int32_t e, int64_t column)
{
    while (s < e) {
        const int32_t mid = s + ((e - s) >> 1);
        if ((int64_t)crd[mid] < column) s = mid + 1; else e = mid;
    }
    return s;
}

// Blocks of at most br rows that end where a row's stretch of columns and the next row's have no column in common, by one workgroup.
// row0[0 .. count]: their first rows, and m.
__global__ __launch_bounds__(1024) void blocks_kernel(const int32_t *__restrict__ rowptr, const int32_t *__restrict__ crd, int64_t m, int br,
                                                      int32_t *__restrict__ row0, unsigned long long *__restrict__ count)
{
    __shared__ int32_t s_start[16];
    __shared__ int s_count[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int32_t start_before = 0;                            // first row of the stretch that reaches into these rows
    int64_t before = 0;
    for (int64_t i0 = 0; i0 < m; i0 += 1024) {
        const int64_t i = i0 + threadIdx.x;
        bool apart = false;
        if (i > 0 && i < m) {
            const int32_t a = rowptr[i - 1], b = rowptr[i], c = rowptr[i + 1];
            apart = a < b && b < c && (crd[b] > crd[b - 1] || crd[c - 1] < crd[a]);
        }
        int32_t start = apart ? (int32_t)i : 0;          // running maximum: the first row of each row's stretch
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) { const int32_t o = __shfl_up(start, d, 64); if (lane >= d && o > start) start = o; }
        if (lane == 63) s_start[wave] = start;
        __syncthreads();
        int32_t carry = start_before;
        for (int w = 0; w < 16; ++w) { if (w < wave && s_start[w] > carry) carry = s_start[w]; if (s_start[w] > start_before) start_before = s_start[w]; }
        if (carry > start) start = carry;
        const bool first = i < m && (i - start) % br == 0;
        const uint64_t firsts = __builtin_amdgcn_ballot_w64(first);
        if (lane == 0) s_count[wave] = __builtin_popcountll(firsts);
        __syncthreads();
        int64_t at = before;
        for (int w = 0; w < 16; ++w) { at += w < wave ? s_count[w] : 0; before += s_count[w]; }
        if (first) row0[at + __builtin_popcountll(firsts & (((uint64_t)1 << lane) - 1))] = (int32_t)i;
        __syncthreads();
    }
    if (threadIdx.x == 0) { row0[before] = (int32_t)m; *count = (unsigned long long)before; }
}

// FILL = false: counts[block * windows + window] = distinct columns.  FILL = true: counts are scanned (exclusive), chunk0 is there;
// writes cols and bits.
template <bool FILL>
__global__ __launch_bounds__(kThreads) void window_kernel(int64_t first, const int32_t *__restrict__ rowptr, const int32_t *__restrict__ crd,
                                                          const int32_t *__restrict__ row0, int64_t m, int br,
                                                          int windows, int wlog, uint32_t *__restrict__ counts, const int32_t *__restrict__ chunk0,
                                                          int32_t *__restrict__ cols, uint32_t *__restrict__ bits)
{
    extern __shared__ uint32_t bitmap[];                 // 256 << wlog words, and FILL: as many ranks
    __shared__ int32_t s_lo[128], s_hi[128];
    __shared__ uint32_t s_wave[kThreads / 64];
    uint32_t *rank = bitmap + (kThreads << wlog);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t pair = first + blockIdx.x, block = pair / windows, window = pair % windows;
    const int64_t base = window * ((int64_t)kWindow << wlog), end = base + ((int64_t)kWindow << wlog);
    const int words = 1 << wlog;                         // of a thread
    for (int i = 0; i < words; ++i) bitmap[tid * words + i] = 0;
    if (tid < br) {
        const int64_t row = attn_first_row(row0, block, br, m) + tid;
        int32_t lo = 0, hi = 0;
        if (row < attn_first_row(row0, block + 1, br, m)) {
            lo = rowptr[row]; hi = rowptr[row + 1];
            if (windows > 1) { lo = first_at_least(crd, lo, hi, base); hi = first_at_least(crd, lo, hi, end); }
        }
        s_lo[tid] = lo; s_hi[tid] = hi;
    }
    __syncthreads();
    for (int r = wave; r < br; r += kThreads / 64)
        for (int32_t e = s_lo[r] + lane; e < s_hi[r]; e += 64) {
            const uint32_t at = (uint32_t)((int64_t)crd[e] - base);
            atomicOr(&bitmap[at >> 5], 1u << (at & 31));
        }
    __syncthreads();
    uint32_t mine = 0;
    for (int i = 0; i < words; ++i) mine += __builtin_popcount(bitmap[tid * words + i]);
    uint32_t upto = wave_inclusive_scan(mine, lane);
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    uint32_t before = 0, total = 0;
    for (int w = 0; w < kThreads / 64; ++w) { before += w < wave ? s_wave[w] : 0; total += s_wave[w]; }
    if (!FILL) {
        if (tid == 0) counts[pair] = total;
        return;
    }
    if (total == 0) return;                              // the whole workgroup
    // places of this window's columns: behind those of the block's windows before it
    const uint32_t place = (uint32_t)chunk0[block] * kAttnChunk + (counts[pair] - counts[block * windows]);
    uint32_t at = before + upto - mine;
    for (int i = 0; i < words; ++i) {
        const int w = tid * words + i;
        rank[w] = at;
        for (uint32_t left = bitmap[w]; left; left &= left - 1) cols[place + at++] = (int32_t)(base + w * 32 + __builtin_ctz(left));
    }
    __syncthreads();
    for (int r = wave; r < br; r += kThreads / 64) {
        const int32_t hi = s_hi[r];
        for (int32_t e0 = s_lo[r]; e0 < hi; e0 += 64) {
            const int32_t e = e0 + lane;
            uint32_t word = 0xffffffffu, bit = 0;        // no word: lanes behind the end
            if (e < hi) {
                const uint32_t c = (uint32_t)((int64_t)crd[e] - base);
                const uint32_t x = place + rank[c >> 5] + __builtin_popcount(bitmap[c >> 5] & ((1u << (c & 31)) - 1u));
                word = x >> 5; bit = 1u << (x & 31);
            }
            // neighbouring entries meet in a word: ORed together among the lanes first, the first lane of a run writes
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t w = __shfl_down(word, d, 64), b = __shfl_down(bit, d, 64);
                if (lane + d < 64 && w == word) bit |= b;
            }
            const uint32_t left = __shfl_up(word, 1, 64);
            if (word != 0xffffffffu && (lane == 0 || left != word)) atomicOr(&bits[((size_t)(word >> 1) * br + r) * 2 + (word & 1)], bit);
        }
    }
}

// chunks of every block (br > 1: from the scanned counts; br = 1: from the row lengths); stats[0] += chunks, stats[1] = max.
__global__ __launch_bounds__(kThreads) void chunks_kernel(const uint32_t *__restrict__ counts, int windows, const int32_t *__restrict__ rowptr,
                                                          int64_t nblocks, int32_t *__restrict__ chunk0, unsigned long long *__restrict__ stats)
{
    const int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    unsigned long long k = 0;
    if (b < nblocks) {
        const uint32_t cols = counts ? counts[(b + 1) * windows] - counts[b * windows] : (uint32_t)(rowptr[b + 1] - rowptr[b]);
        k = (cols + kAttnChunk - 1) / kAttnChunk;
    }
    if (b <= nblocks) chunk0[b] = (int32_t)k;
    unsigned long long sum = k, top = k;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        sum += __shfl_xor(sum, d, 64);
        const unsigned long long o = __shfl_xor(top, d, 64);
        top = o > top ? o : top;
    }
    if ((threadIdx.x & 63) == 0 && sum) { atomicAdd(&stats[0], sum); atomicMax(&stats[1], top); }
}

// behind a block's last column: that column again
__global__ __launch_bounds__(kThreads) void pad_kernel(const uint32_t *__restrict__ counts, int windows, const int32_t *__restrict__ chunk0,
                                                       int64_t nblocks, int32_t *__restrict__ cols)
{
    for (int64_t b = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); b < nblocks; b += (int64_t)gridDim.x * (kThreads / 64)) {
        const int64_t n = counts[(b + 1) * windows] - counts[b * windows], first = (int64_t)chunk0[b] * kAttnChunk, end = (int64_t)chunk0[b + 1] * kAttnChunk;
        const int64_t x = first + n + (threadIdx.x & 63);
        if (n > 0 && x < end) cols[x] = cols[first + n - 1];
    }
}

__global__ __launch_bounds__(kThreads) void state_kernel(const uint64_t *__restrict__ bits, const int32_t *__restrict__ chunk0,
                                                         const int32_t *__restrict__ row0, int64_t nblocks,
                                                         int64_t nchunks, int64_t m, int br, uint8_t *__restrict__ state)
{
    const int64_t x = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int subs = br / 32;
    if (x >= nchunks * subs) return;
    const int64_t chunk = x / subs, sub = x % subs;
    int64_t lo = 0, hi = nblocks;                        // the block: the last one that begins at or before the chunk
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) >> 1;
        if (chunk0[mid] <= chunk) lo = mid; else hi = mid;
    }
    const int64_t rows = attn_first_row(row0, lo + 1, br, m) - attn_first_row(row0, lo, br, m);
    uint64_t all = ~(uint64_t)0, any = 0;
    for (int r = 0; r < 32; ++r) {
        const uint64_t w = bits[chunk * br + sub * 32 + r];
        any |= w;
        if (sub * 32 + r < rows) all &= w;               // rows behind the block's last one leave no trace
    }
    state[x] = any == 0 ? 0 : all == ~(uint64_t)0 ? 2 : 1;
}

struct level_table { int32_t *item0[kAttnLevels]; };
__global__ __launch_bounds__(kThreads) void items_kernel(const int32_t *__restrict__ chunk0, int64_t nblocks, int levels, level_table t)
{
    const int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (b > nblocks) return;
    const int k = b < nblocks ? chunk0[b + 1] - chunk0[b] : 0;
    for (int l = 0; l < levels; ++l) {
        const int per = attn_level_chunks(l);
        t.item0[l][b] = b < nblocks ? (k <= per ? 1 : (k + per - 1) / per) : 0;
    }
}
// the blocks of several items, ascending, by one workgroup
__global__ __launch_bounds__(1024) void cut_blocks_kernel(const int32_t *__restrict__ item0, int64_t nblocks, int32_t *__restrict__ list,
                                                          unsigned long long *__restrict__ count)
{
    __shared__ int s_wave[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t before = 0;
    for (int64_t b0 = 0; b0 < nblocks; b0 += 1024) {
        const int64_t b = b0 + threadIdx.x;
        const bool cut = b < nblocks && item0[b + 1] - item0[b] > 1;
        const uint64_t some = __builtin_amdgcn_ballot_w64(cut);
        if (lane == 0) s_wave[wave] = __builtin_popcountll(some);
        __syncthreads();
        int64_t at = before;
        for (int w = 0; w < 16; ++w) { at += w < wave ? s_wave[w] : 0; before += s_wave[w]; }
        if (cut && list) list[at + __builtin_popcountll(some & (((uint64_t)1 << lane) - 1))] = (int32_t)b;
        __syncthreads();
    }
    if (threadIdx.x == 0) *count = (unsigned long long)before;
}
__global__ __launch_bounds__(kThreads) void stretches_kernel(const int32_t *__restrict__ item0, const int32_t *__restrict__ chunk0,
                                                             const int32_t *__restrict__ rowptr, const int32_t *__restrict__ row0, int64_t nblocks,
                                                             int64_t m, int br, int per, attn_stretch *__restrict__ items)
{
    const int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (b >= nblocks) return;
    const int32_t i0 = item0[b], i1 = item0[b + 1], k0 = chunk0[b], k1 = chunk0[b + 1];
    for (int32_t x = i0; x < i1; ++x) {
        attn_stretch s;
        s.block = (int32_t)b; s.chunk0 = k0;
        s.c0 = k0 + (x - i0) * per;
        s.c1 = k1 - s.c0 < per ? k1 : s.c0 + per;
        s.first = br == 1 ? rowptr[b] : k0 * kAttnChunk;
        s.count = br == 1 ? rowptr[b + 1] - rowptr[b] : (k1 - k0) * kAttnChunk;
        s.row0 = (int32_t)attn_first_row(row0, b, br, m);
        s.rows_whole = 2 * (int32_t)(attn_first_row(row0, b + 1, br, m) - s.row0) + (i1 - i0 == 1);
        items[x] = s;
    }
}

constexpr int64_t kGroups = 1 << 22;     // workgroups of a launch, where there may be more than one has (attn_launches)

unsigned blocks_for(int64_t n) { return (unsigned)(n > 0 ? ceil_div(n, kThreads) : 1); }

// Arrays that a plan under construction has taken; all of them go back unless the plan is finished.
struct plan_scope {
    const sp_mem &mem;
    sp_attn_plan *plan;
    explicit plan_scope(const sp_mem &m) : mem(m), plan(new sp_attn_plan()) { memset(plan, 0, sizeof(*plan)); }
    void *get(size_t bytes) {
        bytes = ((bytes ? bytes : 1) + 255) & ~(size_t)255;      // an allocator that is asked for nothing may give no address
        void *p = mem.get(bytes);
        if (p) plan->bytes += bytes;
        return p;
    }
    void drop() {
        if (!plan) return;
        mem.put(plan->rowptr); mem.put(plan->row0); mem.put(plan->crd_own); mem.put(plan->chunk0); mem.put(plan->cols); mem.put(plan->bits); mem.put(plan->state);
        for (int l = 0; l < kAttnLevels; ++l) { mem.put(plan->item0[l]); mem.put(plan->item[l]); mem.put(plan->cut_block[l]); }
        delete plan;
        plan = nullptr;
    }
    ~plan_scope() { drop(); }
};

struct cut { int windows = 1, wlog = 0; int64_t blocks = 0; };
// at most 2^20 pairs of a block and a window where windows of up to 2^17 columns allow it
cut cut_for(int64_t blocks, int64_t n)
{
    cut c;
    c.blocks = blocks;
    while (c.wlog < 4 && c.blocks * ceil_div(n, (int64_t)kWindow << c.wlog) > ((int64_t)1 << 20)) ++c.wlog;
    c.windows = (int)(n > 0 ? ceil_div(n, (int64_t)kWindow << c.wlog) : 1);
    return c;
}

// t: CSR / DCSR, or CSC for the transposed plan (its rows are t's columns; never br = 1, which would need t's crd to stay).
sp_status build_plan(const sp_tensor *t, const sp_mem &mem, bool transposed, hipStream_t st, sp_attn_plan **out)
{
    plan_scope scope(mem);
    sp_scratch tmp(mem);
    sp_attn_plan *p = scope.plan;
    const int64_t m = t->shape[transposed ? 1 : 0], n = t->shape[transposed ? 0 : 1], entries = t->nvalues;
    if (m >= ((int64_t)1 << 31) - 256 || n >= ((int64_t)1 << 31) - 256) return SP_ERR_TOO_LARGE;
    p->m = m; p->n = n;
    p->rowptr = (int32_t *)scope.get((size_t)(m + 1) * 4);
    if (!p->rowptr) return SP_ERR_ALLOC;
    const bool some = entries > 0;
    const void *rowid = t->enc.lt[0] == SP_COMPRESSED ? t->crd[0] : nullptr;
    const int64_t stored = rowid ? t->ncrd[0] : m;
#define SPMI_ROWPTR(PT, CT)                                                                                                       \
    hipLaunchKernelGGL((rowptr_kernel<PT, CT>), dim3(blocks_for(m + 1)), dim3(kThreads), 0, st, (const PT *)t->pos[1], (const CT *)rowid, \
                       stored, m, p->rowptr)
    if (!some) hipLaunchKernelGGL(fill_kernel, dim3(blocks_for((m + 4) / 4)), dim3(kThreads), 0, st, (uint32_t *)p->rowptr, m + 1, 0u);
    else if (t->enc.pw == 32 && t->enc.cw == 32) SPMI_ROWPTR(int32_t, int32_t);
    else if (t->enc.pw == 32) SPMI_ROWPTR(int32_t, int64_t);
    else if (t->enc.cw == 32) SPMI_ROWPTR(int64_t, int32_t);
    else SPMI_ROWPTR(int64_t, int64_t);
#undef SPMI_ROWPTR
    SP_HIP(hipGetLastError());
    p->crd = (const int32_t *)t->crd[1];
    if (some && t->enc.cw == 64) {
        p->crd_own = (int32_t *)scope.get((size_t)entries * 4);
        if (!p->crd_own) return SP_ERR_ALLOC;
        hipLaunchKernelGGL(crd32_kernel, dim3(blocks_for(entries)), dim3(kThreads), 0, st, (const int64_t *)t->crd[1], entries, p->crd_own);
        SP_HIP(hipGetLastError());
        p->crd = p->crd_own;
    }
    // Three ways to make blocks: of 128 rows, of 32, and of at most 128 within stretches of rows that have columns in common.  For
    // each: the distinct columns of its blocks by window, their chunks.
    struct way { int br; cut c; uint32_t *counts; int32_t *row0, *chunk0; unsigned long long chunks, most; } ways[3];
    unsigned long long *stats = (unsigned long long *)tmp.get(256);
    int32_t *row0 = (int32_t *)tmp.get((size_t)(m + 1) * 4);
    if (!stats || !row0) return SP_ERR_ALLOC;
    SP_TRY(spmi_fill_zero(stats, 256, st));
    unsigned long long within = 0;
    if (m > 0) {
        hipLaunchKernelGGL(blocks_kernel, dim3(1), dim3(1024), 0, st, p->rowptr, p->crd, m, 128, row0, stats + 8);
        SP_HIP(hipGetLastError());
        SP_HIP(hipMemcpyAsync(&within, stats + 8, 8, hipMemcpyDeviceToHost, st));
        SP_HIP(hipStreamSynchronize(st));
    }
    int tried = 2;
    ways[0].br = 128; ways[0].row0 = nullptr;
    ways[1].br = 32; ways[1].row0 = nullptr;
    ways[2].br = 128; ways[2].row0 = row0;
    if ((int64_t)within > ceil_div(m, 128)) tried = 3;
    for (int k = 0; k < tried; ++k) {
        way &w = ways[k];
        w.c = cut_for(w.row0 ? (int64_t)within : ceil_div(m, w.br), n);
        const int64_t pairs = w.c.blocks * w.c.windows;
        if (pairs >= ((int64_t)1 << 31) - 1) return SP_ERR_TOO_LARGE;
        w.counts = (uint32_t *)tmp.get((size_t)(pairs + 1) * 4);
        w.chunk0 = (int32_t *)tmp.get((size_t)(w.c.blocks + 1) * 4);
        if (!w.counts || !w.chunk0) return SP_ERR_ALLOC;
        hipLaunchKernelGGL(fill_kernel, dim3(1), dim3(kThreads), 0, st, w.counts + pairs, (int64_t)1, 0u);
        for (int64_t first = 0; first < pairs; first += kGroups)
            hipLaunchKernelGGL((window_kernel<false>), dim3((unsigned)(pairs - first < kGroups ? pairs - first : kGroups)), dim3(kThreads),
                               (size_t)(kThreads << w.c.wlog) * 4, st, first, p->rowptr, p->crd, w.row0, m, w.br, w.c.windows, w.c.wlog, w.counts, nullptr, nullptr, nullptr);
        SP_HIP(hipGetLastError());
        SP_TRY(spmi_exclusive_scan(w.counts, pairs + 1, 32, tmp, st));
        hipLaunchKernelGGL(chunks_kernel, dim3(blocks_for(w.c.blocks + 1)), dim3(kThreads), 0, st, w.counts, w.c.windows, p->rowptr, w.c.blocks, w.chunk0,
                           stats + 2 * k);
        SP_HIP(hipGetLastError());
    }
    unsigned long long host[6] = {0};
    SP_HIP(hipMemcpyAsync(host, stats, sizeof(host), hipMemcpyDeviceToHost, st));
    SP_HIP(hipStreamSynchronize(st));
    for (int k = 0; k < tried; ++k) { ways[k].chunks = host[2 * k]; ways[k].most = host[2 * k + 1]; }
    // What a block of rows costs for each of its chunks' columns: about 64 rows' worth of work to fetch it, and its rows' worth of work,
    // used or not.  A row by itself fetches its columns for itself, but makes one tile of all heads of a group, where a block makes one for
    // each head: it is the better choice until a block of 32 rows has every column twice on average, as long as the rows run at
    // once.  How many do depends on the heads, which a plan does not know; beyond 512 rows, beginning and ending one is taken to cost as
    // much as 400 columns (measured at these two: 4096 rows of 96 columns out of 65,536, 8
    // heads: 95 us in blocks of 32, 378 by themselves; 276 rows of 79 out of 17,791, 8 heads of one key head, f32: 54 and 38).
    // Whatever makes more blocks than a launch has workgroups is left out.
    auto fits = [](int64_t blocks) { return attn_launches(blocks, 256); };
    const int wide = tried == 3 && ways[2].chunks * 10 <= ways[0].chunks * 11 && fits(ways[2].c.blocks) ? 2 : 0;
    const double cost128 = (double)ways[wide].chunks * 64 * (64 + 128), cost32 = (double)ways[1].chunks * 64 * (64 + 32), cost1 = ((double)entries + 400.0 * (double)(m > 512 ? m - 512 : 0)) * (64 + 32) / 2;
    const way *chosen = nullptr;                         // null: rows by themselves
    if (transposed || cost1 > cost32 || cost1 > cost128 || !fits(m)) chosen = &ways[cost32 < cost128 && fits(ways[1].c.blocks) ? 1 : wide];
    p->br = chosen ? chosen->br : 1;
    p->nblocks = chosen ? chosen->c.blocks : m;
    p->chunk0 = (int32_t *)scope.get((size_t)(p->nblocks + 1) * 4);
    if (!p->chunk0) return SP_ERR_ALLOC;
    if (chosen && chosen->row0) {
        p->row0 = (int32_t *)scope.get((size_t)(p->nblocks + 1) * 4);
        if (!p->row0) return SP_ERR_ALLOC;
        SP_HIP(hipMemcpyAsync(p->row0, chosen->row0, (size_t)(p->nblocks + 1) * 4, hipMemcpyDeviceToDevice, st));
    }
    if (chosen) {
        SP_HIP(hipMemcpyAsync(p->chunk0, chosen->chunk0, (size_t)(p->nblocks + 1) * 4, hipMemcpyDeviceToDevice, st));
        p->nchunks = (int64_t)chosen->chunks; p->max_chunks = (int64_t)chosen->most;
    } else {
        SP_TRY(spmi_fill_zero(stats, 256, st));
        hipLaunchKernelGGL(chunks_kernel, dim3(blocks_for(m + 1)), dim3(kThreads), 0, st, nullptr, 1, p->rowptr, m, p->chunk0, stats);
        SP_HIP(hipGetLastError());
        SP_HIP(hipMemcpyAsync(host, stats, 16, hipMemcpyDeviceToHost, st));
        SP_HIP(hipStreamSynchronize(st));
        p->nchunks = (int64_t)host[0]; p->max_chunks = (int64_t)host[1];
    }
    SP_TRY(spmi_exclusive_scan(p->chunk0, p->nblocks + 1, 32, tmp, st));
    if (p->nchunks >= ((int64_t)1 << 25)) return SP_ERR_TOO_LARGE;       // 2^31 columns of blocks
    if (p->br > 1) {
        const size_t words = (size_t)p->nchunks * p->br;
        p->cols = (int32_t *)scope.get((size_t)p->nchunks * kAttnChunk * 4);
        p->bits = (uint64_t *)scope.get(words * 8);
        p->state = (uint8_t *)scope.get(words / 32);
        if (!p->cols || !p->bits || !p->state) return SP_ERR_ALLOC;
        if (p->nchunks > 0) {
            SP_TRY(spmi_fill_zero(p->bits, words * 8, st));
            const cut &c = chosen->c;
            const int64_t pairs = c.blocks * c.windows, pads = ceil_div(p->nblocks, kThreads / 64);
            for (int64_t first = 0; first < pairs; first += kGroups)
                hipLaunchKernelGGL((window_kernel<true>), dim3((unsigned)(pairs - first < kGroups ? pairs - first : kGroups)), dim3(kThreads),
                                   (size_t)(kThreads << c.wlog) * 8, st, first, p->rowptr, p->crd, p->row0, m, p->br, c.windows, c.wlog, chosen->counts, p->chunk0,
                                   p->cols, (uint32_t *)p->bits);
            hipLaunchKernelGGL(pad_kernel, dim3((unsigned)(pads < kGroups ? pads : kGroups)), dim3(kThreads), 0, st, chosen->counts, c.windows, p->chunk0,
                               p->nblocks, p->cols);
            hipLaunchKernelGGL(state_kernel, dim3(blocks_for(p->nchunks * (p->br / 32))), dim3(kThreads), 0, st, p->bits, p->chunk0, p->row0, p->nblocks,
                               p->nchunks, m, p->br, p->state);
            SP_HIP(hipGetLastError());
        }
    }
    p->levels = 1;
    while ((int64_t)attn_level_chunks(p->levels - 1) < p->max_chunks) ++p->levels;       // 2^25 chunks: 24 levels
    level_table table;
    memset(&table, 0, sizeof(table));
    for (int l = 0; l < p->levels; ++l) {
        p->item0[l] = table.item0[l] = (int32_t *)scope.get((size_t)(p->nblocks + 1) * 4);
        if (!p->item0[l]) return SP_ERR_ALLOC;
    }
    hipLaunchKernelGGL(items_kernel, dim3(blocks_for(p->nblocks + 1)), dim3(kThreads), 0, st, p->chunk0, p->nblocks, p->levels, table);
    SP_HIP(hipGetLastError());
    int32_t total[kAttnLevels];
    unsigned long long cut[kAttnLevels];
    unsigned long long *cuts_dev = (unsigned long long *)tmp.get(kAttnLevels * 8);
    if (!cuts_dev) return SP_ERR_ALLOC;
    for (int l = 0; l < p->levels; ++l) {
        SP_TRY(spmi_exclusive_scan(p->item0[l], p->nblocks + 1, 32, tmp, st));
        hipLaunchKernelGGL(cut_blocks_kernel, dim3(1), dim3(1024), 0, st, p->item0[l], p->nblocks, nullptr, cuts_dev + l);
        SP_HIP(hipMemcpyAsync(&total[l], p->item0[l] + p->nblocks, 4, hipMemcpyDeviceToHost, st));
    }
    SP_HIP(hipMemcpyAsync(cut, cuts_dev, (size_t)p->levels * 8, hipMemcpyDeviceToHost, st));
    SP_HIP(hipStreamSynchronize(st));
    for (int l = 0; l < p->levels; ++l) {
        p->items[l] = total[l];
        p->item[l] = (attn_stretch *)scope.get((size_t)(total[l] > 0 ? total[l] : 1) * sizeof(attn_stretch));
        p->cut[l] = (int64_t)cut[l];
        p->cut_block[l] = (int32_t *)scope.get((size_t)(cut[l] > 0 ? cut[l] : 1) * 4);
        if (!p->item[l] || !p->cut_block[l]) return SP_ERR_ALLOC;
        if (cut[l]) hipLaunchKernelGGL(cut_blocks_kernel, dim3(1), dim3(1024), 0, st, p->item0[l], p->nblocks, p->cut_block[l], cuts_dev + l);
        hipLaunchKernelGGL(stretches_kernel, dim3(blocks_for(p->nblocks)), dim3(kThreads), 0, st, p->item0[l], p->chunk0, p->rowptr, p->row0, p->nblocks,
                           m, p->br, attn_level_chunks(l), p->item[l]);
        SP_HIP(hipGetLastError());
    }
    SP_HIP(hipStreamSynchronize(st));                    // temporaries go back, and another stream may use the plan from now on
    if (p->br > 1) p->crd = nullptr;                     // not read any more; the transposed pattern's is about to go
    *out = scope.plan;
    scope.plan = nullptr;
    return SP_OK;
}

void free_plan(const sp_mem &mem, sp_attn_plan *p)
{
    if (!p) return;
    plan_scope scope(mem);
    delete scope.plan;
    scope.plan = p;                                      // goes back with the scope
}

}  // namespace

void spmi_free_attention(sp_tensor *t)
{
    sp_mem mem{t->alloc, t->free_, t->ctx};
    for (sp_attn_plan *&p : t->attention) { free_plan(mem, p); p = nullptr; }
}

size_t spmi_attention_bytes(const sp_tensor *t)
{
    size_t bytes = 0;
    for (const sp_attn_plan *p : t->attention) bytes += p ? p->bytes : 0;
    return bytes;
}

extern "C" sp_status sp_prepare_attention(sp_tensor *S, int grad, void *stream)
{
    if (!S) return SP_ERR_NULL;
    if (S->enc.rank != 2) return SP_ERR_RANK;
    if (S->enc.perm[0] != 0 || S->enc.lt[1] != SP_COMPRESSED) return SP_ERR_UNSUPPORTED;   // row-major with a compressed inner level
    if (S->nvalues >= ((int64_t)1 << 31)) return SP_ERR_TOO_LARGE;
    hipStream_t st = (hipStream_t)stream;
    if (S->attention[0] && (!grad || S->attention[1])) return SP_OK;
    if (spmi_recording(st)) return SP_ERR_UNSUPPORTED;   // it waits for the stream
    sp_tensor *T = nullptr;
    try {
        sp_mem mem{S->alloc, S->free_, S->ctx};
        if (!S->attention[0]) SP_TRY(build_plan(S, mem, false, st, &S->attention[0]));
        if (grad && !S->attention[1]) {
            sp_encoding enc = S->enc;
            enc.lt[0] = SP_DENSE; enc.lt[1] = SP_COMPRESSED;
            enc.perm[0] = 1; enc.perm[1] = 0;
            enc.pw = enc.cw = enc.pw_store = enc.cw_store = 32;
            if (S->shape[0] >= ((int64_t)1 << 31) - 256) return SP_ERR_TOO_LARGE;
            SP_TRY(spmi_repack(S, &enc, st, &T));
            const sp_status s = build_plan(T, mem, true, st, &S->attention[1]);
            sp_tensor_free(T);
            T = nullptr;
            SP_TRY(s);
        }
    } catch (...) {                                      // host memory ran out: no exception leaves a C entry
        sp_tensor_free(T);
        return SP_ERR_ALLOC;
    }
    return SP_OK;
}
