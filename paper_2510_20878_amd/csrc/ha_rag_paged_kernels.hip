// gfx950 kernels that keep the books of a paged cache on the device and write new rows to it.
//
//  k9_page_scan   one workgroup: which requests get the pages that their new rows need, in request order, from what is
//      free and what is given back; row and page offsets of every request (prefix sums); how the attention of the step is
//      cut into pieces.  With FILL it also does k9_page_fill's work.
//  k9_page_fill   one thread per row (its slot, its position, and the page table's entry where a row opens a page), per
//      page given back, and per piece of attention.
//  k10_append     16 bytes per thread: the new rows' keys and values to their slots.
//
// The formulas.  Request r holds t rows in b = ceil(t / P) pages and adds d rows (drops -d if d < 0):
//   need = ceil((t + d) / P) - b, freed = b - ceil(max(t + d, 0) / P);
//   r is granted if its rows fit the table and the step's row arrays, and the needs of the requests up to it fit what can be
//   taken: free pages + all pages given back.
// The j-th page taken is the j-th page given back while there are any (pages given back go to the top of the free stack,
// the first one uppermost), then the top of what was free.  So taking reads nothing that giving back writes, and both
// can go on side by side.
//
// Bound: latency.  Every sum over the requests is a barrier, every table entry a dependent load, so there are three sums (by lane
// steps and one trip through LDS each), and where the step is small everything happens in one launch.  us a step: 4 requests that
// decode 5.8, 256 requests with 10,000 rows, pages given back and a pool that runs dry 12, 1,024 requests' first chunks (355,000
// rows: 2.8 MB of slots and positions) 13.  One launch for up to 2,048 rows: 1,300 rows 8.7 instead of 9.5, 2,600 rows 9.4 to
// 12.7 instead of 9.6 to 11.2.
#include "ha_rag_paged.h"

namespace ha_rag {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kScanThreads = 1024;

// Sums stop at 2^32 - 1 instead of wrapping: every sum is compared with something smaller, or known to stay below.
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// x + the value of the lane that CTRL names; 0 where there is none, or where the row of 16 lanes is not in MASK
template <int CTRL, int MASK>
__device__ __forceinline__ uint32_t add_lane(uint32_t x)
{
    return add_sat(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, MASK, 0xF, true));
}

// inclusive prefix sums over the wave, by steps within rows of 16 lanes (row_shr 1, 2, 4, 8), then from row to row (row_bcast 15,
// 31): no trip through LDS
__device__ __forceinline__ uint32_t wave_inclusive(uint32_t x)
{
    x = add_lane<0x111, 0xF>(x);
    x = add_lane<0x112, 0xF>(x);
    x = add_lane<0x114, 0xF>(x);
    x = add_lane<0x118, 0xF>(x);
    x = add_lane<0x142, 0xA>(x);
    return add_lane<0x143, 0xC>(x);
}

// the wave's largest value, in lane 63
__device__ __forceinline__ uint32_t wave_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, true));
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, true));
}

// Exclusive prefixes (in x) and sums (in all) of N values over the workgroup's threads.  lds: one row per wave, of this call alone.
template <int N>
__device__ __forceinline__ void block_exclusive(uint32_t (&x)[N], uint32_t (*lds)[N], uint32_t (&all)[N])
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    uint32_t before[N] = {};
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const uint32_t inc = wave_inclusive(x[n]);
        if (lane == 63) lds[wave][n] = inc;
        const uint32_t left = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)inc, 0x138, 0xF, 0xF, true);  // of the lane before
        x[n] = lane == 0 ? 0u : left;
        all[n] = 0u;
    }
    __syncthreads();
    for (uint32_t w = 0; w < waves; ++w)
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t s = lds[w][n];
            if (w < wave) before[n] = add_sat(before[n], s);
            all[n] = add_sat(all[n], s);
        }
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] = add_sat(x[n], before[n]);
}

// index of the first of ex[1..n] above i, i.e. the r with ex[r] <= i < ex[r + 1] (empty ranges passed over); n if none
template <class T>
__device__ __forceinline__ uint32_t find_range(const T *ex, uint32_t n, T i)
{
    uint32_t lo = 0, hi = n;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) >> 1;
        if (ex[mid + 1] <= i) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

struct FillView {  // prefix sums of the requests, in LDS
    const int32_t *start;
    const uint32_t *freed_ex, *line_ex;  // pages given back; tiles (whole) or units (cut) of the attention
};

__device__ __forceinline__ uint32_t freed_page(const K9Params &p, const FillView &v, const StepReq *req, uint32_t f)
{
    const uint32_t r = min(find_range(v.freed_ex, p.n_requests, f), p.n_requests - 1u);
    const uint32_t col = req[r].kept + (f - v.freed_ex[r]);
    return p.table[(uint64_t)r * p.n_table + min(col, p.n_table - 1u)];
}

__device__ __forceinline__ void fill(const K9Params &p, const FillView &v, const StepReq *req, const StepHdr &h, uint32_t id, uint32_t n_threads)
{
    const uint32_t R = p.n_requests, P = p.page_tokens;
    for (uint32_t i = id; i < p.n_rows; i += n_threads) {
        int32_t slot = -1, pos = -1;
        const uint32_t r = find_range(v.start, R, (int32_t)i);
        if (r < R) {
            const StepReq q = req[r];
            if (q.granted) {
                const uint32_t at = q.t + (i - (uint32_t)v.start[r]), col = at / P, row = at - col * P;
                uint32_t page;
                if (col < q.before) {
                    page = p.table[(uint64_t)r * p.n_table + col];
                } else {
                    const uint32_t j = q.need_ex + col - q.before;
                    page = j < h.n_freed ? freed_page(p, v, req, j) : p.free_pages[h.height - 1u - (j - h.n_freed)];
                    if (row == 0) p.table[(uint64_t)r * p.n_table + col] = page;
                }
                pos = (int32_t)at;
                if (page < p.n_pages) slot = (int32_t)(page * P + row);
            }
        }
        p.slots[i] = slot;
        if (p.positions) p.positions[i] = pos;
    }
    for (uint32_t f = id; f < h.n_freed; f += n_threads) {
        const uint32_t at = h.height + h.n_freed - 1u - f;
        if (at < p.n_pages) p.free_pages[at] = freed_page(p, v, req, f);
    }
    StepStart *starts = reinterpret_cast<StepStart *>(p.plan + p.lay.starts);
    for (uint32_t w = id; w < h.n_wgs; w += n_threads) {
        const uint32_t at = h.run ? w * h.run : w;
        const uint32_t r = min(find_range(v.line_ex, R, at), R - 1u), off = at - v.line_ex[r];
        StepStart s;
        s.work = req[r].work;
        const uint32_t units = req[r].units + kTileUnits;
        if (h.run) {
            s.tile = off / units;
            s.unit = off - s.tile * units;
            s.n_units = min(h.run, v.line_ex[R] - at);
        } else {
            s.tile = req[r].tiles - 1u - off;
            s.unit = 0;
            s.n_units = units;
        }
        starts[w] = s;
    }
    uint32_t *counters = reinterpret_cast<uint32_t *>(p.plan + p.lay.counters);
    if (h.run)
        for (uint32_t k = id; k < p.lay.target * p.n_kv_heads; k += n_threads) counters[k] = 0u;
}

// K requests per thread (R <= K * threads).  FILL: K is 1
template <uint32_t K, bool FILL>
__global__ __launch_bounds__(kScanThreads) void k9_page_scan(const K9Params p)
{
    extern __shared__ uint32_t dyn[];  // FILL: requests, then row starts, pages given back, tiles or units: R + 1 each
    __shared__ uint32_t sum2[kScanThreads / 64][2], sum1[kScanThreads / 64][1], sum6[kScanThreads / 64][6], longest;
    const uint32_t tid = threadIdx.x, R = p.n_requests, P = p.page_tokens;
    const uint32_t room = p.n_table * P;

    uint32_t t[K], before[K], freed[K], need[K], add[K], start[K];
    int32_t d[K];
    bool fits[K];
    uint32_t x2[2] = {}, all2[2];
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) {
        const uint32_t r = tid * K + k;
        const int32_t held = r < R ? p.n_tokens[r] : 0;
        d[k] = r < R ? p.n_new[r] : 0;
        t[k] = min((uint32_t)max(held, 0), room);
        add[k] = (uint32_t)max(d[k], 0);
        const uint32_t drop = d[k] < 0 ? 0u - (uint32_t)d[k] : 0u, left = t[k] > drop ? t[k] - drop : 0u;
        before[k] = (t[k] + P - 1u) / P;
        freed[k] = before[k] - (left + P - 1u) / P;
        x2[0] = add_sat(x2[0], add[k]);
        x2[1] += freed[k];
    }
    const uint32_t height = (uint32_t)min(max(*p.n_free, 0), (int32_t)p.n_pages);
    if (tid == 0) longest = 0;
    block_exclusive(x2, sum2, all2);
    uint32_t end = x2[0], freed_ex = x2[1];
    const uint32_t n_add = all2[0], n_freed = all2[1], avail = height + n_freed;

    uint32_t x1[1] = {}, all1[1];
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) {
        start[k] = min(end, p.n_rows);
        end = add_sat(end, add[k]);
        fits[k] = add[k] <= room - t[k] && (add[k] == 0 || end <= p.n_rows);
        need[k] = fits[k] ? (t[k] + add[k] + P - 1u) / P - before[k] : 0u;
        x1[0] += need[k];
    }
    block_exclusive(x1, sum1, all1);
    uint32_t need_ex = x1[0];

    const uint32_t share = p.n_q_heads / p.n_kv_heads;
    uint32_t after[K], tiles[K], tile_rows[K], units[K], rows[K], my_need_ex[K];
    bool granted[K];
    uint32_t x6[6] = {}, all6[6], my_longest = 0;
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) {
        const uint32_t r = tid * K + k;
        my_need_ex[k] = need_ex;
        need_ex += need[k];
        granted[k] = fits[k] && (need[k] == 0 || need_ex <= avail);
        const uint32_t drop = d[k] < 0 ? 0u - (uint32_t)d[k] : 0u;
        after[k] = d[k] < 0 ? (t[k] > drop ? t[k] - drop : 0u) : granted[k] ? t[k] + add[k] : t[k];
        rows[k] = r < R ? min(add_sat(start[k], add[k]), p.n_rows) - start[k] : 0u;
        tile_rows[k] = p.lay.rows_only || rows[k] * share <= 16u ? 16u : kStepTileRows;
        tiles[k] = (rows[k] * share + tile_rows[k] - 1u) / tile_rows[k];
        const uint32_t seen = granted[k] ? (after[k] + p.unit - 1u) / p.unit : 0u;
        units[k] = max(seen, 1u);
        x6[0] += granted[k] ? need[k] : 0u;
        x6[1] += tiles[k] != 0;
        x6[2] += tiles[k];
        x6[3] = add_sat(x6[3], (uint32_t)min((uint64_t)tiles[k] * (units[k] + kTileUnits), 0xFFFFFFFFull));
        if (tiles[k]) my_longest = max(my_longest, units[k] + kTileUnits);
        x6[4] = add_sat(x6[4], tiles[k] ? seen : 0u);
        x6[5] = add_sat(x6[5], tile_rows[k] == 16u ? tiles[k] * (units[k] + kTileUnits) : 0u);
    }
    my_longest = wave_max(my_longest);
    if ((tid & 63u) == 63u) atomicMax(&longest, my_longest);
    block_exclusive(x6, sum6, all6);
    uint32_t work_ex = x6[1];
    const uint32_t n_taken = all6[0], n_tiles = all6[2], n_units = all6[3], n_seen = all6[4], n_units16 = all6[5];
    // Whole tiles, or runs.  All figures: 8 KV heads of 128, 4 query heads each, pages of 16 rows, us cut / whole in a graph.
    // Tiles of 16 rows, whose partial results are small: whole from more than 3 times as many as workgroups that run at once (64 a
    // head), if they count less than 12 units on average (550 rows).  224 tiles of 100 rows 29.7 / 25.1, of 400 73.5 / 69.4, of 550
    // 93.1 / 88.3, of 1,500 225 / 219, of 2,500 359 / 373; 192 of 100 24.3 / 22.2, of 400 59.4 / 59.5, of 1,000 127 / 129; 300 of 1,500 299 / 302;
    // 1,000 of 100 129 / 117, of 400 315 / 304.  Just beyond the borders the choice costs 5 to 9 %; far fewer tiles come out
    // even only where their number happens to go into that of the workgroups (160 of 100 rows 24.3 / 20.1, 100 of 1,500 108 / 115).
    // Large ones (64 KiB of partial results each way) where there are more than workgroups and none takes longer than a run
    // would: four chunks of 1,000 rows over 1,000 144 / 133, 16 of 160 over 1,000 84 / 75, 5 of 1,000 over 100 107 / 84.  The longest may
    // be 1.0 of a run (three of 1,000 over 1,500 to 6,000 253 / 226) and 1.2 (16 of 160 over 500 to 2,000 94 / 85) before it is even (1.3, 40 of 48
    // rows over 500 to 2,000 83 / 86) and lost (1.5, 70 of 30 rows over 1,000 to 4,000 174 / 187): the border is on the safe side.
    // That rule is for steps whose large tiles have two thirds of the units: 32 requests of one row and 16 of 100, over 500, 56 / 43.  With
    // fewer, the few long ones may end last (16 of one row and one of 100, over 2,500, 48 to 55 / 60) or not (64 and 16, over 500, 61 / 53;
    // 64 and 8 49 / 49): all cut.
    // (A line that 32 bits do not hold is not cut.)
    const bool small = n_units16 >= n_units / 3u;
    const bool whole = n_units == 0xFFFFFFFFu || (small ? n_tiles > kManyTiles * p.lay.target && n_units / 12u < n_tiles
                                                        : n_tiles > p.lay.target && longest <= n_units / p.lay.target);
    // Streaming (tiles of 16 rows, pages of whole blocks) is fastest with one workgroup a compute unit; a second one hides what happens
    // between two tiles, and matters where tiles are short and a workgroup has several.  us with one / two: 32 requests of 400
    // rows 14.3 / 19.4, of 5,000 102 / 114, 40 of 1,500 43.3 / 44.6, 48 of 1,000 36.9 / 39.9, 64 of 200 17.0 / 15.4, of 1,000 44.9 / 43.7, of 1,500
    // 64.1 / 65.7, of 2,500 101 / 105, 160 of 200 35.4 / 30.5, of 1,000 110 / 115, of 2,500 248 / 262, 300 of 700 154 / 152, of 1,500
    // 288 / 299.  So: one where there are few tiles (five eighths of the workgroups that run at once; it is even between that and as many)
    // and where they are long (32 units on average; it is even between 14 and 27).  A few large tiles among them gain from two (64 requests
    // of one row and 4 of 100, over 2,500, 154 / 140).  Pages of 12 rows: 48 requests of 4,000 rows, 32 heads, 512 / 499.  Large tiles
    // alone (40 of them, 11 units each) 57 / 50.
    const bool one = P % 16u == 0 && small && (n_tiles <= p.lay.target * 5u / 8u || n_units / 32u >= n_tiles);
    const uint32_t target = one ? max(p.lay.target / 2u, 1u) : p.lay.target;
    const uint32_t run = whole ? 0u : max(n_units / target + (n_units % target != 0u), kLeastRun);
    const uint32_t n_wgs = whole ? n_tiles : n_units / run + (n_units % run != 0u);
    uint32_t line_ex = whole ? x6[2] : x6[3];

    StepReq *req = FILL ? reinterpret_cast<StepReq *>(dyn) : reinterpret_cast<StepReq *>(p.plan + p.lay.req);
    uint32_t *g_freed = reinterpret_cast<uint32_t *>(p.plan + p.lay.freed_ex);
    uint32_t *g_line = reinterpret_cast<uint32_t *>(p.plan + p.lay.line_ex);
    StepWork *work = reinterpret_cast<StepWork *>(p.plan + p.lay.work);
    uint32_t *l_arrays = dyn + R * (uint32_t)(sizeof(StepReq) / 4u);
    int32_t *l_start = reinterpret_cast<int32_t *>(l_arrays);
    uint32_t *l_freed = l_arrays + (R + 1u), *l_line = l_arrays + 2u * (R + 1u);
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) {
        const uint32_t r = tid * K + k;
        if (r <= R) {  // entry R: the sums
            p.row_start[r] = (int32_t)start[k];
            if (FILL) {
                l_start[r] = (int32_t)start[k];
                l_freed[r] = freed_ex;
                l_line[r] = line_ex;
            } else {
                g_freed[r] = freed_ex;
                g_line[r] = line_ex;
            }
        }
        if (r < R) {
            req[r] = StepReq{t[k], before[k], before[k] - freed[k], my_need_ex[k], granted[k], work_ex, tiles[k], units[k]};
            p.n_tokens_after[r] = (int32_t)after[k];
            if (p.refused) p.refused[r] = !granted[k] && d[k] > 0;
            if (tiles[k])
                work[work_ex] = StepWork{r, start[k], rows[k], granted[k] ? after[k] : 0u, tile_rows[k], tiles[k], units[k], line_ex};
        }
        freed_ex += freed[k];
        work_ex += tiles[k] != 0;
        line_ex += whole ? tiles[k] : tiles[k] * (units[k] + kTileUnits);
    }
    StepHdr h = {};
    h.magic = kStepMagic;
    h.n_requests = R;
    h.n_rows = p.n_rows;
    h.n_q_heads = p.n_q_heads;
    h.n_kv_heads = p.n_kv_heads;
    h.head_dim = p.head_dim;
    h.n_wgs = n_wgs;
    h.run = run;
    h.unit = p.unit;
    h.past = (uint64_t)n_seen * p.unit * p.n_layers * p.n_kv_heads * p.head_dim * 4u > kPastBytes;
    h.n_freed = n_freed;
    h.height = height;
    if (tid == 0) {
        *reinterpret_cast<StepHdr *>(p.plan) = h;
        *p.n_free_after = (int32_t)min(avail - n_taken, p.n_pages);
        if (K * blockDim.x == R) {  // no thread has an entry R of its own
            const int32_t rows_all = (int32_t)min(n_add, p.n_rows);
            const uint32_t line_all = whole ? n_tiles : n_units;
            p.row_start[R] = rows_all;
            if (FILL) l_start[R] = rows_all, l_freed[R] = n_freed, l_line[R] = line_all;
            else g_freed[R] = n_freed, g_line[R] = line_all;
        }
    }
    if (FILL) {
        __syncthreads();
        fill(p, FillView{l_start, l_freed, l_line}, req, h, tid, blockDim.x);
    }
}

__global__ __launch_bounds__(kScanThreads) void k9_page_fill(const K9Params p)
{
    extern __shared__ uint32_t dyn[];
    const uint32_t R = p.n_requests;
    int32_t *l_start = reinterpret_cast<int32_t *>(dyn);
    uint32_t *l_freed = dyn + (R + 1u), *l_line = dyn + 2u * (R + 1u);
    const uint32_t *g_freed = reinterpret_cast<const uint32_t *>(p.plan + p.lay.freed_ex);
    const uint32_t *g_line = reinterpret_cast<const uint32_t *>(p.plan + p.lay.line_ex);
    for (uint32_t r = threadIdx.x; r <= R; r += kScanThreads) {
        l_start[r] = p.row_start[r];
        l_freed[r] = g_freed[r];
        l_line[r] = g_line[r];
    }
    const StepHdr h = *reinterpret_cast<const StepHdr *>(p.plan);
    __syncthreads();
    fill(p, FillView{l_start, l_freed, l_line}, reinterpret_cast<const StepReq *>(p.plan + p.lay.req), h, blockIdx.x * kScanThreads + threadIdx.x, gridDim.x * kScanThreads);
}

// Bound by HBM: 12,976 rows of 4 KiB in 19.4 us, 52,000 in 64 (6.7 TB/s read and written; with ordinary stores and an eighth of the
// workgroups, which then go round, 89).
__global__ __launch_bounds__(256) void k10_append(const K10Params p)
{
    const uint32_t octets = p.head_dim / 8u, tile = p.n_kv_heads * octets, per_row = 2u * tile;  // 16-byte pieces
    const uint64_t n = (uint64_t)p.n_rows * per_row;
    for (uint64_t x = (uint64_t)blockIdx.x * 256u + threadIdx.x; x < n; x += (uint64_t)gridDim.x * 256u) {
        const uint32_t i = (uint32_t)(x / per_row), c = (uint32_t)(x - (uint64_t)i * per_row);
        const int32_t slot = p.slots[i];
        if (slot < 0) continue;
        const uint32_t kv = c >= tile, hc = c - kv * tile, h = hc / octets, o = hc - h * octets;
        const uint32_t page = (uint32_t)slot / p.page_tokens, row = (uint32_t)slot - page * p.page_tokens;
        if (page >= p.n_pages) {
            if (p.bad_pages) atomicAdd(p.bad_pages, 1u);
            continue;
        }
        const uint8_t *src = kv ? p.v + i * p.v_row + h * p.v_head : p.k + i * p.k_row + h * p.k_head;
        uint8_t *dst = p.base + page * p.page_stride + ((uint64_t)(p.layer * 2u + kv) * p.n_kv_heads + h) * p.tile_stride +
                       (uint64_t)row * p.head_dim * 2u;
        __builtin_nontemporal_store(*reinterpret_cast<const u32x4 *>(src + o * 16u), reinterpret_cast<u32x4 *>(dst + o * 16u));
    }
}

}  // namespace

hipError_t launch_k9(const K9Params &p, hipStream_t stream)
{
    const uint32_t lds = 3u * (p.n_requests + 1u) * 4u, lds_req = p.n_requests * (uint32_t)sizeof(StepReq);
    const bool together = p.n_rows <= 2048u && p.n_requests <= kScanThreads;
    // few requests and rows: fewer waves to wait for at each of the three sums
    const uint32_t threads = p.n_requests <= 256u && p.n_rows <= 512u ? 256u : kScanThreads;
    if (together) k9_page_scan<1, true><<<1, threads, lds + lds_req, stream>>>(p);
    else if (p.n_requests <= kScanThreads) k9_page_scan<1, false><<<1, kScanThreads, 0, stream>>>(p);
    else k9_page_scan<4, false><<<1, kScanThreads, 0, stream>>>(p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || together) return e;
    const uint32_t blocks = (uint32_t)(((uint64_t)p.n_rows + kScanThreads - 1u) / kScanThreads);
    k9_page_fill<<<blocks < 512u ? blocks : 512u, kScanThreads, lds, stream>>>(p);
    return hipGetLastError();
}

hipError_t launch_k10(const K10Params &p, hipStream_t stream)
{
    const uint64_t n = (uint64_t)p.n_rows * 2u * p.n_kv_heads * (p.head_dim / 8u), blocks = (n + 255u) / 256u;
    k10_append<<<(uint32_t)(blocks < 64u * kChipCUs ? blocks : 64u * kChipCUs), 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace ha_rag
