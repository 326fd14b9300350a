// gfx950 kernels for attention of a step's new rows over what their requests hold in a paged cache.
//
//  k11_attend_rows    steps whose tiles are all of 16 query rows: decode
//  k11_attend_mixed   steps with tiles of 16 and of 128 query rows: questions, chunks of a prefill, and decode next to them
//
// One workgroup of four waves per run of the plan (StepHdr in ha_rag_paged.h: how a step is shared out) and KV head; heads change
// fastest, so that with 8 heads each XCD's L2 holds one head's keys and values for all the tiles that read them.
//
// The formulas.  Query rows of a request and KV head: row m = (new row m / G, query head m % G of the G that share the KV head);
// new row i of n sees the tokens below held - n + i + 1.  With s = q k scale over these, one pass keeps per row a reference r (the
// largest s so far, moved only when a score exceeds it by kLazyMaxSlack), l = sum exp(s - r) and o = sum exp(s - r) v:
// out = o / l, lse = r + log l.  Two such results over different tokens join as r = max, o = o1 exp(r1 - r) + o2 exp(r2 - r), l
// likewise: waves of a workgroup, pieces of a tile and the prior attention are joined so.  Scores, references and sums are
// binary32.  The weights are rounded to BF16 because the matrix instructions that multiply v take no more; out is divided by
// the sum of the rounded ones (so rounding does not scale it), the lse keeps the unrounded sum.  Against 64 bits out is off by 1.9e-3 of its
// norm, of which 1.6e-3 to 1.7e-3 are its own rounding to BF16; a second product with what the weights lose would save the rest for twice
// the matrix instructions of O, which tiles of 128 rows have no room for and which would leave the two forms unlike.
//
// Tiles of 16 rows (attend_rows).  Bound: HBM.  Every wave reads its own share of the tokens, 16 at a time, straight into
// registers, one block on its way while one is worked on; no LDS until the waves are joined.  Scores are computed
// transposed, S^T = K Q^T (16x16x32 MFMA): lane (c = lane / 16, n = lane % 16) supplies of K token n, dims 32 y + 8 c .. + 7, which
// is how rows lie in memory, and receives the scores of tokens 4 c .. 4 c + 3 for query row n: the layout in which P^T is
// the second operand of O^T = V^T P^T (16x16x16 MFMA).  V's operand is 4 tokens of one dim: the lane loads D / 16 neighbouring
// dims of its tokens 4 c + i and regroups them by pairs.  Measured: 32 requests of 5,130 rows, 8 KV heads of 128, 105 us (6.4 TB/s);
// one of 131,072 rows 88 us (6.1); 48 of 900 rows, 32 KV heads, pages of 12 rows, 129 us (5.5).  Heads of 64 and 96, 32 requests of 5,130
// rows: 62.5 us (5.4) and 90 us (5.6).
//
// Tiles of 128 rows (attend_tiles).  Bound: the matrix and the vector unit, which share their SIMD's issue.  A wave owns 32 rows
// (32x32x16 MFMA, S^T and O^T as above); keys and values of 64 tokens at a time go to LDS past the registers for all four waves.
// Measured: chunks of 517 to 1,024 rows over up to 5,120, 64 query heads on 8, 315 to 345 us, by card (850 to 925 TFLOP/s of 1,256 that a product
// of 8,192 x 8,192 matrices reaches); 24 questions of 5 to 64 rows over 16 to 2,112, 43 us in a graph.  Heads of 64 and 96, chunks of 1,024 over 4,096: 709
// and 843 TFLOP/s (of 128: 927), since exponentials are as many and products fewer.  Where that goes, of 320 us with parts
// left out: exponentials and sums 35, the second product 68, the loads to LDS 40; the matrix unit is busy 41 % of the
// clocks, the vector unit 49 %, LDS 21 % and free of bank conflicts.
#include "ha_rag_attend_dev.h"
#include "ha_rag_paged.h"

namespace ha_rag {

namespace {

// The kernel's arguments where they lie.  late() is the same place again, unknown to the compiler: what is read through it is read then and
// there, not at the start and then kept in scalar registers (of which 114 were spilled to lanes of vector registers, 28 of them
// in the loop).
typedef const K11Params __attribute__((address_space(4))) *Params;
__device__ __forceinline__ Params late(Params p)
{
    uint64_t a = (uint64_t)p;
    asm volatile("" : "+s"(a));
    return (Params)a;
}

typedef uint32_t u32x3 __attribute__((ext_vector_type(3), aligned(4)));
typedef uint8_t __attribute__((address_space(1))) *gout;

template <bool PAST, class T>
__device__ __forceinline__ T ldg_of(gbytes p)
{
    if (PAST) return __builtin_nontemporal_load((const T __attribute__((address_space(1))) *)p);
    return *(const T __attribute__((address_space(1))) *)p;
}

// NW dwords from global memory, at an address of 4-byte (NW odd), 8-byte or 16-byte alignment
template <int NW, bool PAST>
__device__ __forceinline__ void ldg_words(gbytes p, uint32_t (&w)[NW])
{
    if constexpr (NW == 2) {
        const u32x2 a = ldg_of<PAST, u32x2>(p);
        w[0] = a.x, w[1] = a.y;
    } else if constexpr (NW == 3) {
        const u32x3 a = ldg_of<PAST, u32x3>(p);
        w[0] = a.x, w[1] = a.y, w[2] = a.z;
    } else {
        static_assert(NW % 4 == 0, "dwords per row and lane");
#pragma unroll
        for (int k = 0; k < NW / 4; ++k) {
            const u32x4 a = ldg16_of<PAST>(p + 16 * k);
            w[4 * k] = a.x, w[4 * k + 1] = a.y, w[4 * k + 2] = a.z, w[4 * k + 3] = a.w;
        }
    }
}

template <int D>
struct RowsBlock {              // what a lane loads for 16 tokens
    u32x4 k[D / 32];            // token n, dims 32 y + 8 c ..
    uint32_t v[4][D / 32];      // tokens 4 c + i, dims n D / 16 .. (D / 32 dwords)
};


// natural logarithm of the sum of exponentials, from its base-2 reference and the sum relative to it
__device__ __forceinline__ float lse_of(float m2, float l)
{
    return l > 0.0f ? m2 * 0.69314718055994531f + __logf(l) : neg_inf();
}

// What a row of an attention becomes with another over other keys: out = o * a + prior * b
struct Merged {
    float a, b, lse;
};
__device__ __forceinline__ Merged merge_with(float lse, float prior_lse)
{
    if (!(prior_lse > neg_inf())) return Merged{1.0f, 0.0f, lse};  // there is no other, whatever its output says
    const float big = __builtin_fmaxf(lse, prior_lse), ea = __expf(lse - big), eb = __expf(prior_lse - big), inv = 1.0f / (ea + eb);
    return Merged{ea * inv, eb * inv, big + __logf(ea + eb)};
}

// N quads of normalised rows (o[k]: dims 4 dq[k] .. of query head hq[k] of row row[k], a row of the step also where it is
// not live) are merged with the prior attention and stored.  What they read is asked for before any of it is used: one wait
// for all.  ONE: all quads are of one row.
template <int D, int N, bool ONE>
__device__ __forceinline__ void store_quads(Params p, const uint32_t (&row)[N], const uint32_t (&hq)[N], const uint32_t (&dq)[N],
                                            const bool (&live)[N], f32x4 (&o)[N], float (&lse)[N])
{
    if (p->prior_out) {
        f32x4 w[N];
        float z[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint64_t at = (uint64_t)row[k] * p->n_q_heads + hq[k];
            if (k == 0 || !ONE) z[k] = ((const float __attribute__((address_space(1))) *)p->prior_lse)[at];
            w[k] = *(const f32x4 __attribute__((address_space(1))) *)(p->prior_out + at * D + 4u * dq[k]);
        }
        __builtin_amdgcn_sched_barrier(0);
        Merged m = {};
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (k == 0 || !ONE) m = merge_with(lse[k], z[k]);
            lse[k] = m.lse;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[k][e] = o[k][e] * m.a + (m.b > 0.0f ? w[k][e] * m.b : 0.0f);
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if (!live[k]) continue;
        *(u32x2 __attribute__((address_space(1))) *)(p->out + row[k] * p->out_row + hq[k] * p->out_head + dq[k] * 8u) =
            u32x2{pack_bf16(o[k].x, o[k].y), pack_bf16(o[k].z, o[k].w)};
        if (dq[k] == 0 && p->lse) ((gfloats)p->lse)[(uint64_t)row[k] * p->n_q_heads + hq[k]] = lse[k];
    }
}

// What one workgroup leaves for another, which may run on another XCD behind another L2, goes past those caches: stores and loads
// of device scope, each 8 bytes.  A release and an acquire fence instead write back and throw away the whole L2 of
// their XCD, per wave: decode of 32 requests took 312 us so and 134 this way (both as first built).
__device__ __forceinline__ void put2(float *p, float a, float b)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    __hip_atomic_store(reinterpret_cast<uint64_t *>(p), __builtin_bit_cast(uint64_t, f2{a, b}), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get2(const float *p)
{
    return __builtin_bit_cast(float2, __hip_atomic_load(reinterpret_cast<const uint64_t *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}
// every store of the wave has been performed where all workgroups see it
__device__ __forceinline__ void stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// A workgroup's share of a tile: tokens [t0, t1), for n_rows new rows of request req that holds `held`; the split-th of n_splits
struct Piece {
    uint32_t req, row0, n_rows, held, tile, t0, t1;
    uint32_t first_wg, split, n_splits;
    uint32_t past;  // its keys and values are read past the last-level cache
};

// ---- the pieces of a tile: whoever comes last joins them.  True for that workgroup; `flag`: a word of its LDS
__device__ __forceinline__ bool last_of_tile(Params p, const Piece &it, uint32_t h, uint32_t *flag)
{
    stores_done();
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t *counter = reinterpret_cast<uint32_t *>(p->plan + p->lay.counters) + (uint64_t)it.first_wg * p->n_kv_heads + h;
        const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *flag = before + 1u == it.n_splits;
        if (*flag) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // for the next layer's call
    }
    __syncthreads();
    return *flag != 0;
}

// A partial result: the sums of R rows in the order in which the workgroup's threads hold them (so that every store and load is
// of whole lines), then per row its reference, the sum of weights, the sum of rounded weights, nothing.
// A workgroup has room for two: its run's first tile, which the one before has a part of, and its last.
__device__ __forceinline__ float *part_of(Params p, uint32_t D, const Piece &it, uint32_t h, uint32_t split)
{
    const uint32_t slot = split == 0 ? 2u * it.first_wg + 1u : 2u * (it.first_wg + split);
    return reinterpret_cast<float *>(p->plan + p->lay.parts) + ((uint64_t)slot * p->n_kv_heads + h) * step_part_floats(D, p->lay.part_rows);
}

template <int D, int WAVES>
struct RowsLds {
    float o[WAVES][16][D + 4];  // 4: the 16 rows that are written side by side begin in different banks
    float m[WAVES][16], l[WAVES][16], r[WAVES][16];
    uint32_t last;
};

// The thread's index as a fresh value: what is derived from it is computed once per piece, not once for all pieces and then kept
// in registers across everything else (which spilled 103 of them).
__device__ __forceinline__ uint32_t fresh_tid()
{
    uint32_t t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// 16 query rows
template <int D, bool PAGE16, int WAVES, bool PAST>
__device__ __forceinline__ void attend_rows(Params p, const Piece &it, uint32_t h, RowsLds<D, WAVES> &lds)
{
    constexpr int Y = D / 32;            // MFMAs of a score; dwords of V per lane and token
    constexpr uint32_t kRowBytes = D * 2u;
    const uint32_t tid = fresh_tid(), lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t c_ = lane >> 4, n_ = lane & 15u;
    const uint32_t G = p->n_q_heads / p->n_kv_heads, M = it.n_rows * G, m0 = it.tile * 16u, mine = min(M - m0, 16u);
    const uint32_t P = p->page_tokens;

    // queries: row n, dims 32 y + 8 c .. (rows beyond the tile's: zero)
    const uint32_t qm = m0 + n_, qi = qm / G, qg = qm - qi * G;
    bf16x8 qb[Y];
#pragma unroll
    for (int y = 0; y < Y; ++y) qb[y] = __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u});
    if (n_ < mine) {
        gbytes qp = (gbytes)p->q + (it.row0 + qi) * p->q_row + (h * G + qg) * p->q_head + c_ * 16u;
#pragma unroll
        for (int y = 0; y < Y; ++y) qb[y] = __builtin_bit_cast(bf16x8, ldg16(qp + 64 * y));
    }
    // tokens that the lane's query row sees; the tile's least
    const int32_t limit = n_ < mine ? (int32_t)it.held - (int32_t)it.n_rows + (int32_t)qi + 1 : 0;
    const int32_t least = (int32_t)it.held - (int32_t)it.n_rows + (int32_t)(m0 / G) + 1;

    // the wave's blocks
    const uint32_t n_blk = it.t1 > it.t0 ? (it.t1 - it.t0 + 15u) / 16u : 0u, per = (n_blk + WAVES - 1u) / WAVES;
    const uint32_t b0 = wave * per, b1 = min(b0 + per, n_blk);

    const uint64_t head_tile = (uint64_t)(p->layer * 2u) * p->n_kv_heads + h;
    gbytes kbase = (gbytes)p->base + head_tile * p->tile_stride;
    gbytes vbase = kbase + (uint64_t)p->n_kv_heads * p->tile_stride;
    const uint32_t *table = p->table + (uint64_t)it.req * p->n_table;

    float m_run = neg_inf(), l_run = 0.0f, r_run = 0.0f;
    f32x4 O[D / 16];
#pragma unroll
    for (int x = 0; x < D / 16; ++x) O[x] = f32x4{0.f, 0.f, 0.f, 0.f};

    // Byte offsets, within a head's tile, of where rows lie.  PAGE16 (pages of whole blocks): lane l holds block
    // group + l's; else token 16 group + l's.  Bad pages, and columns beyond the table, count as rows that nobody sees, and are
    // read as page 0; so are tokens from t1 on, which are not asked for.
    constexpr uint32_t kGroup = PAGE16 ? 64u : 4u;
    auto offset_of = [&](uint32_t tok, uint32_t &lo, uint32_t &hi, bool &bad) {
        const uint32_t col = tok / P, row = tok - col * P;
        uint32_t page = tok >= it.t1 ? 0u : col < p->n_table ? table[col] : 0xFFFFFFFFu;
        bad = page >= p->n_pages;
        if (bad) page = 0u;
        const uint64_t off = page * p->page_stride + (uint64_t)row * kRowBytes;
        lo = (uint32_t)off, hi = (uint32_t)(off >> 32);
    };
    uint32_t off_lo = 0, off_hi = 0;
    uint64_t bad_mask = 0, n_bad = 0;
    uint32_t group = ~0u;

    auto fetch_group = [&](uint32_t g) {
        bool bad;
        offset_of(it.t0 + (PAGE16 ? (g + lane) * 16u : g * 16u + lane), off_lo, off_hi, bad);
        bad_mask = __ballot(bad);
        n_bad += __popcll(bad_mask);
        group = g;
    };
    auto load_block = [&](uint32_t b, RowsBlock<D> &r) -> uint32_t {
        const uint32_t g = (b - b0) / kGroup * kGroup + b0;
        if (g != group) fetch_group(g);
        const uint32_t j = b - g;
        uint32_t bad = 0;
        if (PAGE16) {
            // (the builtin's result is signed: without the casts an offset with bit 31 set came out with its upper half all ones)
            const uint64_t off = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_hi, j) << 32 | (uint32_t)__builtin_amdgcn_readlane(off_lo, j);
            bad = (bad_mask >> j) & 1u ? 15u : 0u;
#pragma unroll
            for (int y = 0; y < Y; ++y) r.k[y] = ldg16_of<PAST>(kbase + off + (n_ * kRowBytes + c_ * 16u + 64u * y));
#pragma unroll
            for (int i = 0; i < 4; ++i) ldg_words<Y, PAST>(vbase + off + ((4u * c_ + i) * kRowBytes + n_ * (D / 8u)), r.v[i]);
        } else {
            const int ks = j * 16u + n_;
            const uint64_t ko = (uint64_t)(uint32_t)__shfl((int)off_hi, ks) << 32 | (uint32_t)__shfl((int)off_lo, ks);
#pragma unroll
            for (int y = 0; y < Y; ++y) r.k[y] = ldg16_of<PAST>(kbase + ko + (c_ * 16u + 64u * y));
            bad = (uint32_t)(bad_mask >> (j * 16u + 4u * c_)) & 15u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int vs = j * 16u + 4u * c_ + i;
                const uint64_t vo = (uint64_t)(uint32_t)__shfl((int)off_hi, vs) << 32 | (uint32_t)__shfl((int)off_lo, vs);
                ldg_words<Y, PAST>(vbase + vo + n_ * (D / 8u), r.v[i]);
            }
        }
        return bad;
    };

    auto process = [&](uint32_t b, RowsBlock<D> &r, uint32_t bad) {
        const int32_t tok0 = (int32_t)(it.t0 + b * 16u);
        f32x4 S = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < Y; ++y) S = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, r.k[y]), qb[y], S, 0, 0, 0);
        mfma_result_wait();
        if (tok0 + 16 > least || __ballot(bad != 0)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int32_t tok = tok0 + 4 * (int32_t)c_ + i;
                const bool gone = (bad >> i) & 1u;
                if (tok >= limit || gone) S[i] = neg_inf();
                if (tok >= (int32_t)it.t1 || gone) {  // nobody's row: it may hold anything
#pragma unroll
                    for (int w = 0; w < Y; ++w) r.v[i][w] = 0u;
                }
            }
        }
        float top = __builtin_fmaxf(__builtin_fmaxf(S[0], S[1]), __builtin_fmaxf(S[2], S[3]));
        top = max_over_lane_groups(top) * p->scale_log2;
        if (__ballot(top > m_run + kLazyMaxSlack)) {
            const float m_new = __builtin_fmaxf(m_run, top);
            const float f = m_run == neg_inf() ? 0.0f : __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= f;
            r_run *= f;
#pragma unroll
            for (int x = 0; x < D / 16; ++x) O[x] *= f;
        }
        const float ref = m_run == neg_inf() ? 0.0f : m_run;
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[i], p->scale_log2, -ref));
            l_run += w[i];
        }
        const uint32_t p01 = pack_bf16(w[0], w[1]), p23 = pack_bf16(w[2], w[3]);
        r_run = add_weights(p23, add_weights(p01, r_run));
        const s16x4 P4 = __builtin_bit_cast(s16x4, u32x2{p01, p23});
#pragma unroll
        for (int x = 0; x < D / 16; ++x) {
            const uint32_t sel = x & 1 ? 0x07060302u : 0x05040100u;
            const u32x2 a = {__builtin_amdgcn_perm(r.v[1][x >> 1], r.v[0][x >> 1], sel),
                             __builtin_amdgcn_perm(r.v[3][x >> 1], r.v[2][x >> 1], sel)};
            O[x] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a), P4, O[x], 0, 0, 0);
        }
    };

    if (b0 < b1) {  // one block is worked on, one is on its way: with two or three on their way decode is 2 to 7 % slower
        RowsBlock<D> ra, rb;
        uint32_t ba = load_block(b0, ra), bb = 0;
        for (uint32_t b = b0; b < b1; b += 2) {
            bb = load_block(min(b + 1u, b1 - 1u), rb);
            process(b, ra, ba);
            if (b + 1u >= b1) break;
            ba = load_block(min(b + 2u, b1 - 1u), ra);
            process(b + 1u, rb, bb);
        }
    }
    mfma_result_wait();
    if (p->bad_pages && n_bad && lane == 0 && h == 0) atomicAdd(p->bad_pages, (uint32_t)n_bad);

    // ---- the waves of the workgroup
    p = late(p);
    l_run = sum_over_lane_groups(l_run);
    r_run = sum_over_lane_groups(r_run);
    if (c_ == 0) lds.m[wave][n_] = m_run;
    __syncthreads();
    float m_all = neg_inf();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) m_all = __builtin_fmaxf(m_all, lds.m[w][n_]);
    const float f = m_run == neg_inf() ? 0.0f : __builtin_amdgcn_exp2f(m_run - m_all);
    if (c_ == 0) {
        lds.l[wave][n_] = l_run * f;
        lds.r[wave][n_] = r_run * f;
    }
    // O[x][i]: dim (4 c + i) D / 16 + x of row n
    if (n_ < mine) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int x = 0; x < D / 16; x += 2)
                *reinterpret_cast<float2 *>(&lds.o[wave][n_][(4u * c_ + i) * (D / 16) + x]) = float2{O[x][i] * f, O[x + 1][i] * f};
    }
    __syncthreads();
    constexpr uint32_t kQuads = D / 4;
    constexpr int kN = (16 * kQuads + WAVES * 64 - 1) / (WAVES * 64);
    float *rec = part_of(p, D, it, h, it.split);
    uint32_t row[kN], hq[kN], dq[kN];
    bool live[kN];
    float lse[kN];
    f32x4 out[kN];
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        const uint32_t x = tid + k * WAVES * 64u, m = min(x / kQuads, mine - 1u);
        dq[k] = x % kQuads;
        live[k] = x / kQuads < mine;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        float l = 0.0f, r = 0.0f, mm = neg_inf();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            o += *reinterpret_cast<const f32x4 *>(&lds.o[w][m][4u * dq[k]]);
            l += lds.l[w][m];
            r += lds.r[w][m];
            mm = __builtin_fmaxf(mm, lds.m[w][m]);
        }
        if (it.n_splits > 1u && live[k]) {
            put2(rec + 2u * x, o.x, o.y);
            put2(rec + 8u * D + 2u * x, o.z, o.w);
            if (dq[k] == 0) {
                put2(rec + 16u * D + 4u * m, mm, l);
                put2(rec + 16u * D + 4u * m + 2u, r, 0.0f);
            }
        }
        const uint32_t i = (m0 + m) / G;
        row[k] = it.row0 + i, hq[k] = h * G + (m0 + m - i * G);
        out[k] = o * (r > 0.0f ? 1.0f / r : 0.0f);
        lse[k] = lse_of(mm, l);
    }
    if (it.n_splits == 1u) store_quads<D, kN, false>(p, row, hq, dq, live, out, lse);
    if (it.n_splits == 1u || !last_of_tile(p, it, h, &lds.last)) return;
    // References and sums of up to kJoin pieces come by one round of loads of all threads, the rows kAtOnce pieces at a time.
    constexpr int kAtOnce = 16;
    constexpr uint32_t kJoin = 64, kPairs = kJoin * 16 / (WAVES * 64);
    float2 (*ml)[16] = reinterpret_cast<float2 (*)[16]>(&lds.o[0][0][0]);
    float (*rr)[16] = reinterpret_cast<float (*)[16]>(&lds.o[0][0][0] + 2 * kJoin * 16);
    static_assert(sizeof(lds.o) >= 3 * kJoin * 16 * 4, "LDS of the join");
    float mm[kN], l[kN], r[kN];
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        mm[k] = neg_inf(), l[k] = r[k] = 0.0f;
        out[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (uint32_t s0 = 0; s0 < it.n_splits; s0 += kJoin) {
        const uint32_t ns = min(it.n_splits - s0, kJoin);
        float2 a[kPairs], b[kPairs], u[kAtOnce], v[kAtOnce];
        auto get = [&](uint32_t x, uint32_t e0) {
#pragma unroll
            for (int e = 0; e < kAtOnce; ++e) {
                const float *q = part_of(p, D, it, h, s0 + min(e0 + e, ns - 1u)) + 2u * x;
                u[e] = get2(q), v[e] = get2(q + 8 * D);
            }
        };
#pragma unroll
        for (uint32_t e = 0; e < kPairs; ++e) {
            const uint32_t x = tid + e * WAVES * 64u;
            const float *q = part_of(p, D, it, h, s0 + min(x / 16u, ns - 1u)) + 16u * D + 4u * min(x % 16u, mine - 1u);
            a[e] = get2(q), b[e] = get2(q + 2);
        }
        get(min(tid, mine * kQuads - 1u), 0);  // together with the references: one wait for both
        __syncthreads();
#pragma unroll
        for (uint32_t e = 0; e < kPairs; ++e) {
            const uint32_t x = tid + e * WAVES * 64u;
            ml[x / 16u][x % 16u] = a[e], rr[x / 16u][x % 16u] = b[e].x;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            if (k * WAVES * 64u >= mine * kQuads) break;
            const uint32_t x = min(tid + k * WAVES * 64u, mine * kQuads - 1u), m = x / kQuads;
            float top = mm[k];
#pragma unroll 8
            for (uint32_t e = 0; e < ns; ++e) top = __builtin_fmaxf(top, ml[e][m].x);
            const float f = mm[k] == neg_inf() ? 0.0f : __builtin_amdgcn_exp2f(mm[k] - top);
            out[k] *= f, l[k] *= f, r[k] *= f, mm[k] = top;
            for (uint32_t e0 = 0; e0 < ns; e0 += kAtOnce) {
                if (k != 0 || e0 != 0) get(x, e0);
#pragma unroll
                for (int e = 0; e < kAtOnce; ++e) {
                    if (e0 + e >= ns) break;
                    const float ms = ml[e0 + e][m].x, g = ms == neg_inf() ? 0.0f : __builtin_amdgcn_exp2f(ms - top);
                    out[k] += f32x4{u[e].x, u[e].y, v[e].x, v[e].y} * g;
                    l[k] += ml[e0 + e][m].y * g;
                    r[k] += rr[e0 + e][m] * g;
                }
            }
        }
    }
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        out[k] *= r[k] > 0.0f ? 1.0f / r[k] : 0.0f;
        lse[k] = lse_of(mm[k], l[k]);
    }
    store_quads<D, kN, false>(p, row, hq, dq, live, out, lse);
}

// ---- 128 query rows: a wave owns 32 of them, the keys and values lie in LDS for all four waves

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ uint32_t lds_base(uint8_t *p) { return (uint32_t)(uintptr_t)(uint8_t __attribute__((address_space(3))) *)p; }

// a value that is computed anew where it is used
__device__ __forceinline__ uint32_t fresh(uint32_t v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// a value that is the same in all lanes, in scalar registers
__device__ __forceinline__ uint64_t uniform(uint64_t v)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)v);
}

// 16 bytes per lane from base + off to LDS at `to` + 16 lane, past the registers.  Nothing waits for it: loads_done() does.
// m0 is the compiler's own register, which it warns of: each use writes it first, and the code built here has no other write or read of it.
__device__ __forceinline__ void load_to_lds(uint32_t to, gbytes base, uint32_t off)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(uniform((uint64_t)base)) : "memory", "m0");
}
__device__ __forceinline__ void load_to_lds(uint32_t to, gbytes at)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"((uint64_t)at) : "memory", "m0");
}
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// the other half of the wave's value
__device__ __forceinline__ void swap_halves(float x, float &a, float &b)
{
    typedef unsigned u2 __attribute__((ext_vector_type(2)));
    const unsigned xi = __builtin_bit_cast(unsigned, x);
    const u2 t = __builtin_amdgcn_permlane32_swap(xi, xi, false, false);
    const unsigned t0 = t.x, t1 = t.y;
    a = __builtin_bit_cast(float, t0), b = __builtin_bit_cast(float, t1);
}

// Tokens come to LDS in stages of 64.
constexpr uint32_t kStage = 64;

// Where 16-byte slot s of row t lies in its row of a tile in LDS: slot s ^ key_slot(t) for keys, s ^ value_slot(t) for values.  Keys
// are read by 16 lanes of 16 rows at the same slot, values by 16 lanes of 4 rows at two neighbouring slots: both then touch
// every bank once, with rows of 128, 192 and 256 bytes.
template <int D>
__device__ __forceinline__ uint32_t key_slot(uint32_t t)
{
    return D == 128 ? t & 15u : D == 64 ? (t >> 1) & 7u : (t >> 2) & 3u;
}
template <int D>
__device__ __forceinline__ uint32_t value_slot(uint32_t t)
{
    return D == 128 ? (t & 3u) << 2 : D == 64 ? ((t >> 1) & 1u) << 2 : 0u;
}

template <int D>
struct alignas(256) TilesLds {  // rows of 256 bytes at multiples of that: their slots are changed by exclusive ors
    uint8_t k[2][kStage * D * 2];
    uint8_t v[2][kStage * D * 2];
    uint16_t absent[2][4];  // bit t of the 64: a row that nobody sees
    uint32_t last;
};

template <int D, bool PAGE16>
__device__ __forceinline__ void attend_tiles(Params p, const Piece &it, uint32_t h, TilesLds<D> &lds)
{
    constexpr int KS = D / 16, DT = D / 32;
    constexpr uint32_t SL = D / 8, kRowBytes = D * 2u;
    constexpr int kLoads = SL / 4;  // loads of a wave per stage, for its 16 rows of keys or values
    const uint32_t tid = fresh_tid(), lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t col = lane & 31u, half = lane >> 5;
    const uint32_t G = p->n_q_heads / p->n_kv_heads, M = it.n_rows * G, m0 = it.tile * 128u, P = p->page_tokens;
    const uint32_t w0 = m0 + wave * 32u, mine = w0 < M ? min(M - w0, 32u) : 0u;

    // queries: row col, dims 16 y + 8 half ..
    const uint32_t qm = min(w0 + col, M - 1u), qi = qm / G, qg = qm - qi * G;
    bf16x8 qb[KS];
    {
        gbytes qp = (gbytes)p->q + (it.row0 + qi) * p->q_row + (h * G + qg) * p->q_head + half * 16u;
#pragma unroll
        for (int y = 0; y < KS; ++y) qb[y] = __builtin_bit_cast(bf16x8, ldg16(qp + 32 * y));
    }
    const int32_t past = (int32_t)it.held - (int32_t)it.n_rows + 1;
    const int32_t limit = past + (int32_t)qi;                      // tokens that the lane's row sees
    const int32_t least = past + (int32_t)(w0 / G);                // ... the wave's first, and its last row
    const int32_t most = mine ? past + (int32_t)((w0 + mine - 1u) / G) : 0;

    const uint64_t head_tile = (uint64_t)(p->layer * 2u) * p->n_kv_heads + h;
    gbytes kbase = (gbytes)p->base + head_tile * p->tile_stride;
    gbytes vbase = kbase + (uint64_t)p->n_kv_heads * p->tile_stride;
    const uint32_t *table = p->table + (uint64_t)it.req * p->n_table;
    const uint32_t n_stages = it.t1 > it.t0 ? (it.t1 - it.t0 + kStage - 1u) / kStage : 0u;

    // This wave brings rows 16 wave .. + 15 of every stage.  16-byte piece x = 64 n + lane of them is slot x % SL of row x / SL.
    const uint32_t row0 = wave * 16u;
    // Rows of 128 and 256 bytes: n changes the slot by an exclusive or and the row by a constant, so that one register says where all are
    // (three arrays of them spilled).
    constexpr bool kPow2 = (D & (D - 1)) == 0;
    const uint32_t t0_ = lane / SL, s0_ = lane - t0_ * SL;
    const uint32_t k_first = (PAGE16 ? t0_ * kRowBytes : 0u) + (s0_ ^ key_slot<D>(t0_)) * 16u;
    const uint32_t v_first = (PAGE16 ? t0_ * kRowBytes : 0u) + (s0_ ^ value_slot<D>(t0_)) * 16u;
    auto row_of = [&](int n) { return kPow2 ? t0_ + n * (64u / SL) : (n * 64u + lane) / SL; };
    auto from = [&](int n, bool v, uint32_t first) {
        if (kPow2) return (first ^ ((v ? value_slot<D>(n * (64u / SL)) : key_slot<D>(n * (64u / SL))) * 16u)) + (PAGE16 ? n * 1024u : 0u);
        const uint32_t t = row_of(n), x = n * 64u + lane - t * SL;
        return (PAGE16 ? t * kRowBytes : 0u) + (x ^ (v ? value_slot<D>(t) : key_slot<D>(t))) * 16u;
    };
    const uint32_t lds_k = lds_base(&lds.k[0][0]) + row0 * kRowBytes, lds_v = lds_base(&lds.v[0][0]) + row0 * kRowBytes;
    uint32_t n_bad = 0;

    // Pages of this wave's rows, many stages at once, since whoever waits for these loads waits for all before them.  PAGE16 (pages of
    // whole 16 rows): lane l has that of stage l's rows, 64 stages; else lane l has that of row l % 16 of stages l / 16, + 4, ..
    constexpr uint32_t kBulk = PAGE16 ? 64u : 16u;
    constexpr int kPages = PAGE16 ? 1 : 4;
    uint32_t pages[kPages];
    auto fetch_pages = [&](uint32_t j) {
#pragma unroll
        for (int n = 0; n < kPages; ++n) {
            const uint32_t tok = it.t0 + row0 + (PAGE16 ? (j + lane) * kStage : (j + 4u * n + (lane >> 4)) * kStage + (lane & 15u));
            const uint32_t at = tok / P;
            pages[n] = tok < it.t1 && at < p->n_table ? table[at] : 0xFFFFFFFFu;
            n_bad += tok < it.t1 && pages[n] >= p->n_pages;
        }
    };
    // Where stage j's rows are: PAGE16, of all 16 (those of the last ones that do not exist lie in the same page); else of row
    // lane % 16.  absent: which of the 16 nobody sees.
    struct Rows16 {
        uint64_t off;
        uint32_t absent;
    };
    auto locate = [&](uint32_t j) -> Rows16 {
        if (j % kBulk == 0) fetch_pages(j);
        const uint32_t tok0 = it.t0 + j * kStage + row0;
        const uint32_t none = tok0 >= it.t1 ? 0xFFFFu : it.t1 - tok0 < 16u ? 0xFFFFu << (it.t1 - tok0) & 0xFFFFu : 0u;
        if (PAGE16) {
            const uint32_t page = (uint32_t)__builtin_amdgcn_readlane(pages[0], j % kBulk);
            const bool gone = page >= p->n_pages;
            return Rows16{(gone ? 0u : page) * p->page_stride + (uint64_t)(tok0 % P) * kRowBytes, gone ? 0xFFFFu : none};
        }
        uint32_t page = pages[0];
#pragma unroll
        for (int n = 1; n < kPages; ++n)
            if ((j % kBulk) / 4u == (uint32_t)n) page = pages[n];
        page = (uint32_t)__shfl((int)page, (int)((j & 3u) * 16u + (lane & 15u)));
        const bool gone = page >= p->n_pages;
        return Rows16{(gone ? 0u : page) * p->page_stride + (uint64_t)((tok0 + (lane & 15u)) % P) * kRowBytes,
                      ((uint32_t)__ballot(gone) & 0xFFFFu) | none};
    };
    auto bring = [&](gbytes base, uint32_t to, uint64_t off, bool v) {
        const uint32_t first = kPow2 ? fresh(v ? v_first : k_first) : 0u;
#pragma unroll
        for (int n = 0; n < kLoads; ++n) {
            if (PAGE16) {
                load_to_lds(to + n * 1024u, base + off, from(n, v, first));
            } else {
                const int t = (int)row_of(n);
                const uint64_t o = (uint64_t)(uint32_t)__shfl((int)(off >> 32), t) << 32 | (uint32_t)__shfl((int)off, t);
                load_to_lds(to + n * 1024u, base + (o + from(n, v, first)));
            }
        }
    };

    float m_run = neg_inf(), l_run = 0.0f, r_run = 0.0f;
    f32x16 O[DT];
#pragma unroll
    for (int x = 0; x < DT; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[x][i] = 0.0f;

    // Where the lane reads: keys, token col (+ 32), slot 2 y + half; values, 4 tokens of 16 dims per 16 lanes.  As above: one register
    // each and an exclusive or per read, where rows allow it.
    const uint32_t i16 = lane & 15u, vt = 4u * half + (i16 >> 2);
    const uint32_t k_x = half ^ key_slot<D>(col), v_s = ((lane >> 4) & 1u) * 2u + ((i16 & 3u) >> 1), v_x = value_slot<D>(vt);
    const uint32_t k_rd = lds_base(&lds.k[0][0]) + col * kRowBytes + (kPow2 ? k_x * 16u : 0u);
    const uint32_t v_rd = lds_base(&lds.v[0][0]) + vt * kRowBytes + (i16 & 1u) * 8u + (kPow2 ? (v_s ^ v_x) * 16u : 0u);
    constexpr uint32_t kBuf = kStage * kRowBytes;

    // S[e]: scores of tokens 32 e .. + 31 of stage j.  The two chains take turns: each MFMA waits for the one before in its chain.
    // What lies between two sched_barriers is meant to run side by side: matrix instructions, the vector instructions that `beside(y)`
    // adds, and the next step's reads.
    auto scores = [&](uint32_t j, f32x16 (&S)[2], auto beside) {
        const uint32_t at = fresh(k_rd + (j & 1u) * kBuf);
        auto key = [&](int y, int e) {
            const uint32_t x = kPow2 ? at ^ (32u * y) : at + (k_x ^ (2u * y)) * 16u;
            return *(const bf16x8 __attribute__((address_space(3))) *)(uintptr_t)(x + e * 32u * kRowBytes);
        };
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) S[e][i] = 0.0f;
        bf16x8 a[KS][2];  // read two steps ahead of their MFMAs
#pragma unroll
        for (int y = 0; y < 2; ++y) a[y][0] = key(y, 0), a[y][1] = key(y, 1);
#pragma unroll
        for (int y = 0; y < KS; ++y) {
            if (y + 2 < KS) a[y + 2][0] = key(y + 2, 0), a[y + 2][1] = key(y + 2, 1);
            S[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[y][0], qb[y], S[0], 0, 0, 0);
            S[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[y][1], qb[y], S[1], 0, 0, 0);
            beside(y);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto absent_of = [&](uint32_t j) { return *(const u32x2 *)&lds.absent[j & 1u][0]; };
    auto mask = [&](uint32_t j, f32x16 (&S)[2], u32x2 ab) {
        const int32_t tok0 = (int32_t)(it.t0 + j * kStage);
        const uint64_t absent = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane(ab.y) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane(ab.x);
        mfma_result_wait();
        if (tok0 + (int32_t)kStage > least || absent) {
            // the lane's tokens are 4 half + constants: what they are compared with is moved instead
            const int32_t sees = limit - tok0 - 4 * (int32_t)half;
            const uint64_t gone = absent >> (4u * half);
            const uint32_t gone2[2] = {(uint32_t)gone, (uint32_t)(gone >> 32)};
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int t = 8 * (i / 4) + i % 4;
                    if (sees <= e * 32 + t || gone2[e] & (1u << t)) S[e][i] = neg_inf();
                }
        }
    };
    // moves the rows' references if scores as large as `top` (of the lane's own) have outgrown them
    auto settle = [&](float top) {
        float ta, tb;
        swap_halves(top, ta, tb);
        top = __builtin_fmaxf(ta, tb) * p->scale_log2;
        if (__ballot(top > m_run + kLazyMaxSlack)) {
            mfma_result_wait();
            const float m_new = __builtin_fmaxf(m_run, top);
            const float f = m_run == neg_inf() ? 0.0f : __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= f;
            r_run *= f;
#pragma unroll
            for (int x = 0; x < DT; ++x) O[x] *= f;
        }
    };
    auto weights = [&](const f32x16 (&S)[2], uint32_t (&pk)[16], float ref, int from, int to) {
#pragma unroll
        for (int i = from; i < to; ++i) {
            const float wa = __builtin_amdgcn_exp2f(__builtin_fmaf(S[i / 8][2 * (i % 8)], p->scale_log2, -ref));
            const float wb = __builtin_amdgcn_exp2f(__builtin_fmaf(S[i / 8][2 * (i % 8) + 1], p->scale_log2, -ref));
            l_run += wa;
            l_run += wb;
            pk[i] = fresh(pack_bf16(wa, wb));  // here, not behind the next branch, where they are used
            r_run = add_weights(pk[i], r_run);
        }
    };
    auto value = [&](uint32_t j, int s, int x) {
        typedef s16x4 __attribute__((address_space(3))) *lq;
        const uint32_t at = v_rd + (j & 1u) * kBuf;
        const uint32_t to = (kPow2 ? at ^ (64u * x) : at + ((v_s + 4u * x) ^ v_x) * 16u) + s * 16u * kRowBytes;
        const u32x2 ua = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lq)(uintptr_t)to));
        const u32x2 uc = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lq)(uintptr_t)(to + 8u * kRowBytes)));
        return __builtin_bit_cast(bf16x8, u32x4{ua.x, ua.y, uc.x, uc.y});
    };
    // first: the values of step 0, read before
    auto add_values = [&](uint32_t j, const uint32_t (&pk)[16], const bf16x8 (&first)[DT], auto beside) {
        bf16x8 a[DT], b[DT];
#pragma unroll
        for (int x = 0; x < DT; ++x) a[x] = first[x];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const bf16x8 w = __builtin_bit_cast(bf16x8, u32x4{pk[4 * s], pk[4 * s + 1], pk[4 * s + 2], pk[4 * s + 3]});
            if (s < 3) {
#pragma unroll
                for (int x = 0; x < DT; ++x) b[x] = value(j, s + 1, x);
            }
#pragma unroll
            for (int x = 0; x < DT; ++x) O[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[x], w, O[x], 0, 0, 0);
            beside(s);
#pragma unroll
            for (int x = 0; x < DT; ++x) a[x] = b[x];
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto top_of = [&](const f32x16 (&S)[2], int from, int to, float top) {
#pragma unroll
        for (int i = from; i < to; ++i) top = __builtin_fmaxf(top, S[i / 16][i % 16]);
        return top;
    };
    auto nothing = [](int) {};

    // Stage j's weights and values are worked on next to the scores of stage j + 1: its keys come a stage earlier than its values.
    // One barrier a stage.  Behind barrier j keys j + 2 and values j + 1 are asked for: their places were read last, by every wave,
    // before it reached that barrier (keys j and values j - 1).  At the next barrier they have arrived.
    if (n_stages) {
        Rows16 now = locate(0), next = {0u, 0u};  // of stages j and j + 1
        bring(kbase, lds_k, now.off, false);
        bring(vbase, lds_v, now.off, true);
        if (n_stages > 1u) {
            next = locate(1);
            bring(kbase, lds_k + kBuf, next.off, false);
        }
        if (lane == 0) lds.absent[0][wave] = (uint16_t)now.absent;
        loads_done();
        __syncthreads();
        auto turn = [&](uint32_t j) {  // of the stages
            loads_done();
            if (now.absent) {  // their values would meet weights of zero: NaN and infinity must not
#pragma unroll
                for (int n = 0; n < kLoads; ++n)
                    if ((now.absent >> row_of(n)) & 1u)
                        *reinterpret_cast<u32x4 *>(&lds.v[j & 1u][row0 * kRowBytes + (n * 64u + lane) * 16u]) = u32x4{0u, 0u, 0u, 0u};
            }
            if (lane == 0) lds.absent[(j + 1u) & 1u][wave] = (uint16_t)next.absent;
            __syncthreads();
        };
        auto ask = [&](uint32_t j) {  // for what stage j + 1 needs
            Rows16 after = {0u, 0u};
            if (j + 2u < n_stages) {
                after = locate(j + 2u);
                bring(kbase, lds_k + (j & 1u) * kBuf, after.off, false);
            }
            if (j + 1u < n_stages) bring(vbase, lds_v + ((j + 1u) & 1u) * kBuf, next.off, true);
            now = next, next = after;
        };
        // S: the scores of stage j; T: those of the next stage go there
        auto work = [&](uint32_t j, f32x16 (&S)[2], f32x16 (&T)[2]) {
            uint32_t pk[16];
            bf16x8 first[DT];
            const float ref = m_run == neg_inf() ? 0.0f : m_run;
            const u32x2 ab = absent_of(j + 1u);
            scores(j + 1u, T, [&](int y) {
                if (y == 0) ask(j);
                if (y == KS - 2) {
#pragma unroll
                    for (int x = 0; x < DT; ++x) first[x] = value(j, 0, x);
                }
                weights(S, pk, ref, y * 16 / KS, (y + 1) * 16 / KS);
            });
            mask(j + 1u, T, ab);
            float top = neg_inf();
            add_values(j, pk, first, [&](int s) { top = top_of(T, 8 * s, 8 * s + 8, top); });
            settle(top);
        };
        auto last_work = [&](uint32_t j, f32x16 (&S)[2]) {
            uint32_t pk[16];
            bf16x8 first[DT];
#pragma unroll
            for (int x = 0; x < DT; ++x) first[x] = value(j, 0, x);
            weights(S, pk, m_run == neg_inf() ? 0.0f : m_run, 0, 16);
            add_values(j, pk, first, nothing);
        };
        // stages of which the wave's rows see something
        const uint32_t mine_stages = most > (int32_t)it.t0 ? min(((uint32_t)most - it.t0 + kStage - 1u) / kStage, n_stages) : 0u;
        uint32_t j = 0;
        if (mine_stages) {
            f32x16 S[2], T[2];
            scores(0, S, nothing);
            mask(0, S, absent_of(0));
            settle(top_of(S, 0, 32, neg_inf()));
            for (; j + 2u < mine_stages; j += 2u) {  // in pairs: the scores change places without being moved
                turn(j);
                work(j, S, T);
                turn(j + 1u);
                work(j + 1u, T, S);
            }
            turn(j);
            if (j + 1u < mine_stages) {
                work(j, S, T);
                turn(++j);
                S[0] = T[0], S[1] = T[1];
            }
            ask(j);
            last_work(j++, S);
        }
        for (; j < n_stages; ++j) turn(j), ask(j);
    }
    mfma_result_wait();
    if (p->bad_pages && h == 0 && __ballot(n_bad != 0) && lane == 0) atomicAdd(p->bad_pages, 1u);

    float a, c;
    swap_halves(l_run, a, c);
    l_run = a + c;
    swap_halves(r_run, a, c);
    r_run = a + c;
    // O[x][i]: dim 32 x + 8 (i / 4) + 4 half + i % 4 of row col
    p = late(p);
    if (it.n_splits > 1u) {
        constexpr uint32_t kSums = 128u * D;  // then a row's four floats
        float *rec = part_of(p, D, it, h, it.split);
        const uint32_t m = wave * 32u + col, at = 2u * tid;
        const bool live_row = col < mine;  // rows that do not exist are neither written nor read
        if (live_row) {
#pragma unroll
            for (int x = 0; x < DT * 8; ++x) put2(rec + x * 512u + at, O[x / 8][2 * (x % 8)], O[x / 8][2 * (x % 8) + 1]);
        }
        if (half == 0 && live_row) {
            put2(rec + kSums + 4u * m, m_run, l_run);
            put2(rec + kSums + 4u * m + 2u, r_run, 0.0f);
        }
        if (!last_of_tile(p, it, h, &lds.last)) return;
        // The same threads hold the same sums of every piece: added up in the order of the pieces.  A load past the L2 takes about a
        // microsecond, so what counts is how often one is waited for: eight pieces' references come together with the first one's sums,
        // and the next one's sums are on their way while one's are added.
        constexpr int kRefs = 8;
        m_run = neg_inf(), l_run = r_run = 0.0f;
#pragma unroll
        for (int x = 0; x < DT; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) O[x][i] = 0.0f;
        for (uint32_t s0 = 0; live_row && s0 < it.n_splits; s0 += kRefs) {
            float2 ml[kRefs], rr[kRefs], v[2][DT * 8];
            auto get = [&](uint32_t s, float2 (&to)[DT * 8]) {
                const float *q = part_of(p, D, it, h, s) + at;
#pragma unroll
                for (int x = 0; x < DT * 8; ++x) to[x] = get2(q + x * 512u);
            };
#pragma unroll
            for (int e = 0; e < kRefs; ++e) {
                const float *q = part_of(p, D, it, h, min(s0 + e, it.n_splits - 1u)) + kSums + 4u * m;
                ml[e] = get2(q), rr[e] = get2(q + 2);
            }
            get(s0, v[0]);
            float top = m_run;
#pragma unroll
            for (int e = 0; e < kRefs; ++e) top = __builtin_fmaxf(top, ml[e].x);
            const float f = m_run == neg_inf() ? 0.0f : __builtin_amdgcn_exp2f(m_run - top);
            m_run = top;
            l_run *= f;
            r_run *= f;
#pragma unroll
            for (int x = 0; x < DT; ++x) O[x] *= f;
#pragma unroll
            for (int e = 0; e < kRefs; ++e) {
                if (s0 + e >= it.n_splits) break;
                if (e + 1 < kRefs && s0 + e + 1u < it.n_splits) get(s0 + e + 1u, v[(e + 1) & 1]);
                const float g = ml[e].x == neg_inf() ? 0.0f : __builtin_amdgcn_exp2f(ml[e].x - m_run);
                l_run += ml[e].y * g;
                r_run += rr[e].x * g;
#pragma unroll
                for (int x = 0; x < DT * 8; ++x) {
                    O[x / 8][2 * (x % 8)] += v[e & 1][x].x * g;
                    O[x / 8][2 * (x % 8) + 1] += v[e & 1][x].y * g;
                }
            }
        }
    }
    const float inv = r_run > 0.0f ? 1.0f / r_run : 0.0f;
    uint32_t row[DT * 4], hq[DT * 4], dq[DT * 4];
    bool live[DT * 4];
    float lse[DT * 4];
    f32x4 o[DT * 4];
#pragma unroll
    for (int x = 0; x < DT * 4; ++x) {
        row[x] = it.row0 + qi, hq[x] = h * G + qg, dq[x] = 2u * x + half;
        live[x] = col < mine;
        lse[x] = lse_of(m_run, l_run);
        o[x] = f32x4{O[x / 4][4 * (x % 4)] * inv, O[x / 4][4 * (x % 4) + 1] * inv, O[x / 4][4 * (x % 4) + 2] * inv, O[x / 4][4 * (x % 4) + 3] * inv};
    }
    store_quads<D, DT * 4, true>(p, row, hq, dq, live, o, lse);
}

constexpr int kWaves = 4;

// Calls body(piece, tile_rows) for the pieces of this workgroup's run.  Everything here is the same for all its threads.
template <class F>
__device__ __forceinline__ void for_pieces(Params p, uint32_t D, uint32_t wg, F body)
{
    const StepHdr hdr = *reinterpret_cast<const StepHdr *>(p->plan);
    StepStart at = reinterpret_cast<const StepStart *>(p->plan + p->lay.starts)[wg];
    if (hdr.magic != kStepMagic || hdr.n_requests != p->n_requests || hdr.n_rows != p->n_rows || hdr.n_q_heads != p->n_q_heads ||
        hdr.n_kv_heads != p->n_kv_heads || hdr.head_dim != D || wg >= hdr.n_wgs)
        return;
    const StepWork *work = reinterpret_cast<const StepWork *>(p->plan + p->lay.work);
    const uint32_t share = p->n_q_heads / p->n_kv_heads;
    while (at.n_units) {
        const StepWork w = work[at.work];
        Piece it;
        it.req = w.req, it.row0 = w.row0, it.n_rows = w.n_rows, it.held = w.held, it.tile = at.tile;
        const uint32_t line = kTileUnits + w.units, n = min(at.n_units, line - at.unit);
        const uint32_t from = max(at.unit, kTileUnits) - kTileUnits, to = max(at.unit + n, kTileUnits) - kTileUnits;
        // what the tile's last row sees
        const uint32_t last = min((at.tile + 1u) * w.tile_rows, w.n_rows * share) - 1u;
        const uint32_t sees = w.held ? w.held - w.n_rows + last / share + 1u : 0u;
        it.t0 = min(from * hdr.unit, sees);
        it.t1 = min(to * hdr.unit, sees);
        it.first_wg = wg, it.split = 0, it.n_splits = 1, it.past = hdr.past;
        if (hdr.run) {
            const uint32_t begin = w.begin + at.tile * line + kTileUnits;
            it.first_wg = begin / hdr.run;
            it.n_splits = (begin + w.units - 1u) / hdr.run - it.first_wg + 1u;
            it.split = wg - it.first_wg;
        }
        if (to > from) {  // else the run ends before the tile's first unit
            body(it, w.tile_rows);
            p = late(p);
        }
        at.n_units -= n;
        at.unit = 0;
        if (++at.tile == w.tiles) at.tile = 0, ++at.work;
        if (at.n_units) __syncthreads();  // the next piece uses the same LDS
    }
}

// every tile is one of 16 rows
template <int D, bool PAGE16>
__global__ __launch_bounds__(kWaves * 64, 2) void k11_attend_rows(const K11Params)
{
    Params p = (Params)__builtin_amdgcn_kernarg_segment_ptr();
    __shared__ RowsLds<D, kWaves> lds;
    const uint32_t wg = blockIdx.x / p->n_kv_heads, h = blockIdx.x - wg * p->n_kv_heads;
    for_pieces(p, D, wg, [&](const Piece &it, uint32_t) {
        if (it.past) attend_rows<D, PAGE16, kWaves, true>(p, it, h, lds);
        else attend_rows<D, PAGE16, kWaves, false>(p, it, h, lds);
    });
}

// tiles of 16 and of 128 rows
template <int D, bool PAGE16>
__global__ __launch_bounds__(kWaves * 64, 2) void k11_attend_mixed(const K11Params)
{
    Params p = (Params)__builtin_amdgcn_kernarg_segment_ptr();
    __shared__ union Lds {
        RowsLds<D, kWaves> rows;
        TilesLds<D> tiles;
    } lds;
    const uint32_t wg = blockIdx.x / p->n_kv_heads, h = blockIdx.x - wg * p->n_kv_heads;
    for_pieces(p, D, wg, [&](const Piece &it, uint32_t tile_rows) {
        if (tile_rows == 16u && it.past) attend_rows<D, PAGE16, kWaves, true>(p, it, h, lds.rows);
        else if (tile_rows == 16u) attend_rows<D, PAGE16, kWaves, false>(p, it, h, lds.rows);
        else attend_tiles<D, PAGE16>(p, it, h, lds.tiles);
    });
}

template <int D>
hipError_t launch_d(const K11Params &p, hipStream_t stream)
{
    const uint32_t grid = p.lay.cap_wgs * p.n_kv_heads, threads = kWaves * 64;
    const bool page16 = p.page_tokens % 16u == 0;
    if (p.lay.rows_only) {
        if (page16) k11_attend_rows<D, true><<<grid, threads, 0, stream>>>(p);
        else k11_attend_rows<D, false><<<grid, threads, 0, stream>>>(p);
    } else {
        if (page16) k11_attend_mixed<D, true><<<grid, threads, 0, stream>>>(p);
        else k11_attend_mixed<D, false><<<grid, threads, 0, stream>>>(p);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_k11(const K11Params &p, uint32_t head_dim, hipStream_t stream)
{
    switch (head_dim) {
    case 64: return launch_d<64>(p, stream);
    case 96: return launch_d<96>(p, stream);
    case 128: return launch_d<128>(p, stream);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace ha_rag
