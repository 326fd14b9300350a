// Serving new tokens from a paged cache: what the host entry points (ha_rag_paged.hip) and the kernels
// (ha_rag_paged_kernels.hip, ha_rag_paged_attend.hip) share.  Not part of the C ABI.
#pragma once
#include "ha_rag_kernels.h"

namespace ha_rag {

constexpr uint32_t kStepMagic = 0x53544550u;  // the first word of a plan that k9 has written

// The plan of a step, in the caller's device memory: written by k9, read by k11.  Sections in this order, each 256-byte
// aligned; sizes follow from (n_requests, n_rows, n_q_heads) and the context alone, because lengths are on the device.
//
// How the attention is shared out.  A request's query rows of a KV head are cut into tiles of 16 or kStepTileRows; a tile's tokens
// are counted in units.  The tiles of all requests, one after the other, are a line, the same for every KV head: each tile
// has a place of kTileUnits units for what it costs to begin and end it, then those of its tokens.
//   cut:    the line is cut into runs of `run` units, one per workgroup and head, wherever that falls: every workgroup has the
//           same to read where tiles see what their request holds, as in decode.  A tile that lies in several runs gets one partial
//           result of each.  (Every tile of a request counts the units of all rows held, but sees those up to its last row.  A chunk
//           over much less than its own length is therefore shared out unevenly: of a prompt of 2,000 rows from nothing, 8 x 4
//           heads, the busiest workgroup works on 32 units, the mean is 16; 62 us, where a chunk of 2,000 over 2,000, which is three
//           times as much, takes 150.  Pieces of rows that a tile does not see are written and joined like others.)
//   whole:  each tile has a workgroup of its own, in request order, the last tile of a request (which sees most) first; where there
//           are enough of them, and of such lengths, that this comes out about even (k9_page_scan says when).
struct StepHdr {
    uint32_t magic, n_requests, n_rows, n_q_heads;  // what the plan was made for
    uint32_t n_kv_heads, head_dim;                  // ... and this
    uint32_t n_wgs;                                 // workgroups with work, per KV head
    uint32_t run;                                   // units of a workgroup; 0: whole tiles
    uint32_t unit;                                  // tokens
    uint32_t past;                                  // 1: the keys and values are read past the last-level cache (kPastBytes)
    uint32_t n_freed, height;                       // pages given back; free pages before
    uint32_t pad[4];
};

struct StepReq {  // what the scan leaves per request for the threads that fill the arrays
    uint32_t t, before, kept;  // rows held before, the pages of these, and those of them that stay
    uint32_t need_ex;          // pages taken by the requests before
    uint32_t granted;          // 1: new rows are stored
    uint32_t work;             // index among the requests with rows
    uint32_t tiles, units;     // as in StepWork
};

struct StepWork {  // a request with rows
    uint32_t req, row0, n_rows, held;  // its first row, its rows, the rows it holds now (0: refused, its rows see nothing)
    uint32_t tile_rows, tiles, units;  // rows of a tile; tiles; units of the tokens of each
    uint32_t begin;                    // where its first tile begins on the line of units (cut)
};

struct StepStart {  // where a workgroup begins
    uint32_t work, tile, unit, n_units;  // unit: on the line, from the tile's begin; n_units: of the run
};
static_assert(sizeof(StepReq) == 32 && sizeof(StepHdr) == 64 && sizeof(StepWork) == 32, "plan layout");

struct StepLayout {  // bytes from the plan's start
    uint64_t req, freed_ex, line_ex, work, starts, counters, parts, total;
    uint32_t cap_wgs;      // workgroups per KV head, at most
    uint32_t target;       // workgroups per KV head that run at once
    uint32_t rows_only;    // 1: every tile is one of 16 rows
    uint32_t part_rows;    // rows that a partial result has room for
};

constexpr uint32_t kStepTileRows = 128;  // query rows of a large tile
constexpr uint32_t step_part_floats(uint32_t head_dim, uint32_t rows) { return rows * (head_dim + 4u); }

// A unit: 64 tokens, more for tables so long that the line of units could pass 32 bits
constexpr uint32_t step_unit(uint32_t n_table, uint32_t page_tokens)
{
    uint32_t unit = 64;
    while ((uint64_t)n_table * page_tokens / unit > (1u << 20)) unit *= 2;
    return unit;
}
constexpr uint32_t kTileUnits = 3;    // a workgroup takes about as long to begin and end a tile as to work on this many units
constexpr uint32_t kLeastRun = 7;     // units: shorter runs cost more to join than they save
constexpr uint32_t kManyTiles = 3;    // tiles of 16 rows are taken whole from so many times more of them than workgroups that run at once

// A step's layers come one after the other, and what one leaves in the last-level cache (256 MB) is of use only if the keys and values of
// all of them fit there until the next step.  Beyond this many bytes they are read past it.  us a layer of decode over 5,000 rows a
// request (20.5 MB), layers in turn, through the cache / past it: 128 requests 416 / 381, 32 requests of two layers 115 / 102, of one
// layer 109 / 97, 18 requests (369 MB in all) 66.4 / 61.3, 16 (328 MB) 57.2 / 54.4, 14 (287 MB) 48.7 / 49.3, 8 requests of two layers
// (328 MB) 33.5 / 32.8, 4 of four 22.2 / 22.0, 4 of two (164 MB) 21.2 / 21.3: even below the border, and past it from there on.
constexpr uint64_t kPastBytes = 320ull << 20;

struct K9Params {
    uint32_t *table;
    const int32_t *n_tokens;
    int32_t *n_tokens_after;
    uint32_t *free_pages;
    const int32_t *n_free;
    int32_t *n_free_after;
    const int32_t *n_new;
    int32_t *row_start, *slots, *positions;
    uint32_t *refused;
    uint8_t *plan;
    StepLayout lay;
    uint32_t n_requests, n_table, n_pages, page_tokens, n_rows, n_q_heads, n_kv_heads, head_dim, n_layers;
    uint32_t unit;
};

struct K10Params {
    const uint8_t *k, *v;
    uint64_t k_row, k_head, v_row, v_head;  // bytes
    const int32_t *slots;
    uint8_t *base;
    uint32_t *bad_pages;
    uint64_t page_stride, tile_stride;
    uint32_t n_rows, n_kv_heads, head_dim, page_tokens, n_pages, layer;
};

struct K11Params {
    const uint8_t *q;
    uint64_t q_row, q_head;  // bytes
    uint8_t *out;
    uint64_t out_row, out_head;
    float *lse;
    const float *prior_out, *prior_lse;
    const uint8_t *base;
    const uint32_t *table;
    uint32_t *bad_pages;
    uint64_t page_stride, tile_stride;
    uint8_t *plan;
    StepLayout lay;
    float scale_log2;
    uint32_t n_requests, n_rows, n_table, n_pages, page_tokens, n_kv_heads, n_q_heads, layer;
};

inline bool step_head_dim(uint32_t d) { return d == 64u || d == 96u || d == 128u; }  // head_dim of k11_attend_rows

hipError_t launch_k9(const K9Params &p, hipStream_t stream);
hipError_t launch_k10(const K10Params &p, hipStream_t stream);
hipError_t launch_k11(const K11Params &p, uint32_t head_dim, hipStream_t stream);

}  // namespace ha_rag
