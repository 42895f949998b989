// What the kernels of obc_paged_attention share: how the work is cut into pieces, and where partial results go.
//
// An item is a tile of `ROWS` query rows of one KV list (row r = i G + g is query i of the group's head g, so that a tile's rows are near
// one another in position and stop at the same tokens).  An item costs as many token tiles of 128 as its last row sees, and kSegCost tiles'
// time for its beginning and end.  All items, in order, are cut into a run of equal cost per CTA, so that ragged batches, lists per
// head and causal chunks load every CTA alike whatever the lengths, which only the device knows.  (Without the constant the CTA with
// the shortest items of a 4096-token prompt took half again as long as the others; with 3 it took 170 us, with 4 161, with 5 159 to 172.)  A CTA's run is a sequence of segments, each a
// range of tiles of one item.  An item that lies within one run is finished there; the others leave partial results (maximum, sum,
// unnormalised output) that the merge kernel joins in the order of the tiles.  A run has at most two such segments, its first
// and its last, and an item that is shared is the last one of the CTA that it begins in: the merge goes by these CTAs.
#pragma once
#include "obc_common.cuh"
#include <cuda_fp16.h>

namespace obc {
namespace {

constexpr int kTokTile = 128;

struct AttnParams {
    PagesView c;
    int G, T, causal;
    const int32_t* q_lens;
    float sl2;                               // scale * log2(e)
    TensorView q, o;
    int o_aligned;                           // rows of o begin on 32-byte boundaries
    float* lse;                              // or nullptr
    int nrt, items;                          // row tiles per list, items in all
    FastDiv by_G, by_nrt;
    int box, box_shift, one_head;            // tokens per bulk copy (a power of two); pages of one head
    unsigned int* status;                    // workspace header: source line of the wait that gave up
    int4* info;                              // per CTA: the shared item that begins in it (or -1), the item's last CTA, its slot here
    float *part_m, *part_l, *part_o;         // [2 gridDim][ROWS] (x d): slots of a CTA's first and last segment
};

struct Item { int b, h, len, ql, r0, rows, tiles; };      // rows: rows of this tile; tiles: 0 if it has none

template <int ROWS>
__device__ __forceinline__ Item item_of(const AttnParams& p, int it) {
    Item m;
    const int unit = p.by_nrt.div(it);
    m.b = p.c.by_H.div(unit); m.h = unit - m.b * p.c.Hkv;
    m.len = p.c.len(m.b, m.h);
    m.ql = p.q_lens ? min(max(p.q_lens[m.b], 0), p.T) : p.T;
    m.r0 = (it - unit * p.nrt) * ROWS;
    m.rows = min(p.G * m.ql - m.r0, ROWS);
    m.tiles = 0;
    if (m.rows > 0) {                        // (one tile at least: rows that see nothing have results, too)
        const int seen = p.causal ? min(max(m.len - m.ql + p.by_G.div(m.r0 + m.rows - 1) + 1, 0), m.len) : m.len;
        m.tiles = max((seen + kTokTile - 1) / kTokTile, 1);
    }
    return m;
}
// tokens that row r of the item's tile sees: p < the result (r beyond the tile's rows: none)
__device__ __forceinline__ int seen_by(const AttnParams& p, const Item& m, int r) {
    if (r >= m.rows) return 0;
    return p.causal ? min(max(m.len - m.ql + p.by_G.div(m.r0 + r) + 1, 0), m.len) : m.len;
}

// four e4m3 codes as fp16 pairs: (b0, b1) and (b2, b3)
__device__ __forceinline__ void expand_adjacent(uint32_t x, uint32_t& p01, uint32_t& p23) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(p01), "=r"(p23) : "r"(x));
}
// a row's scale from its byte
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s == 255u ? 0x7fc00000u : s == 0u ? 0x00400000u : s << 23); }
// codes that stand for NaN (all bits but the sign set): the top bit of their bytes
__device__ __forceinline__ uint32_t nan_codes(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// infinity or NaN in either half
__device__ __forceinline__ bool not_finite(uint32_t bf16x2) { return (bf16x2 & 0x7f80u) == 0x7f80u || (bf16x2 & 0x7f800000u) == 0x7f800000u; }
// The maximum that logits are taken relative to, kept finite: with infinite logits sums become infinite or NaN as they should, where a difference of two infinities
// would be NaN always; and if all are -inf their weights are 0.
__device__ __forceinline__ float reference(float top) { return fminf(fmaxf(top, -3.402823466e38f), 3.402823466e38f); }
// what sums relative to `top` count for relative to the reference of a maximum that is no smaller
__device__ __forceinline__ float share_of(float top, float ref) { return exp2f(fminf(top, 3.402823466e38f) - ref); }
// natural log-sum-exp from the reference in log2 units and the sum above it; a row that saw nothing has sum 0 (and log2(0) = -inf)
__device__ __forceinline__ float lse_of(float ref, float total) { return (ref + log2f(total)) * 0.6931471805599453f; }

constexpr int kSegCost = 4;

struct Run { int begin, end, size, longer; int item, off; };      // runs of size + 1 (the first `longer`) and of size
struct RunScratch { int warp_sum[32]; int item, off; };

// This CTA's run; all threads of the block take part.
template <int ROWS>
__device__ __forceinline__ Run find_run(const AttnParams& p, RunScratch* s) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, nwarps = blockDim.x >> 5;
    const int per = (p.items + blockDim.x - 1) / blockDim.x, i0 = tid * per, i1 = min(i0 + per, p.items);
    auto cost = [&](int i) { const int n = item_of<ROWS>(p, i).tiles; return n > 0 ? n + kSegCost : 0; };
    int mine = 0;
    for (int i = i0; i < i1; ++i) mine += cost(i);
    int scan = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, scan, o);
        if (lane >= o) scan += up;
    }
    if (lane == 31) s->warp_sum[warp] = scan;
    if (tid == 0) { s->item = 0; s->off = 0; }
    __syncthreads();
    int before = scan - mine, total = 0;
#pragma unroll 4
    for (int w = 0; w < nwarps; ++w) {
        const int x = s->warp_sum[w];
        if (w < warp) before += x;
        total += x;
    }
    // (no empty runs between two others: the merge goes by CTA numbers)
    const int ctas = min((int)gridDim.x, total), cta = min((int)blockIdx.x, ctas);
    Run run;
    run.size = ctas ? (int)((unsigned)total / (unsigned)ctas) : 1; run.longer = total - run.size * ctas;
    run.begin = cta * run.size + min(cta, run.longer);
    run.end = cta < ctas ? run.begin + run.size + (cta < run.longer ? 1 : 0) : run.begin;
    if (run.begin >= before && run.begin < before + mine) {
        int at = before;
        for (int i = i0; i < i1; ++i) {
            const int n = cost(i);
            if (run.begin < at + n) { s->item = i; s->off = run.begin - at; break; }
            at += n;
        }
    }
    __syncthreads();
    run.item = s->item; run.off = s->off;
    return run;
}

// Walks the segments of a run; every role of a CTA has its own copy.
template <int ROWS>
struct Segments {
    const AttnParams& p;
    int at, end;                             // where the next item begins; the run's end
    int next_item, off;                      // off: what of the next item's cost lies before the run
    Item m;                                  // the segment: tiles [ta, tb) of item `item`
    int item, ta, tb;
    bool first;
    __device__ __forceinline__ Segments(const AttnParams& p_, const Run& r) : p(p_), at(r.begin - r.off), end(r.end), next_item(r.item), off(r.off), first(true) { item = -1; }
    __device__ __forceinline__ bool next() {
        if (item >= 0) first = false;
        while (at + off < end) {
            m = item_of<ROWS>(p, next_item++);
            if (m.tiles == 0) continue;
            ta = max(off - kSegCost, 0);
            tb = max(min(end - at - kSegCost, m.tiles), 0);
            at += m.tiles + kSegCost;
            off = 0;
            if (ta < tb) { item = next_item - 1; return true; }
        }
        return false;
    }
    __device__ __forceinline__ void copy(const Segments& s) { at = s.at; end = s.end; next_item = s.next_item; off = s.off; m = s.m; item = s.item; ta = s.ta; tb = s.tb; first = s.first; }
    __device__ __forceinline__ bool whole() const { return ta == 0 && tb == m.tiles; }
    __device__ __forceinline__ size_t slot() const { return 2 * (size_t)blockIdx.x + (first ? 0 : 1); }
    // of the current segment, for the merge
    __device__ __forceinline__ int4 shared_item(const Run& r) const {
        if (ta != 0 || tb == m.tiles) return make_int4(-1, 0, 0, 0);
        const int last = at - 1, split = r.longer * (r.size + 1);                  // the item's last tile
        const int cta = last < split ? last / (r.size + 1) : r.longer + (last - split) / r.size;
        return make_int4(item, cta, first ? 0 : 1, 0);
    }
};

// The tiles of a CTA's run, for the warp that asks for their pages.  A lane holds the page number of one box in a window of 32
// consecutive boxes (a tile has at most 16 of them, so it lies within one window); the next window's, or the next segment's first,
// travel while the current ones are used.  (With the numbers of one tile at a time, asked for one tile ahead, 32 sequences of up
// to 8192 tokens took 124 us against 97 without any look-up.)
template <int ROWS, int TILE_TOKENS = kTokTile>
struct TileWalk {
    static constexpr int kParts = kTokTile / TILE_TOKENS;      // tiles of the walk in one of a segment's
    static constexpr int kBits = TILE_TOKENS == 128 ? 7 : 6;
    static_assert(TILE_TOKENS == 1 << kBits, "tile");
    const AttnParams& p;
    Segments<ROWS> cur, nxt;
    bool more, more_next;
    int lane, tile, pages, pages_next;
    int slot, slot8, step;                   // places in their pages of the lane's box and of the lane's eight tokens (of 16 lanes); a tile's tokens mod P
    __device__ __forceinline__ TileWalk(const AttnParams& p_, const Run& r, int lane_) : p(p_), cur(p_, r), nxt(p_, r), lane(lane_) {
        step = p.c.by_P.mod(TILE_TOKENS);
        more = cur.next();
        pages = pages_next = -1;
        more_next = false;
        if (more) { begin(); pages = asked(cur.m, window(tile)); }
    }
    // what need not be known before the first tile's copies are on their way
    __device__ __forceinline__ void look_ahead() {
        if (!more) return;
        nxt.copy(cur); more_next = nxt.next();
        ahead();
    }
    __device__ __forceinline__ int boxes() const { return TILE_TOKENS >> p.box_shift; }
    __device__ __forceinline__ int window(int t) const { return t >> (p.box_shift + 5 - kBits); }         // 32 boxes = 2^(shift + 5) tokens
    __device__ __forceinline__ void begin() {
        tile = cur.ta * kParts;
        slot = p.c.by_P.mod(tile * TILE_TOKENS + (lane << p.box_shift)); slot8 = p.c.by_P.mod(tile * TILE_TOKENS + (lane & 15) * 8);
    }
    __device__ __forceinline__ int asked(const Item& m, int win) const {
        const int t = (win * 32 + lane) << p.box_shift;
        int v = -1;
        if (t < m.len) v = p.c.table[m.b * p.c.tb + m.h * p.c.th + p.c.by_P.div(t)];
        return v;
    }
    __device__ __forceinline__ void ahead() {
        if (window(tile) < window(cur.tb * kParts - 1)) pages_next = asked(cur.m, window(tile) + 1);
        else if (more_next) pages_next = asked(nxt.m, window(nxt.ta * kParts));
    }
    // page of the lane's box of the current tile; -1 for rows of zeros (behind the list, or a page that is not there)
    __device__ __forceinline__ int page() const {
        const int v = __shfl_sync(0xffffffffu, pages, (tile * boxes() + lane) & 31);
        return lane < boxes() && (unsigned)v < (unsigned)p.c.n_pages ? v : -1;
    }
    __device__ __forceinline__ void advance() {
        if (++tile < cur.tb * kParts) {
            slot += step; slot8 += step;
            if (slot >= p.c.P) slot -= p.c.P;
            if (slot8 >= p.c.P) slot8 -= p.c.P;
            if (window(tile) != window(tile - 1)) { pages = pages_next; ahead(); }
            return;
        }
        more = more_next;
        if (!more) return;
        cur.copy(nxt);
        begin();
        pages = pages_next;
        more_next = nxt.next();
        ahead();
    }
};

// where the row (i G + g) of an item's list stands in q, o and lse
__device__ __forceinline__ void row_place(const AttnParams& p, const Item& m, int r, int& head, int& i) {
    const int row = m.r0 + r;
    i = p.by_G.div(row);
    head = m.h * p.G + (row - i * p.G);
}

}  // namespace
}  // namespace obc
