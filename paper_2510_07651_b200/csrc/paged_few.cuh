// Attention of at most 16 rows per KV list (single tokens of a GQA group, a few tokens of a small one) over a paged cache.
//
// Bound by the K and V bytes.  Pages arrive as bulk copies (TMA) in a ring of 128-token tiles; a warp takes 16 tokens of a tile and runs
// warp-level MMAs with the tokens on the M side, so that the (at most 8 per step) rows lie on N and nothing is padded to more:
//     S^T = K q^T      16 tokens x 8 rows, 8 steps of 16 channels
//     O^T += V^T P^T   16 channels x 8 rows, 8 tiles, one step of 16 tokens; P^T is S^T's accumulator turned by movmatrix
// A warp keeps (m, l, O) of its own tokens; they meet once per segment.  P enters as two bf16 parts, so that o is off by no
// more than its own rounding (the MMAs are nowhere near their limit here).  With up to 8 rows two CTAs share an SM, so that one's segment
// beginnings and ends (q, the joining of its warps' results) hide behind the other's tiles: 256 lists of 4096 tokens in 8 bits 74 -> 65 us.
// Tiles of 16-bit rows are halved for it (three stages of 64 tokens each).
//
// e4m3 rows become fp16 in registers, which holds every code exactly (one conversion for two codes; to bf16 it took seven instructions for
// four and, since P then needs two parts, twice the MMAs: 256 lists of 4096 tokens 80 us against 76).  The channels of a 16-channel step are
// taken in the order in which ldmatrix hands out their bytes (q is loaded in the same order), and the rows of an O^T tile are eight even and
// eight odd channels.  q is scaled by a power of two per row, so that its largest value is near 2^14 (what falls below fp16's range is less
// than 2^-38 of it).  The scale of a K row goes into its logit, that of a V row into its P, relative to a reference exponent that O carries: P is
// fp16 then, off by at most 2^-11 of itself.  Where one of 16 tokens' weights (V's scale included) is above 0 and below 2^-14, where fp16 has fewer bits,
// they are taken by classes of exponents, each scaled into fp16's normal range and added to O from accumulators of its own: beside a first token that
// takes nearly all of the weight, with a row of V near 0, o consists of such weights.
#pragma once
#include "paged_common.cuh"
#include "tc_ptx.cuh"
#include "warp_mma.cuh"

namespace obc {
namespace {

template <int NT, bool E4M3> struct FewLayout {
    static constexpr int kRows = 8 * NT, kCtas = NT == 1 ? 2 : 1;                          // CTAs per SM
    static constexpr int kTile = !E4M3 && NT == 1 ? 64 : kTokTile;                         // tokens per stage
    static constexpr int kWarps = 8, kPerTile = kTile / 16, kGroups = kWarps / kPerTile, kThreads = 32 * kWarps + 64;
    static constexpr uint32_t kOperand = kTile * (E4M3 ? 128u : 256u), kStage = 2 * kOperand;
    static constexpr int kStages = E4M3 ? 6 / kCtas : 3, kFull = kStages * kGroups;
    static constexpr int kSlots = 4 / kCtas;                                               // warps whose O the merge buffer holds
    static constexpr int kPitch = kD + 4;                                                  // floats per row of O in the merge buffer
    static constexpr uint32_t kMerge = kStages * kStage, kMergeBytes = kSlots * 8 * kPitch * 4;
    static constexpr uint32_t kScales = kMerge + kMergeBytes;                              // [stage][K, V][128] scale bytes
    static constexpr uint32_t kBars = kScales + (E4M3 ? (uint32_t)kStages * 256u : 0u);    // full, empty
    static constexpr uint32_t kSmem = kBars + (kFull + kStages) * 8u + 1024;               // + alignment slack
};

// (b0, b2) and (b1, b3)
__device__ __forceinline__ void expand_alternate(uint32_t x, uint32_t& p02, uint32_t& p13) { expand_adjacent(__byte_perm(x, 0u, 0x3120), p02, p13); }
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// a weight above 0 that fp16 holds with fewer than its 11 bits, or not at all
__device__ __forceinline__ bool below_f16(float x) { return __float_as_uint(x) - 1u < 0x387fffffu; }
// 2^e for whole e (0 and infinity beyond fp32's exponents)
__device__ __forceinline__ float pow2i(int e) { return e < -126 ? 0.f : e > 127 ? INFINITY : __uint_as_float((uint32_t)(e + 127) << 23); }

// B operands of all steps from one row of q (nullptr: zeros): channels 16 ks + 2 c, + 1 and + 8, + 9.  e4m3: 16 ks + 4 c, .. + 3 as fp16 times a
// power of two; the result is what undoes it.  The four lanes of a row call together.
template <bool E4M3>
__device__ __forceinline__ float q_fragments(uint32_t (&b)[8][2], const __nv_bfloat16* src, int c) {
    if (!E4M3) {
        const uint32_t* u = reinterpret_cast<const uint32_t*>(src);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) { b[ks][0] = u ? u[ks * 8 + c] : 0u; b[ks][1] = u ? u[ks * 8 + 4 + c] : 0u; }
        return 1.f;
    }
    uint32_t top = 0;                        // largest |q|, as bf16 bits
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
        const uint2 u = src ? *reinterpret_cast<const uint2*>(src + ks * 16 + c * 4) : make_uint2(0u, 0u);
        b[ks][0] = u.x; b[ks][1] = u.y;
        top = max(top, max(max(u.x & 0x7fffu, u.x >> 16 & 0x7fffu), max(u.y & 0x7fffu, u.y >> 16 & 0x7fffu)));
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int e = (int)(top >> 7);           // biased exponent; 0: zeros or subnormals, 255: infinity or NaN (beside which finite values only have to stay finite)
    const int up = e == 255 ? -114 : min(141 - e, 126);   // (2^-up has to be a normal number)
    const float f = pow2i(up);
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
#pragma unroll
        for (int j = 0; j < 2; ++j) b[ks][j] = pack_f16x2(__uint_as_float(b[ks][j] << 16) * f, __uint_as_float(b[ks][j] & 0xffff0000u) * f);
    return pow2i(-up);
}
// Two weights (0 or more) as bf16 pairs hi + lo, off by at most 2^-16 of themselves.  Both parts of a weight above 2^-110 are above 0 (hi is cut off below the weight), so that
// an infinity of V times them stays one: with hi rounded to nearest, lo may be 0 or negative, and their sum NaN.
__device__ __forceinline__ void split_weights(float x, float y, uint32_t& hi, uint32_t& lo) {
    const uint32_t u = max(__float_as_uint(x), 1u) - 1u, v = max(__float_as_uint(y), 1u) - 1u;
    hi = __byte_perm(u, v, 0x7632);
    lo = pack_bf16x2(x - __uint_as_float(u & 0xffff0000u), y - __uint_as_float(v & 0xffff0000u));
}
// an 8x8 tile of 16-bit values turned: the lane's pair (row lane / 4, columns 2 (lane % 4), + 1) becomes that of the transpose
__device__ __forceinline__ uint32_t turned(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
// barriers of the consumer warps
template <int N> __device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(N) : "memory"); }
template <int N> __device__ __forceinline__ bool consumers_or(bool x) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)x), "n"(N) : "memory");
    return r != 0;
}
// Copies the pages (and scales) of the walk's tile into a stage, K or V (`scale` and `stage` are that operand's); all lanes of a warp.  A copy takes a
// warp some hundred cycles to issue, one lane after the other, which is what two warps and the map that takes both halves of the rows at
// once are for: a tile in pages of 16 tokens is 8 copies per warp.
template <typename L, bool E4M3, typename W>
__device__ __forceinline__ void few_issue(const W& walk, const CUtensorMap* map, const uint8_t* scale, uint32_t stage, uint32_t scales, uint32_t bar) {
    const AttnParams& p = walk.p;
    const int lane = walk.lane, page = walk.page(), h = walk.cur.m.h;
    if (lane == 0) mbar_expect_tx(bar, L::kOperand);
    __syncwarp();
    if (lane < walk.boxes()) {
        const uint32_t d = stage + (lane << (p.box_shift + (E4M3 ? 7 : 8)));
        const int hh = p.one_head ? 0 : h, slot = walk.slot;
        if (E4M3) tma_load_4d(d, map, bar, 0, slot, hh, page);
        else tma_load_5d(d, map, bar, 0, slot, 0, hh, page);
    }
    if (E4M3) {                              // 8 scale bytes per lane of the first 16
        const int t8 = (lane & 15) * 8, pg = __shfl_sync(0xffffffffu, page, t8 >> p.box_shift);
        const uint8_t* src = scale + (pg < 0 ? 0ll : pg * p.c.ss_p + h * p.c.ss_h + walk.slot8);
        if (lane < 16) asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(scales + t8), "l"(src), "r"(pg < 0 ? 0 : 8) : "memory");
        asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
    }
}
// 16-byte piece `piece` of row `row` of a staged tile of 16-bit values: [box][half of the channels][row of the box][128 bytes], swizzled
__device__ __forceinline__ uint32_t few_piece(int box_shift, int row, int piece) {
    const int in_box = row & ((1 << box_shift) - 1);
    return (uint32_t)((row >> box_shift) << (box_shift + 8)) + (uint32_t)((piece >> 3) << (box_shift + 7)) + in_box * 128 + (((piece & 7) ^ (row & 7)) << 4);
}

template <int NT, bool E4M3>
__global__ void __launch_bounds__(FewLayout<NT, E4M3>::kThreads, FewLayout<NT, E4M3>::kCtas)
few_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttnParams p) {
    using L = FewLayout<NT, E4M3>;
    constexpr int ROWS = L::kRows, CONS = 32 * L::kWarps;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t sbase = smem_u32(smem);
    __shared__ RunScratch scratch;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // Tile n of the CTA goes through stage n mod kStages and announces itself on barrier n mod kFull: a stage has a barrier for each group, since
    // a group waits for every other tile only and could not tell by its parity how often a barrier that it had not watched has turned.
    auto full = [&](int i) { return sbase + L::kBars + 8u * (uint32_t)i; };
    auto empty = [&](int i) { return sbase + L::kBars + 8u * (uint32_t)(L::kFull + i); };
    if (threadIdx.x == 0) {
        prefetch_tmap(&map_k); prefetch_tmap(&map_v);
        for (int i = 0; i < L::kFull; ++i) mbar_init(full(i), E4M3 ? 66 : 2);
        for (int i = 0; i < L::kStages; ++i) mbar_init(empty(i), L::kPerTile);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = 0u;        // no wait of this call can have given up yet (each lasts seconds)
    const Run run = find_run<ROWS>(p, &scratch);                    // (its barriers also publish the mbarriers)
    int fail_site = 0;

    if (warp >= L::kWarps) {
        // ============================ producers: a warp for K, one for V =====================
        const bool is_v = warp > L::kWarps;
        TileWalk<ROWS, L::kTile> walk(p, run, lane);
        int n = 0, st = 0, fb = 0;                                  // tiles issued; stage and barrier of the next
        uint32_t phase = 1;
        while (walk.more) {
            if (!__all_sync(0xffffffffu, mbar_wait(empty(st), phase))) { fail_site = __LINE__; break; }
            few_issue<L, E4M3>(walk, is_v ? &map_v : &map_k, is_v ? p.c.vs : p.c.ks, sbase + st * L::kStage + (is_v ? L::kOperand : 0u), sbase + L::kScales + st * 256 + (is_v ? 128 : 0), full(fb));
            if (n == 0) walk.look_ahead();
            walk.advance();
            ++n;
            if (++fb == L::kFull) fb = 0;
            if (++st == L::kStages) { st = 0; phase ^= 1u; }
        }
        for (int back = 0; back < L::kStages && back < n; ++back) { // no copy may be under way when the CTA leaves
            const int k = n - 1 - back;
            (void)mbar_wait(full(k % L::kFull), (k / L::kFull) & 1);
        }
    } else {
        // ===================================== consumers ====================================
        const int g = lane >> 2, c = lane & 3, group = warp / L::kPerTile, wg = warp;
        const int tok0 = warp % L::kPerTile * 16;                   // the warp's tokens of a tile
        Segments<ROWS> seg(p, run);
        int4 info = make_int4(-1, 0, 0, 0);
        int st = 0, fb = 0, turn = 0;                               // stage, barrier and group of the next tile
        uint32_t phase = 0;
        while (seg.next()) {
            const Item m = seg.m;
            info = seg.shared_item(run);
            uint32_t qf[NT][8][2];
            int seen[NT][2];                                        // of rows 2 c, 2 c + 1
            float mx[NT][2], l[NT][2], sl2[NT][2];
            int e_ref = -1;                                         // biased exponent that the warp's O is relative to (e4m3); -1: none yet
            float o[NT][8][4];                                      // O^T: channel tile; (row g, columns 2 c, 2 c + 1), (row g + 8, ..)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const __nv_bfloat16* src = nullptr;
                if (nt * 8 + g < m.rows) {
                    int head, i;
                    row_place(p, m, nt * 8 + g, head, i);
                    src = static_cast<const __nv_bfloat16*>(p.q.ptr) + m.b * p.q.sb + head * p.q.sh + i * p.q.st;
                }
                const float down = q_fragments<E4M3>(qf[nt], src, c);
#pragma unroll
                for (int j = 0; j < 2; ++j) sl2[nt][j] = E4M3 ? p.sl2 * __shfl_sync(0xffffffffu, down, 4 * (2 * c + j)) : p.sl2;
#pragma unroll
                for (int j = 0; j < 2; ++j) { seen[nt][j] = seen_by(p, m, nt * 8 + 2 * c + j); mx[nt][j] = -INFINITY; l[nt][j] = 0.f; }
#pragma unroll
                for (int j = 0; j < 8; ++j) { o[nt][j][0] = 0.f; o[nt][j][1] = 0.f; o[nt][j][2] = 0.f; o[nt][j][3] = 0.f; }
            }
            const int first_masked = p.causal ? min(max(m.len - m.ql + p.by_G.div(m.r0) + 1, 0), m.len) : m.len;   // tokens that not every row sees begin here

            constexpr int kParts = kTokTile / L::kTile;
            for (int tile = seg.ta * kParts; tile < seg.tb * kParts; ++tile) {
                const bool mine = L::kGroups == 1 || turn == group;
                const int s_at = st, f_at = fb;
                const uint32_t par = phase;
                if (++turn == L::kGroups) turn = 0;
                if (++st == L::kStages) st = 0;
                if (++fb == L::kFull) { fb = 0; phase ^= 1u; }
                if (!mine) continue;
                uint8_t* sk = smem + s_at * L::kStage;
                uint8_t* sv = sk + L::kOperand;
                if (!__all_sync(0xffffffffu, mbar_wait(full(f_at), par))) { fail_site = __LINE__; break; }
                const int t0 = tile * L::kTile + tok0;              // the warp's first token
                const bool edge = t0 + 16 > first_masked;           // some row does not see some of the 16 tokens
                if (t0 < m.len) {
                    float s[NT][4], s2[NT][4];                      // even and odd steps: half the chain
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) { s[nt][j] = 0.f; s2[nt][j] = 0.f; }
                    const int a_row = tok0 + (lane & 15), a_pc = lane >> 4;      // tiles in A's order: (tokens 0-7, p), (8-15, p), (0-7, p + 1), (8-15, p + 1)
                    if (E4M3) {
#pragma unroll
                        for (int pc = 0; pc < 8; pc += 2) {
                            uint32_t r[4];
                            ldsm_x4(r, sk + a_row * 128 + (((pc + a_pc) ^ (a_row & 7)) << 4));
                            uint32_t a[4], b[4];
                            expand_adjacent(r[0], a[0], a[2]); expand_adjacent(r[1], a[1], a[3]);
                            expand_adjacent(r[2], b[0], b[2]); expand_adjacent(r[3], b[1], b[3]);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma_f16(s[nt], a, qf[nt][pc][0], qf[nt][pc][1]);
                                mma_f16(s2[nt], b, qf[nt][pc + 1][0], qf[nt][pc + 1][1]);
                            }
                        }
                    } else {
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks) {
                            const int piece = 2 * ks + a_pc;
                            uint32_t a[4];
                            ldsm_x4(a, sk + few_piece(p.box_shift, a_row, piece));
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma_bf16(ks & 1 ? s2[nt] : s[nt], a, qf[nt][ks][0], qf[nt][ks][1]);
                        }
                    }
                    float fk[2] = {1.f, 1.f}, fv[2] = {1.f, 1.f};                // factors of the lane's tokens g and g + 8
                    int ev[2] = {0, 0};
                    bool classes = false;
                    if (E4M3) {
                        const uint8_t* sc = smem + L::kScales + s_at * 256 + tok0 + g;
                        fk[0] = scale_of(sc[0]); fk[1] = scale_of(sc[8]);
                        ev[0] = sc[128]; ev[1] = sc[136];
                        // highest exponent of the V rows that the list has (of the finite ones; 1 at least: O's factor 2^(e_ref - 127) has to be a normal number)
                        const bool in0 = t0 + g < m.len, in1 = t0 + g + 8 < m.len;
                        const int hi = __reduce_max_sync(0xffffffffu, max(max(in0 && ev[0] < 255 ? ev[0] : 0, in1 && ev[1] < 255 ? ev[1] : 0), 1));
                        if (e_ref < 0 || hi > e_ref + 4) {          // O follows: P stays below 2^12
                            const float f = e_ref < 0 ? 0.f : pow2i(e_ref - hi);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int j = 0; j < 8; ++j) { o[nt][j][0] *= f; o[nt][j][1] *= f; o[nt][j][2] *= f; o[nt][j][3] *= f; }
                            e_ref = hi;
                        }
                        fv[0] = in0 ? pow2i(ev[0] - e_ref) : 0.f; fv[1] = in1 ? pow2i(ev[1] - e_ref) : 0.f;
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            if (ev[j] == 255 && fv[j] != 0.f) fv[j] = __uint_as_float(0x7fc00000u);
                    }
                    uint32_t ph[NT][2], pl[NT][2];                  // P^T as B operands: high and low parts
                    float e[NT][4];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float tm[2];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float x = (s[nt][j] + s2[nt][j]) * (E4M3 ? sl2[nt][j & 1] * fk[j >> 1] : p.sl2);
                            if (edge && t0 + g + 8 * (j >> 1) >= seen[nt][j & 1]) x = -INFINITY;
                            s[nt][j] = x;
                        }
                        tm[0] = fmaxf(s[nt][0], s[nt][2]); tm[1] = fmaxf(s[nt][1], s[nt][3]);
                        // the reference moves only when the maximum exceeds it by 2^8 (P stays far inside fp32's and bf16's range): first asked
                        // of every lane's own two tokens, so that most tiles need no exchange
                        if (__any_sync(0xffffffffu, tm[0] > mx[nt][0] + 8.f || tm[1] > mx[nt][1] + 8.f)) {
                            float f[2];
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
#pragma unroll
                                for (int w = 4; w < 32; w <<= 1) tm[j] = fmaxf(tm[j], __shfl_xor_sync(0xffffffffu, tm[j], w));
                                f[j] = 1.f;
                                if (tm[j] > mx[nt][j] + 8.f) { f[j] = exp2f(mx[nt][j] - tm[j]); mx[nt][j] = tm[j]; }
                                l[nt][j] *= f[j];
                            }
#pragma unroll
                            for (int j = 0; j < 8; ++j) { o[nt][j][0] *= f[0]; o[nt][j][1] *= f[1]; o[nt][j][2] *= f[0]; o[nt][j][3] *= f[1]; }
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float x = fast_exp2(s[nt][j] - reference(mx[nt][j & 1]));
                            l[nt][j & 1] += x;
                            e[nt][j] = x;
                        }
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            uint32_t hi, lo;
                            if (E4M3) {
                                const float x = e[nt][2 * j] * fv[j], y = e[nt][2 * j + 1] * fv[j];
                                classes |= below_f16(x) || below_f16(y);
                                ph[nt][j] = turned(pack_f16x2(x, y));
                            } else {
                                split_weights(e[nt][2 * j], e[nt][2 * j + 1], hi, lo);
                                ph[nt][j] = turned(hi); pl[nt][j] = turned(lo);
                            }
                        }
                    }
                    if (!E4M3 && edge) {
                        // rows that not every query sees: those behind the list's end may hold anything and become zeros; one that
                        // is not finite must reach the queries that see it alone
                        bool odd = false;
                        const int row = tok0 + (lane >> 1), t = t0 + (lane >> 1);
                        uint4* at = reinterpret_cast<uint4*>(sv + (few_piece(p.box_shift, row, (lane & 1) * 8) & ~127u));      // the row's half
                        if (t >= m.len) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) at[j] = make_uint4(0u, 0u, 0u, 0u);
                        } else if (t >= first_masked) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const uint4 u = at[j];
                                odd |= not_finite(u.x) || not_finite(u.y) || not_finite(u.z) || not_finite(u.w);
                            }
                        }
                        __syncwarp();
                        unsigned bad = __ballot_sync(0xffffffffu, odd);
                        while (bad) {                               // token by token, on CUDA cores; the row is zeroed for the MMAs
                            const int tk = (__ffs(bad) - 1) >> 1, rw = tok0 + tk;
                            bad &= ~(3u << (2 * tk));
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                float w[2];
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    w[j] = __shfl_sync(0xffffffffu, tk & 8 ? e[nt][2 + j] : e[nt][j], (tk & 7) * 4 + c);
                                    if (t0 + tk >= seen[nt][j]) continue;
#pragma unroll
                                    for (int x = 0; x < 16; ++x) {  // channels 8 x + g
                                        const __nv_bfloat16 v = *reinterpret_cast<const __nv_bfloat16*>(sv + few_piece(p.box_shift, rw, x) + g * 2);
                                        o[nt][x >> 1][(x & 1) * 2 + j] += w[j] * __bfloat162float(v);
                                    }
                                }
                            }
                            __syncwarp();
                            if (lane < 16) *reinterpret_cast<uint4*>(sv + few_piece(p.box_shift, rw, lane)) = make_uint4(0u, 0u, 0u, 0u);
                            __syncwarp();
                        }
                    }
                    unsigned odd = 0;                               // tokens that not every query sees and whose rows hold NaN
                    if (E4M3 && edge) {                             // rows behind the list's end may hold codes that stand for NaN
                        const int row = tok0 + (lane >> 1), t = t0 + (lane >> 1);
                        uint4* at = reinterpret_cast<uint4*>(sv + row * 128 + (lane & 1) * 64);
                        uint32_t any = 0;
                        if (t >= m.len) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) at[j] = make_uint4(0u, 0u, 0u, 0u);
                        } else if (t >= first_masked) {
                            any = smem[L::kScales + s_at * 256 + 128 + row] == 255 ? 1u : 0u;
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint4 u = at[j];
                                any |= nan_codes(u.x) | nan_codes(u.y) | nan_codes(u.z) | nan_codes(u.w);
                            }
                        }
                        __syncwarp();
                        odd = __ballot_sync(0xffffffffu, any != 0u);
                        odd = (odd | odd >> 1) & 0x55555555u;       // bit 2 i: token i
                        classes |= odd != 0u;
                    }
                    const int v_row = tok0 + (lane & 7) + (lane >> 4) * 8, v_pc = (lane >> 3) & 1;   // (tokens 0-7, p), (0-7, p + 1), (8-15, p), (8-15, p + 1)
                    if (E4M3) {
                        auto v_pieces = [&](int pc, uint32_t lo, uint32_t hi, uint32_t (&a)[4], uint32_t (&b)[4]) {      // lo, hi: bytes of the tokens 2 c, + 1 and + 8, + 9 to be taken
                            uint32_t r[4];
                            ldsm_x4_trans(r, sv + v_row * 128 + (((pc + v_pc) ^ (v_row & 7)) << 4));
                            r[0] &= lo; r[1] &= lo; r[2] &= hi; r[3] &= hi;
                            expand_alternate(r[0], a[0], a[1]); expand_alternate(r[2], a[2], a[3]);      // piece pc: even channels, odd channels
                            expand_alternate(r[1], b[0], b[1]); expand_alternate(r[3], b[2], b[3]);
                        };
                        if (!__any_sync(0xffffffffu, classes)) {
#pragma unroll
                            for (int pc = 0; pc < 8; pc += 2) {
                                uint32_t a[4], b[4];
                                v_pieces(pc, ~0u, ~0u, a, b);
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    mma_f16(o[nt][pc], a, ph[nt][0], ph[nt][1]);
                                    mma_f16(o[nt][pc + 1], b, ph[nt][0], ph[nt][1]);
                                }
                            }
                        } else {
                            // Weights by classes of exponents, each scaled into fp16's normal range.  First all tokens but the odd ones, whose NaN would reach queries of weight 0;
                            // then those one by one, for the queries that see them.
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int j = 0; j < 4; ++j) e[nt][j] *= fv[j >> 1];
                            unsigned now = 0x55555555u & ~odd;
                            bool once = true;
                            int alone = -1;                         // the one token of the pass
                            for (;;) {
                                uint32_t big = 0;
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int j = 0; j < 4; ++j)
                                        if (now >> (2 * g + 16 * (j >> 1)) & 1u) big = max(big, __float_as_uint(e[nt][j]) & 0x7fffffffu);
                                const int top = (int)(__reduce_max_sync(0xffffffffu, big) >> 23);       // biased exponent of the largest; 255: NaN
                                if (top == 0 && !once) {            // (a NaN counts whatever its weight: one pass is there in any case)
                                    if (!odd) break;
                                    now = odd & (0u - odd); odd ^= now;
                                    alone = t0 + ((__ffs(now) - 1) >> 1);
                                    once = true;
                                    continue;
                                }
                                once = false;
                                auto bytes = [&](int at) { const unsigned two = now >> at; return (two & 1u ? 0xffffu : 0u) | (two & 4u ? 0xffff0000u : 0u); };
                                const uint32_t lo = bytes(4 * c), hi = bytes(4 * c + 16);
                                const int up = top == 255 ? 0 : min(141 - top, 126), last = top == 255 ? 255 : top - 28;     // (into [2^14, 2^15); down to 2^-14)
                                const float f = pow2i(up), back = pow2i(-up);
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int j = 0; j < 2; ++j) {
                                        float x = e[nt][2 * j], y = e[nt][2 * j + 1];
                                        const bool mine_now = now >> (2 * g + 16 * j) & 1u;
                                        const bool in_x = mine_now && (int)(__float_as_uint(x) >> 23 & 255u) >= last, in_y = mine_now && (int)(__float_as_uint(y) >> 23 & 255u) >= last;
                                        if (in_x) e[nt][2 * j] = 0.f;
                                        if (in_y) e[nt][2 * j + 1] = 0.f;
                                        x = in_x ? x * f : 0.f; y = in_y ? y * f : 0.f;
                                        ph[nt][j] = turned(pack_f16x2(x, y));
                                    }
#pragma unroll
                                for (int pc = 0; pc < 8; pc += 2) {
                                    uint32_t a[4], b[4];
                                    v_pieces(pc, lo, hi, a, b);
#pragma unroll
                                    for (int nt = 0; nt < NT; ++nt) {
                                        float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
                                        mma_f16(x, a, ph[nt][0], ph[nt][1]);
                                        mma_f16(y, b, ph[nt][0], ph[nt][1]);
#pragma unroll
                                        for (int j = 0; j < 4; ++j)
                                            if (alone < seen[nt][j & 1]) { o[nt][pc][j] = fmaf(x[j], back, o[nt][pc][j]); o[nt][pc + 1][j] = fmaf(y[j], back, o[nt][pc + 1][j]); }
                                    }
                                }
                            }
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const int piece = 2 * j + v_pc;
                            uint32_t a[4];
                            ldsm_x4_trans(a, sv + few_piece(p.box_shift, v_row, piece));
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma_bf16(o[nt][j], a, ph[nt][0], ph[nt][1]);
                                mma_bf16(o[nt][j], a, pl[nt][0], pl[nt][1]);
                            }
                        }
                    }
                }
                if (edge) fence_async_smem();              // this thread's writes to the stage precede the bulk copy into it
                __syncwarp();
                if (lane == 0) mbar_arrive(empty(s_at));
            }

            // ---- the warps' results meet: maxima and sums, then O, eight rows at a time ----
            float* sm = reinterpret_cast<float*>(smem + L::kMerge);            // [warp][ROWS] maxima, then sums
            float* sl = sm + L::kWarps * ROWS;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int w = 4; w < 32; w <<= 1) l[nt][j] += __shfl_xor_sync(0xffffffffu, l[nt][j], w);
                    if (g == 0) { sm[warp * ROWS + nt * 8 + 2 * c + j] = mx[nt][j]; sl[warp * ROWS + nt * 8 + 2 * c + j] = l[nt][j]; }
                }
            if (consumers_or<CONS>(fail_site != 0)) {               // one warp's wait gave up: all leave
                if (!fail_site) fail_site = __LINE__;
                break;
            }
            // the reference and the sum of a row over all warps
            auto joined = [&](int r, float& ref, float& total) {
                float top = -INFINITY;
#pragma unroll
                for (int w = 0; w < L::kWarps; ++w) top = fmaxf(top, sm[w * ROWS + r]);
                ref = reference(top);
                total = 0.f;
#pragma unroll
                for (int w = 0; w < L::kWarps; ++w) total = fmaf(share_of(sm[w * ROWS + r], ref), sl[w * ROWS + r], total);
            };
            float f[NT][2], ref_w[NT], sum_w[NT];                   // factors of the lane's rows; statistics of row 8 nt + wg
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float top = -INFINITY;
#pragma unroll
                    for (int w = 0; w < L::kWarps; ++w) top = fmaxf(top, sm[w * ROWS + nt * 8 + 2 * c + j]);
                    f[nt][j] = share_of(mx[nt][j], reference(top)) * (E4M3 ? (e_ref < 0 ? 1.f : pow2i(e_ref - 127)) : 1.f);
                }
                joined(nt * 8 + wg, ref_w[nt], sum_w[nt]);
            }
            const bool whole = seg.whole();
            float* buf = reinterpret_cast<float*>(smem + L::kMerge);           // [warp][row][channel]
            // as many warps at a time as there is room for, the last ones first, the others adding to what they find
            auto put = [&](int nt, bool add) {
                float* at = buf + warp % L::kSlots * 8 * L::kPitch + 2 * c * L::kPitch;
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        float* to = at + (x & 1) * L::kPitch + 16 * j + (E4M3 ? 2 * g + (x >> 1) : g + 8 * (x >> 1));
                        const float v = o[nt][j][x] * f[nt][x & 1];
                        *to = add ? *to + v : v;
                    }
            };
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (nt * 8 >= m.rows) break;
#pragma unroll 1
                for (int k = L::kWarps / L::kSlots - 1; k >= 0; --k) {
                    consumers_sync<CONS>();                         // (before the first: the buffer is free)
                    if (warp / L::kSlots == k) put(nt, k < L::kWarps / L::kSlots - 1);
                }
                consumers_sync<CONS>();
                // a warp sums and stores one row
                const int r = nt * 8 + wg;
                if (r >= m.rows) continue;
                float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < L::kSlots; ++w) {
                    const float4 x = *reinterpret_cast<const float4*>(buf + (w * 8 + wg) * L::kPitch + lane * 4);
                    a.x += x.x; a.y += x.y; a.z += x.z; a.w += x.w;
                }
                const float sum = sum_w[nt], k = whole ? (sum != 0.f ? 1.f / sum : 0.f) : 1.f;
                a.x *= k; a.y *= k; a.z *= k; a.w *= k;
                if (whole) {
                    int head, i;
                    row_place(p, m, r, head, i);
                    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(const_cast<void*>(p.o.ptr)) + m.b * p.o.sb + head * p.o.sh + i * p.o.st;
                    *reinterpret_cast<uint2*>(dst + lane * 4) = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
                    if (p.lse && lane == 0) p.lse[((size_t)m.b * p.c.Hkv * p.G + head) * p.T + i] = lse_of(ref_w[nt], sum);
                } else {
                    const size_t at = seg.slot() * ROWS + r;
                    *reinterpret_cast<float4*>(p.part_o + at * kD + lane * 4) = a;
                    if (lane == 0) { p.part_m[at] = sum == 0.f ? -INFINITY : ref_w[nt]; p.part_l[at] = sum; }
                }
            }
            consumers_sync<CONS>();                                 // the buffer is free for the next segment's statistics
        }
        if (threadIdx.x == 0) p.info[blockIdx.x] = info;
    }
    if (fail_site && lane == 0) atomicCAS(p.status, 0u, (unsigned)fail_site);
}

}  // namespace
}  // namespace obc
