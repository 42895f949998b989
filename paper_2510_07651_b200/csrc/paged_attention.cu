// Attention of new tokens over a paged cache (obc_paged_attention): o = softmax(scale q K^T) V with the causal mask of a chunk at the
// list's end, by one pass over the list with running maxima and sums.
//
//   few_rows_kernel      up to 32 rows per KV list (single tokens of a GQA group): bound by the K/V bytes.  Pages arrive as bulk copies
//                        (TMA) in a ring; eight warps take 16 tokens of every 128-token tile each and run warp-level MMAs.
//   chunk_kernel         more rows: tcgen05 MMAs (paged_chunk.cuh)
//   paged_f32_kernel     fp32 caches on CUDA cores
//   paged_merge_kernel   joins the partial results of items that several CTAs shared
// How the work is shared out: paged_common.cuh.
#include "paged_chunk.cuh"
#include "warp_mma.cuh"

#include <math.h>

namespace obc {
namespace {

// ---- merge ------------------------------------------------------------------------------------------
// One warp per row of an item that was shared: o = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s over the CTAs' slots, in
// their order.
template <typename OT, int ROWS>
__global__ void __launch_bounds__(256)
paged_merge_kernel(const __grid_constant__ AttnParams p) {
    pdl_wait();
    const int blocks = ROWS / 8, it = blockIdx.x / blocks, r = (blockIdx.x % blocks) * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    const Item m = item_of<ROWS>(p, it);
    if (r >= m.rows) return;
    const int4 f = p.info[it];
    if (f.x < 0) return;
    const int n = f.y - f.x + 1;
    auto at = [&](int s) { return (2 * (size_t)(f.x + s) + (s == 0 ? f.z : 0)) * ROWS + r; };
    float top = -INFINITY;
    for (int s = lane; s < n; s += 32) top = fmaxf(top, p.part_m[at(s)]);
    top = warp_max(top);
    const float ref = top == -INFINITY ? 0.f : top;
    float total = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < n; s0 += 32) {
        const int s = s0 + lane, cnt = min(32, n - s0);
        const float w = s < n ? exp2f(p.part_m[at(s)] - ref) : 0.f;
        if (s < n) total = fmaf(w, p.part_l[at(s)], total);
#pragma unroll 4
        for (int j = 0; j < cnt; ++j) {
            const float wj = __shfl_sync(0xffffffffu, w, j);
            const float4 o = *reinterpret_cast<const float4*>(p.part_o + at(s0 + j) * kD + lane * 4);
            if (wj == 0.f) continue;         // nothing was seen there (or nothing that counts)
            acc.x = fmaf(wj, o.x, acc.x); acc.y = fmaf(wj, o.y, acc.y); acc.z = fmaf(wj, o.z, acc.z); acc.w = fmaf(wj, o.w, acc.w);
        }
    }
    total = warp_sum(total);
    const float inv = total != 0.f ? 1.f / total : 0.f;
    int head, i;
    row_place(p, m, r, head, i);
    OT* dst = static_cast<OT*>(const_cast<void*>(p.o.ptr)) + m.b * p.o.sb + head * p.o.sh + i * p.o.st + lane * 4;
    if constexpr (sizeof(OT) == 4) *reinterpret_cast<float4*>(dst) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    else *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    if (p.lse && lane == 0)
        p.lse[((size_t)m.b * p.c.Hkv * p.G + head) * p.T + i] = lse_of(ref, total);
}

// ---- few rows ---------------------------------------------------------------------------------------
// S = Q K^T and O += P V as m16n8k16 MMAs with the rows (padded to 16) on the M side: a warp's P comes out of its S accumulators in
// the layout that the next MMA wants.  Each warp keeps (m, l, O) of its own tokens; they meet once per segment.  P enters as
// bf16(P) + bf16(P - bf16(P)), so that o is off by no more than its own rounding (the MMAs are nowhere near their limit here).
//
// e4m3 rows are expanded in registers: the code's bits, shifted into bf16's fields, are the value times 2^-120 (subnormals included).  The
// channels of a 16-channel step are taken in the order in which ldmatrix hands out their bytes (q is loaded in the same order), and the
// MMAs' columns of O alternate between even and odd channels.  2^60 goes into q; the scale of a K row, 2^60 and the rest of 2^120 into
// its logit, that of a V row and 2^60 into its P, and the last 2^60 into the result.
constexpr int kFewThreads = 288;
constexpr int kFewWarps = 8;
constexpr uint32_t kFewMerge = 32 * 1024;

template <bool E4M3> struct FewLayout {
    static constexpr uint32_t kOperand = kTokTile * (E4M3 ? 128u : 256u);
    static constexpr uint32_t kStage = 2 * kOperand;
    static constexpr int kStages = E4M3 ? 6 : 3;
    static constexpr uint32_t kMerge = kStages * kStage, kScales = kMerge + kFewMerge;             // [stage][K, V][128] scale bytes
    static constexpr uint32_t kBars = kScales + (E4M3 ? (uint32_t)kStages * 256u : 0u);    // full, empty
    static constexpr uint32_t kEnd = kBars + 2u * kStages * 8u;
    static constexpr uint32_t kSmem = kEnd + 1024;                                         // + alignment slack
};

// (b0, b1) and (b2, b3), or (b0, b2) and (b1, b3), of four codes as bf16 pairs, each value times 2^-120
__device__ __forceinline__ void expand_adjacent(uint32_t x, uint32_t& p01, uint32_t& p23) {
    uint32_t lo, hi;
    expand(x, lo, hi);
    p01 = __byte_perm(lo, hi, 0x5140); p23 = __byte_perm(lo, hi, 0x7362);
}
__device__ __forceinline__ void expand_alternate(uint32_t x, uint32_t& p02, uint32_t& p13) {
    uint32_t lo, hi;
    expand(x, lo, hi);
    p02 = __byte_perm(lo, hi, 0x6240); p13 = __byte_perm(lo, hi, 0x7351);
}
// A operand of step ks: channels 16 ks + 2 c, + 1 (then + 8) of rows g and g + 8; e4m3: 16 ks + 4 c, + 1 (then + 2), times 2^60.
// A row that is not there (nullptr) is zero.
template <bool E4M3>
__device__ __forceinline__ uint4 q_fragment(const __nv_bfloat16* lo, const __nv_bfloat16* hi, int ks, int c) {
    uint32_t w[4];
    const __nv_bfloat16* src[2] = {lo, hi};
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
        if (E4M3) {
            const uint2 u = src[hf] ? *reinterpret_cast<const uint2*>(src[hf] + ks * 16 + c * 4) : make_uint2(0u, 0u);
            const __nv_bfloat162 up = __floats2bfloat162_rn(0x1p60f, 0x1p60f);
            const __nv_bfloat162 x = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&u.x), up), y = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&u.y), up);
            w[hf] = *reinterpret_cast<const uint32_t*>(&x); w[2 + hf] = *reinterpret_cast<const uint32_t*>(&y);
        } else {
            const uint32_t* u = reinterpret_cast<const uint32_t*>(src[hf]);
            w[hf] = u ? u[ks * 8 + c] : 0u; w[2 + hf] = u ? u[ks * 8 + 4 + c] : 0u;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void mma_q(float (&d)[4], uint4 q, uint32_t b0, uint32_t b1) {
    const uint32_t a[4] = {q.x, q.y, q.z, q.w};
    mma_bf16(d, a, b0, b1);
}
// barriers of the eight consumer warps
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
__device__ __forceinline__ bool consumers_or(bool x) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)x) : "memory");
    return r != 0;
}
// 2^(s - 67): a row's scale with the 2^60 that is due beside it
__device__ __forceinline__ float scale_60(uint32_t s) { return __uint_as_float(s > 186u ? 0x7fc00000u : (s + 60u) << 23); }

// Copies the tile's pages (and scales) into a stage; all lanes of a warp.  `page`: of the lane's box, -1 for rows of zeros.
template <bool E4M3>
__device__ __forceinline__ void few_issue(const AttnParams& p, const CUtensorMap* mk, const CUtensorMap* mv, uint32_t stage, uint32_t scales, uint32_t bar,
                                          int lane, int page, int h, int t0) {
    using L = FewLayout<E4M3>;
    if (lane == 0) mbar_expect_tx(bar, L::kStage);
    __syncwarp();
    const int n = kTokTile / p.box, slot = (t0 + lane * p.box) % p.c.P, hh = p.one_head ? 0 : h;
    if (lane < n) {
        if (E4M3) {
            const uint32_t d = stage + lane * p.box * 128;
            tma_load_4d(d, mk, bar, 0, slot, hh, page);
            tma_load_4d(d + L::kOperand, mv, bar, 0, slot, hh, page);
        } else {
            const uint32_t d = stage + lane * p.box * 128;
            tma_load_4d(d, mk, bar, 0, slot, hh, page);
            tma_load_4d(d + kHalfBytes, mk, bar, 64, slot, hh, page);
            tma_load_4d(d + L::kOperand, mv, bar, 0, slot, hh, page);
            tma_load_4d(d + L::kOperand + kHalfBytes, mv, bar, 64, slot, hh, page);
        }
    }
    if (E4M3) {                              // 8 scale bytes per lane: lanes 0-15 K, 16-31 V
        const int t8 = (lane & 15) * 8, pg = __shfl_sync(0xffffffffu, page, t8 / p.box);
        const uint8_t* base = lane < 16 ? p.c.ks : p.c.vs;
        const uint8_t* src = base + (pg < 0 ? 0ll : pg * p.c.ss_p + h * p.c.ss_h + (t0 + t8) % p.c.P);
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(scales + (lane >> 4) * 128 + t8), "l"(src), "r"(pg < 0 ? 0 : 8) : "memory");
        asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
    }
}

template <int MT, bool E4M3>
__global__ void __launch_bounds__(kFewThreads, 1)
few_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttnParams p) {
    constexpr int ROWS = 16 * MT;
    using L = FewLayout<E4M3>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t sbase = smem_u32(smem);
    __shared__ RunScratch scratch;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto full = [&](int i) { return sbase + L::kBars + 8u * (uint32_t)i; };
    auto empty = [&](int i) { return sbase + L::kBars + 8u * (uint32_t)(L::kStages + i); };
    if (threadIdx.x == 0) {
        prefetch_tmap(&map_k); prefetch_tmap(&map_v);
        for (int i = 0; i < L::kStages; ++i) { mbar_init(full(i), E4M3 ? 33 : 1); mbar_init(empty(i), kFewWarps); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = 0u;        // no wait of this call can have given up yet (each lasts seconds)
    const Run run = find_run<ROWS>(p, &scratch);                    // (its barriers also publish the mbarriers)
    int fail_site = 0;

    if (warp == kFewWarps) {
        // ===================================== producer =====================================
        Segments<ROWS> seg(p, run);
        bool more = seg.next();
        int tile = seg.ta;
        auto page_at = [&]() -> int {                               // the lane's box of the current tile
            const int t = tile * kTokTile + lane * p.box;
            return lane < kTokTile / p.box && t < seg.m.len ? p.c.page_of(seg.m.b, seg.m.h, t) : -1;
        };
        int page = more ? page_at() : -1;
        int n = 0;
        while (more) {
            const int pg = page, h = seg.m.h, t0 = tile * kTokTile;
            if (++tile == seg.tb) { more = seg.next(); tile = seg.ta; }
            if (more) page = page_at();                             // the next tile's page numbers travel meanwhile
            const int st = n % L::kStages;
            if (!__all_sync(0xffffffffu, mbar_wait(empty(st), ((n / L::kStages) & 1) ^ 1))) { fail_site = __LINE__; break; }
            few_issue<E4M3>(p, &map_k, &map_v, sbase + st * L::kStage, sbase + L::kScales + st * 256, full(st), lane, pg, h, t0);
            ++n;
        }
        for (int back = 0; back < L::kStages && back < n; ++back) { // no copy may be under way when the CTA leaves
            const int k = n - 1 - back;
            (void)mbar_wait(full(k % L::kStages), (k / L::kStages) & 1);
        }
    } else {
        // ===================================== consumers ====================================
        const int g = lane >> 2, c = lane & 3;
        const int tok0 = warp * 16;                                 // the warp's tokens of a tile
        Segments<ROWS> seg(p, run);
        int n = 0;
        while (seg.next()) {
            const Item m = seg.m;
            // q in the MMAs' layout: in registers, or, two row tiles (which would not fit), in the merge buffer, a step of 16 channels per warp
            uint4* sq = reinterpret_cast<uint4*>(smem + L::kMerge);            // [mt][ks][lane]
            uint4 qf[8];
            int seen[MT][2];
            float mx[MT][2], l[MT][2];
            float o[MT][16][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const __nv_bfloat16* src[2];
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const int r = mt * 16 + hf * 8 + g;
                    seen[mt][hf] = seen_by(p, m, r);
                    mx[mt][hf] = -INFINITY; l[mt][hf] = 0.f;
                    src[hf] = nullptr;
                    if (r < m.rows) {
                        int head, i;
                        row_place(p, m, r, head, i);
                        src[hf] = static_cast<const __nv_bfloat16*>(p.q.ptr) + m.b * p.q.sb + head * p.q.sh + i * p.q.st;
                    }
                }
                if (MT == 1) {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) qf[ks] = q_fragment<E4M3>(src[0], src[1], ks, c);
                } else {
                    sq[(mt * 8 + warp) * 32 + lane] = q_fragment<E4M3>(src[0], src[1], warp, c);
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) { o[mt][j][0] = 0.f; o[mt][j][1] = 0.f; o[mt][j][2] = 0.f; o[mt][j][3] = 0.f; }
            }
            if (MT > 1) consumers_sync();
            auto q_at = [&](int mt, int ks) { return MT == 1 ? qf[ks] : sq[(mt * 8 + ks) * 32 + lane]; };
            const int first_masked = p.causal ? min(max(m.len - m.ql + m.r0 / p.G + 1, 0), m.len) : m.len;   // tokens that not every row sees begin here

            for (int tile = seg.ta; tile < seg.tb; ++tile, ++n) {
                const int st = n % L::kStages;
                uint8_t* sk = smem + st * L::kStage;
                uint8_t* sv = sk + L::kOperand;
                if (!__all_sync(0xffffffffu, mbar_wait(full(st), (n / L::kStages) & 1))) { fail_site = __LINE__; break; }
                const int t0 = tile * kTokTile + tok0;              // the warp's first token
                const bool edge = t0 + 16 > first_masked;           // some row does not see some of the 16 tokens
                float s[MT][2][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[mt][nt][j] = 0.f;
                if (E4M3) {
#pragma unroll
                    for (int pc = 0; pc < 8; pc += 2) {
                        const int mi = lane >> 3, row = tok0 + (mi >> 1) * 8 + (lane & 7), piece = pc + (mi & 1);
                        uint32_t r[4];
                        ldsm_x4(r, sk + row * 128 + ((piece ^ (row & 7)) << 4));
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            uint32_t b0, b1, b2, b3;
                            expand_adjacent(r[u], b0, b1);
                            expand_adjacent(r[2 + u], b2, b3);
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                const uint4 q = q_at(mt, pc + u);
                                mma_q(s[mt][0], q, b0, b1);
                                mma_q(s[mt][1], q, b2, b3);
                            }
                        }
                    }
                } else {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) {
                        const int mi = lane >> 3, row = tok0 + (mi >> 1) * 8 + (lane & 7), piece = 2 * ks + (mi & 1);
                        uint32_t r[4];
                        ldsm_x4(r, sk + (piece >> 3) * kHalfBytes + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            const uint4 q = q_at(mt, ks);
                            mma_q(s[mt][0], q, r[0], r[1]);
                            mma_q(s[mt][1], q, r[2], r[3]);
                        }
                    }
                }
                float fk[2][2], fv[2][2];                           // factors of the lane's tokens 8 nt + 2 c, + 1
                if (E4M3) {
                    const uint8_t* sc = smem + L::kScales + st * 256 + tok0 + 2 * c;
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) {
                        const uint32_t k2 = *reinterpret_cast<const uint16_t*>(sc + nt * 8), v2 = *reinterpret_cast<const uint16_t*>(sc + 128 + nt * 8);
                        fk[nt][0] = scale_60(k2 & 255u) * p.sl2; fk[nt][1] = scale_60(k2 >> 8) * p.sl2;
                        fv[nt][0] = scale_60(v2 & 255u); fv[nt][1] = scale_60(v2 >> 8);
                    }
                }
                uint32_t ph[MT][4], pl[MT][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    float tm[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float x = s[mt][nt][j] * (E4M3 ? fk[nt][j & 1] : p.sl2);
                            if (edge && t0 + nt * 8 + 2 * c + (j & 1) >= seen[mt][j >> 1]) x = -INFINITY;
                            s[mt][nt][j] = x;
                            tm[j >> 1] = fmaxf(tm[j >> 1], x);
                        }
                    bool move = false;
                    float f[2] = {1.f, 1.f};
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        tm[hf] = fmaxf(tm[hf], __shfl_xor_sync(0xffffffffu, tm[hf], 1));
                        tm[hf] = fmaxf(tm[hf], __shfl_xor_sync(0xffffffffu, tm[hf], 2));
                        // the reference moves only when the maximum exceeds it by 2^8: P stays far inside fp32's and bf16's range
                        if (tm[hf] > mx[mt][hf] + 8.f) { f[hf] = exp2f(mx[mt][hf] - tm[hf]); mx[mt][hf] = tm[hf]; move = true; }
                        l[mt][hf] *= f[hf];
                    }
                    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) { o[mt][j][0] *= f[0]; o[mt][j][1] *= f[0]; o[mt][j][2] *= f[1]; o[mt][j][3] *= f[1]; }
                    }
                    float e[2][4];
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float ref = mx[mt][j >> 1];
                            const float x = fast_exp2(s[mt][nt][j] - (ref == -INFINITY ? 0.f : ref));
                            l[mt][j >> 1] += x;
                            e[nt][j] = E4M3 ? (x > 0.f ? x * fv[nt][j & 1] : x) : x;      // (a NaN logit stays NaN; a token not seen has weight 0 whatever its scale)
                        }
                    split_bf16x2(e[0][0], e[0][1], ph[mt][0], pl[mt][0]);
                    split_bf16x2(e[0][2], e[0][3], ph[mt][1], pl[mt][1]);
                    split_bf16x2(e[1][0], e[1][1], ph[mt][2], pl[mt][2]);
                    split_bf16x2(e[1][2], e[1][3], ph[mt][3], pl[mt][3]);
                }
                if (E4M3) {
#pragma unroll
                    for (int pc = 0; pc < 8; pc += 2) {
                        const int mi = lane >> 3, row = tok0 + (mi & 1) * 8 + (lane & 7), piece = pc + (mi >> 1);
                        uint32_t r[4];
                        ldsm_x4_trans(r, sv + row * 128 + ((piece ^ (row & 7)) << 4));
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            uint32_t e0, o0, e1, o1;                // even and odd channels of tokens 0-7 and 8-15
                            expand_alternate(r[2 * u], e0, o0);
                            expand_alternate(r[2 * u + 1], e1, o1);
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                mma_bf16(o[mt][2 * (pc + u)], ph[mt], e0, e1);
                                mma_bf16(o[mt][2 * (pc + u) + 1], ph[mt], o0, o1);
                                mma_bf16(o[mt][2 * (pc + u)], pl[mt], e0, e1);
                                mma_bf16(o[mt][2 * (pc + u) + 1], pl[mt], o0, o1);
                            }
                        }
                    }
                } else {
                    if (edge) {
                        // rows that not every query sees: those behind the list's end may hold anything and become zeros; one that
                        // is not finite must reach the queries that see it alone
                        bool odd = false;
                        const int row = tok0 + (lane >> 1), t = t0 + (lane >> 1);
                        uint4* at = reinterpret_cast<uint4*>(sv + (lane & 1) * kHalfBytes + row * 128);
                        if (t >= m.len) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) at[j] = make_uint4(0u, 0u, 0u, 0u);
                        } else if (t >= first_masked) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const uint4 u = at[j];
                                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                                for (int x = 0; x < 4; ++x) odd |= (w[x] & 0x7f80u) == 0x7f80u || (w[x] & 0x7f800000u) == 0x7f800000u;
                            }
                        }
                        __syncwarp();
                        unsigned bad = __ballot_sync(0xffffffffu, odd);
                        while (bad) {                               // token by token, on CUDA cores; the row is zeroed for the MMAs
                            const int tk = (__ffs(bad) - 1) >> 1;
                            bad &= ~(3u << (2 * tk));
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                const int src = (lane & ~3) | ((tk & 7) >> 1);
                                float w[2];
#pragma unroll
                                for (int hf = 0; hf < 2; ++hf) {
                                    const uint32_t hi = __shfl_sync(0xffffffffu, tk & 8 ? ph[mt][2 + hf] : ph[mt][hf], src);
                                    const uint32_t lo = __shfl_sync(0xffffffffu, tk & 8 ? pl[mt][2 + hf] : pl[mt][hf], src);
                                    w[hf] = tk & 1 ? __uint_as_float(hi & 0xffff0000u) + __uint_as_float(lo & 0xffff0000u)
                                                   : __uint_as_float(hi << 16) + __uint_as_float(lo << 16);
                                }
#pragma unroll
                                for (int j = 0; j < 16; ++j) {
                                    const int rw = tok0 + tk;
                                    const uint32_t two = *reinterpret_cast<const uint32_t*>(sv + (j >> 3) * kHalfBytes + rw * 128 + (((j & 7) ^ (rw & 7)) << 4) + c * 4);
                                    const float v0 = __uint_as_float(two << 16), v1 = __uint_as_float(two & 0xffff0000u);
                                    if (t0 + tk < seen[mt][0]) { o[mt][j][0] += w[0] * v0; o[mt][j][1] += w[0] * v1; }
                                    if (t0 + tk < seen[mt][1]) { o[mt][j][2] += w[1] * v0; o[mt][j][3] += w[1] * v1; }
                                }
                            }
                            __syncwarp();
                            if (lane < 16) *reinterpret_cast<uint4*>(sv + (lane >> 3) * kHalfBytes + (tok0 + tk) * 128 + ((lane & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
                            __syncwarp();
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int mi = lane >> 3, row = tok0 + (mi & 1) * 8 + (lane & 7), piece = 2 * j + (mi >> 1);
                        uint32_t r[4];
                        ldsm_x4_trans(r, sv + (piece >> 3) * kHalfBytes + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            mma_bf16(o[mt][2 * j], ph[mt], r[0], r[1]);
                            mma_bf16(o[mt][2 * j + 1], ph[mt], r[2], r[3]);
                            mma_bf16(o[mt][2 * j], pl[mt], r[0], r[1]);
                            mma_bf16(o[mt][2 * j + 1], pl[mt], r[2], r[3]);
                        }
                    }
                }
                if (edge && !E4M3) fence_async_smem();              // this thread's writes to the stage precede the bulk copy into it
                __syncwarp();
                if (lane == 0) mbar_arrive(empty(st));
            }

            // ---- the warps' results meet: maxima and sums, then O, eight rows at a time ----
            float* sm = reinterpret_cast<float*>(smem + L::kMerge + 8192);     // [warp][ROWS] maxima, then sums (behind q, which slower warps still read)
            float* sl = sm + kFewWarps * ROWS;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    l[mt][hf] += __shfl_xor_sync(0xffffffffu, l[mt][hf], 1);
                    l[mt][hf] += __shfl_xor_sync(0xffffffffu, l[mt][hf], 2);
                    if (c == 0) { sm[warp * ROWS + mt * 16 + hf * 8 + g] = mx[mt][hf]; sl[warp * ROWS + mt * 16 + hf * 8 + g] = l[mt][hf]; }
                }
            if (consumers_or(fail_site != 0)) {                     // one warp's wait gave up: all leave
                if (!fail_site) fail_site = __LINE__;
                break;
            }
            float ref[MT][2], total[MT][2];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const int r = mt * 16 + hf * 8 + g;
                    float top = -INFINITY;
#pragma unroll
                    for (int w = 0; w < kFewWarps; ++w) top = fmaxf(top, sm[w * ROWS + r]);
                    ref[mt][hf] = top == -INFINITY ? 0.f : top;
                    total[mt][hf] = 0.f;
#pragma unroll
                    for (int w = 0; w < kFewWarps; ++w) total[mt][hf] = fmaf(exp2f(sm[w * ROWS + r] - ref[mt][hf]), sl[w * ROWS + r], total[mt][hf]);
                }
            const bool whole = seg.whole();
            float2* buf = reinterpret_cast<float2*>(smem + L::kMerge);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    if (mt * 16 + hf * 8 >= m.rows) break;
                    consumers_sync();                               // the buffer is free (again)
                    const int r = mt * 16 + hf * 8 + g;
                    const float f = exp2f(mx[mt][hf] - ref[mt][hf]), sum = total[mt][hf];
#pragma unroll
                    for (int j = 0; j < 16; ++j) buf[(warp * 16 + j) * 32 + lane] = make_float2(o[mt][j][2 * hf] * f, o[mt][j][2 * hf + 1] * f);
                    consumers_sync();
                    // this thread: columns 2 * warp and 2 * warp + 1 of the lane's row, from all warps
                    float2 a = make_float2(0.f, 0.f), b = a;
#pragma unroll
                    for (int w = 0; w < kFewWarps; ++w) {
                        const float2 x = buf[(w * 16 + 2 * warp) * 32 + lane], y = buf[(w * 16 + 2 * warp + 1) * 32 + lane];
                        a.x += x.x; a.y += x.y; b.x += y.x; b.y += y.y;
                    }
                    if (r >= m.rows) continue;
                    const float k = (E4M3 ? 0x1p60f : 1.f) * (whole ? (sum != 0.f ? 1.f / sum : 0.f) : 1.f);
                    a.x *= k; a.y *= k; b.x *= k; b.y *= k;
                    if (whole) {
                        int head, i;
                        row_place(p, m, r, head, i);
                        __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(const_cast<void*>(p.o.ptr)) + m.b * p.o.sb + head * p.o.sh + i * p.o.st + 16 * warp;
                        if (E4M3) {                                 // channels 4 c .. 4 c + 3
                            *reinterpret_cast<uint2*>(dst + 4 * c) = make_uint2(pack_bf16x2(a.x, b.x), pack_bf16x2(a.y, b.y));
                        } else {
                            *reinterpret_cast<uint32_t*>(dst + 2 * c) = pack_bf16x2(a.x, a.y);
                            *reinterpret_cast<uint32_t*>(dst + 8 + 2 * c) = pack_bf16x2(b.x, b.y);
                        }
                        if (p.lse && warp == 0 && c == 0) p.lse[((size_t)m.b * p.c.Hkv * p.G + head) * p.T + i] = lse_of(ref[mt][hf], sum);
                    } else {
                        const size_t at = seg.slot() * ROWS + r;
                        float* dst = p.part_o + at * kD + 16 * warp;
                        if (E4M3) {
                            *reinterpret_cast<float4*>(dst + 4 * c) = make_float4(a.x, b.x, a.y, b.y);
                        } else {
                            *reinterpret_cast<float2*>(dst + 2 * c) = a;
                            *reinterpret_cast<float2*>(dst + 8 + 2 * c) = b;
                        }
                        if (warp == 0 && c == 0) { p.part_m[at] = sum == 0.f ? -INFINITY : ref[mt][hf]; p.part_l[at] = sum; }
                    }
                }
            consumers_sync();                                       // the buffer is free for the next segment's statistics
            if (threadIdx.x == 0) note_item<ROWS>(p, run, seg);
        }
    }
    if (fail_site && lane == 0) atomicCAS(p.status, 0u, (unsigned)fail_site);
}

// ---- fp32 on CUDA cores ---------------------------------------------------------------------------------
// 16 rows x 64 tokens at a time: logits by (token, four rows) per thread, softmax and P V by warps of two rows each, whose
// statistics and outputs stay in registers.  Bound by fp32 multiply-adds from 16 rows on, by the bytes below.
constexpr int kF32Threads = 256, kF32Rows = 16, kF32Tok = 64, kF32Pitch = kD + 4;
constexpr size_t kF32Smem = sizeof(float) * (kF32Tok * kF32Pitch + kF32Tok * kD + kF32Rows * kD + kF32Rows * kF32Tok);

__global__ void __launch_bounds__(kF32Threads, 2)
paged_f32_kernel(const __grid_constant__ AttnParams p) {
    extern __shared__ __align__(16) float sf[];
    float* sK = sf;                                   // [64][132]
    float* sV = sK + kF32Tok * kF32Pitch;             // [64][128]
    float* sQ = sV + kF32Tok * kD;                    // [16][128]
    float* sS = sQ + kF32Rows * kD;                   // [16][64]
    __shared__ RunScratch scratch;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_wait();
    if (blockIdx.x == 0 && tid == 0) *p.status = 0u;
    const Run run = find_run<kF32Rows>(p, &scratch);
    Segments<kF32Rows> seg(p, run);
    while (seg.next()) {
        const Item m = seg.m;
        __syncthreads();
        for (int e = tid; e < kF32Rows * (kD / 4); e += kF32Threads) {
            const int r = e / (kD / 4), c4 = e % (kD / 4);
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < m.rows) {
                int head, i;
                row_place(p, m, r, head, i);
                x = load4(static_cast<const float*>(p.q.ptr) + m.b * p.q.sb + head * p.q.sh + i * p.q.st + c4 * 4);
            }
            *reinterpret_cast<float4*>(sQ + r * kD + c4 * 4) = x;
        }
        const int r0 = 2 * warp;                      // this warp's rows in the softmax and in P V
        const int seen[2] = {seen_by(p, m, r0), seen_by(p, m, r0 + 1)};
        float mx[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
        for (int t0 = seg.ta * kTokTile; t0 < min(seg.tb * kTokTile, m.len); t0 += kF32Tok) {
            float4 kx[8], vx[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {             // a warp fetches whole rows: token warp + 8 u
                const int t = t0 + warp + 8 * u;
                kx[u] = make_float4(0.f, 0.f, 0.f, 0.f); vx[u] = kx[u];
                const int page = t < m.len ? p.c.page_of(m.b, m.h, t) : -1;
                if (page >= 0) {
                    kx[u] = load4(static_cast<const float*>(p.c.k.ptr) + page * p.c.k.sb + m.h * p.c.k.sh + (t % p.c.P) * p.c.k.st + lane * 4);
                    vx[u] = load4(static_cast<const float*>(p.c.v.ptr) + page * p.c.v.sb + m.h * p.c.v.sh + (t % p.c.P) * p.c.v.st + lane * 4);
                }
            }
            __syncthreads();                          // the preceding tile is no longer read
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                *reinterpret_cast<float4*>(sK + (warp + 8 * u) * kF32Pitch + lane * 4) = kx[u];
                *reinterpret_cast<float4*>(sV + (warp + 8 * u) * kD + lane * 4) = vx[u];
            }
            __syncthreads();
            {
                const int tk = tid & (kF32Tok - 1), q0 = (tid / kF32Tok) * 4;
                float s[4] = {0.f, 0.f, 0.f, 0.f};
                if (q0 < m.rows) {
#pragma unroll 8
                    for (int c4 = 0; c4 < kD / 4; ++c4) {
                        const float4 kv = *reinterpret_cast<const float4*>(sK + tk * kF32Pitch + c4 * 4);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float4 qv = *reinterpret_cast<const float4*>(sQ + (q0 + j) * kD + c4 * 4);
                            s[j] = fmaf(qv.x, kv.x, s[j]); s[j] = fmaf(qv.y, kv.y, s[j]); s[j] = fmaf(qv.z, kv.z, s[j]); s[j] = fmaf(qv.w, kv.w, s[j]);
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) sS[(q0 + j) * kF32Tok + tk] = s[j] * p.sl2;
            }
            __syncthreads();
            if (r0 < m.rows) {
                int n[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    n[j] = min(seen[j] - t0, kF32Tok);                  // tokens of this step that the row sees
                    float* row = sS + (r0 + j) * kF32Tok;
                    const float a = lane < n[j] ? row[lane] : -INFINITY, b = lane + 32 < n[j] ? row[lane + 32] : -INFINITY;
                    const float top = fmaxf(warp_max(fmaxf(a, b)), mx[j]);
                    const float ref = top == -INFINITY ? 0.f : top, f = exp2f(mx[j] - ref);
                    const float ea = exp2f(a - ref), eb = exp2f(b - ref);
                    l[j] = fmaf(l[j], f, ea + eb);                      // per lane; joined at the end
                    acc[j].x *= f; acc[j].y *= f; acc[j].z *= f; acc[j].w *= f;
                    mx[j] = top;
                    row[lane] = ea; row[lane + 32] = eb;
                }
                __syncwarp();
                const int both = min(n[0], n[1]), most = max(n[0], n[1]);
                for (int t = 0; t < most; ++t) {                        // (a row's later queries see at least what its earlier ones see)
                    const float4 v = *reinterpret_cast<const float4*>(sV + t * kD + lane * 4);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (t >= both && t >= n[j]) continue;           // tokens it does not see, infinite ones among them, stay out
                        const float w = sS[(r0 + j) * kF32Tok + t];
                        acc[j].x = fmaf(w, v.x, acc[j].x); acc[j].y = fmaf(w, v.y, acc[j].y);
                        acc[j].z = fmaf(w, v.z, acc[j].z); acc[j].w = fmaf(w, v.w, acc[j].w);
                    }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = r0 + j;
            const float total = warp_sum(l[j]), ref = mx[j] == -INFINITY ? 0.f : mx[j];
            if (r >= m.rows) continue;
            if (seg.whole()) {
                const float inv = total != 0.f ? 1.f / total : 0.f;
                int head, i;
                row_place(p, m, r, head, i);
                float* dst = static_cast<float*>(const_cast<void*>(p.o.ptr)) + m.b * p.o.sb + head * p.o.sh + i * p.o.st + lane * 4;
                *reinterpret_cast<float4*>(dst) = make_float4(acc[j].x * inv, acc[j].y * inv, acc[j].z * inv, acc[j].w * inv);
                if (p.lse && lane == 0) p.lse[((size_t)m.b * p.c.Hkv * p.G + head) * p.T + i] = lse_of(ref, total);
            } else {
                const size_t at = seg.slot() * kF32Rows + r;
                *reinterpret_cast<float4*>(p.part_o + at * kD + lane * 4) = acc[j];
                if (lane == 0) { p.part_m[at] = mx[j]; p.part_l[at] = total; }
            }
        }
        if (tid == 0) note_item<kF32Rows>(p, run, seg);
    }
}

// ---- host side --------------------------------------------------------------------------------------
struct AttnPlan { int rows, grid, nrt, items; size_t off_info, off_m, off_l, off_o, bytes; };

AttnPlan make_plan(const PagesView& c, const AttnShape& s) {
    AttnPlan p{};
    const long long rows = (long long)s.G * s.T;
    p.rows = c.dtype == OBC_F32 ? kF32Rows : rows <= 16 ? 16 : rows <= 32 ? 32 : kChunkRows;
    p.grid = sm_count() * (c.dtype == OBC_F32 ? 2 : 1);
    p.nrt = (int)((rows + p.rows - 1) / p.rows);
    p.items = c.B * c.Hkv * p.nrt;
    size_t off = 256;                                  // header: the status word
    p.off_info = off; off = align_up(off + (size_t)p.items * sizeof(int4), 256);
    const size_t slots = 2 * (size_t)p.grid * p.rows;
    p.off_m = off; off = align_up(off + slots * 4, 256);
    p.off_l = off; off = align_up(off + slots * 4, 256);
    p.off_o = off; off = align_up(off + slots * kD * 4, 256);
    p.bytes = off;
    return p;
}

}  // namespace

size_t paged_attention_bytes(const PagesView& c, const AttnShape& s) { return make_plan(c, s).bytes; }

obc_status launch_paged_attention(const PagesView& c, const AttnShape& s, TensorView q, TensorView o, float* lse, void* ws, cudaStream_t stream) {
    const AttnPlan plan = make_plan(c, s);
    char* w = static_cast<char*>(ws);
    AttnParams p{};
    p.c = c; p.G = s.G; p.T = s.T; p.causal = s.causal; p.q_lens = s.q_lens; p.sl2 = s.scale * kLog2e;
    p.q = q; p.o = o; p.lse = lse; p.nrt = plan.nrt; p.items = plan.items;
    p.one_head = c.k.sh == 0 && c.v.sh == 0 ? 1 : 0;
    p.box = 8;
    while (p.box < kTokTile && c.P % (2 * p.box) == 0) p.box *= 2;
    p.status = reinterpret_cast<unsigned int*>(w);
    p.info = reinterpret_cast<int4*>(w + plan.off_info);
    p.part_m = reinterpret_cast<float*>(w + plan.off_m); p.part_l = reinterpret_cast<float*>(w + plan.off_l);
    p.part_o = reinterpret_cast<float*>(w + plan.off_o);
    cudaError_t e;
    if (c.dtype == OBC_F32) {
        OBC_CUDA_TRY(allow_smem(paged_f32_kernel, kF32Smem));
        ProfScope prof("paged_attention_f32", stream);
        e = launch_pdl(paged_f32_kernel, dim3(plan.grid), dim3(kF32Threads), kF32Smem, stream, 1, p);
    } else {
        CUtensorMap mk, mv;
        if (!make_page_map(&mk, c, c.k, p.box) || !make_page_map(&mv, c, c.v, p.box)) return OBC_ERR_CUDA;
        auto few = [&](auto kernel, size_t smem) {
            const cudaError_t a = allow_smem(kernel, smem);
            if (a != cudaSuccess) return a;
            ProfScope prof("paged_attention_few", stream);
            return launch_pdl(kernel, dim3(plan.grid), dim3(kFewThreads), smem, stream, 1, mk, mv, p);
        };
        auto chunk = [&](auto kernel, size_t smem, int threads, int regs) {
            cudaFuncAttributes fa{};
            cudaError_t a = cudaFuncGetAttributes(&fa, kernel);
            if (a != cudaSuccess) return a;
            if (fa.numRegs < regs) return cudaErrorInvalidKernelImage;      // its warps would wait for registers that the launch does not bring
            if ((a = allow_smem(kernel, smem)) != cudaSuccess) return a;
            ProfScope prof("paged_attention_chunk", stream);
            return launch_pdl(kernel, dim3(plan.grid), dim3(threads), smem, stream, 1, mk, mv, p);
        };
        if (plan.rows == kChunkRows)
            e = c.dtype == OBC_E4M3 ? chunk(chunk_kernel<true>, ChunkLayout<true>::kSmem, ChunkLayout<true>::kThreads, 128)
                                    : chunk(chunk_kernel<false>, ChunkLayout<false>::kSmem, ChunkLayout<false>::kThreads, 168);
        else if (c.dtype == OBC_E4M3)
            e = plan.rows == 16 ? few(few_rows_kernel<1, true>, FewLayout<true>::kSmem) : few(few_rows_kernel<2, true>, FewLayout<true>::kSmem);
        else
            e = plan.rows == 16 ? few(few_rows_kernel<1, false>, FewLayout<false>::kSmem) : few(few_rows_kernel<2, false>, FewLayout<false>::kSmem);
    }
    OBC_CUDA_TRY(e);
    auto merge = [&](auto kernel) {
        ProfScope prof("paged_attention_merge", stream);
        return launch_pdl(kernel, dim3((unsigned)plan.items * (plan.rows / 8)), dim3(256), 0, stream, 1, p);
    };
    OBC_CUDA_TRY(c.dtype == OBC_F32 ? merge(paged_merge_kernel<float, 16>)
                 : plan.rows == 16  ? merge(paged_merge_kernel<__nv_bfloat16, 16>)
                 : plan.rows == 32  ? merge(paged_merge_kernel<__nv_bfloat16, 32>)
                                    : merge(paged_merge_kernel<__nv_bfloat16, kChunkRows>));
    return OBC_OK;
}

}  // namespace obc
