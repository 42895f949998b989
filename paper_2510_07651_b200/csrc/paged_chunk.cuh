// Attention of many rows per KV list (chunks of a prompt) over a paged cache: tcgen05 MMAs with TMEM accumulators.
//
// A CTA works on 256 query rows of a list, 128 per softmax warpgroup, one row per thread.  For tile i of 128 tokens and warpgroup w:
//     S_w  = Q_w K_i^T                       accumulator in TMEM
//     P_w  = 2^(S_w scale log2 e - m_w)      registers -> bf16 -> shared memory (8-bit pages: TMEM, over S_w's first columns)
//     O_w += P_w V_i                         V as MN-major B
// A K or V tile is fetched once for both warpgroups.  m_w only moves when a tile's maximum exceeds it by more than 2^8, so that O_w is
// rescaled (in TMEM, by the thread that owns the row) a few times per list.
// With P in shared memory S_w(i+1) is formed while P_w(i) is still at work (S_w is free as soon as its values are in registers), so that a
// warpgroup finds its next logits ready: 512 rows over 16384 tokens, 32 heads on 8, 137 -> 130 us; a 4096-token prompt 163 -> 157 us; the last 512 of 131072 tokens
// 913 -> 865 us.  It takes 64 KB, which leaves the ring three operands of 32 KB.  8-bit pages need raw tiles beside that ring and would be left with two: there P
// stays in TMEM, the MMAs of a warpgroup execute in order (S_w(i+1) cannot overwrite P_w(i) before P_w V(i) has read it), and those of one
// run while the other is at its exponentials.
//
//   warps 0, 2   producers of K and of V: pages -> ring of 32 KB operands; 8-bit pages -> a raw tile each and its scales.  In V tiles at a list's end (16 bits)
//                rows behind it become zeros; rows that are not finite and that not every query sees become zeros, too, and are named to the softmax warps,
//                which add them by hand where they are seen
//   warps 1, 3   MMA issuers, one for each softmax warpgroup (one thread for both was what set the pace)
//   warps 4-11   softmax, two warpgroups; each fetches its Q
//   warps 12-15  (8-bit pages) codes -> bf16 tiles, the scale multiplied in exactly; and what warp 2 does for V tiles
// TMEM columns: S_0 [0,128)  S_1 [128,256)  O_0 [256,384)  O_1 [384,512)
#pragma once
#include "paged_common.cuh"
#include "tc_ptx.cuh"

namespace obc {
namespace {

constexpr int kChunkRows = 256;

template <bool E4M3> struct ChunkLayout {
    static constexpr int kThreads = E4M3 ? 512 : 384;
    static constexpr bool kPS = !E4M3;                                              // P in shared memory
    // quarters of a tile's exponentials before the other warpgroup's turn.  With P in TMEM all: then the MMAs of one run beside the exponentials of the other.  Else half
    // of them: one warp alone does not keep the unit busy (512 rows over 16384 tokens: 136 us with all, 133, 125, 126
    // with 1, 2, 3; the last 512 of 131072 tokens on another GPU: 930 us with all, 995 without turns)
    static constexpr int kTurn = kPS ? 2 : 4;
    static constexpr int kSlots = E4M3 ? 4 : 3;                                        // bf16 operands of 32 KB
    static constexpr int kRaw = E4M3 ? 2 : 0;                                          // raw operands of 16 KB
    static constexpr uint32_t kQ = 0, kP = 2 * kOperandBytes, kRing = (kPS ? 4 : 2) * kOperandBytes, kRawAt = kRing + kSlots * kOperandBytes;
    static constexpr uint32_t kScales = kRawAt + kRaw * 16384u;                        // [raw slot][128]
    static constexpr uint32_t kBad = kScales + kRaw * 128u;                            // [slot][4] words: tokens to be added by hand
    static constexpr uint32_t kBars = kBad + kSlots * 16u;
    enum { FULL = 0, EMPTY = kSlots, EDGE = 2 * kSlots, QFULL = 3 * kSlots, SFULL = QFULL + 2, PFULL = SFULL + 2, TURN = PFULL + 2, ODONE = TURN + 8, SFREE = ODONE + 2, RAWFULL = SFREE + 2,
           RAWEMPTY = RAWFULL + 2, NBARS = RAWEMPTY + 2 };
    static constexpr uint32_t kTmem = kBars + NBARS * 8u;
    static constexpr uint32_t kSmem = kTmem + 16 + 1024;
    // registers: softmax warpgroups against the others, out of what the launch gives all threads
    static constexpr int kSoftRegs = E4M3 ? 184 : 208, kOtherRegs = E4M3 ? 72 : 88;
    static_assert(!kPS || kSlots >= 3, "places between two operands of a producer");
    static_assert(256 * kSoftRegs + (kThreads - 256) * kOtherRegs <= kThreads * (E4M3 ? 128 : 168), "registers");
};

// a segment as the roles of the CTA see it
struct ChunkSeg {
    int n, cnt0, cnt1;                       // tiles; of warpgroup 0 and 1 (from the segment's first tile on)
    int first_masked;                        // tokens from here on are not seen by every row of the item
    __device__ __forceinline__ int cnt(int w) const { return w ? cnt1 : cnt0; }
};
__device__ __forceinline__ ChunkSeg chunk_seg(const AttnParams& p, const Segments<kChunkRows>& s) {
    ChunkSeg c;
    c.n = s.tb - s.ta;
    const int t0 = max((seen_by(p, s.m, min(s.m.rows, 128) - 1) + kTokTile - 1) / kTokTile, 1);
    const int t1 = s.m.rows > 128 ? (seen_by(p, s.m, s.m.rows - 1) + kTokTile - 1) / kTokTile : 0;
    c.cnt0 = min(max(min(t0, s.tb) - s.ta, 0), c.n);
    c.cnt1 = min(max(min(t1, s.tb) - s.ta, 0), c.n);
    c.first_masked = seen_by(p, s.m, 0);
    return c;
}

// a value that all lanes of the warp have, known as such
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ bool elect_one() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void tc_ld1(uint32_t taddr, uint32_t& r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;" : "=r"(r) : "r"(taddr) : "memory");
}
// 32 bytes in one store (a whole sector; two stores of 16 bytes by each of 32 lanes in rows of their own take twice the requests)
__device__ __forceinline__ void store32(void* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f, uint32_t g, uint32_t h) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e), "r"(f), "r"(g), "r"(h) : "memory");
}
template <int N> __device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// Four bytes (e4m3 codes) -> two bf16 pairs times m (a power of two).  Through fp16 and fp32, of which a code's values need the upper half alone: the
// hardware's conversion knows NaN.
__device__ __forceinline__ void codes_to_bf16(uint32_t x, __nv_bfloat162 m, uint32_t& p01, uint32_t& p23) {
    uint32_t h[2];
    expand_adjacent(x, h[0], h[1]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        const uint32_t b = __byte_perm(__float_as_uint(f.x), __float_as_uint(f.y), 0x7632);
        const __nv_bfloat162 u = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&b), m);
        (i ? p23 : p01) = *reinterpret_cast<const uint32_t*>(&u);
    }
}

// 16 bytes of shared memory
__device__ __forceinline__ uint4 lds16(uint32_t at) {
    uint4 u;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(at) : "memory");
    return u;
}
__device__ __forceinline__ void sts16(uint32_t at, uint4 u) { asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(u.x), "r"(u.y), "r"(u.z), "r"(u.w) : "memory"); }

template <bool E4M3>
__global__ void __launch_bounds__(ChunkLayout<E4M3>::kThreads, 1)
chunk_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ AttnParams p) {
    using L = ChunkLayout<E4M3>;
    constexpr int NS = L::kSlots;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t sbase = smem_u32(smem);
    __shared__ RunScratch scratch;
    auto bar = [&](int i) { return sbase + L::kBars + 8u * (uint32_t)i; };
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + L::kTmem);
    uint32_t* bad_words = reinterpret_cast<uint32_t*>(smem + L::kBad);
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        prefetch_tmap(&map_k); prefetch_tmap(&map_v);
        for (int i = 0; i < NS; ++i) { mbar_init(bar(L::FULL + i), E4M3 ? 4 : 1); mbar_init(bar(L::EMPTY + i), 2); mbar_init(bar(L::EDGE + i), 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(L::QFULL + i), 128); mbar_init(bar(L::SFULL + i), 1); mbar_init(bar(L::PFULL + i), 4); mbar_init(bar(L::ODONE + i), 1); mbar_init(bar(L::SFREE + i), 4);
            mbar_init(bar(L::RAWFULL + i), 33); mbar_init(bar(L::RAWEMPTY + i), 4);
        }
        for (int i = 0; i < 8; ++i) mbar_init(bar(L::TURN + i), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sbase + L::kTmem), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(*tmem_slot);
    pdl_wait();
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.status = 0u;        // no wait of this call can have given up yet (each lasts seconds)
    const Run run = find_run<kChunkRows>(p, &scratch);
    int fail_site = 0;
    auto wait = [&](int b, uint32_t parity, int line) -> bool {
        if (mbar_wait(bar(b), parity & 1u)) return true;
        fail_site = line;
        return false;
    };
    // (for whole warps that go on together: where one lane gave up all do)
    auto all_wait = [&](int b, uint32_t parity, int line) -> bool {
        if (__all_sync(0xffffffffu, wait(b, parity, line))) return true;
        fail_site = line;
        return false;
    };
    // V tiles that reach behind what every row sees pass through warp 2 before anyone else may read them (16-bit pages): their copies complete
    // on the slot's EDGE barrier, whose parity warp 2 keeps (a bit per slot), and warp 2 arrives on FULL in their stead.
    // The two producers' operands share the ring, and a wait by parity passes for a slot that is two rounds behind, too.  That cannot be as long as each
    // issuer releases operands in their order: a producer's next operand, number k, is at most three places (the ring's slots) behind its last, for which
    // operand k - 6 or a later one was released, and so k - 6 itself, the one two rounds earlier in k's slot, was.  An operand that a warpgroup does
    // not see is therefore released by a commit as well: a plain arrival would overtake the MMAs that still read the operands before it.
    // Operands are numbered in the order in which they are fetched and used.  Of a segment's n tiles, of which tile 0 is the run's tile `base`: K(0) V(0) K(1)
    // V(1) .., or with P in shared memory, where S is formed a tile ahead of P V, K(0) K(1) V(0) K(2) V(1) .. K(n-1) V(n-2) V(n-1).
    auto k_number = [](uint32_t base, int i) { return 2 * base + (L::kPS && i > 0 ? 2 * i - 1 : 2 * i); };
    auto v_number = [](uint32_t base, int i, int n) { return 2 * base + (L::kPS && i + 1 < n ? 2 * i + 2 : 2 * i + 1); };
    auto is_edge = [&](const ChunkSeg& c, int t0) { return t0 + kTokTile > c.first_masked; };

    if (warp < 4) {
        fewer_registers<L::kOtherRegs>();
        if ((warp & 1) == 0) {
            // ===================================== producers ====================================
            // (A copy takes a warp some 90 cycles to issue, one lane after the other: with pages of 16 tokens an operand is 16 of them.)
            const int op = warp >> 1;                               // K or V
            const CUtensorMap* map = op ? &map_v : &map_k;
            TileWalk<kChunkRows> walk(p, run, lane);
            uint32_t n = 0, base = 0, edges = 0;                    // tiles fetched, before this segment; EDGE parities, a bit per slot
            uint32_t recent[NS] = {};                               // the last operands
            while (walk.more && !fail_site) {
                const int pg = walk.page(), h = walk.cur.m.h, slot = walk.slot, hh = p.one_head ? 0 : h, at = lane << (p.box_shift + 7);
                if (E4M3) {
                    const uint32_t full = bar(L::RAWFULL + op);
                    if (!all_wait(L::RAWEMPTY + op, n ^ 1u, __LINE__)) break;
                    if (lane == 0) mbar_expect_tx(full, 16384);
                    __syncwarp();
                    if (lane < walk.boxes()) tma_load_4d(sbase + L::kRawAt + op * 16384u + at, map, full, 0, slot, hh, pg);
                    const int t8 = (lane & 15) * 8, ps = __shfl_sync(0xffffffffu, pg, t8 >> p.box_shift);
                    if (lane < 16) {
                        const uint8_t* src = (op ? p.c.vs : p.c.ks) + (ps < 0 ? 0ll : ps * p.c.ss_p + h * p.c.ss_h + walk.slot8);
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(sbase + L::kScales + op * 128u + t8), "l"(src), "r"(ps < 0 ? 0 : 8) : "memory");
                    }
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(full) : "memory");
                } else {
                    const int i = walk.tile - walk.cur.ta, t0 = walk.tile * kTokTile, len = walk.cur.m.len, masked = seen_by(p, walk.cur.m, 0);
                    const bool edge = op && t0 + kTokTile > masked;
                    const uint32_t k = op ? v_number(base, i, walk.cur.tb - walk.cur.ta) : k_number(base, i), st = k % NS, full = bar((edge ? L::EDGE : L::FULL) + st);
                    if (!all_wait(L::EMPTY + st, (k / NS) ^ 1u, __LINE__)) break;
#pragma unroll
                    for (int j = 0; j < NS; ++j) recent[j] = j + 1 < NS ? recent[j + 1] : k;
                    if (lane == 0) mbar_expect_tx(full, kOperandBytes);
                    __syncwarp();
                    if (lane < walk.boxes()) {
                        const uint32_t d = sbase + L::kRing + st * kOperandBytes + at;
                        tma_load_4d(d, map, full, 0, slot, hh, pg);
                        tma_load_4d(d + kHalfBytes, map, full, 64, slot, hh, pg);
                    }
                    // rows behind the list become zeros; so do rows that are not finite and that not every query sees, which are named to the softmax warps
                    if (edge) {
                        if (!all_wait(L::EDGE + st, edges >> st, __LINE__)) break;
                        edges ^= 1u << st;
                        uint8_t* tile = smem + L::kRing + st * kOperandBytes;
#pragma unroll 1
                        for (int j = 0; j < 4; ++j) {
                            const int row = j * 32 + lane, t = t0 + row;
                            bool odd = false;
                            if (t >= masked && t < len) {
#pragma unroll
                                for (int ch = 0; ch < 16; ++ch) {
                                    const uint4 u = *reinterpret_cast<const uint4*>(tile + (ch >> 3) * kHalfBytes + row * 128 + (((ch & 7) ^ (row & 7)) << 4));
                                    odd |= not_finite(u.x) || not_finite(u.y) || not_finite(u.z) || not_finite(u.w);
                                }
                            }
                            if (odd || t >= len) {
#pragma unroll
                                for (int ch = 0; ch < 16; ++ch)
                                    *reinterpret_cast<uint4*>(tile + (ch >> 3) * kHalfBytes + row * 128 + (((ch & 7) ^ (row & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
                            }
                            const uint32_t word = __ballot_sync(0xffffffffu, odd);
                            if (lane == 0) bad_words[st * 4 + j] = word;
                        }
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(L::FULL + st));
                    }
                }
                if (n++ == 0) walk.look_ahead();
                if (walk.tile + 1 == walk.cur.tb) base = n;
                walk.advance();
            }
            // no copy may be under way when the CTA leaves, and no commit's arrival: the last operand of every slot
            if (E4M3) {
                if (n > 0) (void)mbar_wait(bar(L::RAWFULL + op), (n - 1) & 1u);
            } else {
#pragma unroll
                for (int j = 0; j < NS; ++j)
                    if (j + n >= NS && recent[j] + NS >= 2 * n) {
                        (void)mbar_wait(bar(L::FULL + recent[j] % NS), (recent[j] / NS) & 1u);
                        if (!fail_site) (void)all_wait(L::EMPTY + recent[j] % NS, recent[j] / NS, __LINE__);
                    }
            }
        } else if (warp & 1) {
            // ===================================== MMA issuers ======================================
            // The whole warp walks the loop and one lane issues: slots and addresses are then uniform values, which the instruction takes as they
            // are (issued from a loop of one thread each MMA cost the moves of its descriptors, too).
            const int w = warp >> 1;
            const bool leader = elect_one();
            const uint32_t idesc_s = idesc_bf16(kTokTile);
            const uint32_t idesc_pv = idesc_bf16(kD) | (1u << 16);               // B operand (V) is MN-major
            const uint32_t aq = desc_lo_k(sbase + L::kQ + w * kOperandBytes), ap = desc_lo_k(sbase + L::kP + w * kOperandBytes), tS = tmem + w * 128u, tO = tmem + 256u + w * 128u;
            Segments<kChunkRows> seg(p, run);
            uint32_t slot = 0, phase = 0, ns = 0, np = 0, nq = 0;                // the operand's slot and round; S tiles begun, P and Q tiles taken
            auto next_op = [&]() { if (++slot == NS) { slot = 0; phase ^= 1u; } };
            while (seg.next()) {
                const ChunkSeg c = chunk_seg(p, seg);
                const int n = uniform(c.n), cnt = uniform(c.cnt(w));
                // S(i), or, past the tiles that this warpgroup sees, its word that K(i) may go
                auto step_s = [&](int i) -> bool {
                    if (!all_wait(L::FULL + slot, phase, __LINE__)) return false;
                    if (i < cnt) {
                        if (L::kPS && ns++ > 0 && !all_wait(L::SFREE + w, ns, __LINE__)) return false;
                        tc_fence_after();
                        if (leader) {
                            const uint32_t ak = desc_lo_k(sbase + L::kRing + slot * kOperandBytes);
#pragma unroll
                            for (int ks = 0; ks < 8; ++ks)
                                tc_mma(tS, desc_make(aq + desc_kstep(ks, kHalfBytes)), desc_make(ak + desc_kstep(ks, kHalfBytes)), idesc_s, ks > 0);
                            tc_commit(bar(L::SFULL + w));
                            tc_commit(bar(L::EMPTY + slot));
                        }
                    } else if (leader) {
                        tc_commit(bar(L::EMPTY + slot));
                    }
                    __syncwarp();
                    next_op();
                    return true;
                };
                if (cnt > 0 && !all_wait(L::QFULL + w, nq++, __LINE__)) break;
                if (!step_s(0)) break;
                for (int i = 0; i < n; ++i) {
                    if (L::kPS && i + 1 < n && !step_s(i + 1)) break;
                    if (!all_wait(L::FULL + slot, phase, __LINE__)) break;
                    if (i < cnt) {
                        const uint32_t av = desc_lo_mn(sbase + L::kRing + slot * kOperandBytes);
                        if (!all_wait(L::PFULL + w, np, __LINE__)) break;
                        tc_fence_after();
                        if (leader) {
#pragma unroll
                            for (int ks = 0; ks < 8; ++ks)               // steps of K = 16 tokens (2048 bytes of V each)
                                if constexpr (L::kPS) tc_mma(tO, desc_make(ap + desc_kstep(ks, kHalfBytes)), desc_make(av + ks * (2048 >> 4)), idesc_pv, 1u);
                                else tc_mma_ts(tO, tS + ks * 8, desc_make(av + ks * (2048 >> 4)), idesc_pv, 1u);
                        }
                        ++np;
                        if (leader) {
                            tc_commit(bar(L::EMPTY + slot));
                            if (L::kPS || i == cnt - 1) tc_commit(bar(L::ODONE + w));
                        }
                    } else if (leader) {
                        tc_commit(bar(L::EMPTY + slot));
                    }
                    __syncwarp();
                    next_op();
                    if (!L::kPS && i + 1 < n && !step_s(i + 1)) break;
                }
                if (fail_site) break;
            }
        }
    } else if (warp < 12) {
        // ======================================= softmax ========================================
        more_registers<L::kSoftRegs>();
        const int w = (warp - 4) >> 2, lane_grp = warp & 3, row = lane_grp * 32 + lane, r = w * 128 + row;
        const uint32_t lane_addr = (uint32_t)(lane_grp * 32) << 16;
        const uint32_t tS = tmem + lane_addr + w * 128u, tO = tmem + lane_addr + 256u + w * 128u;
        const float2 sl2v = make_float2(p.sl2, p.sl2);
        // Q of a segment: sixteen lanes per row; rows that are not there become zeros.  Asked for as soon as the segment before has its last logits.
        auto ask_q = [&](const Item& m) {
            const int tid = lane_grp * 32 + lane, piece = tid & 15;
            int head = 0, i = 0;
            row_place(p, m, w * 128 + (tid >> 4), head, i);         // eight rows further on: di queries and dg heads
            const int g0 = m.h * p.G, di = p.by_G.div(8), dg = 8 - di * p.G;
            int g = head - g0;
            const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q.ptr) + m.b * p.q.sb + head * p.q.sh + i * p.q.st + piece * 8;
            const long long step = di * p.q.st + dg * p.q.sh, wrap = p.q.st - p.G * p.q.sh;
            const uint32_t dst = sbase + L::kQ + w * kOperandBytes + (piece >> 3) * kHalfBytes;
#pragma unroll 4
            for (int rr = tid >> 4; rr < 128; rr += 8) {
                const bool there = w * 128 + rr < m.rows;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + rr * 128 + (((piece & 7) ^ (rr & 7)) << 4)),
                             "l"(there ? src : static_cast<const __nv_bfloat16*>(p.q.ptr)), "r"(there ? 16 : 0) : "memory");
                src += step; g += dg;
                if (g >= p.G) { g -= p.G; src += wrap; }
            }
        };
        auto q_there = [&]() {
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_async_smem();
            mbar_arrive(bar(L::QFULL + w));
        };
        Segments<kChunkRows> seg(p, run);
        uint32_t base = 0, ns = 0, no = 0, turns = 0;
        int4 info = make_int4(-1, 0, 0, 0);
        bool more = seg.next();
        if (more && chunk_seg(p, seg).cnt(w) > 0) { ask_q(seg.m); q_there(); }
        while (more && !fail_site) {
            const Item m = seg.m;
            const ChunkSeg c = chunk_seg(p, seg);
            const int cnt = c.cnt(w), both = min(c.cnt0, c.cnt1), seen = seen_by(p, m, r), ta = seg.ta;
            const bool whole = seg.whole(), there = r < m.rows;
            const size_t at = seg.slot() * kChunkRows + r;
            int head = 0, iq = 0;
            if (there) row_place(p, m, r, head, iq);
            __nv_bfloat16* const dst = static_cast<__nv_bfloat16*>(const_cast<void*>(p.o.ptr)) + m.b * p.o.sb + head * p.o.sh + iq * p.o.st;
            const int lse_at = (m.b * p.c.Hkv * p.G + head) * p.T + iq;
            info = seg.shared_item(run);
            more = seg.next();                                      // (looked up while the first logits are on their way)
            const bool next_q = more && chunk_seg(p, seg).cnt(w) > 0;
            float m_used = -INFINITY, l = 0.f;
            if (cnt > 0) {                                          // O starts at 0 (all of its MMAs accumulate)
                uint32_t z[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) z[j] = 0u;
#pragma unroll
                for (int q = 0; q < 4; ++q) tc_st32(tO + q * 32, z);
                tc_wait_st();                                       // (ordered before the MMAs by the first P's barrier)
            }
            for (int i = 0; i < cnt; ++i) {
                const int t0 = (ta + i) * kTokTile;
                const bool edge = is_edge(c, t0);
                {
                    if (!all_wait(L::SFULL + w, ns, __LINE__)) break;
                    ++ns;
                    tc_fence_after();
                    uint32_t s[128];
#pragma unroll
                    for (int q = 0; q < 4; ++q) tc_ld32(tS + q * 32, s + q * 32);
                    tc_wait_ld32(s);
#pragma unroll
                    for (int q = 1; q < 4; ++q) tc_wait_ld32(s + q * 32);
                    if (L::kPS) {                                   // S is read: the next one may be formed
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bar(L::SFREE + w));
                    }
                    const int nvis = seen - t0;                     // columns j < nvis are seen
                    if (edge && __any_sync(0xffffffffu, nvis < kTokTile)) {
#pragma unroll
                        for (int j = 0; j < 128; ++j) if (j >= nvis) s[j] = 0xff800000u;
                    }
                    float t4[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        t4[q] = fmaxf(__uint_as_float(s[q]), __uint_as_float(s[q + 4]));
#pragma unroll
                        for (int j = 8; j < 128; j += 8) t4[q] = fmax3(t4[q], __uint_as_float(s[j + q]), __uint_as_float(s[j + q + 4]));
                    }
                    const float mt = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])) * p.sl2;
                    // The two warps of an SM sub-partition take turns at the exponentials, one per warpgroup: left alone they run side by side, and then
                    // wait side by side for their MMAs.  (Warpgroup 0 begins; its turn k follows turn k - 1 of warpgroup 1.)
                    if (i < both) {
                        if ((w == 1 || turns > 0) && !all_wait(L::TURN + 4 * w + lane_grp, w ? turns : turns - 1u, __LINE__)) break;
                        ++turns;
                    }
                    if (L::kPS && no > 0) {                         // P V of the tile before
                        if (!all_wait(L::ODONE + w, no - 1u, __LINE__)) break;
                        tc_fence_after();
                    }
                    if (L::kPS) ++no;
                    const bool need = mt > m_used + 8.f;            // also true for the first tile that is seen
                    if (__any_sync(0xffffffffu, need)) {
                        const float factor = need ? fast_exp2(m_used - mt) : 1.f;
                        if (__any_sync(0xffffffffu, need && m_used != -INFINITY)) {
                            // P V of this warpgroup's previous tile is complete (waited for above, or covered by the commit that signalled S)
#pragma unroll 1
                            for (int q = 0; q < 8; ++q) {
                                uint32_t ov[16];
                                tc_ld16(tO + q * 16, ov);
                                asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(ov[0]), "+r"(ov[1]), "+r"(ov[2]), "+r"(ov[3]), "+r"(ov[4]), "+r"(ov[5]), "+r"(ov[6]), "+r"(ov[7]),
                                             "+r"(ov[8]), "+r"(ov[9]), "+r"(ov[10]), "+r"(ov[11]), "+r"(ov[12]), "+r"(ov[13]), "+r"(ov[14]), "+r"(ov[15]) :: "memory");
#pragma unroll
                                for (int j = 0; j < 16; ++j) ov[j] = __float_as_uint(__uint_as_float(ov[j]) * factor);
                                tc_st16(tO + q * 16, ov);
                            }
                        }
                        l *= factor;
                        if (need) m_used = mt;
                    }
                    const float m_eff = reference(m_used);
                    const float2 negm = make_float2(-m_eff, -m_eff);
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t pk[16];
                        if (q == L::kTurn && i < both && lane == 0) mbar_arrive(bar(L::TURN + 4 * (w ^ 1) + lane_grp));
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            float2 x = make_float2(__uint_as_float(s[q * 32 + j]), __uint_as_float(s[q * 32 + j + 1]));
                            x = __ffma2_rn(x, sl2v, negm);
                            const float2 ex = make_float2(fast_exp2(x.x), fast_exp2(x.y));
                            sum[(j >> 1) & 1] = __fadd2_rn(sum[(j >> 1) & 1], ex);
                            pk[j >> 1] = pack_bf16x2(ex.x, ex.y);
                        }
                        if constexpr (L::kPS) {
                            uint8_t* d = smem + L::kP + w * kOperandBytes + (q >> 1) * kHalfBytes + row * 128;
#pragma unroll
                            for (int x = 0; x < 4; ++x)
                                *reinterpret_cast<uint4*>(d + ((((q & 1) * 4 + x) ^ (row & 7)) << 4)) = make_uint4(pk[4 * x], pk[4 * x + 1], pk[4 * x + 2], pk[4 * x + 3]);
                        } else {
                            tc_st16(tS + q * 16, pk);
                        }
                    }
                    if (L::kTurn == 4 && i < both && lane == 0) mbar_arrive(bar(L::TURN + 4 * (w ^ 1) + lane_grp));
                    l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                    tc_wait_st();
                    if (edge) {                                     // rows of V that are added by hand
                        const uint32_t vop = v_number(base, i, c.n), vs = vop % NS;
                        if (!all_wait(L::FULL + vs, vop / NS, __LINE__)) break;
#pragma unroll 1
                        for (int b = 0; b < 4; ++b) {
                            uint32_t word = bad_words[vs * 4 + b];
                            while (word) {
                                const int j = b * 32 + __ffs(word) - 1;
                                word &= word - 1;
                                float wt;
                                if constexpr (L::kPS) {
                                    wt = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(smem + L::kP + w * kOperandBytes + (j >> 6) * kHalfBytes + row * 128 + ((((j >> 3) & 7) ^ (row & 7)) << 4) + (j & 7) * 2));
                                } else {
                                    uint32_t two;
                                    tc_ld1(tS + (j >> 1), two);
                                    wt = __uint_as_float(j & 1 ? two & 0xffff0000u : two << 16);
                                }
                                const int t = t0 + j, page = p.c.page_of(m.b, m.h, t), at_slot = p.c.by_P.mod(t);
                                const long long at_row = page * p.c.v.sb + m.h * p.c.v.sh + at_slot * p.c.v.st;
                                float sv = 1.f;
                                if (E4M3) sv = scale_of(p.c.vs[page * p.c.ss_p + m.h * p.c.ss_h + at_slot]);
#pragma unroll 1
                                for (int q = 0; q < 8; ++q) {
                                    uint32_t ov[16];
                                    tc_ld16(tO + q * 16, ov);
                                    asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(ov[0]), "+r"(ov[1]), "+r"(ov[2]), "+r"(ov[3]), "+r"(ov[4]), "+r"(ov[5]), "+r"(ov[6]), "+r"(ov[7]),
                                                 "+r"(ov[8]), "+r"(ov[9]), "+r"(ov[10]), "+r"(ov[11]), "+r"(ov[12]), "+r"(ov[13]), "+r"(ov[14]), "+r"(ov[15]) :: "memory");
#pragma unroll
                                    for (int x = 0; x < 16; ++x) {
                                        float v;
                                        if constexpr (E4M3) {
                                            uint32_t two, none;
                                            expand_adjacent(static_cast<const uint8_t*>(p.c.v.ptr)[at_row + q * 16 + x], two, none);
                                            v = __low2float(*reinterpret_cast<const __half2*>(&two)) * sv;
                                        } else {
                                            v = __bfloat162float(static_cast<const __nv_bfloat16*>(p.c.v.ptr)[at_row + q * 16 + x]);
                                        }
                                        if (j < nvis) ov[x] = __float_as_uint(fmaf(wt, v, __uint_as_float(ov[x])));
                                    }
                                    tc_st16(tO + q * 16, ov);
                                }
                                tc_wait_st();
                            }
                        }
                    }
                    if (L::kPS) fence_async_smem();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(L::PFULL + w));

                }
            }
            base += c.n;
            if (fail_site) break;
            if (next_q) ask_q(seg.m);
            // ---- the segment's result ----
            if (cnt > 0) {
                if (!all_wait(L::ODONE + w, L::kPS ? no - 1u : no, __LINE__)) break;
                if (!L::kPS) ++no;
                tc_fence_after();
            }
            const float k = whole ? (l != 0.f ? 1.f / l : 0.f) : 1.f;
            if (cnt > 0 || whole) {
#pragma unroll 1
                for (int q = 0; q < 4; ++q) {
                    uint32_t ov[32];
                    if (cnt > 0) {
                        tc_ld32(tO + q * 32, ov);
                        tc_wait_ld32(ov);
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) ov[j] = 0u;
                    }
                    if (!there) continue;
#pragma unroll
                    for (int j = 0; j < 32; ++j) ov[j] = __float_as_uint(__uint_as_float(ov[j]) * k);
                    if (whole) {
#pragma unroll
                        for (int j = 0; j < 32; j += 16) {
                            uint32_t h[8];
#pragma unroll
                            for (int x = 0; x < 8; ++x) h[x] = pack_bf16x2(__uint_as_float(ov[j + 2 * x]), __uint_as_float(ov[j + 2 * x + 1]));
                            if (p.o_aligned) {
                                store32(dst + q * 32 + j, h[0], h[1], h[2], h[3], h[4], h[5], h[6], h[7]);
                            } else {
                                *reinterpret_cast<uint4*>(dst + q * 32 + j) = make_uint4(h[0], h[1], h[2], h[3]);
                                *reinterpret_cast<uint4*>(dst + q * 32 + j + 8) = make_uint4(h[4], h[5], h[6], h[7]);
                            }
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; j += 8)
                            store32(p.part_o + at * kD + q * 32 + j, ov[j], ov[j + 1], ov[j + 2], ov[j + 3], ov[j + 4], ov[j + 5], ov[j + 6], ov[j + 7]);
                    }
                }
            }
            if (there && whole && p.lse) p.lse[lse_at] = lse_of(reference(m_used), l);
            if (there && !whole) { p.part_m[at] = m_used; p.part_l[at] = l; }
            tc_fence_before();                                      // (O is read: the next segment's MMAs follow the next P's barrier)
            if (next_q) q_there();
        }
        if (threadIdx.x == 128) p.info[blockIdx.x] = info;
    } else {
        // ======================= 8-bit codes -> bf16 tiles, the row's scale multiplied in =======================
        fewer_registers<L::kOtherRegs>();
        const int row = threadIdx.x - 384, sw = row & 7;
        Segments<kChunkRows> seg(p, run);
        uint32_t n = 0;
        while (!fail_site && seg.next()) {
            const ChunkSeg c = chunk_seg(p, seg);
            for (int i = 0; i < c.n && !fail_site; ++i) {
                const int t = (seg.ta + i) * kTokTile + row;
                for (int op = 0; op < 2; ++op, ++n) {
                    const uint32_t st = n & 1, slot = n % NS;
                    if (!all_wait(L::RAWFULL + st, n >> 1, __LINE__)) break;
                    const uint32_t raw = sbase + L::kRawAt + st * 16384u + row * 128 + (sw << 4);      // (a row begins on a 128-byte boundary: its pieces' places differ by exclusive or)
                    uint4 x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = lds16(raw ^ (j << 4));
                    uint32_t s = smem[L::kScales + st * 128u + row];
                    // (the loads above may still be under way, and nothing below uses them soon: without the fence the bulk copy that the
                    // arrival lets go has been seen to overtake them)
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(L::RAWEMPTY + st));
                    // rows of V that not every query sees and that hold NaN become zeros here and are added by hand; so do rows behind the list's end
                    bool odd = false;
                    if (op && is_edge(c, (seg.ta + i) * kTokTile)) {
                        uint32_t codes = s == 255u ? 1u : 0u;
#pragma unroll
                        for (int j = 0; j < 8; ++j) codes |= nan_codes(x[j].x) | nan_codes(x[j].y) | nan_codes(x[j].z) | nan_codes(x[j].w);
                        odd = codes != 0u && t >= c.first_masked && t < seg.m.len;
                        if (odd || t >= seg.m.len) {
                            s = 0;
#pragma unroll
                            for (int j = 0; j < 8; ++j) x[j] = make_uint4(0u, 0u, 0u, 0u);
                        }
                    }
                    const __nv_bfloat16 f = __float2bfloat16(scale_of(s));
                    const __nv_bfloat162 m = __halves2bfloat162(f, f);
                    if (!all_wait(L::EMPTY + slot, (n / NS) ^ 1u, __LINE__)) break;
                    const uint32_t dst = sbase + L::kRing + slot * kOperandBytes + row * 128 + (sw << 4);
#pragma unroll
                    for (int j = 0; j < 16; ++j) {                  // 8 channels at a time
                        uint4 y;
                        codes_to_bf16(j & 1 ? x[j >> 1].z : x[j >> 1].x, m, y.x, y.y);
                        codes_to_bf16(j & 1 ? x[j >> 1].w : x[j >> 1].y, m, y.z, y.w);
                        sts16((dst ^ ((j & 7) << 4)) + (j >> 3) * kHalfBytes, y);
                    }
                    const uint32_t word = __ballot_sync(0xffffffffu, odd);
                    if (op && lane == 0) bad_words[slot * 4 + (warp - 12)] = word;
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(L::FULL + slot));
                }
            }
        }
        for (uint32_t k = n > NS ? n - NS : 0u; k < n && !fail_site; ++k) (void)all_wait(L::EMPTY + k % NS, k / NS, __LINE__);      // (no commit's arrival may be under way when the CTA leaves)
    }
    if (fail_site) atomicCAS(p.status, 0u, (unsigned)fail_site);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

}  // namespace
}  // namespace obc
