// Attention of new tokens over a paged cache (obc_paged_attention): o = softmax(scale q K^T) V with the causal mask of a chunk at the
// list's end, by one pass over the list with running maxima and sums.
//
//   few_rows_kernel      up to 16 rows per KV list (single tokens of a GQA group): warp-level MMAs (paged_few.cuh)
//   chunk_kernel         more rows: tcgen05 MMAs (paged_chunk.cuh)
//   paged_f32_kernel     fp32 caches on CUDA cores
//   paged_merge_kernel   joins the partial results of items that several CTAs shared
// How the work is shared out: paged_common.cuh.
#include "paged_chunk.cuh"
#include "paged_few.cuh"

#include <math.h>

namespace obc {
namespace {

// ---- merge ------------------------------------------------------------------------------------------
// One warp per row of an item that was shared: o = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s over the CTAs' slots, in
// their order.  A block takes eight rows of the item that begins in CTA blockIdx.x / (blocks per item).
template <typename OT, int ROWS>
__global__ void __launch_bounds__(256)
paged_merge_kernel(const __grid_constant__ AttnParams p) {
    constexpr int kBlocks = ROWS / 8;
    pdl_wait();
    const int cta = blockIdx.x / kBlocks, lane = threadIdx.x & 31;
    const int4 f = p.info[cta];
    if (f.x < 0) return;
    const Item m = item_of<ROWS>(p, f.x);
    const int n = f.y - cta + 1;
    const int r = (blockIdx.x % kBlocks) * 8 + (threadIdx.x >> 5);
    if (r >= m.rows) return;
    auto at = [&](int s) { return (2 * (size_t)(cta + s) + (s == 0 ? f.z : 0)) * ROWS + r; };
    float top = -INFINITY;
    for (int s = lane; s < n; s += 32) top = fmaxf(top, p.part_m[at(s)]);
    top = warp_max(top);
    const float ref = reference(top);
    float total = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < n; s0 += 32) {
        const int s = s0 + lane, cnt = min(32, n - s0);
        const float w = s < n ? share_of(p.part_m[at(s)], ref) : 0.f;
        if (s < n) total = fmaf(w, p.part_l[at(s)], total);
#pragma unroll 8
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
    int4 info = make_int4(-1, 0, 0, 0);
    while (seg.next()) {
        const Item m = seg.m;
        info = seg.shared_item(run);
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
                const int page = t < m.len ? p.c.page_of(m.b, m.h, t) : -1, slot = p.c.by_P.mod(t);
                if (page >= 0) {
                    kx[u] = load4(static_cast<const float*>(p.c.k.ptr) + page * p.c.k.sb + m.h * p.c.k.sh + slot * p.c.k.st + lane * 4);
                    vx[u] = load4(static_cast<const float*>(p.c.v.ptr) + page * p.c.v.sb + m.h * p.c.v.sh + slot * p.c.v.st + lane * 4);
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
                    const float ref = reference(top), f = share_of(mx[j], ref);
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
            const float total = warp_sum(l[j]), ref = reference(mx[j]);
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
    }
    if (tid == 0) p.info[blockIdx.x] = info;
}

// ---- host side --------------------------------------------------------------------------------------
struct AttnPlan { int rows, grid, nrt, items; size_t off_info, off_m, off_l, off_o, bytes; };

AttnPlan make_plan(const PagesView& c, const AttnShape& s) {
    AttnPlan p{};
    const long long rows = (long long)s.G * s.T;
    p.rows = c.dtype == OBC_F32 ? kF32Rows : rows <= 8 ? 8 : rows <= 16 ? 16 : kChunkRows;
    p.grid = sm_count() * (c.dtype == OBC_F32 || p.rows == 8 ? 2 : 1);
    p.nrt = (int)((rows + p.rows - 1) / p.rows);
    p.items = c.B * c.Hkv * p.nrt;
    size_t off = 256;                                  // header: the status word
    p.off_info = off; off = align_up(off + (size_t)p.grid * sizeof(int4), 256);
    const size_t slots = 2 * (size_t)p.grid * p.rows;
    p.off_m = off; off = align_up(off + slots * 4, 256);
    p.off_l = off; off = align_up(off + slots * 4, 256);
    p.off_o = off; off = align_up(off + slots * kD * 4, 256);
    p.bytes = off;
    return p;
}

}  // namespace

bool paged_attention_fits(const PagesView& c, const AttnShape& s) {
    const AttnPlan p = make_plan(c, s);
    return (long long)p.items * (c.max_len / kTokTile + 1 + kSegCost) <= 0x7fffffffLL;
}

size_t paged_attention_bytes(const PagesView& c, const AttnShape& s) { return make_plan(c, s).bytes; }

obc_status launch_paged_attention(const PagesView& c, const AttnShape& s, TensorView q, TensorView o, float* lse, void* ws, cudaStream_t stream) {
    const AttnPlan plan = make_plan(c, s);
    char* w = static_cast<char*>(ws);
    AttnParams p{};
    p.c = c; p.G = s.G; p.T = s.T; p.causal = s.causal; p.q_lens = s.q_lens; p.sl2 = s.scale * kLog2e;
    p.q = q; p.o = o; p.lse = lse;
    p.o_aligned = ((uintptr_t)o.ptr & 31) == 0 && o.sb % 16 == 0 && o.sh % 16 == 0 && o.st % 16 == 0;      // (elements of 2 bytes)
    p.nrt = plan.nrt; p.items = plan.items;
    p.one_head = c.k.sh == 0 && c.v.sh == 0 ? 1 : 0;
    const int tile = c.dtype == OBC_BF16 && plan.rows == 8 ? FewLayout<1, false>::kTile : kTokTile;
    p.box = 8; p.box_shift = 3;
    while (p.box < tile && c.P % (2 * p.box) == 0) { p.box *= 2; ++p.box_shift; }
    p.by_G = FastDiv(s.G); p.by_nrt = FastDiv(plan.nrt);
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
        const bool whole_rows = plan.rows != kChunkRows;
        if (!make_page_map(&mk, c, c.k, p.box, whole_rows) || !make_page_map(&mv, c, c.v, p.box, whole_rows)) return OBC_ERR_CUDA;
        auto few = [&](auto kernel, auto layout) {
            using L = decltype(layout);
            const cudaError_t a = allow_smem(kernel, L::kSmem);
            if (a != cudaSuccess) return a;
            ProfScope prof("paged_attention_few", stream);
            return launch_pdl(kernel, dim3(plan.grid), dim3(L::kThreads), L::kSmem, stream, 1, mk, mv, p);
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
            e = plan.rows == 8 ? few(few_rows_kernel<1, true>, FewLayout<1, true>()) : few(few_rows_kernel<2, true>, FewLayout<2, true>());
        else
            e = plan.rows == 8 ? few(few_rows_kernel<1, false>, FewLayout<1, false>()) : few(few_rows_kernel<2, false>, FewLayout<2, false>());
    }
    OBC_CUDA_TRY(e);
    auto merge = [&](auto kernel, int blocks) {
        ProfScope prof("paged_attention_merge", stream);
        return launch_pdl(kernel, dim3((unsigned)(plan.grid * blocks)), dim3(256), 0, stream, 1, p);
    };
    OBC_CUDA_TRY(c.dtype == OBC_F32 ? merge(paged_merge_kernel<float, kF32Rows>, kF32Rows / 8)
                 : plan.rows == 8   ? merge(paged_merge_kernel<__nv_bfloat16, 8>, 8 / 8)
                 : plan.rows == 16  ? merge(paged_merge_kernel<__nv_bfloat16, 16>, 16 / 8)
                                    : merge(paged_merge_kernel<__nv_bfloat16, kChunkRows>, kChunkRows / 8));
    return OBC_OK;
}

}  // namespace obc
