// Rows into and out of a paged cache: obc_paged_write (quantising on the way) and obc_paged_read.
//
// Every row is read once and written once.  Eight lanes take one row of K and of V, 16 channels each, so that the addresses (64-bit strides,
// page numbers) and the row's maximum, which the scale of an 8-bit row needs, are worked out four times per warp; with 16 lanes and
// 8 channels each these instructions were what set the pace (four prompts of up to 8191 tokens, 8 heads, into 8 bits: 48 us, now 27).
#include "obc_common.cuh"
#include <cuda_fp8.h>

namespace obc {
namespace {

constexpr int kLanes = 8;                         // lanes per row
constexpr int kCh = kD / kLanes;                  // channels per lane
constexpr int kBlock = 256;
constexpr int kSpan = kBlock / kLanes;            // rows that a block takes at a time

// ---- 16 channels of a row in registers ----------------------------------------------------------
struct Floats { float x[kCh]; };

template <typename T> struct Chunk;
template <> struct Chunk<float> {
    float4 w[kCh / 4];
    __device__ __forceinline__ void load(const float* p) {
#pragma unroll
        for (int i = 0; i < kCh / 4; ++i) w[i] = reinterpret_cast<const float4*>(p)[i];
    }
    __device__ __forceinline__ Floats values() const {
        Floats r;
#pragma unroll
        for (int i = 0; i < kCh / 4; ++i) { r.x[4 * i] = w[i].x; r.x[4 * i + 1] = w[i].y; r.x[4 * i + 2] = w[i].z; r.x[4 * i + 3] = w[i].w; }
        return r;
    }
    // The largest |x| as the upper half of its bits, rounded up: that keeps what the row's scale goes by, namely its exponent and whether its
    // mantissa is above 1.75.  As whole numbers infinity and NaN are above all others.
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
        const Floats f = values();
#pragma unroll
        for (int i = 0; i < kCh; ++i) m = max(m, __float_as_uint(f.x[i]) & 0x7fffffffu);
        return m >= 0x7f800000u ? m >> 16 : min((m + 0xffffu) >> 16, 0x7f7fu);
    }
};
template <> struct Chunk<__nv_bfloat16> {
    uint4 w[kCh / 8];
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
#pragma unroll
        for (int i = 0; i < kCh / 8; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ Floats values() const {
        Floats r;
#pragma unroll
        for (int i = 0; i < kCh / 8; ++i) {
            const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) { r.x[8 * i + 2 * j] = __uint_as_float(u[j] << 16); r.x[8 * i + 2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u); }
        }
        return r;
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kCh / 8; ++i) {
            const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) m = __vmaxu2(m, u[j] & 0x7fff7fffu);
        }
        return max(m & 0xffffu, m >> 16);
    }
};
__device__ __forceinline__ void store(float* p, const Floats& r) {
#pragma unroll
    for (int i = 0; i < kCh / 4; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(r.x[4 * i], r.x[4 * i + 1], r.x[4 * i + 2], r.x[4 * i + 3]);
}
__device__ __forceinline__ void store(__nv_bfloat16* p, const Floats& r) {
#pragma unroll
    for (int i = 0; i < kCh / 8; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(r.x[8 * i + 2 * j], r.x[8 * i + 2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t*>(&h);
        }
        reinterpret_cast<uint4*>(p)[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// ---- 8 bits -------------------------------------------------------------------------------------
// Biased exponent of a row's scale from the upper half of the largest |x|: 448 = 1.75 * 2^8, so the exponent of the maximum less 8, one
// more if its mantissa is above 1.75.  Infinity or NaN: 255.
__device__ __forceinline__ int scale_exponent(uint32_t top) {
    const int e = (int)(top >> 7);
    return e == 255 ? 255 : max(e - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0), 1);
}
// codes of 16 channels.  x / 2^(s - 127) is exact: the quotient's exponent stays within fp32's range.
__device__ __forceinline__ uint4 e4m3_codes(const Floats& r, int s) {
    if (s == 255) return make_uint4(0u, 0u, 0u, 0u);
    const float inv = __uint_as_float((uint32_t)(254 - s) << 23);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(r.x[4 * i] * inv, r.x[4 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(r.x[4 * i + 2] * inv, r.x[4 * i + 3] * inv), __NV_SATFINITE, __NV_E4M3);
        w[i] = lo | hi << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ Floats e4m3_values(uint4 c, int s) {
    const float scale = s == 255 ? __uint_as_float(0x7fc00000u) : s == 0 ? __uint_as_float(0x00400000u) : __uint_as_float((uint32_t)s << 23);
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
    Floats r;
#pragma unroll
    for (int i = 0; i < kCh / 2; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1)) & 0xffffu), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        r.x[2 * i] = f.x * scale; r.x[2 * i + 1] = f.y * scale;
    }
    return r;
}

// ---- rows of pages ------------------------------------------------------------------------------
// the 16 channels of page row (page, h, slot) that a lane holds, as they lie there (8-bit rows are expanded when all have been asked for)
template <int DT> struct PageRow {
    Chunk<typename std::conditional<DT == OBC_F32, float, __nv_bfloat16>::type> c;
    __device__ __forceinline__ Floats values() const { return c.values(); }
};
template <> struct PageRow<OBC_E4M3> {
    uint4 codes; int s;
    __device__ __forceinline__ Floats values() const { return e4m3_values(codes, s); }
};
template <int DT>
__device__ __forceinline__ PageRow<DT> page_row(const PagesView& c, const TensorView& t, const uint8_t* scale, int page, int h, int slot, int lane) {
    const long long at = page * t.sb + h * t.sh + slot * t.st + lane * kCh;
    PageRow<DT> r;
    if constexpr (DT == OBC_E4M3) {
        r.codes = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(t.ptr) + at);
        r.s = scale[page * c.ss_p + h * c.ss_h + slot];
    } else if constexpr (DT == OBC_BF16) {
        r.c.load(static_cast<const __nv_bfloat16*>(t.ptr) + at);
    } else {
        r.c.load(static_cast<const float*>(t.ptr) + at);
    }
    return r;
}
template <int DT>
__device__ __forceinline__ void put_page_row(const PagesView& c, const TensorView& t, uint8_t* scale, int page, int h, int slot, int lane, const Floats& r, uint32_t top) {
    const long long at = page * t.sb + h * t.sh + slot * t.st + lane * kCh;
    if constexpr (DT == OBC_E4M3) {
        const int s = scale_exponent(top);
        *reinterpret_cast<uint4*>(static_cast<uint8_t*>(const_cast<void*>(t.ptr)) + at) = e4m3_codes(r, s);
        if (lane == 0) scale[page * c.ss_p + h * c.ss_h + slot] = (uint8_t)s;
    } else if constexpr (DT == OBC_BF16) {
        store(static_cast<__nv_bfloat16*>(const_cast<void*>(t.ptr)) + at, r);
    } else {
        store(static_cast<float*>(const_cast<void*>(t.ptr)) + at, r);
    }
}

// Both kernels take the rows of all lists, one after the other.
template <typename S, int DT>
__global__ void __launch_bounds__(kBlock, 6)
paged_write_kernel(const __grid_constant__ PagesView c, const __grid_constant__ PagedWrite w, const __grid_constant__ TensorView k,
                   const __grid_constant__ TensorView v, int total) {
    pdl_wait();
    const int lane = threadIdx.x % kLanes, f = blockIdx.x * kSpan + threadIdx.x / kLanes;
    int page = -1, slot = 0, h = 0;
    Chunk<S> rk{}, rv{};
    if (f < total) {
        const int unit = w.by_rows.div(f), j = f - unit * w.rows, b = c.by_H.div(unit);
        h = unit - b * c.Hkv;
        const int n = w.new_lens ? min(max(w.new_lens[b * w.nb + h * w.nh], 0), w.rows) : w.rows;
        const int pos = c.len(b, h) - n + j, src = w.idx ? w.idx[f] : j;
        if (j < n && pos >= 0 && (unsigned)src < (unsigned)w.src_tokens) {
            // (the row is asked for before the page number is waited for)
            rk.load(static_cast<const S*>(k.ptr) + b * k.sb + h * k.sh + src * k.st + lane * kCh);
            rv.load(static_cast<const S*>(v.ptr) + b * v.sb + h * v.sh + src * v.st + lane * kCh);
            page = c.page_of(b, h, pos);
            slot = c.by_P.mod(pos);
        }
    }
    uint32_t top = 0;                                  // K's largest in the lower half, V's in the upper
    if (DT == OBC_E4M3) {                              // (every lane of the warp takes part)
        top = rk.top() | rv.top() << 16;
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    if (page < 0) return;
    put_page_row<DT>(c, c.k, c.ks, page, h, slot, lane, rk.values(), top & 0xffffu);
    put_page_row<DT>(c, c.v, c.vs, page, h, slot, lane, rv.values(), top >> 16);
}

template <typename D, int DT>
__global__ void __launch_bounds__(kBlock, 4)
paged_read_kernel(const __grid_constant__ PagesView c, int n_tokens, FastDiv by_tokens, const __grid_constant__ TensorView k, const __grid_constant__ TensorView v,
                  int zero_rows, int total) {
    pdl_wait();
    const int lane = threadIdx.x % kLanes, f = blockIdx.x * kSpan + threadIdx.x / kLanes;
    if (f >= total) return;
    const int unit = by_tokens.div(f), t = f - unit * n_tokens, b = c.by_H.div(unit), h = unit - b * c.Hkv;
    PageRow<DT> rk{}, rv{};
    if (t < c.len(b, h)) {
        const int page = c.page_of(b, h, t), slot = c.by_P.mod(t);
        if (page >= 0) {
            rk = page_row<DT>(c, c.k, c.ks, page, h, slot, lane);
            rv = page_row<DT>(c, c.v, c.vs, page, h, slot, lane);
        }
    } else if (!zero_rows) {
        return;
    }
    store(static_cast<D*>(const_cast<void*>(k.ptr)) + b * k.sb + h * k.sh + t * k.st + lane * kCh, rk.values());
    store(static_cast<D*>(const_cast<void*>(v.ptr)) + b * v.sb + h * v.sh + t * v.st + lane * kCh, rv.values());
}

}  // namespace

obc_status launch_paged_write(const PagesView& c, const PagedWrite& w, TensorView k, TensorView v, cudaStream_t stream) {
    const long long total = (long long)c.B * c.Hkv * w.rows, blocks = (total + kSpan - 1) / kSpan;
    if (total > 0x7fffffffLL - kSpan) return OBC_ERR_SHAPE;
    auto go = [&](auto kernel) {
        ProfScope prof("paged_write", stream);
        return launch_pdl(kernel, dim3((unsigned)blocks), dim3(kBlock), 0, stream, 1, c, w, k, v, (int)total);
    };
    auto by_pages = [&](auto src) {
        using S = decltype(src);
        return c.dtype == OBC_E4M3 ? go(paged_write_kernel<S, OBC_E4M3>) : c.dtype == OBC_BF16 ? go(paged_write_kernel<S, OBC_BF16>)
                                                                                               : go(paged_write_kernel<S, OBC_F32>);
    };
    OBC_CUDA_TRY(w.src_dtype == OBC_BF16 ? by_pages(__nv_bfloat16()) : by_pages(float()));
    return OBC_OK;
}

obc_status launch_paged_read(const PagesView& c, int n_tokens, int out_dtype, TensorView k, TensorView v, bool zero_rows, cudaStream_t stream) {
    const long long total = (long long)c.B * c.Hkv * n_tokens, blocks = (total + kSpan - 1) / kSpan;
    if (total > 0x7fffffffLL - kSpan) return OBC_ERR_SHAPE;
    auto go = [&](auto kernel) {
        ProfScope prof("paged_read", stream);
        return launch_pdl(kernel, dim3((unsigned)blocks), dim3(kBlock), 0, stream, 1, c, n_tokens, FastDiv(n_tokens), k, v, (int)zero_rows, (int)total);
    };
    auto by_pages = [&](auto dst) {
        using D = decltype(dst);
        return c.dtype == OBC_E4M3 ? go(paged_read_kernel<D, OBC_E4M3>) : c.dtype == OBC_BF16 ? go(paged_read_kernel<D, OBC_BF16>)
                                                                                              : go(paged_read_kernel<D, OBC_F32>);
    };
    OBC_CUDA_TRY(out_dtype == OBC_BF16 ? by_pages(__nv_bfloat16()) : by_pages(float()));
    return OBC_OK;
}

}  // namespace obc
