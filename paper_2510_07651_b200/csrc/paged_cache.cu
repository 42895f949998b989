// Rows into and out of a paged cache: obc_paged_write (quantising on the way) and obc_paged_read.
//
// Both are bound by HBM traffic: every row is read once and written once.  Sixteen lanes take one row of K and of V, 8 channels each:
// the row's maximum, which the scale of an 8-bit row needs, is four shuffles away and a row is one full 128- to 512-byte access
// either way.  The page number (a dependent load) is asked for together with the source row, not before it.
#include "obc_common.cuh"
#include <cuda_fp8.h>

namespace obc {
namespace {

constexpr int kLanes = 16;                        // lanes per row
constexpr int kBlock = 256;
constexpr int kRows = 2;                          // rows of K and V per thread: four 16-byte loads in flight
constexpr int kRowsPerBlock = kBlock / kLanes * kRows;

struct Row8 { float x[8]; };

template <typename T> __device__ __forceinline__ Row8 load8(const T* p);
template <> __device__ __forceinline__ Row8 load8<float>(const float* p) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    return Row8{{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
}
template <> __device__ __forceinline__ Row8 load8<__nv_bfloat16>(const __nv_bfloat16* p) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    Row8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) { r.x[2 * i] = __uint_as_float(w[i] << 16); r.x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    return r;
}
__device__ __forceinline__ void store8(float* p, const Row8& r) {
    reinterpret_cast<float4*>(p)[0] = make_float4(r.x[0], r.x[1], r.x[2], r.x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(r.x[4], r.x[5], r.x[6], r.x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const Row8& r) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(r.x[2 * i], r.x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Biased exponent of a row's scale from the largest |x| of the row: 448 = 1.75 * 2^8, so the exponent of the maximum less 8, one
// more if its mantissa is above 1.75.  Infinity or NaN: 255.
__device__ __forceinline__ int scale_exponent(float amax) {
    const uint32_t bits = __float_as_uint(amax);
    const int e = (int)(bits >> 23);
    return e == 255 ? 255 : max(e - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), 1);
}
// (fmaxf drops NaN: a NaN counts as infinity here, which is all the row's scale asks)
__device__ __forceinline__ float row_amax(const Row8& r) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, r.x[i] != r.x[i] ? INFINITY : fabsf(r.x[i]));
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    return m;
}
// codes of 8 channels.  x / 2^(s - 127) is exact: the quotient's exponent stays within fp32's range.
__device__ __forceinline__ uint2 e4m3_codes(const Row8& r, int s) {
    if (s == 255) return make_uint2(0u, 0u);
    const float inv = __uint_as_float((uint32_t)(254 - s) << 23);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = __nv_cvt_float2_to_fp8x2(make_float2(r.x[2 * i] * inv, r.x[2 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
    return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}
__device__ __forceinline__ Row8 e4m3_values(uint2 c, int s) {
    const float scale = s == 255 ? __uint_as_float(0x7fc00000u) : s == 0 ? __uint_as_float(0x00400000u) : __uint_as_float((uint32_t)s << 23);
    Row8 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = (i < 2 ? c.x : c.y) >> (16 * (i & 1)) & 0xffffu;
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        r.x[2 * i] = f.x * scale; r.x[2 * i + 1] = f.y * scale;
    }
    return r;
}

// the 8 channels of page row (page, h, slot) that a lane holds, as values
template <int DT>
__device__ __forceinline__ Row8 page_row(const PagesView& c, const TensorView& t, const uint8_t* scale, int page, int h, int slot, int ch) {
    const long long at = page * t.sb + h * t.sh + slot * t.st + ch;
    if (DT == OBC_E4M3) {
        const uint2 codes = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.ptr) + at);
        return e4m3_values(codes, scale[page * c.ss_p + h * c.ss_h + slot]);
    }
    if (DT == OBC_BF16) return load8(static_cast<const __nv_bfloat16*>(t.ptr) + at);
    return load8(static_cast<const float*>(t.ptr) + at);
}
template <int DT>
__device__ __forceinline__ void put_page_row(const PagesView& c, const TensorView& t, uint8_t* scale, int page, int h, int slot, int lane, const Row8& r, float amax) {
    const long long at = page * t.sb + h * t.sh + slot * t.st + lane * 8;
    if (DT == OBC_E4M3) {
        const int s = scale_exponent(amax);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(const_cast<void*>(t.ptr)) + at) = e4m3_codes(r, s);
        if (lane == 0) scale[page * c.ss_p + h * c.ss_h + slot] = (uint8_t)s;
    } else if (DT == OBC_BF16) {
        store8(static_cast<__nv_bfloat16*>(const_cast<void*>(t.ptr)) + at, r);
    } else {
        store8(static_cast<float*>(const_cast<void*>(t.ptr)) + at, r);
    }
}

template <typename S, int DT>
__global__ void __launch_bounds__(kBlock)
paged_write_kernel(PagesView c, PagedWrite w, TensorView k, TensorView v, long long total) {
    pdl_wait();
    const int lane = threadIdx.x % kLanes;
    const long long f0 = (long long)blockIdx.x * kRowsPerBlock + threadIdx.x / kLanes;
    Row8 rk[kRows], rv[kRows];
    int page[kRows], slot[kRows], head[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const long long f = f0 + i * (kBlock / kLanes);
        page[i] = -1; slot[i] = 0; head[i] = 0;
        rk[i] = Row8{}; rv[i] = Row8{};
        if (f >= total) continue;
        const int unit = (int)(f / w.rows), j = (int)(f % w.rows);
        const int b = c.by_H.div(unit), h = unit - b * c.Hkv;
        const int n = w.new_lens ? min(max(w.new_lens[b * w.nb + h * w.nh], 0), w.rows) : w.rows;
        const int pos = c.len(b, h) - n + j;
        const int src = w.idx ? w.idx[f] : j;
        if (j >= n || pos < 0 || (unsigned)src >= (unsigned)w.src_tokens) continue;
        page[i] = c.page_of(b, h, pos);
        slot[i] = c.by_P.mod(pos); head[i] = h;
        rk[i] = load8(static_cast<const S*>(k.ptr) + b * k.sb + h * k.sh + src * k.st + lane * 8);
        rv[i] = load8(static_cast<const S*>(v.ptr) + b * v.sb + h * v.sh + src * v.st + lane * 8);
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        float mk = 0.f, mv = 0.f;
        if (DT == OBC_E4M3) { mk = row_amax(rk[i]); mv = row_amax(rv[i]); }       // (every lane of the warp takes part)
        if (page[i] < 0) continue;
        put_page_row<DT>(c, c.k, c.ks, page[i], head[i], slot[i], lane, rk[i], mk);
        put_page_row<DT>(c, c.v, c.vs, page[i], head[i], slot[i], lane, rv[i], mv);
    }
}

template <typename D, int DT>
__global__ void __launch_bounds__(kBlock)
paged_read_kernel(PagesView c, int n_tokens, TensorView k, TensorView v, int zero_rows, long long total) {
    pdl_wait();
    const int lane = threadIdx.x % kLanes;
    const long long f0 = (long long)blockIdx.x * kRowsPerBlock + threadIdx.x / kLanes;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const long long f = f0 + i * (kBlock / kLanes);
        if (f >= total) continue;
        const int unit = (int)(f / n_tokens), t = (int)(f % n_tokens);
        const int b = c.by_H.div(unit), h = unit - b * c.Hkv;
        Row8 rk{}, rv{};
        if (t < c.len(b, h)) {
            const int page = c.page_of(b, h, t);
            if (page >= 0) {
                rk = page_row<DT>(c, c.k, c.ks, page, h, c.by_P.mod(t), lane * 8);
                rv = page_row<DT>(c, c.v, c.vs, page, h, c.by_P.mod(t), lane * 8);
            }
        } else if (!zero_rows) {
            continue;
        }
        store8(static_cast<D*>(const_cast<void*>(k.ptr)) + b * k.sb + h * k.sh + t * k.st + lane * 8, rk);
        store8(static_cast<D*>(const_cast<void*>(v.ptr)) + b * v.sb + h * v.sh + t * v.st + lane * 8, rv);
    }
}

}  // namespace

obc_status launch_paged_write(const PagesView& c, const PagedWrite& w, TensorView k, TensorView v, cudaStream_t stream) {
    const long long total = (long long)c.B * c.Hkv * w.rows, blocks = (total + kRowsPerBlock - 1) / kRowsPerBlock;
    if (blocks > 0x7fffffffLL) return OBC_ERR_SHAPE;
    auto go = [&](auto kernel) {
        ProfScope prof("paged_write", stream);
        return launch_pdl(kernel, dim3((unsigned)blocks), dim3(kBlock), 0, stream, 1, c, w, k, v, total);
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
    const long long total = (long long)c.B * c.Hkv * n_tokens, blocks = (total + kRowsPerBlock - 1) / kRowsPerBlock;
    if (blocks > 0x7fffffffLL) return OBC_ERR_SHAPE;
    auto go = [&](auto kernel) {
        ProfScope prof("paged_read", stream);
        return launch_pdl(kernel, dim3((unsigned)blocks), dim3(kBlock), 0, stream, 1, c, n_tokens, k, v, (int)zero_rows, total);
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
