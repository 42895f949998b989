// Tiled tensor maps (TMA descriptors) for bf16 arrays whose innermost dimension is head_dim, with a
// small per-thread cache: a map depends only on the base pointer, the extents, the strides and the box,
// and a caller that scores the same cache layer after layer, or decodes step after step, asks for the
// same few maps every call.
#include "obc_common.cuh"
#include <cudaTypedefs.h>
#include <string.h>

namespace obc {
namespace {

PFN_cuTensorMapEncodeTiled get_encode() {
    static PFN_cuTensorMapEncodeTiled fn = nullptr;
    if (!fn) {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) == cudaSuccess &&
            qres == cudaDriverEntryPointSuccess)
            fn = (PFN_cuTensorMapEncodeTiled)ptr;
    }
    return fn;
}

struct MapKey {
    const void* base;
    int rank;
    uint32_t box_rows;
    uint64_t dims[4];
    uint64_t strides[3];
};
struct MapEntry { MapKey key; CUtensorMap map; bool used; };
constexpr int kCacheSlots = 16;

}  // namespace

bool make_map(CUtensorMap* map, const void* base, int rank, const uint64_t* dims, const uint64_t* strides_bytes,
              uint32_t box_rows) {
    thread_local MapEntry cache[kCacheSlots] = {};
    thread_local int next_slot = 0;
    MapKey key;
    memset(&key, 0, sizeof(key));
    key.base = base; key.rank = rank; key.box_rows = box_rows;
    for (int i = 0; i < rank; ++i) key.dims[i] = dims[i];
    for (int i = 0; i < rank - 1; ++i) key.strides[i] = strides_bytes[i];
    for (int i = 0; i < kCacheSlots; ++i)
        if (cache[i].used && memcmp(&cache[i].key, &key, sizeof(key)) == 0) { *map = cache[i].map; return true; }

    PFN_cuTensorMapEncodeTiled enc = get_encode();
    if (!enc) return false;
    cuuint64_t gdim[4]; cuuint64_t gstr[3]; cuuint32_t box[4] = {64, box_rows, 1, 1}; cuuint32_t estr[4] = {1, 1, 1, 1};
    for (int i = 0; i < rank; ++i) gdim[i] = dims[i];
    for (int i = 0; i < rank - 1; ++i) gstr[i] = strides_bytes[i];
    if (enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(base), gdim, gstr, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return false;
    MapEntry& e = cache[next_slot];
    next_slot = (next_slot + 1) % kCacheSlots;
    e.key = key; e.map = *map; e.used = true;
    return true;
}

// (made anew for every call: a pool's map is not worth a slot of the cache above)
bool make_page_map(CUtensorMap* map, const PagesView& c, const TensorView& t, int box, bool whole_rows) {
    PFN_cuTensorMapEncodeTiled enc = get_encode();
    if (!enc) return false;
    const bool e4m3 = c.dtype == OBC_E4M3;
    const cuuint64_t es = e4m3 ? 1 : 2, row = (cuuint64_t)t.st * es;
    // (a stride of 0, which the encoding refuses, belongs to a dimension of extent 1)
    cuuint64_t dims[5] = {e4m3 ? 128u : 64u, (cuuint64_t)c.P}, strides[4] = {row};
    cuuint32_t boxes[5] = {e4m3 ? 128u : 64u, (cuuint32_t)box, 1, 1, 1};
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    int n = 2;
    if (whole_rows && !e4m3) { dims[n] = 2; strides[n - 1] = 128; boxes[n++] = 2; }
    else dims[0] = kD;
    dims[n] = (cuuint64_t)(t.sh ? c.Hkv : 1); strides[n - 1] = t.sh ? (cuuint64_t)t.sh * es : row; ++n;
    dims[n] = (cuuint64_t)(t.sb ? c.n_pages : 1); strides[n - 1] = t.sb ? (cuuint64_t)t.sb * es : row; ++n;
    return enc(map, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)n, const_cast<void*>(t.ptr), dims, strides, boxes, ones,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace obc
