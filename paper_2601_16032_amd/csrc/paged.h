// What the operators over a paged key-value cache share: sums over lanes, and checks on the host.
#pragma once

namespace sawattn {

// Sum over the lanes up to and including this one.
template <int CONTROL, int ROWS>
__device__ __forceinline__ int from_lane(int x) { return __builtin_amdgcn_update_dpp(0, x, CONTROL, ROWS, 0xf, false); }
template <int CONTROL, int ROWS>
__device__ __forceinline__ long long from_lane(long long x) {
    const unsigned low = from_lane<CONTROL, ROWS>((int)x), high = from_lane<CONTROL, ROWS>((int)(x >> 32));
    return (long long)((unsigned long long)high << 32 | low);
}
template <typename T>
__device__ __forceinline__ T lanes_upto(T x) {
    x += from_lane<0x111, 0xf>(x);      // row_shr 1, 2, 4, 8: within rows of 16 lanes
    x += from_lane<0x112, 0xf>(x);
    x += from_lane<0x114, 0xf>(x);
    x += from_lane<0x118, 0xf>(x);
    x += from_lane<0x142, 0xa>(x);      // the last lane of rows 0 and 2 into rows 1 and 3
    x += from_lane<0x143, 0xc>(x);      // lane 31 into rows 2 and 3
    return x;
}

// log2 of a page size, or -1 where it is none: a power of two from 16 (the attention reads sixteen rows of a page at a time) to 2^20.
inline int page_shift(int page_size) {
    if (page_size < 16 || page_size > (1 << 20) || (page_size & (page_size - 1))) return -1;
    return __builtin_ctz((unsigned)page_size);
}

struct Range {      // of memory
    uintptr_t begin, end;
    Range(const void* p, unsigned long long bytes) : begin((uintptr_t)p), end((uintptr_t)p + bytes) {}
    bool meets(const Range& o) const { return begin < o.end && o.begin < end; }
};

// Whether n places `stride` elements apart are in order: no step backwards, whole 16-byte pieces, far from overflowing.  (A single one has no stride.)
inline bool good_stride(int64_t stride, long long n) {
    return n <= 1 || (stride >= 0 && stride % 8 == 0 && (double)stride * (double)n < 1e17);
}

inline int check_cache(const sawattn_kv_cache* c, bool pointers) {
    if (!c) return fail(SAWATTN_ERR_INVALID_ARG, "cache must be non-null");
    if (c->pages <= 0 || c->heads <= 0) return fail(SAWATTN_ERR_INVALID_ARG, "cache: pages and heads must be positive");
    if (c->d != 64 && c->d != 128) return fail(SAWATTN_ERR_UNSUPPORTED, "head dimension must be 64 or 128");
    if (page_shift(c->page_size) < 0) return fail(SAWATTN_ERR_UNSUPPORTED, "page size must be a power of two from 16 to 2^20");
    if (c->dtype != SAWATTN_F16 && c->dtype != SAWATTN_BF16)
        return fail(SAWATTN_ERR_INVALID_ARG, "cache: dtype must be SAWATTN_F16 or SAWATTN_BF16");
    if (!pointers) return SAWATTN_OK;
    if (!c->k || !c->v) return fail(SAWATTN_ERR_INVALID_ARG, "cache: k and v must be non-null");
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15u) return fail(SAWATTN_ERR_INVALID_ARG, "cache: k and v must be 16-byte aligned");
    for (int64_t s : {c->k_page, c->v_page})
        if (!good_stride(s, c->pages)) return fail(SAWATTN_ERR_INVALID_ARG, "cache: page strides must be multiples of 8, not negative");
    for (int64_t s : {c->k_head, c->v_head})
        if (!good_stride(s, c->heads)) return fail(SAWATTN_ERR_INVALID_ARG, "cache: head strides must be multiples of 8, not negative");
    for (int64_t s : {c->k_row, c->v_row})
        if (!good_stride(s, c->page_size)) return fail(SAWATTN_ERR_INVALID_ARG, "cache: row strides must be multiples of 8, not negative");
    return SAWATTN_OK;
}

inline int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return SAWATTN_OK;
    char msg[200];
    std::snprintf(msg, sizeof msg, "%s: kernel launch failed: %s", what, hipGetErrorString(e));
    return fail(SAWATTN_ERR_RUNTIME, msg);
}

}  // namespace sawattn
